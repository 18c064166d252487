"""The example of beam search under a grammar: what it writes fits the grammar, and each beam's cache holds what its own history put there."""
import os
import re
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WANTS = [r"\d{4}-\d\d-\d\d", r'"[a-z ]{3,12}"', r"(yes|no)", r"\d+(\.\d+)*", r"[abc]{2,40}!"]


def _decoder(beams, steps, page_tokens):
    import torch
    import paper_2507_16768_amd as wg
    import wg_synth as ws
    assert torch.cuda.is_available(), "this test needs the GPU"
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import beam_decode
    v = ws.make_vocab(3000, ("geometric", 4, 16), seed=1)
    vocab = wg.Vocab(v.bytes, v.offsets, v.eos_id)
    h = wg.Handle([wg.regex_to_template(w) for w in WANTS], None, vocab, flags=wg.EOS_STOP)
    prompts = [[(7 * i + 13 * g) % vocab.V for i in range(1 + 17 * g)] for g in range(len(WANTS))]
    return torch, v, beam_decode.BeamDecoder(h, beam_decode.Model(vocab.V), prompts, beams, steps, page_tokens), prompts


@pytest.mark.parametrize("beams,steps,page_tokens", [(1, 20, 16), (4, 40, 16), (5, 33, 32), (8, 50, 16)])
def test_beams_write_what_the_grammar_allows_and_keep_their_caches(beams, steps, page_tokens):
    torch, v, d, prompts = _decoder(beams, steps, page_tokens)
    history, scores = d.run()
    history, scores = history.cpu().numpy(), scores.cpu().numpy()
    table, lens = d.now["table"].cpu().numpy(), d.now["lens"].cpu().numpy()
    parents = d.parents.cpu().numpy()
    finished = 0
    for g, want in enumerate(WANTS):
        s = scores[g * beams:(g + 1) * beams]
        assert s[0] > -np.inf and (np.diff(s[np.isfinite(s)]) <= 0).all()
        seen = set()
        for r in range(g * beams, (g + 1) * beams):
            if scores[r] == -np.inf:
                continue
            row = history[r].tolist()
            assert min(row) >= 0 and tuple(row) not in seen
            seen.add(tuple(row))
            end = row.index(v.eos_id) if v.eos_id in row else None
            assert end is None or row[end:] == [v.eos_id] * (steps - end)
            text = b"".join(bytes(v.bytes[v.offsets[t]:v.offsets[t + 1]]) for t in row[:end]).decode("latin-1")
            if end is not None:
                finished += 1
                assert re.fullmatch(want, text), (want, text)
    assert finished > 0
    # What each row's pages hold after the last step but one: the keys and values of its prompt and of the tokens on the way to it.  (The last
    # selection came after the last append: rows have its parents' histories then.)
    model = d.model
    held = {}
    for r in range(d.R):
        if scores[r] > -np.inf:
            held.setdefault(int(parents[r]), history[r][:steps - 1].tolist())
    assert held
    for r, row in held.items():
        tokens = prompts[r // beams] + row
        assert lens[r] == len(tokens)
        t = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        _, _, k, val = model.project(t, torch.arange(len(tokens), dtype=torch.int32, device="cuda"))
        at = torch.arange(len(tokens), device="cuda")
        page = torch.from_numpy(table[r]).cuda().long()[at // page_tokens]
        off = at % page_tokens
        k8 = d.k_cache.float()[page, :, off] * d.k_scale[page][:, :, None]
        v8 = d.v_cache.float()[page, :, :, off] * d.v_scale[page][:, :, None]
        # a number is rounded to 4 bits of mantissa (2^-4 of itself) or, at the low end, to 2^-10 of 448 / 448 times the scale; where the scale grew, once more
        # at the low end for each time.  (The projection's own product may differ in its last bit with the number of its rows: 2^-8.)
        for x, y, scale in ((k, k8, d.k_scale[page]), (val, v8, d.v_scale[page])):
            x = x.float()
            assert ((x - y).abs() <= (2.0 ** -4 + 2.0 ** -7) * x.abs() + scale[:, :, None] * 2.0 ** -9).all(), r


def test_one_beam_is_the_greedy_choice():
    """With one beam the tokens are those that masked_argmax takes from the same logits."""
    torch, v, d, prompts = _decoder(1, 15, 16)
    import paper_2507_16768_amd as wg
    picked = []
    select = wg.beam_select

    def both(logits, mask, *rest):
        t = torch.empty(logits.shape[0], dtype=torch.int32, device="cuda")
        wg.masked_argmax(logits, mask, t)
        picked.append(t)
        select(logits, mask, *rest)

    wg.beam_select = both
    try:
        history, _ = d.run()
    finally:
        wg.beam_select = select
    assert torch.equal(torch.stack(picked, 1), history)
