"""Beam search under a grammar, with the model's cache in 8-bit pages that follow the beams.

Every request decodes with `K` beams.  A step is: the beams' masks (Handle.fill_masks), their best continuations with the
grammar states that go with them (beam_select, Handle.advance), the token histories after their parents (reorder_rows), the pages of
the cache after them too, with a place for each new token (page_step), the tokens' keys and values into them (cache_append) and
attention over them (cache_attend).  Nothing in a step waits for the GPU.  The model is one layer of random weights: what matters
here is what is called, on what, and in which order.

    python examples/beam_decode.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_16768_amd as wg  # noqa: E402


class Model:
    """One layer of attention: 4 query heads over 2 cached ones of 64 values."""

    Q, H, D = 4, 2, 64

    def __init__(self, V, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *shape: (torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5).to(torch.bfloat16)
        E = 256
        self.embedding = (torch.randn((V, E), generator=g, device="cuda")).to(torch.bfloat16)
        self.frequency = torch.exp(-torch.arange(E, device="cuda") / 20.0)
        self.qkv, self.out, self.head = w(E, (self.Q + 2 * self.H) * self.D), w(self.Q * self.D, E), w(E, V)

    def project(self, tokens, positions):
        x = self.embedding[tokens.clamp(min=0).long()] + torch.sin(positions[:, None] * self.frequency).to(torch.bfloat16)
        heads = (x @ self.qkv).view(-1, self.Q + 2 * self.H, self.D)
        return x, heads[:, :self.Q], heads[:, self.Q:self.Q + self.H], heads[:, self.Q + self.H:]

    def logits(self, x, attended):
        return (x + attended.flatten(1) @ self.out) @ self.head * 3.0


class BeamDecoder:
    """`prompts`: a list of token lists, one for each of the handle's instances; `steps` tokens are decoded with `beams` beams."""

    def __init__(self, handle, model, prompts, beams, steps, page_tokens=16):
        G, K = len(prompts), beams
        self.h, self.model, self.prompts, self.G, self.K, self.R, self.P, self.steps = handle, model, prompts, G, K, G * K, page_tokens, steps
        R, i32 = self.R, dict(dtype=torch.int32, device="cuda")
        columns = -(-(max(map(len, prompts)) + steps) // page_tokens)
        pages = R * columns + R
        # what a step reads and what it writes, in turn
        state = lambda: dict(table=torch.zeros((R, columns), **i32), lens=torch.zeros(R, **i32), counters=torch.zeros(2, dtype=torch.int64, device="cuda"),
                             scores=torch.zeros(R, device="cuda"), states=torch.zeros((R, 2), **i32), history=torch.full((R, steps), -1, **i32))
        self.now, self.next = state(), state()
        self.now["counters"][1] = pages
        self.ring = torch.arange(pages, **i32)
        self.k_cache = torch.zeros((pages, model.H, page_tokens, model.D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        self.v_cache = torch.zeros((pages, model.H, model.D, page_tokens), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        self.k_scale, self.v_scale = (torch.ones((pages, model.H), device="cuda") for _ in range(2))
        self.mask = torch.empty((R, handle.W), **i32)
        self.parents, self.tokens = torch.arange(R, **i32), torch.empty(R, **i32)
        self.starts = torch.empty(R + 1, **i32)
        tokens = max(R, sum(map(len, prompts)))
        self.work = torch.empty(max(wg.beam_select_workspace(R, handle.V, K), wg.page_step_workspace(R, K, columns),
                                    *(wg.cache_attend_workspace(t, R, model.Q, model.H, model.D, columns, page_tokens) for t in (R, tokens))),
                                dtype=torch.uint8, device="cuda")

    def forward(self, tokens, counts):
        """The tokens' attention behind what the rows' caches hold: logits of all of them.  Rows follow self.parents first."""
        T, i32, a, b = tokens.numel(), dict(dtype=torch.int32, device="cuda"), self.now, self.next
        slots, positions, origins = (torch.empty(T, **i32) for _ in range(3))
        wg.page_step(a["table"], a["lens"], counts, self.parents, self.K, self.P, self.ring, a["counters"], b["table"], b["lens"], self.starts, slots, positions,
                     origins, b["counters"], self.work)
        x, q, k, v = self.model.project(tokens, positions)
        wg.cache_append(k, v, slots, origins, self.k_cache, self.v_cache, self.k_scale, self.v_scale)
        attended = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        wg.cache_attend(q, self.k_cache, self.v_cache, self.k_scale, self.v_scale, b["table"], b["lens"], self.starts, self.model.D ** -0.5, attended, self.work)
        for name in ("table", "lens", "counters"):
            a[name], b[name] = b[name], a[name]
        return self.model.logits(x, attended)

    def run(self):
        """Histories [R, steps] and scores [R], a request's best beam first."""
        R, K, a, b = self.R, self.K, self.now, self.next
        # the prompts, once for each request: in the row of its first beam, which alone lives before the first step
        counts = torch.zeros(R, dtype=torch.int32, device="cuda")
        counts[::K] = torch.tensor([len(p) for p in self.prompts], dtype=torch.int32, device="cuda")
        prompt = torch.tensor([t for p in self.prompts for t in p], dtype=torch.int32, device="cuda")
        last = self.forward(prompt, counts)[counts[::K].cumsum(0) - 1]
        logits = last.repeat_interleave(K, 0)
        a["scores"].view(-1, K)[:, 1:] = -torch.inf
        a["states"].copy_(torch.from_numpy(self.h.start_states.view("int32")).cuda().repeat_interleave(K, 0))
        one = torch.ones(R, dtype=torch.int32, device="cuda")
        for step in range(self.steps):
            if step:
                logits = self.forward(self.tokens, one)
            self.h.fill_masks(a["states"], self.mask)
            wg.beam_select(logits, self.mask, a["scores"], a["states"], K, b["scores"], self.parents, self.tokens, b["states"], self.work)
            self.h.advance(b["states"], self.tokens)
            wg.reorder_rows(a["history"], self.parents, b["history"])
            b["history"][:, step] = self.tokens
            for name in ("scores", "states", "history"):
                a[name], b[name] = b[name], a[name]
        return a["history"], a["scores"]


def main():
    import wg_synth as ws
    v = ws.make_vocab(4000, ("geometric", 4, 16), seed=1)
    vocab = wg.Vocab(v.bytes, v.offsets, v.eos_id)
    wants = [r"\d{4}-\d\d-\d\d", r'"[a-z ]{3,12}"', r"(yes|no)", r"\d+(\.\d+)*"]
    h = wg.Handle([wg.regex_to_template(w) for w in wants], None, vocab, flags=wg.EOS_STOP)
    model = Model(vocab.V)
    prompts = [[(7 * i + 13 * g) % vocab.V for i in range(5 + 17 * g)] for g in range(len(wants))]
    decoder = BeamDecoder(h, model, prompts, beams=4, steps=24)
    history, scores = decoder.run()
    for r, (row, score) in enumerate(zip(history.cpu().tolist(), scores.cpu().tolist())):
        text = b"".join(bytes(v.bytes[v.offsets[t]:v.offsets[t + 1]]) for t in row if t >= 0 and t != v.eos_id)
        print("%-24s beam %d  %8.3f  %s" % (wants[r // 4], r % 4, score, text.decode("latin-1") if score > float("-inf") else "-"))


if __name__ == "__main__":
    main()
