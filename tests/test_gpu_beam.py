"""Beam selection and the rows that follow the parents, against the definition in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# A score is score + ((x - m) - log Z) in fp32.  Z is a sum of up to 151,936 terms in threads, wavefronts and parts: at most some 200
# additions follow one another, each off by 2^-24, and exp by 2^-22 (its argument is below 40 where its term counts), so log Z is off by
# 200 * 2^-24 + 40 * 2^-24 + 2^-22 < 1.5e-5; the three roundings of the rest are below 3 * 2^-24 * |s| each.
def close(s):
    return 1.5e-5 + 2e-7 * np.abs(s)


def _wg():
    import torch
    import paper_2507_16768_amd as wg
    assert torch.cuda.is_available(), "this test needs the GPU"
    return torch, wg


def definition(x, allowed, scores, K):
    """x float64 [R, V], allowed bool, scores float64 [R]: per request the list of (score, row, token), best first, and all scores [R, V]."""
    R, V = x.shape
    ok = allowed & (x > -np.inf) & (scores > -np.inf)[:, None]          # (a NaN is not above -inf)
    tame = np.where(ok, np.minimum(x, np.finfo(np.float32).max), -np.inf)
    top = np.where(ok.any(1), tame.max(1), 0.0)[:, None]
    with np.errstate(all="ignore"):
        z = np.exp(tame - top).sum(1, keepdims=True)
        s = np.where(ok, scores[:, None] + (tame - top) - np.log(z), -np.inf)
    out = []
    for r0 in range(0, R, K):
        found = []
        for r in range(r0, r0 + K):
            ids = np.flatnonzero(ok[r])
            ids = ids[np.lexsort((ids, -x[r, ids]))][:K]
            found += [(-s[r, t], r, j, t) for j, t in enumerate(ids)]
        found.sort()
        out.append([(-a, r, t) for a, r, _, t in found[:K]])
    return out, s


def pack(torch, allowed):
    R, V = allowed.shape
    W = (V + 31) // 32
    bits = np.zeros((R, W * 32), dtype=np.uint8)
    bits[:, :V] = allowed
    words = np.packbits(bits, axis=1, bitorder="little").view(np.uint32)
    return torch.from_numpy(words.view(np.int32).copy()).cuda()


class Call:
    def __init__(self, torch, wg, R, V, K, states=True):
        self.torch, self.wg, self.K = torch, wg, K
        self.scores = torch.full((R,), 7.0, device="cuda")
        self.parents = torch.full((R,), -7, dtype=torch.int32, device="cuda")
        self.tokens = torch.full((R,), -7, dtype=torch.int32, device="cuda")
        self.states = torch.full((R, 2), -7, dtype=torch.int32, device="cuda") if states else None
        self.work = torch.empty(wg.beam_select_workspace(R, V, K), dtype=torch.uint8, device="cuda")

    def run(self, logits, mask, scores, states, stream=None):
        self.wg.beam_select(logits, mask, scores, states, self.K, self.scores, self.parents, self.tokens, self.states, self.work, stream)

    def host(self):
        return self.scores.cpu().numpy().astype(np.float64), self.parents.cpu().numpy(), self.tokens.cpu().numpy()


def check(got, states_in, states_out, want, s, K, exact_ids=True):
    scores, parents, tokens = got
    for g, best in enumerate(want):
        for j in range(K):
            r = g * K + j
            if j >= len(best):
                assert scores[r] == -np.inf and parents[r] == -1 and tokens[r] == -1, (g, j)
                if states_out is not None:
                    assert tuple(states_out[r]) == (-1, 0)
                continue
            v, row, token = best[j]
            assert abs(scores[r] - v) <= close(v), (g, j, scores[r], v)
            assert g * K <= parents[r] < g * K + K
            assert abs(s[parents[r], tokens[r]] - scores[r]) <= close(v), (g, j)
            if exact_ids:
                assert (parents[r], tokens[r]) == (row, token), (g, j)
            if states_out is not None:
                assert (states_out[r] == states_in[parents[r]]).all()
        pairs = [(parents[g * K + j], tokens[g * K + j]) for j in range(len(best))]
        assert len(set(pairs)) == len(pairs)


def apart(want, s, K):
    """Whether every neighbour among the best of each request, and the first left out, is further apart than two errors."""
    R = s.shape[0]
    for g, best in enumerate(want):
        v = np.sort(s[g * K:(g + 1) * K].reshape(-1))[::-1][:K + 1]
        v = v[v > -np.inf]
        if len(v) > 1 and (np.abs(np.diff(v)) <= 2 * close(v[:-1])).any():
            return False
    return True


def data(seed, G, K, V, dtype, density=None):
    rng = np.random.default_rng(seed)
    R = G * K
    x = (rng.standard_normal((R, V)) * 3).astype(np.float32)
    if dtype == "bf16":
        x = (x.view(np.uint32) & 0xFFFF0000).view(np.float32)
    allowed = np.ones((R, V), dtype=bool)
    if density is not None:
        share = np.array([0.97, 0.5, 0.02, 0.0, 2.0 / V])[np.arange(R) % 5][:, None]
        allowed = rng.random((R, V)) < share
    scores = (-20 * rng.random(R)).astype(np.float32)
    return x, allowed, scores, rng


def device_logits(torch, x, dtype):
    t = torch.from_numpy(x).cuda()
    return t if dtype == "f32" else t.to(torch.bfloat16)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("G,K,V", [(1, 1, 1), (1, 4, 33), (3, 2, 31), (2, 5, 1000), (1, 4, 32000), (5, 3, 8191), (7, 8, 20011), (2, 64, 5000),
                                   (1, 16, 151936), (40, 4, 16385), (1, 1, 300000), (300, 2, 700)])
def test_the_best_continuations(G, K, V, masked, dtype):
    torch, wg = _wg()
    x, allowed, scores, rng = data(G * 1000 + K, G, K, V, dtype, 1 if masked else None)
    R = G * K
    want, s = definition(x.astype(np.float64), allowed, scores.astype(np.float64), K)
    states = rng.integers(1, 1 << 30, (R, 2)).astype(np.int32)
    call = Call(torch, wg, R, V, K)
    call.run(device_logits(torch, x, dtype), pack(torch, allowed) if masked else None, torch.from_numpy(scores).cuda(), torch.from_numpy(states).cuda())
    check(call.host(), states, call.states.cpu().numpy(), want, s, K, exact_ids=dtype == "f32" and apart(want, s, K))


@pytest.mark.parametrize("K,V", [(64, 40000), (33, 16500), (20, 100003), (17, 20000)])
def test_many_beams_whose_best_come_from_one_place(K, V):
    """All of a request's continuations out of one beam's neighbouring tokens, out of one beam, and out of all alike."""
    torch, wg = _wg()
    x, allowed, scores, rng = data(K, 3, K, V, "f32")
    x[K // 2, 700:700 + 2 * K] += 30 + np.arange(2 * K, dtype=np.float32) / 8
    scores[K + 3] += 60
    scores[2 * K:] = -7.0
    want, s = definition(x.astype(np.float64), allowed, scores.astype(np.float64), K)
    states = rng.integers(1, 1 << 30, (3 * K, 2)).astype(np.int32)
    call = Call(torch, wg, 3 * K, V, K)
    call.run(device_logits(torch, x, "f32"), None, torch.from_numpy(scores).cuda(), torch.from_numpy(states).cuda())
    check(call.host(), states, call.states.cpu().numpy(), want, s, K, exact_ids=apart(want, s, K))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_anywhere_in_memory_and_on_another_stream(dtype):
    torch, wg = _wg()
    G, K, V = 4, 3, 4099
    x, allowed, scores, rng = data(5, G, K, V, dtype, 1)
    want, s = definition(x.astype(np.float64), allowed, scores.astype(np.float64), K)
    size = 4 if dtype == "f32" else 2
    for shift in (0, size, 3 * size, 1):                # bytes in front of the first row; an odd one too
        stride = V + 5
        raw = torch.zeros((G * K * stride + 16) * size, dtype=torch.uint8, device="cuda")
        host = device_logits(torch, x, dtype).contiguous().view(torch.uint8).view(G * K, V * size)
        rows = raw[shift:shift + G * K * stride * size].view(G * K, stride * size)
        rows[:, :V * size] = host
        rows[:, V * size:] = 0x7F                       # NaNs behind every row
        call = Call(torch, wg, G * K, V, K, states=False)
        mask, sc = pack(torch, allowed), torch.from_numpy(scores).cuda()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            if shift % size:
                L = wg.load_library()                   # (torch has no tensors at odd addresses)
                import ctypes as C
                p = lambda t: C.c_void_p(t.data_ptr())
                rc = L.wg_beam_select(C.c_void_p(raw.data_ptr() + shift), 0 if dtype == "f32" else 1, G * K, V, stride, p(mask), K, p(sc), None, p(call.scores),
                                      p(call.parents), p(call.tokens), None, p(call.work), call.work.numel(), C.c_void_p(side.cuda_stream))
                assert rc == 0
            else:
                at = raw[shift:].view(torch.float32 if dtype == "f32" else torch.bfloat16).as_strided((G * K, V), (stride, 1))
                call.run(at, mask, sc, None)
        side.synchronize()
        check(call.host(), None, None, want, s, K, exact_ids=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,V", [(4, 3000), (64, 40000), (1, 9000)])
def test_ties_go_to_the_lower_beam_and_token(K, V, dtype):
    """All logits are equal (more ties than any list holds), then all but some that stand out together."""
    torch, wg = _wg()
    x = np.full((2 * K, V), 1.5, dtype=np.float32)
    x[K:, V // 2:V // 2 + 2] = 9.0
    scores = np.full(2 * K, -1.0, dtype=np.float32)
    call = Call(torch, wg, 2 * K, V, K)
    states = torch.arange(4 * K, dtype=torch.int32, device="cuda").view(2 * K, 2)
    call.run(device_logits(torch, x, dtype), None, torch.from_numpy(scores).cuda(), states)
    got, parents, tokens = call.host()
    assert (parents[:K] == 0).all() and (tokens[:K] == np.arange(K)).all()
    top = [(K + i // 2, V // 2 + i % 2) for i in range(K)]
    assert [(parents[K + i], tokens[K + i]) for i in range(K)] == top
    assert (np.abs(got[:K] - (-1.0 - np.log(V))) <= close(20.0)).all()
    mask = np.zeros((2 * K, V), dtype=bool)
    mask[:, 7::3] = True                                 # the same under a mask
    call.run(device_logits(torch, x, dtype), pack(torch, mask), torch.from_numpy(scores).cuda(), states)
    _, parents, tokens = call.host()
    assert (parents[:K] == 0).all() and (tokens[:K] == 7 + 3 * np.arange(K)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_numbers_that_are_none(dtype):
    """NaN and -inf are no continuations and not in the sum, +inf is the largest number; dead beams have no continuations."""
    torch, wg = _wg()
    K, V, inf, nan = 4, 500, np.inf, np.nan
    x, allowed, scores, rng = data(9, 6, K, V, dtype)
    x[0, ::2] = nan
    x[1] = -inf
    x[2] = nan
    x[4, 17] = inf; x[4, 400] = inf
    x[5] = -inf; x[5, 3] = -3.0e38
    x = x.astype(np.float32)
    if dtype == "bf16":
        keep = np.isnan(x)
        x = (x.view(np.uint32) & 0xFFFF0000).view(np.float32)
        x[keep] = nan
    scores[6] = nan
    scores[7] = -inf
    scores[8:12] = -inf                                   # a request all of whose beams are gone
    scores[12:16] = [0.0, -inf, -inf, -inf]               # the first step
    allowed[16:20] = False
    allowed[16, 3] = True                                 # one continuation in all
    allowed[20:24] = False                                # none
    want, s = definition(x.astype(np.float64), allowed, scores.astype(np.float64), K)
    assert [len(b) for b in want] == [4, 4, 0, 4, 1, 0]
    states = rng.integers(1, 1 << 30, (24, 2)).astype(np.int32)
    call = Call(torch, wg, 24, V, K)
    call.run(device_logits(torch, x, dtype), pack(torch, allowed), torch.from_numpy(scores).cuda(), torch.from_numpy(states).cuda())
    check(call.host(), states, call.states.cpu().numpy(), want, s, K, exact_ids=False)
    got, parents, _ = call.host()
    assert got[16] == np.float32(scores[16]) and (parents[12:16] == 12).all()    # the only allowed token adds nothing


def test_a_finished_hypothesis_keeps_its_score():
    """A grammar's FINAL state allows the end of sequence alone, which has probability 1 there."""
    torch, wg = _wg()
    import wg_synth as ws
    from wg_synth.vocab import tiny_vocab
    v = tiny_vocab(b"ab", 2)
    vocab = wg.Vocab(v.bytes, v.offsets, v.eos_id)
    h = wg.Handle(['Sequence(Write("a"))'], None, vocab, flags=wg.EOS_STOP)
    states = torch.tensor([[wg.SID_FINAL, 0], [int(h.start_states[0][0]), 0]], dtype=torch.int32, device="cuda")
    mask = torch.empty((2, h.W), dtype=torch.int32, device="cuda")
    h.fill_masks(states, mask)
    x = torch.randn((2, vocab.V), device="cuda") * 10
    scores = torch.tensor([-3.25, -100.0], device="cuda")
    call = Call(torch, wg, 2, vocab.V, 2)
    call.run(x, mask, scores, states)
    got, parents, tokens = call.host()
    assert got[0] == -3.25 and parents[0] == 0 and tokens[0] == v.eos_id
    h.advance(call.states, call.tokens)
    assert tuple(call.states[0].tolist()) == (wg.SID_FINAL, 0)


def test_same_bits_every_time_and_in_a_graph():
    torch, wg = _wg()
    G, K, V = 8, 4, 50021
    x, allowed, scores, _ = data(3, G, K, V, "bf16", 1)
    lg, mask, sc = device_logits(torch, x, "bf16"), pack(torch, allowed), torch.from_numpy(scores).cuda()
    call = Call(torch, wg, G * K, V, K, states=False)
    call.run(lg, mask, sc, None)
    first = [t.clone() for t in (call.scores, call.parents, call.tokens)]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call.run(lg, mask, sc, None)
        with torch.cuda.graph(graph, stream=side):
            call.run(lg, mask, sc, None)
    torch.cuda.synchronize()
    for i in range(4):
        lg.copy_(device_logits(torch, x * (1 + i), "bf16"))
        call.run(lg, mask, sc, None)
        want = [t.clone() for t in (call.scores, call.parents, call.tokens)]
        for t in (call.scores, call.parents, call.tokens):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (call.scores, call.parents, call.tokens)):
            assert torch.equal(a, b)
        if i == 0:
            for a, b in zip(first, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("shape,axis,dtype", [((7, 64), 0, "float32"), ((8, 1000), 0, "bfloat16"), ((3, 8, 4099), 1, "float32"), ((2, 5, 3, 33), 1, "bfloat16"),
                                              ((6, 1), 0, "uint8"), ((4, 9, 7), 1, "uint8"), ((1, 3), 0, "int32"), ((16,), 0, "int64"), ((2, 16), 1, "int16"),
                                              ((5, 300000), 0, "uint8")])
def test_rows_follow_their_parents(shape, axis, dtype):
    torch, wg = _wg()
    dt = getattr(torch, dtype)
    g = torch.Generator().manual_seed(1)
    src = torch.randint(-100, 100, shape, generator=g).to(dt).cuda()
    R = shape[axis]
    parents = torch.randint(-1, R, (R,), generator=g, dtype=torch.int32)
    parents[R // 2] = R + 5                              # not a row either
    dst = torch.full(shape, 77, dtype=dt, device="cuda")
    wg.reorder_rows(src, parents.cuda(), dst, axis=axis)
    there = (parents >= 0) & (parents < R)
    want = src.cpu().index_select(axis, torch.where(there, parents, 0).long())
    view = [1] * len(shape)
    view[axis] = R
    want = torch.where(there.view(view), want, torch.zeros_like(want))
    assert torch.equal(dst.cpu(), want)


def test_rows_of_a_larger_array_follow_too():
    torch, wg = _wg()
    big = torch.arange(3 * 10 * 50, dtype=torch.int32, device="cuda").view(3, 10, 50)
    src, out = big[:, 2:8, 5:30], torch.zeros((3, 6, 41), dtype=torch.int32, device="cuda")
    dst = out[:, :, 7:32]
    parents = torch.tensor([5, 0, -1, 3, 3, 1], dtype=torch.int32, device="cuda")
    wg.reorder_rows(src, parents, dst, axis=1)
    want = src[:, parents.clamp(min=0).long()] * (parents >= 0).int()[None, :, None]
    assert torch.equal(dst, want) and int(out[:, :, :7].abs().sum()) == 0 and int(out[:, :, 32:].abs().sum()) == 0


@pytest.mark.parametrize("R,V,dtype", [(1, 40_000_003, "f32"), (256, 200_003, "bf16"), (64, 700_001, "bf16"), (1, 60_000_000, "bf16")])
def test_the_sum_over_a_large_vocabulary(R, V, dtype):
    """One beam a request: the score is its row's largest logit less the log of the sum, which is off by what the header says; the score's three roundings on top."""
    torch, wg = _wg()
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn((R, V), generator=g, device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    call = Call(torch, wg, R, V, 1, states=False)
    call.run(x, None, torch.zeros(R, device="cuda"), None)
    for r in range(0, R, 37):
        y = x[r].double()
        want = float(y.max() - torch.logsumexp(y, 0))
        assert abs(float(call.scores[r]) - want) <= (V / 1600 + 80) * 2.0 ** -24 + 2e-7 * abs(want)
        assert int(call.tokens[r]) == int((y == y.max()).nonzero()[0])
