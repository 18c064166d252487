"""What the operators of rotary positions and of attention over a cache of latent vectors are timed on.

A token's keys and values come from one latent vector of `C` numbers that all heads share, and a key of 64 numbers that
carries the position and is shared too.  A case names the operator (`op`) and its sizes:

  rotate  rotate: `T` tokens of `Q` query heads and `K` key heads of `D` numbers, the first `turned` of which are rotated by
          the token's position (up to `reach`), in pairs that lie side by side (`pairs`) or half of them apart
  append  latent_append: the latent vectors and shared keys of up to `new` tokens of each of `R` rows (requests of `K` beams)
          behind up to `len` cached ones, into pages of `P` tokens, in 8 bits with a scale for each token, or in 16
  read    latent_read: the cached tokens of `R` rows of up to `len`, out of their pages into one piece, in 16 bits
  attend  latent_attend: up to `new` tokens of each row, `H` heads, over the cached latent vectors themselves: what a head makes
          of a latent vector is in its query already, and is applied to its output later
  prompt  latent_prompt: the same attention with the keys and values of every head made beforehand (`D` numbers each, and the
          shared key): up to `new` tokens a row behind up to `len` earlier ones

Rows have lengths of their own, spread over the range up to `len` (and `new`).  Where `own` is false the operators are
computed in elementary operations in 32 bits; where it is true by this library's kernels.
"""
import math

import torch

own = False

BLOCK_MAX = 448.0                     # the largest value of the 8-bit format (e4m3)
LEAST, MOST = -64, 120                # exponents that a scale may have
E = 64                                # numbers of a shared key


def listed():
    return [
        # a token of one request: latency of a launch
        {"name": "rotate one token", "op": "rotate", "T": 1, "Q": 32, "K": 8, "D": 128, "turned": 128, "pairs": False, "type": "bf16", "reach": 8000},
        # prompts whose heads are rotated in part, far into a long context
        {"name": "rotate prompts", "op": "rotate", "T": 7001, "Q": 40, "K": 8, "D": 128, "turned": 64, "pairs": True, "type": "bf16", "reach": 1000000},
        # a token for each of 256 rows, beams that fork among them
        {"name": "append latent decode", "op": "append", "R": 256, "K": 4, "len": 1024, "new": 1, "P": 64, "C": 512, "bits": 8},
        # sixteen prompts
        {"name": "append latent prompts", "op": "append", "R": 16, "K": 1, "len": 500, "new": 2048, "P": 32, "C": 512, "bits": 8},
        # one short row
        {"name": "read one", "op": "read", "R": 1, "len": 500, "P": 16, "C": 512, "bits": 16},
        # the cached prefixes of a batch, before they are expanded
        {"name": "read batch", "op": "read", "R": 32, "len": 8000, "P": 64, "C": 512, "bits": 8},
        # one request with a long context, a token at a time, few heads
        {"name": "attend latent one", "op": "attend", "R": 1, "len": 30000, "new": 1, "P": 16, "H": 16, "C": 512, "bits": 8},
        # a batch that decodes with all heads of a large model
        {"name": "attend latent batch", "op": "attend", "R": 100, "len": 4096, "new": 1, "P": 64, "H": 128, "C": 512, "bits": 16},
        # a few drafted tokens a row to be verified
        {"name": "attend latent drafts", "op": "attend", "R": 64, "len": 8192, "new": 4, "P": 32, "H": 16, "C": 512, "bits": 8},
        # parts of prompts behind a cached prefix, a narrow latent vector
        {"name": "attend latent chunks", "op": "attend", "R": 3, "len": 1500, "new": 203, "P": 64, "H": 24, "C": 256, "bits": 16},
        # whole prompts
        {"name": "prompt batch", "op": "prompt", "R": 4, "len": 0, "new": 2001, "H": 32, "D": 128},
        # the last part of one long prompt
        {"name": "prompt tail", "op": "prompt", "R": 1, "len": 9000, "new": 131, "H": 16, "D": 128},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    lo, hi = min(lo, hi), max(lo, hi)
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("rotate", "append", "read", "attend", "attend", "prompt"))
    if op == "rotate":
        D = rng.choice((64, 64, 80, 128, 128, 192, 256))
        Q, K = rng.choice(((1, 0), (8, 1), (12, 4), (16, 1), (32, 8), (40, 8)))
        return {"op": op, "T": _spread(rng, 1, 7001 * 48 * 128 // ((Q + K) * D * 2)), "Q": Q, "K": K, "D": D, "turned": rng.choice((D, D, D // 2, D // 4)),
                "pairs": rng.random() < 0.5, "type": rng.choice(("bf16", "bf16", "f32")), "reach": _spread(rng, 100, 1000000)}
    P, C, bits = rng.choice((16, 32, 64)), rng.choice((256, 512, 512)), rng.choice((8, 16))
    if op == "append":
        if rng.random() < 0.5:
            K = rng.choice((1, 2, 4))
            return {"op": op, "R": K * _spread(rng, 1, 256 // K), "K": K, "len": _spread(rng, 20, 2048), "new": 1, "P": P, "C": C, "bits": bits}
        return {"op": op, "R": _spread(rng, 1, 16), "K": 1, "len": _spread(rng, 16, 1024), "new": _spread(rng, 2, 2048 if bits == 8 else 1500), "P": P, "C": C, "bits": bits}
    if op == "read":
        R = _spread(rng, 1, 32)
        return {"op": op, "R": R, "len": _spread(rng, 20, 8000 if bits == 8 else 6000), "P": P, "C": C, "bits": bits}
    if op == "attend":
        H = rng.choice((4, 8, 16, 24, 32, 64, 128))
        if rng.random() < 0.7:
            new = rng.choice((1, 1, 1, 1, 2, 5))
            R = _spread(rng, 1, 100)
            return {"op": op, "R": R, "len": _spread(rng, 20, min(32768, 400_000 // R, 52_000_000 // (R * H * new))), "new": new, "P": P, "H": H, "C": C, "bits": bits}
        R, new = _spread(rng, 1, 4), _spread(rng, 6, 300)
        return {"op": op, "R": R, "len": _spread(rng, 16, max(20, min(4096, 36_000_000 // (R * H * new) - new))), "new": new, "P": P, "H": H, "C": C, "bits": bits}
    R, H, D = _spread(rng, 1, 4), rng.choice((2, 8, 16, 32)), rng.choice((64, 128))
    new = _spread(rng, 2, 2000)
    most = min(9000, 220_000_000 // (R * new * H) - new, 32_000_000 // (R * H * D) - new)
    return {"op": op, "R": R, "len": rng.choice((0, _spread(rng, 10, most))) if most > 10 else 0, "new": new, "H": H, "D": D}


# ---- the rows of a case -----------------------------------------------------------------------

def _shares(R):
    """A share of the range for each row, spread evenly: the first row has all of it."""
    return [((r * 0.6180339887498949) % 1.0) for r in range(R)]


def _lens(c):
    """Cached tokens of each row before the step: beams of a request agree."""
    K = c.get("K", 1)
    n = c["R"] // K
    return [int(c["len"] * (1.0 - 0.75 * f)) for f in _shares(n) for _ in range(K)]


def _news(c):
    """Tokens that each row takes in the step."""
    if c["new"] == 1:
        return [1] * c["R"]
    return [max(1, int(c["new"] * (1.0 - 0.6 * f))) for f in reversed(_shares(c["R"]))]


def _pages(tokens, P):
    return (tokens + P - 1) // P


def _token_bytes(c):
    return c["C"] + 4 + 2 * E if c["bits"] == 8 else 2 * (c["C"] + E)


def work(case):
    c = case
    if c["op"] == "rotate":
        e = 4 if c["type"] == "f32" else 2
        numbers = c["T"] * (c["Q"] + c["K"]) * c["D"]
        turned = c["T"] * (c["Q"] + c["K"]) * c["turned"]
        return {"bytes": 2.0 * numbers * e + 4.0 * c["T"] + 4.0 * c["turned"], "flops": 3.0 * turned}
    lens = _lens(c)
    if c["op"] == "read":
        return {"bytes": float(sum(lens) * (_token_bytes(c) + 2 * (c["C"] + E))), "flops": 0.0}
    news = _news(c)
    T = sum(news)
    if c["op"] == "append":
        # (a row that forks takes its begun page along)
        forked = sum(a % c["P"] for r, a in enumerate(lens) if r % c["K"] < c["K"] - 1)
        return {"bytes": float(T * (2 * (c["C"] + E) + _token_bytes(c)) + 2 * forked * _token_bytes(c)), "flops": 2.0 * T * c["C"]}
    seen = sum(b * a + b * (b + 1) // 2 for a, b in zip(lens, news))
    keys = sum(lens) + T
    if c["op"] == "attend":
        return {"bytes": float(keys * _token_bytes(c) + 2 * T * c["H"] * (2 * c["C"] + E)), "flops": 2.0 * c["H"] * (2 * c["C"] + E) * seen}
    return {"bytes": 2.0 * (T * c["H"] * (2 * c["D"] + E) + keys * (c["H"] * 2 * c["D"] + E)), "flops": 2.0 * c["H"] * (2 * c["D"] + E) * seen}


# ---- inputs -----------------------------------------------------------------------------------

def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return _ints(at)


def _bf16(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def _frequencies(turned, reach):
    """Radians a position of each pair: a geometric series whose slow ones are stretched from 8,192 positions to the reach."""
    f = [10000.0 ** (-2.0 * i / turned) for i in range(turned // 2)]
    factor = max(1.0, reach / 8192.0)
    out = []
    for x in f:
        turns = 8192.0 * x / (2.0 * math.pi)
        kept = min(1.0, max(0.0, (turns - 1.0) / 3.0))
        out.append(kept * x + (1.0 - kept) * x / factor)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _prepare_rotate(c, g):
    T, Q, K, D = c["T"], c["Q"], c["K"], c["D"]
    # queries and keys as they leave one projection, side by side
    x = torch.randn((T, Q + K, D), generator=g, device="cuda").to(torch.float32 if c["type"] == "f32" else torch.bfloat16)
    q, k = x[:, :Q], x[:, Q:] if K else None
    # prompts: runs of positions that begin somewhere
    run = max(1, T // 5)
    begin = torch.randint(max(1, c["reach"] - run), (T // run + 1,), generator=g, device="cuda")
    t = torch.arange(T, device="cuda")
    positions = (begin[t // run] + t % run).to(torch.int32)
    return {"op": "rotate", "q": q, "k": k, "positions": positions, "frequencies": _frequencies(c["turned"], c["reach"]), "pairs": c["pairs"], "magnitude": 1.0 + 0.1 * math.log(max(1.0, c["reach"] / 8192.0)),
            "q_out": torch.empty((T, Q, D), dtype=x.dtype, device="cuda"), "k_out": torch.empty((T, K, D), dtype=x.dtype, device="cuda") if K else None}


def _held(x, bits):
    """Latent vectors [..., C] as a cache holds them, and their scales."""
    if bits == 16:
        return x.to(torch.bfloat16), None
    top = x.abs().amax(-1)
    s = torch.exp2(torch.ceil(torch.log2(top / BLOCK_MAX)).clamp(LEAST, MOST))
    return (x / s[..., None]).clamp(-BLOCK_MAX, BLOCK_MAX).to(torch.float8_e4m3fn), s


def _cache(c, N, g):
    """Latent vectors [N, P, C], shared keys [N, P, 64] and scales [N, P] of tokens whose magnitudes differ."""
    size = torch.exp2(2.0 * torch.rand((N, c["P"], 1), generator=g, device="cuda") - 1.5)
    held, s = _held(torch.randn((N, c["P"], c["C"]), generator=g, device="cuda") * size, c["bits"])
    return held, _bf16(g, N, c["P"], E), s


def _tables(c, lens, g):
    """A table for each row, whose pages lie in any order, and the number of pages."""
    R, P = c["R"], c["P"]
    M = max(1, _pages(max(lens), P))
    N = sum(_pages(a, P) for a in lens) + 3
    order = torch.randperm(N, generator=g, device="cuda").to(torch.int32)
    table, at = torch.zeros((R, M), dtype=torch.int32, device="cuda"), 0
    for r, a in enumerate(lens):
        n = _pages(a, P)
        table[r, :n] = order[at:at + n]
        at += n
    return table, N


def _prepare_append(c, g):
    R, K, P, C = c["R"], c["K"], c["P"], c["C"]
    lens, news = _lens(c), _news(c)
    T = sum(news)
    # pages that the step touches: a row's begun one and those behind it
    touched = [_pages(a + b, P) - a // P for a, b in zip(lens, news)]
    N = sum(touched) + R + 8
    ids = torch.randperm(N, generator=g, device="cuda").tolist()
    slots, origins, at = [], [], R
    for r, (a, b) in enumerate(zip(lens, news)):
        o = a % P
        for i in range(b):
            slots.append(ids[at + (o + i) // P] * P + (o + i) % P)
            # beams of one parent take a copy each of its begun page; a request's last row has a parent of its own
            origins.append(ids[r // K] if i == 0 and o and r % K < K - 1 else -1)
        at += touched[r]
    c_cache, r_cache, scale = _cache(c, N, g)
    # latent vectors and shared keys as they leave one projection, side by side
    x = torch.randn((T, C + E), generator=g, device="cuda") * torch.exp2(4.0 * torch.rand((T, 1), generator=g, device="cuda") - 2.0)
    x = x.to(torch.bfloat16)
    return {"op": "append", "P": P, "starts": _starts(news), "c": x[:, :C], "r": x[:, C:], "slots": _ints(slots), "origins": _ints(origins),
            "c_cache": c_cache, "r_cache": r_cache, "scale": scale}


def _prepare_read(c, g):
    lens = _lens(c)
    table, N = _tables(c, lens, g)
    c_cache, r_cache, scale = _cache(c, N, g)
    return {"op": "read", "P": c["P"], "c_cache": c_cache, "r_cache": r_cache, "scale": scale, "table": table, "starts": _starts(lens),
            "c_out": torch.empty((sum(lens), c["C"]), dtype=torch.bfloat16, device="cuda"), "r_out": torch.empty((sum(lens), E), dtype=torch.bfloat16, device="cuda")}


def _prepare_attend(c, g):
    lens, news = _lens(c), _news(c)
    all_ = [a + b for a, b in zip(lens, news)]
    table, N = _tables(c, all_, g)
    c_cache, r_cache, scale = _cache(c, N, g)
    T = sum(news)
    return {"op": "attend", "P": c["P"], "new": max(news), "q_c": _bf16(g, T, c["H"], c["C"]), "q_r": _bf16(g, T, c["H"], E), "c_cache": c_cache, "r_cache": r_cache,
            "scale": scale, "table": table, "lens": _ints(all_), "starts": _starts(news), "factor": 0.08, "out": torch.empty((T, c["H"], c["C"]), dtype=torch.bfloat16, device="cuda"),
            "workspace": torch.empty(1 << 30, dtype=torch.uint8, device="cuda")}


def _prepare_prompt(c, g):
    lens, news, H, D = _lens(c), _news(c), c["H"], c["D"]
    T, keys = sum(news), sum(lens) + sum(news)
    # a head's keys and values leave one product, side by side, and so do the two parts of its queries
    kv, q = _bf16(g, keys, H, 2 * D), _bf16(g, T, H, D + E)
    return {"op": "prompt", "new": max(news), "most": max(a + b for a, b in zip(lens, news)), "q_n": q[..., :D], "q_r": q[..., D:], "k_n": kv[..., :D], "k_r": _bf16(g, keys, E), "v": kv[..., D:],
            "starts": _starts(news), "key_starts": _starts([a + b for a, b in zip(lens, news)]), "factor": 1.3 * (D + E) ** -0.5,
            "out": torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda"), "workspace": torch.empty(1 << 28, dtype=torch.uint8, device="cuda")}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"rotate": _prepare_rotate, "append": _prepare_append, "read": _prepare_read, "attend": _prepare_attend, "prompt": _prepare_prompt}[case["op"]](case, g)


# ---- the plain forms ----------------------------------------------------------------------------

def _turned(x, cos, sin, pairs):
    """x [T, heads, D] with its first pairs of numbers turned: cos and sin [T, 1, pairs]."""
    n = cos.shape[-1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if pairs else (x[..., :n], x[..., n:2 * n])
    a, b = a.float(), b.float()
    u, v = a * cos - b * sin, a * sin + b * cos
    front = torch.stack((u, v), -1).flatten(-2) if pairs else torch.cat((u, v), -1)
    return torch.cat((front.to(x.dtype), x[..., 2 * n:]), -1)


def _rotate_plain(s):
    angle = s["positions"].double()[:, None, None] * s["frequencies"]              # (64 bits: far positions are many turns)
    cos, sin = (torch.cos(angle) * s["magnitude"]).float(), (torch.sin(angle) * s["magnitude"]).float()
    return tuple(_turned(x, cos, sin, s["pairs"]) for x in (s["q"], s["k"]) if x is not None)


def _append_plain(s):
    P, slots, first = s["P"], s["slots"].long(), s["starts"][:-1].long()
    c, scale = _held(s["c"].float(), 16 if s["scale"] is None else 8)
    # the begun pages of rows that fork
    page, o, origin = slots[first] // P, slots[first] % P, s["origins"][first].long()
    take = ((torch.arange(P, device=slots.device) < o[:, None]) & (origin >= 0)[:, None])
    source = torch.where(origin >= 0, origin, page)

    def put(cache, new):
        cache[page] = torch.where(take[..., None] if cache.dim() == 3 else take, cache[source], cache[page])
        cache.view(-1, *cache.shape[2:])[slots] = new

    put(s["c_cache"].view(torch.uint8) if s["scale"] is not None else s["c_cache"], c.view(torch.uint8) if s["scale"] is not None else c)
    put(s["r_cache"], s["r"])
    if s["scale"] is None:
        return s["c_cache"], s["r_cache"]
    put(s["scale"], scale)
    return s["c_cache"], s["r_cache"], s["scale"]


def _row_of(starts, n):
    """The row of each of n tokens that lie behind one another, and its place there."""
    t = torch.arange(n, device=starts.device)
    row = torch.searchsorted(starts, t, right=True) - 1
    return row, t - starts[row]


def _latent(s, slots):
    """The latent vectors of slots, in 32 bits."""
    flat = s["c_cache"].view(-1, s["c_cache"].shape[-1])
    if s["scale"] is None:
        return flat[slots].float()
    return flat.view(torch.uint8)[slots].view(torch.float8_e4m3fn).float() * s["scale"].view(-1)[slots][..., None]


def _read_plain(s):
    P = s["P"]
    row, i = _row_of(s["starts"].long(), s["c_out"].shape[0])
    slots = s["table"][row, i // P].long() * P + i % P
    return _latent(s, slots).to(torch.bfloat16), s["r_cache"].view(-1, E)[slots]


def _softmax(w, seen):
    """Weights and their sum: w [..., keys], seen what each may see."""
    w = w.masked_fill_(~seen, -torch.inf)
    top = w.amax(-1, keepdim=True)
    w = torch.exp(w - torch.where(top > -torch.inf, top, 0.0))
    return w, w.sum(-1, keepdim=True)


def _padded(x, starts, n):
    """x [T, ...] as [R, n, ...]: what is behind a row's tokens is whatever follows."""
    return x[(starts[:-1, None] + torch.arange(n, device=x.device)).clamp(max=x.shape[0] - 1)]


def _attend_plain(s):
    starts, lens, P, n = s["starts"].long(), s["lens"].long(), s["P"], s["new"]
    T, H, C = s["q_c"].shape
    R, M = s["table"].shape
    dev = lens.device
    slots = (s["table"].long()[..., None] * P + torch.arange(P, device=dev)).view(R, M * P)
    c, r = _latent(s, slots), s["r_cache"].view(-1, E)[slots].float()
    q_c = _padded(s["q_c"], starts, n).float().view(R, n * H, C)
    q_r = _padded(s["q_r"], starts, n).float().view(R, n * H, E)
    w = torch.baddbmm(torch.bmm(q_r, r.transpose(1, 2).contiguous()), q_c, c.transpose(1, 2).contiguous()) * s["factor"]
    i = torch.arange(n, device=dev)
    seen = (lens - (starts[1:] - starts[:-1]))[:, None] + i + 1                        # keys that token i of a row sees
    w, total = _softmax(w.view(R, n, H, M * P), (torch.arange(M * P, device=dev) < seen[:, :, None])[:, :, None])
    o = torch.bmm(w.view(R, n * H, M * P), c).view(R, n, H, C)
    row, place = _row_of(starts, T)
    return torch.where(total > 0, o / total, 0.0)[row, place].to(torch.bfloat16)


def _prompt_plain(s):
    starts, key_starts, n, m = s["starts"].long(), s["key_starts"].long(), s["new"], s["most"]
    T, H, D = s["q_n"].shape
    dev = starts.device
    q = torch.cat((s["q_n"], s["q_r"]), -1)
    k = torch.cat((s["k_n"], s["k_r"][:, None].expand(-1, H, -1)), -1)
    q = _padded(q, starts, n).permute(0, 2, 1, 3).float()                              # [R, H, n, D + 64]
    k = _padded(k, key_starts, m).permute(0, 2, 3, 1).float().contiguous()             # [R, H, D + 64, m]
    v = _padded(s["v"], key_starts, m).permute(0, 2, 1, 3).float().contiguous()        # [R, H, m, D]
    count, keys = starts[1:] - starts[:-1], key_starts[1:] - key_starts[:-1]
    seen = (keys - count)[:, None] + torch.arange(n, device=dev) + 1
    w, total = _softmax(torch.matmul(q, k) * s["factor"], (torch.arange(m, device=dev) < seen[:, :, None])[:, None])
    o = torch.matmul(w, v)
    o = torch.where(total > 0, o / total, 0.0)
    row, place = _row_of(starts, T)
    return o.permute(0, 2, 1, 3)[row, place].to(torch.bfloat16)


# ---- the library's calls ------------------------------------------------------------------------

def _rotate_own(s):
    import paper_2507_16768_amd as wg
    wg.rotate(s["q"], s["k"], s["positions"], s["frequencies"], s["q_out"], s["k_out"], interleaved=s["pairs"], magnitude=s["magnitude"])
    return (s["q_out"],) if s["k"] is None else (s["q_out"], s["k_out"])


def _append_own(s):
    import paper_2507_16768_amd as wg
    wg.latent_append(s["c"], s["r"], s["slots"], s["origins"], s["c_cache"], s["r_cache"], s["scale"])
    return (s["c_cache"], s["r_cache"]) if s["scale"] is None else (s["c_cache"], s["r_cache"], s["scale"])


def _read_own(s):
    import paper_2507_16768_amd as wg
    wg.latent_read(s["c_cache"], s["r_cache"], s["scale"], s["table"], s["starts"], s["c_out"], s["r_out"])
    return s["c_out"], s["r_out"]


def _attend_own(s):
    import paper_2507_16768_amd as wg
    wg.latent_attend(s["q_c"], s["q_r"], s["c_cache"], s["r_cache"], s["scale"], s["table"], s["lens"], s["starts"], s["factor"], s["out"], s["workspace"])
    return s["out"]


def _prompt_own(s):
    import paper_2507_16768_amd as wg
    wg.latent_prompt(s["q_n"], s["q_r"], s["k_n"], s["k_r"], s["v"], s["starts"], s["key_starts"], s["factor"], s["out"], s["workspace"])
    return s["out"]


PLAIN = {"rotate": _rotate_plain, "append": _append_plain, "read": _read_plain, "attend": _attend_plain, "prompt": _prompt_plain}
OWN = {"rotate": _rotate_own, "append": _append_own, "read": _read_own, "attend": _attend_own, "prompt": _prompt_own}


def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _rotate_exact(s):
    """Pairs as complex numbers times magnitude * e^(i * position * frequency)."""
    f = s["frequencies"]
    n = f.numel()
    angle = s["positions"].double()[:, None] * f[None]
    z = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None, :]
    out = []
    for x in (s["q"], s["k"]):
        if x is None:
            continue
        y = x.double().clone()
        T, heads, _ = y.shape
        if s["pairs"]:
            p = torch.view_as_complex(y[..., :2 * n].reshape(T, heads, n, 2).contiguous()) * z
            y[..., :2 * n] = torch.view_as_real(p).reshape(T, heads, 2 * n)
        else:
            p = torch.complex(y[..., :n].contiguous(), y[..., n:2 * n].contiguous()) * z
            y[..., :n], y[..., n:2 * n] = p.real, p.imag
        out.append(y)
    return tuple(out)


def _to_8_bits(x):
    """The nearest value of the format, ties to even, 448 at most (x float64)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    unit = torch.exp2(e - 3)
    return (torch.round(x / unit) * unit).clamp(-BLOCK_MAX, BLOCK_MAX)


def _append_exact(s):
    P, slots, origins = s["P"], s["slots"].tolist(), s["origins"].tolist()
    c, r = s["c"].double(), s["r"].double()
    caches = [s["c_cache"].double(), s["r_cache"].double()]
    new = [c, r]
    if s["scale"] is not None:
        top = c.abs().amax(1) / BLOCK_MAX
        fraction, e = torch.frexp(top)
        e = torch.where(fraction == 0.5, e - 1, e)                       # the least power of two that is not below
        scale = torch.exp2(torch.where(top == 0, LEAST, e).clamp(LEAST, MOST).double())
        new = [_to_8_bits(c / scale[:, None]), r, scale]
        caches.append(s["scale"].double())
    for t, origin in enumerate(origins):
        if origin >= 0:
            page, o = divmod(slots[t], P)
            for held in caches:
                held[page, :o] = held[origin, :o]
    at = torch.tensor(slots, device=c.device)
    for held, x in zip(caches, new):
        held.reshape(-1, *held.shape[2:])[at] = x
    return tuple(caches)


def _row_slots(s, r, n):
    i = torch.arange(n, device=s["table"].device)
    return s["table"][r].long()[i // s["P"]] * s["P"] + i % s["P"]


def _exact_latent(s, at):
    x = s["c_cache"].double().reshape(-1, s["c_cache"].shape[-1])[at] if s["scale"] is None else \
        s["c_cache"].view(torch.uint8).reshape(-1, s["c_cache"].shape[-1])[at].view(torch.float8_e4m3fn).double() * s["scale"].reshape(-1)[at].double()[:, None]
    return x, s["r_cache"].reshape(-1, E)[at].double()


def _read_exact(s):
    starts = s["starts"].tolist()
    parts = [_exact_latent(s, _row_slots(s, r, starts[r + 1] - starts[r])) for r in range(len(starts) - 1)]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def _attend_exact(s):
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    out = torch.zeros(s["q_c"].shape, dtype=torch.float64, device="cuda")
    for r, total in enumerate(lens):
        c, e = _exact_latent(s, _row_slots(s, r, total))
        both = torch.cat((c, e), 1).T.contiguous()
        for t in range(starts[r], starts[r + 1]):
            n = total - (starts[r + 1] - 1 - t)
            q = torch.cat((s["q_c"][t], s["q_r"][t]), 1).double()
            out[t] = torch.softmax(q @ both[:, :n] * s["factor"], 1) @ c[:n]
    return out


def _prompt_exact(s):
    starts, key_starts = s["starts"].tolist(), s["key_starts"].tolist()
    T, H, D = s["q_n"].shape
    out = torch.zeros((T, H, D), dtype=torch.float64, device="cuda")
    for r in range(len(starts) - 1):
        a, b, ka, kb = starts[r], starts[r + 1], key_starts[r], key_starts[r + 1]
        n, m = b - a, kb - ka
        ahead = torch.arange(m, device="cuda")[None, :] - torch.arange(n, device="cuda")[:, None] > m - n
        shared = s["k_r"][ka:kb].double().T.contiguous()
        for h in range(H):
            w = s["q_n"][a:b, h].double() @ s["k_n"][ka:kb, h].double().T.contiguous() + s["q_r"][a:b, h].double() @ shared
            out[a:b, h] = torch.softmax((w * s["factor"]).masked_fill(ahead, -torch.inf), 1) @ s["v"][ka:kb, h].double()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _rotate_exact, "append": _append_exact, "read": _read_exact, "attend": _attend_exact, "prompt": _prompt_exact}[case["op"]](s)
