"""What the operators of beam search over a paged 8-bit cache are timed on.

A case names the operator (`op`) and its sizes:

  beam    beam_select and reorder_rows: the best `K` continuations of each of `G` requests over beams and a
          vocabulary of `V` tokens under the grammar's masks, and `L` layers of `row` values of recurrent state
          that follow their parents.  `type` is that of the logits, `masked` is false where no grammar is in force,
          `first` is the step after the prompt, when one beam of each request lives
  pages   page_step: tables, slots and positions of `R` rows (requests of `K` beams each) of up to `len` cached
          tokens that take up to `new` tokens more, in pages of `P`
  append  cache_append: the keys and values of those tokens into the 8-bit cache of `H` heads of `D` values, with a
          scale for each page and head
  attend  cache_attend: attention of up to `new` tokens of each of `R` rows, `Q` query heads over `H` cached ones

Rows have lengths of their own, spread over the range up to `len` (and `new`).  Where `own` is false the operators
are computed in elementary operations in 32 bits; where it is true by this library's kernels.
"""
import torch

own = False

BLOCK_MAX = 448.0                     # the largest value of the 8-bit format (e4m3)
LEAST, MOST = -64, 120                # exponents that a scale may have


def listed():
    return [
        # one request with four beams on a small vocabulary: latency of a step
        {"name": "beam one request", "op": "beam", "G": 1, "K": 4, "V": 32000, "type": "f32", "masked": True, "first": False, "L": 1, "row": 64},
        # the step after the prompts of sixteen outline requests: one live beam each
        {"name": "beam first step", "op": "beam", "G": 16, "K": 4, "V": 128256, "type": "bf16", "masked": True, "first": True, "L": 4, "row": 1000},
        # a batch of 256 rows on the largest vocabulary, states of eight layers
        {"name": "beam batch", "op": "beam", "G": 32, "K": 8, "V": 151936, "type": "bf16", "masked": True, "first": False, "L": 8, "row": 8192},
        # free generation: no mask, fp32, an odd vocabulary and an odd number of beams
        {"name": "beam unmasked", "op": "beam", "G": 24, "K": 5, "V": 100003, "type": "f32", "masked": False, "first": False, "L": 2, "row": 4099},
        # a token for each of 256 requests without beams: nothing but new slots and now and then a page
        {"name": "pages decode", "op": "pages", "R": 256, "K": 1, "len": 4096, "new": 1, "P": 16},
        # 64 requests of eight beams with long outputs, whose beams change parents
        {"name": "pages beams", "op": "pages", "R": 512, "K": 8, "len": 16384, "new": 1, "P": 16},
        # prompts of ragged lengths for 64 requests, some of which have a cached prefix
        {"name": "pages prompts", "op": "pages", "R": 64, "K": 1, "len": 2000, "new": 1500, "P": 32},
        # a token for each of 256 rows, beams that fork among them
        {"name": "append decode", "op": "append", "R": 256, "K": 4, "len": 1024, "new": 1, "P": 16, "H": 8, "D": 128},
        # eight prompts
        {"name": "append prompts", "op": "append", "R": 8, "K": 1, "len": 500, "new": 2048, "P": 32, "H": 8, "D": 128},
        # one request with a long context, a token at a time
        {"name": "attend one long", "op": "attend", "R": 1, "len": 30000, "new": 1, "P": 16, "Q": 32, "H": 8, "D": 128},
        # a batch of rows of ragged lengths, an odd number of query heads per cached one
        {"name": "attend batch", "op": "attend", "R": 128, "len": 8192, "new": 1, "P": 32, "Q": 28, "H": 4, "D": 128},
        # prompts in chunks behind a cached prefix
        {"name": "attend prompts", "op": "attend", "R": 4, "len": 2048, "new": 2000, "P": 32, "Q": 32, "H": 8, "D": 128},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("beam", "pages", "append", "attend"))
    if op == "beam":
        K = rng.choice((2, 3, 4, 5, 8, 16))
        V = _spread(rng, 1000, 151936)
        most = max(1, min(64, 38_000_000 // (V * K)))
        return {"op": op, "G": _spread(rng, 1, most), "K": K, "V": V, "type": rng.choice(("f32", "bf16")), "masked": rng.random() < 0.7,
                "first": rng.random() < 0.2, "L": rng.choice((1, 2, 4, 8)), "row": _spread(rng, 16, 8192)}
    if op == "pages":
        K = rng.choice((1, 1, 2, 4, 5, 8))
        return {"op": op, "R": K * _spread(rng, 1, 512 // K), "K": K, "len": _spread(rng, 40, 16384), "new": rng.choice((1, 1, 4, _spread(rng, 2, 1500))) if K == 1 else 1,
                "P": rng.choice((16, 32, 64))}
    P, H, D = rng.choice((16, 32, 64)), rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 256))
    if op == "append":
        if rng.random() < 0.5:
            K = rng.choice((1, 2, 4))
            return {"op": op, "R": K * _spread(rng, 1, 256 // K), "K": K, "len": _spread(rng, 20, 2048), "new": 1, "P": P, "H": H, "D": D}
        return {"op": op, "R": _spread(rng, 1, 8), "K": 1, "len": _spread(rng, 16, 1024), "new": _spread(rng, 2, 2048), "P": P, "H": H, "D": min(D, 128)}
    Q = H * rng.choice((1, 4, 7, 8) if H < 8 else (1, 4))
    if rng.random() < 0.6:
        R = _spread(rng, 1, 128)
        return {"op": op, "R": R, "len": _spread(rng, 30, min(30000, 1_000_000 // R)), "new": rng.choice((1, 1, 1, 5)), "P": P, "Q": Q, "H": H if D < 256 else min(H, 2), "D": D} \
            if D < 256 else {"op": op, "R": R, "len": _spread(rng, 30, min(16000, 500_000 // R)), "new": 1, "P": P, "Q": min(H, 2) * 4, "H": min(H, 2), "D": D}
    return {"op": op, "R": _spread(rng, 1, 4), "len": _spread(rng, 16, 2048), "new": _spread(rng, 20, 2000), "P": P, "Q": Q, "H": H, "D": min(D, 128)}


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


def _kinds(R):
    """What the mask of each row allows: free text, a class of tokens, a literal's few tokens."""
    return [(0.97, 0.97, 0.02, 0.0)[r % 4] for r in range(R)]


def work(case):
    c = case
    if c["op"] == "beam":
        R, V, e = c["G"] * c["K"], c["V"], 4 if c["type"] == "f32" else 2
        live = [r for r in range(R) if not c["first"] or r % c["K"] == 0]
        logits = sum((_kinds(R)[r] if c["masked"] else 1.0) * V for r in live)
        read = logits * e + (len(live) * ((V + 31) // 32) * 4 if c["masked"] else 0) + R * 12
        return {"bytes": read + R * 20 + 2.0 * c["L"] * R * c["row"] * 4, "flops": 4.0 * logits}
    lens, news = _lens(c), _news(c)
    T = sum(news)
    if c["op"] == "pages":
        entries = sum(_pages(n, c["P"]) for n in lens) if c["K"] > 1 else 0
        fresh = sum(_pages(a + b, c["P"]) - _pages(a, c["P"]) for a, b in zip(lens, news))
        return {"bytes": 8.0 * entries + 8.0 * fresh + 12.0 * T + 20.0 * c["R"], "flops": 0.0}
    values = T * c["H"] * c["D"]
    if c["op"] == "append":
        return {"bytes": 2.0 * (2 * values + values), "flops": 4.0 * values}
    seen = sum(b * a + b * (b + 1) // 2 for a, b in zip(lens, news))
    cached = sum(a + b for a, b in zip(lens, news)) * c["H"] * c["D"] * 2
    return {"bytes": cached + 4.0 * T * c["Q"] * c["D"], "flops": 4.0 * c["Q"] * c["D"] * seen}


# ---- inputs -----------------------------------------------------------------------------------

def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _prepare_beam(c, g):
    G, K, V = c["G"], c["K"], c["V"]
    R, W = G * K, (V + 31) // 32
    x = torch.randn((R, V), generator=g, device="cuda") * 2.0
    # what a model favours stands out
    likely = torch.randint(V, (R, 64), generator=g, device="cuda")
    x.scatter_add_(1, likely, torch.empty((R, 64), device="cuda").exponential_(0.25, generator=g))
    x = x.to(torch.float32 if c["type"] == "f32" else torch.bfloat16)
    mask = None
    if c["masked"]:
        share = torch.tensor(_kinds(R), device="cuda")[:, None]
        allowed = torch.rand((R, W * 32), generator=g, device="cuda") < share
        few = torch.randint(V, (R, 6), generator=g, device="cuda")
        allowed.scatter_(1, few, True)
        allowed[:, V:] = False
        bit = torch.ones(1, dtype=torch.int64, device="cuda") << torch.arange(32, device="cuda")
        mask = (allowed.view(R, W, 32) * bit).sum(2)
        mask = torch.where(mask >= 1 << 31, mask - (1 << 32), mask).to(torch.int32)
    scores = -20.0 * torch.rand(R, generator=g, device="cuda")
    if c["first"]:
        scores.view(G, K)[:, 0] = 0.0
        scores.view(G, K)[:, 1:] = -torch.inf
    states = torch.randint(1, 1 << 20, (R, 2), generator=g, device="cuda", dtype=torch.int32)
    layers = torch.randn((c["L"], R, c["row"]), generator=g, device="cuda")
    return {"op": "beam", "K": K, "logits": x, "mask": mask, "scores": scores, "states": states, "layers": layers,
            "out_scores": torch.empty_like(scores), "parents": torch.empty(R, dtype=torch.int32, device="cuda"),
            "tokens": torch.empty(R, dtype=torch.int32, device="cuda"), "out_states": torch.empty_like(states),
            "out_layers": torch.empty_like(layers), "workspace": torch.empty(64 << 20, dtype=torch.uint8, device="cuda")}


def _prepare_pages(c, g):
    R, K, P = c["R"], c["K"], c["P"]
    lens, news = _lens(c), _news(c)
    n = _ints([_pages(a, P) for a in lens])
    M = max(_pages(a + b, P) for a, b in zip(lens, news)) + 1
    N = R * M + 16
    order = torch.randperm(N, generator=g, device="cuda").to(torch.int32)
    table = order[:R * M].view(R, M).clone()
    if K > 1:
        # beams share what they had in common: a request's rows have its first row's pages up to a place of their own
        fork = (torch.rand(R, generator=g, device="cuda") * n).to(torch.int32)
        shared = torch.arange(M, device="cuda") < fork[:, None]
        first = table.view(R // K, K, M)[:, :1].expand(-1, K, -1).reshape(R, M)
        table = torch.where(shared, first, table)
    used = torch.zeros(N, dtype=torch.bool, device="cuda")
    inside = torch.arange(M, device="cuda") < n[:, None]
    used[table[inside].long()] = True
    free = order[~used[order.long()]]
    ring_and_one = torch.full((N + 1,), -1, dtype=torch.int32, device="cuda")
    ring, taken = ring_and_one[:N], 1000
    ring[(torch.arange(free.numel(), device="cuda") + taken) % N] = free
    parents = None
    if K > 1:
        parents = torch.arange(R, device="cuda") // K * K + torch.randint(K, (R,), generator=g, device="cuda")
        parents = torch.where(torch.rand(R, generator=g, device="cuda") < 0.02, -1, parents).to(torch.int32)
    T = sum(news)
    empty = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
    return {"op": "pages", "K": K, "P": P, "table": table, "new_table": torch.full_like(table, -1) if K > 1 else table, "lens": _ints(lens), "counts": _ints(news),
            "parents": parents, "ring": ring, "ring_and_one": ring_and_one, "counters": torch.tensor([taken, taken + free.numel()], dtype=torch.int64, device="cuda"),
            "new_counters": torch.zeros(2, dtype=torch.int64, device="cuda"), "new_lens": empty(R), "starts": empty(R + 1), "slots": empty(T),
            "positions": empty(T), "origins": empty(T), "workspace": torch.empty(1 << 20, dtype=torch.uint8, device="cuda")}


def _quantised(x):
    """A cache's values and scales for each page and head: x [pages, heads, ., .]."""
    top = x.abs().amax((2, 3))
    e = torch.ceil(torch.log2(top / BLOCK_MAX)).clamp(LEAST, MOST)
    s = torch.exp2(e)
    return (x / s[:, :, None, None]).clamp(-BLOCK_MAX, BLOCK_MAX).to(torch.float8_e4m3fn), s


def _cache(N, H, P, D, g):
    """Keys [N, H, P, D] and values [N, H, D, P] of pages whose magnitudes differ."""
    size = torch.exp2(3.0 * torch.rand((N, H, 1, 1), generator=g, device="cuda") - 2.0)
    k, ks = _quantised(torch.randn((N, H, P, D), generator=g, device="cuda") * size)
    v, vs = _quantised(torch.randn((N, H, D, P), generator=g, device="cuda") * size)
    return k, v, ks, vs


def _prepare_append(c, g):
    R, K, P, H, D = c["R"], c["K"], c["P"], c["H"], c["D"]
    lens, news = _lens(c), _news(c)
    T = sum(news)
    # pages that the step touches: a row's begun one and those behind it
    touched = [_pages(a + b, P) - a // P for a, b in zip(lens, news)]
    N = sum(touched) + R + 64
    ids = torch.randperm(N, generator=g, device="cuda").tolist()
    slots, origins, at = [], [], R
    for r, (a, b) in enumerate(zip(lens, news)):
        o = a % P
        for i in range(b):
            slots.append(ids[at + (o + i) // P] * P + (o + i) % P)
            # beams of one parent take a copy each of its begun page; a request's last row has a parent of its own
            origins.append(ids[r // K] if i == 0 and o and r % K < K - 1 else -1)
        at += touched[r]
    k_cache, v_cache, k_scale, v_scale = _cache(N, H, P, D, g)
    # keys and values as they leave one projection, side by side
    kv = torch.randn((T, 2, H, D), generator=g, device="cuda") * torch.exp2(4.0 * torch.rand((T, 2, H, 1), generator=g, device="cuda") - 2.0)
    kv = kv.to(torch.bfloat16)
    return {"op": "append", "R": R, "P": P, "k": kv[:, 0], "v": kv[:, 1], "slots": _ints(slots), "origins": _ints(origins),
            "k_cache": k_cache, "v_cache": v_cache, "k_scale": k_scale, "v_scale": v_scale}


def _prepare_attend(c, g):
    R, P, Q, H, D = c["R"], c["P"], c["Q"], c["H"], c["D"]
    lens, news = _lens(c), _news(c)
    all_ = [a + b for a, b in zip(lens, news)]
    T, M = sum(news), _pages(max(all_), P)
    N = sum(_pages(a, P) for a in all_) + 3
    order = torch.randperm(N, generator=g, device="cuda").to(torch.int32)
    table, at = torch.zeros((R, M), dtype=torch.int32, device="cuda"), 0
    for r, a in enumerate(all_):
        n = _pages(a, P)
        table[r, :n] = order[at:at + n]
        at += n
    k_cache, v_cache, k_scale, v_scale = _cache(N, H, P, D, g)
    starts = [0]
    for b in news:
        starts.append(starts[-1] + b)
    q = (torch.randn((T, Q, D), generator=g, device="cuda") * 1.5).to(torch.bfloat16)
    return {"op": "attend", "P": P, "new": max(news), "q": q, "k_cache": k_cache, "v_cache": v_cache, "k_scale": k_scale, "v_scale": v_scale,
            "table": table, "lens": _ints(all_), "starts": _ints(starts), "out": torch.empty_like(q), "scale": D ** -0.5,
            "workspace": torch.empty(128 << 20, dtype=torch.uint8, device="cuda")}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"beam": _prepare_beam, "pages": _prepare_pages, "append": _prepare_append, "attend": _prepare_attend}[case["op"]](case, g)


# ---- the plain forms ----------------------------------------------------------------------------

def _beam_plain(s):
    K, x, scores = s["K"], s["logits"].float(), s["scores"]
    R, V = x.shape
    rows = torch.arange(R, device=x.device)
    allowed = x > -torch.inf
    if s["mask"] is not None:
        t = torch.arange(V, device=x.device)
        allowed &= (s["mask"][:, t >> 5] >> (t & 31) & 1).bool()
    allowed &= (scores > -torch.inf)[:, None]
    x = torch.where(allowed, x, -torch.inf)
    top = x.amax(1, keepdim=True)
    gap = torch.where(x == top, 0.0, x - top)                  # (also where both are infinite)
    total = torch.where(allowed, torch.exp(gap), 0.0).sum(1, keepdim=True)
    step = torch.where(allowed, gap - torch.log(total), -torch.inf)
    # the K best of a row: the larger logit, then the lower token
    bits = (x + 0.0).view(torch.int32)
    order = (bits ^ (bits >> 31 & 0x7FFFFFFF)).long() << 32 | (V - 1 - torch.arange(V, device=x.device))
    best = order.topk(min(K, V), dim=1).indices
    found = scores[:, None] + step.gather(1, best)
    # the K best of a request's rows: the better score, then the lower beam
    n = best.shape[1]
    found = found.view(R // K, K * n)
    value, at = found.sort(dim=1, descending=True, stable=True)
    value, at = value[:, :K].reshape(R), at[:, :K].reshape(R)
    there = value > -torch.inf
    parent = rows // K * K + at // n
    token = best[parent, at % n]
    parents = torch.where(there, parent, -1).to(torch.int32)
    states = torch.where(there[:, None], s["states"][parent], torch.tensor([-1, 0], dtype=torch.int32, device=x.device))
    layers = torch.where(there[None, :, None], s["layers"][:, parent], 0.0)
    return torch.where(there, value, -torch.inf), parents, torch.where(there, token, -1).to(torch.int32), states, layers


def _pages_plain(s):
    K, P, table, lens, counts = s["K"], s["P"], s["table"], s["lens"].long(), s["counts"].long()
    R, M = table.shape
    N, T = s["ring"].numel(), s["slots"].numel()
    G, dev, out = R // K, table.device, s["new_table"]
    rows, cols = torch.arange(R, device=dev), torch.arange(M, device=dev)
    taken, given = s["counters"][0], s["counters"][1]
    if s["parents"] is None:
        length, kept = lens, table
        have = _pages(length, P)
        at = (length // P).clamp(max=M - 1)
        fork = torch.zeros(R, dtype=torch.bool, device=dev)
    else:
        p = s["parents"].long()
        of = (p // K == rows // K) & (p >= 0)
        source = torch.where(of, p, rows)
        length = torch.where(of, lens[source], 0)
        have = _pages(length, P)
        kept = torch.where(cols < have[:, None], table[source], -1)
        # a begun page that another row of the request has too is copied
        begun = (length % P != 0) & (counts > 0)
        at = (length // P).clamp(max=M - 1)
        mine = torch.where(begun, kept.gather(1, at[:, None])[:, 0], -2).view(G, K)
        theirs = kept.view(G, K, M).gather(2, at.view(G, 1, K).expand(-1, K, -1))                  # [request, other, row]
        other = ~torch.eye(K, dtype=torch.bool, device=dev)
        fork = (other & (theirs == mine[:, None, :])).any(1).reshape(R)
    want = _pages(length + counts, P)
    fits = (want <= M).view(G, K).all(1)
    need = (fork.long() + want - have).view(G, K) * fits[:, None]
    total = need.sum(1)
    end = total.cumsum(0)
    served = fits & ((total == 0) | (end <= given - taken))
    begin = ((end - total)[:, None] + need.cumsum(1) - need).reshape(R)
    used = torch.where(served, total, 0).sum()
    served = served[:, None].expand(G, K).reshape(R)
    fork = fork & served
    released = torch.zeros((), dtype=torch.int64, device=dev)
    if s["parents"] is not None:
        out.copy_(torch.where(cols < have[:, None], kept, out))
        # pages that no row refers to any more go back, by request, place and row
        old = torch.where(cols < _pages(lens, P)[:, None], table, -1).view(G, K, M)
        now = torch.where(fork[:, None] & (cols == at[:, None]), -1, kept).view(G, K, M)
        k = torch.arange(K, device=dev)
        again = (old[:, :, None] == old[:, None, :]) & (k[:, None] > k[None, :])[None, :, :, None]
        gone = (old >= 0) & ~again.any(2) & ~(old[:, :, None] == now[:, None, :]).any(2)
        gone, old = gone.transpose(1, 2).reshape(-1), old.transpose(1, 2).reshape(-1)
        rank = gone.cumsum(0)
        released = rank[-1]
        s["ring_and_one"][torch.where(gone, (given + rank - 1) % N, N)] = old       # (what is not released goes behind the ring)
    place = cols - have[:, None] + fork[:, None].long()
    page = s["ring"][(taken + begin[:, None] + place.clamp(min=0)) % N]
    fresh = served[:, None] & (cols >= have[:, None]) & (cols < want[:, None])
    first = s["ring"][(taken + begin) % N]
    moved = fork[:, None] & (cols == at[:, None])
    before = kept.gather(1, at[:, None])[:, 0]
    out.copy_(torch.where(fresh, page, torch.where(moved, first[:, None], out)))
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), counts.cumsum(0)])
    t = torch.arange(T, device=dev)
    row = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[row]
    position = length[row] + i
    slot = torch.where(served[row], out[row, (position // P).clamp(max=M - 1)].long() * P + position % P, -1)
    origin = torch.where((i == 0) & fork[row], before[row].long(), -1)
    counters = torch.stack([taken + used, given + released])
    i32 = torch.int32
    return (out, torch.where(served, length + counts, length).to(i32), starts.to(i32), slot.to(i32), position.to(i32), origin.to(i32), counters, s["ring"])


def _rounded(x, scale):
    return (x / scale).clamp(-BLOCK_MAX, BLOCK_MAX).to(torch.float8_e4m3fn)


def _append_one(x, cache, scale, slots, origins, runs, P, flip):
    """x [T, H, D] into cache [N, H, P, D] (flip: [N, H, D, P]) and scale [N, H]."""
    T, H, D = x.shape
    dev = x.device
    slot = slots.long()
    page, off = slot // P, slot % P
    lead = torch.ones(T, dtype=torch.bool, device=dev)
    lead[1:] = page[1:] != page[:-1]
    run = lead.cumsum(0) - 1
    # of each run of tokens in one page: the page, where its earlier tokens are, how many
    at = torch.where(lead, run, runs)
    spread = lambda v: torch.zeros(runs + 1, dtype=torch.int64, device=dev).index_put((at,), v)[:runs]
    real = torch.arange(runs, device=dev) <= run[-1]
    page_of, begin = spread(page), spread(off)
    from_ = spread(torch.where(origins.long() >= 0, origins.long(), page))
    buf = torch.zeros((runs, P, H, D), device=dev)
    buf[run, off] = x.float()
    new = torch.zeros((runs, P), dtype=torch.bool, device=dev)
    new[run, off] = True
    buf = buf.permute(0, 2, 1, 3)
    top = torch.where(buf.abs() < torch.inf, buf.abs(), 0.0).amax((2, 3))
    need = torch.exp2(torch.ceil(torch.log2(top / BLOCK_MAX)).clamp(LEAST, MOST))
    was = torch.where((begin > 0)[:, None], scale[from_], 0.0)
    now = torch.maximum(need, was)
    old = cache.view(torch.uint8)[from_].view(cache.dtype).float()
    if flip:
        old = old.transpose(2, 3)
    old = _rounded(old * was[:, :, None, None], now[:, :, None, None])
    there = cache.view(torch.uint8)[page_of].view(cache.dtype)
    if flip:
        there = there.transpose(2, 3)
    p = torch.arange(P, device=dev)
    first = (p < begin[:, None])[:, None, :, None]
    put = torch.where(new[:, None, :, None], _rounded(buf, now[:, :, None, None]).view(torch.uint8),
                      torch.where(first, old.view(torch.uint8), there.contiguous().view(torch.uint8)))
    if flip:
        put = put.transpose(2, 3)
    # (what is behind the last run repeats the first)
    pick = torch.where(real, torch.arange(runs, device=dev), 0)
    cache.view(torch.uint8)[page_of[pick]] = put[pick]
    scale[page_of[pick]] = now[pick]


def _append_plain(s):
    T = s["slots"].numel()
    runs = min(T, T // s["P"] + 2 * s["R"])
    _append_one(s["k"], s["k_cache"], s["k_scale"], s["slots"], s["origins"], runs, s["P"], False)
    _append_one(s["v"], s["v_cache"], s["v_scale"], s["slots"], s["origins"], runs, s["P"], True)
    return s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]


def _attend_plain(s):
    q, table, lens, starts, P = s["q"], s["table"].long(), s["lens"].long(), s["starts"].long(), s["P"]
    T, Q, D = q.shape
    R, M = table.shape
    H, dev, n = s["k_cache"].shape[1], q.device, s["new"]
    k = s["k_cache"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * s["k_scale"][table][..., None, None]      # [R, M, H, P, D]
    v = s["v_cache"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * s["v_scale"][table][..., None, None]      # [R, M, H, D, P]
    k = k.permute(0, 2, 4, 1, 3).reshape(R, H, D, M * P)
    v = v.permute(0, 2, 1, 4, 3).reshape(R, H, M * P, D)
    i = torch.arange(n, device=dev)
    count = starts[1:] - starts[:-1]
    padded = q.float()[(starts[:-1, None] + i).clamp(max=T - 1)]                       # [R, n, Q, D]
    padded = padded.view(R, n, H, Q // H, D).permute(0, 2, 3, 1, 4).reshape(R, H, Q // H * n, D)
    w = torch.matmul(padded, k) * s["scale"]
    seen = (lens - count)[:, None] + i + 1                                             # keys that token i of a row sees
    masked = torch.arange(M * P, device=dev) >= seen[:, :, None]
    w = w.view(R, H, Q // H, n, M * P).masked_fill_(masked[:, None, None], -torch.inf)
    top = w.amax(-1, keepdim=True)
    w = torch.exp(w - torch.where(top > -torch.inf, top, 0.0))
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(R, H, Q // H * n, M * P), v).view(R, H, Q // H, n, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(R, n, Q, D)
    t = torch.arange(T, device=dev)
    row = torch.searchsorted(starts, t, right=True) - 1
    return o[row, t - starts[row]].to(q.dtype)


# ---- the library's calls ------------------------------------------------------------------------

def _beam_own(s):
    import paper_2507_16768_amd as wg
    wg.beam_select(s["logits"], s["mask"], s["scores"], s["states"], s["K"], s["out_scores"], s["parents"], s["tokens"], s["out_states"], s["workspace"])
    wg.reorder_rows(s["layers"], s["parents"], s["out_layers"], axis=1)
    return s["out_scores"], s["parents"], s["tokens"], s["out_states"], s["out_layers"]


def _pages_own(s):
    import paper_2507_16768_amd as wg
    wg.page_step(s["table"], s["lens"], s["counts"], s["parents"], s["K"], s["P"], s["ring"], s["counters"],
                 s["new_table"], s["new_lens"], s["starts"], s["slots"], s["positions"], s["origins"], s["new_counters"], s["workspace"])
    return s["new_table"], s["new_lens"], s["starts"], s["slots"], s["positions"], s["origins"], s["new_counters"], s["ring"]


def _append_own(s):
    import paper_2507_16768_amd as wg
    wg.cache_append(s["k"], s["v"], s["slots"], s["origins"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]


def _attend_own(s):
    import paper_2507_16768_amd as wg
    wg.cache_attend(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["starts"], s["scale"], s["out"], s["workspace"])
    return s["out"]


PLAIN = {"beam": _beam_plain, "pages": _pages_plain, "append": _append_plain, "attend": _attend_plain}
OWN = {"beam": _beam_own, "pages": _pages_own, "append": _append_own, "attend": _attend_own}


def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _beam_exact(s):
    K, R = s["K"], s["scores"].numel()
    V = s["logits"].shape[1]
    scores, states = s["scores"].double().tolist(), s["states"].cpu()
    best = []
    for r in range(R):
        if not scores[r] > -float("inf"):
            best.append([])
            continue
        x = s["logits"][r].double()
        ok = x > -torch.inf
        if s["mask"] is not None:
            words = s["mask"][r].long() & 0xFFFFFFFF
            ok &= (words[:, None] >> torch.arange(32, device=x.device) & 1).bool().reshape(-1)[:V]
        ids = ok.nonzero()[:, 0]
        values, by = x[ids].sort(descending=True, stable=True)
        norm = torch.logsumexp(values, 0) if len(values) else 0.0
        best.append(list(zip((scores[r] + (values[:K] - norm)).tolist(), ids[by[:K]].tolist())))
    out_s, out_p, out_t, out_st = [], [], [], []
    for r0 in range(0, R, K):
        found = [(-v, r, j, t) for r in range(r0, r0 + K) for j, (v, t) in enumerate(best[r])]
        found = sorted(found)[:K]
        for v, r, _, t in found:
            out_s.append(-v); out_p.append(r); out_t.append(t); out_st.append(states[r].tolist())
        for _ in range(K - len(found)):
            out_s.append(-float("inf")); out_p.append(-1); out_t.append(-1); out_st.append([-1, 0])
    layers = s["layers"].double()
    moved = torch.stack([layers[:, p] if p >= 0 else torch.zeros_like(layers[:, 0]) for p in out_p], 1)
    return torch.tensor(out_s, dtype=torch.float64), torch.tensor(out_p, dtype=torch.int32), torch.tensor(out_t, dtype=torch.int32), torch.tensor(out_st, dtype=torch.int32), moved


def _to_8_bits(x):
    """The nearest value of the format, ties to even, 448 at most (x float64)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    unit = torch.exp2(e - 3)
    return (torch.round(x / unit) * unit).clamp(-BLOCK_MAX, BLOCK_MAX)


def _append_exact(s):
    P, slots, origins = s["P"], s["slots"].tolist(), s["origins"].tolist()
    out = []
    for x, cache, scale, flip in ((s["k"], s["k_cache"], s["k_scale"], False), (s["v"], s["v_cache"], s["v_scale"], True)):
        x = x.double()
        held, sc = cache.double(), scale.double()
        was, was_scale = held.clone(), sc.clone()
        t = 0
        while t < len(slots):
            page, o = divmod(slots[t], P)
            n = 1
            while t + n < len(slots) and slots[t + n] == slots[t] + n and o + n < P:
                n += 1
            part = x[t:t + n].transpose(0, 1)                       # [H, n, D]
            _, e = torch.frexp(part.abs().amax((1, 2)) / BLOCK_MAX)
            top = part.abs().amax((1, 2)) / BLOCK_MAX
            e = torch.where(top == torch.exp2(e.double() - 1), e - 1, e)          # the least power of two that is not below
            e = torch.where(top == 0, LEAST, e).clamp(LEAST, MOST)
            new = torch.exp2(e.double())
            source = origins[t] if origins[t] >= 0 else page
            if o:
                new = torch.maximum(new, was_scale[source])
                early = was[source][:, :, :o] if flip else was[source][:, :o]
                early = _to_8_bits(early * (was_scale[source] / new)[:, None, None])
                if flip:
                    held[page, :, :, :o] = early
                else:
                    held[page, :, :o] = early
            late = _to_8_bits(part / new[:, None, None])
            if flip:
                held[page, :, :, o:o + n] = late.transpose(1, 2)
            else:
                held[page, :, o:o + n] = late
            sc[page] = new
            t += n
        out.append((held, sc))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _attend_exact(s):
    P, starts, lens = s["P"], s["starts"].tolist(), s["lens"].tolist()
    T, Q, D = s["q"].shape
    H = s["k_cache"].shape[1]
    out = torch.zeros((T, Q, D), dtype=torch.float64, device="cuda")
    for r, length in enumerate(lens):
        n = starts[r + 1] - starts[r]
        pages = s["table"][r, :_pages(length, P)].long()
        k = (s["k_cache"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * s["k_scale"].double()[pages][:, :, None, None])
        v = (s["v_cache"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).double() * s["v_scale"].double()[pages][:, :, None, None])
        visible = torch.arange(length, device="cuda")[None, :] <= (length - n + torch.arange(n, device="cuda"))[:, None]
        for h in range(Q):
            kh = k[:, h // (Q // H)].reshape(-1, D)[:length]
            vh = v[:, h // (Q // H)].transpose(1, 2).reshape(-1, D)[:length]
            w = s["q"][starts[r]:starts[r + 1], h].double() @ kh.T * s["scale"]
            w = torch.softmax(w.masked_fill(~visible, -torch.inf), -1)
            out[starts[r]:starts[r + 1], h] = w @ vh
    return out


def exact(case, seed):
    if case["op"] == "pages":
        return None                                 # whole numbers only
    if case["op"] == "attend" and case["R"] * case["Q"] > 6000:
        return None                                 # (a product for each row and head: over twenty seconds)
    return {"beam": _beam_exact, "append": _append_exact, "attend": _attend_exact}[case["op"]](prepare(case, seed))
