"""Rotary positions and the cache of latent vectors against their definitions in 64 bits (GPU)."""
import math

import pytest
import torch

import paper_2507_16768_amd as wg

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
HALF = 2.0 ** -8                      # the rounding of a bfloat16 number, relative
E = 64


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def bf16(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


# ---- rotary positions ---------------------------------------------------------------------------

def turned(x, positions, f, beside, magnitude):
    """The definition in 64 bits, and how large the numbers are that an output is a sum of."""
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    n = f.numel()
    a = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if beside else (slice(0, n), slice(n, 2 * n))
    angle = positions.double()[:, None, None] * f
    c, s = torch.cos(angle) * magnitude, torch.sin(angle) * magnitude
    p, q = x[..., a[0]].double(), x[..., a[1]].double()
    y[..., a[0]], y[..., a[1]] = p * c - q * s, p * s + q * c
    size[..., a[0]] = size[..., a[1]] = (p.abs() + q.abs()) * magnitude
    return y, size


def close_turned(got, x, positions, f, beside, magnitude):
    """Sines and cosines are off by a few units of 2^-24 (the angle's rounding, the series', the factor's), products and sums by as many: 2^-21 of what is
    summed; then the rounding of the type."""
    want, size = turned(x, positions, f, beside, magnitude)
    step = HALF if x.dtype == torch.bfloat16 else 2.0 ** -24
    off = (got.double() - want).abs()
    assert (off <= want.abs() * step + size * 2.0 ** -21).all(), (off - want.abs() * step).max()
    behind = got[..., 2 * f.numel():]
    assert torch.equal(behind, x[..., 2 * f.numel():])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("beside", [False, True])
@pytest.mark.parametrize("T,Q,K,D,rotated", [(1, 32, 8, 128, 128), (3, 1, 0, 64, 64), (257, 5, 2, 80, 20), (70, 3, 3, 192, 64), (19, 2, 1, 7, 6), (33, 4, 1, 66, 2), (2, 1, 1, 1024, 1024), (1000, 16, 1, 64, 64), (150, 4, 2, 80, 40), (61, 7, 1, 36, 12),
                                               (3001, 24, 2, 80, 20), (9, 300, 5, 1022, 514)])
def test_rotate(dtype, beside, T, Q, K, D, rotated):
    g = gen(T * D + beside)
    x = torch.randn((T, Q + K, D), generator=g, device="cuda").to(dtype)
    q, k = x[:, :Q], x[:, Q:] if K else None
    positions = torch.randint(0, 1 << 20, (T,), generator=g, device="cuda").to(torch.int32)
    f = torch.tensor(wg.rotary_frequencies(rotated), device="cuda")
    q_out, k_out = torch.full_like(q, 7.0).contiguous(), torch.full_like(k, 7.0).contiguous() if K else None
    wg.rotate(q, k, positions, f, q_out, k_out, interleaved=beside, magnitude=1.3)
    close_turned(q_out, q, positions, f, beside, 1.3)
    if K:
        close_turned(k_out, k, positions, f, beside, 1.3)
    # in place: the same numbers
    y = x.clone()
    wg.rotate(y[:, :Q], y[:, Q:] if K else None, positions, f, y[:, :Q], y[:, Q:] if K else None, interleaved=beside, magnitude=1.3)
    assert torch.equal(y[:, :Q], q_out) and (not K or torch.equal(y[:, Q:], k_out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("beside", [False, True])
def test_rotate_part_of_wider_heads_at_odd_places(dtype, beside):
    """The last 64 of heads of 192, as latent attention's queries have them, and rows that begin between multiples of 16 bytes; what lies around stays."""
    for shift, D in ((0, 64), (1, 64), (3, 33)):
        g = gen(shift)
        room = torch.randn((11, 4, 192 + 4), generator=g, device="cuda").to(dtype)
        at = slice(128 + shift, 128 + shift + D)
        x = room[:, :, at].clone()
        positions = torch.arange(11, dtype=torch.int32, device="cuda") * 1001
        f = torch.tensor(wg.rotary_frequencies(32), device="cuda")
        was = room.clone()
        wg.rotate(room[:, :, at], None, positions, f, room[:, :, at], None, interleaved=beside)
        close_turned(room[:, :, at], x, positions, f, beside, 1.0)
        was[:, :, at] = room[:, :, at]
        assert torch.equal(room, was)


def test_rotate_far_and_negative_positions():
    positions = ints([0, -1, 2 ** 31 - 1, -2 ** 31, 1, 123456789])
    x = torch.randn((6, 2, 8), generator=gen(5), device="cuda")
    f = torch.tensor([1.0, 0.1, 1e-5, 0.0], dtype=torch.float64, device="cuda")
    out = torch.empty_like(x)
    wg.rotate(x, None, positions, f, out, None)
    close_turned(out, x, positions, f, False, 1.0)
    assert torch.equal(out[0], x[0])


# ---- the cache ------------------------------------------------------------------------------------

def to_8_bits(x):
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    unit = torch.exp2(e - 3)
    return (torch.round(x / unit) * unit).clamp(-448, 448)


def held(c):
    """Vectors [T, C] in 8 bits, as values, and their scales (64 bits, from the definition)."""
    x = c.double()
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(1) / 448
    f, e = torch.frexp(top)
    e = torch.where(f == 0.5, e - 1, e)
    scale = torch.exp2(torch.where(top == 0, -64, e).clamp(-64, 120).double())
    y = torch.where(x.isinf(), torch.sign(x) * 448, x / scale[:, None])
    return torch.where(x.isnan(), x, to_8_bits(y)), scale


def new_cache(g, N, P, C, bits):
    size = torch.exp2(2.0 * torch.rand((N, P, 1), generator=g, device="cuda") - 1.5)
    x = torch.randn((N, P, C), generator=g, device="cuda") * size
    r = bf16(g, N, P, E)
    if bits == 16:
        return x.to(torch.bfloat16), r, None
    v, s = held(x.view(-1, C))
    return v.float().to(torch.float8_e4m3fn).view(N, P, C), r, s.float().view(N, P)


def values(c_cache, scale):
    """What the cache's vectors stand for, [slots, C] in 64 bits."""
    x = c_cache.double() if scale is None else c_cache.double() * scale.double()[..., None]
    return x.reshape(-1, x.shape[-1])


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("T,P", [(1, 16), (5, 32), (300, 64), (1100, 16)])
def test_append(bits, C, T, P):
    g = gen(T + C)
    N = T // P * 2 + 6
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    both = torch.randn((T, C + E), generator=g, device="cuda") * torch.exp2(40 * torch.rand((T, 1), generator=g, device="cuda") - 20)
    both = both.to(torch.bfloat16)
    if T >= 300:
        for i, v in enumerate((0.0, INF, -INF, NAN, 3.38e38, 1e-38, 448.0, 2.0 ** -120)):
            both[10 + i, 17] = v
        both[20, :C] = 0.0
        both[21, :C] = INF
        both[22, :C] = NAN
        both[23, :C] = 2.0 ** -90
    c, r = both[:, :C], both[:, C:]
    slots = torch.randperm(N * P, generator=g, device="cuda")[:T].to(torch.int32)
    if T > 4:
        slots[1], slots[2], slots[3] = -1, N * P, -2 ** 31
    want = [c_cache.clone(), r_cache.clone(), None if scale is None else scale.clone()]
    ok = (slots >= 0) & (slots < N * P)
    at = slots[ok].long()
    if bits == 8:
        v, s = held(c)
        want[0].view(torch.uint8).view(-1, C)[at] = v.float().to(torch.float8_e4m3fn).view(torch.uint8)[ok]
        want[2].view(-1)[at] = s.float()[ok]
    else:
        want[0].view(-1, C)[at] = c[ok]
    want[1].view(-1, E)[at] = r[ok]
    wg.latent_append(c, r, slots, None, c_cache, r_cache, scale)
    if bits == 8:                     # a NaN's sign is of no account
        nan = c_cache.float().isnan()
        both_nan = torch.equal(nan, want[0].float().isnan())
        numbers = same(torch.where(nan, 0, c_cache.view(torch.uint8)), torch.where(nan, 0, want[0].view(torch.uint8)))
        assert both_nan and numbers
    else:
        assert same(c_cache, want[0])
    assert same(r_cache, want[1]) and (scale is None or same(scale, want[2]))


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("P,T", [(16, 7), (64, 40), (32, 1500)])
def test_append_forks(bits, P, T):
    """Rows that take a begun page along: at every place of a page, from pages that others take too, with origins that are none."""
    g = gen(P)
    C, R = 512, min(T, 40)
    N = 2 * R + T // P + 4
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    slots, origins = [], []
    for i in range(R):
        slots.append((R + i) * P + i * 5 % P)
        origins.append([i // 2, -1, N, 2 ** 31 - 1][0 if i % 4 < 2 else i % 4] if i else R)      # (the first: its own page)
    for i in range(T - R):
        slots.append((2 * R + i // P) * P + i % P)
        origins.append(-1)
    c, r = bf16(g, T, C), bf16(g, T, E)
    v, s = held(c)
    caches = [c_cache.view(torch.uint8) if bits == 8 else c_cache, r_cache] + ([scale] if bits == 8 else [])
    new = [v.float().to(torch.float8_e4m3fn).view(torch.uint8) if bits == 8 else c, r, s.float()]
    want = [x.clone() for x in caches]
    for t in range(T):
        page, o = divmod(slots[t], P)
        for w, x in zip(want, new):
            if 0 <= origins[t] < N:
                w[page, :o] = w[origins[t], :o].clone()
            w[page, o] = x[t]
    wg.latent_append(c, r, ints(slots), ints(origins), c_cache, r_cache, scale)
    for w, x in zip(want, caches):
        assert same(x, w)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("P,lens", [(16, [1]), (32, [0, 100, 0, 31, 32, 33, 0]), (64, [700, 65, 1, 900])])
def test_read(bits, C, P, lens):
    g = gen(C + P)
    R, M = len(lens), max(1, max((n + P - 1) // P for n in lens))
    N = R * M + 2
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    if bits == 8:
        scale[1, 2], scale[2, 3] = 2.0 ** -64, 2.0 ** 110
    table = torch.randperm(N, generator=g, device="cuda")[:R * M].view(R, M).to(torch.int32)
    bad = R > 3
    if bad:
        table[R - 1, 0], table[1, 1] = -5, N            # pages that are none read as zeros
    head, tail = 3, 5
    starts = [head]
    for n in lens:
        starts.append(starts[-1] + n)
    total = starts[-1] + tail
    c_out = torch.full((total, C + 16), 9.0, dtype=torch.bfloat16, device="cuda")
    r_out = torch.full((total, E), 9.0, dtype=torch.bfloat16, device="cuda")
    wg.latent_read(c_cache, r_cache, scale, table, ints(starts), c_out[:, 8:8 + C], r_out)
    v, r = values(c_cache, scale), r_cache.view(-1, E)
    want_c, want_r = torch.full_like(c_out, 9.0), torch.full_like(r_out, 9.0)
    for row, n in enumerate(lens):
        for i in range(n):
            page = int(table[row, i // P])
            there = 0 <= page < N
            want_c[starts[row] + i, 8:8 + C] = v[page * P + i % P].to(torch.bfloat16) if there else 0.0
            want_r[starts[row] + i] = r[page * P + i % P] if there else 0.0
    assert torch.equal(c_out, want_c) and torch.equal(r_out, want_r)


def test_read_behind_the_table():
    """More tokens asked of a row than its table has pages for."""
    g = gen(1)
    c_cache, r_cache, _ = new_cache(g, 4, 16, 256, 16)
    c_out, r_out = torch.full((40, 256), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((40, E), 9.0, dtype=torch.bfloat16, device="cuda")
    wg.latent_read(c_cache, r_cache, None, ints([[2, 1]]), ints([0, 37]), c_out, r_out)
    assert torch.equal(c_out[:32], torch.cat((c_cache[2], c_cache[1]))) and (c_out[32:37] == 0).all() and (c_out[37:] == 9).all()
    assert torch.equal(r_out[:32], torch.cat((r_cache[2], r_cache[1]))) and (r_out[32:37] == 0).all() and (r_out[37:] == 9).all()


# ---- attention ------------------------------------------------------------------------------------

def attention(q, k, v, seen, factor):
    """q [n, H, A], k [m, H or 1, A], v [m, H or 1, B], seen [n]: outputs [n, H, B] and how far a kernel's may be off, in 64 bits.

    A score, a sum of A products in fp32, is off by A * 2^-24 of the sum of their magnitudes at the most, and so is its weight, relatively (with some units for exp2).  A weight's rounding is
    HALF of it; with d_j the relative errors, sum w_j (1 + d_j) v_j / sum w_j (1 + d_j) is off by sum w_j |d_j| |v_j - out| <= max |d| (sum w_j |v_j| + |out|).  Then the output's rounding."""
    q, k, v = q.double(), k.double(), v.double()
    m = k.shape[0]
    dead = torch.arange(m, device=q.device)[None, None, :] >= seen[:, None, None]
    kt = k.permute(1, 2, 0).contiguous()
    s = torch.matmul(q.permute(1, 0, 2), kt).permute(1, 0, 2) * factor                  # [n, H, m]
    size = torch.matmul(q.abs().permute(1, 0, 2), kt.abs()).permute(1, 0, 2) * abs(factor)
    d = HALF + ((q.shape[-1] * 2.0 ** -24) * torch.where(dead, 0.0, size).amax(-1, keepdim=True) + 2.0 ** -20 if m else 0.0)
    w = torch.softmax(s.masked_fill(dead, -INF), -1)
    w = torch.where(dead, 0.0, w)
    if not m:
        return torch.zeros((*q.shape[:2], v.shape[-1]), dtype=torch.float64, device=q.device), torch.zeros((*q.shape[:2], v.shape[-1]), dtype=torch.float64, device=q.device)
    vt = v.permute(1, 0, 2)
    out = torch.matmul(w.permute(1, 0, 2), vt).permute(1, 0, 2)
    spread = torch.matmul(w.permute(1, 0, 2), vt.abs()).permute(1, 0, 2)
    return out, d * (spread + out.abs()) * 1.01 + HALF * out.abs()


def pages_of(g, lens, P, extra=3, columns=0):
    R, M = len(lens), max(1, columns, max((n + P - 1) // P for n in lens))
    N = sum((n + P - 1) // P for n in lens) + extra
    order = torch.randperm(N, generator=g, device="cuda").to(torch.int32)
    table, at = torch.full((R, M), -77, dtype=torch.int32, device="cuda"), 0
    for r, n in enumerate(lens):
        n = (n + P - 1) // P
        table[r, :n] = order[at:at + n]
        at += n
    return table, N


def starts_of(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def check_attend(g, lens, counts, H, C, bits, P, factor=0.06, extra=0, spoil=None, columns=0):
    """lens: cached tokens, those of the call among them.  extra: tokens of the call that belong to no row."""
    table, N = pages_of(g, lens, P, columns=columns)
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    starts = starts_of(counts)
    T = starts[-1] + extra
    v, r = values(c_cache, scale), r_cache.view(-1, E).double()
    # what lies behind the rows' tokens, in their last pages and in pages of none, is nothing to them
    used = torch.zeros(N * P, dtype=torch.bool, device="cuda")
    slots = []
    for row, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        slots.append(table[row].long()[i // P] * P + i % P)
        used[slots[-1]] = True
    c_cache.view(torch.uint8).view(N * P, -1)[~used] = 0xFF
    r_cache.view(-1, E)[~used] = NAN
    if scale is not None:
        scale.view(-1)[~used] = INF
    wide = torch.randn((T, H, C + E + 16), generator=g, device="cuda").to(torch.bfloat16)
    q_c, q_r = wide[..., 8:8 + C], wide[..., 8 + C:8 + C + E]
    if spoil:
        spoil(c_cache, r_cache, scale, slots)
        v, r = values(c_cache, scale), r_cache.view(-1, E).double()
    out = torch.full((T, H, C), 5.0, dtype=torch.bfloat16, device="cuda")
    work = torch.full((max(16, wg.latent_attend_workspace(T, len(lens), H, C, table.shape[1], P)),), 0xFF, dtype=torch.uint8, device="cuda")
    wg.latent_attend(q_c, q_r, c_cache, r_cache, scale, table, ints(lens), ints(starts), factor, out, work)
    assert (out[starts[-1]:] == 5.0).all()
    for row, n in enumerate(counts):
        at = slice(starts[row], starts[row + 1])
        c, e = v[slots[row]], r[slots[row]]
        seen = (lens[row] - n + 1 + torch.arange(n, device="cuda")).clamp(min=0)
        if spoil:
            yield out[at], torch.cat((q_c[at], q_r[at]), -1), torch.cat((c, e), -1)[:, None], c[:, None], seen
            continue
        want, off = attention(torch.cat((q_c[at], q_r[at]), -1), torch.cat((c, e), -1)[:, None], c[:, None], seen, factor)
        got = out[at].double()
        assert ((got - want).abs() <= off).all(), (row, n, lens[row], ((got - want).abs() - off).max())
        assert (got[seen == 0] == 0).all()


def run_attend(*a, **k):
    assert list(check_attend(*a, **k)) == []


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("H", [1, 3, 16, 24, 128])
def test_attend_single_tokens(bits, C, H):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 513]
    run_attend(gen(H), lens, [1] * len(lens), H, C, bits, 16, extra=2)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("H,P,lens,counts", [
    (16, 32, [700, 40, 4, 1000], [4, 4, 4, 3]), (16, 64, [0, 3, 900, 130], [0, 5, 130, 130]), (24, 16, [600, 77], [203, 77]), (128, 64, [1300, 129], [2, 7]),
    (5, 16, [2000, 0, 1, 33], [13, 0, 0, 33]), (1, 32, [500, 333], [200, 333]), (40, 64, [90], [90])])
def test_attend_many_tokens(bits, H, P, lens, counts):
    run_attend(gen(H + P), lens, counts, H, 512, bits, P, extra=3)
    run_attend(gen(H + P), lens, counts, H, 256, bits, P)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("H,lens,counts", [(16, [9001], [1]), (128, [5003], [1]), (16, [6000, 100, 12001, 1], [1, 1, 2, 1]), (32, [7000], [6]), (8, [4000] * 3 + [130], [40, 1, 7, 130]), (128, [3000, 2500], [1, 1])])
def test_attend_in_shares(bits, H, lens, counts):
    """Long rows, whose keys are cut; the table has room for more."""
    run_attend(gen(H), lens, counts, H, 512, bits, 64, columns=300)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("columns", [2500, 200, 0])
@pytest.mark.parametrize("H,P,lens,counts", [
    (128, 16, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 513], [1] * 20), (64, 32, [700, 0, 33, 129, 1000], [1] * 5), (24, 16, [600, 77], [203, 77]),
    (5, 16, [2000, 0, 1, 33], [13, 0, 0, 33]), (40, 64, [90], [90]), (32, 64, [1, 400, 64, 5], [1, 2, 1, 0]), (16, 64, [500, 40, 4, 1000], [4, 4, 4, 3])])
def test_attend_tables_of_other_widths(bits, C, columns, H, P, lens, counts):
    """How wide a table is decides over how many query rows a workgroup takes; what it holds behind the rows' tokens is nothing to them."""
    run_attend(gen(H + P), lens, counts, H, C, bits, P, extra=1, columns=columns)


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("H,lens,counts,at", [(128, [200], [3], 198), (16, [130], [130], 100), (64, [64], [64], 33)])
def test_attend_numbers_that_are_none_under_wide_tables(bad, H, lens, counts, at):
    def spoil(c_cache, r_cache, scale, slots):
        c_cache.view(-1, 512)[int(slots[0][at]), 5] = bad
    for got, q, k, v, seen in check_attend(gen(at), lens, counts, H, 512, 16, 64, spoil=spoil, columns=2000):
        v, k = v.clone(), k.clone()
        v[at, :, 5], k[at, :, 5] = 0.0, 0.0
        blind = seen <= at
        want, off = attention(q[blind], k, v, seen[blind], 0.06)
        assert ((got[blind].double() - want).abs() <= off).all()
        assert got[~blind][..., 5].isnan().all()


def test_attend_rows_without_tokens_and_many_rows():
    counts = [1 if r % 3 else 0 for r in range(150)]
    run_attend(gen(9), [(r * 37) % 290 if r % 5 else 0 for r in range(150)], counts, 16, 256, 8, 16)


def test_attend_more_rows_than_have_their_keys_cut():
    counts = [1] * 1100
    run_attend(gen(2), [(r * 7) % 300 for r in range(1100)], counts, 2, 256, 16, 64)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("R,H,n", [(600, 16, 400), (520, 128, 300), (300, 48, 1400), (1024, 2, 150)])
def test_attend_many_rows_of_few_tokens(bits, R, H, n):
    """More tiles than the chip holds at a time, and rows of no tokens and of none cached among them."""
    lens = [r * 7919 % n if r % 11 else 0 for r in range(R)]
    run_attend(gen(R), lens, [(1, 1, 0, 2, 1)[r % 5] for r in range(R)], H, 512, bits, 64, columns=50)


@pytest.mark.parametrize("bits", [8, 16])
def test_attend_large_scores_and_scales(bits):
    """Scores in the hundreds, so that one key has all the weight, and vectors whose sizes differ by 2^12."""
    run_attend(gen(4), [300, 1000, 77], [1, 2, 3], 16, 512, bits, 32, factor=1.0)
    run_attend(gen(4), [300, 1000, 77], [1, 2, 3], 16, 512, bits, 32, factor=-0.5)
    run_attend(gen(4), [300, 1000, 77], [1, 2, 3], 16, 512, bits, 32, factor=0.0)


@pytest.mark.parametrize("bits,bad", [(8, NAN), (16, NAN), (16, INF), (16, -INF)])
@pytest.mark.parametrize("H,lens,counts,at", [(16, [300], [4], 298), (16, [130], [130], 100), (128, [200], [3], 198), (3, [200], [50], 170), (64, [64], [64], 33)])
def test_attend_numbers_that_are_none_are_nothing_to_those_that_do_not_see_them(bits, bad, H, lens, counts, at):
    def spoil(c_cache, r_cache, scale, slots):
        s = int(slots[0][at])
        c_cache.view(-1, 512)[s, 5] = bad
    for got, q, k, v, seen in check_attend(gen(at), lens, counts, H, 512, bits, 64, spoil=spoil):
        v = v.clone()
        k = k.clone()
        v[at, :, 5], k[at, :, 5] = 0.0, 0.0
        blind = seen <= at
        want, off = attention(q[blind], k, v, seen[blind], 0.06)
        assert ((got[blind].double() - want).abs() <= off).all()
        assert got[~blind][..., 5].isnan().all()


def test_attend_pages_that_are_none():
    """A page number out of range among a row's own reads as zeros."""
    g = gen(3)
    c_cache, r_cache, _ = new_cache(g, 5, 16, 256, 16)
    q_c, q_r, out = bf16(g, 1, 16, 256), bf16(g, 1, 16, E), torch.empty((1, 16, 256), dtype=torch.bfloat16, device="cuda")
    wg.latent_attend(q_c, q_r, c_cache, r_cache, None, ints([[1, 5, -1, 2]]), ints([64]), ints([0, 1]), 0.1, out)
    c = torch.cat((c_cache[1], torch.zeros_like(c_cache[:2]).view(32, 256), c_cache[2]))
    r = torch.cat((r_cache[1], torch.zeros_like(r_cache[:2]).view(32, E), r_cache[2]))
    want, off = attention(torch.cat((q_c, q_r), -1), torch.cat((c, r), -1)[:, None], c[:, None], torch.tensor([64], device="cuda"), 0.1)
    assert ((out.double() - want).abs() <= off).all()


def check_prompt(g, counts, keys, H, D, extra=0, factor=0.08, spoil=None):
    starts, key_starts = starts_of(counts), starts_of(keys)
    T, N = starts[-1] + extra, key_starts[-1] + 5
    q, kv = bf16(g, T, H, D + E + 8), bf16(g, N, H, 2 * D + 8)
    q_n, q_r, k_n, v = q[..., :D], q[..., D:D + E], kv[..., :D], kv[..., D:2 * D]
    k_r = bf16(g, N, E + 8)[:, 8:]
    kv[key_starts[-1]:] = NAN
    k_r[key_starts[-1]:] = NAN
    if spoil:
        spoil(v)
    out = torch.full((T, H, D), 5.0, dtype=torch.bfloat16, device="cuda")
    work = torch.full((max(16, wg.latent_prompt_workspace(T, len(counts), H, D, N)),), 0xFF, dtype=torch.uint8, device="cuda")
    wg.latent_prompt(q_n, q_r, k_n, k_r, v, ints(starts), ints(key_starts), factor, out, work)
    assert (out[starts[-1]:] == 5.0).all()
    for row, n in enumerate(counts):
        at, to = slice(starts[row], starts[row + 1]), slice(key_starts[row], key_starts[row + 1])
        seen = (keys[row] - n + 1 + torch.arange(n, device="cuda")).clamp(min=0)
        k = torch.cat((k_n[to], k_r[to][:, None].expand(-1, H, -1)), -1)
        if spoil:
            yield out[at], torch.cat((q_n[at], q_r[at]), -1), k, v[to], seen
            continue
        want, off = attention(torch.cat((q_n[at], q_r[at]), -1), k, v[to], seen, factor)
        got = out[at].double()
        assert ((got - want).abs() <= off).all(), (row, n, keys[row], ((got - want).abs() - off).max())
        assert (got[seen == 0] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,counts,keys", [
    (1, [1], [1]), (2, [1, 1, 1], [5, 64, 65]), (3, [127, 128, 129], [127, 128, 129]), (4, [300, 0, 70, 10], [300, 20, 500, 0]), (2, [20, 5], [10, 5]), (8, [40], [4000]), (16, [131], [2500]),
    (1, [1000], [1000]), (5, [3, 600, 64], [1000, 601, 64]), (32, [200] * 6, [200] * 6), (2, [1] * 70, list(range(70)))])
def test_prompt(D, H, counts, keys):
    for _ in check_prompt(gen(H + D), counts, keys, H, D, extra=2):
        pass


@pytest.mark.parametrize("H,R", [(16, 100), (4, 500), (2, 1030)])
def test_prompt_many_rows_of_few_tokens(H, R):
    counts = [(1, 4, 0, 7)[r % 4] for r in range(R)]
    for _ in check_prompt(gen(H), counts, [r * 31 % 290 for r in range(R)], H, 128, extra=1):
        pass


def test_prompt_large_scores():
    for factor in (1.5, -1.0, 0.0):
        for _ in check_prompt(gen(7), [100, 200], [130, 200], 2, 128, factor=factor):
            pass


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("at", [0, 63, 64, 130, 199])
def test_prompt_values_that_are_none(bad, at):
    def spoil(v):
        v[at, :, 7] = bad
    for got, q, k, v, seen in check_prompt(gen(at), [200], [200], 2, 128, spoil=spoil):
        v = v.clone()
        v[at, :, 7] = 0.0
        want, off = attention(q, k, v, seen, 0.08)
        fine = ((got.double() - want).abs() <= off)
        blind = seen <= at
        assert fine[blind].all() and not got[~blind][..., 7].isfinite().any()
        fine[..., 7] = True
        assert fine.all()


def test_attend_fewer_tokens_than_the_rows_have():
    """A call with the first tokens of a step alone: they see what they see in the whole call.  And rows that begin behind the first token."""
    for H, lens, counts in ((16, [700, 90, 3000], [3, 40, 200]), (128, [300, 2000], [2, 5])):
        g = gen(H)
        table, N = pages_of(g, lens, 32)
        c_cache, r_cache, _ = new_cache(g, N, 32, 512, 16)
        T = sum(counts)
        q_c, q_r = bf16(g, T, H, 512), bf16(g, T, H, E)
        starts, lens_t, out = ints(starts_of(counts)), ints(lens), torch.empty((T, H, 512), dtype=torch.bfloat16, device="cuda")
        work = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        wg.latent_attend(q_c, q_r, c_cache, r_cache, None, table, lens_t, starts, 0.07, out, work)
        v, r = values(c_cache, None), r_cache.view(-1, E).double()
        for few in (1, counts[0], counts[0] + 1, T - 1):
            part = torch.empty((few, H, 512), dtype=torch.bfloat16, device="cuda")
            wg.latent_attend(q_c[:few], q_r[:few], c_cache, r_cache, None, table, lens_t, starts, 0.07, part, work)
            at = 0
            for row, n in enumerate(counts):
                m = max(0, min(n, few - at))
                if m:
                    i = torch.arange(lens[row], device="cuda")
                    slots = table[row].long()[i // 32] * 32 + i % 32
                    seen = lens[row] - n + 1 + torch.arange(m, device="cuda")
                    want, off = attention(torch.cat((q_c[at:at + m], q_r[at:at + m]), -1), torch.cat((v[slots], r[slots]), -1)[:, None], v[slots][:, None], seen, 0.07)
                    assert ((part[at:at + m].double() - want).abs() <= off).all()
                at += n
        # the rows begin at token 5
        moved = torch.full((T + 7, H, 512), 5.0, dtype=torch.bfloat16, device="cuda")
        q_c2, q_r2 = torch.zeros((T + 7, H, 512), dtype=torch.bfloat16, device="cuda"), torch.zeros((T + 7, H, E), dtype=torch.bfloat16, device="cuda")
        q_c2[5:5 + T], q_r2[5:5 + T] = q_c, q_r
        wg.latent_attend(q_c2, q_r2, c_cache, r_cache, None, table, lens_t, starts + 5, 0.07, moved, work)
        assert (moved[:5] == 5).all() and (moved[5 + T:] == 5).all()
        at = 0
        for row, n in enumerate(counts):
            i = torch.arange(lens[row], device="cuda")
            slots = table[row].long()[i // 32] * 32 + i % 32
            seen = lens[row] - n + 1 + torch.arange(n, device="cuda")
            want, off = attention(torch.cat((q_c[at:at + n], q_r[at:at + n]), -1), torch.cat((v[slots], r[slots]), -1)[:, None], v[slots][:, None], seen, 0.07)
            assert ((moved[5 + at:5 + at + n].double() - want).abs() <= off).all()
            at += n


def test_prompt_fewer_tokens_and_shifted_rows():
    g = gen(31)
    H, D, counts, keys = 4, 128, [200, 30], [900, 31]
    T, N = sum(counts), sum(keys)
    q_n, q_r, k_n, k_r, v = bf16(g, T + 4, H, D), bf16(g, T + 4, H, E), bf16(g, N + 3, H, D), bf16(g, N + 3, E), bf16(g, N + 3, H, D)
    work = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    for few in (T + 4, 150, 201):
        out = torch.full((few, H, D), 5.0, dtype=torch.bfloat16, device="cuda")
        wg.latent_prompt(q_n[:few], q_r[:few], k_n, k_r, v, ints([2, 202, 232]), ints([3, 903, 934]), 0.08, out, work)
        assert (out[:2] == 5).all() and (out[232:] == 5).all()
        for b, n, kb, m in ((2, 200, 3, 900), (202, 30, 903, 31)):
            have = max(0, min(n, few - b))
            if have:
                seen = m - n + 1 + torch.arange(have, device="cuda")
                k = torch.cat((k_n[kb:kb + m], k_r[kb:kb + m][:, None].expand(-1, H, -1)), -1)
                want, off = attention(torch.cat((q_n[b:b + have], q_r[b:b + have]), -1), k, v[kb:kb + m], seen, 0.08)
                assert ((out[b:b + have].double() - want).abs() <= off).all()


def test_prompt_shared_and_broadcast_keys():
    """Heads that share keys and values (a stride of 0), as one cached head read by many."""
    g = gen(32)
    q_n, q_r, k_n, k_r, v = bf16(g, 70, 6, 64), bf16(g, 70, 6, E), bf16(g, 300, 1, 64), bf16(g, 300, E), bf16(g, 300, 1, 64)
    out = torch.empty((70, 6, 64), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    wg.latent_prompt(q_n, q_r, k_n.expand(-1, 6, -1), k_r, v.expand(-1, 6, -1), ints([0, 70]), ints([0, 300]), 0.1, out, work)
    want, off = attention(torch.cat((q_n, q_r), -1), torch.cat((k_n, k_r[:, None]), -1).expand(-1, 6, -1), v.expand(-1, 6, -1), 231 + torch.arange(70, device="cuda"), 0.1)
    assert ((out.double() - want).abs() <= off).all()


@pytest.mark.parametrize("bits", [8, 16])
def test_a_cache_behind_2_to_32_bytes(bits):
    """Slots whose vectors lie more than 2^32 bytes from the first one's."""
    P, C, H = 64, 512, 16
    N = (1 << 32) // (P * C * (1 if bits == 8 else 2)) + 4
    g = gen(bits)
    c_cache = torch.empty((N, P, C), dtype=torch.float8_e4m3fn if bits == 8 else torch.bfloat16, device="cuda")
    r_cache, scale = torch.empty((N, P, E), dtype=torch.bfloat16, device="cuda"), torch.empty((N, P), device="cuda") if bits == 8 else None
    table = ints([[N - 1, 0, N - 3]])
    i = torch.arange(170, device="cuda")
    slots = table[0].long()[i // P] * P + i % P
    c, r = bf16(g, 170, C), bf16(g, 170, E)
    wg.latent_append(c, r, slots.to(torch.int32), None, c_cache, r_cache, scale)
    c_out, r_out = torch.empty_like(c), torch.empty_like(r)
    wg.latent_read(c_cache, r_cache, scale, table, ints([0, 170]), c_out, r_out)
    kept = held(c)[0] * held(c)[1][:, None] if bits == 8 else c.double()
    assert torch.equal(c_out.double(), kept.to(torch.bfloat16).double()) and torch.equal(r_out, r)
    q_c, q_r, out = bf16(g, 1, H, C), bf16(g, 1, H, E), torch.empty((1, H, C), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(max(16, wg.latent_attend_workspace(1, 1, H, C, 3, P)), dtype=torch.uint8, device="cuda")
    wg.latent_attend(q_c, q_r, c_cache, r_cache, scale, table, ints([170]), ints([0, 1]), 0.06, out, work)
    want, off = attention(torch.cat((q_c, q_r), -1), torch.cat((kept, r.double()), -1)[:, None], kept[:, None], torch.tensor([170], device="cuda"), 0.06)
    assert ((out.double() - want).abs() <= off).all()


# ---- together -------------------------------------------------------------------------------------

def test_calls_on_another_stream_and_in_graphs():
    """Each call on a stream of its own, and all of them captured into two graphs that share a workspace, replayed with other work between: the same numbers every time."""
    g = gen(11)
    P, C, H, D, lens, counts = 32, 512, 16, 128, [700, 90, 3000], [3, 1, 2]
    table, N = pages_of(g, lens, P)
    c_cache, r_cache, scale = new_cache(g, N, P, C, 8)
    starts, T = ints(starts_of(counts)), sum(counts)
    q_c, q_r, c, r = bf16(g, T, H, C), bf16(g, T, H, E), bf16(g, T, C), bf16(g, T, E)
    slots = torch.cat([table[row].long()[torch.arange(n - m, n, device="cuda") // P] * P + torch.arange(n - m, n, device="cuda") % P for row, (n, m) in enumerate(zip(lens, counts))]).to(torch.int32)
    positions = torch.cat([torch.arange(n - m, n, device="cuda") for n, m in zip(lens, counts)]).to(torch.int32)
    f = torch.tensor(wg.rotary_frequencies(E), device="cuda")
    key_starts, lens_t = ints(starts_of(lens)), ints(lens)
    total = sum(lens)
    kv, q_n = bf16(g, total, H, 2 * D), bf16(g, T, H, D)
    work = torch.empty(max(wg.latent_attend_workspace(T, 3, H, C, table.shape[1], P), wg.latent_prompt_workspace(T, 3, H, D, total)), dtype=torch.uint8, device="cuda")

    def outputs():
        return [torch.zeros_like(q_r), torch.zeros((T, 1, E), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(q_c), torch.zeros((total, C), dtype=torch.bfloat16, device="cuda"),
                torch.zeros((total, E), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(q_n)]

    def first(o):
        wg.rotate(q_r, r[:, None], positions, f, o[0], o[1])
        wg.latent_append(c, o[1][:, 0], slots, None, c_cache, r_cache, scale)
        wg.latent_attend(q_c, o[0], c_cache, r_cache, scale, table, lens_t, starts, 0.05, o[2], work)

    def second(o):
        wg.latent_read(c_cache, r_cache, scale, table, key_starts, o[3], o[4])
        wg.latent_prompt(q_n, o[0], kv[..., :D], o[4], kv[..., D:], starts, key_starts, 0.07, o[5], work)

    eager = outputs()
    first(eager); second(eager)
    torch.cuda.synchronize()
    other, side = outputs(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first(other); second(other)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    o = outputs()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        first(o)
    with torch.cuda.graph(graphs[1]):
        second(o)
    for _ in range(4):
        for t in o:
            t.zero_()
        work.fill_(0xAA)
        graphs[0].replay()
        graphs[1].replay()
        busy = torch.randn(1000, device="cuda").sum().item()
        assert math.isfinite(busy) and all(torch.equal(a, b) for a, b in zip(eager, o))


@pytest.mark.parametrize("bits", [8, 16])
def test_a_model_s_steps(bits):
    """Prompts, then steps of beams that fork, through pages, rotary positions, the cache and attention in both forms, against the same model without pages in 64 bits."""
    g = gen(21)
    H, C, D, P, K, G, V = 4, 256, 64, 16, 3, 2, 64
    R, pages, columns = K * G, 200, 12
    w_k, w_v = torch.randn((H, D, C), generator=g, device="cuda") / 16, torch.randn((H, D, C), generator=g, device="cuda") / 16
    f = torch.tensor(wg.rotary_frequencies(E, factor=4.0, original=64), device="cuda")
    factor = (D + E) ** -0.5
    c_cache = torch.empty((pages, P, C), dtype=torch.float8_e4m3fn if bits == 8 else torch.bfloat16, device="cuda")
    r_cache, scale = torch.empty((pages, P, E), dtype=torch.bfloat16, device="cuda"), torch.empty((pages, P), device="cuda") if bits == 8 else None
    ring, counters = torch.randperm(pages, generator=g, device="cuda").to(torch.int32), torch.tensor([0, pages], device="cuda")
    table, lens = torch.zeros((R, columns), dtype=torch.int32, device="cuda"), ints([0] * R)
    past = [[] for _ in range(R)]                          # of each row: (vector as the cache holds it, turned key)
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    for step in range(12):
        counts = [[37, 0, 0, 50, 0, 0][r] if step == 0 else 1 for r in range(R)]
        parents = None if step == 0 else ints([r // K * K + (0 if step == 1 else (r * 7 + step) % K) for r in range(R)])
        T = sum(counts)
        table2, lens2, counters2 = table if parents is None else torch.zeros_like(table), torch.empty_like(lens), torch.empty_like(counters)
        starts, slots, positions, origins = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (R + 1, T, T, T))
        wg.page_step(table, lens, ints(counts), parents, K if parents is not None else 1, P, ring, counters, table2, lens2, starts, slots, positions, origins, counters2, work)
        table, lens, counters = table2, lens2, counters2
        c, r, q_n, q_r = bf16(g, T, C), bf16(g, T, 1, E), bf16(g, T, H, D), bf16(g, T, H, E)
        r2, q2 = torch.empty_like(r), torch.empty_like(q_r)
        wg.rotate(q_r, r, positions, f, q2, r2, interleaved=True)
        wg.latent_append(c, r2[:, 0], slots, origins, c_cache, r_cache, scale)
        # the model without pages
        if parents is not None:
            past = [list(past[p]) for p in parents.tolist()]
        kept = held(c)
        kept = kept[0] * kept[1][:, None] if bits == 8 else c.double()
        want_r, _ = turned(r, positions, f, True, 1.0)
        close_turned(r2, r, positions, f, True, 1.0)
        at = starts.tolist()
        assert positions.tolist() == [len(past[r]) + i for r in range(R) for i in range(counts[r])]
        for row in range(R):
            past[row] += [(kept[t], r2[t, 0].double()) for t in range(at[row], at[row + 1])]
        assert lens.tolist() == [len(p) for p in past]
        q_c = torch.matmul(q_n.float().permute(1, 0, 2), w_k).permute(1, 0, 2).to(torch.bfloat16)          # [T, H, C]
        out_c = torch.empty((T, H, C), dtype=torch.bfloat16, device="cuda")
        wg.latent_attend(q_c, q2, c_cache, r_cache, scale, table, lens, starts, factor, out_c, work)
        total = sum(len(p) for p in past)
        key_starts = ints(starts_of([len(p) for p in past]))
        all_c, all_r = torch.empty((total, C), dtype=torch.bfloat16, device="cuda"), torch.empty((total, E), dtype=torch.bfloat16, device="cuda")
        wg.latent_read(c_cache, r_cache, scale, table, key_starts, all_c, all_r)
        assert torch.equal(all_c.double(), torch.stack([x[0] for p in past for x in p]).to(torch.bfloat16).double())
        k_n = torch.matmul(all_c.float(), w_k.transpose(1, 2).contiguous()).permute(1, 0, 2).to(torch.bfloat16).contiguous()    # [N, H, D]
        v = torch.matmul(all_c.float(), w_v.transpose(1, 2).contiguous()).permute(1, 0, 2).to(torch.bfloat16).contiguous()
        out = torch.empty_like(q_n)
        wg.latent_prompt(q_n, q2, k_n, all_r, v, starts, key_starts, factor, out, work)
        for row in range(R):
            part, m = slice(at[row], at[row + 1]), len(past[row])
            if not counts[row]:
                continue
            cs, rs = torch.stack([x[0] for x in past[row]]), torch.stack([x[1] for x in past[row]])
            seen = m - counts[row] + 1 + torch.arange(counts[row], device="cuda")
            want, off = attention(torch.cat((q_c[part], q2[part]), -1), torch.cat((cs, rs), -1)[:, None], cs[:, None], seen, factor)
            assert ((out_c[part].double() - want).abs() <= off).all()
            keys = slice(int(key_starts[row]), int(key_starts[row + 1]))
            want, off = attention(torch.cat((q_n[part], q2[part]), -1), torch.cat((k_n[keys], all_r[keys][:, None].expand(-1, H, -1)), -1), v[keys], seen, factor)
            assert ((out[part].double() - want).abs() <= off).all()


# ---- values at the ends of the range ------------------------------------------------------------

def one_takes_all(got, want, q, keys, winners, factor):
    """Scores so far apart that all weight lies with one key, or with some whose scores are equal, bit for bit: then its weights are equal too, and 2^a / (n 2^a) leaves but the output's rounding and that of 1 / n.

    q [n, H, A] and keys [m, A] as a kernel sees them, winners [m].  A score in fp32 is off by A * 2^-24 of the sum of its products' magnitudes; behind that 200 in log2 have to be left."""
    s = torch.matmul(q.double(), keys.double().T.contiguous()) * (factor * math.log2(math.e))
    size = torch.matmul(q.double().abs(), keys.double().abs().T.contiguous()).amax() * abs(factor) * math.log2(math.e)
    best = s[..., winners]
    assert (best == best[..., :1]).all()
    assert (best[..., 0] - s[..., ~winners].amax(-1)).min() > 200 + 2 * q.shape[-1] * 2.0 ** -24 * size
    assert ((got.double() - want).abs() <= 2 * HALF * want.abs()).all(), (got.double() - want).abs().max()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("H,n,columns", [(16, 100, 2), (32, 500, 8), (64, 300, 2000), (128, 200, 4), (128, 200, 2000), (16, 6000, 100), (128, 2500, 50)])
@pytest.mark.parametrize("size,factor", [(14, 0.06), (14, -0.08), (19, 0.1), (12, 1.0)])
def test_attend_scores_beyond_2_to_31(bits, C, H, n, columns, size, factor):
    """Numbers of 2^12 to 2^20, and scores of up to 2^48: a key takes all the weight, or two whose scores are the same; the two lie in different parts where keys are cut."""
    g = gen(n + size)
    P = 64
    sign = torch.where(torch.rand(C + E, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    heads = (1.0 + (torch.arange(H, device="cuda") * 37 % 128) / 128.0)[:, None]         # (sums of all these are whole multiples below 2^24: fp32 has them exactly)
    q = (math.copysign(1.0, factor) * 2.0 ** size * heads * sign).to(torch.bfloat16)[None]
    keys = torch.where(torch.rand((n, C + E), generator=g, device="cuda") < 0.5, -1.0, 1.0) * 2.0 ** size
    a, b = n // 7, n - 3
    by = torch.where(torch.arange(C + E, device="cuda") % 2 == 0, 3.0, 1.0)
    keys[a], keys[b] = sign * by * 2.0 ** size, sign * by.roll(1) * 2.0 ** size
    table, N = pages_of(g, [n], P, columns=columns)
    i = torch.arange(n, device="cuda")
    slots = table[0].long()[i // P] * P + i % P
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    wg.latent_append(keys[:, :C].to(torch.bfloat16), keys[:, C:].to(torch.bfloat16), slots.to(torch.int32), None, c_cache, r_cache, scale)
    assert torch.equal(values(c_cache, scale)[slots], keys[:, :C].double())               # (1 and 3 times powers of two have a place in 8 bits)
    work = torch.empty(max(16, wg.latent_attend_workspace(1, 1, H, C, table.shape[1], P)), dtype=torch.uint8, device="cuda")
    out = torch.empty((1, H, C), dtype=torch.bfloat16, device="cuda")
    for seen, winners in ((n, [a, b]), (b, [a])):
        wg.latent_attend(q[..., :C], q[..., C:], c_cache, r_cache, scale, table, ints([seen]), ints([0, 1]), factor, out, work)
        at = torch.zeros(seen, dtype=torch.bool, device="cuda")
        at[winners] = True
        one_takes_all(out, keys[:seen, :C][at].double().mean(0).expand(1, H, C), q, keys[:seen], at, factor)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,n,m", [(2, 1, 100), (4, 150, 300), (8, 40, 4000), (1, 1, 9000)])
@pytest.mark.parametrize("size,factor", [(14, 0.06), (14, -0.08), (19, 0.1), (12, 1.0)])
def test_prompt_scores_beyond_2_to_31(D, H, n, m, size, factor):
    g = gen(m + size)
    sign = torch.where(torch.rand(D + E, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    tokens = (1.0 + (torch.arange(n * H, device="cuda") * 37 % 128) / 128.0).view(n, H, 1)
    q = (math.copysign(1.0, factor) * 2.0 ** size * tokens * sign).to(torch.bfloat16)
    keys = torch.where(torch.rand((m, D + E), generator=g, device="cuda") < 0.5, -1.0, 1.0) * 2.0 ** size
    a, b = m // 7, m - n
    by = torch.where(torch.arange(D + E, device="cuda") % 2 == 0, 3.0, 1.0)
    keys[a], keys[b] = sign * by * 2.0 ** size, sign * by.roll(1) * 2.0 ** size
    v = bf16(g, m, H, D)
    k = keys.to(torch.bfloat16)
    work = torch.empty(max(16, wg.latent_prompt_workspace(n, 1, H, D, m)), dtype=torch.uint8, device="cuda")
    out = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda")
    for winners in ([a, b], [a]):
        if len(winners) == 1:
            k[b] = 0
            keys[b] = 0
        wg.latent_prompt(q[..., :D], q[..., D:], k[:, None, :D].expand(-1, H, -1), k[:, D:], v, ints([0, n]), ints([0, m]), factor, out, work)
        at = torch.zeros(m, dtype=torch.bool, device="cuda")
        at[winners] = True
        one_takes_all(out, v[at].double().mean(0).expand(n, H, D), q, keys, at, factor)       # (every token sees the winners: the second is the first token's own key)


def levels(n, first, last, size):
    """Keys [n] whose scores are 0, and 7.75 in log2 for one behind the first 64 of every 128; values of about 2^size there, and none elsewhere.  (A softmax whose base is the first scores' may not weigh the later ones with 2^7.75.)"""
    i = torch.arange(n, device="cuda")
    late = i % 128 == 100
    v = torch.where(late, 1.0 + (i * 37 % 128) / 128.0, 0.0) * 2.0 ** size
    return torch.where(late, last, first), v


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("H,n,columns", [(16, 120, 2), (32, 120, 2), (64, 120, 2), (128, 250, 4), (64, 250, 2000), (16, 3000, 50), (128, 2500, 50), (32, 4000, 2000)])
@pytest.mark.parametrize("size", [120, -122])
def test_attend_values_near_the_ends_of_the_range(bits, C, H, n, columns, size):
    """2^120 to 2^121: the largest weight times it is beyond 2^128 if a weight may be 2^7.75; up to 32 of them with weights of 1 at the most are not."""
    g = gen(n)
    P = 64
    level, v = levels(n, 0.0, 7.75, size)
    table, N = pages_of(g, [n], P, columns=columns)
    i = torch.arange(n, device="cuda")
    slots = table[0].long()[i // P] * P + i % P
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    c, r = torch.zeros((n, C), device="cuda"), torch.zeros((n, E), device="cuda")
    c[:, ::3], r[:, 5] = v[:, None], level
    wg.latent_append(c.to(torch.bfloat16), r.to(torch.bfloat16), slots.to(torch.int32), None, c_cache, r_cache, scale)
    q_c, q_r = torch.zeros((1, H, C), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, H, E), dtype=torch.bfloat16, device="cuda")
    q_r[..., 5] = 1.0
    out, work = torch.empty_like(q_c), torch.empty(max(16, wg.latent_attend_workspace(1, 1, H, C, table.shape[1], P)), dtype=torch.uint8, device="cuda")
    wg.latent_attend(q_c, q_r, c_cache, r_cache, scale, table, ints([n]), ints([0, 1]), math.log(2.0), out, work)
    held_c, held_r = values(c_cache, scale)[slots], r_cache.view(-1, E)[slots].double()
    want, off = attention(torch.cat((q_c, q_r), -1), torch.cat((held_c, held_r), -1)[:, None], held_c[:, None], torch.tensor([n], device="cuda"), math.log(2.0))
    assert ((out.double() - want).abs() <= off).all(), (out.double() - want).abs().max()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,n,m", [(2, 1, 120), (4, 150, 300), (8, 40, 4000), (1, 1, 4000)])
@pytest.mark.parametrize("size", [120, -122])
def test_prompt_values_near_the_ends_of_the_range(D, H, n, m, size):
    level, of = levels(m, 0.0, 7.75, size)
    q_n, q_r = torch.zeros((n, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, H, E), dtype=torch.bfloat16, device="cuda")
    k_n, k_r = bf16(gen(m), m, H, D), torch.zeros((m, E), dtype=torch.bfloat16, device="cuda")
    q_r[..., 5], k_r[:, 5] = 1.0, level.to(torch.bfloat16)
    v = of[:, None, None].expand(-1, H, D).to(torch.bfloat16)
    out, work = torch.empty_like(q_n), torch.empty(max(16, wg.latent_prompt_workspace(n, 1, H, D, m)), dtype=torch.uint8, device="cuda")
    wg.latent_prompt(q_n, q_r, k_n, k_r, v, ints([0, n]), ints([0, m]), math.log(2.0), out, work)
    k = torch.cat((k_n, k_r[:, None].expand(-1, H, -1)), -1)
    want, off = attention(torch.cat((q_n, q_r), -1), k, v, m - n + 1 + torch.arange(n, device="cuda"), math.log(2.0))
    assert ((out.double() - want).abs() <= off).all(), (out.double() - want).abs().max()


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,n,m", [(2, 100, 200), (8, 40, 4000), (1, 1, 9000), (16, 131, 2500)])
def test_prompt_values_that_are_none_where_weights_vanish(bad, D, H, n, m):
    """A value that is none times a weight of 0 is none, also where keys are cut and all of a part's weights vanish beside those of another."""
    g = gen(m)
    u = torch.where(torch.rand(D, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    q_n, q_r = u.to(torch.bfloat16).expand(n, H, D).contiguous(), bf16(g, n, H, E)
    k_n, k_r, v = torch.zeros((m, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((m, E), dtype=torch.bfloat16, device="cuda"), bf16(g, m, H, D)
    k_n[m // 2:] = (u * 4.0).to(torch.bfloat16)                # scores of 4 D, which is 369 in log2 and more
    fine = v.clone()
    v[m // 50, :, 7], fine[m // 50, :, 7] = bad, 0.0
    out, work = torch.empty_like(q_n), torch.empty(max(16, wg.latent_prompt_workspace(n, 1, H, D, m)), dtype=torch.uint8, device="cuda")
    wg.latent_prompt(q_n, q_r, k_n, k_r, v, ints([0, n]), ints([0, m]), 1.0, out, work)
    want, off = attention(torch.cat((q_n, q_r), -1), torch.cat((k_n, k_r[:, None].expand(-1, H, -1)), -1), fine, m - n + 1 + torch.arange(n, device="cuda"), 1.0)
    close = (out.double() - want).abs() <= off
    assert not out[..., 7].isfinite().any()
    close[..., 7] = True
    assert close.all()


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("H,n,columns", [(16, 200, 4), (16, 3000, 50), (128, 2500, 50), (32, 30000, 500), (64, 250, 2000)])
def test_attend_numbers_that_are_none_where_weights_vanish(bad, C, H, n, columns):
    """An infinity that makes its key's score -inf, among keys whose scores are far below the others'."""
    g = gen(n)
    P = 64
    table, N = pages_of(g, [n], P, columns=columns)
    i = torch.arange(n, device="cuda")
    slots = table[0].long()[i // P] * P + i % P
    c_cache, r_cache, _ = new_cache(g, N, P, C, 16)
    c, r = bf16(g, n, C), torch.zeros((n, E), dtype=torch.bfloat16, device="cuda")
    c[:, 5], r[n // 2:] = 0.0, 8.0
    c[n // 50, 5] = bad
    wg.latent_append(c, r, slots.to(torch.int32), None, c_cache, r_cache, None)
    q_c, q_r = torch.zeros((1, H, C), dtype=torch.bfloat16, device="cuda"), torch.ones((1, H, E), dtype=torch.bfloat16, device="cuda")
    q_c[..., 5] = 1.0 if bad < 0 else -1.0
    out, work = torch.empty_like(q_c), torch.empty(max(16, wg.latent_attend_workspace(1, 1, H, C, table.shape[1], P)), dtype=torch.uint8, device="cuda")
    wg.latent_attend(q_c, q_r, c_cache, r_cache, None, table, ints([n]), ints([0, 1]), 1.0, out, work)
    assert not out[..., 5].isfinite().any()
    c[n // 50, 5] = 0.0
    others = torch.arange(n, device="cuda") != n // 50
    want, off = attention(torch.cat((q_c, q_r), -1), torch.cat((c, r), -1)[:, None][others], c[:, None][others], torch.tensor([n - 1], device="cuda"), 1.0)
    close = (out.double() - want).abs() <= off
    close[..., 5] = True
    assert (close | out.isnan()).all()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("C", [256, 512])
@pytest.mark.parametrize("T", [1023, 1024, 1025, 16384, 16385, 16391])
def test_append_many(bits, C, T):
    """On both sides of where workgroups take more tokens, wavefronts and workgroups that are not full; slots that are none inside a wavefront's tokens, and several tokens of a workgroup whose pages have begun in others."""
    g = gen(T + C)
    P, forks = 32, 60
    N = 2 * (T // P + 1) + forks + 3
    c_cache, r_cache, scale = new_cache(g, N, P, C, bits)
    both = (torch.randn((T, C + E), generator=g, device="cuda") * torch.exp2(20 * torch.rand((T, 1), generator=g, device="cuda") - 10)).to(torch.bfloat16)
    c, r = both[:, :C], both[:, C:]
    pages = torch.randperm(N, generator=g, device="cuda")
    origin_pages, fork_pages, other = pages[:2], pages[2:2 + forks], pages[2 + forks:]
    slots = (other[:T // P + 1, None] * P + torch.arange(P, device="cuda")).view(-1)[torch.randperm(T // P * P + P, generator=g, device="cuda")[:T]]
    origins = torch.full((T,), -1, device="cuda")
    # tokens that take a begun page along: some behind one another, the call's last ones, and some with a slot or an origin that is none
    at = torch.cat((torch.arange(5, 12), torch.arange(0, 40 * 13, 13) + 100, torch.arange(T - 13, T))).to("cuda")
    assert at.numel() == forks and at.unique().numel() == forks
    places = torch.arange(forks, device="cuda") * 7 % P
    slots[at], origins[at] = fork_pages * P + places, origin_pages[torch.arange(forks, device="cuda") % 2]
    origins[at[::9]] = N
    none = torch.tensor([0, 2, 7, 17, 33, 34, 35, 37, 113, T - 2], device="cuda")
    slots[none] = torch.tensor([-1, N * P, -2 ** 31, 2 ** 31 - 1, -1, -1, -1, N * P + 5, -3, N * P], device="cuda")
    v, s = held(c)
    caches = [c_cache.view(torch.uint8) if bits == 8 else c_cache, r_cache] + ([scale] if bits == 8 else [])
    new = [v.float().to(torch.float8_e4m3fn).view(torch.uint8) if bits == 8 else c, r, s.float()]
    want = [x.clone() for x in caches]
    ok = (slots >= 0) & (slots < N * P)
    for w, x in zip(want, new):
        for t in at.tolist():
            if ok[t] and 0 <= origins[t] < N:
                page, o = divmod(int(slots[t]), P)
                w[page, :o] = w[int(origins[t]), :o].clone()
        w.view(-1, *w.shape[2:])[slots[ok]] = x[ok]
    wg.latent_append(c, r, slots.to(torch.int32), origins.to(torch.int32), c_cache, r_cache, scale)
    for w, x in zip(want, caches):
        assert same(x, w)
