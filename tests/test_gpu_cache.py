"""The 8-bit cache: what is appended bit by bit, and attention over it, against the definitions in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _wg():
    import torch
    import paper_2507_16768_amd as wg
    assert torch.cuda.is_available(), "this test needs the GPU"
    return torch, wg


def numbers_of_bytes():
    """The 256 numbers of the format, by its definition."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = np.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = -x if b & 128 else x
    return out


NUMBERS = numbers_of_bytes()


def to_bytes(x):
    """Nearest byte of float64 numbers, ties to the even mantissa, beyond 448 the largest; NaN is 0x7F."""
    grid = NUMBERS[:127]
    a = np.minimum(np.abs(x), 448.0)
    nan = np.isnan(x)
    a = np.where(nan, 0.0, a)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    b = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    b = np.where(grid[hi] == a, hi, b)
    return np.where(nan, 0x7F, b | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(top):
    """The least power of two from 2^-64 on times which 448 reaches top."""
    s = 2.0 ** -64
    while 448.0 * s < top:
        s *= 2
    return s


def same_bytes(a, b):
    """NaNs of either sign are one."""
    return (a == b) | (((a & 127) == 127) & ((b & 127) == 127))


class Cache:
    def __init__(self, N, H, P, D, seed=0):
        rng = np.random.default_rng(seed)
        self.N, self.H, self.P, self.D = N, H, P, D
        self.k = rng.integers(0, 127, (N, H, P, D)).astype(np.uint8)          # what pages held before: any numbers
        self.v = rng.integers(0, 127, (N, H, D, P)).astype(np.uint8)
        self.ks = 2.0 ** rng.integers(-6, 3, (N, H)).astype(np.float32)
        self.vs = 2.0 ** rng.integers(-6, 3, (N, H)).astype(np.float32)

    def device(self, torch):
        f8 = lambda x: torch.from_numpy(x.copy()).cuda().view(torch.float8_e4m3fn)
        return f8(self.k), f8(self.v), torch.from_numpy(self.ks.copy()).cuda(), torch.from_numpy(self.vs.copy()).cuda()

    def append(self, k, v, slots, origins):
        """In 64 bits, token run by token run; k and v float64 [T, H, D]."""
        P, t, T = self.P, 0, len(slots)
        before = [x.copy() for x in (self.k, self.v, self.ks, self.vs)]
        while t < T:
            page, o = divmod(int(slots[t]), P)
            if not 0 <= slots[t] < self.N * P:
                t += 1
                continue
            n = 1
            while t + n < T and slots[t + n] == slots[t] + n and o + n < P:
                n += 1
            src = page if origins is None or not 0 <= origins[t] < self.N else int(origins[t])
            for h in range(self.H):
                for x, cache, scale, old, old_scale in ((k, self.k, self.ks, before[0], before[2]), (v, self.v, self.vs, before[1], before[3])):
                    part = x[t:t + n, h]
                    fine = np.abs(part[np.isfinite(part)])
                    s = scale_of(fine.max() if fine.size else 0.0)
                    if o:
                        s = max(s, float(old_scale[src, h]))
                        early = old[src, h, :o] if cache is self.k else old[src, h, :, :o].T
                        early = to_bytes(NUMBERS[early] * float(old_scale[src, h]) / s)
                        if cache is self.k:
                            cache[page, h, :o] = early
                        else:
                            cache[page, h, :, :o] = early.T
                    b = to_bytes(part / s)
                    if cache is self.k:
                        cache[page, h, o:o + n] = b
                    else:
                        cache[page, h, :, o:o + n] = b.T
                    scale[page, h] = s
            t += n

    def check(self, k, v, ks, vs):
        import torch
        assert (ks.cpu().numpy() == self.ks).all() and (vs.cpu().numpy() == self.vs).all()
        for got, want in ((k, self.k), (v, self.v)):
            got = got.view(torch.uint8).cpu().numpy()
            assert same_bytes(got, want).all(), np.argwhere(~same_bytes(got, want))[:4].tolist()


def bf16(torch, x):
    t = torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)
    return t, t.double().numpy()


def rows_of(rng, pages, lens, news, P):
    """Slots of rows that lie in pages of their own: their lens[r] earlier tokens are there."""
    slots = []
    for a, b in zip(lens, news):
        mine = [pages.pop() for _ in range(-(-(a + b) // P))]
        slots += [mine[p // P] * P + p % P for p in range(a, a + b)]
    return np.array(slots, np.int32)


@pytest.mark.parametrize("H,P,D", [(1, 16, 64), (3, 16, 128), (8, 32, 128), (2, 64, 256), (5, 64, 64), (4, 32, 256)])
@pytest.mark.parametrize("kind", ["one", "few", "long"])
def test_append(H, P, D, kind):
    torch, wg = _wg()
    rng = np.random.default_rng(H * P + D)
    R = 6
    lens = rng.integers(0, 3 * P, R)
    lens[:2] = [0, P - 1]
    news = {"one": np.ones(R, int), "few": rng.integers(1, 7, R), "long": rng.integers(1, 4 * P, R)}[kind]
    N = int(sum(-(-(a + b) // P) for a, b in zip(lens, news))) + 3
    slots = rows_of(rng, list(rng.permutation(N)), lens, news, P)
    T = len(slots)
    cache = Cache(N, H, P, D, seed=1)
    # side by side, as one projection leaves them, and of magnitudes that grow and shrink a page's scale
    kv = rng.standard_normal((T, 2, H, D)) * 2.0 ** rng.integers(-9, 9, (T, 2, H, 1))
    t, x = bf16(torch, kv)
    dev = t.cuda()
    on = cache.device(torch)
    d_slots = torch.from_numpy(slots).cuda()
    for _ in range(2):                                   # a second time changes nothing
        wg.cache_append(dev[:, 0], dev[:, 1], d_slots, None, *on)
    cache.append(x[:, 0], x[:, 1], slots, None)
    cache.check(*on)


@pytest.mark.parametrize("P,D", [(16, 128), (32, 64), (64, 256)])
def test_tokens_in_front_of_a_fork_come_with_it(P, D):
    torch, wg = _wg()
    rng = np.random.default_rng(P)
    H, o, N = 3, P // 2 + 3, 9
    cache = Cache(N, H, P, D, seed=2)
    slots = np.array([2 * P + o, 4 * P + o, 5 * P, 7 * P + o, 8 * P + o], np.int32)
    origins = np.array([0, 0, -1, -1, 1], np.int32)
    x = rng.standard_normal((5, 2, H, D)) * 4.0
    x[1] *= 2.0 ** 12                                   # this one's scale grows, that one's stays
    x[4] = 0
    t, x = bf16(torch, x)
    on = cache.device(torch)
    wg.cache_append(t.cuda()[:, 0], t.cuda()[:, 1], torch.from_numpy(slots).cuda(), torch.from_numpy(origins).cuda(), *on)
    cache.append(x[:, 0], x[:, 1], slots, origins)
    cache.check(*on)


def test_numbers_of_all_sizes():
    """Every byte's number, what lies between two, zeros, infinities, NaN, and pages of zeros alone; slots that are none."""
    torch, wg = _wg()
    H, P, D, N = 1, 16, 128, 12
    cache = Cache(N, H, P, D, seed=3)
    x = np.zeros((11, 1, D))
    grid = NUMBERS[:127]
    x[0, 0] = np.concatenate([grid, [448.0]])
    x[1, 0] = np.concatenate([-grid, [448.0]])
    x[2, 0, :126] = (grid[1:] + grid[:-1]) / 2
    x[2, 0, 126:] = [449.0, 464.0]                       # above 448: the next scale
    x[3, 0, :4] = [np.inf, -np.inf, np.nan, 1.0]
    x[4, 0] = np.inf
    x[5, 0] = np.nan
    x[6, 0] = 0.0
    x[7, 0, :3] = [1e-30, -2e-38, 3e-39]                 # below the least scale
    x[8, 0, :2] = [3.0e38, 1.0]
    x[9, 0, :] = 5.0
    x[10, 0, :] = 7.0
    t, x = bf16(torch, x)
    slots = np.array([0, 1 * P, 2 * P + 3, 3 * P, 4 * P, 5 * P, 6 * P, 7 * P, 8 * P, -1, N * P], np.int32)
    on = cache.device(torch)
    dev = t.cuda()
    wg.cache_append(dev, dev, torch.from_numpy(slots).cuda(), None, *on)
    cache.append(x, x, slots, None)
    cache.check(*on)


# ---- attention --------------------------------------------------------------------------------

def attention(cache, q, table, lens, starts, scale):
    """float64; returns the output and, for the bound, the weighted sum of the values' magnitudes."""
    T, Q, D = q.shape
    H, P = cache.H, cache.P
    out, size = np.zeros((T, Q, D)), np.zeros((T, Q, D))
    for r, L in enumerate(lens):
        n = starts[r + 1] - starts[r]
        pages = [min(int(p), cache.N - 1) if p >= 0 else 0 for p in table[r][:-(-L // P)]]
        for h in range(H):
            if not pages:
                continue
            k = np.concatenate([NUMBERS[cache.k[p, h]] * cache.ks[p, h] for p in pages])[:L]
            v = np.concatenate([NUMBERS[cache.v[p, h]].T * cache.vs[p, h] for p in pages])[:L]
            for i in range(n):
                sees = L - n + i + 1
                if sees <= 0:
                    continue
                for j in range(h * (Q // H), (h + 1) * (Q // H)):
                    w = k[:sees] @ q[starts[r] + i, j] * scale
                    w = np.exp(w - w.max())
                    w /= w.sum()
                    out[starts[r] + i, j] = w @ v[:sees]
                    size[starts[r] + i, j] = w @ np.abs(v[:sees])
    return out, size


# Products of the cache's numbers are exact in fp32.  A weight is rounded to float16 (2^-11 of itself at the most), the output to bfloat16 (2^-8 of
# itself: half a unit of its 8 bits).  Scores are sums of up to 256 products in fp32, off by 256 * 2^-24 of some tens, which moves a weight by 2^-11; sums
# of L weighted values add up to L * 2^-24 of the sum of their magnitudes, exp 2^-22.  With |out| <= the weighted sum of magnitudes that is below
# 2^-8 of that sum and 2^-9 of the output together.
def check_attention(got, want, size):
    off = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
    most = 2.0 ** -8 * size + 2.0 ** -9 * np.abs(want) + 1e-30
    assert np.isfinite(off).all() and (off <= most).all(), (float((off / most).max()), np.argwhere(~(off <= most))[:4].tolist())


def case(seed, P, H, G, D, lens, news, extra=0):
    rng = np.random.default_rng(seed)
    R = len(lens)
    M = max(1, max(-(-a // P) for a in lens)) + extra
    N = sum(-(-a // P) for a in lens) + 2
    cache = Cache(N, H, P, D, seed)
    cache.k = to_bytes(rng.standard_normal((N, H, P, D)) * 30)
    cache.v = to_bytes(rng.standard_normal((N, H, D, P)) * 30)
    cache.ks[:] = 2.0 ** rng.integers(-7, -3, (N, H))
    cache.vs[:] = 2.0 ** rng.integers(-7, 2, (N, H))
    pages = list(rng.permutation(N))
    # behind a row's pages anything: numbers of no page among them
    table = rng.choice([-1, N, 2 ** 31 - 1, 0, -2 ** 31], (R, M)).astype(np.int32)
    for r, a in enumerate(lens):
        for j in range(-(-a // P)):
            table[r, j] = pages.pop()
        if a % P:                                        # behind its tokens anything: NaNs too
            cache.k[table[r, a // P], :, a % P:] = 0x7F
            cache.v[table[r, a // P], :, :, a % P:] = 0xFF
    for p in pages:                                      # and in pages that belong to no row
        cache.k[p], cache.v[p], cache.ks[p], cache.vs[p] = 0x7F, 0x7F, np.nan, np.nan
    starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    q = rng.standard_normal((starts[-1], H * G, D))
    return cache, table, np.asarray(lens, np.int32), starts, q


def run(torch, wg, cache, table, lens, starts, q, scale, out=None, strided=False):
    on = cache.device(torch)
    t, x = bf16(torch, q)
    t = t.cuda()
    if strided:                                          # among other things, as a projection leaves them
        wide = torch.randn((t.shape[0] + 1, t.shape[1] + 3, t.shape[2] * 2), device="cuda").to(torch.bfloat16)
        wide[1:, 2:-1, 8:8 + t.shape[2]] = t
        t = wide[1:, 2:-1, 8:8 + t.shape[2]]
    if out is None:
        out = torch.full(q.shape, 77.0, device="cuda", dtype=torch.bfloat16)
    d = lambda a: torch.from_numpy(a).cuda()
    need = wg.cache_attend_workspace(q.shape[0], len(lens), q.shape[1], cache.H, cache.D, table.shape[1], cache.P)
    work = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if need else None
    wg.cache_attend(t, *on, d(table), d(lens), d(starts), scale, out, work)
    return out, x


@pytest.mark.parametrize("P,H,G,D", [(16, 1, 1, 64), (16, 2, 4, 128), (32, 4, 7, 128), (64, 2, 16, 64), (16, 1, 20, 128), (32, 2, 3, 256), (64, 8, 1, 128)])
def test_a_token_for_each_row(P, H, G, D):
    torch, wg = _wg()
    lens = [1, 2, 63, 64, 65, 1000, 17, P, P + 1, 3 * P - 1, 0, 300, 2049]
    cache, table, lens, starts, q = case(1, P, H, G, D, lens, [1] * len(lens), extra=3)
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))
    assert float(out[10].abs().max()) == 0.0             # the row without a key


@pytest.mark.parametrize("P,H,G,D", [(16, 1, 1, 64), (16, 2, 4, 128), (32, 1, 7, 128), (64, 2, 2, 256), (16, 1, 24, 64)])
def test_several_tokens_of_a_row(P, H, G, D):
    """Prompts and parts of them, rows without tokens, and more tokens than keys: the first ones see nothing."""
    torch, wg = _wg()
    lens, news = [70, 33, 0, 5, 200, 64, 129, 3, 1, 90], [70, 5, 0, 5, 100, 1, 17, 6, 0, 64]
    cache, table, lens, starts, q = case(2, P, H, G, D, lens, news)
    out, x = run(torch, wg, cache, table, lens, starts, q, 0.125, strided=True)
    check_attention(out, *attention(cache, x, table, lens, starts, 0.125))
    first = starts[7]
    assert float(out[first:first + 3].abs().max()) == 0.0 and float(out[first + 3].abs().max()) > 0.0


@pytest.mark.parametrize("L", [5000, 40000])
def test_a_long_row(L):
    torch, wg = _wg()
    cache, table, lens, starts, q = case(3, 16, 2, 4, 128, [L, 40], [1, 2])
    out, x = run(torch, wg, cache, table, lens, starts, q, 128 ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, 128 ** -0.5))


@pytest.mark.parametrize("G,n", [(12, 5), (6, 10), (20, 3), (7, 9)])
def test_tokens_that_lie_in_two_tiles_of_a_row_in_shares(G, n):
    """A token's query heads may be split between two tiles, whose last tokens do not see the same blocks of keys."""
    torch, wg = _wg()
    lens = [64 * b + e for b in (16, 32, 48) for e in range(1, 9)]
    cache, table, lens, starts, q = case(6, 16, 1, G, 64, lens, [n] * len(lens))
    assert wg.cache_attend_workspace(q.shape[0], len(lens), G, 1, 64, table.shape[1], 16) > 0
    out, x = run(torch, wg, cache, table, lens, starts, q, 0.125)
    check_attention(out, *attention(cache, x, table, lens, starts, 0.125))


@pytest.mark.parametrize("lens,news", [([3000, 700], [1, 2]), ([60, 20], [3, 1]), ([400, 300], [200, 100])], ids=["shares", "one share", "prompts"])
def test_outputs_of_tokens_behind_the_rows_stay(lens, news):
    torch, wg = _wg()
    cache, table, lens, starts, q = case(7, 16, 2, 4, 128, lens, news)
    more = np.concatenate([q, np.full((5,) + q.shape[1:], np.nan)])
    out, _ = run(torch, wg, cache, table, lens, starts, more, 0.1)
    alone, x = run(torch, wg, cache, table, lens, starts, q, 0.1)
    check_attention(out[:len(q)], *attention(cache, x, table, lens, starts, 0.1))
    assert (out[len(q):] == 77.0).all()


@pytest.mark.parametrize("n,P,H,G,D", [(130, 32, 2, 4, 128), (700, 32, 2, 4, 128), (333, 16, 1, 7, 64), (150, 64, 3, 5, 256), (65, 16, 8, 1, 128), (260, 64, 1, 16, 64)])
def test_a_long_prompt(n, P, H, G, D):
    torch, wg = _wg()
    cache, table, lens, starts, q = case(4, P, H, G, D, [n + 77, 20, n], [n, 3, n // 2])
    # query rows of all sizes, and numbers of a row that are far below its largest
    q *= 2.0 ** np.random.default_rng(1).integers(-3, 2, q.shape[:2] + (1,))
    q[::3] *= 2.0 ** np.random.default_rng(2).integers(-24, 1, q[::3].shape)
    q[5] = 0.0
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5, strided=G == 5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


@pytest.mark.parametrize("H,G,D,n", [(2, 2, 64, 1), (1, 16, 128, 2), (1, 3, 256, 1)])
def test_more_rows_than_have_their_keys_cut(H, G, D, n):
    torch, wg = _wg()
    rng = np.random.default_rng(D)
    lens = rng.integers(n, 90, 1100).tolist()
    cache, table, lens, starts, q = case(10, 16, H, G, D, lens, [n] * len(lens))
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


@pytest.mark.parametrize("P,H,G,D", [(16, 64, 2, 64), (32, 64, 2, 128), (64, 32, 2, 256)])
def test_prompts_that_fill_the_chip(P, H, G, D):
    """Enough of them for no row's keys to be cut."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(8, P, H, G, D, [270, 100], [260, 33])
    assert wg.cache_attend_workspace(q.shape[0], 2, H * G, H, D, table.shape[1], P) == 0
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


@pytest.mark.parametrize("P,H,G,D", [(16, 2, 4, 64), (32, 1, 12, 128), (64, 1, 5, 256)])
def test_prompts_behind_long_rows(P, H, G, D):
    """Few query rows and many keys: the rows' keys are cut, one row's into more shares than another's."""
    torch, wg = _wg()
    lens, news = [5000, 1090, 70, 0, 3], [61, 66, 50, 0, 1]
    cache, table, lens, starts, q = case(9, P, H, G, D, lens, news)
    assert wg.cache_attend_workspace(q.shape[0], len(lens), H * G, H, D, table.shape[1], P) > 0
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


@pytest.mark.parametrize("D,size", [(128, 1e30), (128, 1e-30), (256, 1e36), (64, 1e-37)])
def test_queries_at_the_ends_of_the_range(D, size):
    """What the scale brings back to the middle of it."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(9, 16, 1, 4, D, [90, 70], [90, 40])
    out, x = run(torch, wg, cache, table, lens, starts, q * size, 0.1 / size)
    check_attention(out, *attention(cache, x, table, lens, starts, 0.1 / size))


def test_scores_that_rise_and_fall_along_a_prompt():
    """The first keys far below the later ones, and far above; in tiles that see few of either."""
    torch, wg = _wg()
    D, n = 128, 400
    for sign in (1, -1):
        cache, table, lens, starts, q = case(10, 16, 1, 2, D, [n, n], [n, n])
        for r in range(2):
            for i in range(n):
                p, o = table[r, i // 16], i % 16
                cache.k[p, 0, o] = to_bytes(np.full(D, sign * (i / 8.0 if r else (i // 64) * 40.0 % 130)))
                cache.ks[p, 0] = 1.0
        q[:] = 0.0
        q[:, :, 3] = 1.0
        q[::2, 1, 3] = 0.01
        out, x = run(torch, wg, cache, table, lens, starts, q, 1.0)
        check_attention(out, *attention(cache, x, table, lens, starts, 1.0))


def test_scores_that_are_far_apart_or_equal():
    """One key far above the others, all equal, and scores that grow from block to block."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(5, 16, 1, 4, 64, [300, 300, 300, 300], [1, 1, 1, 5])
    def key(r, i, x):
        p, o = table[r, i // 16], i % 16
        cache.k[p, 0, o], cache.ks[p, 0] = to_bytes(np.full(64, x)), 1.0
    for i in range(300):
        key(0, i, 0.0 if i != 170 else 300.0)
        key(1, i, 2.0)
        key(2, i, i // 4 * 1.0)
        key(3, i, -i // 4 * 1.0)
    q[:] = 1.0
    out, x = run(torch, wg, cache, table, lens, starts, q, 1.0)
    check_attention(out, *attention(cache, x, table, lens, starts, 1.0))


def test_slots_that_pass_32_bits_of_bytes():
    """A cache of more than 4 GiB: its last pages are written and read."""
    torch, wg = _wg()
    H, P, D = 8, 64, 256
    N = (1 << 32) // (H * P * D) + 40
    k = torch.zeros((N, H, P, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros((N, H, D, P), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks, vs = (torch.ones((N, H), device="cuda") for _ in range(2))
    kv = torch.randn((100, 2, H, D), device="cuda").to(torch.bfloat16)
    pages = [N - 1, N - 3]
    slots = torch.tensor([pages[p // P] * P + p % P for p in range(100)], dtype=torch.int32, device="cuda")
    wg.cache_append(kv[:, 0], kv[:, 1], slots, None, k, v, ks, vs)
    small = [t[[N - 1, N - 3]].clone() for t in (k.view(torch.uint8), v.view(torch.uint8))]
    c = Cache(2, H, P, D)
    c.k, c.v, c.ks, c.vs = small[0].cpu().numpy(), small[1].cpu().numpy(), ks[pages].cpu().numpy(), vs[pages].cpu().numpy()
    want = Cache(2, H, P, D)
    want.k[:], want.v[:], want.ks[:], want.vs[:] = 0, 0, 1, 1
    x = kv.double().cpu().numpy()
    want.append(x[:, 0], x[:, 1], np.arange(100), None)
    assert same_bytes(c.k, want.k).all() and same_bytes(c.v, want.v).all() and (c.ks == want.ks).all() and (c.vs == want.vs).all()
    q = torch.randn((1, 8, D), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    work = torch.empty(max(16, wg.cache_attend_workspace(1, 1, 8, H, D, 2, P)), dtype=torch.uint8, device="cuda")
    wg.cache_attend(q, k, v, ks, vs, i32([pages]), i32([100]), i32([0, 1]), 0.0625, out, work)
    check_attention(out, *attention(c, q.double().cpu().numpy(), np.array([[0, 1]]), [100], [0, 1], 0.0625))


def test_same_bits_every_time_and_in_a_graph():
    torch, wg = _wg()
    cache, table, lens, starts, q = case(6, 16, 2, 4, 128, [3000, 100, 900], [1, 1, 1])
    on = cache.device(torch)
    t, _ = bf16(torch, q)
    t = t.cuda()
    d = lambda a: torch.from_numpy(a).cuda()
    dt, dl, ds = d(table), d(lens), d(starts)
    out = torch.empty_like(t)
    work = torch.empty(max(16, wg.cache_attend_workspace(3, 3, 8, 2, 128, table.shape[1], 16)), dtype=torch.uint8, device="cuda")
    kv = torch.randn((3, 2, 2, 128), device="cuda").to(torch.bfloat16)
    slots = torch.tensor([int(table[r, (lens[r] - 1) // 16]) * 16 + (lens[r] - 1) % 16 for r in range(3)], dtype=torch.int32, device="cuda")

    def step():
        wg.cache_append(kv[:, 0], kv[:, 1], slots, None, *on)
        wg.cache_attend(t, *on, dt, dl, ds, 0.1, out, work)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for i in range(4):
        t.copy_(torch.randn(t.shape, device="cuda") * (1 + i))
        kv.copy_(torch.randn(kv.shape, device="cuda"))
        step()
        want = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and float(want.float().abs().sum()) > 0


def test_what_a_token_does_not_see_is_nothing_to_it():
    """A NaN or an infinity in a key or value reaches the tokens from its own on, and no other."""
    torch, wg = _wg()
    for D, P, n, G in ((64, 16, 40, 4), (128, 32, 40, 4), (256, 64, 40, 4), (64, 64, 19, 1), (128, 16, 19, 2), (256, 32, 19, 2)):
        L = 70
        cache, table, lens, starts, q = case(7, P, 1, G, D, [L, L, L], [n, n, n])
        at = L - n + 17                                  # the 18th token's own key
        page, o = table[0, at // P], at % P
        cache.k[page, 0, o, 5] = 0x7F
        page, o = table[1, at // P], at % P
        cache.v[page, 0, 7, o] = 0xFF
        out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
        got = torch.isnan(out).cpu().numpy()
        assert not got[:17].any() and got[17:n].all()
        assert not got[n:n + 17].any() and got[n + 17:2 * n, :, 7].all() and got[n + 17:2 * n].sum() == (n - 17) * G
        assert not got[2 * n:].any()
        clean = np.ones(out.shape, bool)
        clean[17:n] = False
        clean[n + 17:2 * n, :, 7] = False
        with np.errstate(all="ignore"):
            cache.v[table[1, at // P], 0, 7, at % P] = 0     # (for what is clean the definition without it)
            cache.k[table[0, at // P], 0, at % P, 5] = 0
            want, size = attention(cache, x, table, lens, starts, D ** -0.5)
        off = np.abs(np.where(clean, out.double().cpu().numpy() - want, 0.0))
        assert (off <= 2.0 ** -8 * size + 2.0 ** -9 * np.abs(want) + 1e-30).all()


def test_weights_that_are_small_beside_the_largest():
    """A key of weight 1 and very many of weight 2^-14 to 2^-24 each, which together count; pages whose values' scales differ by 2^40, and one of zeros."""
    torch, wg = _wg()
    L, D, P = 20000, 64, 16
    for least in (14, 24):
        cache, table, lens, starts, q = case(8, P, 1, 1, D, [L], [1])
        cache.k[:], cache.ks[:], cache.v[:] = to_bytes(np.zeros(1)), 1.0, to_bytes(np.full(1, 1.0))
        q[:] = 0.0
        q[0, 0, 0] = 1.0
        page = table[0, 100]
        cache.k[page, 0, 3, 0] = to_bytes(np.full(1, float(least)))[0]
        cache.v[page] = to_bytes(np.full(1, -0.5))
        cache.vs[:] = 2.0 ** -20
        cache.vs[table[0, ::2]] = 2.0 ** 20
        cache.v[table[0, 1]], cache.vs[table[0, 1]] = 0, 0.0
        scale = float(np.log(2.0))
        out, x = run(torch, wg, cache, table, lens, starts, q, scale)
        check_attention(out, *attention(cache, x, table, lens, starts, scale))


# ---- pages whose values differ in scale ---------------------------------------------------------
# A weight is held as float16 and with it the scale of its page's values, the largest of a query at 2^8 or more: what is below 2^-25 is lost from the products, and with
# n keys of at most 448 that is n * 448 * 2^-25 beside 2^8 times the largest key's own value: below 2^-15 of the sum of magnitudes for the thousands of keys here, whose
# values are 2^4 on average.  The sum of the weights is fp32 and loses nothing.  The bounds above hold as they are.
SMALL = {"zeros": (2.0 ** -64, True), "zeros without a scale": (0.0, True), "far below": (2.0 ** -40, False), "below": (2.0 ** -30, False)}


def small_pages(cache, table, r, which, kind, times=1.0):
    """Some of row r's pages have values of zero, or of a scale far below the others'."""
    scale, zeros = SMALL[kind]
    for j in which:
        p = table[r, j]
        if zeros:
            cache.v[p] = 0
        cache.vs[p] = scale * times


def places(n, where):
    """The first pages, the last ones, every other one, all but one."""
    return {"first": range(n // 2), "last": range(n // 2, n), "every other": range(1, n, 2), "all but one": [j for j in range(n) if j != 1]}[where]


@pytest.mark.parametrize("where", ["first", "last", "every other", "all but one"])
@pytest.mark.parametrize("kind", list(SMALL))
@pytest.mark.parametrize("P,H,G,D", [(16, 1, 4, 64), (32, 2, 2, 128), (64, 1, 4, 256), (16, 1, 4, 128)])
def test_prompts_over_pages_of_small_values(P, H, G, D, kind, where):
    torch, wg = _wg()
    lens, news = [300, 200, 130], [190, 70, 130]
    cache, table, lens, starts, q = case(11, P, H, G, D, lens, news)
    cache.vs[cache.vs > 0] = 2.0 ** -4
    for r, L in enumerate(lens):
        small_pages(cache, table, r, places(-(-int(L) // P), where), kind)
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


@pytest.mark.parametrize("where", ["last", "all but one"])
@pytest.mark.parametrize("P,H,G,D", [(16, 2, 4, 64), (32, 1, 12, 128), (64, 1, 5, 256)])
def test_prompts_behind_long_rows_of_small_values(P, H, G, D, where):
    """The same where a row's keys are cut: shares of zeros alone are among them."""
    torch, wg = _wg()
    lens, news = [5000, 1090, 70], [61, 66, 50]
    cache, table, lens, starts, q = case(12, P, H, G, D, lens, news)
    assert wg.cache_attend_workspace(q.shape[0], len(lens), H * G, H, D, table.shape[1], P) > 0
    for r, L in enumerate(lens):
        small_pages(cache, table, r, places(-(-int(L) // P), where), "zeros")
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


def test_a_prompt_and_single_tokens_agree():
    """The last token of a prompt over pages of zeros, by itself and among the prompt's."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(13, 16, 1, 4, 128, [160], [160])
    small_pages(cache, table, 0, range(4, 10), "zeros")
    whole, x = run(torch, wg, cache, table, lens, starts, q, 0.1)
    alone, _ = run(torch, wg, cache, table, lens, np.array([0, 1], np.int32), q[-1:], 0.1)
    want, size = attention(cache, x, table, lens, starts, 0.1)
    check_attention(whole, want, size)
    check_attention(alone, want[-1:], size[-1:])


@pytest.mark.parametrize("where", ["first", "last", "every other", "all but one"])
@pytest.mark.parametrize("P,H,G,D,lens,news", [(16, 1, 4, 64, [300, 200], [1, 2]), (32, 2, 7, 128, [5000, 300], [1, 1]), (64, 1, 3, 256, [300, 700], [1, 1]),
                                               (16, 1, 4, 64, [300, 200], [100, 90]), (32, 1, 12, 128, [5000, 70], [61, 50]), (64, 1, 5, 256, [200, 100], [100, 20])])
def test_pages_of_zeros_beside_very_large_values(P, H, G, D, lens, news, where):
    """What float32 holds of a scale: 2^90 beside the least one."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(14, P, H, G, D, lens, news)
    cache.vs[cache.vs > 0] = 2.0 ** 90
    for r, L in enumerate(lens):
        small_pages(cache, table, r, places(-(-int(L) // P), where), "zeros")
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    check_attention(out, *attention(cache, x, table, lens, starts, D ** -0.5))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 2, 40])
def test_queries_with_numbers_that_are_none(D, n):
    """An infinity or a NaN in a query makes its output NaN (infinite scores less their infinite maximum are none) and no other; a query that sees nothing has zeros."""
    torch, wg = _wg()
    G, lens = 4, [90, 70, 0, 1500]
    cache, table, lens, starts, q = case(15, 16, 1, G, D, lens, [n] * len(lens))
    cache.k[table[1, 0], 0, :, 5] = to_bytes(np.full(16, -2.0))            # numbers of one sign, of both, zeros
    for j in range(5):
        cache.k[table[1, j], 0, :, 9] = to_bytes(np.full(16, -1.5))
        cache.k[table[0, j], 0, :, 9] = 0
    bad = np.zeros(q.shape[:2], bool)
    for r, L in enumerate(lens):
        t = int(starts[r + 1]) - 1
        q[t, 0, 9], q[t, 1, 9], q[t, 2, 5] = np.inf, -np.inf, np.nan
        bad[t, :3] = L > 0
        if n > 2:
            q[t - 7, 3, D - 1] = np.inf
            bad[t - 7, 3] = L > 0
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    got = torch.isnan(out).cpu().numpy()
    assert (got == bad[:, :, None]).all(), np.argwhere(got != bad[:, :, None])[:4].tolist()
    assert float(out[starts[2]:starts[3]].abs().max()) == 0.0
    want, size = attention(cache, np.where(np.isfinite(x), x, 0.0), table, lens, starts, D ** -0.5)
    keep = ~bad
    check_attention(out[torch.from_numpy(keep).cuda()], want[keep], size[keep])


@pytest.mark.parametrize("G,D,lens,news,cut", [(4, 128, [300, 200, 90], [100, 80, 90], 130), (4, 64, [300, 200, 90], [100, 80, 90], 37), (2, 256, [90, 300], [64, 200], 100),
                                               (4, 128, [300, 200], [5, 4], 7), (3, 64, [2000, 300], [3, 2], 2), (12, 128, [5000, 70], [61, 50], 50)])
def test_fewer_tokens_than_the_rows_take(G, D, lens, news, cut):
    """The first tokens of a step by themselves: the rows' lengths and starts say where they are, and what they see does not change."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(16, 16, 1, G, D, lens, news)
    out, x = run(torch, wg, cache, table, lens, starts, q[:cut], D ** -0.5)
    want, size = attention(cache, bf16(torch, q)[1], table, lens, starts, D ** -0.5)
    check_attention(out, want[:cut], size[:cut])


def sum_of_two(x):
    """A row of bfloat16 numbers as the header says that calls with 32 query rows and more to a row of the table take it: the largest in [128, 256), sums of two
    8-bit numbers, the second 2^-5 of what it is."""
    e = np.floor(np.log2(np.abs(x).max(-1, keepdims=True))) - 7
    y = x / 2.0 ** e
    first = NUMBERS[to_bytes(y)]
    return (first + NUMBERS[to_bytes((y - first) * 32)] / 32) * 2.0 ** e


@pytest.mark.parametrize("D,n", [(128, 8), (256, 16), (128, 7), (64, 8)])
def test_what_queries_are_rounded_to(D, n):
    """One large number of a query meets keys of zeros, and its small ones keys that tell what they are: as they are below the limit and for heads of 64, else in two parts."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(17, 16, 1, 4, D, [40, 40], [n, n])
    cache.k[:, :, :, 0] = 0
    cache.ks[cache.ks > 0] = 2.0 ** 13
    q *= 2.0 ** -16
    q[:, :, 0] = 1.9
    out, x = run(torch, wg, cache, table, lens, starts, q, D ** -0.5)
    parts = sum_of_two(x)
    off = np.abs(parts - x).max()
    assert 2.0 ** -24 < off <= 2.0 ** -22
    taken = parts if D != 64 and n * 4 >= 32 else x
    check_attention(out, *attention(cache, taken, table, lens, starts, D ** -0.5))
    other, size = attention(cache, x if taken is parts else parts, table, lens, starts, D ** -0.5)
    assert (np.abs(out.double().cpu().numpy() - other) > 2 * (2.0 ** -8 * size + 2.0 ** -9 * np.abs(other))).any()


@pytest.mark.parametrize("high,others", [(20.0, 0), (40.0, 0), (80.0, 0), (80.0, 90)])
@pytest.mark.parametrize("D,lens,news", [(64, [300, 200], [1, 2]), (128, [2500, 200], [1, 2]), (64, [300, 200], [200, 90]), (128, [300, 200], [200, 90]), (256, [300, 200], [200, 90]),
                                         (128, [2500, 200], [70, 90])])
def test_pages_of_zeros_with_the_highest_scores(D, lens, news, high, others):
    """What the other pages leave beside them is as small as their terms.  Here the largest weight, of a score e^80 times the others' and the least scale, may be on a page of
    zeros, and the sum of magnitudes says nothing of it: what is below 2^-33 of it is lost, for len keys of at most 448."""
    torch, wg = _wg()
    cache, table, lens, starts, q = case(18, 16, 1, 4, D, lens, news)
    cache.ks[cache.ks > 0] = 1.0
    cache.vs[cache.vs > 0] *= np.float32(2.0 ** others)
    for r, L in enumerate(lens):
        for i in range(int(L)):
            page = table[r, i // 16]
            cache.k[page, 0, i % 16] = to_bytes(np.full(D, high if i // 16 % 3 == 2 else i % 16 / 8.0))
        small_pages(cache, table, r, range(2, -(-int(L) // 16), 3), "zeros")
    q[:] = 0.0
    q[:, :, 3] = 1.0
    q[::2, 1, 3] = -1.0
    out, x = run(torch, wg, cache, table, lens, starts, q, 1.0)
    want, size = attention(cache, x, table, lens, starts, 1.0)
    off = np.abs(out.double().cpu().numpy() - want)
    lost = 2500 * 448 * 2.0 ** -33 * 2.0 ** -64
    assert (off <= 2.0 ** -8 * size + 2.0 ** -9 * np.abs(want) + lost).all(), float((off / (size + lost)).max())
    assert others == 0 or (np.abs(want) > 1e3 * lost).mean() > 0.9
