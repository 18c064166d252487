"""Arguments that the calls of rotary positions and the cache of latent vectors refuse, on the host, before anything is launched, and the frequencies, which are made
there (CPU; no pointer is followed)."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2507_16768_amd as wg

P, Q = C.c_void_p(4096), C.c_void_p(1 << 20)
OFF = C.c_void_p(4104)


def refused(name, good, cases):
    """Each case differs from the good call in what it names, and is refused."""
    L = wg.load_library()
    for case in cases:
        args = dict(good, **case)
        assert getattr(L, name)(*args.values()) == -1, case
        assert L.wg_last_error().startswith(name.encode()), (case, L.wg_last_error())


def test_rotate():
    good = dict(q=P, k=P, dtype=1, tokens=4, q_heads=8, k_heads=2, dim=128, rotated=64, beside=0, q0=1024, q1=128, k0=256, k1=128, positions=P, frequencies=P, magnitude=1.0,
                q_out=Q, qo0=1024, qo1=128, k_out=C.c_void_p(1 << 21), ko0=256, ko1=128, stream=None)
    refused("wg_rotate", good, [
        dict(q=None), dict(k=None), dict(positions=None), dict(frequencies=None), dict(q_out=None), dict(k_out=None), dict(dtype=2), dict(tokens=0), dict(tokens=1 << 31), dict(tokens=1 << 24),
        dict(q_heads=0), dict(q_heads=4097), dict(k_heads=4097), dict(dim=1025), dict(dim=63), dict(rotated=0), dict(rotated=63), dict(rotated=130),
        dict(magnitude=math.nan), dict(magnitude=math.inf), dict(q=C.c_void_p(4097)), dict(q_out=C.c_void_p(4097)), dict(k=C.c_void_p(4097)), dict(frequencies=C.c_void_p(4100)),
        dict(q_out=P, qo0=2048), dict(q_out=P, qo1=64), dict(k_out=P, ko0=512), dict(k_out=Q), dict(dtype=0, q=C.c_void_p(4098))])


def test_latent_append():
    good = dict(c=P, r=P, tokens=4, latent=512, c0=576, r0=576, slots=P, origins=P, c_cache=Q, r_cache=Q, scale=Q, pages=10, page_tokens=16, stream=None)
    refused("wg_latent_append", good, [
        dict(c=None), dict(r=None), dict(slots=None), dict(c_cache=None), dict(r_cache=None), dict(tokens=0), dict(tokens=(1 << 29) + 1), dict(tokens=(1 << 27) + 1), dict(latent=128), dict(latent=576), dict(pages=0),
        dict(page_tokens=24), dict(pages=1 << 27), dict(c=OFF), dict(r=OFF), dict(c0=580), dict(r0=4), dict(c_cache=OFF), dict(r_cache=OFF), dict(scale=C.c_void_p(4098))])


def test_latent_read():
    good = dict(c_cache=P, r_cache=P, scale=P, latent=256, pages=10, page_tokens=32, table=P, rows=3, columns=5, starts=P, tokens=100, c_out=Q, c0=256, r_out=Q, r0=64, stream=None)
    refused("wg_latent_read", good, [
        dict(c_cache=None), dict(r_cache=None), dict(table=None), dict(starts=None), dict(c_out=None), dict(r_out=None), dict(tokens=0), dict(tokens=1 << 31), dict(tokens=(1 << 29) + 1), dict(rows=0), dict(rows=65536),
        dict(columns=0), dict(columns=1 << 26), dict(latent=64), dict(page_tokens=8), dict(pages=0), dict(pages=1 << 26), dict(c_out=OFF), dict(r_out=OFF), dict(c0=250), dict(r0=68),
        dict(c_cache=OFF), dict(r_cache=OFF)])


def test_latent_attend():
    need = wg.latent_attend_workspace(4, 2, 16, 512, 100, 64)
    assert need > 0
    assert wg.latent_attend_workspace(0, 2, 16, 512, 100, 64) == 0 and wg.latent_attend_workspace(4, 2, 16, 512, 100, 60) == 0 and wg.latent_attend_workspace(4, 2, 16, 512, 1, 64) == 0
    good = dict(q_c=P, q_r=P, tokens=4, heads=16, latent=512, c0=8192, c1=512, r0=1024, r1=64, c_cache=P, r_cache=P, scale=P, pages=300, page_tokens=64, table=P, rows=2, columns=100,
                lens=P, starts=P, factor=0.1, out=Q, work=Q, bytes=need, stream=None)
    refused("wg_latent_attend", good, [
        dict(q_c=None), dict(q_r=None), dict(c_cache=None), dict(r_cache=None), dict(table=None), dict(lens=None), dict(starts=None), dict(out=None), dict(work=None), dict(tokens=0),
        dict(heads=0), dict(heads=4097), dict(latent=320), dict(pages=0), dict(pages=1 << 25), dict(page_tokens=0), dict(rows=0), dict(rows=65536), dict(columns=0), dict(columns=1 << 25),
        dict(tokens=1 << 27, heads=16), dict(tokens=(1 << 27) - 1, heads=16, rows=65535), dict(c0=8190), dict(c1=508), dict(r0=1020), dict(r1=60), dict(q_c=OFF), dict(q_r=OFF), dict(c_cache=OFF),
        dict(r_cache=OFF), dict(out=OFF), dict(factor=math.nan), dict(factor=-math.inf), dict(factor=3e38), dict(bytes=need - 1), dict(work=OFF)])


def test_latent_prompt():
    need = wg.latent_prompt_workspace(100, 2, 4, 128, 9000)
    assert need > 0
    assert wg.latent_prompt_workspace(100, 2, 4, 128, 0) == 0 and wg.latent_prompt_workspace(8000, 4, 32, 128, 8000) == 0
    good = dict(q_n=P, q_r=P, k_n=P, k_r=P, v=P, tokens=100, keys=9000, heads=4, dim=128, qn0=768, qn1=192, qr0=768, qr1=192, kn0=1024, kn1=256, kr0=64, v0=1024, v1=256, rows=2, starts=P,
                key_starts=P, factor=0.1, out=Q, work=Q, bytes=need, stream=None)
    refused("wg_latent_prompt", good, [
        dict(q_n=None), dict(q_r=None), dict(k_n=None), dict(k_r=None), dict(v=None), dict(starts=None), dict(key_starts=None), dict(out=None), dict(work=None), dict(tokens=0), dict(keys=0),
        dict(heads=0), dict(heads=4097), dict(dim=96), dict(dim=256), dict(rows=0), dict(rows=65536), dict(tokens=1 << 31), dict(keys=1 << 31), dict(tokens=1 << 29, heads=4),
        dict(qn0=769), dict(qn1=4), dict(qr0=4), dict(qr1=4), dict(kn0=4), dict(kn1=4), dict(kr0=4), dict(v0=4), dict(v1=4), dict(kn0=1 << 24), dict(kr0=1 << 24), dict(v0=1 << 24), dict(kn0=-1024), dict(kr0=-64), dict(v0=-1024), dict(q_n=OFF), dict(q_r=OFF), dict(k_n=OFF), dict(k_r=OFF), dict(v=OFF),
        dict(out=OFF), dict(factor=math.nan), dict(factor=-3e38), dict(heads=4096, rows=65535, keys=100), dict(bytes=need - 1), dict(work=OFF)])


def test_frequencies():
    """pow, log and the few products behind them are off by some units in the last place: 1e-13 is a thousand of them."""
    i = np.arange(32)
    f = 10000.0 ** (-i / 32)
    np.testing.assert_allclose(wg.rotary_frequencies(64), f, rtol=1e-13)
    np.testing.assert_allclose(wg.rotary_frequencies(64, factor=8.0, low=math.inf), f / 8, rtol=1e-13)
    turns = 4096 * f / (2 * math.pi)
    kept = np.clip((turns - 1) / 3, 0, 1)
    assert kept.min() == 0 and kept.max() == 1 and ((kept > 0) & (kept < 1)).any()
    np.testing.assert_allclose(wg.rotary_frequencies(64, factor=4.0, original=4096), kept * f + (1 - kept) * f / 4, rtol=1e-12)
    kept = np.clip(np.log(turns / 1) / math.log(32), 0, 1)
    np.testing.assert_allclose(wg.rotary_frequencies(64, factor=40.0, original=4096, low=1, high=32, log_ramp=True), kept * f + (1 - kept) * f / 40, rtol=1e-12)
    assert wg.rotary_frequencies(2).tolist() == [1.0]
    for bad in (dict(rotated=0), dict(rotated=7), dict(rotated=2048), dict(base=0.0), dict(base=math.nan), dict(factor=0.5), dict(factor=math.inf), dict(factor=2.0), dict(factor=2.0, original=4096, low=4, high=4),
                dict(factor=2.0, original=4096, low=-1), dict(factor=2.0, original=4096, low=0, log_ramp=True), dict(factor=2.0, original=math.inf)):
        with pytest.raises(wg.WgError):
            wg.rotary_frequencies(**dict(dict(rotated=64), **bad))


def test_calls_that_no_launch_holds():
    """A launch has fewer than 2^32 threads: 2^24 - 1 workgroups of 256, of four tokens each in 8 bits (sixteen in 16, which other limits end), or of sixteen that are read."""
    append = dict(c=P, r=P, tokens=4, latent=512, c0=576, r0=576, slots=P, origins=P, c_cache=Q, r_cache=Q, scale=Q, pages=10, page_tokens=16, stream=None)
    refused("wg_latent_append", append, [dict(tokens=n, latent=latent) for n in ((1 << 26) - 3, 1 << 26, (1 << 26) + 1, 1 << 27) for latent in (256, 512)] + [dict(scale=None, tokens=(1 << 27) + 1)])
    read = dict(c_cache=P, r_cache=P, scale=P, latent=256, pages=10, page_tokens=32, table=P, rows=3, columns=5, starts=P, tokens=100, c_out=Q, c0=256, r_out=Q, r0=64, stream=None)
    refused("wg_latent_read", read, [dict(tokens=n, scale=scale) for n in ((1 << 28) - 15, 1 << 28, (1 << 28) + 1, 1 << 29) for scale in (P, None)])
