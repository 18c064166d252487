"""Arguments that the calls of rotary positions and the cache of latent vectors refuse, on the host, before anything is launched, and the frequencies, which are made
there (CPU; no pointer is followed)."""
import ctypes as C
import math
import os
import subprocess
import sys

import numpy as np
import pytest

import paper_2507_16768_amd as wg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


CALLS = r"""
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2507_16768_amd as wg
from paper_2507_16768_amd import binding
binding.load_library()
i32, f32, f8, b16, f64 = (dict(dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.float8_e4m3fn, torch.bfloat16, torch.float64))


def e(how, *shape):
    return torch.empty(shape, **how)


def make(n=()):
    # what each call takes, in its order; n: a batch in front
    return {
        "rotate": dict(q=e(b16, *n, 4, 3, 64), k=e(b16, *n, 4, 2, 64), positions=e(i32, *n, 4), frequencies=e(f64, *n, 16), q_out=e(b16, *n, 4, 3, 64), k_out=e(b16, *n, 4, 2, 64), interleaved=False,
                       magnitude=1.0, stream=0),
        "latent_append": dict(c=e(b16, *n, 4, 256), r=e(b16, *n, 4, 64), slots=e(i32, *n, 4), origins=e(i32, *n, 4), c_cache=e(f8, *n, 7, 16, 256), r_cache=e(b16, *n, 7, 16, 64),
                              c_scale=e(f32, *n, 7, 16), stream=0),
        "latent_read": dict(c_cache=e(f8, *n, 7, 16, 256), r_cache=e(b16, *n, 7, 16, 64), c_scale=e(f32, *n, 7, 16), table=e(i32, *n, 3, 5), starts=e(i32, *n, 4), c_out=e(b16, *n, 9, 256),
                            r_out=e(b16, *n, 9, 64), stream=0),
        "latent_attend": dict(q_c=e(b16, *n, 4, 3, 256), q_r=e(b16, *n, 4, 3, 64), c_cache=e(f8, *n, 7, 16, 256), r_cache=e(b16, *n, 7, 16, 64), c_scale=e(f32, *n, 7, 16), table=e(i32, *n, 2, 5),
                              lens=e(i32, *n, 2), starts=e(i32, *n, 3), scale=0.1, out=e(b16, *n, 4, 3, 256), workspace=e(dict(dtype=torch.uint8, device="cuda"), *n, 1 << 20), stream=0),
        "latent_prompt": dict(q_n=e(b16, *n, 4, 3, 128), q_r=e(b16, *n, 4, 3, 64), k_n=e(b16, *n, 9, 3, 128), k_r=e(b16, *n, 9, 64), v=e(b16, *n, 9, 3, 128), starts=e(i32, *n, 3),
                              key_starts=e(i32, *n, 3), scale=0.1, out=e(b16, *n, 4, 3, 128), workspace=e(dict(dtype=torch.uint8, device="cuda"), *n, 1 << 20), stream=0)}
"""

NO_STORAGE = r"""
with FakeTensorMode(allow_non_fake_inputs=True):
    for (name, given), batched in zip(make().items(), make((5,)).values()):
        for a in [a for a, x in given.items() if torch.is_tensor(x)]:
            def body(x):
                getattr(wg, name)(**dict(given, **{a: x}))
                return x
            try:
                torch.func.vmap(body)(batched[a])
                print(name, a, "returned")
            except RuntimeError as error:
                assert not isinstance(error, wg.WgError) and "storage" in str(error), (name, a, error)
print("done")
"""

REFUSED = r"""
import re


def refusals():
    cpu = dict(device="cpu")
    caches = [(ValueError, "must be a contiguous device tensor", dict(c_cache=e(dict(f8, **cpu), 7, 16, 256))), (ValueError, "c_cache must be", dict(c_cache=e(f8, 7, 256))),
              (ValueError, "c_cache must be", dict(r_cache=e(b16, 6, 16, 64))), (ValueError, "c_cache must be", dict(r_cache=e(b16, 7, 16, 32))), (ValueError, "c_cache must be", dict(c_scale=e(f32, 7))),
              (ValueError, "float8_e4m3fn", dict(c_scale=None)), (ValueError, "float8_e4m3fn", dict(c_cache=e(b16, 7, 16, 256))), (ValueError, "contiguous", dict(c_cache=e(f8, 7, 256, 16).transpose(1, 2))),
              (ValueError, "r_cache must", dict(r_cache=e(f32, 7, 16, 64))), (ValueError, "c_scale must have dtype torch.float32", dict(c_scale=e(b16, 7, 16))), (TypeError, "c_cache must be a tensor", dict(c_cache=None)),
              (TypeError, "r_cache must be a tensor", dict(r_cache=3)), (TypeError, "c_scale must be a tensor", dict(c_scale=1.0))]
    tables = [(ValueError, "table must", dict(table=e(i32, 5))), (ValueError, "starts", dict(starts=e(i32, 7))), (ValueError, "table must have dtype torch.int32", dict(table=e(f32, 3, 5), starts=e(i32, 4), lens=e(i32, 3))),
              (ValueError, "contiguous", dict(table=e(i32, 5, 3).t(), starts=e(i32, 4), lens=e(i32, 3))), (TypeError, "table must be a tensor", dict(table=None)), (TypeError, "starts must be a tensor", dict(starts=None))]
    return {
        "rotate": [(ValueError, "float32 or bfloat16", dict(q=e(dict(b16, dtype=torch.float16), 4, 3, 64))), (ValueError, "of the dtype of q", dict(k=e(f32, 4, 2, 64))), (ValueError, "of the dtype of q", dict(q_out=e(f32, 4, 3, 64))),
                   (ValueError, "k must be", dict(k=e(b16, 4, 64))), (ValueError, "q must be", dict(q=e(dict(b16, **cpu), 4, 3, 64))), (ValueError, "unit inner stride", dict(q=e(b16, 4, 64, 3).transpose(1, 2))),
                   (ValueError, "in and out", dict(k=None)), (ValueError, "in and out", dict(k_out=None)), (ValueError, "inputs' shapes", dict(q_out=e(b16, 4, 2, 64))), (ValueError, "inputs' shapes", dict(k_out=e(b16, 4, 3, 64))),
                   (ValueError, "inputs' shapes", dict(k=e(b16, 5, 2, 64), k_out=e(b16, 5, 2, 64))), (ValueError, "inputs' shapes", dict(k=e(b16, 4, 2, 32), k_out=e(b16, 4, 2, 32))), (ValueError, "positions must", dict(positions=e(i32, 5))),
                   (ValueError, "positions must", dict(frequencies=e(f64, 2, 8))), (ValueError, "more frequencies", dict(frequencies=e(f64, 65))), (ValueError, "positions must have dtype torch.int32", dict(positions=e(f32, 4))),
                   (ValueError, "frequencies must have dtype torch.float64", dict(frequencies=e(f32, 16))), (ValueError, "contiguous", dict(frequencies=e(f64, 32)[::2])), (TypeError, "q must be a tensor", dict(q=None)),
                   (TypeError, "k must be a tensor", dict(k=7)), (TypeError, "", dict(magnitude="1")), (TypeError, "", dict(stream=[]))],
        "latent_append": caches + [(ValueError, "c must be a \\[T, 256\\]", dict(c=e(b16, 4, 512))), (ValueError, "c must be", dict(c=e(f32, 4, 256))), (ValueError, "c must be", dict(c=e(b16, 256, 4).t())), (ValueError, "r must be a \\[T, 64\\]", dict(r=e(b16, 4, 32))),
                                   (ValueError, "r must be", dict(r=e(dict(b16, **cpu), 4, 64))), (ValueError, "slots and origins", dict(r=e(b16, 5, 64))), (ValueError, "slots and origins", dict(slots=e(i32, 5))), (ValueError, "slots and origins", dict(origins=e(i32, 3))),
                                   (ValueError, "slots must have dtype torch.int32", dict(slots=e(f32, 4))), (ValueError, "origins must have dtype torch.int32", dict(origins=e(f64, 4))), (TypeError, "slots must be a tensor", dict(slots=None))],
        "latent_read": caches + [c for c in tables if "lens" not in c[2]] + [(ValueError, "c_out must be a \\[T, 256\\]", dict(c_out=e(b16, 9, 512))), (ValueError, "r_out must be", dict(r_out=e(b16, 9, 32))), (ValueError, "same tokens", dict(r_out=e(b16, 8, 64))),
                                                                             (ValueError, "c_out must be", dict(c_out=e(f32, 9, 256))), (ValueError, "starts must have dtype torch.int32", dict(starts=e(f32, 4)))],
        "latent_attend": caches + tables + [(ValueError, "q_c must be", dict(q_c=e(f32, 4, 3, 256))), (ValueError, "q_c and out must be", dict(q_c=e(b16, 4, 3, 512), out=e(b16, 4, 3, 512))), (ValueError, "q_c and out must be", dict(out=e(b16, 4, 2, 256))),
                                            (ValueError, "q_c and out must be", dict(q_r=e(b16, 5, 3, 64))), (ValueError, "q_c and out must be", dict(q_r=e(b16, 4, 3, 32))), (ValueError, "q_r must be", dict(q_r=e(b16, 4, 64))), (ValueError, "lens", dict(lens=e(i32, 3))),
                                            (ValueError, "out must have dtype torch.bfloat16", dict(out=e(f32, 4, 3, 256))), (ValueError, "contiguous", dict(out=e(b16, 4, 256, 3).transpose(1, 2))), (ValueError, "lens must have dtype torch.int32", dict(lens=e(f32, 2))),
                                            (TypeError, "out must be a tensor", dict(out=None)), (TypeError, "", dict(scale=None)), (ValueError, "", dict(workspace=e(dict(dtype=torch.uint8, device="cpu"), 64)))],
        "latent_prompt": [(ValueError, "q_n must be", dict(q_n=e(f32, 4, 3, 128))), (ValueError, "q_n and out must be", dict(out=e(b16, 4, 3, 64))), (ValueError, "q_n and out must be", dict(q_r=e(b16, 4, 2, 64))), (ValueError, "q_n and out must be", dict(q_r=e(b16, 4, 3, 128))),
                          (ValueError, "q_n and out must be", dict(k_n=e(b16, 9, 2, 128), v=e(b16, 9, 2, 128))), (ValueError, "q_n and out must be", dict(k_n=e(b16, 9, 3, 64), v=e(b16, 9, 3, 64))), (ValueError, "q_n and out must be", dict(v=e(b16, 8, 3, 128))),
                          (ValueError, "q_n and out must be", dict(k_r=e(b16, 8, 64))), (ValueError, "k_r must be", dict(k_r=e(b16, 9, 32))), (ValueError, "v must be", dict(v=e(f32, 9, 3, 128))), (ValueError, "k_n must be", dict(k_n=e(dict(b16, **cpu), 9, 3, 128))),
                          (ValueError, "starts and key_starts", dict(starts=e(i32, 1), key_starts=e(i32, 1))), (ValueError, "starts and key_starts", dict(key_starts=e(i32, 4))), (ValueError, "starts and key_starts", dict(starts=e(i32, 3, 1))),
                          (ValueError, "starts must have dtype torch.int32", dict(starts=e(f32, 3))), (ValueError, "key_starts must have dtype torch.int32", dict(key_starts=e(f64, 3))), (ValueError, "out must", dict(out=e(f32, 4, 3, 128))),
                          (TypeError, "k_r must be a tensor", dict(k_r=None)), (TypeError, "", dict(scale="x")), (TypeError, "", dict(workspace=4))]}


with FakeTensorMode(allow_non_fake_inputs=True):
    cases = refusals()
    for name, given in make().items():
        for kind, text, change in cases[name]:
            try:
                getattr(wg, name)(**dict(given, **change))
                print(name, list(change), "returned")
            except Exception as error:
                if not isinstance(error, kind) or isinstance(error, wg.WgError) or not re.search(text, str(error)): print(name, list(change), repr(error))
        try:                                                   # as they are, the arguments pass these checks; the C call finds that they have no memory
            getattr(wg, name)(**given)
            print(name, "returned")
        except wg.WgError as error:
            if "null argument" not in str(error): print(name, error)
print("done")
"""


def in_a_process(source):
    r = subprocess.run([sys.executable, "-c", source], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["done"], (r.returncode, r.stdout, r.stderr[-2000:])


def test_tensors_without_storage_raise():
    in_a_process(CALLS + NO_STORAGE)


def test_tensors_that_do_not_fit():
    """Device tensors without memory: every check of types, shapes and strides is reached without a GPU."""
    in_a_process(CALLS + REFUSED)
