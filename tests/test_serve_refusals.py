"""Arguments that the calls of beam search and the paged cache refuse, on the host, before anything is launched (CPU; no pointer is followed)."""
import ctypes as C
import subprocess
import sys
import os

import pytest

import paper_2507_16768_amd as wg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, Q = C.c_void_p(4096), C.c_void_p(1 << 20)


def refused(call, name, good, cases):
    """Each case differs from the good call in what it names, and is refused."""
    L = wg.load_library()
    for case in cases:
        args = dict(good, **case)
        rc = getattr(L, call)(*args.values())
        assert rc == -1, case
        assert L.wg_last_error().startswith(name.encode()), (case, L.wg_last_error())


def test_beam_select():
    need = wg.beam_select_workspace(8, 2000, 4)
    assert need == 8 * 1 * 5 * 8 and wg.beam_select_workspace(0, 5, 1) == 0 and wg.beam_select_workspace(4, 5, 0) == 0 and wg.beam_select_workspace(4, 32000, 4) == 4 * 16 * 5 * 8
    good = dict(logits=P, dtype=0, rows=8, V=2000, stride=2000, mask=P, beams=4, scores=P, states=P, out=Q, parents=Q, tokens=Q, out_states=Q,
                work=Q, bytes=need, stream=None)
    refused("wg_beam_select", "wg_beam_select", good, [
        dict(logits=None), dict(scores=None), dict(out=None), dict(parents=None), dict(tokens=None), dict(work=None), dict(states=None),
        dict(out_states=None), dict(dtype=2), dict(rows=0), dict(V=0), dict(stride=1999), dict(rows=65536, bytes=1 << 40), dict(beams=0), dict(beams=65, rows=65),
        dict(beams=3), dict(out=P), dict(out_states=P), dict(bytes=need - 1), dict(work=C.c_void_p(4100))])


def test_reorder_rows():
    good = dict(src=P, dst=Q, parents=P, outer=1, rows=4, row_bytes=16, so=0, sr=16, do=0, dr=16, stream=None)
    refused("wg_reorder_rows", "wg_reorder_rows", good, [dict(src=None), dict(dst=None), dict(parents=None), dict(dst=P), dict(outer=0), dict(rows=0), dict(row_bytes=0),
                                                         dict(outer=65536), dict(rows=65536), dict(sr=15), dict(dr=8)])


def test_page_step():
    need = wg.page_step_workspace(8, 4, 10)
    assert need == 2 * (8 + 8) + 8 * 4 and wg.page_step_workspace(8, 0, 10) == 0 and wg.page_step_workspace(64, 64, 300) == 8 + 10 * 8 + 64 * 4
    good = dict(table=P, rows=8, columns=10, lens=P, counts=P, parents=P, beams=4, page=16, ring=P, pages=100, counters=P, table_out=Q, lens_out=Q, starts=Q, slots=Q,
                positions=Q, origins=Q, tokens=8, counters_out=Q, work=Q, bytes=need, stream=None)
    refused("wg_page_step", "wg_page_step", good, [
        dict([(k, None)]) for k in ("table", "lens", "counts", "ring", "counters", "table_out", "lens_out", "starts", "slots", "positions", "origins", "counters_out", "work")] + [
        dict(rows=0), dict(columns=0), dict(pages=0), dict(rows=65536, bytes=1 << 30), dict(page=8), dict(page=48), dict(page=128), dict(page=0), dict(columns=1 << 27),
        dict(pages=1 << 27), dict(tokens=1 << 31), dict(beams=0), dict(beams=3), dict(beams=65, rows=65), dict(parents=None), dict(table_out=P), dict(lens_out=P),
        dict(counters_out=P), dict(bytes=need - 1), dict(work=C.c_void_p(4104))])


def test_cache_append():
    good = dict(k=P, v=P, tokens=4, heads=2, dim=64, k0=128, k1=64, v0=128, v1=64, slots=P, origins=None, k_cache=Q, v_cache=Q, k_scale=Q, v_scale=Q, pages=10, page=16,
                stream=None)
    refused("wg_cache_append", "wg_cache_append", good, [
        dict([(k, None)]) for k in ("k", "v", "slots", "k_cache", "v_cache", "k_scale", "v_scale")] + [
        dict(tokens=0), dict(heads=0), dict(pages=0), dict(heads=65536), dict(dim=96), dict(dim=512), dict(page=24), dict(pages=1 << 27), dict(k0=129), dict(v1=4),
        dict(k=C.c_void_p(4104)), dict(v=C.c_void_p(4098)), dict(k_cache=C.c_void_p(4104)), dict(v_cache=C.c_void_p(4104)), dict(tokens=1 << 31),
        dict(k0=1 << 24), dict(v0=-128)])


def test_cache_attend():
    shape = dict(tokens=2, rows=2, q_heads=8, heads=2, dim=64, columns=100, page_tokens=16)
    need = wg.cache_attend_workspace(**shape)
    assert need == (2 * 8 * 2 * 66 + 2) * 4 and wg.cache_attend_workspace(**dict(shape, columns=8)) == 0 and wg.cache_attend_workspace(**dict(shape, heads=0)) == 0
    good = dict(q=P, tokens=2, q_heads=8, heads=2, dim=64, q0=512, q1=64, k_cache=P, v_cache=P, k_scale=P, v_scale=P, pages=200, page=16, table=P, rows=2, columns=100,
                lens=P, starts=P, scale=0.125, out=Q, work=Q, bytes=need, stream=None)
    refused("wg_cache_attend", "wg_cache_attend", good, [
        dict([(k, None)]) for k in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "table", "lens", "starts", "out", "work")] + [
        dict(tokens=0), dict(rows=0), dict(columns=0), dict(pages=0), dict(heads=0), dict(rows=65536), dict(tokens=1 << 31), dict(q_heads=7), dict(q_heads=1),
        dict(q_heads=65536), dict(heads=4096, q_heads=4096), dict(dim=32), dict(page=17), dict(columns=1 << 27), dict(pages=1 << 27), dict(q0=513), dict(q1=4),
        dict(q=C.c_void_p(4104)), dict(k_cache=C.c_void_p(4104)), dict(v_cache=C.c_void_p(4104)), dict(out=C.c_void_p(4104)), dict(scale=float("nan")), dict(scale=float("inf")),
        dict(bytes=need - 1), dict(work=C.c_void_p(4104))])


def test_calls_that_no_launch_holds():
    append = dict(k=P, v=P, tokens=(1 << 29) + 1, heads=2, dim=64, k0=128, k1=64, v0=128, v1=64, slots=P, origins=None, k_cache=Q, v_cache=Q, k_scale=Q, v_scale=Q, pages=10,
                  page=16, stream=None)
    refused("wg_cache_append", "wg_cache_append", append, [{}])
    refused("wg_reorder_rows", "wg_reorder_rows", dict(src=P, dst=Q, parents=P, outer=1, rows=1, row_bytes=(1 << 33) + 16, so=0, sr=1 << 40, do=0, dr=1 << 40, stream=None), [{}])
    attend = dict(q=P, tokens=1 << 27, q_heads=64, heads=8, dim=64, q0=512, q1=64, k_cache=P, v_cache=P, k_scale=P, v_scale=P, pages=200, page=16, table=P, rows=2, columns=100,
                  lens=P, starts=P, scale=0.125, out=Q, work=Q, bytes=1 << 62, stream=None)
    refused("wg_cache_attend", "wg_cache_attend", attend, [{}, dict(tokens=0x7FFFFFFF), dict(rows=65535, heads=4095, q_heads=4095 * 16, tokens=65535 * 16)])


NO_STORAGE = r"""
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2507_16768_amd as wg
from paper_2507_16768_amd import binding
binding.load_library()
with FakeTensorMode(allow_non_fake_inputs=True):
    given, CALLS = make(torch, wg)
    for name, (names, call) in CALLS.items():
        for batched in names:
            def body(x):
                call(**{a: (x if a == batched else given[a][0]) for a in names})
                return x
            try:
                torch.func.vmap(body)(given[batched])
                print(name, batched, "returned")
            except RuntimeError as e:
                assert not isinstance(e, wg.WgError) and "storage" in str(e), (name, batched, e)
print("done")
"""

BEAM = r"""
def make(torch, wg):
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(device="cuda")
    given = dict(logits=torch.empty((5, 4, 64), **f32), mask=torch.empty((5, 4, 2), **i32), scores=torch.empty((5, 4), **f32), states=torch.empty((5, 4, 2), **i32),
                 out=torch.empty((5, 4), **f32), parents=torch.empty((5, 4), **i32), tokens=torch.empty((5, 4), **i32), ends=torch.empty((5, 4, 2), **i32),
                 work=torch.empty((5, 4096), dtype=torch.uint8, device="cuda"), src=torch.empty((5, 4, 8), **f32), dst=torch.empty((5, 4, 8), **f32))
    return given, {
        "beam_select": (("logits", "mask", "scores", "states", "out", "parents", "tokens", "ends", "work"),
                        lambda logits, mask, scores, states, out, parents, tokens, ends, work:
                        wg.beam_select(logits, mask, scores, states, 2, out, parents, tokens, ends, work, 0)),
        "reorder_rows": (("src", "parents", "dst"), lambda src, parents, dst: wg.reorder_rows(src, parents, dst, 0, 0))}
"""


CACHE = r"""
def make(torch, wg):
    i32, f32, f8, b16 = dict(dtype=torch.int32, device="cuda"), dict(device="cuda"), dict(dtype=torch.float8_e4m3fn, device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
    i64 = dict(dtype=torch.int64, device="cuda")
    given = dict(table=torch.empty((5, 4, 6), **i32), lens=torch.empty((5, 4), **i32), counts=torch.empty((5, 4), **i32), parents=torch.empty((5, 4), **i32),
                 ring=torch.empty((5, 30), **i32), counters=torch.empty((5, 2), **i64), out_table=torch.empty((5, 4, 6), **i32), out_lens=torch.empty((5, 4), **i32),
                 starts=torch.empty((5, 5), **i32), slots=torch.empty((5, 4), **i32), positions=torch.empty((5, 4), **i32), origins=torch.empty((5, 4), **i32),
                 out_counters=torch.empty((5, 2), **i64), work=torch.empty((5, 1 << 16), dtype=torch.uint8, device="cuda"),
                 k=torch.empty((5, 4, 2, 64), **b16), v=torch.empty((5, 4, 2, 64), **b16), q=torch.empty((5, 4, 4, 64), **b16), out=torch.empty((5, 4, 4, 64), **b16),
                 kc=torch.empty((5, 7, 2, 16, 64), **f8), vc=torch.empty((5, 7, 2, 64, 16), **f8), ks=torch.empty((5, 7, 2), **f32), vs=torch.empty((5, 7, 2), **f32))
    return given, {
        "page_step": (("table", "lens", "counts", "parents", "ring", "counters", "out_table", "out_lens", "starts", "slots", "positions", "origins", "out_counters", "work"),
                      lambda table, lens, counts, parents, ring, counters, out_table, out_lens, starts, slots, positions, origins, out_counters, work:
                      wg.page_step(table, lens, counts, parents, 2, 16, ring, counters, out_table, out_lens, starts, slots, positions, origins, out_counters, work, 0)),
        "cache_append": (("k", "v", "slots", "origins", "kc", "vc", "ks", "vs"),
                         lambda k, v, slots, origins, kc, vc, ks, vs: wg.cache_append(k, v, slots, origins, kc, vc, ks, vs, 0)),
        "cache_attend": (("q", "kc", "vc", "ks", "vs", "table", "lens", "starts", "out", "work"),
                         lambda q, kc, vc, ks, vs, table, lens, starts, out, work: wg.cache_attend(q, kc, vc, ks, vs, table, lens, starts, 0.1, out, work, 0))}
"""


def no_storage(make):
    r = subprocess.run([sys.executable, "-c", make + NO_STORAGE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["done"], (r.returncode, r.stdout, r.stderr[-2000:])


@pytest.mark.parametrize("make", [BEAM, CACHE], ids=["beam", "cache"])
def test_tensors_without_storage_raise(make):
    no_storage(make)


def test_tensors_that_do_not_fit():
    import torch
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError, match="device tensor"):
        wg.beam_select(x, None, x[:, 0], None, 2, x[:, 0], x[:, 0], x[:, 0], None, x)
    with pytest.raises(TypeError, match="logits must be a tensor"):
        wg.beam_select(None, None, x, None, 2, x, x, x, None, x)
    with pytest.raises(ValueError, match="agree in shape"):
        wg.reorder_rows(x, x, x[:2])
    with pytest.raises(ValueError, match="device tensors"):
        wg.reorder_rows(x, x, x)
    i = torch.zeros((4, 6), dtype=torch.int32)
    with pytest.raises(ValueError, match="out_table must be"):
        wg.page_step(i, i[:, 0], i[:, 0], None, 1, 16, i[0], i[0], i, i[:, 0], i[0], i[0], i[0], i[0], i[0])
    with pytest.raises(ValueError, match="out of range"):
        wg.page_step(i, i, i, None, 1 << 40, 16, i[0], i[0], i, i, i, i[0], i[0], i[0], i[0])
    f8 = torch.zeros((3, 2, 16, 64)).to(torch.float8_e4m3fn)
    s = torch.ones((3, 2))
    kv = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k_cache must be"):
        wg.cache_append(kv, kv, i[0], None, f8, f8, s, s)
    with pytest.raises(ValueError, match="device tensor"):
        wg.cache_append(kv, kv, i[0], None, f8, f8.transpose(2, 3).contiguous(), s, s)
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        wg.cache_attend(kv, f8.float(), f8.float().transpose(2, 3), s, s, i, i[:, 0], i[0], 1.0, kv)
