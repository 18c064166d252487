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
    assert need == 8 * 1 * 5 * 8 and wg.beam_select_workspace(0, 5, 1) == 0 and wg.beam_select_workspace(4, 32000, 4) == 4 * 4 * 5 * 8
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


def no_storage(make):
    r = subprocess.run([sys.executable, "-c", make + NO_STORAGE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["done"], (r.returncode, r.stdout, r.stderr[-2000:])


def test_tensors_without_storage_raise():
    no_storage(BEAM)


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
