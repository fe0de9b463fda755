"""The calls of gfwa_layer.h on the host: every declared function is exported and bound, and bad arguments are refused before anything is
launched (no compute calls here)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
A = P(0x10000)
LL = 1 << 62


@pytest.fixture(scope="module")
def lib():
    import paper_2512_07782_amd as g
    return g.load_library()


def heads(data=0x1000000, batch=0, token=0, head=0):
    import paper_2512_07782_amd as g
    return g.GfwaHeads(data, batch, token, head)


def test_declared_functions_are_exported_and_bound(lib):
    import paper_2512_07782_amd as g
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gfwa_layer.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(gfwa_[a-z_]+)\s*\(", text)))
    assert names == sorted(["gfwa_qk_norm_rope", "gfwa_qk_norm_rope_backward", "gfwa_qk_norm_rope_backward_workspace_bytes", "gfwa_append_paged",
                            "gfwa_decode_paged", "gfwa_decode_paged_workspace_bytes"])
    for n in names:
        assert hasattr(lib, n) and callable(getattr(g, n)) and n in g.binding.EXPORTS, n


def test_status_texts(lib):
    import paper_2512_07782_amd as g
    assert "overlap" in g.gfwa_strerror(-7)


def test_profile_read_serves_callers_of_the_first_ids(lib):
    ms, n = (ctypes.c_float * 13)(), (ctypes.c_int * 13)()
    assert lib.gfwa_profile_read(ms, n, 13) == 0
    assert lib.gfwa_profile_read(ms, n, 12) == -2
    import paper_2512_07782_amd as g
    assert len(g.gfwa_profile_read()) == 19 and "" not in g.gfwa_profile_read()


# ---- norm and rotation.  q, k, v of one packed tensor [2, 10, (4 + 2 + 2) 64] of bf16: 20480 bytes at 0x1000000

def rope(lib, **kw):
    q = kw.get("q", heads(0x1000000, 5120, 512, 64))
    k = kw.get("k", heads(0x1000000 + 512, 5120, 512, 64))
    v = kw.get("v", heads(0x1000000 + 768, 5120, 512, 64))
    r = lambda x: None if x is None else ctypes.byref(x)
    return lib.gfwa_qk_norm_rope(kw.get("dt", 0), r(q), r(k), r(v), kw.get("wq", A), A, kw.get("eps", 1e-6), kw.get("freq", A), kw.get("rot", 64),
                                 kw.get("pos", None), kw.get("flags", 1), kw.get("Q", P(0x2000000)), kw.get("K", P(0x3000000)), kw.get("V", P(0x4000000)),
                                 kw.get("B", 2), kw.get("H", 4), kw.get("Hkv", 2), kw.get("N", 10), kw.get("d", 64), None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(q=None)), (-1, dict(k=None)), (-1, dict(q=heads(0))), (-1, dict(v=heads(0))), (-1, dict(V=None)), (-1, dict(Q=None)), (-1, dict(freq=None)),
    (-2, dict(B=0)), (-2, dict(N=-1)), (-2, dict(H=0)), (-2, dict(Hkv=3)), (-2, dict(Hkv=0)), (-2, dict(rot=8)), (-2, dict(rot=80)), (-2, dict(rot=-16)),
    (-2, dict(eps=-1.0)), (-2, dict(eps=float("nan"))), (-2, dict(B=1 << 20, N=1 << 20)), (-2, dict(B=1 << 14, N=1 << 18)),
    (-2, dict(q=heads(0x1000000, -5120, 512, 64))), (-2, dict(q=heads(0x1000000, LL, 512, 64))), (-2, dict(q=heads(0x1000000, 1 << 40, 512, 64))),
    (-3, dict(d=96)), (-3, dict(dt=2)), (-3, dict(flags=4)),
    (-4, dict(q=heads(0x1000008, 5120, 512, 64))), (-4, dict(q=heads(0x1000000, 5120, 516, 64))), (-4, dict(q=heads(0x1000000, 5120, 512, 68))),
    (-4, dict(Q=P(0x2000008))), (-4, dict(wq=P(0x10002))), (-4, dict(pos=P(0x10002))), (-4, dict(freq=P(0x10004))),
    (-7, dict(Q=P(0x1000000))), (-7, dict(Q=P(0x1000000 - 16))), (-7, dict(K=P(0x2000000))), (-7, dict(V=P(0x1000000 + 20480 - 16))),
])
def test_rope_refuses(lib, status, kw):
    assert rope(lib, **kw) == status


def rope_bwd(lib, **kw):
    r = lambda x: None if x is None else ctypes.byref(x)
    ins = [r(kw.get("q", heads(0x1000000, 5120, 512, 64))), r(kw.get("k", heads(0x1000000 + 512, 5120, 512, 64)))]
    outs = [r(kw.get("dq", heads(0x8000000, 5120, 512, 64))), r(kw.get("dk", heads(0x8000000 + 512, 5120, 512, 64))),
            r(kw.get("dv", heads(0x8000000 + 768, 5120, 512, 64)))]
    return lib.gfwa_qk_norm_rope_backward(kw.get("dt", 0), *ins, A, A, kw.get("eps", 1e-6), A, kw.get("rot", 64), None, kw.get("flags", 1),
                                          kw.get("dQ", P(0x2000000)), P(0x3000000), kw.get("dV", P(0x4000000)), *outs, kw.get("dwq", A), kw.get("dwk", P(0x20000)),
                                          kw.get("ws", P(0x5000000)), kw.get("wsb", 1 << 30), 2, 4, kw.get("Hkv", 2), 10, kw.get("d", 64), None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(q=None)), (-1, dict(dQ=None)), (-1, dict(dq=None)), (-1, dict(dV=None)), (-1, dict(dv=None)),
    (-2, dict(Hkv=3)), (-2, dict(rot=24)), (-2, dict(eps=-1.0)), (-3, dict(d=32)), (-3, dict(dt=5)), (-3, dict(flags=0)), (-3, dict(flags=8)),
    (-4, dict(dQ=P(0x2000004))), (-4, dict(dwq=P(0x10001))), (-4, dict(dq=heads(0x8000004, 5120, 512, 64))), (-4, dict(ws=P(0x5000008))),
    (-5, dict(ws=None)), (-5, dict(wsb=1000)),
    (-7, dict(dwk=A)), (-7, dict(dwk=P(0x10000 + 128))), (-7, dict(dq=heads(0x1000000, 5120, 512, 64))), (-7, dict(dq=heads(0x2000000, 5120, 512, 64))),
    (-7, dict(dq=heads(0x8000000, 0, 512, 64))), (-7, dict(dq=heads(0x8000000, 5120, 128, 64))), (-7, dict(dq=heads(0x8000000, 5120, 512, 0))),
])
def test_rope_backward_refuses(lib, status, kw):
    assert rope_bwd(lib, **kw) == status


def test_rope_backward_workspace(lib):
    f = lib.gfwa_qk_norm_rope_backward_workspace_bytes
    assert f(2, 4, 2, 10, 64) > 0 and f(2, 4, 3, 10, 64) == 0 and f(2, 4, 2, 10, 96) == 0 and f(0, 4, 2, 10, 64) == 0


# ---- the paged cache: 6 pages of 32 rows

def append(lib, **kw):
    r = lambda x: None if x is None else ctypes.byref(x)
    q, k, v = (r(kw.get(n, heads(0x1000000 + o, 0, 512, 64))) for n, o in (("q", 0), ("k", 512), ("v", 768)))
    return lib.gfwa_append_paged(kw.get("dt", 0), q, k, v, A, A, kw.get("eps", 1e-6), kw.get("freq", A), kw.get("rot", 64), kw.get("flags", 1),
                                 kw.get("alpha", P(0x1800000)), kw.get("at", 4), kw.get("ah", 1), kw.get("start", A), kw.get("cached", A),
                                 kw.get("table", A), kw.get("Q", P(0x2000000)), kw.get("Kp", P(0x3000000)), kw.get("Vp", P(0x4000000)),
                                 kw.get("cp", P(0x5000000)), kw.get("rows", 10), kw.get("B", 2), kw.get("H", 4), kw.get("Hkv", 2), kw.get("d", 64),
                                 kw.get("pages", 6), kw.get("page", 32), kw.get("M", 3), None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(k=None)), (-1, dict(v=None)), (-1, dict(v=heads(0))), (-1, dict(Q=None)), (-1, dict(Kp=None)), (-1, dict(cp=None)), (-1, dict(start=None)),
    (-1, dict(cached=None)), (-1, dict(table=None)), (-1, dict(freq=None)),
    (-2, dict(rows=0)), (-2, dict(B=0)), (-2, dict(Hkv=3)), (-2, dict(pages=0)), (-2, dict(page=0)), (-2, dict(page=24)), (-2, dict(page=8)), (-2, dict(M=0)),
    (-2, dict(M=1 << 26)), (-2, dict(rot=72)), (-2, dict(at=-1)), (-2, dict(ah=LL)), (-2, dict(at=1 << 40)),
    (-3, dict(d=80)), (-3, dict(dt=-1)), (-3, dict(flags=16)),
    (-4, dict(Kp=P(0x3000008))), (-4, dict(cp=P(0x5000002))), (-4, dict(alpha=P(0x1800002))), (-4, dict(start=P(0x10001))), (-4, dict(k=heads(0x1000200, 0, 516, 64))),
    (-7, dict(Kp=P(0x1000000))), (-7, dict(Q=P(0x3000000))), (-7, dict(cp=P(0x1800000))), (-7, dict(Vp=P(0x3000000 + 16))),
])
def test_append_refuses(lib, status, kw):
    assert append(lib, **kw) == status


def decode(lib, **kw):
    return lib.gfwa_decode_paged(kw.get("dt", 0), kw.get("q", A), kw.get("Kp", A), A, kw.get("cp", A), kw.get("table", A), kw.get("pos", A), kw.get("o", A),
                                 kw.get("L", None), kw.get("ws", A), kw.get("wsb", 1 << 30), kw.get("B", 2), kw.get("H", 4), kw.get("Hkv", 2), kw.get("d", 64),
                                 kw.get("pages", 6), kw.get("page", 32), kw.get("M", 3), kw.get("w", 50), 0.1, None)


@pytest.mark.parametrize("status,kw", [
    (-1, dict(q=None)), (-1, dict(cp=None)), (-1, dict(table=None)), (-1, dict(pos=None)), (-1, dict(o=None)),
    (-2, dict(B=0)), (-2, dict(Hkv=3)), (-2, dict(pages=-1)), (-2, dict(page=20)), (-2, dict(M=0)), (-2, dict(w=0)), (-2, dict(M=1 << 27)), (-2, dict(B=1 << 21)),
    (-3, dict(d=96)), (-3, dict(dt=9)), (-4, dict(q=P(0x10008))), (-4, dict(o=P(0x10008))), (-4, dict(L=P(0x10002))), (-4, dict(pos=P(0x10001))), (-4, dict(ws=P(0x10008))),
    (-5, dict(ws=None)), (-5, dict(wsb=8)),
])
def test_decode_refuses(lib, status, kw):
    assert decode(lib, **kw) == status


# what a call writes against what it reads besides the rows, and against its workspace
@pytest.mark.parametrize("call,kw", [
    (rope, dict(pos=P(0x2000000))), (rope, dict(pos=P(0x2000000 - 76))), (rope, dict(freq=P(0x3000000))), (rope, dict(freq=P(0x4000000 - 248))), (rope, dict(wq=P(0x4000000 + 16))),
    (rope_bwd, dict(dwq=P(0x5000000))), (rope_bwd, dict(dwq=P(0x2000000))), (rope_bwd, dict(dwq=P(0x8000000))), (rope_bwd, dict(dwq=P(0x1000000))), (rope_bwd, dict(dwq=P(0x10000))),
    (rope_bwd, dict(dwq=P(0x11000), ws=P(0x4000000))), (rope_bwd, dict(dwq=P(0x11000), ws=P(0x8000000))), (rope_bwd, dict(dq=heads(0x10000, 5120, 512, 64))),
    (append, dict(start=P(0x3000000))), (append, dict(cached=P(0x2000000))), (append, dict(table=P(0x5000000 - 20))), (append, dict(freq=P(0x4000000))),
    (decode, dict(o=P(0x900000 + 512), q=P(0x900000), L=P(0x800000))), (decode, dict(o=P(0x900000), L=P(0x900000 + 1020), ws=P(0xa00000))),
    (decode, dict(o=P(0x900000), ws=P(0x900000 + 1008))), (decode, dict(o=P(0x900000), ws=P(0xa00000), pos=P(0xa00000))),
    (decode, dict(o=P(0x900000), ws=P(0xa00000), table=P(0x900000))), (decode, dict(o=P(0x900000), ws=P(0xa00000), Kp=P(0x900000 - 16))),
    (decode, dict(o=P(0x900000), ws=P(0xa00000), cp=P(0xa00000 + 64))),
])
def test_overlaps_are_refused(lib, call, kw):
    assert call(lib, **kw) == -7


def test_decode_workspace(lib):
    f = lib.gfwa_decode_paged_workspace_bytes
    assert f(2, 4, 2, 128, 32, 100, 1000) >= 2 * 4 * 130 * 4
    assert f(2, 4, 3, 128, 32, 100, 1000) == 0 and f(2, 4, 2, 128, 24, 100, 1000) == 0 and f(2, 4, 2, 128, 32, 100, 0) == 0 and f(2, 4, 2, 100, 32, 100, 10) == 0
    # it does not grow without bound with the length of the cache
    assert f(64, 32, 8, 128, 64, 1 << 20, 1 << 30) <= 64 << 20


def test_binding_refuses_on_the_host():
    import torch
    import paper_2512_07782_amd as g
    x = torch.zeros(1, 4, 2, 64)
    with pytest.raises(ValueError, match="GPU"):
        g.gfwa_qk_norm_rope(x, x)
    with pytest.raises(ValueError):
        g.gfwa_qk_norm_rope(x[0], x)
    with pytest.raises(TypeError):
        g.gfwa_qk_norm_rope(x.half(), x.half())
    with pytest.raises(TypeError):
        g.gfwa_qk_norm_rope(None, x)
    with pytest.raises(ValueError, match="divide"):
        g.gfwa_qk_norm_rope(x, torch.zeros(1, 4, 3, 64))
