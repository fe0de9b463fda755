"""Gradients that share memory with each other are refused on the host, strided ones that only interleave are not (nothing is launched here)."""
import ctypes

import numpy as np
import pytest

from test_layer_abi import A, P, heads, lib, rope_bwd  # noqa: F401 (lib is a fixture)

BASE = 0x8000000


@pytest.mark.parametrize("kw", [
    dict(dk=heads(BASE, 5120, 512, 64)),                       # the same tensor twice
    dict(dv=heads(BASE + 512, 5120, 512, 64)),                 # dk's
    dict(dk=heads(BASE + 384, 5120, 512, 64)),                 # begins inside dq's last head
    dict(dk=heads(BASE - 128, 5120, 512, 64)),                 # its second head is dq's first one
    dict(dv=heads(BASE + 512 + 16, 5120, 512, 64)),            # eight elements off dk's rows
    dict(dk=heads(BASE + 19 * 1024 + 256, 5120, 512, 64)),     # all behind each other, its first row inside dq's last token
    dict(dk=heads(BASE - 19 * 1024 - 128, 5120, 512, 64)),     # its last row is dq's first one
    dict(dv=heads(BASE + 768 - 112, 5120, 512, 64)),           # dk's last row ends inside its first one
    dict(dk=heads(BASE + 1024 * 10, 5120, 512, 64)),           # dq's second sequence
])
def test_gradients_that_share_elements_are_refused(lib, kw):
    assert rope_bwd(lib, ws=None, **kw) == -7


@pytest.mark.parametrize("kw", [
    dict(),                                                                                                            # packed by kind
    dict(dq=heads(BASE, 5120, 512, 128), dk=heads(BASE + 128, 5120, 512, 256), dv=heads(BASE + 128 + 256, 5120, 512, 256)),  # heads of each kind in turn
    dict(dv=heads(BASE - 0x10000, 5120, 512, 64)), dict(dk=heads(BASE + 20480, 5120, 512, 64)),                        # behind each other
    dict(dq=heads(BASE, 64 * 4, 64 * 16, 64), dk=heads(BASE + 1024, 64 * 2, 64 * 16, 64), dv=heads(BASE + 1536, 64 * 2, 64 * 16, 64)),  # [N,B,..]
])
def test_gradients_that_interleave_are_not(lib, kw):
    assert rope_bwd(lib, ws=None, **kw) == -5  # the next thing in order: no workspace


def test_the_look_at_rows_agrees_with_counting():
    """Random strided outputs of few elements: the status against the elements themselves, where ends decide."""
    import paper_2512_07782_amd as g
    lib = g.load_library()
    rng = np.random.default_rng(3)
    B, N, H, Hkv, d = 2, 3, 4, 2, 64
    seen = set()
    for _ in range(3000):
        def tensor(count):
            order = rng.permutation(3)
            counts, strides, reach = [B, N, count], [0, 0, 0], d
            for i in order:
                strides[i] = reach + 64 * int(rng.integers(0, 4))
                reach = strides[i] * counts[i]
            at = 64 * int(rng.integers(0, 60)) + 8 * int(rng.integers(0, 2))
            rows = [at + b * strides[0] + n * strides[1] + h * strides[2] for b in range(B) for n in range(N) for h in range(count)]
            return at, strides, rows
        t = [tensor(c) for c in (H, Hkv, Hkv)]
        sets = [set(r + e for r in rows for e in range(0, d, 8)) for _, _, rows in t]
        ends = [set(r + e for r in (rows[0], rows[-1]) for e in range(0, d, 8)) for _, _, rows in t]
        meet = any(ends[i] & sets[j] for i in range(3) for j in range(3) if i != j)
        apart = not any(sets[i] & sets[j] for i in range(3) for j in range(i))
        h = [heads(BASE + 2 * at, *s) for at, s, _ in t]
        got = rope_bwd_sized(lib, h, B, N, H, Hkv, d)
        assert got == (-7 if meet else -5), (t, got)
        seen.add((meet, apart))
    assert (True, False) in seen and (False, True) in seen


def rope_bwd_sized(lib, outs, B, N, H, Hkv, d):
    r = ctypes.byref
    q, k = heads(0x1000000, N * H * d, H * d, d), heads(0x1800000, N * Hkv * d, Hkv * d, d)
    return lib.gfwa_qk_norm_rope_backward(0, r(q), r(k), A, A, 1e-6, A, 64, None, 1, P(0x2000000), P(0x3000000), P(0x4000000), *[r(x) for x in outs], A, P(0x20000),
                                          None, 0, B, H, Hkv, N, d, None)


def test_gradient_without_inputs_on_the_host():
    import torch
    import paper_2512_07782_amd as g
    x = torch.zeros(1, 2, 4, 64)
    with pytest.raises(TypeError, match="q must be a tensor"):
        g.gfwa_qk_norm_rope_backward(None, None, x, x)
    with pytest.raises(TypeError, match="dQ must be a tensor"):
        g.gfwa_qk_norm_rope_backward(None, None, None, x, norm=False)
    with pytest.raises(ValueError, match="dQ .B,H,N,d."):
        g.gfwa_qk_norm_rope_backward(None, None, x[0], x, norm=False)
    with pytest.raises(ValueError, match="divide"):
        g.gfwa_qk_norm_rope_backward(None, None, x, torch.zeros(1, 3, 4, 64), norm=False)
    with pytest.raises(ValueError, match="GPU"):
        g.gfwa_qk_norm_rope_backward(None, None, x, x, norm=False)
