"""The operators around the attention on the GPU against the fp64 oracle (oracle/layer.py).

Tolerances.  half = eps / 2 of the storage type (2^-8 bf16, 2^-24 fp32): one rounding of the result.  u = 2^-24, one fp32 rounding.
  norm: the sum of squares of d elements, 16 in a chain and three exchanges, is off by 20 u of itself, its root by 10 u, then root, quotient
  and two products: 16 u in all.  rotation: the angle is rounded at 2^-25 half turns (pi / 2 u of a turn's arc), sin and cos at 2 units, two
  products and a sum: 8 u of |a| + |b|.  Together below 32 u times the sum of the pair's magnitudes; angles in fp64 add 2^-51 of the angle.
  dx = r (g w - u mean(g w u)): 64 u of r (|g w| + |u| mean|g w u|), the rotated g being off by 8 u of its pair's sum.
  dw: products off by 32 u, sums of at most 16 + 3 + 4 + 64 + 32 terms in a chain (rows of a lane: the tests' sizes give each lane at most 16): 160 u of
  the sum of magnitudes.
  c: fp64 sums rounded once: u.
  decode: scores from n = d products in fp32, d + 8 units of scale sum|q||k| and 8 units of |S|: E; weights off by 2 E + 8 u and, in bf16, taken
  as two bf16 numbers into the second product (2^-16 of each, twice that for the sums of their parts); sums of n keys off by at most n units; the quotient is rounded to the storage type.
"""
import numpy as np
import pytest
import torch

import gfwa_inputs as gi
from oracle import layer as ol

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


@pytest.fixture(scope="module")
def g():
    import paper_2512_07782_amd as mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mod.load_library()
    return mod


def host(t):
    return t.detach().double().cpu().numpy()


def store(x, dtype):
    """fp32 numpy values of the storage type and the GPU tensor that holds them."""
    x = np.asarray(x, dtype=np.float32)
    x = gi.round_to_bf16(x) if dtype == "bf16" else x
    return x, torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(TORCH[dtype])


def freq_of(rot):
    return None if rot == 0 else 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)


def dev64(f):
    return None if f is None else torch.from_numpy(f).to(DEV)


def layout(x, kind, dtype):
    """x [B,N,heads,d] on the GPU in the strides a caller may have, and its values."""
    x, t = store(x, dtype)
    B, N, h, d = x.shape
    if kind == "dense":
        return x, t
    if kind == "packed":  # the middle heads of a wider token
        wide = torch.full((B, N, h + 3, d), float("nan"), dtype=t.dtype, device=DEV)
        wide[:, :, 2:2 + h] = t
        return x, wide[:, :, 2:2 + h]
    if kind == "head_major":  # [B,heads,N,d] seen through a transpose
        return x, t.transpose(1, 2).contiguous().transpose(1, 2)
    if kind == "padded_rows":  # rows of d + 16 elements
        wide = torch.full((N, B, h, d + 16), float("nan"), dtype=t.dtype, device=DEV)
        wide[..., :d] = t.transpose(0, 1)
        return x, wide[..., :d].transpose(0, 1)
    raise AssertionError(kind)


def pair_sums(y, rot, paired):
    """|y_i| + |y_j| of the element's pair, which is what its rotation mixes."""
    out = np.abs(y).copy()
    i, j = ol._pairs(y.shape[-1], rot, paired)
    both = np.abs(y[..., i]) + np.abs(y[..., j])
    out[..., i], out[..., j] = both, both
    return out


# B, H, Hkv, N, d, rot, paired, norm, layout, positions
ROPE = [
    (1, 1, 1, 1, 64, 64, False, True, "dense", None), (1, 1, 1, 1, 128, 128, False, True, "packed", None),
    (2, 8, 2, 37, 128, 128, False, True, "packed", None), (2, 8, 2, 37, 128, 128, True, True, "packed", None),
    (3, 6, 3, 131, 64, 32, False, True, "head_major", "random"), (3, 6, 3, 131, 64, 32, True, True, "padded_rows", "random"),
    (1, 4, 1, 517, 128, 16, False, True, "padded_rows", "far"), (1, 4, 1, 517, 64, 16, True, True, "dense", "far"),
    (2, 5, 5, 65, 128, 0, False, True, "packed", None), (2, 5, 5, 65, 64, 48, False, False, "packed", "random"),
    (70, 3, 1, 1, 128, 96, False, True, "packed", "far"), (1, 16, 4, 1003, 64, 64, False, False, "head_major", None),
    (4, 12, 4, 300, 128, 128, False, True, "packed", "negative"), (2, 2, 1, 9, 64, 0, True, False, "dense", None),
]


def positions(kind, B, N, rng):
    if kind is None:
        return np.broadcast_to(np.arange(N), (B, N)), None
    p = {"random": lambda: rng.integers(0, 5000, (B, N)), "far": lambda: rng.integers(2 ** 20, 2 ** 31 - 1, (B, N)),
         "negative": lambda: rng.integers(-3000, 3000, (B, N))}[kind]().astype(np.int32)
    return p, torch.from_numpy(p).to(DEV)


def rope_inputs(B, H, Hkv, N, d, rot, kind, pos_kind, dtype):
    rng = np.random.default_rng(B * 1000 + N + d + rot)
    pos, pos_dev = positions(pos_kind, B, N, rng)
    q, tq = layout(rng.standard_normal((B, N, H, d)) * np.exp(rng.standard_normal((1, 1, H, 1))), kind, dtype)
    k, tk = layout(rng.standard_normal((B, N, Hkv, d)) * 3, kind, dtype)
    v, tv = layout(rng.standard_normal((B, N, Hkv, d)), kind, dtype)
    wq, wk = (1 + 0.3 * rng.standard_normal((2, d))).astype(np.float32)
    return rng, pos, pos_dev, (q, tq), (k, tk), (v, tv), (wq, torch.from_numpy(wq).to(DEV)), (wk, torch.from_numpy(wk).to(DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,N,d,rot,paired,norm,kind,pos_kind", ROPE)
def test_norm_and_rotation(g, B, H, Hkv, N, d, rot, paired, norm, kind, pos_kind, dtype):
    print("rope", B, H, Hkv, N, d, rot, paired, norm, kind, pos_kind, dtype, flush=True)
    _, pos, pos_dev, (q, tq), (k, tk), (v, tv), (wq, twq), (wk, twk) = rope_inputs(B, H, Hkv, N, d, rot, kind, pos_kind, dtype)
    freq = freq_of(rot)
    Q, K, V = g.gfwa_qk_norm_rope(tq, tk, tv, twq if norm else None, twk if norm else None, EPS, dev64(freq), pos_dev, norm=norm, paired=paired)
    assert Q.is_contiguous() and Q.shape == (B, H, N, d) and K.shape == V.shape == (B, Hkv, N, d)
    assert torch.equal(V, tv.transpose(1, 2))
    for x, wt, got in ((q, wq, Q), (k, wk, K)):
        plain = ol.norm_rope_rows(x, wt, EPS, norm, pos, None, paired)
        ref = ol.norm_rope_rows(x, wt, EPS, norm, pos, freq, paired)
        off = U * 32 + (2.0 ** -51 * np.abs(pos).max() if rot else 0)
        tol = HALF[dtype] * np.abs(ref) + off * pair_sums(plain, rot, paired) * (1 + HALF[dtype])
        err = np.abs(host(got.transpose(1, 2)) - ref)
        assert (err <= tol + 1e-38).all(), (err / (tol + 1e-38)).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,N,d", [(8, 8, 22223, 128), (16, 8, 33335, 64)])
def test_large_inputs_as_small_ones(g, H, Hkv, N, d, dtype):
    """More than 128 MiB, which a wave walks through in another order: the bits of calls for a part of the tokens."""
    gen = torch.Generator(device=DEV).manual_seed(N)
    x = torch.randn(1, N, H + 2 * Hkv, d, device=DEV, generator=gen).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    assert x.numel() * x.element_size() > 128 << 20
    w = 1 + 0.3 * torch.randn(2, d, device=DEV, generator=gen)
    f = dev64(freq_of(d))
    for kw in (dict(freq=f, wq=w[0], wk=w[1]), dict(freq=f, norm=False, paired=True)):
        whole = g.gfwa_qk_norm_rope(q, k, v, **kw)
        for i in range(0, N, 5000):
            at = slice(i, min(i + 5000, N))
            pos = torch.arange(at.start, at.stop, dtype=torch.int32, device=DEV)[None]
            part = g.gfwa_qk_norm_rope(q[:, at], k[:, at], v[:, at], pos=pos, **kw)
            assert all(torch.equal(a[:, :, at], b) for a, b in zip(whole, part)), i


@pytest.mark.parametrize("H,Hkv,N,d", [(8, 8, 22223, 128), (16, 8, 33335, 64), (7, 7, 40001, 64), (5, 5, 20003, 128), (3, 1, 70007, 64), (5, 5, 13001, 128)])
def test_large_gradients_as_small_ones(g, H, Hkv, N, d):
    """The derivative of 45 to 137 MB of inputs: the bits of calls for a part of the tokens, and the weights' gradients to the tolerance of the small ones
    (no chain is longer: eight heads of a lane, five items of a wave; the rest in fp64)."""
    gen = torch.Generator(device=DEV).manual_seed(N)
    mk = lambda *s: torch.randn(s, device=DEV, generator=gen).bfloat16()
    x, dx = mk(1, N, H + 2 * Hkv, d), torch.zeros(1, N, H + 2 * Hkv, d, device=DEV, dtype=torch.bfloat16)
    assert x.numel() * 2 > 40 << 20
    parts = lambda t: (t[:, :, :H], t[:, :, H:H + Hkv], t[:, :, H + Hkv:])
    q, k, _ = parts(x)
    dQ, dK, dV = mk(1, H, N, d), mk(1, Hkv, N, d), mk(1, Hkv, N, d)
    w = 1 + 0.3 * torch.randn(2, d, device=DEV, generator=gen)
    f = dev64(freq_of(d))
    outs = parts(dx)
    dw = g.gfwa_qk_norm_rope_backward(q, k, dQ, dK, dV, w[0], w[1], EPS, f, dq=outs[0], dk=outs[1], dv=outs[2])[3:]
    for i in range(0, N, 6000):
        at = slice(i, min(i + 6000, N))
        pos = torch.arange(at.start, at.stop, dtype=torch.int32, device=DEV)[None]
        part = g.gfwa_qk_norm_rope_backward(q[:, at], k[:, at], *(t[:, :, at].contiguous() for t in (dQ, dK, dV)), w[0], w[1], EPS, f, pos=pos)
        assert all(torch.equal(a[:, at], b) for a, b in zip(outs, part)), i
    for i, (y, dy) in enumerate(((q, dQ), (k, dK))):
        y, back = y.double(), dy.double().transpose(1, 2)
        u = y * (y * y).mean(-1, keepdim=True).add(EPS).rsqrt()
        angle = torch.arange(N, device=DEV, dtype=torch.float64)[:, None] * f
        c, s = angle.cos()[None, :, None], angle.sin()[None, :, None]
        lo, hi = back[..., :d // 2], back[..., d // 2:]
        terms = torch.cat((lo * c + hi * s, hi * c - lo * s), -1) * u
        assert ((dw[i].double() - terms.sum((0, 1, 2))).abs() <= 160 * U * (torch.cat((lo.abs() + hi.abs(),) * 2, -1) * u.abs()).sum((0, 1, 2))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,N,d,rot,paired,norm,kind,pos_kind", ROPE)
def test_norm_and_rotation_backward(g, B, H, Hkv, N, d, rot, paired, norm, kind, pos_kind, dtype):
    print("rope bwd", B, H, Hkv, N, d, rot, paired, norm, kind, pos_kind, dtype, flush=True)
    rng, pos, pos_dev, (q, tq), (k, tk), (v, tv), (wq, twq), (wk, twk) = rope_inputs(B, H, Hkv, N, d, rot, kind, pos_kind, dtype)
    freq = freq_of(rot)
    dQ, tdQ = store(rng.standard_normal((B, H, N, d)), dtype)
    dK, tdK = store(rng.standard_normal((B, Hkv, N, d)), dtype)
    dV, tdV = store(rng.standard_normal((B, Hkv, N, d)), dtype)
    outs = [layout(np.zeros((B, N, h, d)), kind, dtype)[1] for h in (H, Hkv, Hkv)]
    bases = [t._base if t._base is not None else t for t in outs]
    poison = [b.isnan() for b in bases]
    args = (tq, tk, tdQ, tdK, tdV, twq if norm else None, twk if norm else None, EPS, dev64(freq), pos_dev)
    got = g.gfwa_qk_norm_rope_backward(*args, norm=norm, paired=paired, dq=outs[0], dk=outs[1], dv=outs[2])
    assert all(a is b for a, b in zip(got, outs))
    for b, n in zip(bases, poison):
        assert torch.equal(b.isnan(), n), "what lies between the rows was written"
    fresh = g.gfwa_qk_norm_rope_backward(*args, norm=norm, paired=paired)
    for a, b in zip(got, fresh):
        assert (a is None and b is None) or torch.equal(a, b), "two runs, or two layouts, differ"
    assert torch.equal(got[2], tdV.transpose(1, 2))
    if not norm:
        assert got[3] is None and got[4] is None
    for x, wt, dy, dx, dwt in ((q, wq, dQ, got[0], got[3]), (k, wk, dK, got[1], got[4])):
        dyt = dy.transpose(0, 2, 1, 3).astype(np.float64)
        ref, dref = ol.norm_rope_rows_backward(x, wt, EPS, norm, pos, freq, paired, dyt)
        off = 8 * U + (2.0 ** -51 * np.abs(pos).max() if rot else 0)
        if norm:
            x64 = x.astype(np.float64)
            r = ol._rms(x64, EPS)
            u = x64 * r
            gg = np.abs(ol.rotate(dyt, np.broadcast_to(pos[..., None], dyt.shape[:-1]), freq, paired, back=True))
            goff = off * pair_sums(dyt, rot, paired)
            mag = lambda a: r * (a * np.abs(wt) + np.abs(u) * np.mean(a * np.abs(wt * u), axis=-1, keepdims=True))
            tol = HALF[dtype] * np.abs(ref) + (64 * U * mag(gg) + mag(goff)) * (1 + HALF[dtype])
            derr = np.abs(host(dwt) - dref)
            dtol = 160 * U * (gg * np.abs(u)).reshape(-1, d).sum(0) + (goff * np.abs(u)).reshape(-1, d).sum(0)
            assert (derr <= dtol).all(), (derr / dtol).max()
        else:
            tol = HALF[dtype] * np.abs(ref) + off * pair_sums(dyt, rot, paired) * (1 + HALF[dtype])
        err = np.abs(host(dx) - ref)
        assert (err <= tol + 1e-38).all(), (err / (tol + 1e-38)).max()


def test_rope_without_values_or_weights(g):
    rng = np.random.default_rng(3)
    q, tq = store(rng.standard_normal((2, 19, 4, 64)), "f32")
    k, tk = store(rng.standard_normal((2, 19, 2, 64)), "f32")
    Q, K, V = g.gfwa_qk_norm_rope(tq, tk)
    one = torch.ones(64, device=DEV)
    Q1, K1, _ = g.gfwa_qk_norm_rope(tq, tk, wq=one, wk=one)
    assert V is None and torch.equal(Q, Q1) and torch.equal(K, K1)
    ref = ol.norm_rope_rows(q, None, EPS, True, 0, None, False)
    assert np.abs(host(Q.transpose(1, 2)) - ref).max() <= 32 * U * np.abs(ref).max()
    dq, dk, dv, dwq, dwk = g.gfwa_qk_norm_rope_backward(tq, tk, Q, K)
    assert dv is None and dwq is None and dwk is None
    dq2, dk2, _, dwq, dwk = g.gfwa_qk_norm_rope_backward(tq, tk, Q, K, dwk=torch.empty(64, device=DEV))
    assert dwq is None and torch.equal(dq, dq2) and torch.equal(dk, dk2)
    ref = (ol.norm_rope_rows(k, None, EPS, True, 0, None, False) ** 2).reshape(-1, 64).sum(0)
    assert np.abs(host(dwk) - ref).max() <= 256 * U * ref.max()


def test_rope_rows_of_zeros_and_infinities(g):
    # a row of zeros stays zero (eps > 0); an infinity spoils its own row alone, and without the norm only what it is mixed with
    x = np.ones((1, 4, 2, 64), dtype=np.float32)
    x[0, 1] = 0
    x[0, 2, 0, 40] = np.inf
    t = torch.from_numpy(x).to(DEV)
    f = dev64(freq_of(32))
    Q, K, _ = g.gfwa_qk_norm_rope(t, t, freq=f)
    assert (Q[0, :, 1] == 0).all() and not torch.isfinite(Q[0, 0, 2]).all()
    rest = [(0, 0), (0, 1), (0, 3), (1, 0), (1, 1), (1, 2), (1, 3)]
    assert all(torch.isfinite(Q[0, h, n]).all() for h, n in rest)
    Q, _, _ = g.gfwa_qk_norm_rope(t, t, freq=f, norm=False)
    assert Q[0, 0, 2, 40] == np.inf and torch.isfinite(Q[0, 0, 2, :40]).all() and (Q[0, 0, 2, 41:] == 1).all()
    dq, _, _, _, _ = g.gfwa_qk_norm_rope_backward(t, t, Q, Q, freq=f, norm=False)
    assert dq[0, 2, 0, 40] == np.inf and torch.isfinite(dq[0, 2, 0, :40]).all()


def test_rope_reads_broadcast_inputs(g):
    # one token, one head expanded over all (strides of zero); the gradient is per row, its sum is the shared row's
    x = torch.randn(1, 1, 1, 128, device=DEV)
    q, k = x.expand(2, 11, 4, 128), x.expand(2, 11, 2, 128)
    Q, K, V = g.gfwa_qk_norm_rope(q, k, k)
    Qd, Kd, Vd = g.gfwa_qk_norm_rope(q.contiguous(), k.contiguous(), k.contiguous())
    assert torch.equal(Q, Qd) and torch.equal(K, Kd) and torch.equal(V, Vd)
    with pytest.raises(g.GfwaError):
        g.gfwa_qk_norm_rope_backward(q, k, Q, K, dq=torch.empty(1, 1, 1, 128, device=DEV).expand(2, 11, 4, 128))


# ---- the paged cache

def paged_case(seed, lens, H, Hkv, d, page, dtype, M=None, missing=()):
    """Sequences (cached, new) of a batch on a shuffled cache of NaN whose cached prefixes are finite."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    M = M or max((a + b + page - 1) // page for a, b in lens) + 1
    pages = B * M + 2
    table = rng.permutation(pages)[:B * M].reshape(B, M).astype(np.int32)
    for b, i in missing:
        table[b, i] = rng.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
    cp = np.full((pages, H, page), np.nan, dtype=np.float32)
    Kp, Vp = (np.full((pages, Hkv, page, d), np.nan, dtype=np.float32) for _ in range(2))
    for b, (before, _) in enumerate(lens):
        c = np.zeros(H)
        for p in range(before):
            c = c + rng.random(H) * 0.2
            at = table[b, p // page]
            if 0 <= at < pages:
                cp[at, :, p % page] = c
                Kp[at, :, p % page], Vp[at, :, p % page] = rng.standard_normal((2, Hkv, d))
    return rng, table, Kp, Vp, cp


def gpu(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(TORCH[dtype])


# (cached, new) of each sequence, H, Hkv, d, page, rot, paired, norm, rows in front and behind, missing pages
APPEND = [
    ([(0, 1)], 1, 1, 64, 16, 64, False, True, 0, 0, ()), ([(31, 1)], 4, 1, 128, 16, 128, False, True, 0, 0, ()),
    ([(7, 1), (0, 1), (48, 1), (16, 1), (100, 1)], 8, 2, 128, 16, 128, False, True, 0, 0, ()),
    ([(0, 37), (50, 1), (3, 0), (95, 70), (0, 0)], 6, 3, 64, 48, 32, True, True, 0, 5, ()),
    ([(0, 300), (17, 211)], 4, 4, 128, 64, 64, False, True, 3, 13, ()),
    ([(5, 1)] * 70, 2, 1, 64, 16, 16, False, False, 0, 2, ()),
    ([(40, 60), (64, 30), (10, 80)], 8, 1, 64, 32, 0, False, True, 1, 1, ((0, 1), (0, 2), (1, 1), (2, 0))),
    ([(0, 1500), (2, 3)], 16, 2, 64, 128, 64, False, True, 0, 0, ()),
    ([(0, 0), (0, 0), (9, 2), (0, 0)], 3, 3, 128, 16, 128, True, True, 4, 4, ()),
    ([(0, 5)] * 9 + [(0, 3000)] + [(1, 1)] * 5, 2, 2, 64, 256, 64, False, True, 0, 7, ()),
    ([(40, 2600), (0, 1), (7, 511), (0, 0), (5, 513)], 9, 3, 64, 64, 0, False, False, 2, 3, ((0, 20),)),  # prefixes in segments
    ([(3, 40000)], 1, 1, 64, 512, 16, False, True, 0, 0, ()), ([(5, 0)] * 69 + [(9, 70)], 5, 5, 64, 16, 0, False, False, 0, 0, ()),
    ([(31, 8), (16, 9), (0, 7), (3, 64), (40, 65), (15, 1)], 9, 3, 64, 16, 32, False, True, 1, 0, ()), ([(9, 2)] * 40, 12, 4, 64, 16, 0, False, False, 0, 0, ()),
    ([(7, 129)] + [(2, 1)] * 150, 10, 5, 64, 64, 0, False, False, 0, 1, ()),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(g, case, dtype):
    lens, H, Hkv, d, page, rot, paired, norm, front, behind, missing = APPEND[case]
    print("append", case, dtype, flush=True)
    rng, table, Kp, Vp, cp = paged_case(case, lens, H, Hkv, d, page, dtype, missing=missing)
    new = np.array([n for _, n in lens])
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) + front
    rows = int(start[-1]) + behind
    cached = np.array([c for c, _ in lens], dtype=np.int32)
    q, k, v = (layout(rng.standard_normal((1, rows, h, d)), "packed", dtype) for h in (H, Hkv, Hkv))
    alpha = (rng.random((rows, H)) * 0.3).astype(np.float32)
    wq, wk = (1 + 0.3 * rng.standard_normal((2, d))).astype(np.float32)
    freq = freq_of(rot)
    (Kp, tK), (Vp, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    Q0, tQ = store(rng.standard_normal((rows, H, d)), dtype)
    out = g.gfwa_append_paged(k[1][0], v[1][0], tK, tV, gpu(start), gpu(cached), gpu(table), q=q[1][0], wq=gpu(wq) if norm else None,
                              wk=gpu(wk) if norm else None, eps=EPS, freq=dev64(freq), norm=norm, paired=paired, alpha=gpu(alpha), cp=tc, Q=tQ)
    assert out is tQ
    refs = [ol.append_paged(q[0][0], k[0][0], v[0][0], wq, wk, EPS, norm, f, paired, alpha, start, cached, table, Q0, Kp, Vp, cp) for f in (freq, None)]
    (Qr, Kr, Vr, cr), (Qn, Kn, _, _) = refs
    assert np.array_equal(host(tV), Vr, equal_nan=True), "values"
    for name, got, ref, plain, old in (("Q", tQ, Qr, Qn, Q0), ("K", tK, Kr, Kn, Kp)):
        got = host(got)
        same = (ref == old) | (np.isnan(ref) & np.isnan(old))
        assert np.array_equal(got[same], ref[same], equal_nan=True), name + ": what belongs to no new token has changed"
        tol = HALF[dtype] * np.abs(ref) + (32 * U + 2.0 ** -51 * (cached + new).max()) * pair_sums(plain, rot, paired) * (1 + HALF[dtype])
        bad = ~same & ~(np.abs(got - ref) <= tol)
        assert not bad.any(), (name, np.argwhere(bad)[:3])
    got = host(tc)
    assert np.array_equal(np.isnan(got), np.isnan(cr))
    fin = ~np.isnan(cr)
    assert (np.abs(got[fin] - cr[fin]) <= U * np.abs(cr[fin])).all()
    assert np.array_equal(got[~np.isnan(cp)], cp[~np.isnan(cp)].astype(np.float64)), "cached prefixes"


def test_append_variants(g):
    """Without queries, without a gate, a head-major gate, a fresh Q: the same bits."""
    lens = [(3, 40), (0, 9)]
    rng, table, Kp, Vp, cp = paged_case(5, lens, 4, 2, 64, 16, "bf16")
    start, cached = gpu(np.array([0, 40, 49], dtype=np.int32)), gpu(np.array([3, 0], dtype=np.int32))
    q, k, v = (store(rng.standard_normal((49, h, 64)), "bf16")[1] for h in (4, 2, 2))
    alpha = gpu(rng.random((49, 4)).astype(np.float32))
    state = lambda: (store(Kp, "bf16")[1], store(Vp, "bf16")[1], gpu(cp))
    same = lambda a, b: torch.equal(torch.nan_to_num(a.float(), nan=7e7), torch.nan_to_num(b.float(), nan=7e7))
    f = dev64(freq_of(64))
    K1, V1, c1 = state()
    Q1 = g.gfwa_append_paged(k, v, K1, V1, start, cached, gpu(table), q=q, freq=f, alpha=alpha, cp=c1)
    K2, V2, c2 = state()
    assert g.gfwa_append_paged(k, v, K2, V2, start, cached, gpu(table), freq=f) is None
    assert same(K1, K2) and same(V1, V2) and same(c2, gpu(cp))
    K3, V3, c3 = state()
    Q3 = g.gfwa_append_paged(k, v, K3, V3, start, cached, gpu(table), q=q, freq=f, alpha=alpha.t().contiguous().t(), cp=c3)
    assert same(Q1, Q3) and same(K1, K3) and same(c1, c3)
    K4, V4, c4 = state()
    assert g.gfwa_append_paged(k, v, K4, V4, start, cached, gpu(table), freq=f, alpha=alpha, cp=c4) is None and same(c1, c4)


def test_append_survives_bad_offsets(g):
    """Offsets and lengths a caller must not give: nothing is written outside the cache, whatever else comes out."""
    rng, table, Kp, Vp, cp = paged_case(6, [(0, 8)] * 4, 2, 1, 64, 16, "f32")
    k, v, q = (store(rng.standard_normal((32, h, 64)), "f32")[1] for h in (1, 1, 2))
    alpha = gpu(rng.random((32, 2)).astype(np.float32))
    for start, cached in (([0, 40, 99, -5, 7], [0, 0, 0, 0]), ([9, 8, 7, 6, 5], [0, 1, 2, 3]), ([0, 8, 16, 24, 32], [-1, 10 ** 9, 2 ** 31 - 1, -2 ** 31]),
                          ([-100, -50, 0, 16, 10 ** 9], [5, 5, 5, 5])):
        bufs = []
        for x in (Kp, Vp, cp):
            b = torch.full((x.size + 8192,), 3.25, device=DEV)
            b[4096:-4096] = gpu(x).flatten()
            bufs.append(b)
        tK, tV, tc = (b[4096:-4096].view(x.shape) for b, x in zip(bufs, (Kp, Vp, cp)))
        g.gfwa_append_paged(k, v, tK, tV, gpu(np.array(start, dtype=np.int32)), gpu(np.array(cached, dtype=np.int32)), gpu(table), q=q, alpha=alpha, cp=tc)
        torch.cuda.synchronize()
        for b in bufs:
            assert (b[:4096] == 3.25).all() and (b[-4096:] == 3.25).all()


# positions (-1: no sequence), H, Hkv, d, page, w, missing pages, spare columns of the table
DECODE = [
    ([0], 1, 1, 64, 16, 1, ()), ([0, 1, 15, 16, 17], 4, 2, 128, 16, 5, ()), ([299, 3, 120], 8, 2, 128, 16, 64, ()),
    ([999, -1, 57, 500], 4, 1, 64, 48, 333, ()), ([776, 100, 5, 31], 6, 3, 64, 32, 2000, ()), ([1499, 1023], 3, 3, 128, 64, 1024, ()),
    ([2098, 1, 700, -1, 2047], 16, 4, 128, 128, 1024, ()), ([599, 256], 8, 8, 64, 16, 257, ()),
    ([300, 200, 100], 16, 2, 128, 16, 250, ((0, 0), (0, 5), (0, 12), (1, 12), (2, 2), (2, 3))),  # the second one's own page is missing
    ([700, 650], 32, 2, 64, 32, 1 << 30, ((0, 3), (0, 20))), ([5000], 20, 1, 128, 256, 4097, ()), ([130] * 40, 40, 2, 64, 16, 70, ()),
    ([90, 35, 64], 51, 3, 128, 16, 40, ()),
]


def decode_check(g, dtype, q, tq, Kp, Vp, cp, tK, tV, tc, table, pos, w, **kw):
    d = q.shape[-1]
    scale = d ** -0.5
    o, L = g.gfwa_decode_paged(tq, tK, tV, tc, gpu(table), gpu(np.array(pos, dtype=np.int32)), w, scale, **kw)
    o_ref, L_ref, absv, dots, top, count = ol.decode_paged(q, Kp, Vp, cp, table, pos, w, scale, detail=True)
    E = ((d + 8) * dots + 8 * top) * U
    n = count[:, None]
    rel = 2 * E + (n + 16) * U
    tol = HALF[dtype] * np.abs(o_ref) + (rel + (2.0 ** -15 if dtype == "bf16" else 0))[..., None] * absv
    with np.errstate(invalid="ignore"):  # empty rows: minus infinity on both sides
        err, lerr = np.abs(host(o) - o_ref), host(L) - L_ref
    empty = np.isinf(L_ref)
    assert np.array_equal(np.isinf(host(L)), empty) and (host(o)[empty] == 0).all()
    assert (err <= tol + 1e-30).all(), (err / (tol + 1e-30)).max()
    ltol = E + (n + 16) * U + 8 * U * np.abs(np.where(empty, 0, L_ref))
    lerr[empty] = 0
    assert (np.abs(lerr) <= ltol).all(), (np.abs(lerr) / ltol).max()
    return o, L


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(g, case, dtype):
    pos, H, Hkv, d, page, w, missing = DECODE[case]
    print("decode", case, dtype, flush=True)
    # slots that hold no token, and those in front of the window, are NaN
    rng, table, Kp, Vp, cp = paged_case(case, [(p + 1, 0) for p in pos], H, Hkv, d, page, dtype, missing=missing)
    for b, p in enumerate(pos):
        for i in range(max(0, p - w + 1)):
            if 0 <= table[b, i // page] < len(Kp):
                Kp[table[b, i // page], :, i % page] = Vp[table[b, i // page], :, i % page] = cp[table[b, i // page], :, i % page] = np.nan
    q, tq = store(rng.standard_normal((len(pos), H, d)), dtype)
    (Kp, tK), (Vp, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    o, L = decode_check(g, dtype, q, tq, Kp, Vp, cp, tK, tV, tc, table, pos, w)
    o2, L2 = g.gfwa_decode_paged(tq, tK, tV, tc, gpu(table), gpu(np.array(pos, dtype=np.int32)), w, d ** -0.5)
    assert torch.equal(o, o2) and torch.equal(L, L2), "two runs differ"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,d,T,w", [(3, 8, 2, 128, 600, 300), (2, 4, 4, 64, 333, 1 << 20), (40, 8, 1, 64, 200, 70), (300, 16, 2, 64, 90, 50)])
def test_decode_agrees_with_the_dense_cache(g, B, H, Hkv, d, T, w, dtype):
    page = 16
    rng, table, Kp, Vp, cp = paged_case(1, [(T, 0)] * B, H, Hkv, d, page, dtype)
    q, tq = store(rng.standard_normal((B, H, d)), dtype)
    tK, tV, tc = store(Kp, dtype)[1], store(Vp, dtype)[1], gpu(cp)
    rows = gpu(table).long()
    dense = lambda x: x[rows].transpose(1, 2).flatten(2, 3)[:, :, :T].contiguous()
    pos = torch.randint(0, T, (B,), dtype=torch.int32, device=DEV)
    o, L = g.gfwa_decode_paged(tq, tK, tV, tc, gpu(table), pos, w, d ** -0.5)
    o1, L1 = g.gfwa_decode(tq, dense(tK), dense(tV), dense(tc), pos, w, d ** -0.5)
    # both are off by the bounds of their tests: the outputs are averages of values of magnitude below 6
    assert (o.float() - o1.float()).abs().max() <= 6 * (4 * HALF["bf16"] if dtype == "bf16" else 2000 * U)
    assert (L - L1).abs().max() <= 1e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(4, 4), (8, 2), (16, 1)])
def test_decode_masked_keys_and_scores_far_apart(g, H, Hkv, dtype):
    """Keys of the type's lowest value score minus infinity, wherever they stand: no weight, and where they are all of the window an empty row; one key far
    above the rest; values of infinity under a weight of zero stay out where the key is outside the window."""
    T, page, d, w = 300, 16, 128, 200
    rng, table, Kp, Vp, cp = paged_case(2, [(T, 0)] * 2, H, Hkv, d, page, dtype)
    q, tq = store(np.concatenate([np.full((2, H, 1), 12.0), rng.standard_normal((2, H, d - 1))], -1), dtype)
    back = T - 1 - np.arange(T)
    at = lambda x, b, mask: (table[b][np.flatnonzero(mask) // page], slice(None), np.flatnonzero(mask) % page)
    low = torch.finfo(TORCH[dtype]).min
    for name, mask in (("two of three", back % 3 != 1), ("newest", back < 40), ("oldest", back >= 100), ("all but one", back != 77), ("all", back >= 0)):
        K1 = Kp.copy()
        for b in range(2):
            K1[at(K1, b, mask) + (0,)] = low
        K1, tK1 = store(K1, dtype)
        assert np.nanmin(K1) < -3e38
        print("  masked:", name, flush=True)
        if name == "all":
            o, L = g.gfwa_decode_paged(tq, tK1, store(Vp, dtype)[1], gpu(cp), gpu(table), torch.full((2,), T - 1, dtype=torch.int32, device=DEV), w, 1e3)
            assert (o == 0).all() and (L == -np.inf).all()
            continue
        # 1e-5 of the scores of masked keys is far below any weight; the oracle's scores are finite in fp64
        o, L = g.gfwa_decode_paged(tq, tK1, store(Vp, dtype)[1], gpu(cp), gpu(table), torch.full((2,), T - 1, dtype=torch.int32, device=DEV), w, d ** -0.5)
        o_ref, L_ref = ol.decode_paged(q, K1, store(Vp, dtype)[0], cp, table, [T - 1] * 2, w, d ** -0.5)
        assert np.abs(host(o) - o_ref).max() <= 6 * (3 * HALF["bf16"] if dtype == "bf16" else 2000 * U)
        assert np.abs(host(L) - L_ref).max() <= 1e-3
    # queries and keys of large norm: a score hundreds above all others, in the middle of the window
    Kp2 = 4 * Kp
    for b in range(2):
        Kp2[table[b, (T - 90) // page], :, (T - 90) % page] = 4 * q[b, ::H // Hkv]
    Kp2, tK2 = store(Kp2, dtype)
    Vp2, tV2 = store(Vp, dtype)
    decode_check(g, dtype, q, tq, Kp2, Vp2, cp, tK2, tV2, gpu(cp), table, [T - 1] * 2, w)
    # infinities and NaN next to the window, in its first and last page
    K3, V3 = Kp.copy(), Vp.copy()
    outside = (np.arange(T) > T - 5) | (np.arange(T) < T - 5 - w + 1)
    for b in range(2):
        V3[at(V3, b, outside)] = np.inf
        K3[at(K3, b, outside)] = np.nan
    (K3, tK3), (V3, tV3) = store(K3, dtype), store(V3, dtype)
    decode_check(g, dtype, q, tq, K3, V3, cp, tK3, tV3, gpu(cp), table, [T - 5] * 2, w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 2500])
def test_decode_masked_keys_with_finite_scores(g, T, dtype):
    """Where every key holds the type's lowest value and the query little there, scores are of the order of -1e37, all equal in 32 bits: weights
    are even, not none.  With one key unmasked it has all the weight."""
    H, Hkv, page, d = 4, 2, 16, 64
    rng, table, Kp, Vp, cp = paged_case(7, [(T, 0)], H, Hkv, d, page, dtype)
    q, tq = store(np.concatenate([np.full((1, H, 1), 0.25), rng.standard_normal((1, H, d - 1))], -1), dtype)
    low = torch.finfo(TORCH[dtype]).min
    Kp[..., 0] = np.where(np.isnan(Kp[..., 0]), np.nan, low)
    (K1, tK), (V1, tV) = store(Kp, dtype), store(Vp, dtype)
    pos = torch.tensor([T - 1], dtype=torch.int32, device=DEV)
    o, L = g.gfwa_decode_paged(tq, tK, tV, gpu(cp), gpu(table), pos, 1 << 30, 0.125)
    i = np.arange(T)
    V = V1[table[0, i // page], :, i % page].astype(np.float64)
    mean = np.repeat(V.mean(0), H // Hkv, 0)
    # even weights: sums of T terms and the rounding of the result, in bf16 of the weights too (1 is exact in it)
    assert (np.abs(host(o)[0] - mean) <= HALF[dtype] * np.abs(mean) + (T + 16) * U * np.abs(V).mean(0).max()).all()
    assert np.allclose(host(L), 0.125 * 0.25 * float(low), rtol=1e-6)
    Kp[table[0, 3 // page], :, 3 % page, 0] = 0.0
    o, L = g.gfwa_decode_paged(tq, store(Kp, dtype)[1], tV, gpu(cp), gpu(table), pos, 1 << 30, 0.125)
    one = np.repeat(V[3], H // Hkv, 0)
    assert (np.abs(host(o)[0] - one) <= HALF[dtype] * np.abs(one)).all() and np.isfinite(host(L)).all() and (host(L) > -1e6).all()


def test_decode_clamps_positions_past_the_table(g):
    rng, table, Kp, Vp, cp = paged_case(3, [(64, 0)] * 3, 4, 2, 64, 16, "bf16", M=4)
    q, tq = store(rng.standard_normal((3, 4, 64)), "bf16")
    args = (tq, store(Kp, "bf16")[1], store(Vp, "bf16")[1], gpu(cp), gpu(table))
    o1, L1 = g.gfwa_decode_paged(*args, gpu(np.array([64, 2 ** 31 - 1, 63], dtype=np.int32)), 30, 0.125)
    o2, L2 = g.gfwa_decode_paged(*args, gpu(np.array([63, 63, 63], dtype=np.int32)), 30, 0.125)
    assert torch.equal(o1, o2) and torch.equal(L1, L2)
    o, L = g.gfwa_decode_paged(*args, gpu(np.array([-1, -2 ** 31, -7], dtype=np.int32)), 30, 0.125)
    assert (o == 0).all() and (L == -np.inf).all()


def test_caches_beyond_32_bit_offsets(g):
    """The last pages of caches of more than 2^31 elements."""
    Hkv, H, page, d = 8, 16, 256, 128
    pages = (1 << 31) // (Hkv * page * d) + 5
    Kp, Vp = (torch.empty((pages, Hkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cp = torch.empty((pages, H, page), device=DEV)
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device=DEV)
    small = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    Ks, Vs, cs = torch.empty_like(Kp[:2]), torch.empty_like(Vp[:2]), torch.empty_like(cp[:2])
    n = 400
    q, k, v = (torch.randn((n, h, d), device=DEV).bfloat16() for h in (H, Hkv, Hkv))
    alpha = torch.rand((n, H), device=DEV)
    start, cached = torch.tensor([0, n], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    pos = torch.tensor([n - 1], dtype=torch.int32, device=DEV)
    outs = []
    for K, V, c, tab in ((Kp, Vp, cp, table), (Ks, Vs, cs, small)):
        Q = g.gfwa_append_paged(k, v, K, V, start, cached, tab, q=q, alpha=alpha, cp=c, freq=dev64(freq_of(128)))
        outs.append((Q,) + g.gfwa_decode_paged(Q[n - 1:], K, V, c, tab, pos, 300, 0.1))
    assert torch.isfinite(outs[0][1]).all()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_rows_beyond_32_bit_offsets(g):
    """Projections and head-major tensors of more than 2^31 elements: the last rows are those of a small call."""
    N, H, Hkv, d = 132000, 112, 8, 128
    x = torch.empty((1, N, H + 2 * Hkv, d), dtype=torch.bfloat16, device=DEV).normal_()
    assert x.numel() > 1 << 31
    wt, f = 1 + 0.1 * torch.randn(d, device=DEV), dev64(freq_of(d))
    split = lambda t: (t[:, :, :H], t[:, :, H:H + Hkv], t[:, :, H + Hkv:])
    pos = torch.arange(N, dtype=torch.int32, device=DEV)[None]
    Q, K, V = g.gfwa_qk_norm_rope(*split(x), wt, wt, freq=f)
    n = 100
    tail = x[:, -n:].contiguous()
    for a, b in zip((Q, K, V), g.gfwa_qk_norm_rope(*split(tail), wt, wt, freq=f, pos=pos[:, -n:].contiguous())):
        assert torch.equal(a[:, :, -n:], b)
    dx = torch.empty_like(x)
    dq, dk, dv = split(dx)
    g.gfwa_qk_norm_rope_backward(*split(x)[:2], Q, K, V, wt, wt, freq=f, dq=dq, dk=dk, dv=dv)
    got = g.gfwa_qk_norm_rope_backward(*split(tail)[:2], Q[:, :, -n:].contiguous(), K[:, :, -n:].contiguous(), V[:, :, -n:].contiguous(), wt, wt, freq=f,
                                       pos=pos[:, -n:].contiguous())
    for a, b in zip((dq, dk, dv), got):
        assert torch.equal(a[:, -n:], b)


def test_append_past_the_table_and_from_unaligned_vectors(g):
    """Positions that the table has no column for are not written, their queries are; vectors may start at any multiple of their own size."""
    lens = [(30, 20), (0, 40)]
    rng, table, Kp, Vp, cp = paged_case(8, lens, 4, 2, 64, 16, "f32", M=2)
    start, cached = np.array([0, 20, 60], dtype=np.int32), np.array([30, 0], dtype=np.int32)
    q, k, v = (store(rng.standard_normal((60, h, 64)), "f32") for h in (4, 2, 2))
    alpha = (rng.random((60, 4)) * 0.3).astype(np.float32)
    wt = (1 + 0.3 * rng.standard_normal(64)).astype(np.float32)

    def odd(x):  # the same values one element into a buffer
        b = torch.zeros(x.size + 1, dtype=torch.from_numpy(x).dtype, device=DEV)
        b[1:] = gpu(x).flatten()
        return b[1:].view(x.shape)

    tK, tV, tc, tQ = store(Kp, "f32")[1], store(Vp, "f32")[1], odd(cp), torch.zeros((60, 4, 64), device=DEV)
    freq = freq_of(64)
    g.gfwa_append_paged(k[1], v[1], tK, tV, odd(start), odd(cached), odd(table), q=q[1], wq=odd(wt), wk=odd(wt), eps=EPS, freq=odd(freq), alpha=odd(alpha),
                        cp=tc, Q=tQ)
    Qr, Kr, Vr, cr = ol.append_paged(q[0], k[0], v[0], wt, wt, EPS, True, freq, False, alpha, start, cached, table, np.zeros((60, 4, 64)), Kp, Vp, cp)
    for got, ref in ((tK, Kr), (tV, Vr), (tc, cr), (tQ, Qr)):
        got = host(got)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        fin = ~np.isnan(ref)
        assert (np.abs(got[fin] - ref[fin]) <= 128 * U * max(1, np.abs(ref[fin]).max())).all()
    pos = np.array([31, 31], dtype=np.int32)
    o, L = g.gfwa_decode_paged(tQ[[1, 51]].contiguous(), tK, tV, tc, odd(table), odd(pos), 20, 0.125)
    o1, L1 = g.gfwa_decode_paged(tQ[[1, 51]].contiguous(), tK, tV, tc.clone(), gpu(table), gpu(pos), 20, 0.125)
    assert torch.equal(o, o1) and torch.equal(L, L1) and torch.isfinite(o).all()


# ---- as they are used

def test_training_step_through_all(g, oracle):
    """Packed projection -> norm and rotation -> attention -> loss, and back down to the projection and the norm weights, against the same chain of
    oracles in fp64 (fp32 storage: a chain of four operators, each within 1e-4 of its own result)."""
    B, N, H, Hkv, d, w = 2, 75, 4, 2, 64, 33
    rng = np.random.default_rng(9)
    x = rng.standard_normal((B, N, H + 2 * Hkv, d)).astype(np.float32)
    alpha = (rng.random((B, H, N)) * 0.3).astype(np.float32)
    wq, wk = (1 + 0.2 * rng.standard_normal((2, d))).astype(np.float32)
    dO = rng.standard_normal((B, H, N, d)).astype(np.float32)
    freq, scale, pos = freq_of(d), d ** -0.5, np.broadcast_to(np.arange(N), (B, N))
    t = gpu(x)
    q, k, v = t[:, :, :H], t[:, :, H:H + Hkv], t[:, :, H + Hkv:]
    how = dict(wq=gpu(wq), wk=gpu(wk), eps=EPS, freq=dev64(freq))
    Q, K, V = g.gfwa_qk_norm_rope(q, k, v, **how)
    c = g.gfwa_gate_prefix(gpu(alpha))
    O, L = g.gfwa_forward_gqa(Q, K, V, c, w, scale)
    dQ, dK, dV, _ = g.gfwa_backward_gqa(Q, K, V, O, gpu(dO), c, L, w, scale)
    dt = torch.full_like(t, float("nan"))
    _, _, _, dwq, dwk = g.gfwa_qk_norm_rope_backward(q, k, dQ, dK, dV, dq=dt[:, :, :H], dk=dt[:, :, H:H + Hkv], dv=dt[:, :, H + Hkv:], **how)

    hm = lambda y: np.ascontiguousarray(y.transpose(0, 2, 1, 3), dtype=np.float64)
    xq, xk, xv = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    Qr, Kr = hm(ol.norm_rope_rows(xq, wq, EPS, True, pos, freq, False)), hm(ol.norm_rope_rows(xk, wk, EPS, True, pos, freq, False))
    cr = oracle.gate_prefix(alpha)
    gr = oracle.backward_gqa_from_c(Qr, Kr, hm(xv), cr, dO, w, scale)
    dxq, dwqr = ol.norm_rope_rows_backward(xq, wq, EPS, True, pos, freq, False, hm(gr["dQ"]))
    dxk, dwkr = ol.norm_rope_rows_backward(xk, wk, EPS, True, pos, freq, False, hm(gr["dK"]))
    ref = np.concatenate([dxq, dxk, hm(gr["dV"])], axis=2)
    close = lambda a, b: np.linalg.norm(host(a) - b) <= 4e-4 * np.linalg.norm(b)
    assert close(dt, ref) and close(dwq, dwqr) and close(dwk, dwkr)
    # ... and against differences of the GPU's own forward along a direction: the loss is <dO, O>
    dirx = rng.standard_normal(x.shape).astype(np.float32)

    def loss(s):
        y = gpu(x + np.float32(s) * dirx)
        Q1, K1, V1 = g.gfwa_qk_norm_rope(y[:, :, :H], y[:, :, H:H + Hkv], y[:, :, H + Hkv:], **how)
        return float((host(g.gfwa_forward_gqa(Q1, K1, V1, c, w, scale)[0]) * dO).sum())

    h = 2.0 ** -7  # h^2 times third derivatives of the loss's size, and 2^-20 of it over h
    slope = (loss(h) - loss(-h)) / (2 * h)
    size = np.linalg.norm(ref) * np.linalg.norm(dirx) / np.sqrt(ref.size)
    assert abs(slope - (host(dt) * dirx).sum()) <= 0.02 * size + 2e-4 * np.abs(host(O) * dO).sum()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("captured", [False, True])
def test_serving_run(g, oracle, captured, dtype):
    """Prompts of different lengths through norm and rotation, appended in two chunks, then tokens one by one (eagerly, or as one captured graph that is
    replayed), on a stream of its own; every step's output against the oracle's forward of the whole sequence."""
    H, Hkv, d, page, w, steps = 8, 2, 64, 16, 45, 6
    prompts = [70, 1, 33]
    B, M = len(prompts), 6
    rng = np.random.default_rng(12)
    total = [n + steps for n in prompts]
    x = [store(rng.standard_normal((n, H + 2 * Hkv, d)), dtype) for n in total]
    alpha = [(rng.random((n, H)) * 0.3).astype(np.float32) for n in total]
    wq, wk = (1 + 0.2 * rng.standard_normal((2, d))).astype(np.float32)
    freq, scale = freq_of(d), d ** -0.5
    how = dict(wq=gpu(wq), wk=gpu(wk), eps=EPS, freq=dev64(freq))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    pages = B * M
    Kp, Vp = (torch.full((pages, Hkv, page, d), float("nan"), dtype=TORCH[dtype], device=DEV) for _ in range(2))
    cp = torch.full((pages, H, page), float("nan"), device=DEV)
    table = gpu(rng.permutation(pages).reshape(B, M).astype(np.int32))
    split = lambda t: (t[..., :H, :], t[..., H:H + Hkv, :], t[..., H + Hkv:, :])
    refs = []
    for b in range(B):
        xq, xk, xv = split(x[b][0].astype(np.float64))
        pos = np.arange(total[b])
        Qr, Kr = ol.norm_rope_rows(xq, wq, EPS, True, pos, freq, False), ol.norm_rope_rows(xk, wk, EPS, True, pos, freq, False)
        hm = lambda y: np.ascontiguousarray(y.transpose(1, 0, 2))[None]
        refs.append(oracle.forward_gqa_from_c(hm(Qr), hm(Kr), hm(xv), oracle.gate_prefix(alpha[b].T[None].copy()), w, scale))
    # three operators' roundings to bf16 of queries, keys and weights: scores off by 2 * 2^-8 of sum|q||k| scale (about 5) at most
    bar = (0.15, 0.02) if dtype == "bf16" else (2e-4, 2e-5)

    def check(b, p, o):
        err = np.abs(host(o) - refs[b][0][0, :, p])
        assert err.max() <= bar[0] and err.mean() <= bar[1], (b, p, err.max(), err.mean())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = [n // 2 for n in prompts]
        done = [0] * B
        for chunk in (first, [n - f for n, f in zip(prompts, first)]):
            rows = torch.cat([x[b][1][done[b]:done[b] + chunk[b]] for b in range(B)])
            al = torch.cat([gpu(alpha[b][done[b]:done[b] + chunk[b]]) for b in range(B)])
            q, k, v = split(rows)
            start = np.concatenate([[0], np.cumsum(chunk)])
            Q = g.gfwa_append_paged(k, v, Kp, Vp, i32(start.tolist()), i32(done), table, q=q, alpha=al, cp=cp, **how)
            done = [a + b for a, b in zip(done, chunk)]
            last = [int(s) - 1 for s in start[1:]]
            o, L = g.gfwa_decode_paged(Q[[max(i, 0) for i in last]].contiguous(), Kp, Vp, cp, table, i32([n - 1 if c else -1 for n, c in zip(done, chunk)]), w, scale)
            for b in range(B):
                if chunk[b]:
                    check(b, done[b] - 1, o[b])
        # tokens: static buffers
        row, al, cached, pos = torch.empty_like(torch.stack([x[b][1][0] for b in range(B)])), torch.empty((B, H), device=DEV), i32(done), i32(done)
        start = i32(list(range(B + 1)))
        Q, o, L = torch.empty((B, H, d), dtype=TORCH[dtype], device=DEV), torch.empty((B, H, d), dtype=TORCH[dtype], device=DEV), torch.empty((B, H), device=DEV)
        ws = torch.empty(g.gfwa_decode_paged_workspace_bytes(B, H, Hkv, d, page, M, w), dtype=torch.uint8, device=DEV)

        def step():
            q, k, v = split(row)
            g.gfwa_append_paged(k, v, Kp, Vp, start, cached, table, q=q, alpha=al, cp=cp, Q=Q, **how)
            g.gfwa_decode_paged(Q, Kp, Vp, cp, table, pos, w, scale, o=o, L=L, workspace=ws)

        graph = None
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        for s in range(steps):
            for b in range(B):
                row[b].copy_(x[b][1][done[b]])
                al[b].copy_(gpu(alpha[b][done[b]]))
            cached.copy_(i32(done))
            pos.copy_(i32(done))
            graph.replay() if captured else step()
            for b in range(B):
                check(b, done[b], o[b])
            done = [n + 1 for n in done]
            torch.cuda.synchronize()


def test_two_streams_at_once(g):
    """Calls that share nothing but the library, on two streams: the results of each alone."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    mk = lambda *s: torch.randn(s, generator=gen, device=DEV).bfloat16()
    sets = []
    for n in (700, 900):
        q, k, v = mk(1, n, 8, 128), mk(1, n, 2, 128), mk(1, n, 2, 128)
        wt = torch.rand(128, generator=gen, device=DEV)
        sets.append((q, k, v, wt, mk(1, 8, n, 128), mk(1, 2, n, 128)))
    f = dev64(freq_of(128))

    def work(s):
        q, k, v, wt, dQ, dK = s
        return g.gfwa_qk_norm_rope(q, k, v, wt, wt, freq=f) + tuple(x for x in g.gfwa_qk_norm_rope_backward(q, k, dQ, dK, None, wt, wt, freq=f) if x is not None)

    alone = [work(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i].append(work(sets[i]))
    torch.cuda.synchronize()
    for a, many in zip(alone, outs):
        for got in many:
            assert all(torch.equal(x, y) for x, y in zip(a, got))


def test_bench_line_of_the_paged_step(g, capsys):
    import json
    import sys
    import bench
    argv, sys.argv = sys.argv, ["bench.py", "--decode", "3,8,2,700,64,100", "--paged", "16", "--steps", "3", "--warmup", "1"]
    try:
        assert bench.main() == 0
    finally:
        sys.argv = argv
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["unit"] == "GB/s" and line["value"] > 0 and line["steps"] == 3
    assert {"append_paged_ms", "decode_paged_partial_ms", "algorithmic_bytes", "tokens_per_s"} <= set(line["detail"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hkv,G,d", [(1, 2, 4, 128), (5, 1, 3, 64), (40, 8, 1, 64)])
def test_decode_short_sequences_in_a_long_table(g, B, Hkv, G, d, dtype):
    """Columns for 65536 positions, sequences of up to a few hundred: the steps of a table that just holds them, to the order of the sums."""
    page, H = 16, Hkv * G
    rng, table, Kp, Vp, cp = paged_case(11, [(int(n), 0) for n in np.random.default_rng(B).integers(1, 500, B)], H, Hkv, d, page, dtype)
    lens = [int((~np.isnan(cp[table[b], 0])).sum()) for b in range(B)]
    q, tq = store(rng.standard_normal((B, H, d)), dtype)
    (K1, tK), (V1, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    wide = np.full((B, 4096), -1, dtype=np.int32)
    wide[:, :table.shape[1]] = table
    pos = [n - 1 for n in lens]
    decode_check(g, dtype, q, tq, K1, V1, cp, tK, tV, tc, table, pos, 1 << 30)
    decode_check(g, dtype, q, tq, K1, V1, cp, tK, tV, tc, wide, pos, 1 << 30)
    # ... and one position at the far end among them: a window over the sequence's first tokens, seen there
    n = min(lens[0], 38)
    wide[0, -3:] = np.resize(table[0], 3)
    decode_check(g, dtype, q, tq, K1, V1, cp, tK, tV, tc, wide, [65536 - 48 + n - 1] + pos[1:], n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_training_step_and_prompt(g, dtype):
    """Norm and rotation, its derivative and the append of prompts (prefixes in segments) as one graph, replayed on other contents of the same tensors:
    the bits of eager calls each time."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=DEV).manual_seed(3)
    H, Hkv, N, d, page = 8, 2, 1300, 64, 32
    new = lambda *s: torch.empty(s, device=DEV, dtype=dt)
    x, dx, wt = new(1, N, H + 2 * Hkv, d), new(1, N, H + 2 * Hkv, d), torch.empty(2, d, device=DEV)
    grads = [new(1, h, N, d) for h in (H, Hkv, Hkv)]
    outs, Qn = [new(1, h, N, d) for h in (H, Hkv, Hkv)], new(N, H, d)
    dw = torch.empty(2, d, device=DEV)
    alpha = torch.empty(N, H, device=DEV)
    start, cached = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 1100, N], [5, 40]))
    table = torch.randperm(2 * 36, device=DEV, generator=gen).view(2, 36).int()
    cache = [torch.zeros(72, Hkv, page, d, device=DEV, dtype=dt), torch.zeros(72, Hkv, page, d, device=DEV, dtype=dt), torch.zeros(72, H, page, device=DEV)]
    ws = torch.empty(g.gfwa_qk_norm_rope_backward_workspace_bytes(1, H, Hkv, N, d), dtype=torch.uint8, device=DEV)
    f = dev64(freq_of(d))
    parts = lambda t: (t[..., :H, :], t[..., H:H + Hkv, :], t[..., H + Hkv:, :])

    def step():
        q, k, v = parts(x)
        dq, dk, dv = parts(dx)
        g.gfwa_qk_norm_rope(q, k, v, wt[0], wt[1], freq=f, Q=outs[0], K=outs[1], V=outs[2])
        g.gfwa_qk_norm_rope_backward(q, k, *grads, wt[0], wt[1], freq=f, dq=dq, dk=dk, dv=dv, dwq=dw[0], dwk=dw[1], workspace=ws)
        g.gfwa_append_paged(k[0], v[0], cache[0], cache[1], start, cached, table, q=q[0], wq=wt[0], wk=wt[1], freq=f, alpha=alpha, cp=cache[2], Q=Qn)

    written = [dx, dw, Qn, *outs, *cache]

    def refill(i):
        gen.manual_seed(100 + i)
        for t in [x, wt, *grads]:
            t.copy_(torch.randn(t.shape, device=DEV, generator=gen))
        alpha.copy_(torch.rand(alpha.shape, device=DEV, generator=gen))
        for t in cache:
            t.fill_(0.25)
        for t in written[:-3]:
            t.fill_(7.0)

    refill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        refill(i)
        step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in written]
        refill(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, written)), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_that_share_pages(g, dtype):
    """Three sequences on the same first pages, each appending to a page of its own, one of them twice in the batch of the step."""
    H, Hkv, d, page = 8, 2, 64, 16
    rng, table, Kp, Vp, cp = paged_case(21, [(48, 2), (48, 2), (48, 2)], H, Hkv, d, page, dtype)
    table[1:, :3] = table[0, :3]
    start, cached = np.array([0, 2, 4, 6], dtype=np.int32), np.full(3, 48, dtype=np.int32)
    q, k, v = (store(rng.standard_normal((6, h, d)), dtype) for h in (H, Hkv, Hkv))
    alpha = (rng.random((6, H)) * 0.3).astype(np.float32)
    (K1, tK), (V1, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    g.gfwa_append_paged(k[1], v[1], tK, tV, gpu(start), gpu(cached), gpu(table), norm=False, alpha=gpu(alpha), cp=tc)
    _, Kr, Vr, cr = ol.append_paged(q[0], k[0], v[0], None, None, EPS, False, None, False, alpha, start, cached, table, q[0], K1, V1, cp)
    assert np.array_equal(host(tK), Kr, equal_nan=True) and np.array_equal(host(tV), Vr, equal_nan=True)  # no arithmetic
    got = host(tc)
    fin = ~np.isnan(cr)
    assert np.array_equal(~np.isnan(got), fin) and (np.abs(got[fin] - cr[fin]) <= U * np.abs(cr[fin])).all()
    rows = [0, 1, 2, 1]
    qs, tq = store(rng.standard_normal((4, H, d)), dtype)
    decode_check(g, dtype, qs, tq, Kr, Vr, got.astype(np.float32), tK, tV, tc, table[rows], [49, 49, 49, 48], 30)
