"""Calls of the operators around the attention at the edges of what include/gfwa_layer.h allows, on the GPU, against the fp64 oracle or against calls of
another form of the same kernel (bit for bit).  Tolerances as in test_gpu_layer.py unless a test derives its own."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from test_gpu_layer import DEV, EPS, HALF, TORCH, U, dev64, freq_of, g, gpu, host, paged_case, store  # noqa: F401 (g is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,w,H,Hkv,d", [(40, 40, 4, 2, 64), (700, 650, 8, 2, 128), (3000, 1 << 20, 16, 1, 64)])
@pytest.mark.parametrize("scores", ["even", "random", "faint"])
def test_decode_infinities_among_the_values(g, scores, T, w, H, Hkv, d, dtype):
    """An infinity in a column of a key that has any weight is that column's result, infinities of both signs give NaN, and no other column changes by a
    bit.  even: every weight is 1; faint: the infinities' keys weigh about 2^-122 beside the newest, among the smallest normal numbers of 32 bits.  A
    weight below those is zero in 32 bits, and zero times infinity NaN (random, 3000 keys: gates of 0.1 on average put the oldest e^-300 below the newest)."""
    page, p = 16, T - 1
    rng, table, Kp, Vp, cp = paged_case(31, [(T, 0)], H, Hkv, d, page, dtype)
    q, tq = store(rng.standard_normal((1, H, d)) * (scores == "random"), dtype)
    where = lambda i: (table[0, i // page], slice(None), i % page)
    keys = [p, p - 1, p - 17, max(0, p - w + 1)]  # the newest, its neighbour, another unit, the oldest of the window
    if scores == "faint":
        keys = keys[1:]
    if scores != "random":
        cp[~np.isnan(cp)] = 100.0
    if scores == "faint":
        for i in keys:
            cp[where(i)] = 100.0 - 122.3 * np.log(2.0)
    (_, tK), (Vn, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    V2 = Vp.copy()
    for n, i in enumerate(keys):
        V2[where(i) + (n,)] = np.inf
        V2[where(i) + (10 + n,)] = -np.inf
    V2[where(keys[0]) + (20,)], V2[where(keys[1]) + (20,)] = np.inf, -np.inf
    _, tV2 = store(V2, dtype)
    pos = torch.tensor([p], dtype=torch.int32, device=DEV)
    o, L = g.gfwa_decode_paged(tq, tK, tV, tc, gpu(table), pos, w, d ** -0.5)
    got, L2 = g.gfwa_decode_paged(tq, tK, tV2, tc, gpu(table), pos, w, d ** -0.5)
    want = o.clone()
    for n, i in enumerate(keys):
        want[..., n], want[..., 10 + n] = np.inf, -np.inf
        assert (scores, T, n) == ("random", 3000, 3) or (cp[where(p)] - cp[where(i)] < 86).all()
    if (scores, T) == ("random", 3000):
        assert (cp[where(p)] - cp[where(keys[3])] > 250).all() and got[..., [3, 13]].isnan().all()
        want[..., [3, 13]] = got[..., [3, 13]] = 0
    assert torch.isfinite(o).all() and torch.equal(L, L2)
    assert got[..., 20].isnan().all()
    want[..., 20] = got[..., 20] = 0
    assert torch.equal(got, want), (got != want).nonzero()[:5]
