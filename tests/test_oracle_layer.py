"""What pins the fp64 oracle of the operators around the attention: finite differences, invariances of the rotation, the dense decoding step."""
import numpy as np
import pytest

from oracle import layer as ol


def freqs(rot):
    return None if rot == 0 else 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("rot,paired", [(0, False), (16, False), (32, False), (32, True), (16, True)])
def test_gradient_matches_differences(rot, paired, norm):
    rng = np.random.default_rng(1)
    x, dy, dirx = (rng.standard_normal((2, 3, 32)) for _ in range(3))
    wt, dirw = rng.standard_normal(32), rng.standard_normal(32)
    pos = np.array([5, 77])
    f = lambda x, wt: (dy * ol.norm_rope_rows(x, wt, 1e-3, norm, pos, freqs(rot), paired)).sum()
    dx, dw = ol.norm_rope_rows_backward(x, wt, 1e-3, norm, pos, freqs(rot), paired, dy)
    h = 1e-5  # central differences: error of order h^2 times third derivatives of order ten, and 2^-52 / h
    assert abs((f(x + h * dirx, wt) - f(x - h * dirx, wt)) / (2 * h) - (dx * dirx).sum()) < 1e-7
    if norm:
        assert abs((f(x, wt + h * dirw) - f(x, wt - h * dirw)) / (2 * h) - (dw * dirw).sum()) < 1e-7
    else:
        assert dw is None


@pytest.mark.parametrize("paired", [False, True])
def test_rotation_depends_on_distance_alone(paired):
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal(64), rng.standard_normal(64)
    dot = lambda p, i: ol.rotate(q, p, freqs(64), paired) @ ol.rotate(k, i, freqs(64), paired)
    assert abs(dot(9, 4) - dot(1009, 1004)) < 1e-10
    assert abs(dot(3, 3) - q @ k) < 1e-12
    back = ol.rotate(ol.rotate(q, 7, freqs(64), paired), 7, freqs(64), paired, back=True)
    assert np.abs(back - q).max() < 1e-14


def test_rotation_pairs_are_the_documented_ones():
    x = np.zeros(32)
    x[1] = 1.0
    f = freqs(16)
    half, paired = ol.rotate(x, 3, f, False), ol.rotate(x, 3, f, True)
    assert np.flatnonzero(half).tolist() == [1, 9] and np.allclose(half[[1, 9]], [np.cos(3 * f[1]), np.sin(3 * f[1])])
    assert np.flatnonzero(paired).tolist() == [0, 1] and np.allclose(paired[[0, 1]], [-np.sin(3 * f[0]), np.cos(3 * f[0])])


def test_norm_gives_rows_of_unit_mean_square():
    x = np.random.default_rng(3).standard_normal((4, 64)) * 7
    y = ol.norm_rope_rows(x, None, 0.0, True, 0, None, False)
    assert np.allclose((y * y).mean(-1), 1.0, atol=1e-14)


@pytest.mark.parametrize("w", [1, 5, 40, 1000])
def test_paged_run_is_the_dense_step(oracle, w):
    """Tokens appended in two calls and read back through a shuffled table, against the dense cache."""
    rng = np.random.default_rng(4)
    B, H, Hkv, d, page, M = 3, 4, 2, 64, 16, 4
    lens = [(20, 17), (0, 33), (5, 0)]
    T = M * page
    K, V = rng.standard_normal((B, T, Hkv, d)), rng.standard_normal((B, T, Hkv, d))
    alpha = rng.random((B, T, H))
    table = rng.permutation(B * M + 2)[:B * M].reshape(B, M)
    Kp, Vp, cp = (np.full(s, np.nan) for s in ((B * M + 2, Hkv, page, d), (B * M + 2, Hkv, page, d), (B * M + 2, H, page)))
    cached = np.zeros(B, dtype=int)
    for step in range(2):
        new = np.array([l[step] for l in lens])
        start = np.concatenate([[0], np.cumsum(new)])
        rows = [(b, cached[b] + i) for b in range(B) for i in range(new[b])]
        pick = lambda x: np.stack([x[b, p] for b, p in rows])
        _, Kp, Vp, cp = ol.append_paged(None, pick(K), pick(V), None, None, 0.0, False, None, False, pick(alpha), start, cached, table, None, Kp, Vp, cp)
        cached = cached + new
    c = np.cumsum(alpha, axis=1).transpose(0, 2, 1)
    q = rng.standard_normal((B, H, d))
    o, L = ol.decode_paged(q, Kp, Vp, cp, table, cached - 1, w, 0.125)
    o_ref, L_ref = oracle.decode_from_c(q, K.transpose(0, 2, 1, 3).copy(), V.transpose(0, 2, 1, 3).copy(), c, cached - 1, w, 0.125)
    assert np.abs(o - o_ref).max() < 1e-12 and np.abs(L - L_ref).max() < 1e-12


def test_paged_slots_without_tokens():
    z = lambda *s: np.ones(s)
    table = np.array([[-1, 0], [0, -1], [7, 0]])
    o, L = ol.decode_paged(z(3, 2, 64), z(2, 1, 16, 64), z(2, 1, 16, 64), z(2, 2, 16), table, np.array([20, 20, -1]), 30, 1.0)
    assert np.allclose(o[0], 1.0) and np.allclose(L[0], 64 + np.log(5))  # its first page has left the window: five keys
    assert (o[1:] == 0).all() and (L[1:] == -np.inf).all()
