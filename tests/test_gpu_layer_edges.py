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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[9], [3, 5, 40], [700, 30], [20] + [1] * 40, [2] + [1] * 9, [2600, 1, 0, 77]])
@pytest.mark.parametrize("ahead", [1, 37])
def test_append_of_a_batch_that_begins_in_front_of_row_0(g, ahead, lens, dtype):
    """start[0] = -ahead: the first sequence's tokens in front of row 0 are not here, those from row 0 on stand `ahead` positions further on, and their
    prefix follows the cached one.  Keys, values and prefixes meet in the same slots; the last rows of the batch are not here either."""
    H, Hkv, d, page = 9, 3, 64, 16
    cached = [50] + [(7 * b) % 45 for b in range(1, len(lens))]
    rng, table, Kp, Vp, cp = paged_case(41, [(c + ahead * (b == 0), n) for b, (c, n) in enumerate(zip(cached, lens))], H, Hkv, d, page, dtype)
    for i in range(50, 50 + ahead):  # what stands in front of the first row is the prefix of position 49
        cp[table[0, i // page], :, i % page] = cp[table[0, 49 // page], :, 49 % page]
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    behind = min(2, lens[-1])
    rows = int(start[-1]) - behind
    there = np.minimum(start, rows)
    q, k, v = (store(rng.standard_normal((rows, h, d)), dtype) for h in (H, Hkv, Hkv))
    alpha = (rng.random((rows, H)) * 0.3).astype(np.float32)
    (Kp, tK), (Vp, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    Q0, tQ = store(rng.standard_normal((rows, H, d)), dtype)
    given = start.copy()
    given[0] -= ahead
    g.gfwa_append_paged(k[1], v[1], tK, tV, gpu(given), gpu(np.array(cached, dtype=np.int32)), gpu(table), q=q[1], norm=False, alpha=gpu(alpha), cp=tc, Q=tQ)
    cached[0] += ahead
    Qr, Kr, Vr, cr = ol.append_paged(q[0], k[0], v[0], None, None, EPS, False, None, False, alpha, there, cached, table, Q0, Kp, Vp, cp)
    for name, a, b in (("Q", tQ, Qr), ("K", tK, Kr), ("V", tV, Vr)):  # no arithmetic
        assert np.array_equal(host(a), b, equal_nan=True), name
    got = host(tc)
    assert np.array_equal(np.isnan(got), np.isnan(cr))
    fin = ~np.isnan(cr)
    assert (np.abs(got[fin] - cr[fin]) <= U * np.abs(cr[fin])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("paired", [False, True])
def test_append_rotates_queries_past_the_largest_position(g, paired, dtype):
    """Positions from 2^31 on are outside every table, but their queries are written, rotated by where they stand."""
    H, Hkv, d, page, n = 4, 2, 64, 16, 21
    rng, table, Kp, Vp, cp = paged_case(43, [(16, 0)], H, Hkv, d, page, dtype)
    cached = np.array([2 ** 31 - 10], dtype=np.int32)
    q, tq = store(rng.standard_normal((n, H, d)), dtype)
    (k, tk), (v, tv), tK, tV, tc = store(q[:, :Hkv], dtype), store(q[:, :Hkv], dtype), store(Kp, dtype)[1], store(Vp, dtype)[1], gpu(cp)
    before, freq = tK.clone(), freq_of(d)
    Q = g.gfwa_append_paged(tk, tv, tK, tV, gpu(np.array([0, n], dtype=np.int32)), gpu(cached), gpu(table), q=tq, freq=dev64(freq), norm=False, paired=paired,
                            alpha=gpu(np.ones((n, H), dtype=np.float32)), cp=tc)
    pos = 2 ** 31 - 10 + np.arange(n, dtype=np.int64)
    ref = ol.norm_rope_rows(q, None, EPS, False, pos, freq, paired)
    off = 32 * U + 2.0 ** -51 * pos.max()
    i, j = ol._pairs(d, d, paired)
    both = np.zeros(q.shape)
    both[..., i] = both[..., j] = np.abs(q[..., i]) + np.abs(q[..., j])
    assert (np.abs(host(Q) - ref) <= HALF[dtype] * np.abs(ref) + off * both * (1 + HALF[dtype])).all()
    assert np.array_equal(host(tK), host(before), equal_nan=True) and np.array_equal(host(tc), cp.astype(np.float64), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,N,d,rot", [(1, 1, 1, 1, 64, 64), (3, 6, 2, 77, 128, 32), (2, 4, 4, 9, 64, 0)])
def test_gradient_without_the_norm_needs_no_inputs(g, B, H, Hkv, N, d, rot, dtype):
    """norm=False reads neither q nor k: the same bits without them, or without one of them."""
    rng = np.random.default_rng(N)
    q, k = (store(rng.standard_normal((B, N, h, d)), dtype)[1] for h in (H, Hkv))
    grads = [store(rng.standard_normal((B, h, N, d)), dtype)[1] for h in (H, Hkv, Hkv)]
    f = dev64(freq_of(rot))
    want = g.gfwa_qk_norm_rope_backward(q, k, *grads, freq=f, norm=False)
    assert want[0].shape == q.shape and want[1].shape == want[2].shape == k.shape
    for a, b in ((None, None), (q, None), (None, k)):
        got = g.gfwa_qk_norm_rope_backward(a, b, *grads, freq=f, norm=False)
        assert all(torch.equal(x, y) for x, y in zip(got[:3], want[:3])) and got[3] is got[4] is None
    packed = torch.full((B, N, H + 2 * Hkv, d), float("nan"), dtype=TORCH[dtype], device=DEV)
    dq, dk, dv = packed[:, :, :H], packed[:, :, H:H + Hkv], packed[:, :, H + Hkv:]
    g.gfwa_qk_norm_rope_backward(None, None, *grads, freq=f, norm=False, dq=dq, dk=dk, dv=dv)
    assert all(torch.equal(x, y) for x, y in zip((dq, dk, dv), want))
    for bad in (dict(), dict(norm=True)):
        with pytest.raises(TypeError, match="q must be a tensor"):
            g.gfwa_qk_norm_rope_backward(None, k, *grads, **bad)
    with pytest.raises(ValueError, match="shape"):
        g.gfwa_qk_norm_rope_backward(None, None, grads[0], grads[1], grads[0][:, :, :, :32], norm=False)
    with pytest.raises(ValueError, match="shape"):
        g.gfwa_qk_norm_rope_backward(None, None, *grads, norm=False, dq=dq.transpose(1, 2) if H != N else dk[:, :, :0])


@pytest.mark.parametrize("shape,bound", [("40,32,8,2000,128,512", "hbm"), ("2,8,2,700,64,100", "cache")])
def test_bench_of_the_paged_step_reads_what_no_cache_holds(g, shape, bound, capsys):
    """A rate counts against the memory's only where more than twice the memory-side cache is read between two looks at a window."""
    import json
    import sys
    import bench
    argv, sys.argv = sys.argv, ["bench.py", "--decode", shape, "--paged", "16", "--steps", "20", "--warmup", "2"]
    try:
        assert bench.main() == 0
    finally:
        sys.argv = argv
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    between = line["detail"]["caches_in_turn"] * line["detail"]["algorithmic_bytes"]
    assert line["detail"]["caches_in_turn"] >= 2 and line["roofline"]["bound"] == bound and (between >= 512 << 20) == (bound == "hbm")
    assert line["value"] < line["roofline"]["peak"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_go_through_the_attention_and_into_the_cache(g, dtype):
    """A padded batch of prompts: norm and rotation, attention, append without queries; a second chunk of one sequence with a row of the decoding step for
    each of its tokens; then a token for each sequence.  Outputs against the attention over the whole sequences, the cache against K and V bit for bit."""
    B, N, H, Hkv, d, page, w, more = 2, 133, 8, 2, 64, 16, 60, 9
    lens = [133, 70]
    rng = np.random.default_rng(71)
    total = N + more + 1
    x, tx = store(rng.standard_normal((B, total, H + 2 * Hkv, d)), dtype)
    alpha = gpu((rng.random((B, total, H)) * 0.3).astype(np.float32))
    wt = gpu((1 + 0.2 * rng.standard_normal((2, d))).astype(np.float32))
    how, scale = dict(wq=wt[0], wk=wt[1], eps=EPS, freq=dev64(freq_of(d))), d ** -0.5
    split = lambda t: (t[..., :H, :], t[..., H:H + Hkv, :], t[..., H + Hkv:, :])
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    M = -(-total // page)
    table = gpu(rng.permutation(B * M).reshape(B, M).astype(np.int32))
    Kp, Vp = (torch.full((B * M, Hkv, page, d), float("nan"), dtype=TORCH[dtype], device=DEV) for _ in range(2))
    cp = torch.full((B * M, H, page), float("nan"), device=DEV)
    # the whole sequences at once; sequence 1 goes on from 70, so its rows there are the later tokens
    order = [list(range(total)), list(range(lens[1])) + list(range(N, total)) + list(range(lens[1], N))]
    whole = torch.stack([tx[b, order[b]] for b in range(B)])
    gates = torch.stack([alpha[b, order[b]] for b in range(B)])
    Q, K, V = g.gfwa_qk_norm_rope(*split(whole), **how)
    O, _ = g.gfwa_forward_gqa(Q, K, V, g.gfwa_gate_prefix(gates.transpose(1, 2).contiguous()), w, scale)
    # two roundings of one formula: scores and weights as in the tests of each
    bar = 2.0 ** -5 if dtype == "bf16" else 1e-4

    def check(b, p, o):
        assert (o.float() - O[b, :, p].float()).abs().max() <= bar, (b, p)

    prompt = tx[:, :N].contiguous()
    q, k, v = split(prompt)
    Q1, K1, V1 = g.gfwa_qk_norm_rope(q, k, v, **how)
    O1, _ = g.gfwa_forward_gqa(Q1, K1, V1, g.gfwa_gate_prefix(alpha[:, :N].transpose(1, 2).contiguous()), w, scale)
    for b in range(B):
        check(b, lens[b] - 1, O1[b, :, lens[b] - 1])
    append = lambda x, al, start, cached, tab, **kw: g.gfwa_append_paged(x[1], x[2], Kp, Vp, i32(start), i32(cached), tab, alpha=al, cp=cp, **kw)
    append(split(prompt.flatten(0, 1)), alpha[:, :N].reshape(B * N, H), [0, N, 2 * N], [0, 0], table, **how)
    slots = lambda b, n: (table[b].long()[torch.arange(n, device=DEV) // page], slice(None), torch.arange(n, device=DEV) % page)
    for b in range(B):
        assert torch.equal(Kp[slots(b, N)], K1[b].transpose(0, 1)) and torch.equal(Vp[slots(b, N)], V1[b].transpose(0, 1))
    # the same rows already normed and rotated, a sequence a call
    K2, V2, c2 = torch.zeros_like(Kp), torch.zeros_like(Vp), torch.zeros_like(cp)
    for b in range(B):
        g.gfwa_append_paged(K1[b].transpose(0, 1), V1[b].transpose(0, 1), K2, V2, i32([0, N]), i32([0]), table[b:b + 1].contiguous(), norm=False,
                            alpha=alpha[b, :N], cp=c2)
        assert all(torch.equal(y[slots(b, N)], z[slots(b, N)]) for y, z in ((Kp, K2), (Vp, V2), (cp, c2)))
    # nine more tokens of sequence 1, a row of the step for each
    rows = split(tx[1, N:N + more])
    Qc = append(rows, alpha[1, N:N + more], [0, more], [lens[1]], table[1:].contiguous(), q=rows[0], **how)
    o, _ = g.gfwa_decode_paged(Qc, Kp, Vp, cp, table[1:].expand(more, M).contiguous(), i32([lens[1] + i for i in range(more)]), w, scale)
    for i in range(more):
        check(1, lens[1] + i, o[i])
    lens = [N, lens[1] + more]
    # a token for each
    rows = split(torch.stack([tx[0, N], tx[1, N + more]]))
    Qt = append(rows, torch.stack([alpha[0, N], alpha[1, N + more]]), [0, 1, 2], lens, table, q=rows[0], **how)
    o, _ = g.gfwa_decode_paged(Qt, Kp, Vp, cp, table, i32(lens), w, scale)
    for b in range(B):
        check(b, lens[b], o[b])


def test_decode_windows_past_32_bits(g):
    """A window longer than any position holds every sequence, however long it is; none below one is taken."""
    rng, table, Kp, Vp, cp = paged_case(3, [(64, 0)], 4, 2, 64, 16, "bf16", M=4)
    args = store(rng.standard_normal((1, 4, 64)), "bf16")[1], store(Kp, "bf16")[1], store(Vp, "bf16")[1], gpu(cp), gpu(table), gpu(np.array([60], dtype=np.int32))
    want = g.gfwa_decode_paged(*args, 64, 0.125)
    for w in (2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, 2 ** 63, 2 ** 70 + 1):
        assert g.gfwa_decode_paged_workspace_bytes(1, 4, 2, 64, 16, 4, w) == g.gfwa_decode_paged_workspace_bytes(1, 4, 2, 64, 16, 4, 64) > 0
        assert all(torch.equal(a, b) for a, b in zip(g.gfwa_decode_paged(*args, w, 0.125), want)), w
    for w in (0, -1, -2 ** 32 + 7, -2 ** 70):
        assert g.gfwa_decode_paged_workspace_bytes(1, 4, 2, 64, 16, 4, w) == 0
        with pytest.raises(g.GfwaError):
            g.gfwa_decode_paged(*args, w, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_whose_squares_leave_32_bits(g, dtype):
    """Squares are taken in 32 bits: rows that overflow them come out as zeros, and so do their gradients; their neighbours do not change."""
    rng = np.random.default_rng(81)
    x = rng.standard_normal((1, 5, 2, 64))
    big = x.copy()
    big[0, 2, 1] = 1e20 * np.sign(x[0, 2, 1])
    (x, t), (big, tb) = store(x, dtype), store(big, dtype)
    f = dev64(freq_of(64))
    Q, K, _ = g.gfwa_qk_norm_rope(t, t, freq=f)
    Qb, _, _ = g.gfwa_qk_norm_rope(tb, t, freq=f)
    grads = g.gfwa_qk_norm_rope_backward(t, t, Q, K, freq=f)[0], g.gfwa_qk_norm_rope_backward(tb, t, Q, K, freq=f)[0]
    assert (Qb[0, 1, 2] == 0).all() and (grads[1][0, 2, 1] == 0).all()
    Qb[0, 1, 2], grads[1][0, 2, 1] = Q[0, 1, 2], grads[0][0, 2, 1]
    assert torch.equal(Q, Qb) and torch.equal(*grads)
