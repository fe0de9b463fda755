"""Every variant of the kernels around the attention that a size may choose, against the same tokens in calls that take another one (bit for bit) or the
fp64 oracle; the profiler says which kernel a call ran."""
import numpy as np
import pytest
import torch

from test_gpu_layer import DEV, TORCH, U, decode_check, dev64, freq_of, g, gpu, paged_case, store  # noqa: F401 (g is a fixture)

pytestmark = pytest.mark.gpu


def kernels(call):
    """Names of the library's kernels that `call` runs, as the profiler gives them."""
    torch.cuda.synchronize()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    return " ".join(e.key for e in prof.key_averages() if "gfwa" in e.key)


def variant(kernel, dtype, *args):
    """A kernel's name with its template arguments: names with bf16 in them come mangled."""
    if dtype == "f32":
        return "%s<float, %s>" % (kernel, ", ".join(str(a).lower() for a in args))
    return kernel + "IDF16b" + "".join(("Lb%dE" if isinstance(a, bool) else "Li%dE") % a for a in args) + "EE"


def normal(seed, shape, dtype="bf16"):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(TORCH[dtype])


@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("lens,H,Hkv,d,page,rot,paired", [
    ([5003, 0, 1, 3990, 97], 10, 5, 128, 64, 128, False), ([22003, 77, 0, 1], 9, 3, 64, 48, 32, True), ([2000] * 9 + [4099], 8, 4, 64, 16, 64, False),
    ([1, 1, 9120], 7, 7, 128, 128, 0, False)])
def test_append_of_many_tokens(g, lens, H, Hkv, d, page, rot, paired, with_q):
    """More than 40 MiB of rows, read past the caches and at d = 64 two rows by the lanes of both: queries, keys and values as calls for a few thousand
    tokens each write them, with padding in front and behind, a missing page, and every other slot of the cache as it was."""
    front, behind, B = 3, 61, len(lens)
    if not with_q:  # what a call without queries reads is its keys and values
        lens = [n * (H + 2 * Hkv) // (2 * Hkv) + n % 2 for n in lens]
    cached = [(31 * b + 5) % 200 for b in range(B)]
    start = front + np.concatenate([[0], np.cumsum(lens)])
    rows = int(start[-1]) + behind
    assert rows * ((H if with_q else 0) + 2 * Hkv) * d * 2 > 40 << 20
    M = max((c + n + page - 1) // page for c, n in zip(cached, lens)) + 1
    gen = torch.Generator(device=DEV).manual_seed(rows)
    table = torch.randperm(B * M + 1, device=DEV, generator=gen)[:B * M].view(B, M).int()
    table[0, 3] = -1
    x = normal(1, (rows, H + 2 * Hkv, d))
    q, k, v = x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]
    alpha = torch.rand((rows, H), device=DEV, generator=gen)
    w = 1 + 0.3 * torch.randn(2, d, device=DEV, generator=gen)
    i32 = lambda y: torch.tensor(np.asarray(y), dtype=torch.int32, device=DEV)
    fresh = lambda: [normal(7, (B * M + 1, Hkv, page, d)), normal(8, (B * M + 1, Hkv, page, d)), normal(9, (rows, H, d)),
                     torch.zeros((B * M + 1, H, page), device=DEV)]

    def append(state, first, last, c, tab, at, gate):  # rows first .. last of the batch
        K, V, Q, cp = state
        part = slice(first, last)
        g.gfwa_append_paged(k[part], v[part], K, V, i32(at), i32(c), tab, q=q[part] if with_q else None, wq=w[0] if with_q else None, wk=w[1],
                            freq=dev64(freq_of(rot)), paired=paired, alpha=alpha[part] if gate else None, cp=cp if gate else None,
                            Q=Q[part] if with_q else None)

    whole, parts = fresh(), fresh()
    names = kernels(lambda: append(whole, 0, rows, cached, table, start, True))
    assert variant("append_paged_kernel", "bf16", d, True) in names, names
    step = 2900
    for b, n in enumerate(lens):
        for done in range(0, n, step):
            first = int(start[b]) + done
            m = min(step, n - done)
            append(parts, first, first + m, [cached[b] + done], table[b:b + 1].contiguous(), [0, m], False)
    small = kernels(lambda: append(fresh(), 0, 2900, [0], table[:1].contiguous(), [0, 7], False))
    assert variant("append_paged_kernel", "bf16", d, False) in small, small
    for name, a, b in zip("KVQ", whole, parts):
        assert torch.equal(a, b), (name, (a != b).nonzero()[:4])
    if with_q:
        assert torch.equal(whole[2][:front], normal(9, (rows, H, d))[:front]) and torch.equal(whole[2][rows - behind:], normal(9, (rows, H, d))[rows - behind:])
    # prefixes: c of the cached tokens is zero; fp64 sums rounded once
    cp = whole[3].double()
    written = torch.zeros(cp[:, 0].shape, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        p = cached[b] + torch.arange(n, device=DEV)
        sums = alpha[int(start[b]):int(start[b]) + n].double().cumsum(0)
        page_id = table[b][p // page].long()
        here = page_id >= 0
        got = cp[page_id[here], :, (p % page)[here]]
        assert ((got - sums[here]).abs() <= (U + 2.0 ** -50 * n) * sums[here]).all()
        written[page_id[here], (p % page)[here]] = True
    assert (cp.transpose(1, 2)[~written] == 0).all()


@pytest.mark.parametrize("H,Hkv,N,d,sides", [(7, 7, 40001, 64, 2), (5, 5, 20003, 128, 4), (12, 4, 27001, 128, 4), (6, 3, 90001, 64, 2), (3, 1, 66000, 128, 4)])
def test_rope_past_the_caches(g, H, Hkv, N, d, sides):
    """Norm and rotation of 70 to 140 MB of bf16 by waves that take two or four heads side by side: the bits of calls for a part of the tokens."""
    x = normal(N, (1, N, H + 2 * Hkv, d))
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    w = 1 + 0.3 * normal(3, (2, d), "f32")
    f = dev64(freq_of(d))
    for kw in (dict(freq=f, wq=w[0], wk=w[1]), dict(freq=f, norm=False, paired=True)):
        outs = []
        names = kernels(lambda: outs.extend(g.gfwa_qk_norm_rope(q, k, v, **kw)))
        assert variant("qk_norm_rope_kernel", "bf16", d, True, sides) in names, names
        for i in range(0, N, 6000):
            at = slice(i, min(i + 6000, N))
            pos = torch.arange(at.start, at.stop, dtype=torch.int32, device=DEV)[None]
            part = g.gfwa_qk_norm_rope(q[:, at], k[:, at], v[:, at], pos=pos, **kw)
            assert all(torch.equal(a[:, :, at], b) for a, b in zip(outs, part)), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,d,T,w", [(32, 16, 8, 128, 1100, 1000), (43, 12, 6, 64, 1000, 900)])
def test_decode_by_eight_waves_past_the_caches(g, B, H, Hkv, d, T, w, dtype):
    """256 to 511 windows of one length and of more than 24 MiB in all: workgroups of eight waves, values past the caches."""
    page = 16
    rng, table, Kp, Vp, cp = paged_case(B, [(T, 0)] * B, H, Hkv, d, page, dtype)
    q, tq = store(rng.standard_normal((B, H, d)), dtype)
    (Kp, tK), (Vp, tV), tc = store(Kp, dtype), store(Vp, dtype), gpu(cp)
    pos = [T - 1 - 3 * b for b in range(B)]
    pos[7] = -1
    call = lambda: decode_check(g, dtype, q, tq, Kp, Vp, cp, tK, tV, tc, table, pos, w)
    names = kernels(call)
    assert variant("decode_paged_kernel", dtype, d, 8, True) in names and "combine" not in names, names


@pytest.mark.parametrize("H,Hkv,N,d", [(4, 2, 37, 64), (8, 2, 3000, 128), (7, 7, 40001, 64)])
def test_weights_gradients_to_their_own_chain(g, H, Hkv, N, d):
    """What is summed in 32 bits is a lane's rows, with one rounding more for a workgroup's sum and one for the result: with r rows to a lane and terms off
    by 32 u, r + 34 u of the sum of magnitudes, and 8 u of the pair's for the rotation.  Rows of a lane, over all its tiles: at most 16 here."""
    q, k = normal(1, (1, N, H, d)), normal(2, (1, N, Hkv, d))
    dQ, dK = normal(3, (1, H, N, d)), normal(4, (1, Hkv, N, d))
    w = 1 + 0.3 * normal(5, (2, d), "f32")
    f = dev64(freq_of(d))
    dw = g.gfwa_qk_norm_rope_backward(q, k, dQ, dK, None, w[0], w[1], freq=f)[3:]
    angle = torch.arange(N, device=DEV, dtype=torch.float64)[:, None] * f
    c, s = angle.cos()[None, :, None], angle.sin()[None, :, None]
    for got, x, dy in zip(dw, (q, k), (dQ, dK)):
        x, dy = x.double(), dy.double().transpose(1, 2)
        u = x * ((x * x).mean(-1, keepdim=True) + 1e-6).rsqrt()
        lo, hi = dy[..., :d // 2], dy[..., d // 2:]
        terms = torch.cat((lo * c + hi * s, hi * c - lo * s), -1) * u
        both = torch.cat((lo.abs() + hi.abs(),) * 2, -1) * u.abs()
        assert ((got.double() - terms.sum((0, 1, 2))).abs() <= U * ((16 + 34) * terms.abs() + 8 * both).sum((0, 1, 2))).all()


def test_sizes_count_what_is_read(g):
    """Keys alone, or without values: 34 MB are read of a projection of 50 MB, which the caches hold.  The same bits as with queries, or values."""
    H, Hkv, N, d, page = 16, 16, 4100, 128, 64
    x, f = normal(1, (1, N, H + 2 * Hkv, d)), dev64(freq_of(d))
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    outs = []
    names = kernels(lambda: outs.extend((g.gfwa_qk_norm_rope(q, k, v, freq=f), g.gfwa_qk_norm_rope(q, k, freq=f))))
    assert all(variant("qk_norm_rope_kernel", "bf16", d, once, 4) in names for once in (True, False)), names
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and outs[1][2] is None
    i32 = lambda y: torch.tensor(y, dtype=torch.int32, device=DEV)
    pages = N // page + 1
    table, alpha, caches = torch.arange(pages, device=DEV, dtype=torch.int32)[None], torch.rand(N, H, device=DEV), []

    def append(**kw):
        Kp, Vp, cp = (torch.zeros(s, dtype=t, device=DEV) for s, t in (((pages, Hkv, page, d), torch.bfloat16),) * 2 + (((pages, H, page), torch.float32),))
        g.gfwa_append_paged(k[0], v[0], Kp, Vp, i32([0, N]), i32([0]), table, freq=f, alpha=alpha, cp=cp, **kw)
        caches.append((Kp, Vp, cp))

    names = kernels(lambda: append(q=q[0]))
    assert variant("append_paged_kernel", "bf16", d, True) in names, names
    names = kernels(append)
    assert variant("append_paged_kernel", "bf16", d, False) in names, names
    assert all(torch.equal(a, b) for a, b in zip(*caches))


@pytest.mark.parametrize("dtype,most", [("bf16", 768), ("f32", 512)])
def test_workgroups_that_leave_sums_are_there_at_once(g, dtype, most):
    """Each leaves one row in the workspace: as many as the type's registers let run together (four waves of three, or two, a SIMD of 256 compute units)."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("counts workgroups of a whole MI355X")
    H, Hkv, N, d = 8, 2, 5900, 128
    x = normal(1, (1, N, H + 2 * Hkv, d), dtype)
    grads = [normal(2 + i, (1, h, N, d), dtype) for i, h in enumerate((H, Hkv, Hkv))]
    w = normal(6, (2, d), "f32")
    ws = torch.full((768, 2 * d), 3.5, device=DEV)
    assert ws.nbytes >= g.gfwa_qk_norm_rope_backward_workspace_bytes(1, H, Hkv, N, d)
    g.gfwa_qk_norm_rope_backward(x[:, :, :H], x[:, :, H:H + Hkv], *grads, w[0], w[1], freq=dev64(freq_of(d)), workspace=ws)
    used = int((ws != 3.5).any(1).nonzero().max()) + 1
    assert used <= most and (dtype == "f32" or used > 512), used
