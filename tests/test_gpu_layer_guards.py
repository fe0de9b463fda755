"""The operators around the attention write what the header says they write and nothing else: every output, cache and workspace stands in the middle of
a poisoned allocation.  Each call runs twice on the same inputs and returns the same bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAD, POISON = 8192, 0xA5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def g():
    import paper_2512_07782_amd as mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    mod.load_library()
    return mod


class Guarded:
    def __init__(self, shape, dtype):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        self.n, self.buf = n, torch.full((PAD + n + PAD,), POISON, dtype=torch.uint8, device=DEV)
        self.t = self.buf[PAD:PAD + n].view(dtype).view(shape)

    def intact(self):
        return bool((self.buf[:PAD] == POISON).all()) and bool((self.buf[PAD + self.n:] == POISON).all())


def normal(seed, shape, dtype):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def freq(rot):
    return None if rot == 0 else 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) * 2 / rot)


def check(named, runs):
    for name, gd in named.items():
        assert gd.intact(), name + ": bytes outside the buffer were written"
    runs.append({k: x.t.clone() for k, x in named.items() if k != "workspace"})
    if len(runs) == 2:
        for k in runs[0]:
            assert torch.equal(runs[0][k].view(torch.uint8), runs[1][k].view(torch.uint8)), k + ": two runs differ"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,Hkv,N,d,rot", [(1, 1, 1, 1, 64, 64), (2, 7, 7, 37, 128, 96), (3, 9, 3, 130, 64, 16), (1, 33, 11, 515, 128, 128),
                                             (1, 3, 1, 40001, 64, 0), (600, 2, 1, 3, 128, 16), (1, 2000, 1000, 1, 64, 64)])
def test_norm_and_rotation(g, B, H, Hkv, N, d, rot, dtype):
    print("guards rope", B, H, Hkv, N, d, rot, dtype, flush=True)
    dt, f, runs, back = DTYPES[dtype], freq(rot), [], []
    x = normal(1, (B, N, H + 2 * Hkv, d), dt)
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    dQ, dK, dV = (normal(2 + i, (B, h, N, d), dt) for i, h in enumerate((H, Hkv, Hkv)))
    wt = normal(9, (d,), torch.float32)
    for _ in range(2):
        o = {n: Guarded((B, h, N, d), dt) for n, h in (("Q", H), ("K", Hkv), ("V", Hkv))}
        g.gfwa_qk_norm_rope(q, k, v, wt, wt, freq=f, **{n: x.t for n, x in o.items()})
        check(o, runs)
        b = {n: Guarded((B, N, h, d), dt) for n, h in (("dq", H), ("dk", Hkv), ("dv", Hkv))}
        b.update({n: Guarded((d,), torch.float32) for n in ("dwq", "dwk")})
        b["workspace"] = Guarded((g.gfwa_qk_norm_rope_backward_workspace_bytes(B, H, Hkv, N, d),), torch.uint8)
        g.gfwa_qk_norm_rope_backward(q, k, dQ, dK, dV, wt, wt, freq=f, **{n: x.t for n, x in b.items()})
        check(b, back)
    for r in (runs[0], back[0]):
        assert all(torch.isfinite(x.float()).all() for x in r.values())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,H,Hkv,d,page,M", [([1], 1, 1, 64, 16, 1), ([1] * 33, 6, 2, 128, 16, 3), ([70, 0, 1, 301], 8, 8, 64, 48, 9),
                                                ([2000, 3], 2, 1, 128, 128, 16), ([5] * 300, 4, 4, 64, 16, 2)])
def test_append_and_decode(g, new, H, Hkv, d, page, M, dtype):
    print("guards paged", new[:4], H, Hkv, d, page, dtype, flush=True)
    dt, B, runs, back = DTYPES[dtype], len(new), [], []
    rng = np.random.default_rng(d + page)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)
    cached = [int(rng.integers(0, M * page - n + 1)) for n in new]
    rows, pages = sum(new) + 9, B * M + 1
    start, table = i32(np.concatenate([[0], np.cumsum(new)])), i32(rng.permutation(pages)[:B * M].reshape(B, M))
    q, k, v = (normal(20 + i, (rows, h, d), dt) for i, h in enumerate((H, Hkv, Hkv)))
    alpha = normal(30, (rows, H), torch.float32).abs() * 0.1
    for _ in range(2):
        o = {"Kp": Guarded((pages, Hkv, page, d), dt), "Vp": Guarded((pages, Hkv, page, d), dt), "cp": Guarded((pages, H, page), torch.float32),
             "Q": Guarded((rows, H, d), dt)}
        for x in o.values():
            x.t.zero_()
        o["Q"].t.fill_(3)
        g.gfwa_append_paged(k, v, o["Kp"].t, o["Vp"].t, start, i32(cached), table, q=q, alpha=alpha, cp=o["cp"].t, Q=o["Q"].t, freq=freq(d))
        check(o, runs)
        assert (o["Q"].t[sum(new):] == 3).all()
        for w in (1, 20, 1 << 20):
            pos = i32([c + n - 1 for c, n in zip(cached, new)])
            r = {"o": Guarded((B, H, d), dt), "L": Guarded((B, H), torch.float32),
                 "workspace": Guarded((g.gfwa_decode_paged_workspace_bytes(B, H, Hkv, d, page, M, w),), torch.uint8)}
            qd = normal(40, (B, H, d), dt)
            g.gfwa_decode_paged(qd, o["Kp"].t, o["Vp"].t, o["cp"].t, table, pos, w, d ** -0.5, **{n: x.t for n, x in r.items()})
            torch.cuda.synchronize()
            for n, x in r.items():
                assert x.intact(), n
            back.append((r["o"].t.clone(), r["L"].t.clone()))
            empty = pos < 0
            assert torch.isfinite(r["o"].t.float()).all() and torch.equal(torch.isinf(r["L"].t).all(1), empty)
    for a, b in zip(back[:3], back[3:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
