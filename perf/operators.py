"""The operators that an attention layer needs next to the attention itself, as cases that a timing program can run.

  rope      queries and keys as the layer's projection gives them, [B,N,heads,d] inside one packed tensor: root-mean-square norm of
            each head, rotation by position, and the head-major layout that the attention reads (values change their layout alone)
  rope_bwd  its derivative: the gradient of the packed projection and of the two norm weights
  append    new tokens of a batch of sequences of different lengths: the same norm and rotation, keys and values written into
            a paged cache, the gate's prefix carried on there, queries handed back for the attention
  decode    one generated token for every sequence of a batch, against the paged cache

`own` false: elementary torch operations in 32 bits (64 for angles and long sums).  `own` true: the calls of `paper_2512_07782_amd`.

Keys of a case, beside its name:
  kind; B sequences; H, Hkv query heads and key/value heads; d head dimension; dtype storage type, "bf16" or "f32"
  N        rope, rope_bwd: length; append: most new tokens of a sequence (1: a decoding step); decode: longest sequence
  norm     whether heads are normed; rot: how many of the d dimensions are rotated; paired: (2j, 2j+1) instead of (j, j + rot/2)
  page, w  page length of the cache; window
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
TORCH_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
LONGEST = 131072           # positions at which an append may start
WHOLE = 1 << 20            # a window that holds every sequence

# What a drawn case may cost at most: the largest listed one of its kind.
MAX_ROWS = 16384 * 48 * 128 * 2        # bytes of the packed projection
MAX_NEW = 16 * 2048 * 48 * 128 * 2     # the same of all tokens that an append may bring
MAX_WINDOWS = 64 * 8 * 1024 * 128 * 2  # bytes of the keys that a decoding step reads


def _case(kind, B, H, Hkv, N, d, dtype="bf16", norm=True, rot=None, paired=False, page=64, w=1024, **name):
    return dict(kind=kind, B=B, H=H, Hkv=Hkv, N=N, d=d, dtype=dtype, norm=norm, rot=d if rot is None else rot, paired=paired, page=page, w=w, **name)


def listed():
    return [
        # a short prompt, batch one, grouped heads: the layer's preprocessing when serving latency counts
        _case("rope", 1, 32, 8, 700, 128, name="rope_prompt"),
        # a numerics check in fp32: odd length, 64-wide heads of which half is rotated, neighbouring dimensions in pairs
        _case("rope", 2, 8, 2, 515, 64, "f32", rot=32, paired=True, name="rope_pairs_f32"),
        # the long-sequence training shape with grouped heads
        _case("rope", 1, 32, 8, 16384, 128, name="rope_long"),
        # a fine-tuning step on short ragged sequences in fp32
        _case("rope_bwd", 2, 8, 2, 515, 64, "f32", rot=32, paired=True, name="rope_bwd_short_f32"),
        # the language-model shape, 64-wide heads in groups of four
        _case("rope_bwd", 4, 16, 4, 4096, 64, name="rope_bwd_lm"),
        # the long-sequence training shape
        _case("rope_bwd", 1, 32, 8, 16384, 128, name="rope_bwd_long"),
        # one conversation: a token's latency
        _case("append", 1, 32, 8, 1, 128, name="append_one"),
        # a serving batch: one token for each of its sequences
        _case("append", 64, 32, 8, 1, 128, page=16, name="append_batch"),
        # prompts (or their chunks) of different lengths written in one call, with rows of padding behind them
        _case("append", 16, 32, 8, 2048, 128, name="append_prompts"),
        # one conversation: a token's latency
        _case("decode", 1, 32, 8, 16384, 128, name="decode_paged_one"),
        # a serving batch of sequences of different lengths, slots without a sequence among them
        _case("decode", 64, 32, 8, 16384, 128, page=16, name="decode_paged_batch"),
        # whole sequences without a window, eight query heads for each key/value head, 64-wide heads
        _case("decode", 16, 32, 4, 16384, 64, page=32, w=WHOLE, name="decode_paged_whole"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the range the listed ones span, evenly in their logarithm."""
    kind = rng.choice(["rope", "rope_bwd", "append", "append", "decode", "decode"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    group = rng.choice([1, 2, 3, 4, 8, 16])
    Hkv = _log_int(rng, 1, 16)
    H = group * Hkv
    d = rng.choice([64, 128])
    norm = rng.random() < 0.8
    rot = rng.choice([d, d, d, d // 2, d // 4, 0 if norm else d])
    paired = rng.random() < 0.3
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    row = (H + 2 * Hkv) * d * SIZE[dtype]
    while True:
        if kind in ("rope", "rope_bwd"):
            B, N = _log_int(rng, 1, 16), _log_int(rng, 1, 16384)
            if B * N * row <= MAX_ROWS:
                return _case(kind, B, H, Hkv, N, d, dtype, norm, rot, paired)
        elif kind == "append":
            B, N = _log_int(rng, 1, 256), 1 if rng.random() < 0.4 else _log_int(rng, 1, 8192)
            if B * N * row <= MAX_NEW:
                return _case(kind, B, H, Hkv, N, d, dtype, norm, rot, paired, page)
        else:
            B, N, w = _log_int(rng, 1, 256), _log_int(rng, 64, 32768), WHOLE if rng.random() < 0.25 else _log_int(rng, 32, 4096)
            if B * Hkv * min(w, N) * d * SIZE[dtype] <= MAX_WINDOWS:
                return _case(kind, B, H, Hkv, N, d, dtype, page=page, w=w)


# ---- inputs

def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _normal(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _packed(gen, shape, H, Hkv, d, dtype):
    """A projection's output: heads of different magnitude, [.., (H + 2 Hkv) d], and its views by head."""
    heads = H + 2 * Hkv
    x = torch.randn(tuple(shape) + (heads, d), generator=gen, device=DEV, dtype=torch.float32)
    x *= torch.exp(0.3 * _normal(gen, (heads, 1)))
    x = x.to(dtype).view(tuple(shape) + (heads * d,))
    return x, _views(x, H, Hkv, d)


def _views(x, H, Hkv, d):
    x = x.view(x.shape[:-1] + (H + 2 * Hkv, d))
    return x[..., :H, :], x[..., H:H + Hkv, :], x[..., H + Hkv:, :]


def _norm_and_rotation(case, gen):
    d, rot = case["d"], case["rot"]
    s = {"wq": None, "wk": None, "freq": None}
    if case["norm"]:
        s["wq"], s["wk"] = 1 + 0.2 * _normal(gen, (d,)), 1 + 0.2 * _normal(gen, (d,))
    if rot:
        s["freq"] = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) * 2 / rot)
    return s


def _page_table(first, last, columns, rng):
    """[B, columns]: a page of its own, in no order, for the columns first .. last of every sequence and -1 for the others."""
    col = torch.arange(columns)
    live = (col >= torch.tensor(first)[:, None]) & (col <= torch.tensor(last)[:, None])
    count = int(live.sum())
    pages = count + 3
    order = torch.tensor(rng.sample(range(pages), count), dtype=torch.int32)
    table = torch.full(live.shape, -1, dtype=torch.int32)
    table[live] = order
    return table.to(DEV), pages


def _lengths(case):
    """The sequences of a case, which are part of it as its sizes are: append: (tokens cached, new ones) of each; decode: the position of the
    new token, -1 in slots without a sequence."""
    B, N = case["B"], case["N"]
    rng = random.Random("%d %d %d" % (B, N, case["page"]))
    if case["kind"] == "decode":
        return [-1 if b % 8 == 5 else rng.randint(N // 4, N - 1) for b in range(B)]
    new = [rng.randint(max(1, N // 4), N) for _ in range(B)]
    return [0 if N > 1 and rng.random() < 0.3 else _log_int(rng, 1, LONGEST) for _ in range(B)], new


def prepare(case, seed):
    kind, B, H, Hkv, N, d, page, w = (case[k] for k in ("kind", "B", "H", "Hkv", "N", "d", "page", "w"))
    dt = TORCH_DTYPE[case["dtype"]]
    gen, rng = _generator(seed), random.Random(seed)
    s = dict(case, scale=1.0 / math.sqrt(d))
    if kind in ("rope", "rope_bwd"):
        s["qkv"], (s["q"], s["k"], s["v"]) = _packed(gen, (B, N), H, Hkv, d, dt)
        s.update(_norm_and_rotation(case, gen))
        if kind == "rope_bwd":
            s["dQ"], s["dK"], s["dV"] = (_normal(gen, (B, h, N, d), dt) for h in (H, Hkv, Hkv))
        return s
    if kind == "append":
        cached, new = _lengths(case)
        rows = sum(new) if N == 1 else -(-sum(new) // 64) * 64
        s["start"] = _int32([sum(new[:b]) for b in range(B + 1)])
        s["cached"] = _int32(cached)
        s["qkv"], (s["q"], s["k"], s["v"]) = _packed(gen, (rows,), H, Hkv, d, dt)
        s.update(_norm_and_rotation(case, gen))
        s["alpha"] = torch.nn.functional.softplus(_normal(gen, (rows, H)) - 2)
        last = [(c + n - 1) // page for c, n in zip(cached, new)]
        s["table"], pages = _page_table([max(0, c - 1) // page for c in cached], last, max(last) + 1, rng)
        s["Kp"], s["Vp"] = _normal(gen, (pages, Hkv, page, d), dt), _normal(gen, (pages, Hkv, page, d), dt)
        s["cp"] = 1000 * torch.rand((pages, H, page), generator=gen, device=DEV)
        s["Q"] = torch.zeros((rows, H, d), dtype=dt, device=DEV)
        return s
    pos = _lengths(case)
    first, last = [max(0, p - w + 1) // page for p in pos], [p // page for p in pos]
    s["pos"] = _int32(pos)
    s["table"], pages = _page_table(first, last, (N + page - 1) // page, rng)
    s["q"] = _normal(gen, (B, H, d), dt)
    s["Kp"], s["Vp"] = _normal(gen, (pages, Hkv, page, d), dt), _normal(gen, (pages, Hkv, page, d), dt)
    # the prefix over every sequence's pages, from what the tokens in front of them have added up to
    most = max(b - a for a, b in zip(first, last)) + 1
    c = torch.nn.functional.softplus(_normal(gen, (B, H, most * page)) - 2).double().cumsum(-1)
    c += 0.2 * page * torch.tensor(first, dtype=torch.float64, device=DEV)[:, None, None]
    c = c.float().view(B, H, most, page)
    s["cp"] = torch.zeros((pages, H, page), device=DEV)
    b, col = torch.nonzero(s["table"] >= 0, as_tuple=True)
    s["cp"][s["table"][b, col].long()] = c[b, :, col - torch.tensor(first, device=DEV)[b]]
    s["o"] = torch.zeros((B, H, d), dtype=dt, device=DEV)
    s["L"] = torch.zeros((B, H), device=DEV)
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    return s


# ---- the plain forms

def _cos_sin(pos, freq, sign):
    """cos and sin of pos * freq, the angle in 64 bits: [.., 1, rot / 2], to go with [.., heads, d]."""
    angle = (pos.double()[..., None] * freq)[..., None, :]
    return torch.cos(angle).float(), torch.sin(angle).float() * sign


def _rotated(x, pos, s, sign=1.0):
    if s["freq"] is None:
        return x
    rot = s["rot"]
    cos, sin = _cos_sin(pos, s["freq"], sign)
    if s["paired"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _normed_and_rotated(x, weight, pos, s):
    x = x.float()
    if s["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    return _rotated(x, pos, s)


def _head_gradient(x, weight, pos, dy, s):
    """(dx, dweight) of _normed_and_rotated, dy as [B,heads,N,d]."""
    g = _rotated(dy.float().transpose(1, 2), pos, s, -1.0)
    if not s["norm"]:
        return g, None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    x = x * r
    dweight = (g * x).sum((0, 1, 2), dtype=torch.float64).float()
    g = g * weight
    return r * (g - x * (g * x).mean(-1, keepdim=True)), dweight


def _plain_append(s):
    start, dt = s["start"].long(), s["q"].dtype
    row = torch.arange(s["q"].shape[0], device=DEV)
    here = row < start[-1]
    row = torch.minimum(row, start[-1] - 1)  # rows behind the last sequence write its last token once more
    seq = torch.searchsorted(start, row, right=True) - 1
    before = s["cached"].long()
    pos = before[seq] + row - start[seq]
    Q, k = (_normed_and_rotated(s[n][row], s["w" + n], pos, s).to(dt) for n in ("q", "k"))
    s["Q"].copy_(torch.where(here[:, None, None], Q, s["Q"]))
    # prefix: what the cache holds at the position before the first new one, and the sums from there on
    page, prev = s["page"], (before - 1).clamp(min=0)
    c0 = s["cp"][torch.gather(s["table"], 1, (prev // page)[:, None])[:, 0].long(), :, prev % page]
    c0 = torch.where(before[:, None] > 0, c0, 0.0).double()
    total = torch.cumsum(torch.where(here[:, None], s["alpha"], 0.0), 0, dtype=torch.float64)
    total = torch.cat((torch.zeros_like(total[:1]), total))
    c = c0[seq] + total[row + 1] - total[start[seq]]
    at = s["table"][seq, pos // page].long(), slice(None), pos % page
    s["Kp"][at], s["Vp"][at], s["cp"][at] = k, s["v"][row], c.float()


def _plain_decode(s):
    B, H, Hkv, d, page, table = (s[k] for k in ("B", "H", "Hkv", "d", "page", "table"))
    keys = min(s["w"], table.shape[1] * page)
    pos = s["pos"].long()[:, None]
    i = pos - torch.arange(keys - 1, -1, -1, device=DEV)
    there = (i >= 0) & (pos >= 0)
    i = i.clamp(min=0)
    at = torch.gather(table, 1, i // page).long()
    there &= at >= 0
    at = at.clamp(min=0), slice(None), i % page
    k, v, c = (s[n][at].float() for n in ("Kp", "Vp", "cp"))  # [B,keys,heads(,d)]
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.transpose(1, 2).contiguous()
    c = (c - c[:, -1:]).transpose(1, 2)
    x = torch.matmul(s["q"].float().view(B, Hkv, H // Hkv, d) * s["scale"], k).view(B, H, keys) + c
    x = torch.where(there[:, None], x, -torch.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, Hkv, H // Hkv, keys), v).view(B, H, d) / total
    s["o"].copy_(torch.where(total > 0, o, 0.0))
    s["L"].copy_((m + torch.log(total))[..., 0])


def _run_plain(s):
    kind = s["kind"]
    if kind == "append":
        _plain_append(s)
        return {k: s[k] for k in ("Q", "Kp", "Vp", "cp")}
    if kind == "decode":
        _plain_decode(s)
        return {"o": s["o"], "L": s["L"]}
    dt = s["qkv"].dtype
    pos = torch.arange(s["N"], device=DEV)
    if kind == "rope":
        Q, K = (_normed_and_rotated(s[n], s["w" + n], pos, s).transpose(1, 2).to(dt).contiguous() for n in ("q", "k"))
        return {"Q": Q, "K": K, "V": s["v"].transpose(1, 2).contiguous()}
    dq, dwq = _head_gradient(s["q"], s["wq"], pos, s["dQ"], s)
    dk, dwk = _head_gradient(s["k"], s["wk"], pos, s["dK"], s)
    dqkv = torch.cat((dq.to(dt), dk.to(dt), s["dV"].transpose(1, 2)), 2)
    return {"dqkv": dqkv.view(s["qkv"].shape), "dwq": dwq, "dwk": dwk}


# ---- the framework's calls

def _run_own(s):
    import paper_2512_07782_amd as g
    kind = s["kind"]
    how = {k: s.get(k) for k in ("wq", "wk", "freq", "norm", "paired")}
    if kind == "rope":
        Q, K, V = g.gfwa_qk_norm_rope(s["q"], s["k"], s["v"], eps=EPS, **how)
        return {"Q": Q, "K": K, "V": V}
    if kind == "rope_bwd":
        dqkv = torch.empty_like(s["qkv"])
        dq, dk, dv = _views(dqkv, s["H"], s["Hkv"], s["d"])
        _, _, _, dwq, dwk = g.gfwa_qk_norm_rope_backward(s["q"], s["k"], s["dQ"], s["dK"], s["dV"], eps=EPS, dq=dq, dk=dk, dv=dv, **how)
        return {"dqkv": dqkv, "dwq": dwq, "dwk": dwk}
    if kind == "append":
        g.gfwa_append_paged(s["k"], s["v"], s["Kp"], s["Vp"], s["start"], s["cached"], s["table"], q=s["q"], Q=s["Q"], alpha=s["alpha"],
                            cp=s["cp"], eps=EPS, **how)
        return {k: s[k] for k in ("Q", "Kp", "Vp", "cp")}
    g.gfwa_decode_paged(s["q"], s["Kp"], s["Vp"], s["cp"], s["table"], s["pos"], s["w"], s["scale"], o=s["o"], L=s["L"], workspace=s["workspace"])
    return {"o": s["o"], "L": s["L"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the definition in 64 bits

def _exact_heads(x, weight, pos, s):
    """[rows, heads, d] normed and rotated, the rotated pairs as complex numbers."""
    if s["norm"]:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / s["d"] + EPS) * weight.double()
    if s["freq"] is None:
        return x
    rot = s["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * s["freq"])[:, None]
    pairs = x[..., :rot].unflatten(-1, (rot // 2, 2)) if s["paired"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    z = z if s["paired"] else z.transpose(-1, -2)
    return torch.cat((z.flatten(-2), x[..., rot:]), -1)


def _exact_append(s):
    page, table, start, cached = s["page"], s["table"].tolist(), s["start"].tolist(), s["cached"].tolist()
    Kp, Vp, cp, Q = (s[k].double() for k in ("Kp", "Vp", "cp", "Q"))
    for b, before in enumerate(cached):
        rows = slice(start[b], start[b + 1])
        pos = torch.arange(before, before + start[b + 1] - start[b], device=DEV)
        Q[rows] = _exact_heads(s["q"][rows].double(), s["wq"], pos, s)
        k, v = _exact_heads(s["k"][rows].double(), s["wk"], pos, s), s["v"][rows].double()
        c = s["alpha"][rows].double().cumsum(0)
        if before:
            c += s["cp"][table[b][(before - 1) // page], :, (before - 1) % page].double()
        done = 0
        while done < len(pos):  # page by page
            p = before + done
            n = min(page - p % page, len(pos) - done)
            to, at = table[b][p // page], slice(p % page, p % page + n)
            for pages, new in ((Kp, k), (Vp, v), (cp, c)):
                pages[to][:, at] = new[done:done + n].transpose(0, 1)
            done += n
    return {"Q": Q, "Kp": Kp, "Vp": Vp, "cp": cp}


def _exact_decode(s):
    page, table, pos = s["page"], s["table"], s["pos"].tolist()
    B, H, Hkv, d = (s[k] for k in ("B", "H", "Hkv", "d"))
    o = torch.zeros((B, H, d), dtype=torch.float64, device=DEV)
    L = torch.full((B, H), -math.inf, dtype=torch.float64, device=DEV)
    for b, p in enumerate(pos):
        if p < 0:
            continue
        lo = max(0, p - s["w"] + 1)
        first = lo // page
        ids = table[b, first:p // page + 1].long()
        k, v, c = (s[n][ids].transpose(0, 1).flatten(1, 2)[:, lo - first * page:p + 1 - first * page].double() for n in ("Kp", "Vp", "cp"))
        q = s["q"][b].double().view(Hkv, H // Hkv, d)
        x = s["scale"] * torch.matmul(q, k.transpose(1, 2)) + (c - c[:, -1:]).view(Hkv, H // Hkv, -1)
        L[b] = torch.logsumexp(x, -1).flatten()
        o[b] = torch.matmul(torch.softmax(x, -1), v).flatten(0, 1)
    return {"o": o, "L": L}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "decode":
        return _exact_decode(s)
    B, N, H, Hkv = (case[k] for k in ("B", "N", "H", "Hkv"))
    pos = torch.arange(N, device=DEV).repeat(B)

    def forward(x, weight):
        return _exact_heads(x, weight, pos, s).unflatten(0, (B, N)).transpose(1, 2)

    q, k = (s[n].flatten(0, 1).double() for n in ("q", "k"))
    if case["kind"] == "rope":
        return {"Q": forward(q, s["wq"]), "K": forward(k, s["wk"]), "V": s["v"].transpose(1, 2).double()}
    grads, weights = [], []
    for x, weight, dy in ((q, s["wq"], s["dQ"]), (k, s["wk"], s["dK"])):
        leaves = [t.double().requires_grad_() for t in (x, weight) if t is not None]
        got = torch.autograd.grad(forward(leaves[0], leaves[-1]), leaves, dy.double())
        grads.append(got[0])
        weights.append(got[1] if case["norm"] else None)
    dqkv = torch.cat(grads + [s["dV"].transpose(1, 2).flatten(0, 1).double()], 1)
    return {"dqkv": dqkv.reshape(s["qkv"].shape), "dwq": weights[0], "dwk": weights[1]}


def work(case):
    """Every input read once, every output written once; of the cache only what new tokens fill or the window holds."""
    kind, B, H, Hkv, N, d = (case[k] for k in ("kind", "B", "H", "Hkv", "N", "d"))
    size = SIZE[case["dtype"]]
    heads = H + 2 * Hkv
    if kind == "decode":
        keys = sum(min(case["w"], p + 1) for p in _lengths(case))
        return {"bytes": keys * (2 * Hkv * d * size + 4 * H) + 2 * B * H * d * size + 4 * B * H, "flops": 4 * H * keys * d}
    if kind == "append":
        rows = sum(_lengths(case)[1])
        return {"bytes": rows * (2 * heads * d * size + 8 * H), "flops": 10 * rows * (H + Hkv) * d}
    rows = B * N
    if kind == "rope":
        return {"bytes": rows * 2 * heads * d * size, "flops": 10 * rows * (H + Hkv) * d}
    read = heads + (H + Hkv if case["norm"] else 0)
    return {"bytes": rows * (read + heads) * d * size, "flops": 20 * rows * (H + Hkv) * d}
