"""What is timed of the operators that stand beside the linear layer: dropout whose mask is never stored, and low-rank
adapters of many requests beside a shared projection, each forward and backward.

Dropout.  Element (R, C) of the full matrix is kept where its 16 random bits are at least T = round(65536 p), and then
multiplied by 65536 / (65536 - T).  The bits come from the counter-based generator Philox4x32-10 (Salmon, Moraes, Dror, Shaw:
"Parallel random numbers: as easy as 1, 2, 3", 2011) with counter (C / 8, R, offset) and key `seed`: the eight columns of a group share
one 128-bit draw, column 8 g + e taking bits 16 e .. 16 e + 15.  So the mask goes by the position in the full matrix, whatever the
partition, and backward draws it again.
    forward    Z = drop(act(X + b)) + R            backward    dX = drop'(dZ) GeLU'(A),  db = 1^T dX

Adapters.  Rows come in segments (a request each); a segment names an adapter of a pool or none (an id outside the pool).  With
the factors A_i: [rank, H] and B_i: [rank, F] and the scale s_i of a row's adapter i
    forward    V = drop(X) A_i^T,  Y = act(C + s_i V B_i + b)          (C: the shared projection's product)
    backward   U = dY B_i^T,  dX = dX_base + drop'(s_i U A_i),  dA_i = s_i U^T drop(X),  dB_i = s_i V^T dY   (sums over the rows of adapter i)
A rank of a grid has blocks of X and A (of dY and B) for every step of its sum.  Rows behind the last segment stay as they were.

A case is one call: `kind` names it.  mode, q, d, p, ri, rj, rk and M, H, F are the rank grid and the full layer; `keep` below 1 asks for
dropout (of probability 1 - keep) on the adapters' input.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

_BF, _F32 = torch.bfloat16, torch.float32
_SEED_MASK = (1 << 64) - 1


def _drop(kind, rows, cols, x, act, **more):
    return dict(dict(kind=kind, rows=rows, cols=cols, x=x, act=act, residual=False, pre=False, y="bf16", keep=0.9, row0=0, col0=0), **more)


def _adapter(kind, mode, M, H, F, rank, pool, requests, q=1, d=1, p=1, ri=0, rj=0, rk=0, **more):
    return dict(dict(kind=kind, mode=mode, q=q, d=d, p=p, ri=ri, rj=rj, rk=rk, M=M, H=H, F=F, rank=rank, pool=pool, requests=requests,
                     tail=0, keep=1.0, c="bf16", y="bf16", act="none"), **more)


def listed():
    return [
        # ---- dropout
        # a few rows of a row-cut layer's sum: launch and host path count
        _drop("drop_fwd", 8, 4096, "f32", "bias", residual=True, name="dropout_few_rows"),
        # what follows the row-cut product of the 4096 / 16384 feed-forward: fp32 sum of partials, bias, dropout, residual
        _drop("drop_fwd", 16384, 4096, "f32", "bias", residual=True, name="dropout_residual_1d"),
        # the same place on a 4 x 4 grid, where the product's own epilogue has added the bias: bf16 in and out, a block inside the matrix
        _drop("drop_fwd", 2048, 8192, "bf16", "none", residual=True, row0=2048, col0=16384, name="dropout_residual_2d"),
        # hidden activations of the ViT-style MLP after their summation: bias, GeLU, dropout, the pre-activation kept; ragged rows
        _drop("drop_fwd", 32896, 2560, "f32", "gelu", pre=True, col0=2560, row0=32896, name="dropout_gelu_vit"),
        # backward of the residual form: dX and the bias gradient in one pass
        _drop("drop_bwd", 16384, 4096, "bf16", "bias", name="dropout_bwd_1d"),
        # backward of the GeLU form
        _drop("drop_bwd", 32896, 2560, "bf16", "gelu", col0=2560, row0=32896, name="dropout_bwd_gelu_vit"),
        # ---- adapters
        # one new token of one request: latency
        _adapter("adapter_fwd", "1d_col", 1, 4096, 16384, 16, 8, 1, p=4, ri=1, name="adapter_token"),
        # a decoding batch of 96 requests over a pool of 48 adapters, some requests without one: streams the factors
        _adapter("adapter_fwd", "1d_col", 96, 4096, 16384, 16, 48, 96, p=4, ri=1, name="adapter_decode"),
        # prompts of 12 requests and a padded tail through a column-cut layer with bias, GeLU and a saved pre-activation
        _adapter("adapter_fwd", "1d_col", 6000, 4096, 16384, 32, 8, 12, p=4, ri=1, tail=77, c="f32", act="gelu", name="adapter_prefill"),
        # fine-tuning one adapter of rank 64 on a 4 x 4 grid's share, forward: four steps, dropout on the adapter's input, bias
        _adapter("adapter_fwd", "2d", 8192, 8192, 32768, 64, 1, 1, q=4, ri=1, rj=2, keep=0.9, act="bias", name="adapter_steps_2d"),
        # fine-tuning with dropout on the adapter's input, backward: dX, dA and dB
        _adapter("adapter_bwd", "1d_col", 16384, 4096, 16384, 16, 1, 1, p=4, ri=1, keep=0.95, c="f32", y="f32", name="adapter_train_bwd"),
        # three tenants' batches on the ViT-style MLP's 2 x 2 x 2 grid, backward over two steps; ragged rows
        _adapter("adapter_bwd", "2.5d", 131584, 1280, 5120, 8, 3, 24, q=2, d=2, ri=1, rk=1, tail=40, name="adapter_bwd_vit"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _eights(rng, lo, hi):
    return max(1, round(_log(rng, lo, hi) / 8)) * 8


def draw(rng):
    kind = rng.choice(["drop_fwd", "drop_bwd", "adapter_fwd", "adapter_fwd", "adapter_bwd"])
    keep = rng.choice([0.9, 0.5, rng.uniform(0.05, 0.999)])
    if kind.startswith("drop"):
        rows, cols = int(_log(rng, 1, 33000)), _eights(rng, 8, 25000)
        rows = min(rows, 80_000_000 // cols)
        at = dict(row0=rng.randrange(0, 1 << 20), col0=8 * rng.randrange(0, 4096), keep=keep)
        if kind == "drop_bwd":
            return _drop(kind, rows, cols, "bf16", rng.choice(["bias", "gelu", "none"]), **at)
        act = rng.choice(["none", "bias", "gelu"])
        return _drop(kind, rows, cols, rng.choice(["f32", "bf16"]), act, residual=rng.random() < 0.6, pre=act == "gelu" and rng.random() < 0.7,
                     y=rng.choice(["bf16", "bf16", "f32"]), **at)
    mode = rng.choice(["1d_col", "1d_row", "2d", "2.5d", "3d"])
    g = dict(q=1, d=1, p=1, ri=0, rj=0, rk=0)
    if mode.startswith("1d"):
        g.update(p=rng.choice([1, 2, 4, 8]))
        g.update(ri=rng.randrange(g["p"]))
    elif mode == "3d":
        g.update(p=2, ri=rng.randrange(2), rj=rng.randrange(2), rk=rng.randrange(2))
    else:
        g.update(q=rng.choice([2, 3, 4]), d=1 if mode == "2d" else rng.choice([1, 2]))
        g.update(ri=rng.randrange(g["q"]), rj=rng.randrange(g["q"]), rk=rng.randrange(g["d"]))
    shape = dict(g, mode=mode, M=1, H=1, F=1)
    rc, kc, cc, steps = _chunks(shape)
    few = kind == "adapter_fwd" and rng.random() < 0.5
    hb, fb = _eights(rng, 64, 4096), _eights(rng, 64, 4096)
    most = 180_000_000 // (steps * (hb + fb) + 2 * (hb + fb))
    mb = max(1, min(int(_log(rng, 1, 256) if few else _log(rng, 200, 20000)), most))
    requests = rng.choice([mb, max(1, mb // 3)]) if few else rng.choice([1, 2, rng.randint(3, 40)])
    pool = rng.choice([1, 3, rng.randint(4, 32)])
    rank = rng.choice([8, 16, 16, 32, 64, 8 * rng.randint(1, 16)])
    pool = max(1, min(pool, 640 // rank))
    partial = mode == "1d_row" and g["p"] > 1
    act = "none" if partial or kind == "adapter_bwd" else rng.choice(["none", "bias", "gelu"])
    out = "f32" if partial or (kind == "adapter_bwd" and mode == "1d_col" and g["p"] > 1) else rng.choice(["bf16", "f32"])
    return dict(_adapter(kind, mode, mb * rc, hb * kc, fb * cc, rank, pool, requests, **g), tail=rng.choice([0, rng.randrange(0, 1 + mb // 4)]),
                keep=1.0 if few else rng.choice([1.0, keep]), c="f32" if partial else rng.choice(["bf16", "f32"]), y=out, act=act)


# ------------------------------------------------------------------------------------------------ extents
def _chunks(case):
    """Row chunks of X, column chunks of X, column chunks of W, steps of the rank's sum."""
    q, d, p = case["q"], case["d"], case["p"]
    return {"1d_col": (1, 1, p, 1), "1d_row": (1, p, 1, 1), "2d": (q, q, q, q), "2.5d": (q * d, q, q, q), "3d": (p * p, p, p, p)}[case["mode"]]


def _share(case):
    """m, k, n of the rank's blocks, its steps, the row chunk and the column chunk of X that are its own."""
    rc, kc, cc, steps = _chunks(case)
    i, j, l = case["ri"], case["rj"], case["rk"]
    row, col = {"1d_col": (0, 0), "1d_row": (0, i), "2d": (i, j), "2.5d": (l * case["q"] + i, j), "3d": (i * case["p"] + l, j)}[case["mode"]]
    return case["M"] // rc, case["H"] // kc, case["F"] // cc, steps, row, col


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(2110 + 7919 * (int(seed) % (1 << 40)))
    return g


def _normal(g, *shape, std=1.0, dtype=_BF):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case=dict(case), seed=(0x9E3779B97F4A7C15 * (int(seed) + 1)) & _SEED_MASK, offset=int(seed) % 1000 + (1 << 33))
    rand = functools.partial(_normal, g)
    empty = lambda *shape, dtype: torch.full(shape, 0.25, dtype=dtype, device="cuda")
    type_of = lambda name: _F32 if name == "f32" else _BF
    if case["kind"].startswith("drop"):
        rows, cols = case["rows"], case["cols"]
        if case["kind"] == "drop_fwd":
            s.update(x=rand(rows, cols, std=1.28, dtype=type_of(case["x"])), y=empty(rows, cols, dtype=type_of(case["y"])),
                     bias=None if case["act"] == "none" else rand(cols, std=0.02), residual=rand(rows, cols) if case["residual"] else None,
                     pre=empty(rows, cols, dtype=_BF) if case["pre"] else None)
        else:
            s.update(dy=rand(rows, cols), dx=empty(rows, cols, dtype=_BF), db=None if case["act"] == "none" else empty(cols, dtype=_F32),
                     pre=rand(rows, cols, std=1.28) if case["act"] == "gelu" else None)
        return s
    m, k, n, steps, row, col = _share(case)
    rank, pool, requests = case["rank"], case["pool"], case["requests"]
    covered = m - case["tail"]
    # cut points of the segments: one row each where there are as many requests as rows, else anywhere (empty requests among them)
    if requests >= covered:
        cuts = torch.arange(requests + 1, device="cuda").clamp(max=covered)
    else:
        cuts = torch.randint(0, covered + 1, (requests + 1,), generator=g, device="cuda").sort().values
        cuts[0], cuts[-1] = 0, covered
    ids = torch.randint(0 if requests == 1 else -1, pool, (requests,), generator=g, device="cuda")
    s.update(offsets=cuts.to(torch.int32), ids=ids.to(torch.int32), scale=torch.rand(pool, generator=g, device="cuda") * 1.5 + 0.5)
    A = lambda: rand(pool, rank, k, std=1.0 / math.sqrt(k * steps))
    B = lambda: rand(pool, rank, n, std=0.2 / math.sqrt(rank))
    if case["kind"] == "adapter_fwd":
        s.update(x=[rand(m, k) for _ in range(steps)], a=[A() for _ in range(steps)], b=B(), c=rand(m, n, std=1.28, dtype=type_of(case["c"])),
                 bias=None if case["act"] == "none" else rand(n, std=0.02), y=empty(m, n, dtype=type_of(case["y"])),
                 pre=empty(m, n, dtype=_BF) if case["act"] == "gelu" else None, v=empty(m, rank, dtype=_F32))
    else:
        s.update(dy=[rand(m, n) for _ in range(steps)], b=[B() for _ in range(steps)], a=A(), x=rand(m, k), v=rand(m, rank, dtype=_F32),
                 c=rand(m, k, std=1.28, dtype=type_of(case["c"])), dx=empty(m, k, dtype=type_of(case["y"])),
                 da=empty(pool, rank, k, dtype=_F32), db=empty(pool, rank, n, dtype=_F32), own_dy=0 if case["mode"].startswith("1d") else case["rj"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _round(state, i, seed):
    """One round of the generator on 32-bit words held in 64 (products wrap at 64 bits; the shifts are masked)."""
    x0, x1, x2, x3 = state
    key0, key1 = ((seed & 0xFFFFFFFF) + 0x9E3779B9 * i) & 0xFFFFFFFF, ((seed >> 32) + 0xBB67AE85 * i) & 0xFFFFFFFF
    a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57
    return (b >> 32 & 0xFFFFFFFF) ^ x1 ^ key0, b & 0xFFFFFFFF, (a >> 32 & 0xFFFFFFFF) ^ x3 ^ key1, a & 0xFFFFFFFF


def _threshold(case):
    return round((1.0 - case["keep"]) * 65536)


def _kept(case, state, rows, cols, row0, col0):
    """Factor of every element: 0, or 65536 / (65536 - T)."""
    r = (torch.arange(rows, device="cuda") + row0)[:, None].expand(rows, cols // 8)
    c = (torch.arange(cols // 8, device="cuda") + col0 // 8)[None].expand(rows, cols // 8)
    lo = torch.full_like(c, state["offset"] & 0xFFFFFFFF)
    hi = torch.full_like(c, state["offset"] >> 32)
    words = functools.reduce(lambda x, i: _round(x, i, state["seed"]), range(10), (c, r, lo, hi))
    bits = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=2).view(rows, cols)
    t = _threshold(case)
    return (bits >= t).float() * (65536.0 / (65536 - t))


def _gelu(a):
    return 0.5 * a * (1.0 + torch.erf(a * math.sqrt(0.5)))


def _gelu_slope(a):
    return 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5))) + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_drop_fwd(case, s):
    a = s["x"].float()
    if s["bias"] is not None:
        a = a + s["bias"].float()
    z = _gelu(a) if case["act"] == "gelu" else a
    z = z * _kept(case, s, case["rows"], case["cols"], case["row0"], case["col0"])
    if s["residual"] is not None:
        z = z + s["residual"].float()
    return dict(y=z.to(s["y"].dtype), pre=None if s["pre"] is None else a.to(_BF))


def _plain_drop_bwd(case, s):
    g = s["dy"].float() * _kept(case, s, case["rows"], case["cols"], case["row0"], case["col0"])
    if s["pre"] is not None:
        g = g * _gelu_slope(s["pre"].float())
    return dict(dx=g.to(_BF), db=None if s["db"] is None else g.sum(0))


def _rows_of(s, m):
    """Of each row: whether a segment holds it, and a 0 / 1 row over the pool that picks its adapter."""
    r = torch.arange(m, device="cuda")
    seg = torch.bucketize(r, s["offsets"][1:].long(), right=True)
    inside = r < s["offsets"][-1]
    who = torch.where(inside, s["ids"].long()[seg.clamp(max=s["ids"].numel() - 1)], -1)
    return inside[:, None], (who[:, None] == torch.arange(s["scale"].numel(), device="cuda")).float()


def _down(pick, p, factor):
    """Each row's product with its own adapter's factor [rank, cols]^T."""
    pool, rank, cols = factor.shape
    return ((p @ factor.reshape(pool * rank, cols).t()).view(-1, pool, rank) * pick[:, :, None]).sum(1)


def _spread(pick, v):
    """[rows, rank] -> [rows, pool * rank] with a row's values at its own adapter."""
    return (v[:, None] * pick[:, :, None]).flatten(1)


def _plain_adapter_fwd(case, s):
    m, k, n, steps, row, col = _share(case)
    inside, pick = _rows_of(s, m)
    x = torch.cat(s["x"], 1).float()
    if case["keep"] < 1:
        x = x * _kept(case, s, m, k * steps, row * m, col * k if case["mode"] == "1d_row" else 0)
    v = _down(pick, x, torch.cat(s["a"], 2).float())
    a = s["c"].float() + _spread(pick * s["scale"], v) @ s["b"].float().flatten(0, 1)
    if s["bias"] is not None:
        a = a + s["bias"].float()
    y = _gelu(a) if case["act"] == "gelu" else a
    return dict(y=torch.where(inside, y.to(s["y"].dtype), s["y"]), v=torch.where(pick.sum(1, keepdim=True) > 0, v, s["v"]),
                pre=None if s["pre"] is None else torch.where(inside, a.to(_BF), s["pre"]))


def _plain_adapter_bwd(case, s):
    m, k, n, steps, row, col = _share(case)
    inside, pick = _rows_of(s, m)
    u = _down(pick, torch.cat(s["dy"], 1).float(), torch.cat(s["b"], 2).float())
    keep = _kept(case, s, m, k, row * m, col * k) if case["keep"] < 1 else 1.0
    dx = s["c"].float() + _spread(pick * s["scale"], u) @ s["a"].float().flatten(0, 1) * keep
    da = _spread(pick * s["scale"], u).t() @ (s["x"].float() * keep)
    db = _spread(pick * s["scale"], s["v"]).t() @ s["dy"][s["own_dy"]].float()
    return dict(dx=torch.where(inside, dx.to(s["dx"].dtype), s["dx"]), da=da.view_as(s["da"]), db=db.view_as(s["db"]))


# ------------------------------------------------------------------------------------------------ the framework's calls
def _handles(T, case, s):
    """What a program makes once and keeps: grid, workspace."""
    if case["kind"].startswith("drop"):
        need = T.tp_bias_grad_workspace_size(case["rows"], case["cols"]) if case["kind"] == "drop_bwd" else 0
        return dict(ws=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    mode = {"1d_col": T.MODE_1D_COL, "1d_row": T.MODE_1D_ROW, "2d": T.MODE_2D, "2.5d": T.MODE_2P5D, "3d": T.MODE_3D}[case["mode"]]
    grid = T.Grid(mode, q=case["q"], d=case["d"], p=case["p"], ri=case["ri"], rj=case["rj"], rk=case["rk"])
    dims = (case["M"], case["H"], case["F"])
    adapters = T.Adapters(s["offsets"], s["ids"], case["pool"], case["rank"], s["scale"])
    need = T.tp_adapter_workspace_size(grid, dims, T.PASS_FWD if case["kind"] == "adapter_fwd" else T.PASS_DX, adapters)
    return dict(grid=grid, dims=dims, adapters=adapters, ws=torch.empty(max(need, 256), dtype=torch.uint8, device="cuda"))


def _own_run(case, s):
    import paper_2110_14883_amd as T

    h = s.get("handles")
    if h is None:
        h = s["handles"] = _handles(T, case, s)
    kind = case["kind"]
    if kind.startswith("drop"):
        drop = T.Dropout(1.0 - case["keep"], s["seed"], s["offset"], row0=case["row0"], col0=case["col0"])
        if kind == "drop_fwd":
            epi = {"none": T.EPI_NONE, "bias": T.EPI_BIAS, "gelu": T.EPI_BIAS_GELU}[case["act"]]
            T.tp_dropout_fwd(drop, s["x"], s["bias"], epi, s["y"], residual=s["residual"], preact=s["pre"])
            return dict(y=s["y"], pre=s["pre"])
        T.tp_dropout_bwd(drop, s["dy"], s["dx"], preact=s["pre"], db=s["db"], workspace=h["ws"])
        return dict(dx=s["dx"], db=s["db"])
    drop = T.Dropout(1.0 - case["keep"], s["seed"], s["offset"]) if case["keep"] < 1 else None
    if kind == "adapter_fwd":
        epi = {"none": T.EPI_NONE, "bias": T.EPI_BIAS, "gelu": T.EPI_BIAS_GELU}[case["act"]]
        T.tp_adapter_fwd(h["grid"], h["dims"], len(s["x"]), h["adapters"], s["x"], s["a"], s["b"], s["c"], s["bias"], epi, s["y"], preact=s["pre"],
                         v=s["v"], dropout=drop, workspace=h["ws"])
        return dict(y=s["y"], v=s["v"], pre=s["pre"])
    T.tp_adapter_bwd(h["grid"], h["dims"], len(s["dy"]), h["adapters"], s["dy"], s["b"], a=s["a"], dx_base=s["c"], dx=s["dx"], x_own=s["x"], da=s["da"],
                     dy_own=s["dy"][s["own_dy"]], v=s["v"], db=s["db"], dropout=drop, workspace=h["ws"])
    return dict(dx=s["dx"], da=s["da"], db=s["db"])


_PLAIN = dict(drop_fwd=_plain_drop_fwd, drop_bwd=_plain_drop_bwd, adapter_fwd=_plain_adapter_fwd, adapter_bwd=_plain_adapter_bwd)


def run(state):
    case = state["case"]
    if own:
        return _own_run(case, state)
    return _PLAIN[case["kind"]](case, state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    size = lambda name: 4 if name == "f32" else 2
    if case["kind"].startswith("drop"):
        n = case["rows"] * case["cols"]
        if case["kind"] == "drop_fwd":
            each = size(case["x"]) + size(case["y"]) + (2 if case["residual"] else 0) + (2 if case["pre"] else 0)
            return dict(bytes=n * each + 2 * case["cols"], flops=2 * n)
        return dict(bytes=n * (6 if case["act"] == "gelu" else 4) + 4 * case["cols"], flops=2 * n)
    m, k, n, steps, row, col = _share(case)
    rows, r, used = m - case["tail"], case["rank"], min(case["pool"], case["requests"])
    if case["kind"] == "adapter_fwd":
        each = 2 * k * steps + n * (size(case["c"]) + size(case["y"]) + (2 if case["act"] == "gelu" else 0)) + 4 * r
        return dict(bytes=rows * each + used * r * (k * steps + n) * 2, flops=2 * rows * r * (k * steps + n))
    each = 2 * n * steps + 2 * k + k * (size(case["c"]) + size(case["y"])) + 4 * r
    return dict(bytes=rows * each + used * r * (n * steps + k) * 2 + case["pool"] * r * (k + n) * 4, flops=2 * rows * r * (n * steps + k + k + n))


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits
def _exact_kept(case, s, rows, cols, row0, col0):
    """The factors, from the generator written with products of 16-bit halves (nothing wraps)."""
    def wide(x, c):                       # (high, low) words of x c
        x0, x1, c0, c1 = x & 0xFFFF, x >> 16, c & 0xFFFF, c >> 16
        low = x0 * c0
        mid = x1 * c0 + (low >> 16)
        mid2 = x0 * c1 + (mid & 0xFFFF)
        return x1 * c1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)

    t = round((1.0 - case["keep"]) * 65536)
    out = torch.empty(rows, cols // 8, 8, dtype=torch.float64, device="cuda")
    for first in range(0, rows, 4096):
        n = min(4096, rows - first)
        x0 = torch.arange(col0 // 8, col0 // 8 + cols // 8, device="cuda").repeat(n, 1)
        x1 = torch.arange(row0 + first, row0 + first + n, device="cuda")[:, None].repeat(1, cols // 8)
        x2 = torch.zeros_like(x0) + (s["offset"] % (1 << 32))
        x3 = torch.zeros_like(x0) + (s["offset"] // (1 << 32))
        k0, k1 = s["seed"] % (1 << 32), s["seed"] // (1 << 32)
        for _ in range(10):
            h0, l0 = wide(x0, 0xD2511F53)
            h2, l2 = wide(x2, 0xCD9E8D57)
            x0, x1, x2, x3 = h2 ^ x1 ^ k0, l2, h0 ^ x3 ^ k1, l0
            k0, k1 = (k0 + 0x9E3779B9) % (1 << 32), (k1 + 0xBB67AE85) % (1 << 32)
        for w, x in enumerate((x0, x1, x2, x3)):
            for h in range(2):
                u = (x // (1 << 16 * h)) % 65536
                out[first:first + n, :, 2 * w + h] = torch.where(u < t, 0.0, 65536.0 / (65536 - t)).double()
    # (the factor is a number of 32 bits in the definition's use: 65536 / (65536 - T) itself here)
    exact = torch.tensor(65536.0 / (65536 - t), dtype=torch.float64, device="cuda")
    return torch.where(out > 0, exact, out).view(rows, cols)


def exact(case, seed):
    s = prepare(case, seed)
    half = math.sqrt(0.5)
    phi = lambda a: 0.5 * torch.special.erfc(-a * half)
    if case["kind"].startswith("drop"):
        keep = _exact_kept(case, s, case["rows"], case["cols"], case["row0"], case["col0"])
        if case["kind"] == "drop_fwd":
            a = s["x"].double()
            if s["bias"] is not None:
                a += s["bias"].double()
            z = (a * phi(a) if case["act"] == "gelu" else a) * keep
            if s["residual"] is not None:
                z += s["residual"].double()
            return dict(y=z, pre=a if case["pre"] else None)
        g = s["dy"].double() * keep
        if s["pre"] is not None:
            a = s["pre"].double()
            g *= phi(a) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
        return dict(dx=g, db=None if s["db"] is None else g.sum(0))
    m, k, n, steps, row, col = _share(case)
    cuts, ids, scale = s["offsets"].tolist(), s["ids"].tolist(), s["scale"].double()
    pool = case["pool"]
    if case["kind"] == "adapter_fwd":
        y, v = s["y"].double(), s["v"].double()
        pre = s["pre"].double() if s["pre"] is not None else None
        x = [t.double() for t in s["x"]]
        if case["keep"] < 1:
            x = [t * _exact_kept(case, s, m, k, row * m, (col if case["mode"] == "1d_row" else i) * k) for i, t in enumerate(x)]
        for lo, hi, i in zip(cuts, cuts[1:], ids):
            if hi == lo:
                continue
            a = s["c"][lo:hi].double()
            if 0 <= i < pool:
                v[lo:hi] = sum(t[lo:hi] @ f[i].double().t().contiguous() for t, f in zip(x, s["a"]))
                a = a + scale[i] * (v[lo:hi] @ s["b"][i].double())
            if s["bias"] is not None:
                a = a + s["bias"].double()
            if pre is not None:
                pre[lo:hi] = a
            y[lo:hi] = a * phi(a) if case["act"] == "gelu" else a
        return dict(y=y, v=v, pre=pre)
    dx = s["dx"].double()
    da, db = torch.zeros_like(s["da"], dtype=torch.float64), torch.zeros_like(s["db"], dtype=torch.float64)
    keep = _exact_kept(case, s, m, k, row * m, col * k) if case["keep"] < 1 else torch.ones(1, 1, dtype=torch.float64, device="cuda").expand(m, k)
    for lo, hi, i in zip(cuts, cuts[1:], ids):
        if hi == lo:
            continue
        dx[lo:hi] = s["c"][lo:hi].double()
        if 0 <= i < pool:
            u = scale[i] * sum(t[lo:hi].double() @ f[i].double().t().contiguous() for t, f in zip(s["dy"], s["b"]))
            dx[lo:hi] += (u @ s["a"][i].double()) * keep[lo:hi]
            da[i] += u.t().contiguous() @ (s["x"][lo:hi].double() * keep[lo:hi])
            db[i] += scale[i] * (s["v"][lo:hi].double().t().contiguous() @ s["dy"][s["own_dy"]][lo:hi].double())
    return dict(dx=dx, da=da, db=db)
