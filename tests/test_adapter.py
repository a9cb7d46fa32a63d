"""Low-rank adapters beside the shared projection: forward and backward against 64 bits over ranks, extents, segment layouts, grids and types; what the
calls refuse; partial sums over ranks, captured graphs, dropout inside the products, and a training step and a serving step put together."""
import math

import pytest
import torch

import paper_2110_14883_amd as T
from paper_2110_14883_amd import binding as B
from test_dropout import factor, gelu64, keep_mask

E24 = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------------ on the host
def _st(fn):
    try:
        fn()
    except T.TpError as e:
        return e.status
    return 0


G1 = T.Grid(T.MODE_1D_COL)
AD = T.Adapters(0x100, 0x200, 4, 16, 0x300, 2)
X, A, Bf, C, Y = (0x10000, 64), (0x20000, 64, 1024), (0x30000, 128, 2048), (0x40000, 128, B.DT_BF16), (0x80000, 128, B.DT_BF16)
WS = (0x1000000, 1 << 30)


def _fwd(**k):
    return _st(lambda: T.tp_adapter_fwd(k.get("grid", G1), k.get("dims", (32, 64, 128)), k.get("steps", 1), k.get("ad", AD), k.get("x", [X]), k.get("a", [A]),
                                        k.get("b", Bf), k.get("c", C), k.get("bias"), k.get("epi", T.EPI_NONE), k.get("y", Y), preact=k.get("pre"), v=k.get("v"),
                                        dropout=k.get("drop"), workspace=k.get("ws", WS), stream=0))


def _bwd(**k):
    return _st(lambda: T.tp_adapter_bwd(k.get("grid", G1), k.get("dims", (32, 64, 128)), k.get("steps", 1), k.get("ad", AD), k.get("dy", [(0x10000, 128)]),
                                        k.get("bs", [Bf]), a=k.get("a", A), dx_base=k.get("base", (0x40000, 64, 0)), dx=k.get("dx", (0x80000, 64, 0)),
                                        x_own=k.get("x", X), da=k.get("da", (0x90000, 64, 1024)), dy_own=k.get("own", (0x10000, 128)), v=k.get("v", 0xA0000),
                                        db=k.get("db", (0xB0000, 128, 2048)), dropout=k.get("drop"), workspace=k.get("ws", WS), stream=0))


def test_refusals_forward():
    """All found on the host, addresses are never followed."""
    ad = lambda **k: AD._replace(**k)
    assert _fwd(ad=ad(n_segments=-1)) == 4 and _fwd(ad=ad(n_adapters=0)) == 4 and _fwd(ad=ad(n_adapters=40000)) == 4
    assert _fwd(ad=ad(rank=0)) == 4 and _fwd(ad=ad(rank=136)) == 4 and _fwd(ad=ad(rank=12)) == 5
    assert _fwd(ad=ad(offsets=0)) == 1 and _fwd(ad=ad(ids=0)) == 1 and _fwd(ad=ad(offsets=0x102)) == 5 and _fwd(ad=ad(scale=0x301)) == 5
    assert _fwd(steps=0) == 4 and _fwd(steps=2) == 4 and _fwd(grid=T.Grid(77)) == 2 and _fwd(dims=(0, 64, 128)) == 4
    assert _fwd(x=None) == 1 and _fwd(x=[]) == 1 and _fwd(a=None) == 1 and _fwd(a=[None]) == 1 and _fwd(b=None) == 1
    assert _fwd(x=[(0x10008, 64)]) == 5 and _fwd(x=[(0x10000, 56)]) == 4 and _fwd(a=[(0x20000, 60, 1024)]) == 5 and _fwd(a=[(0x20000, 56, 1024)]) == 4
    assert _fwd(a=[(0x20000, 64, 1020)]) == 5 and _fwd(a=[(0x20000, 64, 1016)]) == 4 and _fwd(b=(0x30000, 128, 0)) == 4
    assert _fwd(c=None) == 1 and _fwd(y=None) == 1 and _fwd(c=(0x40000, 128, 5)) == 6 and _fwd(y=(0x80000, 128, 5)) == 6
    assert _fwd(epi=9) == 2 and _fwd(epi=T.EPI_BIAS) == 1 and _fwd(epi=T.EPI_BIAS, bias=0x8) == 5 and _fwd(v=0x8) == 5
    assert _fwd(pre=(0xC0000, 128, B.DT_F32)) == 6
    # y over c: the same block, or apart
    for y in ((0x40000, 128, B.DT_F32), (0x40010, 128, B.DT_BF16), (0x40000, 136, B.DT_BF16), (0x40000 + 31 * 256, 128, B.DT_BF16)):
        assert _fwd(y=y) == 4
    assert T.tp_adapter_workspace_size(G1, (32, 64, 128), T.PASS_FWD, AD) == 32 * 16 * 4
    assert _fwd(ws=None) == 7 and _fwd(ws=(0x1000008, 1 << 30)) == 7 and _fwd(ws=(0x1000000, 2047)) == 7
    assert _fwd(drop=T.Dropout(1.5, 1)) == 2 and _fwd(drop=T.Dropout(0.5, 1, col0=4)) == 5 and _fwd(drop=T.Dropout(0.5, 1, row0=2 ** 32 - 31)) == 4
    row = T.Grid(T.MODE_1D_ROW, p=2)
    f = dict(grid=row, dims=(32, 128, 128))
    assert _fwd(y=Y, **f) == 6 and _fwd(y=(0x80000, 128, 1), epi=T.EPI_BIAS, bias=0x100, **f) == 2 and _fwd(y=(0x80000, 128, 1), pre=(0xC0000, 128, 0), **f) == 2
    assert _fwd(ad=ad(n_segments=0)) == 0                # nothing to do
    # more tiles than a launch has threads for
    many = dict(dims=(1 << 23, 64, 128), ws=(0x1000000, 1 << 50), c=(0x4000000000, 128, 0), y=(0x8000000000, 128, 0))
    assert _fwd(ad=ad(n_segments=1 << 23), **many) == 4


def test_refusals_backward():
    ad = lambda **k: AD._replace(**k)
    assert _bwd(ad=ad(rank=20)) == 5 and _bwd(ad=ad(ids=0)) == 1 and _bwd(steps=2) == 4 and _bwd(steps=0) == 4
    assert _bwd(dy=None) == 1 and _bwd(bs=None) == 1 and _bwd(a=None) == 1 and _bwd(base=None) == 1 and _bwd(x=None) == 1 and _bwd(own=None) == 1 and _bwd(v=None) == 1
    assert _bwd(da=(0x90000, 64, 1000)) == 4 and _bwd(da=(0x90000, 60, 1024)) == 5 and _bwd(db=(0xB0004, 128, 2048)) == 5 and _bwd(v=0xA0004) == 5
    assert _bwd(dx=(0x40020, 64, 0)) == 4 and _bwd(dx=(0x80000, 64, 7)) == 6 and _bwd(ws=None) == 7 and _bwd(drop=T.Dropout(float("nan"), 1)) == 2
    assert _bwd(grid=T.Grid(T.MODE_1D_COL, p=2), dims=(32, 64, 256)) == 6          # a partial dX in bf16
    assert _bwd(ad=ad(n_adapters=32767, n_segments=1 << 20), dims=(32, 1 << 18, 1 << 18), dy=[(0x10000, 1 << 18)], bs=[(0x10000, 1 << 18, 1 << 22)],
                own=(0x10000, 1 << 18)) == 4             # more workgroups than a launch has threads for
    none = dict(dx=None, da=None, db=None)
    assert _bwd(dy=None, bs=None, a=None, base=None, x=None, own=None, v=None, ws=None, **none) == 0


def test_workspace_bounds():
    """At most 16 planes of V, and for backward 32 of dA and dB besides; nothing for a prefix or another pass; grows with nothing but the extents."""
    for m, h, f, n, pool, r in ((1, 4096, 4096, 1, 1, 8), (16384, 4096, 4096, 1, 1, 128), (4096, 1024, 512, 4096, 64, 16), (100000, 64, 64, 3, 3, 8)):
        a = T.Adapters(None, None, pool, r, None, n)
        fw = T.tp_adapter_workspace_size(G1, (m, h, f), T.PASS_FWD, a)
        bw = T.tp_adapter_workspace_size(G1, (m, h, f), T.PASS_DX, a)
        assert 0 < fw <= 16 * m * r * 4 + 256 and 0 < bw <= 16 * m * r * 4 + 32 * pool * r * (h + f) * 4 + 4 * pool + 1024
    assert T.tp_adapter_workspace_size(G1, (64, 64, 64), T.PASS_DW, AD) == 0 and T.tp_adapter_workspace_size(G1, (0, 64, 64), T.PASS_FWD, AD) == 0
    assert T.tp_adapter_workspace_size(G1, (64, 64, 64), T.PASS_FWD, AD._replace(rank=9)) == 0


def test_tensors_of_the_wrong_kind_are_refused():
    """Before anything is launched: host tensors, other types, arrays that are too short."""
    i32, bad = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    call = lambda **k: T.tp_adapter_fwd(G1, (32, 64, 128), 1, k.get("ad", AD), k.get("x", [X]), k.get("a", [A]), Bf, C, None, 0, k.get("y", Y), workspace=WS, stream=0)
    for k in (dict(ad=AD._replace(offsets=i32)), dict(x=[torch.zeros(32, 64, dtype=BF)]), dict(a=[torch.zeros(4, 16, 64, dtype=BF)]), dict(y=torch.zeros(32, 128, dtype=BF))):
        with pytest.raises(ValueError, match="not on the GPU"):
            call(**k)
    for ad in ((1, 2, 3), AD._replace(n_segments="x")):
        with pytest.raises((ValueError, TypeError)):
            call(ad=ad)
    assert bad.dtype == torch.int64


# ------------------------------------------------------------------------------------------------ on the GPU
def _g(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _strided(g, *shape, std=1.0, dtype=BF, pad=8):
    """Random values in a block whose rows (and adapters) lie further apart than they are long."""
    big = list(shape)
    big[-1] += pad
    if len(big) == 3:
        big[1] += 1
    t = (torch.randn(big, generator=g, device="cuda") * std).to(dtype)
    return t[..., :shape[-1]] if len(big) == 2 else t[:, :shape[1], :shape[2]]


def _out(*shape, dtype, pad=8):
    big = list(shape)
    big[-1] += pad
    return torch.full(big, 7.0, dtype=dtype, device="cuda")[..., :shape[-1]]


def _cuts(kind, m):
    """offsets of the segments, ids over a pool of three (-1 and 9: none)."""
    if kind == "one":
        return [0, m], [1]
    if kind == "single rows":
        return list(range(m + 1)), [(i * 7 % 5) - 1 for i in range(m)]
    if kind == "gaps and empties":                       # rows before the first and behind the last segment, empty ones between
        a, b, c = m // 7, m // 2, m - m // 5
        return [a, a, b, b, b, c, c], [0, 2, 1, 9, 2, 0]
    if kind == "many":                                   # more segments than lanes, ragged, the same adapter again and again
        cuts = [min(m, i * m // 130 + (i % 3)) for i in range(131)]
        return sorted(cuts), [i % 4 - 1 for i in range(130)]
    raise KeyError(kind)


def _share(grid, dims):
    f, x = T.tp_block_map(grid, dims, T.PASS_FWD), T.tp_block_map(grid, dims, T.PASS_DX)
    return f, x


def check(got, ref, tol, what):
    got, ref, tol = got.double(), ref.double(), tol.double() if torch.is_tensor(tol) else tol
    bad = ~((got - ref).abs() <= tol + 1e-30)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst by {float(((got - ref).abs() - tol).nan_to_num(1e30).max()):.3g}"


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def run_case(grid, dims, rank, kind, c_type=BF, y_type=BF, epi=T.EPI_NONE, p=0.0, scale=True, seed=0, steps=None, in_place=False):
    """Forward and backward of one rank's share, every element.  Tolerances: a sum of K products in fp32 is off by at most (K / 8 + 64) 2^-24 of the
    sum of magnitudes (32 products a matrix instruction, then chains over instructions, waves and planes); V as bf16 terms by 2^-17 (bf16 result) or
    2^-24 (fp32 result) of it; each result by half a step of its type and 8 2^-24 of its addends."""
    f, xm = _share(grid, dims)
    m, n, k = f["m"], f["n"], f["k"]
    steps = steps or f["n_steps"]
    g = _g(seed + 100 * rank + m)
    offsets, ids = _cuts(kind, m)
    pool = 3
    dev = lambda v, t=torch.int32: torch.tensor(v, dtype=t, device="cuda")
    s = [0.5, 2.0, -1.25] if scale else [1.0] * 3
    ad = T.Adapters(dev(offsets), dev(ids), pool, rank, dev(s, F32) if scale else None)
    drop = T.Dropout(p, 1234567 + seed, 89, row0=3, col0=16) if p else None
    xs = [_strided(g, m, k) for _ in range(steps)]
    As = [_strided(g, pool, rank, k, std=1 / math.sqrt(k)) for _ in range(steps)]
    Bn = _strided(g, pool, rank, n, std=1 / math.sqrt(rank))
    c, bias = _strided(g, m, n, dtype=c_type), (_strided(g, 1, n)[0].contiguous() if epi else None)
    y = c if in_place else _out(m, n, dtype=y_type)
    base = c.clone()
    pre, v = _out(m, n, dtype=BF) if epi == T.EPI_BIAS_GELU else None, torch.full((m, rank), 7.0, device="cuda")
    need = T.tp_adapter_workspace_size(grid, dims, T.PASS_FWD, ad)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")          # (planes full of NaN before the call)
    T.tp_adapter_fwd(grid, dims, steps, ad, xs, As, Bn, c, bias, epi, y, preact=pre, v=v, dropout=drop, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()

    def kept(row, col, cols):
        if not p:
            return torch.ones(m, cols, dtype=torch.float64, device="cuda")
        return torch.from_numpy(keep_mask((p, drop.seed, drop.offset, drop.row0 + row * m, drop.col0 + col * cols), m, cols)).cuda().double() * factor(p)

    x64 = [x.double() * kept(*f["a"][i], k) for i, x in enumerate(xs)]
    want_y, want_v, tol_y, tol_v = (torch.full(t, 7.0, dtype=torch.float64, device="cuda") for t in ((m, n), (m, rank), (m, n), (m, rank)))
    tol_y.zero_(); tol_v.zero_()
    if in_place:
        want_y = base.double()
    want_pre = torch.full((m, n), 7.0, dtype=torch.float64, device="cuda")
    sum_off = lambda terms: (terms / 8 + 64) * E24
    split_off = 2.0 ** -17 if y.dtype == BF else E24
    for lo, hi, i in zip(offsets, offsets[1:], ids):
        if hi <= lo:
            continue
        a, t = base[lo:hi].double(), torch.zeros(hi - lo, n, dtype=torch.float64, device="cuda")
        mag = a.abs()
        if 0 <= i < pool:
            want_v[lo:hi] = sum(x[lo:hi] @ q[i].double().t().contiguous() for x, q in zip(x64, As))
            tol_v[lo:hi] = sum(x[lo:hi].abs() @ q[i].double().abs().t().contiguous() for x, q in zip(x64, As)) * sum_off(k * steps)
            b64 = Bn[i].double() * s[i]
            a = a + want_v[lo:hi] @ b64
            big = want_v[lo:hi].abs() @ b64.abs()
            t = tol_v[lo:hi] @ b64.abs() + big * (split_off + sum_off(rank))
            mag = mag + big
        if epi:
            a, mag = a + bias.double(), mag + bias.double().abs()
        t = t + 8 * E24 * mag
        want_pre[lo:hi], t_pre = a, t
        if epi == T.EPI_BIAS_GELU:
            check(pre[lo:hi], a, t_pre + half_step(BF) * (a.abs() + t_pre), "preact")
            a, t = gelu64(a), 1.13 * t + 3e-7 * (1 + a.abs())
        want_y[lo:hi], tol_y[lo:hi] = a, t + half_step(y.dtype) * (a.abs() + t)
    check(v, want_v, tol_v, "V")
    check(y, want_y, tol_y, "Y")
    if not in_place:
        assert (torch.as_strided(y, (m, 8), (y.stride(0), 1), n) == 7).all()

    # ---- backward
    kx, nx = xm["k"], xm["n"]
    back_steps = min(steps, xm["n_steps"])
    dys = [_strided(g, m, kx) for _ in range(back_steps)]
    Bs = [_strided(g, pool, rank, kx, std=1 / math.sqrt(kx)) for _ in range(back_steps)]
    Ax, xo, vo = _strided(g, pool, rank, nx, std=1 / math.sqrt(rank)), _strided(g, m, nx), torch.randn(m, rank, generator=g, device="cuda")
    dyo = _strided(g, m, n)
    dx_type = F32 if xm["partial"] else y_type
    dxb = _strided(g, m, nx, dtype=c_type)
    dx = _out(m, nx, dtype=dx_type)
    da, db = (_out(pool, rank, cols, dtype=F32) for cols in (nx, n))
    need = T.tp_adapter_workspace_size(grid, dims, T.PASS_DX, ad)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    T.tp_adapter_bwd(grid, dims, back_steps, ad, dys, Bs, a=Ax, dx_base=dxb, dx=dx, x_own=xo, da=da, dy_own=dyo, v=vo, db=db, dropout=drop, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()
    keep = kept(*xm["out"], nx)
    want = torch.full((m, nx), 7.0, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(want)
    grads = {name: torch.zeros(pool, rank, cols, dtype=torch.float64, device="cuda") for name, cols in (("da", nx), ("db", n), ("ta", nx), ("tb", n))}
    for lo, hi, i in zip(offsets, offsets[1:], ids):
        if hi <= lo:
            continue
        want[lo:hi] = dxb[lo:hi].double()
        mag = want[lo:hi].abs()
        if 0 <= i < pool:
            u = sum(d[lo:hi].double() @ q[i].double().t().contiguous() for d, q in zip(dys, Bs))
            tu = sum(d[lo:hi].double().abs() @ q[i].double().abs().t().contiguous() for d, q in zip(dys, Bs)) * sum_off(kx * back_steps)
            a64 = Ax[i].double() * s[i]
            want[lo:hi] += (u @ a64) * keep[lo:hi]
            big = (u.abs() @ a64.abs()) * keep[lo:hi]
            tol[lo:hi] = (tu @ a64.abs()) * keep[lo:hi] + big * ((2.0 ** -17 if dx_type == BF else E24) + sum_off(rank))
            mag = mag + big
            xk, dk, vk = xo[lo:hi].double() * keep[lo:hi], dyo[lo:hi].double(), vo[lo:hi].double()
            grads["da"][i] += s[i] * (u.t().contiguous() @ xk)
            grads["db"][i] += s[i] * (vk.t().contiguous() @ dk)
            grads["ta"][i] += abs(s[i]) * ((u.abs() * (sum_off(m) + E24) + tu).t().contiguous() @ xk.abs())
            grads["tb"][i] += abs(s[i]) * (sum_off(m) + E24) * (vk.abs().t().contiguous() @ dk.abs())
        tol[lo:hi] += 8 * E24 * mag
    tol = tol + half_step(dx_type) * (want.abs() + tol) * (want != 7)
    check(dx, want, tol, "dX")
    check(da, grads["da"], grads["ta"] * 1.01, "dA")
    check(db, grads["db"], grads["tb"] * 1.01, "dB")
    # a second call that adds, and one output alone: the same sums
    da2, db2 = da.clone(), torch.full_like(db, 7.0)
    T.tp_adapter_bwd(grid, dims, back_steps, ad, dys, Bs, x_own=xo, da=da2, dropout=drop, accumulate=True, workspace=ws[:need])
    T.tp_adapter_bwd(grid, dims, 0, ad, dy_own=dyo, v=vo, db=db2, workspace=ws[:need])
    assert torch.equal(da2, da + da) and torch.equal(db2, db)


KINDS = ["one", "single rows", "gaps and empties", "many"]


@pytest.mark.gpu
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("kind", KINDS)
def test_ranks_and_segments(rank, kind):
    run_case(T.Grid(T.MODE_1D_COL), (150, 264, 136), rank, kind, seed=1)


@pytest.mark.gpu
@pytest.mark.parametrize("m,h,f", [(1, 8, 8), (1, 4096, 1024), (2, 24, 2056), (15, 64, 128), (17, 1032, 40), (33, 200, 512), (64, 2048, 256), (65, 520, 640), (700, 8, 8),
                                   (1025, 96, 1096), (3000, 328, 24)])
@pytest.mark.parametrize("rank,kind,p", [(16, "one", 0.0), (8, "gaps and empties", 0.3), (64, "one", 0.5)])
def test_extents(m, h, f, rank, kind, p):
    run_case(T.Grid(T.MODE_1D_COL), (m, h, f), rank, kind, p=p, seed=2)


@pytest.mark.gpu
@pytest.mark.parametrize("m,h,f,rank,kind,p", [
    (130, 64, 5000, 16, "single rows", 0.0), (70, 4096, 4104, 48, "single rows", 0.0),       # many strips a wave in one launch
    (3, 16384, 2056, 128, "one", 0.0), (40, 9000, 264, 128, "single rows", 0.0),             # factors too large for that
    (40, 136, 264, 16, "single rows", 0.4),                                                  # and dropout
    (9000, 136, 1288, 16, "many", 0.2), (9000, 136, 640, 64, "gaps and empties", 0.0), (5000, 72, 1160, 128, "many", 0.0), (20000, 328, 520, 8, "one", 0.1),
    (1300, 40, 4104, 32, "gaps and empties", 0.3)])
def test_every_plan(m, h, f, rank, kind, p):
    run_case(T.Grid(T.MODE_1D_COL), (m, h, f), rank, kind, y_type=F32 if rank % 16 else BF, p=p, seed=15)


@pytest.mark.gpu
@pytest.mark.parametrize("q,h,p", [(9, 40, 0.0), (9, 72, 0.3), (16, 8, 0.0)])
def test_many_short_steps(q, h, p):
    """More steps than waves, fewer units than waves, units that end inside a step."""
    run_case(T.Grid(T.MODE_2D, q=q, ri=1, rj=q - 1), (q * 37, q * h, q * 48), 16, "gaps and empties", p=p, seed=16)
    run_case(T.Grid(T.MODE_2D, q=q, ri=1, rj=q - 1), (q * 37, q * h, q * 48), 72, "single rows", p=p, seed=17)


@pytest.mark.gpu
def test_no_segments_and_everything_dropped():
    m, h, n, rank = 50, 72, 136, 16
    g = _g(18)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c, dy = (t.contiguous() for t in (_strided(g, m, h), _strided(g, 2, rank, h), _strided(g, 2, rank, n), _strided(g, m, n), _strided(g, m, n)))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def both(ad, drop, x):
        y, v, dx = torch.full((m, n), 7.0, dtype=BF, device="cuda"), torch.full((m, rank), 7.0, device="cuda"), torch.full((m, h), 7.0, dtype=BF, device="cuda")
        da, db = torch.full((2, rank, h), 7.0, device="cuda"), torch.full((2, rank, n), 7.0, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v, dropout=drop, workspace=ws)
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=c[:, :h], dx=dx, x_own=x, da=da, dy_own=dy, v=v, db=db, dropout=drop, workspace=ws)
        return y, v, dx, da, db

    for ad in (T.Adapters(i32([0]), i32([]), 2, rank), T.Adapters(i32([0, 0, 0]), i32([0, 1]), 2, rank)):
        y, v, dx, da, db = both(ad, None, x)
        assert (y == 7).all() and (v == 7).all() and (dx == 7).all() and (da == 0).all() and (db == 0).all()
    y, v, dx, da, db = both(T.Adapters(i32([0, m]), i32([1]), 2, rank), T.Dropout(1.0, 3), x * float("nan"))
    assert torch.equal(y, c) and (v == 0).all() and torch.equal(dx, c[:, :h]) and (da == 0).all() and (db == 0).all()
    # NaN and infinities where the mask drops them
    drop, ad = T.Dropout(0.5, 4, 5), T.Adapters(i32([0, 20, m]), i32([1, 0]), 2, rank)
    keep = torch.from_numpy(keep_mask((0.5, 4, 5, 0, 0), m, h)).cuda()
    clean = torch.where(keep, x, torch.zeros_like(x))
    dirty = torch.where(keep, x, torch.tensor([float("nan"), float("inf")], device="cuda").repeat(h // 2).to(BF))
    for s, t in zip(both(ad, drop, clean), both(ad, drop, dirty)):
        assert torch.equal(s, t) and torch.isfinite(t).all()


@pytest.mark.gpu
@pytest.mark.parametrize("c_type", [BF, F32])
@pytest.mark.parametrize("y_type", [BF, F32])
@pytest.mark.parametrize("epi", [T.EPI_NONE, T.EPI_BIAS, T.EPI_BIAS_GELU])
@pytest.mark.parametrize("rank", [16, 48])
def test_types_and_epilogues(c_type, y_type, epi, rank):
    run_case(T.Grid(T.MODE_1D_COL), (97, 136, 200), rank, "gaps and empties", c_type, y_type, epi, scale=False, seed=3)
    if c_type == y_type:
        run_case(T.Grid(T.MODE_1D_COL), (97, 136, 200), rank, "gaps and empties", c_type, y_type, epi, seed=4, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("name,grid,dims", [
    ("1D column", T.Grid(T.MODE_1D_COL, p=4, ri=2), (70, 64, 4 * 136)), ("1D row", T.Grid(T.MODE_1D_ROW, p=4, ri=3), (70, 4 * 72, 136)),
    ("2D", T.Grid(T.MODE_2D, q=3, ri=1, rj=2), (3 * 50, 3 * 72, 3 * 104)), ("2.5D", T.Grid(T.MODE_2P5D, q=2, d=2, ri=1, rj=0, rk=1), (4 * 77, 2 * 40, 2 * 136)),
    ("3D", T.Grid(T.MODE_3D, p=2, ri=1, rj=0, rk=1), (4 * 61, 2 * 264, 2 * 88)), ("3D gathered", T.Grid(T.MODE_3D_GATHERED, p=2, ri=1, rj=0, rk=1), (4 * 30, 2 * 64, 2 * 88))])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_grids(name, grid, dims, p):
    partial = T.tp_block_map(grid, dims, T.PASS_FWD)["partial"]
    kw = dict(c_type=F32, y_type=F32) if partial else dict(epi=T.EPI_BIAS_GELU)
    run_case(grid, dims, 24, "gaps and empties", p=p, seed=5, **kw)
    if T.tp_block_map(grid, dims, T.PASS_FWD)["n_steps"] > 1:
        run_case(grid, dims, 32, "one", p=p, seed=6, steps=1, **kw)


@pytest.mark.gpu
def test_leading_dimensions_beyond_32_bit_offsets():
    """Rows 4 MiB apart (the largest leading dimension): byte offsets of a block pass 2^32."""
    m, k, n, rank, ld = 1100, 64, 72, 16, 1 << 21
    big = torch.empty(m * ld, dtype=BF, device="cuda")
    x, y, d = (big[o:].as_strided((m, c), (ld, 1)) for o, c in ((0, k), (1024, n), (2048, n)))
    g = _g(7)
    x.copy_(_strided(g, m, k)); d.copy_(_strided(g, m, n))
    a, b = _strided(g, 1, rank, k, std=0.1), _strided(g, 1, rank, n, std=0.3)
    c = _strided(g, m, n)
    ad = T.Adapters(torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 1, rank)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, k, n)
    ws = torch.empty(max(T.tp_adapter_workspace_size(grid, dims, q, ad) for q in (T.PASS_FWD, T.PASS_DX)), dtype=torch.uint8, device="cuda")
    v, v2 = (torch.empty(m, rank, device="cuda") for _ in range(2))
    y2 = torch.empty(m, n, dtype=BF, device="cuda")
    T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v, workspace=ws)
    T.tp_adapter_fwd(grid, dims, 1, ad, [x.contiguous()], [a], b, c, None, 0, y2, v=v2, workspace=ws)
    assert torch.equal(v, v2) and torch.equal(y.contiguous(), y2)
    out = [[torch.empty(1, rank, cols, device="cuda") for cols in (k, n)] for _ in range(2)]
    for xx, dd, o in ((x, d, out[0]), (x.contiguous(), d.contiguous(), out[1])):
        T.tp_adapter_bwd(grid, dims, 1, ad, [dd], [b], x_own=xx, da=o[0], dy_own=dd, v=v, db=o[1], workspace=ws)
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.gpu
def test_partials_over_ranks_sum_to_the_whole():
    """1D row cut: the ranks' parts, each with its own columns of X and A and the dropout of those, add up to what one rank computes on all of them."""
    m, h, n, rank, p = 90, 256, 136, 16, 4
    g = _g(8)
    x, a, b = _strided(g, m, h), _strided(g, 1, rank, h, std=0.1), _strided(g, 1, rank, n, std=0.3)
    ad = T.Adapters(torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 1, rank)
    drop, zero = T.Dropout(0.3, 5, 6), torch.zeros(m, n, device="cuda")
    whole, parts = torch.empty(m, n, device="cuda"), torch.zeros(m, n, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    T.tp_adapter_fwd(T.Grid(T.MODE_1D_COL), (m, h, n), 1, ad, [x], [a], b, zero, None, 0, whole, dropout=drop, workspace=ws)
    for r in range(p):
        cut = slice(r * h // p, (r + 1) * h // p)
        T.tp_adapter_fwd(T.Grid(T.MODE_1D_ROW, p=p, ri=r), (m, h, n), 1, ad, [x[:, cut]], [a[:, :, cut]], b, parts, None, 0, parts, dropout=drop, workspace=ws)
    check(parts, whole, 2.0 ** -18 * float(whole.abs().max()), "sum over ranks")


@pytest.mark.gpu
def test_gradients_by_differences():
    """y is linear in each factor: <dY, y(A + D) - y(A)> = <dA, D> and so on, D a change that bf16 holds exactly."""
    m, h, n, rank = 80, 72, 104, 16
    g = _g(9)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    offsets, ids = _cuts("gaps and empties", m)
    ad = T.Adapters(torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.tensor(ids, dtype=torch.int32, device="cuda"), 3, rank, torch.tensor([0.5, 2.0, -1.25], device="cuda"))
    r = lambda *shape: torch.randint(-8, 9, shape, generator=g, device="cuda").to(BF) / 8        # sums of these are exact in bf16
    x, a, b, dy, c = r(m, h), r(3, rank, h), r(3, rank, n), r(m, n), torch.zeros(m, n, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    drop, v = T.Dropout(0.5, 1, 2), torch.zeros(m, rank, device="cuda")

    def forward(x, a, b, v=None):
        y = torch.zeros(m, n, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v, dropout=drop, workspace=ws)
        return y.double()

    y0 = forward(x, a, b, v)
    dx, da, db = torch.zeros(m, h, device="cuda"), torch.empty(3, rank, h, device="cuda"), torch.empty(3, rank, n, device="cuda")
    T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=torch.zeros(m, h, device="cuda"), dx=dx, x_own=x, da=da, dy_own=dy, v=v, db=db, dropout=drop, workspace=ws)
    for grad, t, at in ((da, a, 1), (db, b, 2), (dx, x, 0)):
        d = r(*t.shape)
        args = [x, a, b]
        args[at] = t + d
        assert torch.equal((t.double() + d.double()), args[at].double())
        diff = (forward(*args) - y0)
        # both sides are sums of fp32 results: 2^-20 of the magnitudes added up
        lhs, rhs = (diff * dy.double()).sum(), (grad.double() * d.double()).sum()
        mag = ((diff.abs() + 2 * y0.abs()) * dy.double().abs()).sum() + (grad.double().abs() * d.double().abs()).sum()
        assert abs(float(lhs - rhs)) <= 2.0 ** -20 * float(mag)


@pytest.mark.gpu
def test_wild_offsets_and_ids_stay_inside():
    """Descending, negative and too large offsets and ids far out: whatever the rows get, nothing outside the blocks is touched, and the next good call is right."""
    m, h, n, rank = 60, 64, 136, 16
    g = _g(10)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c, dy = _strided(g, m, h), _strided(g, 2, rank, h), _strided(g, 2, rank, n), _strided(g, m, n), _strided(g, m, n)
    room = torch.full((3 * m, n + 8), 7.0, dtype=BF, device="cuda")
    y = room[m:2 * m, :n]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    for offsets, ids in (([50, 10, 55, -5, 2 ** 31 - 1], [0, 1, 2 ** 31 - 1, -2 ** 31]), ([-2 ** 31, 2 ** 31 - 1, 0, 60, 60], [1, 0, 1, 0]), ([60, 60, 60, 60, 60], [0, 0, 0, 0]),
                         ([0, 60, 0, 60, 0], [0, 1, 0, 1])):
        ad = T.Adapters(i32(offsets), i32(ids), 2, rank)
        v = torch.full((3 * m, rank), 7.0, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v[m:2 * m], workspace=ws)
        da, db, dx = torch.full((4, rank, h), 7.0, device="cuda"), torch.full((4, rank, n), 7.0, device="cuda"), torch.full((3 * m, h), 7.0, dtype=BF, device="cuda")
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=x, dx=dx[m:2 * m], x_own=x, da=da[1:3], dy_own=dy, v=v[m:2 * m], db=db[1:3], workspace=ws)
        assert (room[:m] == 7).all() and (room[2 * m:] == 7).all() and (room[:, n:] == 7).all() and (v[:m] == 7).all() and (v[2 * m:] == 7).all()
        assert (da[0] == 7).all() and (da[3] == 7).all() and (db[0] == 7).all() and (db[3] == 7).all() and (dx[:m] == 7).all() and (dx[2 * m:] == 7).all()
    run_case(grid, dims, rank, "gaps and empties", seed=11)


@pytest.mark.gpu
def test_infinities_stay_in_their_rows():
    """An infinite and a NaN row of X, and garbage behind the segments, leave the other rows and other adapters' gradients as they are."""
    m, h, n, rank = 40, 64, 72, 16
    g = _g(12)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c, dy = (t.contiguous() for t in (_strided(g, m, h), _strided(g, 2, rank, h), _strided(g, 2, rank, n), _strided(g, m, n), _strided(g, m, n)))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ad = T.Adapters(i32([0, 17, 30]), i32([0, 1]), 2, rank)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def both(x, dy):
        y, v = torch.full((m, n), 7.0, dtype=BF, device="cuda"), torch.full((m, rank), 7.0, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v, workspace=ws)
        dx, da, db = torch.full((m, h), 7.0, dtype=BF, device="cuda"), torch.empty(2, rank, h, device="cuda"), torch.empty(2, rank, n, device="cuda")
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=c[:, :h], dx=dx, x_own=x, da=da, dy_own=dy, v=v, db=db, workspace=ws)
        return y, v, dx, da, db

    good = both(x, dy)
    x2, dy2 = x.clone(), dy.clone()
    x2[3], x2[5], x2[30:], dy2[30:] = float("inf"), float("nan"), float("nan"), float("inf")
    bad = both(x2, dy2)
    ok = torch.ones(m, dtype=torch.bool, device="cuda")
    ok[[3, 5]] = False
    for i in (0, 1, 2):
        assert torch.equal(good[i][ok], bad[i][ok])
    assert not torch.isfinite(bad[1][3]).any() and torch.isnan(bad[1][5]).all() and not torch.isfinite(bad[0][3]).any()
    for i in (3, 4):
        assert torch.equal(good[i][1], bad[i][1]) and torch.isfinite(good[i]).all() and not torch.isfinite(bad[i][0]).any()


@pytest.mark.gpu
def test_captured_graph_follows_new_lengths():
    """One graph, replayed with other offsets, ids and inputs, on a stream of its own; eager calls on the same tensors between the replays."""
    m, h, n, rank = 200, 256, 264, 16
    g = _g(13)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c, dy = _strided(g, m, h), _strided(g, 3, rank, h), _strided(g, 3, rank, n), _strided(g, m, n), _strided(g, m, n)
    offsets, ids = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (7, 6))
    ad = T.Adapters(offsets, ids, 3, rank)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = T.Dropout(0.2, 1, 2, step)

    def buffers():
        return dict(y=torch.full((m, n), 7.0, dtype=BF, device="cuda"), v=torch.full((m, rank), 7.0, device="cuda"), dx=torch.full((m, h), 7.0, device="cuda"),
                    da=torch.empty(3, rank, h, device="cuda"), db=torch.empty(3, rank, n, device="cuda"),
                    ws=torch.empty(max(T.tp_adapter_workspace_size(grid, dims, q, ad) for q in (T.PASS_FWD, T.PASS_DX)), dtype=torch.uint8, device="cuda"))

    def both(t):
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, t["y"], v=t["v"], dropout=drop, workspace=t["ws"])
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=c[:, :h], dx=t["dx"], x_own=x, da=t["da"], dy_own=dy, v=t["v"], db=t["db"], dropout=drop, workspace=t["ws"])

    t, e = buffers(), buffers()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(t)
    for i, cuts in enumerate(([0, 1, 2, 3, 4, 5, 6], [0, 0, 100, 100, 180, 180, 200], [0, 200, 200, 200, 200, 200, 200], [20, 60, 61, 62, 150, 151, 170])):
        offsets.copy_(torch.tensor(cuts, dtype=torch.int32))
        ids.copy_(torch.tensor([(i + j) % 4 - 1 for j in range(6)], dtype=torch.int32))
        x.normal_(generator=g)
        step.fill_(i)
        for d in (t, e):
            for name in ("y", "v", "dx"):
                d[name].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        both(e)
        torch.cuda.synchronize()
        for name in ("y", "v", "dx", "da", "db"):
            assert torch.equal(t[name], e[name]), (i, name)


@pytest.mark.gpu
def test_fine_tuning_step_of_a_two_layer_share():
    """As a program uses them together: column-cut layer with an adapter (dropout on its input) and GeLU, row-cut layer with one, dropout and residual behind it; all
    gradients, against the same step in 64 bits from the same saved bf16 tensors."""
    M, H, F, rank = 150, 136, 264, 16
    g = _g(14)
    ga, gb = T.Grid(T.MODE_1D_COL), T.Grid(T.MODE_1D_ROW)
    da_, db_ = (M, H, F), (M, F, H)
    x, w1, w2 = _strided(g, M, H), _strided(g, H, F, std=0.1), _strided(g, F, H, std=0.1)
    b1, b2, res, dz = _strided(g, 1, F)[0].contiguous(), _strided(g, 1, H)[0].contiguous(), _strided(g, M, H), _strided(g, M, H)
    a1, f1, a2, f2 = (_strided(g, 2, rank, k, std=0.2) for k in (H, F, F, H))
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ad = T.Adapters(i32([0, 70, M]), i32([1, 0]), 2, rank, torch.tensor([1.5, 0.75], device="cuda"))
    d1, d2, d3 = T.Dropout(0.1, 9, 1), T.Dropout(0.1, 9, 2), T.Dropout(0.3, 9, 3)
    e = lambda r, c, t=BF: torch.empty(r, c, dtype=t, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    y1, pre1, h1, v1, y2, v2, out = e(M, F), e(M, F), e(M, F), e(M, rank, F32), e(M, H, F32), e(M, rank, F32), e(M, H)
    T.tp_linear_fwd(ga, da_, 1, [x], [w1], None, T.EPI_NONE, y1, None, ws)
    T.tp_adapter_fwd(ga, da_, 1, ad, [x], [a1], f1, y1, b1, T.EPI_BIAS_GELU, h1, preact=pre1, v=v1, dropout=d1, workspace=ws)
    T.tp_linear_fwd(gb, db_, 1, [h1], [w2], None, T.EPI_NONE, y2, None, ws)
    T.tp_adapter_fwd(gb, db_, 1, ad, [h1], [a2], f2, y2, None, T.EPI_NONE, y2, v=v2, dropout=d2, workspace=ws)
    T.tp_dropout_fwd(d3, y2, b2, T.EPI_BIAS, out, residual=res)
    # backward
    g2, db2 = e(M, H), torch.empty(H, device="cuda")
    T.tp_dropout_bwd(d3, dz, g2, db=db2, workspace=ws)
    dh, dw2, gr = e(M, F), e(F, H, F32), [torch.empty(2, rank, k, device="cuda") for k in (F, H, H, F)]
    T.tp_linear_bwd(gb, db_, 1, 1, da_row_blocks=[g2], w_blocks_dx=[w2], x_blocks_dw=[h1], da_col_blocks=[g2], dx=dh, dw=dw2, workspace=ws)
    T.tp_adapter_bwd(gb, db_, 1, ad, [g2], [f2], a=a2, dx_base=dh, dx=dh, x_own=h1, da=gr[0], dy_own=g2, v=v2, db=gr[1], dropout=d2, workspace=ws)
    dp, dx, dw1 = e(M, F), e(M, H), e(H, F, F32)
    T.tp_dgelu(dh, pre1, dp)
    T.tp_linear_bwd(ga, da_, 1, 1, da_row_blocks=[dp], w_blocks_dx=[w1], x_blocks_dw=[x], da_col_blocks=[dp], dx=dx, dw=dw1, workspace=ws)
    T.tp_adapter_bwd(ga, da_, 1, ad, [dp], [f1], a=a1, dx_base=dx, dx=dx, x_own=x, da=gr[2], dy_own=dp, v=v1, db=gr[3], dropout=d1, workspace=ws)

    # the same in 64 bits, each stage from the tensors that the stage before it left
    keep = lambda d, c: torch.from_numpy(keep_mask((d.p, d.seed, d.offset, 0, 0), M, c)).cuda().double() * factor(d.p)
    who, sc = [1] * 70 + [0] * (M - 70), [1.5, 0.75]
    rows = {i: torch.tensor([r for r in range(M) if who[r] == i], device="cuda") for i in (0, 1)}

    def adapted(v64, fac):
        o = torch.zeros(M, fac.shape[2], dtype=torch.float64, device="cuda")
        for i, r in rows.items():
            o[r] = sc[i] * (v64[r] @ fac[i].double())
        return o

    def low(z, fac):
        o = torch.zeros(M, rank, dtype=torch.float64, device="cuda")
        for i, r in rows.items():
            o[r] = z[r] @ fac[i].double().t().contiguous()
        return o

    def pair(l, r64):
        return torch.stack([sc[i] * (l[r].t().contiguous() @ r64[r]) for i, r in sorted(rows.items())])

    def close(got, ref, rel, what):      # norm-wise: bf16 tensors between the stages round at 2^-8
        off = float((got.double() - ref).norm() / ref.norm())
        assert off <= rel, (what, off)

    x64, h64 = x.double(), h1.double()
    p1 = x64 @ w1.double() + adapted(low(x64 * keep(d1, H), a1), f1) + b1.double()
    close(pre1, p1, 2.0 ** -7, "pre")
    close(h1, gelu64(p1), 2.0 ** -7, "h")
    z2 = h64 @ w2.double() + adapted(low(h64 * keep(d2, F), a2), f2)
    close(y2, z2, 2.0 ** -18, "y2")
    close(out, (z2 + b2.double()) * keep(d3, H) + res.double(), 2.0 ** -8, "out")
    q2 = dz.double() * keep(d3, H)
    close(g2, q2, 2.0 ** -8, "g2"); close(db2, q2.sum(0), 2.0 ** -18, "db2")
    g64 = g2.double()
    u2 = low(g64, f2)
    close(dh, g64 @ w2.double().t().contiguous() + adapted(u2, a2) * keep(d2, F), 2.0 ** -7, "dh")
    close(gr[0], pair(u2, h64 * keep(d2, F)), 2.0 ** -18, "dA2"); close(gr[1], pair(v2.double(), g64), 2.0 ** -18, "dB2")
    p64 = dp.double()
    u1 = low(p64, f1)
    close(dx, p64 @ w1.double().t().contiguous() + adapted(u1, a1) * keep(d1, H), 2.0 ** -7, "dx")
    close(gr[2], pair(u1, x64 * keep(d1, H)), 2.0 ** -18, "dA1"); close(gr[3], pair(v1.double(), p64), 2.0 ** -18, "dB1")
    close(dw1, x64.t().contiguous() @ p64, 2.0 ** -18, "dW1"); close(dw2, h64.t().contiguous() @ g64, 2.0 ** -18, "dW2")


@pytest.mark.gpu
def test_calls_on_two_streams_at_once():
    """Two calls in flight with buffers of their own give what each gives alone."""
    m, h, n, rank = 300, 512, 520, 32
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    sets = []
    for i in range(2):
        g = _g(20 + i)
        offsets, ids = _cuts("gaps and empties", m)
        ad = T.Adapters(torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.tensor(ids, dtype=torch.int32, device="cuda"), 3, rank)
        sets.append((ad, _strided(g, m, h), _strided(g, 3, rank, h), _strided(g, 3, rank, n), _strided(g, m, n),
                     torch.empty(T.tp_adapter_workspace_size(grid, dims, T.PASS_FWD, ad), dtype=torch.uint8, device="cuda")))
    run = lambda t, y, s=None: T.tp_adapter_fwd(grid, dims, 1, t[0], [t[1]], [t[2]], t[3], t[4], None, 0, y, workspace=t[5], stream=s)
    ys = [[torch.full((m, n), 7.0, dtype=BF, device="cuda") for _ in range(2)] for _ in range(2)]
    for t, y in zip(sets, ys):
        run(t, y[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for t, y, s in zip(sets, ys, streams):
            run(t, y[1], s)
    torch.cuda.synchronize()
    for y in ys:
        assert torch.equal(y[0], y[1])


@pytest.mark.gpu
def test_arrays_that_are_too_short_or_of_another_type_are_refused():
    """Before anything is launched: the outputs keep what they held."""
    m, h, n, rank = 16, 64, 72, 16
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    cuda = lambda *s, dtype=BF: torch.zeros(*s, dtype=dtype, device="cuda")
    i32 = lambda k: cuda(k, dtype=torch.int32)
    ok = T.Adapters(i32(4), i32(3), 2, rank, cuda(2, dtype=F32))
    y, dx = torch.full((m, n), 7.0, device="cuda"), torch.full((m, h), 7.0, device="cuda")
    ws = cuda(1 << 22, dtype=torch.uint8)
    fwd = lambda **k: T.tp_adapter_fwd(grid, dims, 1, k.get("ad", ok), [k.get("x", cuda(m, h))], [k.get("a", cuda(2, rank, h))], k.get("b", cuda(2, rank, n)), k.get("c", cuda(m, n)),
                                       k.get("bias"), T.EPI_BIAS if "bias" in k else 0, y, v=k.get("v"), workspace=ws)
    bwd = lambda **k: T.tp_adapter_bwd(grid, dims, 1, ok, [k.get("dy", cuda(m, n))], [cuda(2, rank, n)], a=cuda(2, rank, h), dx_base=cuda(m, h), dx=dx, x_own=k.get("x", cuda(m, h)),
                                       da=k.get("da"), dy_own=cuda(m, n), v=k.get("v"), db=k.get("db"), workspace=ws)
    ad = lambda **k: ok._replace(**k)
    for call in (lambda: fwd(ad=ad(offsets=cuda(4, dtype=torch.int64))), lambda: fwd(ad=ad(ids=cuda(3, dtype=torch.int64))), lambda: fwd(ad=ad(scale=cuda(2))), lambda: fwd(x=cuda(m, h, dtype=F32)),
                 lambda: fwd(a=cuda(2, rank, h, dtype=F32)), lambda: fwd(b=cuda(2, rank, n, dtype=torch.float16)), lambda: fwd(v=cuda(m, rank)), lambda: fwd(bias=cuda(n, dtype=F32)),
                 lambda: bwd(da=cuda(2, rank, h)), lambda: bwd(db=cuda(2, rank, n), v=cuda(m, rank, dtype=F32)), lambda: bwd(dy=cuda(m, n, dtype=F32))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: fwd(ad=ad(offsets=i32(3))), lambda: fwd(ad=ad(n_segments=4)), lambda: fwd(ad=ad(offsets=i32(8)[::2])), lambda: fwd(ad=ad(scale=cuda(1, dtype=F32))),
                 lambda: fwd(a=cuda(3, rank, h)), lambda: fwd(a=cuda(2, 8, h)), lambda: fwd(a=cuda(rank, h)), lambda: fwd(a=cuda(2, h, rank).transpose(1, 2)),
                 lambda: fwd(x=cuda(h, m).t()), lambda: fwd(v=cuda(m, 2 * rank, dtype=F32)[:, :rank]), lambda: fwd(bias=cuda(2 * n)[::2])):
        with pytest.raises(ValueError):
            call()
    assert _st(lambda: fwd(a=cuda(1, rank, h).expand(2, rank, h))) == 4 and _st(lambda: fwd(c=cuda(m, n, dtype=torch.float16))) == 6
    torch.cuda.synchronize()
    assert (y == 7).all() and (dx == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m,rank,p", [(3, 128, 0.0), (5, 96, 0.25), (260, 40, 0.0)])
def test_first_call_inside_a_capture(m, rank, p):
    """A graph may be captured with no call before it: each replay gives what an eager call gives afterwards."""
    g = _g(31)
    h, n = 136, 200
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c = _strided(g, m, h), _strided(g, 1, rank, h), _strided(g, 1, rank, n), _strided(g, m, n, dtype=F32)
    ad = T.Adapters(torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), 1, rank)
    ws = torch.empty(T.tp_adapter_workspace_size(grid, dims, T.PASS_FWD, ad), dtype=torch.uint8, device="cuda")
    y, z = (torch.full((m, n), 7.0, device="cuda") for _ in range(2))
    call = lambda out: T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, out, dropout=T.Dropout(p, 5) if p else None, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y)
    for _ in range(3):
        x.normal_(generator=g)
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        call(z)
        torch.cuda.synchronize()
        assert torch.equal(y, z)


@pytest.mark.gpu
def test_an_infinite_factor_stays_in_its_columns():
    """One infinite element of B: its column alone is not finite, in the rows of its adapter alone."""
    m, h, n, rank = 70, 64, 136, 16
    g = _g(33)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c = _strided(g, m, h), _strided(g, 2, rank, h), _strided(g, 2, rank, n), _strided(g, m, n)
    ad = T.Adapters(torch.tensor([0, 30, m], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 2, rank)
    ws = torch.empty(T.tp_adapter_workspace_size(grid, dims, T.PASS_FWD, ad), dtype=torch.uint8, device="cuda")
    y, z = (torch.full((m, n), 7.0, dtype=BF, device="cuda") for _ in range(2))
    T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, workspace=ws)
    b[1, 5, 77] = float("inf")
    T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, z, workspace=ws)
    hit = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    hit[30:, 77] = True
    assert torch.equal(y[~hit], z[~hit]) and not torch.isfinite(z[hit]).any()


@pytest.mark.gpu
@pytest.mark.parametrize("m,pool,rank,cuts,ids", [(700, 7, 40, [0, 333, 690], [5, 2]), (900, 1, 128, [0, 1, 900], [0, 0]), (1500, 40, 16, [3, 1490], [39])])
def test_gradients_are_the_same_with_and_without_dx(m, pool, rank, cuts, ids):
    """The factors' gradients of a pool of which few adapters have rows, in shares: right, zeros elsewhere, the same bits whichever launch adds the shares up, and
    added to what is there if that is asked for."""
    h, n = 136, 264
    g = _g(41)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c, dy = _strided(g, m, h), _strided(g, pool, rank, h), _strided(g, pool, rank, n), _strided(g, m, h), _strided(g, m, n)
    ad = T.Adapters(torch.tensor(cuts, dtype=torch.int32, device="cuda"), torch.tensor(ids, dtype=torch.int32, device="cuda"), pool, rank)
    ws = torch.empty(T.tp_adapter_workspace_size(grid, dims, T.PASS_DX, ad), dtype=torch.uint8, device="cuda")
    v = torch.randn(m, rank, generator=g, device="cuda")
    dx = torch.full((m, h), 7.0, device="cuda")

    def grads(with_dx, start=None):
        da, db = (torch.full((pool, rank, k), float("nan"), device="cuda") if start is None else start[i].clone() for i, k in enumerate((h, n)))
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a if with_dx else None, dx_base=c if with_dx else None, dx=dx if with_dx else None, x_own=x, da=da, dy_own=dy, v=v, db=db,
                         accumulate=start is not None, workspace=ws)
        return da, db

    one, two = grads(True), grads(False)
    for p, q in zip(one, two):
        assert torch.equal(p, q)
    start = [torch.randn(t.shape, generator=g, device="cuda") for t in one]
    for p, q, s, t in zip(grads(True, start), grads(False, start), start, one):
        assert torch.equal(p, q) and torch.equal(p, s + t)
    # against 64 bits: U and the terms of both sums are off by what fp32 sums of K products and of a segment's rows are
    d64 = lambda t: t.double()
    want = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in one]
    size = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in one]
    for lo, hi, i in zip(cuts, cuts[1:], ids):
        u, mu = d64(dy[lo:hi]) @ d64(b[i]).t().contiguous(), d64(dy[lo:hi]).abs() @ d64(b[i]).abs().t().contiguous()
        want[0][i] += u.t().contiguous() @ d64(x[lo:hi])
        size[0][i] += mu.t().contiguous() @ d64(x[lo:hi]).abs()
        want[1][i] += d64(v[lo:hi]).t().contiguous() @ d64(dy[lo:hi])
        size[1][i] += d64(v[lo:hi]).abs().t().contiguous() @ d64(dy[lo:hi]).abs()
    for got, w, s in zip(one, want, size):
        assert ((got.double() - w).abs() <= (m + n + 16) * E24 * s).all()
        idle = [i for i in range(pool) if i not in ids]
        assert (got[idle] == 0).all()
