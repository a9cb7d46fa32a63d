"""Dropout and adapters where values and blocks are unusual: blocks over and between one another, infinities beside padded ranks, values that bf16 cannot hold,
adapters that no row uses, many segments."""
import pytest
import torch

import paper_2110_14883_amd as T
import test_adapter
from test_adapter import BF, F32, _g, _strided
from test_dropout import _mask, _rand, factor, near, slope64

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("db", [0, 1])
def test_dropout_blocks_between_each_others_rows_and_over_preact(db):
    """dy, preact and dx as columns of one matrix, and dx over preact itself."""
    rows, cols, d = 70, 136, T.Dropout(0.4, 8, 9, row0=3, col0=16)
    m = _rand(rows, 3 * cols, BF, 51)
    dy, pre, dx = (m[:, i * cols:(i + 1) * cols] for i in range(3))
    ref = torch.where(_mask(d, rows, cols), dy.double() * factor(d.p) * slope64(pre.double()), 0.0)
    keep = dy.clone()
    work = (3 * 2.0 ** -24 + 1e-6) * max(1.0, float(ref.abs().max()))
    sums = torch.empty(cols, device="cuda") if db else None
    T.tp_dropout_bwd(d, dy, dx, preact=pre, db=sums)
    near(dx, ref, BF, work)
    first = dx.clone()
    T.tp_dropout_bwd(d, dy, pre, preact=pre, db=sums)
    assert torch.equal(pre, first) and torch.equal(dx, first) and torch.equal(dy, keep)
    x, y = m[:, :cols], m[:, 2 * cols:]
    want = torch.where(_mask(d, rows, cols), x.double() * factor(d.p), 0.0) + pre.double()
    T.tp_dropout_fwd(d, x, None, T.EPI_NONE, y, residual=pre, preact=x)
    near(y, want, BF, 3 * 2.0 ** -24 * float(want.abs().max()))
    assert torch.equal(x, keep) and torch.equal(pre, first)


def test_adapter_blocks_between_each_others_rows():
    """c and y, dx_base and dx as columns of one matrix: what blocks apart give."""
    m, h, n, rank = 50, 64, 72, 16
    g = _g(52)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, dy = _strided(g, m, h), _strided(g, 1, rank, h), _strided(g, 1, rank, n), _strided(g, m, n)
    ad = T.Adapters(i32([0, 20, m]), i32([0, -1]), 1, rank)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for p in (0.0, 0.3):
        drop = T.Dropout(p, 1) if p else None
        both = _strided(g, m, 2 * n, pad=0)
        c, y, z = both[:, :n], both[:, n:], torch.empty(m, n, dtype=BF, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c.clone(), None, 0, z, dropout=drop, workspace=ws)
        keep = c.clone()
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, dropout=drop, workspace=ws)
        assert torch.equal(y, z) and torch.equal(c, keep)
        base, dx, dz = both[:, n:n + h], both[:, :h], torch.empty(m, h, dtype=BF, device="cuda")
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=base.clone(), dx=dz, dropout=drop, workspace=ws)
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=base, dx=dx, dropout=drop, workspace=ws)
        assert torch.equal(dx, dz) and torch.equal(base, z[:, :h])


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 128])
@pytest.mark.parametrize("rows", [3, 80])           # one launch, two launches
@pytest.mark.parametrize("y_type", [BF, F32])
def test_an_infinite_input_is_infinite_and_no_nan_for_any_rank(rank, rows, y_type):
    """Factors of one sign: an infinite element of X makes its row of Y infinite, whatever lies in the ranks that fill up a matrix operand; the others stay as they are."""
    h, n = 64, 136
    g = _g(60 + rank)
    grid, dims = T.Grid(T.MODE_1D_COL), (rows, h, n)
    x, a, b, c = _strided(g, rows, h), _strided(g, 1, rank, h).abs() + 0.125, _strided(g, 1, rank, n).abs() + 0.125, _strided(g, rows, n)
    ad = T.Adapters(i32([0, rows]), i32([0]), 1, rank)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def forward(x):
        y, v = torch.full((rows, n), 7.0, dtype=y_type, device="cuda"), torch.full((rows, rank), 7.0, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v, workspace=ws)
        return y, v

    good = forward(x)
    inf = float("inf")
    for value in (inf, -inf):
        x2 = x.clone()
        x2[1, 5] = value
        bad = forward(x2)
        for p, q in zip(good, bad):
            assert (q[1] == value).all() and torch.equal(p[0], q[0]) and torch.equal(p[2:], q[2:])


# V's largest values: 2^128 - 2^118 is an fp32 number that would round to an infinite bf16.  Exact as a sum of these three, in any order
TOP = [2.0 ** 128 - 2.0 ** 120, 2.0 ** 119, 2.0 ** 118]


@pytest.mark.parametrize("rank,rows", [(16, 3), (16, 80), (72, 3), (72, 80)])
@pytest.mark.parametrize("y_type", [BF, F32])
def test_finite_values_beyond_bf16s_largest(rank, rows, y_type):
    """V and U of 2^128 - 2^118 and its opposite times factors of 2^-100: Y, dX, dA and dB are finite and right to their type's rounding (the products are exact
    in fp32 but for the sum over ranks: 2^-24 a rank, and 2^-17 for V as two terms)."""
    h, n, tiny = 64, 72, 2.0 ** -100
    grid, dims = T.Grid(T.MODE_1D_COL), (rows, h, n)
    z = lambda *s, t=BF: torch.zeros(*s, dtype=t, device="cuda")
    x, a, b, dy = z(rows, h), z(1, rank, h), torch.full((1, rank, n), tiny, dtype=BF, device="cuda"), z(rows, n)
    a[:, :, :3] = 1
    top = torch.tensor(TOP, dtype=torch.float64, device="cuda").to(BF)
    x[0, :3], x[1, :3] = top, -top
    v_top = sum(TOP)
    ad = T.Adapters(i32([0, rows]), i32([0]), 1, rank)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    y, v = z(rows, n, t=y_type), z(rows, rank, t=F32)
    T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, z(rows, n), None, 0, y, v=v, workspace=ws)
    assert (v[0].double() == v_top).all() and (v[1].double() == -v_top).all() and (v[2:] == 0).all()
    want = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
    want[0], want[1] = rank * v_top * tiny, -rank * v_top * tiny
    off = torch.finfo(y_type).eps / 2 + rank * 2.0 ** -24 + (2.0 ** -17 if y_type == BF else 2.0 ** -24)
    assert ((y.double() - want).abs() <= off * want.abs()).all()
    # backward: U = dY B^T with factors of one, dX = U A, dA = U^T X, dB = V^T dY
    one, small = z(1, rank, n), torch.full((1, rank, h), tiny, dtype=BF, device="cuda")
    one[:, :, :3] = 1
    dy[0, :3], dy[1, :3] = top, -top
    xs, dys = torch.full((rows, h), tiny, dtype=BF, device="cuda"), torch.full((rows, n), tiny, dtype=BF, device="cuda")
    xs[1], dys[1] = -tiny, -tiny
    dx, da, db = z(rows, h, t=y_type), z(1, rank, h, t=F32), z(1, rank, n, t=F32)
    T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [one], a=small, dx_base=z(rows, h), dx=dx, x_own=xs, da=da, dy_own=dys, v=v, db=db, workspace=ws)
    want = torch.zeros(rows, h, dtype=torch.float64, device="cuda")
    want[0], want[1] = rank * v_top * tiny, -rank * v_top * tiny
    assert ((dx.double() - want).abs() <= off * want.abs()).all()
    for t in (da, db):
        assert ((t.double() - 2 * v_top * tiny).abs() <= 2.0 ** -22 * 2 * v_top * tiny).all()


@pytest.mark.parametrize("m", [40, 1500])           # one share of an adapter's rows, several
def test_scales_of_adapters_without_rows_do_not_matter(m):
    """They may be anything, as in a pool that is not full: zeros as the factors' gradients, or what was there."""
    h, n, rank = 64, 72, 16
    g = _g(70)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, dy = _strided(g, m, h), _strided(g, 4, rank, h), _strided(g, 4, rank, n), _strided(g, m, n)
    v = torch.randn(m, rank, generator=g, device="cuda")
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def grads(scale, start):
        ad = T.Adapters(i32([0, m // 2, m]), i32([1, -1]), 4, rank, torch.tensor(scale, device="cuda"))
        da, db = (torch.full((4, rank, k), start, device="cuda") for k in (h, n))
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], x_own=x, da=da, dy_own=dy, v=v, db=db, accumulate=start != 7.0, workspace=ws)
        return da, db

    inf = float("inf")
    for start in (7.0, 0.5):                        # (7: overwritten)
        for p, q in zip(grads([1.0, 2.0, 1.0, 1.0], start), grads([float("nan"), 2.0, inf, -inf], start)):
            assert torch.equal(p, q) and (q[[0, 2, 3]] == (0.0 if start == 7.0 else start)).all() and torch.isfinite(q).all()


def test_bias_gradient_of_no_rows_without_blocks():
    db = torch.full((72,), 7.0, device="cuda")
    T.tp_dropout_bwd(T.Dropout(0.1, 1), None, None, db=db, rows=0, cols=64)
    assert (db[:64] == 0).all() and (db[64:] == 7).all()


@pytest.mark.parametrize("m,pool,rank", [(200, 8, 16), (2050, 3, 16), (3000, 8, 64)])
def test_one_workspace_for_every_number_of_segments(m, pool, rank):
    """A workspace made for the largest number of requests serves calls of fewer, forward and backward, and they give what they give with their own."""
    h, n, most = 1024, 136, 12
    g = _g(80)
    grid, dims = T.Grid(T.MODE_1D_COL), (m, h, n)
    x, a, b, c, dy = _strided(g, m, h), _strided(g, pool, rank, h), _strided(g, pool, rank, n), _strided(g, m, n), _strided(g, m, n)
    size = lambda count: max(T.tp_adapter_workspace_size(grid, dims, q, T.Adapters(None, None, pool, rank, None, count)) for q in (T.PASS_FWD, T.PASS_DX))
    room = torch.full((size(most) + 64,), 0xFF, dtype=torch.uint8, device="cuda")

    def both(count, ws):
        cuts = [i * m // count for i in range(count + 1)]
        ad = T.Adapters(i32(cuts), i32([i % pool for i in range(count)]), pool, rank)
        y, v, dx = torch.empty(m, n, dtype=BF, device="cuda"), torch.empty(m, rank, device="cuda"), torch.empty(m, h, device="cuda")
        da, db = torch.empty(pool, rank, h, device="cuda"), torch.empty(pool, rank, n, device="cuda")
        T.tp_adapter_fwd(grid, dims, 1, ad, [x], [a], b, c, None, 0, y, v=v, workspace=ws)
        T.tp_adapter_bwd(grid, dims, 1, ad, [dy], [b], a=a, dx_base=x, dx=dx, x_own=x, da=da, dy_own=dy, v=v, db=db, workspace=ws)
        return y, v, dx, da, db

    for count in (1, 2, 3, 5, 9, most):
        for p, q in zip(both(count, room[:-64]), both(count, torch.empty(size(count), dtype=torch.uint8, device="cuda"))):
            assert torch.equal(p, q), count
    assert (room[-64:] == 0xFF).all()


@pytest.mark.parametrize("rank,p", [(16, 0.0), (72, 0.3)])
@pytest.mark.parametrize("single", [False, True])
def test_over_a_thousand_segments(monkeypatch, rank, p, single):
    """Ragged ones with empty ones between, and single rows: many rounds of 64 of a workgroup's walk over them, the same adapter again and again."""
    def cuts(kind, m):
        n = 1300
        at = [min(m, i if single else i * m // n + i * 7 % 3) for i in range(n + 1)]
        return sorted(at), [i * 5 % 7 - 1 if i % 3 else i // 400 for i in range(n)]

    monkeypatch.setattr(test_adapter, "_cuts", cuts)
    test_adapter.run_case(T.Grid(T.MODE_1D_COL), (1500, 72, 136), rank, None, p=p, seed=90)
