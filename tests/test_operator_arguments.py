"""What the calls of dropout and adapters refuse of their tensors, and what they take, seen on the host: stand-ins for tensors on the device whose addresses are
never followed (every call that gets past the arguments is turned down by the library for its workspace or probability)."""
import ctypes as C

import pytest
import torch

import paper_2110_14883_amd as T
from paper_2110_14883_amd import binding as B

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Block:
    """A tensor of device 0 as the binding sees one."""
    def __init__(self, *shape, dtype=BF, stride=None, at=0x100000):
        self.shape, self.dtype, self.at = shape, dtype, at
        dense = [1] * len(shape)
        for i in range(len(shape) - 2, -1, -1):
            dense[i] = dense[i + 1] * max(1, shape[i + 1])
        self.dense, self.strides = tuple(dense), tuple(stride or dense)

    def data_ptr(self):
        return self.at

    def stride(self):
        return self.strides

    def numel(self):
        return int(torch.Size(self.shape).numel())

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def get_device(self):
        return 0

    def is_contiguous(self):
        return self.strides == self.dense


@pytest.fixture
def device0(monkeypatch):
    """The binding with device 0 as the current one."""
    get = C.CFUNCTYPE(C.c_int, C.POINTER(C.c_int))(lambda to: to.__setitem__(0, 0) or 0)
    monkeypatch.setattr(B, "_hip_get_device", lambda L: C.cast(get, C.c_void_p).value)
    B._call.cache_clear()
    B._call()
    yield
    monkeypatch.undo()
    B._call.cache_clear()
    B._call()


def status(call):
    with pytest.raises(T.TpError) as e:
        call()
    return e.value.status


M, H, F, RANK = 48, 64, 136, 16
GRID, DIMS = T.Grid(T.MODE_1D_COL), (M, H, F)
AD = T.Adapters(Block(4, dtype=I32), Block(3, dtype=I32), 2, RANK, Block(2, dtype=F32))


def fwd(epi=T.EPI_BIAS_GELU, grid=GRID, dims=DIMS, steps=1, ws=None, **k):
    get = lambda name, *shape, **kw: k.get(name, Block(*shape, **kw))
    T.tp_adapter_fwd(grid, dims, steps, k.get("ad", AD), k.get("xs") or [get("x", M, H)], k.get("as_") or [get("a", 2, RANK, H)], get("b", 2, RANK, F), get("c", M, F, at=0x200000),
                     get("bias", F), epi, get("y", M, F, at=0x300000), preact=get("pre", M, F, at=0x400000), v=get("v", M, RANK, dtype=F32), workspace=ws, stream=0)


def bwd(**k):
    get = lambda name, *shape, **kw: k[name] if name in k else Block(*shape, **kw)
    T.tp_adapter_bwd(GRID, DIMS, 1, AD, [get("dy", M, F)], [get("bs", 2, RANK, F)], a=get("a", 2, RANK, H), dx_base=get("base", M, H, at=0x200000), dx=get("dx", M, H, at=0x300000),
                     x_own=get("x", M, H), da=get("da", 2, RANK, H, dtype=F32), dy_own=get("own", M, F), v=get("v", M, RANK, dtype=F32), db=get("db", 2, RANK, F, dtype=F32),
                     workspace=None, stream=0)


def test_adapters_take_blocks_that_hold_their_extents(device0):
    """Exactly as large, larger, and cut out of a larger one: the workspace is what is missing then."""
    assert status(fwd) == 7 and status(bwd) == 7
    big = dict(x=Block(M + 1, H, stride=(H + 8, 1)), a=Block(2, RANK, H + 8), b=Block(2, RANK, F, stride=(4096, 256, 1)), bias=Block(F + 8), v=Block(M + 5, RANK, dtype=F32))
    assert status(lambda: fwd(**big)) == 7
    assert status(lambda: bwd(x=big["x"], a=big["a"], v=big["v"], db=Block(2, RANK, F + 8, dtype=F32))) == 7
    assert status(lambda: fwd(v=Block(M * RANK, dtype=F32))) == 7 and status(lambda: fwd(epi=T.EPI_NONE, bias=Block(8))) == 7
    # what is not used may be anything
    assert status(lambda: bwd(da=None, x=Block(1, 8))) == 7 and status(lambda: bwd(db=None, own=Block(1, 8), v=Block(1, RANK, dtype=F32))) == 7
    assert status(lambda: bwd(dx=None, a=Block(2, RANK, 8), base=Block(1, 8))) == 7 and status(lambda: bwd(dx=None, da=None, dy=Block(1, 8), bs=Block(2, RANK, 8))) == 7
    # a grid's steps: the first n_steps blocks are read
    grid, dims = T.Grid(T.MODE_2D, q=2, ri=1), (2 * M, 2 * H, 2 * F)
    assert status(lambda: fwd(grid=grid, dims=dims, xs=[Block(M, H), Block(1, 8)], as_=[Block(2, RANK, H), Block(2, RANK, 8)])) == 7
    with pytest.raises(ValueError):
        fwd(grid=grid, dims=dims, steps=2, xs=[Block(M, H), Block(1, 8)], as_=[Block(2, RANK, H)] * 2)
    with pytest.raises(ValueError):
        fwd(grid=grid, dims=dims, steps=2, xs=[Block(M, H)] * 2, as_=[Block(2, RANK, H), Block(2, RANK, 8)])


@pytest.mark.parametrize("name,block", [
    ("v", Block(M - 1, RANK, dtype=F32)), ("bias", Block(F - 8)), ("x", Block(M - 1, H)), ("x", Block(M, H - 8)), ("x", Block(H)), ("a", Block(2, RANK, H - 8)), ("b", Block(2, RANK, F - 8)),
    ("c", Block(M - 1, F)), ("c", Block(M, F - 8)), ("y", Block(M, F - 8)), ("y", Block(M - 1, F)), ("pre", Block(M - 1, F)), ("pre", Block(M, F - 8))])
def test_adapter_forward_refuses_shorter_tensors(device0, name, block):
    with pytest.raises(ValueError):
        fwd(**{name: block})


@pytest.mark.parametrize("name,block", [
    ("v", Block(M - 1, RANK, dtype=F32)), ("dy", Block(M - 1, F)), ("dy", Block(M, F - 8)), ("bs", Block(2, RANK, F - 8)), ("a", Block(2, RANK, H - 8)), ("base", Block(M - 1, H)),
    ("base", Block(M, H - 8)), ("dx", Block(M, H - 8)), ("dx", Block(M - 1, H)), ("x", Block(M - 1, H)), ("x", Block(M, H - 8)), ("own", Block(M - 1, F)), ("own", Block(M, F - 8)),
    ("da", Block(2, RANK, H - 8, dtype=F32)), ("db", Block(2, RANK, F - 8, dtype=F32))])
def test_adapter_backward_refuses_shorter_tensors(device0, name, block):
    with pytest.raises(ValueError):
        bwd(**{name: block})


NO = T.Dropout(2.0, 1)          # (refused by the library, behind the tensors)


def dfwd(x=None, y=None, bias=None, res=None, pre=None, rows=None, cols=None):
    T.tp_dropout_fwd(NO, x or Block(M, F, dtype=F32), bias or Block(F), T.EPI_BIAS, y or Block(M, F, at=0x200000), residual=res or Block(M, F, at=0x300000),
                     preact=pre or Block(M, F, at=0x400000), rows=rows, cols=cols, stream=0)


def dbwd(dy=None, dx=None, pre=None, rows=None, cols=None):
    T.tp_dropout_bwd(NO, dy or Block(M, F), dx or Block(M, F, at=0x200000), preact=pre or Block(M, F, at=0x300000), db=Block(F, dtype=F32), rows=rows, cols=cols, stream=0)


def test_dropout_takes_blocks_that_hold_their_extents(device0):
    assert status(dfwd) == 2 and status(dbwd) == 2
    assert status(lambda: dfwd(y=Block(M + 1, F, stride=(F + 8, 1), at=0x500000), res=Block(M, F + 16, at=0x600000))) == 2
    assert status(lambda: dfwd(x=Block(M + 3, F + 8), rows=M, cols=F)) == 2 and status(lambda: dbwd(dy=Block(M + 3, F + 8), rows=M, cols=F)) == 2
    assert status(lambda: dfwd(x=Block(F), rows=1, cols=F)) == 2


@pytest.mark.parametrize("call,name,block", [(dfwd, "y", Block(M - 1, F)), (dfwd, "y", Block(M, F - 8)), (dfwd, "res", Block(M - 1, F)), (dfwd, "res", Block(M, F - 8)), (dfwd, "pre", Block(M - 1, F)),
                                             (dfwd, "pre", Block(M, F - 8)), (dbwd, "dx", Block(M - 1, F)), (dbwd, "dx", Block(M, F - 8)), (dbwd, "pre", Block(M - 1, F)), (dbwd, "pre", Block(M, F - 8)),
                                             (dfwd, "y", Block(F))])
def test_dropout_refuses_shorter_tensors(device0, call, name, block):
    with pytest.raises(ValueError):
        call(**{name: block})


def test_more_rows_than_the_tensor_has_are_refused(device0):
    for call in (lambda: dfwd(x=Block(M, F, dtype=F32), rows=M + 1, cols=F), lambda: dbwd(dy=Block(M, F), rows=M, cols=F + 8), lambda: dfwd(x=Block(2 * F, stride=(2,)), rows=1, cols=F)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows,pitch,wide", [(1, 256, 256), (5, 256, 256), (5, 512, 256), (5, 512, 384), (3, 1024, 256), (32, 512, 272)])
def test_blocks_that_share_no_byte_may_lie_between_each_others_rows(rows, pitch, wide):
    """Every distance of y from c, against the sets of their bytes: refused where they share one (but for c itself), else the workspace is what is missing."""
    ld, cols, at = pitch // 2, wide // 2, 0x400000
    c_bytes = {i * pitch + b for i in range(rows) for b in range(0, wide, 16)}
    for d in range(-(rows + 1) * pitch, (rows + 1) * pitch + 1, 16):
        shares = any(x + d in c_bytes for x in c_bytes)

        def call():
            T.tp_adapter_fwd(GRID, (rows, H, cols), 1, T.Adapters(0x100, 0x200, 2, RANK, None, 1), [(0x10000, H)], [(0x20000, H, RANK * H)], (0x30000, cols, RANK * cols),
                             (at, ld, B.DT_BF16), None, T.EPI_NONE, (at + d, ld, B.DT_BF16), workspace=None, stream=0)
        assert status(call) == (4 if shares and d else 7), d


def test_dropout_outputs_that_overlap_what_is_read_are_refused():
    """x at 0x100000, 32 rows of 64 columns, bf16 or fp32; a probability that the library refuses behind this stands for a forward call that passes."""
    rows, cols, at = 32, 64, 0x100000
    bf, f32 = B.DT_BF16, B.DT_F32
    f = lambda x, y, res=None, pre=None: status(lambda: T.tp_dropout_fwd(NO, x, None, T.EPI_NONE, y, residual=res, preact=pre, rows=rows, cols=cols, stream=0))
    b = lambda dy, dx, pre=None: status(lambda: T.tp_dropout_bwd(T.Dropout(0.1, 1), dy, dx, preact=pre, rows=rows, cols=cols, stream=0))
    far = (0x900000, cols, bf)
    assert f((at, cols, f32), (at, cols, f32)) == 2 and f((at, cols, bf), (at, cols, bf)) == 2 and f((at, 72, bf), (at, 72, bf)) == 2          # in place
    assert f((at, cols, f32), far, res=(0x900000, cols)) == 2 and f((at, cols, bf), far, pre=(at, cols, bf)) == 2 and f((at, cols, f32), far, res=(0x500000, cols), pre=(0x500000, cols, bf)) == 2
    assert f((at, 128, bf), (at + 128, 128, bf), res=(at, 128)) == 2                                                                          # columns of one matrix
    assert f((at, cols, f32), (at, cols, bf)) == 4 and f((at, cols, bf), (at, cols, f32)) == 4 and f((at, cols, f32), (at, 2 * cols, bf)) == 4  # other types, other strides
    assert f((at, cols, bf), (at, 72, bf)) == 4 and f((at, cols, bf), (at + 16, cols, bf)) == 4 and f((at, cols, bf), (at - 128 * 31, cols, bf)) == 4 and f((at, cols, bf), (at + 128 * 31, cols, bf)) == 4
    one = lambda y: status(lambda: T.tp_dropout_fwd(NO, (at, 64, bf), None, T.EPI_NONE, y, rows=1, cols=cols, stream=0))
    assert one((at, 128, bf)) == 2 and one((at, 64, bf)) == 2 and one((at, 64, f32)) == 4 and one((at + 16, 64, bf)) == 4                       # one row: the same whatever the stride
    assert f((at, cols, bf), (at + 128 * 32, cols, bf)) == 2 and f((at, cols, bf), (at - 128 * 32, cols, bf)) == 2
    assert f((at, cols, f32), far, res=(0x900000, 72)) == 4 and f((at, cols, f32), (0x900000, cols, f32), res=(0x900000, cols)) == 4
    assert f((at, cols, f32), far, pre=far) == 4 and f((at, cols, f32), far, pre=(at, cols, bf)) == 4 and f((at, cols, f32), far, res=(0x500000, cols), pre=(0x500010, cols, bf)) == 4
    assert b((at, cols), (at + 16, cols)) == 4 and b((at, cols), (at, 72)) == 4 and b((at, cols), (0x900000, cols), pre=(0x900080, cols)) == 4


def test_empty_dropout_calls_need_no_blocks():
    """Nothing to do with no rows or columns, blocks left out and of any leading dimension."""
    d = T.Dropout(0.1, 1)
    T.tp_dropout_fwd(d, None, None, T.EPI_BIAS, None, rows=0, cols=64, stream=0)
    T.tp_dropout_fwd(d, None, None, T.EPI_BIAS, None, rows=4, cols=0, stream=0)
    T.tp_dropout_bwd(d, None, None, rows=0, cols=64, stream=0)
    T.tp_dropout_bwd(d, None, None, rows=4, cols=0, stream=0)
    T.tp_dropout_bwd(d, (0x10000, 8), (0x20000, 8), preact=(0x30000, 8), rows=0, cols=64, stream=0)
    # what does not depend on the extents is still looked at
    assert status(lambda: T.tp_dropout_bwd(T.Dropout(1.5, 1), None, None, rows=0, cols=64, stream=0)) == 2 and status(lambda: T.tp_dropout_bwd(d, None, None, db=0x40004, rows=0, cols=64, stream=0)) == 5


def test_negative_extents_of_dropout_are_refused():
    """Also where the other one is zero."""
    d = T.Dropout(0.1, 1)
    for rows, cols in ((0, -8), (-1, 0), (-1, -8), (-1, 64), (4, -8)):
        assert status(lambda: T.tp_dropout_fwd(d, (0x10000, 64, B.DT_BF16), None, T.EPI_NONE, (0x20000, 64, B.DT_BF16), rows=rows, cols=cols, stream=0)) == 4
        assert status(lambda: T.tp_dropout_bwd(d, (0x10000, 64), (0x20000, 64), rows=rows, cols=cols, stream=0)) == 4


def test_adapters_by_address_need_their_number_of_segments(device0):
    """There is no tensor to count them by: an error instead of a call that does nothing.  With none at all there is nothing to count."""
    for ad in (T.Adapters(0x100, 0x200, 2, RANK), T.Adapters(Block(4, dtype=I32), 0x200, 2, RANK)):
        with pytest.raises(ValueError, match="n_segments"):
            fwd(ad=ad)
    assert status(lambda: fwd(ad=T.Adapters(0x100, 0x200, 2, RANK, None, 3))) == 7 and status(lambda: fwd(ad=AD._replace(n_segments=2))) == 7
    assert status(lambda: fwd(ad=T.Adapters(None, None, 2, RANK))) == 7


def test_the_offset_on_the_device_is_a_64_bit_integer(device0):
    """Other types of eight bytes would be read as integers."""
    for dtype in (torch.float64, torch.complex64, torch.int32, torch.float32):
        with pytest.raises(TypeError):
            T.tp_dropout_bwd(T.Dropout(2.0, 1, 0, Block(1, dtype=dtype)), Block(M, F), Block(M, F, at=0x200000), stream=0)
    for dtype in (torch.int64, torch.uint64):
        assert status(lambda: T.tp_dropout_bwd(T.Dropout(2.0, 1, 0, Block(1, dtype=dtype)), Block(M, F), Block(M, F, at=0x200000), stream=0)) == 2
    assert status(lambda: T.tp_dropout_bwd(T.Dropout(2.0, 1, 0, 0x1000), Block(M, F), Block(M, F, at=0x200000), stream=0)) == 2


@pytest.mark.parametrize("m,h,f", [(1, 64, 64), (20, 4096, 512), (33, 16384, 128), (200, 4096, 4096), (700, 1504, 2496), (8200, 4096, 4096), (40000, 1280, 5120)])
def test_a_workspace_serves_every_smaller_number_of_segments(m, h, f):
    """The size for n segments is never below that for fewer, so one made for the most requests there can be is enough for any."""
    for pool in (1, 3, 8, 40, 300):
        for rank in (8, 16, 64, 128):
            for which in (T.PASS_FWD, T.PASS_DX):
                sizes = [T.tp_adapter_workspace_size(GRID, (m, h, f), which, T.Adapters(None, None, pool, rank, None, n)) for n in (*range(0, 60), 97, 300, 301, 1000, 9000, 50000)]
                assert sizes == sorted(sizes) and sizes[0] > 0, (pool, rank, which)


def test_dropout_rows_longer_than_the_kernels_count():
    """Columns are numbered in 32 bits inside a block, whatever its place in the full matrix."""
    d, n = T.Dropout(0.1, 1), 1 << 32
    assert status(lambda: T.tp_dropout_fwd(d, (1 << 40, n, B.DT_BF16), None, T.EPI_NONE, (1 << 45, n, B.DT_BF16), rows=1, cols=n, stream=0)) == 4
    assert status(lambda: T.tp_dropout_bwd(d, (1 << 40, n), (1 << 45, n), rows=1, cols=n, stream=0)) == 4
    for n in ((1 << 32) - 8, 64):           # (the probability is what is refused there)
        assert status(lambda: T.tp_dropout_fwd(T.Dropout(2.0, 1, col0=1 << 34), (1 << 40, n, B.DT_BF16), None, T.EPI_NONE, (1 << 45, n, B.DT_BF16), rows=1, cols=n, stream=0)) == 2
        assert status(lambda: T.tp_dropout_bwd(T.Dropout(2.0, 1, col0=1 << 34), (1 << 40, n), (1 << 45, n), rows=1, cols=n, stream=0)) == 2


def test_bias_gradients_of_more_columns_than_a_launch_has_threads_for():
    """Four threads a column, 2^32 - 1 in a launch: refused before it."""
    d, call = T.Dropout(0.1, 1), lambda d, n: status(lambda: T.tp_dropout_bwd(d, (1 << 40, n), (1 << 45, n), db=1 << 48, rows=1, cols=n, stream=0))
    assert call(d, 1 << 30) == 4 and call(d, (1 << 30) - 248) == 4 and call(d, (1 << 31) - 8) == 4
    assert call(T.Dropout(2.0, 1), (1 << 30) - 256) == 2
