// C ABI of what stands beside the layer's products (see include/tp_linear.h): dropout without a stored mask, low-rank
// adapters.  Everything is checked before the
// first launch; nothing is allocated or synchronised here.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "tp_checks.h"
#include "tp_internal.h"

using namespace tpl;

namespace {

constexpr int64_t kMostCols = ((int64_t)1 << 32) - 8;     // of a block of the dropout calls: its columns are numbered in 32 bits
constexpr int64_t kMostSumCols = ((int64_t)1 << 30) - 256;  // with their sums, strips of 64 or 256 columns at four threads a column: fewer than 2^32 threads

// A mask whose block begins at (row, col) behind the caller's own position
int check_dropout(const tp_dropout_t* d, int64_t row, int64_t col, int64_t rows, int64_t cols, DropArgs* a) {
    if (!(d->p >= 0.0 && d->p <= 1.0)) return TP_ERR_MODE;
    if ((d->col0 & 7) || (col & 7) || (reinterpret_cast<uintptr_t>(d->offset_dev) & 7)) return TP_ERR_ALIGN;
    constexpr int64_t kRows = (int64_t)1 << 32, kCols = (int64_t)1 << 35;      // row and column group are words of the counter
    if (d->row0 < 0 || d->col0 < 0 || d->row0 > kRows || d->col0 > kCols || row > kRows || col > kCols || rows > kRows - d->row0 - row ||
        cols > kCols - d->col0 - col)
        return TP_ERR_SHAPE;
    a->key0 = (uint32_t)d->seed; a->key1 = (uint32_t)(d->seed >> 32);
    a->offset = d->offset; a->offset_dev = d->offset_dev;
    a->threshold = (uint32_t)std::nearbyint(d->p * 65536.0);
    a->factor = a->threshold < 65536 ? (float)(65536.0 / (65536.0 - a->threshold)) : 0.0f;
    a->row0 = (uint32_t)(d->row0 + row); a->group0 = (uint32_t)((d->col0 + col) >> 3);
    return TP_OK;
}

// Memory of a dropout call: a block's address, the bytes from row to row and of a row (no address: none)
struct Bytes { const void* p; int64_t pitch, width; };
Bytes bytes_of(const void* p, int64_t ld, int64_t cols, int dtype) { const int64_t size = dtype == TP_F32 ? 4 : 2; return Bytes{p, ld * size, cols * size}; }
bool apart(const Bytes& a, const Bytes& b, int64_t rows) { return !a.p || !b.p || !rows_overlap(a.p, a.pitch, a.width, b.p, b.pitch, b.width, rows); }
// An output and an input are one block, whose elements a thread reads before it writes them, or apart
bool over_or_apart(const Bytes& out, const Bytes& in, int64_t rows) {
    return (out.p == in.p && out.width == in.width && (out.pitch == in.pitch || rows == 1)) || apart(out, in, rows);
}

// ---------------------------------------------------------------------------------------------
// adapters
// ---------------------------------------------------------------------------------------------
struct Map {            // one pass of tp_block_map
    int n_steps, a_row[TP_MAX_STEPS], a_col[TP_MAX_STEPS], out_row, out_col, partial;
    int64_t m, n, k;
};
int block_map(const tp_grid_t* grid, const tp_dims_t* dims, int pass, Map* s) {
    if (int e = tp_block_map(grid, dims, pass, &s->n_steps, &s->m, &s->n, &s->k, s->a_row, s->a_col, nullptr, nullptr, &s->out_row, &s->out_col, &s->partial))
        return e;
    return s->m > INT32_MAX || s->n > INT32_MAX || s->k > INT32_MAX ? TP_ERR_SHAPE : TP_OK;
}

int check_counts(const tp_adapters_t* a) {
    if (!a) return TP_ERR_NULL;
    if (a->n_segments < 0 || a->n_adapters < 1 || a->n_adapters > TP_ADAPTER_MAX_POOL || a->rank < 1 || a->rank > TP_ADAPTER_MAX_RANK) return TP_ERR_SHAPE;
    return a->rank & 7 ? TP_ERR_ALIGN : TP_OK;
}
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int check_adapters(const tp_adapters_t* a) {
    if (int e = check_counts(a)) return e;
    if (a->n_segments > 0 && (!a->offsets || !a->ids)) return TP_ERR_NULL;
    return aligned4(a->offsets) && aligned4(a->ids) && aligned4(a->scale) ? TP_OK : TP_ERR_ALIGN;
}
int check_factor(const void* ptr, int64_t ld, int64_t stride, const tp_adapters_t* a, int64_t cols) {
    if (int e = check_cblk(tp_cblk_t{ptr, ld}, cols)) return e;
    if (stride & 7) return TP_ERR_ALIGN;
    return a->n_adapters > 1 && stride < (int64_t)(a->rank - 1) * ld + cols ? TP_ERR_SHAPE : TP_OK;
}
// an operand and the output over it: the same block or apart
int check_over(const tp_oblk_t& c, const tp_oblk_t& y, int64_t rows, int64_t cols) {
    if (c.ptr == y.ptr && c.dtype == y.dtype && (c.ld == y.ld || rows == 1)) return TP_OK;
    const int64_t size = c.dtype == TP_F32 ? 4 : 2, size_y = y.dtype == TP_F32 ? 4 : 2;
    return rows_overlap(c.ptr, c.ld * size, cols * size, y.ptr, y.ld * size_y, cols * size_y, rows) ? TP_ERR_SHAPE : TP_OK;
}

// Tiles of at most `tile` rows that segments over `rows` rows can have
int64_t most_tiles(int64_t rows, int64_t segments, int tile) {
    const int64_t some = std::min(rows, std::max<int64_t>(1, segments));        // segments with rows (none: as one)
    return (rows + some * (tile - 1)) / tile;
}
// How the products run.
//   down: short segments (up to 24 rows on average) take tiles of 16 rows, others of 64, or of 32 where 64 make at most 128 tiles or leave the CU with the most
//     tiles more rows (the start of one counted as eight).  us with 64 / 32: 16384 x 4096, 16 ranks 29.6 / 36.5; 32896 x 2 x
//     2560 in 24 segments 50.2 / 46.3; 2048 x 4 x 2048, 64 ranks 15.6 / 15.6, and up 21.5 / 19.3 for half the planes.  K is shared by as many workgroups
//     as make one for every CU, while each has eight units of 64, and while the planes are fewer than what reads them pays for (up, and in backward grad, once
//     for each of its strips; a multiple of four above four, as those are read): us with up to 4 / 8 / 12 planes, forward of 553 rows, 3968 to 432 columns, 64
//     ranks 24.5 / 21.4 / 22.5, 128 ranks 39.5 / - / 35.8; backward of 731 rows of 1504 and 2496 columns, 64 ranks 32.3 / 35.6 / -, 128 ranks 44.9 / 47.9 / -.
//   up: tiles of 32, 64 or 128 rows, whichever leaves the CU with the most workgroups (two at least, or there are too few loads under way) the
//     fewest rows, the start of a workgroup counted as ten.  us with 32 / 64 / 128: 16384 x 4096 fp32 with dropout, 16 ranks
//     118 / 110 / 101; 6000 x 4096 in 12 segments with GeLU, 32 ranks 44.9 / 47.6 / 45.4; 2048 x 8192, 64 ranks 25.1 / 21.8 / 25.2; 32896 x 640 in 24 segments
//     19.2 / 21.6 / 24.3.
struct Split { int tile, splits; int64_t tiles; int up_tile; int64_t up_tiles; };
Split plan_products(int64_t rows, int64_t segments, int64_t k, int n_steps, int64_t up_cols, int rank, bool bwd) {
    Split s;
    const bool brief = rows <= 24 * std::max<int64_t>(1, std::min(rows, segments));
    auto tiles = [&](int tile) { return std::max<int64_t>(1, most_tiles(rows, segments, tile)); };
    auto rounds = [](int64_t groups) { return (groups + 255) / 256; };
    s.tile = 16;
    s.up_tile = 16;
    if (!brief) {
        s.tile = tiles(64) <= 128 || rounds(tiles(32)) * (32 + 8) < rounds(tiles(64)) * (64 + 8) ? 32 : 64;
        int64_t best = INT64_MAX;
        const int strips = (int)((up_cols + 127) / 128);
        for (int tile : {64, 128, 32}) {
            if (tile == 128 && rank > 64) continue;             // (V's terms would not fit)
            const int waves = up_waves(strips, tiles(tile));
            const int64_t cost = std::max<int64_t>(2, rounds(tiles(tile) * ((strips + waves - 1) / waves))) * (tile + 10);
            if (cost < best) { best = cost; s.up_tile = tile; }
        }
    }
    s.tiles = tiles(s.tile);
    s.up_tiles = tiles(s.up_tile);
    const int64_t units = (k + 63) / 64 * n_steps;
    s.splits = (int)std::max<int64_t>(1, std::min<int64_t>({256 / s.tiles, units / 8, 16, bwd ? std::max(4, 256 / rank) : std::max(8, 512 / rank)}));
    if (s.splits > 4) s.splits &= ~3;
    return s;
}
// A launch's threads are counted in 32 bits: at most 2^22 tiles, and 2^23 workgroups of the gradients
constexpr int64_t kMostTiles = (int64_t)1 << 22, kMostGradBlocks = (int64_t)1 << 23;
int check_tiles(const Split& s) { return s.tiles > kMostTiles || s.up_tiles > kMostTiles ? TP_ERR_SHAPE : TP_OK; }

// Whether both products of short segments go into one launch, where every workgroup of a tile reads the factor A whole: by the elements it has.  GPU time in
// us, one launch / two, 4096 columns: one row, 16 ranks x 4096 6.7 / 8.3, x 16384 11.7 / 9.9; 96 single rows, 64 ranks x 4096 15.6 / 17.5, x 8192 20.7 / 20.9,
// x 16384 30.9 / 26.9; 256 single rows, 64 x 16384 35 / 47, 128 x 16384 96 / 97; 1000 single rows, 16 x 4096 50 / 83, 128 x 16384 323 / 330; segments
// of six rows, 16 of them, 16 x 4096 8.0 / 9.4, 64 x 4096 14.1 / 11.7; 50 of twelve rows, 16 x 1024 8.7 / 9.7, 16 x 4096 11.7 / 10.6.
bool in_one_launch(const Split& s, int64_t rows, int64_t segments, int64_t factor) {
    if (s.tile != 16) return false;
    const int64_t most = s.tiles >= 192 ? 1 << 21 : s.tiles >= 80 ? 1 << 19 : 1 << 17;
    return factor <= (rows > 8 * segments ? most / 4 : most);
}
// Shares of an adapter's rows: enough workgroups (a strip of 128 columns by 32 ranks each) of the adapters that can have rows for two a CU (four: 63 us
// for 55, and more planes), but of four units of 32 rows (one a wave) at least where they are all one adapter's, and of two of an adapter's average; and room for
// the planes of 256 adapters at most, or those that the whole pool would ask for (idle adapters have planes too, which nobody writes or reads).  Backward in
// us, by rows and the whole pool before: 222 rows in 29 segments, 56 ranks 34.5 -> 24; 8814 rows, two of 12 adapters, 32 ranks 83.4 -> 67.9; 8124 rows in
// two segments, 27 adapters, 16 ranks 25.7 -> 22; without the average: 642 rows in 28 segments, ten adapters, 64 ranks 35 -> 21.
int64_t grad_blocks(int64_t cols, int pool, int rank) { return (cols + 127) / 128 * ((rank + 31) / 32) * pool; }
int64_t grad_busy(int64_t segments, int pool) { return std::max<int64_t>(1, std::min<int64_t>(pool, segments)); }     // adapters that can have rows
int64_t grad_enough(int64_t cols, int rank, int64_t adapters) { const int64_t blocks = grad_blocks(cols, 1, rank) * adapters; return (512 + blocks - 1) / blocks; }
int64_t grad_room(int64_t cols, int pool, int rank) { return std::max<int64_t>(grad_enough(cols, rank, pool), 256 / pool); }
int plan_grad(int64_t rows, int64_t segments, int64_t cols, int pool, int rank) {
    const int64_t busy = grad_busy(segments, pool), units = most_tiles(rows, segments, 32);
    return (int)std::max<int64_t>(1, std::min<int64_t>({grad_enough(cols, rank, busy), grad_room(cols, pool, rank), units / 4, std::max<int64_t>(1, units / (2 * busy)), 32}));
}
// The most of these that any number of segments up to this one takes: a program has one workspace for batches of more and fewer requests.  K is shared most
// with one segment, which has the fewest tiles (64 rows make more than 128 of them where they are chosen, and K is not shared then); of the shares every
// bound where it is largest.
int most_splits(int64_t rows, int64_t k, int n_steps, int64_t up_cols, int rank, bool bwd) { return plan_products(rows, 1, k, n_steps, up_cols, rank, bwd).splits; }
int most_shares(int64_t rows, int64_t segments, int64_t cols, int pool, int rank) {
    const int64_t units = most_tiles(rows, segments, 32), busy = segments > pool ? pool : 1;
    const int64_t average = std::max(most_tiles(rows, 1, 32) / 2, (segments > pool ? units : 0) / (2 * busy));
    return (int)std::max<int64_t>(1, std::min<int64_t>({grad_enough(cols, rank, 1), grad_room(cols, pool, rank), units / 4, std::max<int64_t>(1, average), 32}));
}
size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
// the workspace, in this order
struct Space { size_t low, da, db, units; size_t all() const { return padded(low) + padded(da) + padded(db) + padded(units); } };
Space space_fwd(const Map& f, const tp_adapters_t* a, int splits) { return Space{(size_t)splits * (size_t)f.m * a->rank * 4, 0, 0, 0}; }
Space space_bwd(const Map& f, const Map& x, const tp_adapters_t* a, int splits, int shares) {
    const size_t each = (size_t)shares * a->n_adapters * a->rank * 4;
    Space w{(size_t)splits * (size_t)x.m * a->rank * 4, 0, 0, 0};
    if (shares > 1) { w.da = each * x.n; w.db = each * f.n; w.units = (size_t)a->n_adapters * 4; }
    return w;
}

SegArgs segments(const tp_adapters_t* a, int64_t rows) { return SegArgs{a->offsets, a->ids, a->n_segments, (int32_t)rows, a->n_adapters}; }

// V = sum P_k F_k^T; n_steps blocks, the plan's planes at `planes`
int fill_down(DownArgs& d, const Split& s, const tp_adapters_t* a, int n_steps, const tp_cblk_t* p, const tp_factor_t* f, int64_t rows, int64_t k, float* planes) {
    for (int i = 0; i < n_steps; ++i) {
        if (int e = check_cblk(p[i], k)) return e;
        if (int e = check_factor(f[i].ptr, f[i].ld, f[i].stride, a, k)) return e;
        d.p[i] = p[i].ptr; d.ldp[i] = (int32_t)p[i].ld;
        d.f[i] = f[i].ptr; d.ldf[i] = (int32_t)f[i].ld; d.strides[i] = f[i].stride;
    }
    d.n_steps = n_steps; d.K = (int32_t)k; d.rank = a->rank;
    d.tile = s.tile; d.tiles = (int32_t)s.tiles; d.splits = s.splits;
    d.seg = segments(a, rows);
    d.out = planes; d.plane = rows * a->rank;
    return TP_OK;
}
int fill_up(UpArgs& u, const Split& s, const tp_adapters_t* a, const tp_factor_t& f, const tp_oblk_t& c, const tp_oblk_t& out, int64_t rows, int64_t cols) {
    if (int e = check_factor(f.ptr, f.ld, f.stride, a, cols)) return e;
    if (int e = check_oblk(c, cols, false)) return e;
    if (int e = check_oblk(out, cols, false)) return e;
    if (int e = check_over(c, out, rows, cols)) return e;
    u.plane = rows * a->rank; u.splits = s.splits;
    u.f = f.ptr; u.ldf = (int32_t)f.ld; u.stride = f.stride; u.rank = a->rank; u.cols = (int32_t)cols;
    u.scale = a->scale;
    u.c = c.ptr; u.ldc = c.ld; u.c_f32 = c.dtype == TP_F32;
    u.out = out.ptr; u.ldo = out.ld; u.out_f32 = out.dtype == TP_F32;
    u.tile = s.up_tile; u.tiles = (int32_t)s.up_tiles;
    u.seg = segments(a, rows);
    return TP_OK;
}

}  // namespace

extern "C" {

size_t tp_adapter_workspace_size(const tp_grid_t* grid, const tp_dims_t* dims, int pass, const tp_adapters_t* adapters) {
    Map f, x;
    if (check_counts(adapters) != TP_OK || block_map(grid, dims, TP_PASS_FWD, &f) != TP_OK || block_map(grid, dims, TP_PASS_DX, &x) != TP_OK) return 0;
    if (pass == TP_PASS_FWD) return space_fwd(f, adapters, most_splits(f.m, f.k, f.n_steps, f.n, adapters->rank, false)).all();
    if (pass != TP_PASS_DX) return 0;
    const int shares = most_shares(x.m, std::max(1, adapters->n_segments), x.n + f.n, adapters->n_adapters, adapters->rank);
    return space_bwd(f, x, adapters, most_splits(x.m, x.k, x.n_steps, x.n, adapters->rank, true), shares).all();
}

int tp_adapter_fwd(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps, const tp_adapters_t* adapters, const tp_cblk_t* x_blocks,
                   const tp_factor_t* a_blocks, const tp_factor_t* b, const tp_dropout_t* drop, tp_oblk_t c, const void* bias, int epi, tp_oblk_t y,
                   tp_oblk_t preact, float* v, void* workspace, size_t workspace_bytes, void* hip_stream) {
    Map s;
    if (int e = block_map(grid, dims, TP_PASS_FWD, &s)) return e;
    if (int e = check_adapters(adapters)) return e;
    if (!x_blocks || !a_blocks || !b) return TP_ERR_NULL;
    if (n_steps < 1 || n_steps > s.n_steps) return TP_ERR_SHAPE;
    if (epi != TP_EPI_NONE && epi != TP_EPI_BIAS && epi != TP_EPI_BIAS_GELU) return TP_ERR_MODE;
    if (epi != TP_EPI_NONE && !bias) return TP_ERR_NULL;
    if ((bias && !aligned16(bias)) || !aligned16(v)) return TP_ERR_ALIGN;
    if (s.partial) {
        if (epi != TP_EPI_NONE || preact.ptr) return TP_ERR_MODE;
        if (y.ptr && y.dtype != TP_F32) return TP_ERR_DTYPE;
    }
    const Split sp = plan_products(s.m, adapters->n_segments, s.k, s.n_steps, s.n, adapters->rank, false);
    if (int e = check_tiles(sp)) return e;
    const Space need = space_fwd(s, adapters, sp.splits);
    float* const planes = v && sp.splits == 1 ? v : static_cast<float*>(workspace);
    DownArgs d{};
    if (int e = fill_down(d, sp, adapters, n_steps, x_blocks, a_blocks, s.m, s.k, planes)) return e;
    if (drop) {
        d.dropped = 1;
        for (int i = 0; i < n_steps; ++i) {
            if (int e = check_dropout(drop, s.a_row[i] * s.m, s.a_col[i] * s.k, s.m, s.k, &d.drop)) return e;
            d.group0[i] = d.drop.group0;
        }
    }
    UpArgs u{};
    if (int e = fill_up(u, sp, adapters, *b, c, y, s.m, s.n)) return e;
    if (preact.ptr) {
        if (int e = check_oblk(preact, s.n, false)) return e;
        if (preact.dtype != TP_BF16) return TP_ERR_DTYPE;
    }
    const bool few = !drop && in_one_launch(sp, s.m, adapters->n_segments, n_steps * s.k * adapters->rank);
    u.v = planes; u.v_out = planes == v && !few ? nullptr : v;
    u.bias = epi == TP_EPI_NONE ? nullptr : bias; u.gelu = epi == TP_EPI_BIAS_GELU;
    u.pre = preact.ptr; u.ldp = preact.ld;
    if (!ws_ok(need.all(), workspace, workspace_bytes)) return TP_ERR_WORKSPACE;
    if (adapters->n_segments == 0) return TP_OK;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (few) return launch_few(d, u, stream) != hipSuccess ? TP_ERR_HIP : TP_OK;
    return launch_down(d, stream) != hipSuccess || launch_up(u, nullptr, stream) != hipSuccess ? TP_ERR_HIP : TP_OK;
}

int tp_adapter_bwd(const tp_grid_t* grid, const tp_dims_t* dims, int n_steps, const tp_adapters_t* adapters, const tp_cblk_t* dy_blocks,
                   const tp_factor_t* b_blocks, const tp_factor_t* a, const tp_dropout_t* drop, tp_oblk_t dx_base, tp_oblk_t dx, const tp_cblk_t* x_own,
                   tp_factor_out_t da, const tp_cblk_t* dy_own, const float* v, tp_factor_out_t db, int accumulate, void* workspace,
                   size_t workspace_bytes, void* hip_stream) {
    Map f, x;
    if (int e = block_map(grid, dims, TP_PASS_FWD, &f)) return e;
    if (int e = block_map(grid, dims, TP_PASS_DX, &x)) return e;
    if (int e = check_adapters(adapters)) return e;
    const bool want_u = dx.ptr || da.ptr;
    if (want_u && (!dy_blocks || !b_blocks)) return TP_ERR_NULL;
    if (want_u && (n_steps < 1 || n_steps > x.n_steps)) return TP_ERR_SHAPE;
    if ((dx.ptr && !a) || (da.ptr && !x_own) || (db.ptr && (!dy_own || !v))) return TP_ERR_NULL;
    if (!aligned16(v)) return TP_ERR_ALIGN;
    if (dx.ptr && x.partial && dx.dtype != TP_F32) return TP_ERR_DTYPE;
    const Split sp = plan_products(x.m, adapters->n_segments, x.k, x.n_steps, x.n, adapters->rank, true);
    if (int e = check_tiles(sp)) return e;
    if (grad_blocks(x.n + f.n, adapters->n_adapters, adapters->rank) > kMostGradBlocks) return TP_ERR_SHAPE;
    const int shares = plan_grad(x.m, adapters->n_segments, x.n + f.n, adapters->n_adapters, adapters->rank);
    const Space need = space_bwd(f, x, adapters, sp.splits, shares);
    char* at = static_cast<char*>(workspace);
    float* const planes = reinterpret_cast<float*>(at);
    DropArgs mask{};
    if (drop)                                         // (rows and columns of the own X block, which dX has too)
        if (int e = check_dropout(drop, x.out_row * x.m, x.out_col * x.n, x.m, x.n, &mask)) return e;
    DownArgs d{};
    if (want_u)
        if (int e = fill_down(d, sp, adapters, n_steps, dy_blocks, b_blocks, x.m, x.k, planes)) return e;
    UpArgs u{};
    if (dx.ptr) {
        if (int e = fill_up(u, sp, adapters, *a, dx_base, dx, x.m, x.n)) return e;
        u.v = planes;
        u.dropped = drop != nullptr; u.drop = mask;
    }
    GradArgs g{};
    auto side = [&](const float* l, int splits, const tp_cblk_t& r, int64_t cols, int dropped, const tp_factor_out_t& out, size_t part) {
        if (int e = check_cblk(r, cols)) return e;
        if (int e = check_factor(out.ptr, out.ld, out.stride, adapters, cols)) return e;
        GradSide& q = g.side[g.sides++];
        q.l = l; q.plane = x.m * adapters->rank; q.splits = splits;
        q.r = r.ptr; q.ldr = (int32_t)r.ld; q.cols = (int32_t)cols; q.dropped = dropped;
        q.out = static_cast<float*>(out.ptr); q.ldo = out.ld; q.stride = out.stride;
        q.part = reinterpret_cast<float*>(at + part);
        return (int)TP_OK;
    };
    if (da.ptr)
        if (int e = side(planes, sp.splits, *x_own, x.n, drop != nullptr, da, padded(need.low))) return e;
    if (db.ptr)
        if (int e = side(v, 1, *dy_own, f.n, 0, db, padded(need.low) + padded(need.da))) return e;
    g.rank = adapters->rank; g.shares = shares; g.accumulate = accumulate != 0;
    g.scale = adapters->scale; g.seg = segments(adapters, x.m); g.drop = mask;
    g.units = reinterpret_cast<int32_t*>(at + padded(need.low) + padded(need.da) + padded(need.db));
    if (!want_u && !db.ptr) return TP_OK;
    if (!ws_ok(need.all(), workspace, workspace_bytes)) return TP_ERR_WORKSPACE;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    // (dA and dB before dX: dY, which U has just read, may still be in the last cache)
    const bool some = adapters->n_segments > 0, up = some && dx.ptr, add_in_up = up && g.sides && g.shares > 1;
    if (some && want_u && launch_down(d, stream) != hipSuccess) return TP_ERR_HIP;
    if (g.sides && launch_grad(g, !add_in_up, stream) != hipSuccess) return TP_ERR_HIP;
    return up && launch_up(u, add_in_up ? &g : nullptr, stream) != hipSuccess ? TP_ERR_HIP : TP_OK;
}

int tp_dropout_fwd(const tp_dropout_t* drop, const void* x, int64_t ld_x, int x_dtype, const void* bias, int epi, tp_cblk_t residual, tp_oblk_t y,
                   tp_oblk_t preact, int64_t rows, int64_t cols, void* hip_stream) {
    if (!drop) return TP_ERR_NULL;
    if (rows < 0 || cols < 0 || cols > kMostCols) return TP_ERR_SHAPE;
    if (rows == 0 || cols == 0) {                // (an empty tensor has no address)
        DropArgs a;
        return check_dropout(drop, 0, 0, rows, cols, &a);
    }
    if (!x || !y.ptr) return TP_ERR_NULL;
    if (epi != TP_EPI_NONE && epi != TP_EPI_BIAS && epi != TP_EPI_BIAS_GELU) return TP_ERR_MODE;
    if (epi != TP_EPI_NONE && !bias) return TP_ERR_NULL;
    if (x_dtype != TP_F32 && x_dtype != TP_BF16) return TP_ERR_DTYPE;
    if (!aligned16(x) || (bias && !aligned16(bias)) || (ld_x & 7)) return TP_ERR_ALIGN;
    if (ld_x < cols) return TP_ERR_SHAPE;
    if (int e = check_oblk(y, cols, false)) return e;
    if (preact.ptr) {
        if (int e = check_oblk(preact, cols, false)) return e;
        if (preact.dtype != TP_BF16) return TP_ERR_DTYPE;
    }
    if (residual.ptr) {
        if (!aligned16(residual.ptr) || (residual.ld & 7)) return TP_ERR_ALIGN;
        if (residual.ld < cols) return TP_ERR_SHAPE;
    }
    const Bytes in[] = {bytes_of(x, ld_x, cols, x_dtype), bytes_of(residual.ptr, residual.ld, cols, TP_BF16)},
                out[] = {bytes_of(y.ptr, y.ld, cols, y.dtype), bytes_of(preact.ptr, preact.ld, cols, TP_BF16)};
    if (!apart(out[0], out[1], rows)) return TP_ERR_SHAPE;
    for (const Bytes& o : out)
        if (!over_or_apart(o, in[0], rows) || !over_or_apart(o, in[1], rows)) return TP_ERR_SHAPE;
    DropArgs a;
    if (int e = check_dropout(drop, 0, 0, rows, cols, &a)) return e;
    if (launch_dropout(a, x, ld_x, x_dtype == TP_F32, epi == TP_EPI_NONE ? nullptr : bias, epi == TP_EPI_BIAS_GELU, residual.ptr, residual.ld, y.ptr, y.ld,
                       y.dtype == TP_F32, preact.ptr, preact.ld, rows, cols, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return TP_ERR_HIP;
    return TP_OK;
}

int tp_dropout_bwd(const tp_dropout_t* drop, const void* dy, int64_t ld_dy, const void* preact, int64_t ld_pre, void* dx, int64_t ld_dx, void* db_f32,
                   int64_t rows, int64_t cols, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!drop || (rows != 0 && cols != 0 && (!dy || !dx))) return TP_ERR_NULL;
    if (rows < 0 || cols < 0 || cols > kMostCols || (db_f32 && cols > kMostSumCols)) return TP_ERR_SHAPE;
    if (!aligned16(dy) || !aligned16(dx) || (cols & 7) || (ld_dy & 7) || (ld_dx & 7)) return TP_ERR_ALIGN;
    if (preact && (!aligned16(preact) || (ld_pre & 7))) return TP_ERR_ALIGN;
    if (db_f32 && !aligned16(db_f32)) return TP_ERR_ALIGN;
    if (rows > 0 && (ld_dy < cols || ld_dx < cols || (preact && ld_pre < cols))) return TP_ERR_SHAPE;
    DropArgs a;
    if (int e = check_dropout(drop, 0, 0, rows, cols, &a)) return e;
    if (db_f32 && workspace && (!aligned16(workspace) || workspace_bytes < colsum_ws_bytes(rows, cols))) return TP_ERR_WORKSPACE;
    if (cols == 0) return TP_OK;
    if (rows > 0) {
        const Bytes out = bytes_of(dx, ld_dx, cols, TP_BF16);
        if (!over_or_apart(out, bytes_of(dy, ld_dy, cols, TP_BF16), rows) || !over_or_apart(out, bytes_of(preact, ld_pre, cols, TP_BF16), rows)) return TP_ERR_SHAPE;
    }
    if (launch_dropout_bwd(a, dy, ld_dy, preact, ld_pre, dx, ld_dx, rows, cols, static_cast<float*>(db_f32), static_cast<float*>(workspace),
                           static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        return TP_ERR_HIP;
    return TP_OK;
}

}  // extern "C"
