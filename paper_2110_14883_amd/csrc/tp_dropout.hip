// gfx950 (MI355X, CDNA4): dropout beside the elementwise passes of the layer (paper Section 2.2: what is applied to a rank's chunk of the
// output), with the mask drawn where it is needed (tp_random.h).
//   forward   z = drop(act(x + bias)) + residual          backward   dx = drop'(dz) GeLU'(a),  db = column sums of dx
// Bound by memory; the draw costs about 55 vector instructions for the eight columns of a thread.
#include "tp_random.h"

namespace tpl {

namespace {

// Eight columns per thread and a grid that covers the block, streaming hints on everything (as tp_dgelu_kernel).  A dropped element is a zero whatever
// its input was: it is chosen, not multiplied.
// With bf16 in and out a thread has the eight columns of a group.  With an fp32 side it has four columns of one group and four of the group 32 further on in
// the block (neighbouring threads the other halves): every access is then 16 or 8 neighbouring bytes a lane.  (32 bytes a lane
// in two halves: 16384 x 4096 fp32 to bf16 with residual 86.4 us against 82.3, fp32 to fp32 96.5 / 83.2, bf16 to fp32 with residual 111 / 83.)
template <bool X_F32, bool GELU, bool PRE, bool Y_F32>
__global__ __launch_bounds__(256) void tp_dropout_kernel(const DropArgs drop, const void* x, int64_t ldx, const uint16_t* bias, const uint16_t* res,
                                                         int64_t ldr, void* y, int64_t ldy, uint16_t* pre, int64_t ldp, const uint32_t total,
                                                         const Divisor d) {
    constexpr int N = X_F32 || Y_F32 ? 2 : 1, C = 8 / N;                  // places, columns in each
    const uint32_t thread = blockIdx.x * 256u + threadIdx.x;
    const uint32_t first = N == 1 ? thread : (thread & ~63u) + ((thread & 63u) >> 1);
    if (first >= total) return;                                           // (both threads of a pair)
    const bool both = N > 1 && first + 32 < total;                        // (else the second place is the first again, and not stored)
    uint32_t g[N], n[N];
    int64_t r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t idx = i && both ? first + 32 : first;
        r[i] = quotient(d, idx);
        g[i] = idx - (uint32_t)r[i] * d.d;
        n[i] = g[i] * 8 + (N == 1 ? 0 : 4 * (thread & 1));
    }
    auto load_bf16 = [&](const uint16_t* p, int64_t ld) __attribute__((always_inline)) {
        if constexpr (N == 1) {
            return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p + r[0] * ld + n[0]));
        } else {
            const u32x2_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p + r[0] * ld + n[0]));
            const u32x2_t w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p + r[N - 1] * ld + n[N - 1]));
            return u32x4_t{v[0], v[1], w[0], w[1]};
        }
    };
    auto store_bf16 = [&](uint16_t* p, int64_t ld, const float (&v)[8]) __attribute__((always_inline)) {
        const u32x4_t o = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        if constexpr (N == 1) {
            __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(p + r[0] * ld + n[0]));
        } else {
            __builtin_nontemporal_store(u32x2_t{o[0], o[1]}, reinterpret_cast<u32x2_t*>(p + r[0] * ld + n[0]));
            if (both) __builtin_nontemporal_store(u32x2_t{o[2], o[3]}, reinterpret_cast<u32x2_t*>(p + r[N - 1] * ld + n[N - 1]));
        }
    };
    // everything is asked for, then the draw, which needs none of it, then the values
    f32x4_t xf[N];
    u32x4_t xb, q = {0u, 0u, 0u, 0u}, b = {0u, 0u, 0u, 0u};
    if constexpr (X_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) xf[i] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(static_cast<const float*>(x) + r[i] * ldx + n[i]));
    } else {
        xb = load_bf16(static_cast<const uint16_t*>(x), ldx);
    }
    if (res) q = load_bf16(res, ldr);
    if (bias) {
        if constexpr (N == 1) {
            b = *reinterpret_cast<const u32x4_t*>(bias + n[0]);
        } else {
            const u32x2_t v = *reinterpret_cast<const u32x2_t*>(bias + n[0]), w = *reinterpret_cast<const u32x2_t*>(bias + n[N - 1]);
            b = u32x4_t{v[0], v[1], w[0], w[1]};
        }
    }
    const Mask m = open_mask(drop);
    const u32x4_t bits = N == 1 ? draw(m, drop.group0 + g[0], drop.row0 + (uint32_t)r[0])
                                : draw_shared(m, drop.group0 + g[0], drop.row0 + (uint32_t)r[0], drop.group0 + g[N - 1], drop.row0 + (uint32_t)r[N - 1]);
    __builtin_amdgcn_sched_barrier(0);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (X_F32) v[j] = xf[j / C][j % C & 3];
        else                 v[j] = j & 1 ? bf16_hi(xb[j >> 1]) : bf16_lo(xb[j >> 1]);
    }
    if (bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] += bf16_lo(b[i]); v[2 * i + 1] += bf16_hi(b[i]); }
    }
    if constexpr (PRE) store_bf16(pre, ldp, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (GELU) v[i] = gelu_f(v[i]);
        v[i] = keeps(m, bits, i) ? v[i] * drop.factor : 0.0f;
    }
    if (res) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] += bf16_lo(q[i]); v[2 * i + 1] += bf16_hi(q[i]); }
    }
    if constexpr (Y_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i == 0 || both)
                __builtin_nontemporal_store(f32x4_t{v[C * i], v[C * i + 1], v[C * i + 2], v[C * i + 3]},
                                            reinterpret_cast<f32x4_t*>(static_cast<float*>(y) + r[i] * ldy + n[i]));
    } else {
        store_bf16(static_cast<uint16_t*>(y), ldy, v);
    }
}

// eight columns of dx = drop'(dz) GeLU'(a) before their rounding
template <bool GELU>
__device__ __forceinline__ void slope8(const Mask& m, float factor, const u32x4_t& bits, const u32x4_t& g, const u32x4_t& a, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = (i & 1 ? bf16_hi(g[i >> 1]) : bf16_lo(g[i >> 1])) * factor;
        float t = s;
        if constexpr (GELU) t = dgelu_times(s, i & 1 ? bf16_hi(a[i >> 1]) : bf16_lo(a[i >> 1]));
        v[i] = keeps(m, bits, i) ? t : 0.0f;
    }
}

template <bool GELU>
__global__ __launch_bounds__(256) void tp_dropout_bwd_kernel(const DropArgs drop, const uint16_t* dy, int64_t ld_dy, const uint16_t* pre,
                                                             int64_t ld_pre, uint16_t* dx, int64_t ld_dx, const uint32_t total, const Divisor d) {
    const uint32_t idx = blockIdx.x * 256u + threadIdx.x;
    if (idx >= total) return;
    const int64_t r = quotient(d, idx);
    const uint32_t g = idx - (uint32_t)r * d.d, n = g * 8;
    const u32x4_t s = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(dy + r * ld_dy + n));
    u32x4_t a = {0u, 0u, 0u, 0u};
    if constexpr (GELU) a = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(pre + r * ld_pre + n));
    const Mask m = open_mask(drop);
    const u32x4_t bits = draw(m, drop.group0 + g, drop.row0 + (uint32_t)r);      // (while the loads are under way)
    __builtin_amdgcn_sched_barrier(0);
    float v[8];
    slope8<GELU>(m, drop.factor, bits, s, a, v);
    const u32x4_t o = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(dx + r * ld_dx + n));
}

// The same with the column sums of dx, taken before its rounding: workgroup (bx, by) writes rows [by * per, ...) of columns COLS bx .. and their sums
// to out[by][cols]; 32 rows side by side, four in flight a thread.  The order of summation is fixed by the rows, the columns and the number of slabs.
constexpr int LANES = 32;
template <bool GELU, int COLS>
__global__ __launch_bounds__(COLS * 4) void tp_dropout_bwd_sum_kernel(const DropArgs drop, const uint16_t* dy, int64_t ld_dy, const uint16_t* pre,
                                                                      int64_t ld_pre, uint16_t* dx, int64_t ld_dx, int64_t rows, int cols, float* out,
                                                                      int64_t per) {
    __shared__ float part[LANES][COLS + 1];
    constexpr int CL = COLS / 8;
    const int cl = threadIdx.x % CL, rl = threadIdx.x / CL;
    const int c = blockIdx.x * COLS + cl * 8;
    const int64_t begin = (int64_t)blockIdx.y * per, end = begin + per < rows ? begin + per : rows;
    const Mask m = open_mask(drop);
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (c < cols) {
        for (int64_t r0 = begin + rl; r0 < end; r0 += 4 * LANES) {
            u32x4_t g[4], a[4], bits[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {                        // (rows past the end: the last one again, dropped below)
                const int64_t r = r0 + LANES * u < end ? r0 + LANES * u : end - 1;
                g[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(dy + r * ld_dy + c));
                if constexpr (GELU) a[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(pre + r * ld_pre + c));
                else                a[u] = g[u];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) bits[u] = draw(m, drop.group0 + (uint32_t)(c >> 3), drop.row0 + (uint32_t)(r0 + LANES * u));   // (while the loads are under way)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t r = r0 + LANES * u;
                if (r >= end) break;
                float v[8];
                slope8<GELU>(m, drop.factor, bits[u], g[u], a[u], v);
                const u32x4_t o = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
                __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(dx + r * ld_dx + c));
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] += v[i];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) part[rl][cl * 8 + i] = s[i];
    __syncthreads();
    if (threadIdx.x < COLS) {
        float tot = 0.0f;
#pragma unroll
        for (int r = 0; r < LANES; ++r) tot += part[r][threadIdx.x];
        const int cc = blockIdx.x * COLS + threadIdx.x;
        if (cc < cols) out[(int64_t)blockIdx.y * cols + cc] = tot;
    }
}

template <bool X_F32, bool GELU, bool PRE, bool Y_F32>
hipError_t forward(const DropArgs& drop, const void* x, int64_t ldx, const void* bias, const void* res, int64_t ldr, void* y, int64_t ldy, void* pre,
                   int64_t ldp, int64_t rows, int64_t cols, hipStream_t s) {
    return over_rows(rows, cols >> 3, [&](int64_t r, int64_t, uint32_t total, Divisor d) {
        DropArgs a = drop;
        a.row0 += (uint32_t)r;
        return launch_kernel(tp_dropout_kernel<X_F32, GELU, PRE, Y_F32>, covering(total), dim3(256), 0, s, a,
                             static_cast<const void*>(static_cast<const char*>(x) + r * ldx * (X_F32 ? 4 : 2)), ldx, static_cast<const uint16_t*>(bias),
                             res ? static_cast<const uint16_t*>(res) + r * ldr : nullptr, ldr,
                             static_cast<void*>(static_cast<char*>(y) + r * ldy * (Y_F32 ? 4 : 2)), ldy,
                             PRE ? static_cast<uint16_t*>(pre) + r * ldp : nullptr, ldp, total, d);
    });
}

// How the sums run: as those of a finished block, but in strips of 256 columns where those have 128 (16384 x 4096 51.1 us for 53.2, 32896 x 2560 with GeLU'
// 106.4 for 108.7: longer pieces of a row, and 32 rows side by side in a workgroup of 16 waves as before), and with the number of slabs, up to what the workspace holds, at which the CU with the most
// workgroups has the fewest rows: these kernels are bound by vector instructions as much as by memory, and a few workgroups beyond a whole round of the
// 256 CUs cost half a round (32896 x 2560 with GeLU', 20 strips of 128: 26 slabs 123.7 us, 25 108.7).
ColsumPlan sums_plan(int64_t rows, int64_t cols, bool has_ws) {
    ColsumPlan p = colsum_plan(rows, cols, has_ws, true);
    const int64_t strips = p.wide ? (cols + 255) / 256 : (cols + 63) / 64, weight = p.wide ? 2 : 1;
    auto slab = [&](int s) { return s == 1 ? rows : ((rows + s - 1) / s + 31) / 32 * 32; };
    auto longest = [&](int s) { return (strips * s * weight + 255) / 256 * slab(s); };
    int best = p.splits;
    for (int s = p.splits - 1; s >= 2; --s)
        if (longest(s) < longest(best)) best = s;
    p.splits = best;
    p.per = slab(best);
    return p;
}
template <bool GELU, int COLS>
hipError_t backward_sums(const DropArgs& drop, const ColsumPlan& p, const uint16_t* dy, int64_t ld_dy, const uint16_t* pre, int64_t ld_pre, uint16_t* dx,
                         int64_t ld_dx, int64_t rows, int64_t cols, float* db, float* ws, hipStream_t s) {
    const dim3 grid((unsigned)((cols + COLS - 1) / COLS), (unsigned)p.splits);
    if (hipError_t e = launch_kernel(tp_dropout_bwd_sum_kernel<GELU, COLS>, grid, dim3(COLS * 4), 0, s, drop, dy, ld_dy, pre, ld_pre, dx, ld_dx, rows,
                                     (int)cols, p.splits == 1 ? db : ws, p.per); e != hipSuccess || p.splits == 1)
        return e;
    return launch_colsum_finish(ws, p.splits, cols, db, s);
}

}  // namespace

hipError_t launch_dropout(const DropArgs& drop, const void* x, int64_t ldx, int x_f32, const void* bias, int gelu, const void* res, int64_t ldr, void* y,
                          int64_t ldy, int y_f32, void* pre, int64_t ldp, int64_t rows, int64_t cols, hipStream_t s) {
    using Y = std::true_type;
    using N = std::false_type;
    auto pick = [&](auto xf, auto g, auto p) {
        constexpr bool X = decltype(xf)::value, G = decltype(g)::value, P = decltype(p)::value;
        return y_f32 ? forward<X, G, P, true>(drop, x, ldx, bias, res, ldr, y, ldy, pre, ldp, rows, cols, s)
                     : forward<X, G, P, false>(drop, x, ldx, bias, res, ldr, y, ldy, pre, ldp, rows, cols, s);
    };
    auto typed = [&](auto xf) { return gelu ? (pre ? pick(xf, Y{}, Y{}) : pick(xf, Y{}, N{})) : (pre ? pick(xf, N{}, Y{}) : pick(xf, N{}, N{})); };
    return x_f32 ? typed(Y{}) : typed(N{});
}

hipError_t launch_dropout_bwd(const DropArgs& drop, const void* dy, int64_t ld_dy, const void* pre, int64_t ld_pre, void* dx, int64_t ld_dx, int64_t rows,
                              int64_t cols, float* db, float* ws, hipStream_t s) {
    const uint16_t *g = static_cast<const uint16_t*>(dy), *a = static_cast<const uint16_t*>(pre);
    uint16_t* const o = static_cast<uint16_t*>(dx);
    if (db) {
        const ColsumPlan p = sums_plan(rows, cols, ws != nullptr);
        auto pick = [&](auto gelu) {
            constexpr bool G = decltype(gelu)::value;
            return p.wide ? backward_sums<G, 256>(drop, p, g, ld_dy, a, ld_pre, o, ld_dx, rows, cols, db, ws, s)
                          : backward_sums<G, 64>(drop, p, g, ld_dy, a, ld_pre, o, ld_dx, rows, cols, db, ws, s);
        };
        return a ? pick(std::true_type{}) : pick(std::false_type{});
    }
    return over_rows(rows, cols >> 3, [&](int64_t r, int64_t, uint32_t total, Divisor d) {
        DropArgs m = drop;
        m.row0 += (uint32_t)r;
        return launch_kernel(a ? tp_dropout_bwd_kernel<true> : tp_dropout_bwd_kernel<false>, covering(total), dim3(256), 0, s, m, g + r * ld_dy, ld_dy,
                             a ? a + r * ld_pre : nullptr, ld_pre, o + r * ld_dx, ld_dx, total, d);
    });
}

}  // namespace tpl
