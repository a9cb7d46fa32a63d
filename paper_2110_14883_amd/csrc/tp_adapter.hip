// gfx950 (MI355X, CDNA4): low-rank adapters of many requests beside a shared projection (paper Section 2.2: the projection is a rank's share of the
// linear layer).  With the factors A_i: [rank, H], B_i: [rank, F] and scale s_i of a row's adapter i
//   forward   V = drop(X) A_i^T,   Y = act(C + s_i V B_i + bias)
//   backward  U = dY B_i^T,        dX = dX_base + drop'(s_i U A_i),    dA_i = s_i U^T drop(X),   dB_i = s_i V^T dY
// Both factors lie as `rank` long rows, so forward and backward are the same three products:
//   down  [rows, K] x [rank, K]^T      both operands contraction-contiguous, through LDS
//   up    [rows, rank] x [rank, cols]  the factor's 8 x 8 blocks transposed in registers
//   grad  [rows, rank]^T x [rows, cols]  the same turn of the second operand, sums over rows
// All three are bound by memory: with 8 to 128 ranks *down* and *grad* take 8 to 128 flops a byte of X or dY, *up* 2 to 64 a byte of C and its result.
// V and U stay in fp32.  Where they are a matrix operand they go in as a sum of bf16 terms, two (2^-17) for bf16 results and three (2^-25) for fp32 ones:
// the matrix unit has the time, and rounding them once would cost a bf16 step of the adapters' part.
// Measured (all of a call, us, and the bytes it cannot do without over that): one token of 4096 x 4096, 16 ranks 7.4; 96 tokens over 48 adapters 9.5; 5923
// rows in 12 segments, 32 ranks, GeLU 56 (4.4 TB/s); 2048 x 4 x 2048 x 8192, 64 ranks, dropout 30 (3.5); backward of 16384 x 4096 x 4096, 16 ranks, dropout,
// fp32 178 (4.5), of 32896 x 640 over 2 x 2560, 8 ranks, three quarters of the rows with an adapter 101 (3.6).  A large copy reaches 5.2 TB/s.
//
// Rows come in segments, a request each, described by device arrays.  A workgroup works on a tile of one segment's rows: it finds its tile from
// the offsets itself (one trip to memory for up to 64 segments), so a call is the same launches whatever the lengths, and can be captured.  Offsets are
// clamped to the rows there are and an adapter that the pool does not have is none: bad ones give wrong rows, never a wild access.
#include "tp_random.h"
#include "tp_stream.h"

namespace tpl {

namespace {

__device__ __forceinline__ float as_float(uint32_t w) { return __builtin_bit_cast(float, w); }   // (of a value: a bit cast of a vector's element takes its first one)

// inclusive sum over the wave's lanes: inside rows of 16 lanes, then the last lane of row 0 (2) to row 1 (3), that of row 1 to rows 2 and 3
__device__ __forceinline__ int wave_sums(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);      // from 1, 2, 4, 8 lanes below
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}
// rows [lo, lo + len) of segment i, clamped, and its adapter (-1: none)
__device__ __forceinline__ void segment(const SegArgs& s, int i, int& lo, int& len, int& id) {
    lo = len = 0;
    id = -1;
    if (i < s.n) {
        lo = s.offsets[i];
        int hi = s.offsets[i + 1];
        const int k = s.ids[i];
        lo = lo < 0 ? 0 : lo > s.rows ? s.rows : lo;
        hi = hi < 0 ? 0 : hi > s.rows ? s.rows : hi;
        len = hi > lo ? hi - lo : 0;
        id = k >= 0 && k < s.pool ? k : -1;
    }
}

// Asks for the scalar arguments that a kernel's start goes through one after the other, so that they come in one trip (the others are loaded where they
// are needed).
__device__ __forceinline__ void preload(const DownArgs& d) {
    asm volatile("" :: "s"(d.seg.offsets), "s"(d.seg.ids), "s"(d.seg.n), "s"(d.seg.rows), "s"(d.seg.pool), "s"(d.n_steps), "s"(d.K), "s"(d.rank), "s"(d.splits));
    asm volatile("" :: "s"(d.p[0]), "s"(d.f[0]), "s"(d.strides[0]), "s"(d.ldp[0]), "s"(d.ldf[0]), "s"(d.out), "s"(d.plane));
}
__device__ __forceinline__ void preload(const UpArgs& u) {
    asm volatile("" :: "s"(u.seg.offsets), "s"(u.seg.ids), "s"(u.seg.n), "s"(u.seg.rows), "s"(u.seg.pool), "s"(u.f), "s"(u.stride), "s"(u.ldf), "s"(u.rank), "s"(u.cols));
    asm volatile("" :: "s"(u.scale), "s"(u.c), "s"(u.ldc), "s"(u.bias), "s"(u.gelu), "s"(u.out), "s"(u.ldo), "s"(u.pre), "s"(u.v), "s"(u.v_out), "s"(u.tile));
}

struct Tile { int row0, rows, id; };
// tile t of the tiles of at most T rows that the segments have, in their order; the same for every lane of a wave
__device__ __forceinline__ bool find_tile(const SegArgs& s, int t, int T, Tile& out) {
    const int l = threadIdx.x & 63;
    int base = 0;
    for (int first = 0; first < s.n; first += 64) {
        int lo, len, id;
        segment(s, first + l, lo, len, id);
        const int count = (len + T - 1) / T, sums = wave_sums(count);
        const uint64_t behind = __ballot(base + sums > t);
        if (behind) {
            const int j = __builtin_ctzll(behind);
            const int at = __builtin_amdgcn_readlane(lo, j), end = at + __builtin_amdgcn_readlane(len, j);
            out.row0 = at + (t - base - (__builtin_amdgcn_readlane(sums, j) - __builtin_amdgcn_readlane(count, j))) * T;
            out.rows = end - out.row0 < T ? end - out.row0 : T;
            out.id = __builtin_amdgcn_readlane(id, j);
            return out.row0 >= at && out.rows > 0;               // (not so only where sums of wild offsets overflow)
        }
        base += __builtin_amdgcn_readlane(sums, 63);
    }
    return false;
}

// 8 values -> their bf16 terms: v = t[0] + t[1] (+ t[2]).  The first is held to bf16's finite range: from 2^128 - 2^119 on fp32 numbers would round to an
// infinity there, and leave another of the other sign.  (So an infinity has bf16's largest value as its first term and itself as the second.)
template <int N>       // 2, 3
__device__ __forceinline__ void split_terms(const float (&v)[8], u32x4_t (&t)[N]) {
    constexpr float TOP = 0x1.FEp127f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[0][i] = pack_bf16(__builtin_amdgcn_fmed3f(v[2 * i], -TOP, TOP), __builtin_amdgcn_fmed3f(v[2 * i + 1], -TOP, TOP));
        const float a = v[2 * i] - bf16_lo(t[0][i]), b = v[2 * i + 1] - bf16_hi(t[0][i]);
        t[1][i] = pack_bf16(a, b);
        if constexpr (N == 3) {
            const float c = a - bf16_lo(t[1][i]), d = b - bf16_hi(t[1][i]);
            t[2][i] = pack_bf16(c == c ? c : 0.0f, d == d ? d : 0.0f);               // (infinity less infinity: nothing is left)
        }
    }
}
// 8 x 8 block: in[j] is row j of eight columns -> out[e] is column e of eight rows
__device__ __forceinline__ void transpose8(const u32x4_t (&in)[8], u32x4_t (&out)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
        for (int i = 0; i < 4; ++i) out[e][i] = __builtin_amdgcn_perm(in[2 * i + 1][e >> 1], in[2 * i][e >> 1], sel);
    }
}
__device__ __forceinline__ f32x4_t mfma(const u32x4_t& a, const u32x4_t& b, const f32x4_t& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// ---------------------------------------------------------------------------------------------
// down.  A tile of 16 MT rows by all 16 RB ranks.  The waves of a workgroup, and the workgroups of a tile, take the units of 64 k in turn (so neighbouring
// waves read neighbouring cache lines of a row), and the waves' sums meet in LDS in their order.  A wave has a ring of LDS slots of its own, filled by
// direct-to-LDS loads of 8 whole lines each, with no barrier in the loop.  (Fragments loaded straight into registers, 64 bytes of 16 rows an
// instruction, kept the address path busy longer: 16384 x 4096, 16 ranks 34.2 us against 28.5, 32896 x 2 x 2560 in 24 segments 67 / 46.)
// ---------------------------------------------------------------------------------------------
// (with a mask to draw, the waves count for more than the slots.  At 128 ranks a slot is 24 KB: six waves with one each 16384 x 4096 46.1 us, four 52.4, three with
// two 45.6, and 7731 x 7296 with a mask, forward, 91.8 / 95.3 / 105; tiles of 32 rows, 731 of 2496: four with two slots 9.2, eight with one 10.4, with a mask 553 of 3968 17.6 / 14.2.)
constexpr int down_waves(int mt, int rb, bool drop) {
    if (rb == 8) return mt == 4 ? 6 : mt == 2 && drop ? 8 : 4;
    return mt + rb <= (drop ? 8 : 5) ? 8 : 4;
}
template <int MT, int RB, bool DROP> struct DownShape {
    static constexpr int WAVES = down_waves(MT, RB, DROP);
    static constexpr int SLOT = (MT + RB) * 2048;                                               // a unit: lines of 16 MT rows, of 16 RB ranks
    static constexpr int FIT = 163840 / (WAVES * SLOT), NS = FIT > 4 ? 4 : FIT;
    static constexpr int PART = 16 * RB + 4, SUMS = WAVES * 16 * PART * 4;                      // the waves' sums of 16 rows
    static constexpr int BYTES = WAVES * NS * SLOT > SUMS ? WAVES * NS * SLOT : SUMS;
    static_assert(NS >= 1 && BYTES <= 163840);
};
// one wave's sums over units share, share + shares, ... of tile t: acc[i][j][e] is row 16 i + c, rank 16 j + 4 g + e.  Its ring begins at byte `mine`.
// XL: loads of eight rows of P each that the tile needs (rows beyond them are whatever LDS holds; so are their sums, which nobody reads).
template <int MT, int RB, int NS, bool DROP, int XL>
__device__ __forceinline__ void down_sums(const DownArgs& p, const Tile& t, const int share, const int shares, const uint32_t mine, f32x4_t (&acc)[MT][RB]) {
    constexpr int X_BYTES = MT * 2048, SLOT = (MT + RB) * 2048, LOADS = XL + 2 * RB;
    const int l = threadIdx.x & 63, c = l & 15, g = l >> 4;
    const int KT = (p.K + 63) / 64, total = p.n_steps * KT;
    Mask m;
    if constexpr (DROP) m = open_mask(p.drop);
    // rows of 128 bytes, 16-byte chunk q of row r at q ^ ((r >> 1) & 7): reads of one chunk of 16 rows lie in different banks
    const int lr = l >> 3;
    // (descriptors and leading dimensions stay in scalar registers until the step changes: asked for again for every unit, they took 0.4 us of it)
    u32x4_t rx, rf;
    int ldp = 0, ldf = 0;
    auto describe = [&](const uint16_t* base, int64_t bytes) __attribute__((always_inline)) {
        const uint64_t at = reinterpret_cast<uint64_t>(base);
        return u32x4_t{(uint32_t)uni((int)(uint32_t)at), (uint32_t)uni((int)((uint32_t)(at >> 32) & 0xffffu)), (uint32_t)uni((int)(uint32_t)bytes), 0x00020000u};
    };
    auto open_step = [&](int s) __attribute__((always_inline)) {
        if (s < p.n_steps) {
            ldp = p.ldp[s];
            ldf = p.ldf[s];
            rx = describe(static_cast<const uint16_t*>(p.p[s]) + (int64_t)t.row0 * ldp, ((int64_t)(t.rows - 1) * ldp + p.K) * 2);
            rf = describe(static_cast<const uint16_t*>(p.f[s]) + t.id * p.strides[s], ((int64_t)(p.rank - 1) * ldf + p.K) * 2);
        } else {
            rx[2] = rf[2] = 0;
        }
    };
    auto load = [&](auto n_loads, const u32x4_t& rs, int ld, int k0, uint32_t dst) __attribute__((always_inline)) {
        static_for<decltype(n_loads)::value>([&](auto n_) __attribute__((always_inline)) {
            constexpr int n = decltype(n_)::value;
            const int r = 8 * n + lr, k = k0 + (((l & 7) ^ ((r >> 1) & 7)) << 3);
            dtl_load16(rs, k < p.K ? (uint32_t)((r * ld + k) * 2) : OOB_OFFSET, dst + n * 1024);
        });
    };
    int f_step = 0, f_kt = share;                                        // the unit to fetch next
    while (f_kt >= KT && f_step < p.n_steps) { f_kt -= KT; ++f_step; }
    rx = rf = u32x4_t{0u, 0u, 0u, 0x00020000u};
    open_step(f_step);
    auto fetch = [&](int slot) __attribute__((always_inline)) {          // (past the end: empty descriptors, zeros that nobody uses)
        const uint32_t dst = mine + (uint32_t)(slot * SLOT);
        load(std::integral_constant<int, XL>{}, rx, ldp, 64 * f_kt, dst);
        load(std::integral_constant<int, 2 * RB>{}, rf, ldf, 64 * f_kt, dst + X_BYTES);
        f_kt += shares;
        if (f_kt >= KT && f_step < p.n_steps) {
            do { f_kt -= KT; ++f_step; } while (f_kt >= KT && f_step < p.n_steps);
            open_step(f_step);
        }
    };
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) fetch(s);
    int slot = 0, step = 0, kt = share;                                  // the unit to multiply
    while (kt >= KT && step < p.n_steps) { kt -= KT; ++step; }
    for (int u = share; u < total; u += shares) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");               // the slot to refill has been read
        fetch(slot == 0 ? NS - 1 : slot - 1);
        u32x4_t bits[DROP ? 2 * MT : 1];
        if constexpr (DROP) {                                            // (the draws need nothing that is under way)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    bits[MT * h + i] = draw(m, p.group0[step] + 8 * kt + 4 * h + g, p.drop.row0 + (uint32_t)(t.row0 + 16 * i + c));
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_vm<(NS - 1) * LOADS>();
        asm volatile("" ::: "memory");
        const uint32_t at = mine + (uint32_t)(slot * SLOT);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            auto frag = [&](uint32_t base, int i) __attribute__((always_inline)) {
                const int r = 16 * i + c;
                return lds_load_frag(base + r * 128 + (((4 * h + g) ^ ((r >> 1) & 7)) << 4));
            };
            bf16x8_t f[RB];
#pragma unroll
            for (int j = 0; j < RB; ++j) f[j] = frag(at + X_BYTES, j);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                u32x4_t x = __builtin_bit_cast(u32x4_t, frag(at, i));
                if constexpr (DROP) x = clear_dropped(m, bits[MT * h + i], x);
#pragma unroll
                for (int j = 0; j < RB; ++j) acc[i][j] = mfma(__builtin_bit_cast(u32x4_t, f[j]), x, acc[i][j]);
            }
        }
        slot = slot + 1 == NS ? 0 : slot + 1;
        for (kt += shares; kt >= KT && step < p.n_steps; ++step) kt -= KT;
    }
    wait_vm<0>();                                                        // (zeros on their way into slots)
}
// four ranks from 4 q on of row `row` of 16 rows: the waves' sums in their order
template <int PART, int WAVES>
__device__ __forceinline__ f32x4_t waves_sum(const float* part, int row, int q) {
    f32x4_t s = *reinterpret_cast<const f32x4_t*>(part + row * PART + 4 * q);
#pragma unroll
    for (int v = 1; v < WAVES; ++v) s += *reinterpret_cast<const f32x4_t*>(part + (v * 16 + row) * PART + 4 * q);
    return s;
}
template <int MT, int RB, bool DROP>
__global__ __launch_bounds__(64 * down_waves(MT, RB, DROP)) void tp_adapter_down_kernel(const DownArgs p) {
    using Sh = DownShape<MT, RB, DROP>;
    constexpr int WAVES = Sh::WAVES;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    preload(p);
    Tile t;
    if (!find_tile(p.seg, blockIdx.x, 16 * MT, t) || t.id < 0) return;
    const int l = threadIdx.x & 63, c = l & 15, g = l >> 4, w = uni(threadIdx.x >> 6);
    f32x4_t acc[MT][RB];
    down_sums<MT, RB, Sh::NS, DROP, 2 * MT>(p, t, blockIdx.y * WAVES + w, p.splits * WAVES, (uint32_t)(w * Sh::NS * Sh::SLOT), acc);
    __syncthreads();
    float* const part = reinterpret_cast<float*>(lds);
    float* const out = p.out + blockIdx.y * p.plane;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int j = 0; j < RB; ++j) *reinterpret_cast<f32x4_t*>(part + (w * 16 + c) * Sh::PART + 16 * j + 4 * g) = acc[i][j];
        __syncthreads();
        for (int x = threadIdx.x; x < 64 * RB; x += 64 * WAVES) {
            const int row = x / (4 * RB), q = x % (4 * RB);
            if (16 * i + row >= t.rows || 4 * q >= p.rank) continue;
            f32x4_t s = waves_sum<Sh::PART, WAVES>(part, row, q);
            if constexpr (DROP) s *= p.drop.factor;
            *reinterpret_cast<f32x4_t*>(out + (int64_t)(t.row0 + 16 * i + row) * p.rank + 4 * q) = s;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The shares' planes of dA and dB (grad, below) added in order, eight on their way at a time; a share without rows has none.  Four elements a thread, block `block` of
// finish_share().  In a backward pass that also wants dX this is done by workgroups of *up* behind its tiles, otherwise by a launch of its own (backward of
// 32896 x 640 over 2 x 2560, 8 ranks 101 us against 105; 16384 x 4096 x 4096, 16 ranks 178.3 against 178.9).
// ---------------------------------------------------------------------------------------------
__host__ __device__ inline int finish_blocks_each(const GradArgs& p, int threads) {
    const int most = p.sides > 1 && p.side[1].cols > p.side[0].cols ? p.side[1].cols : p.side[0].cols;
    return (most * p.rank / 4 + threads - 1) / threads;                  // (up to 2^21 columns)
}
__device__ __forceinline__ void finish_share(const GradArgs& p, unsigned block) {
    const unsigned each = (unsigned)finish_blocks_each(p, blockDim.x), y = block / each;
    if (y >= (unsigned)(p.seg.pool * p.sides)) return;
    const int which = y >= (unsigned)p.seg.pool, a = which ? y - p.seg.pool : y;
    const GradSide& q = p.side[which];
    const unsigned at = ((block - y * each) * blockDim.x + threadIdx.x) * 4, plane = (unsigned)(p.rank * q.cols);      // (up to 128 x 2^21)
    if (at >= plane) return;
    const unsigned k = at / (unsigned)q.cols, cc = at - k * (unsigned)q.cols;
    const float* const part = q.part + (int64_t)a * p.shares * plane + at;
    const unsigned total = (unsigned)p.units[a], shares = (unsigned)p.shares;
    f32x4_t* const to = reinterpret_cast<f32x4_t*>(q.out + a * q.stride + k * q.ldo + cc);
    f32x4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int z0 = 0; z0 < p.shares; z0 += 8) {
        f32x4_t v[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            const int y = z0 + z;
            v[z] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            if (y < p.shares && (total >= shares || total * y / shares < total * (y + 1) / shares))
                v[z] = *reinterpret_cast<const f32x4_t*>(part + (int64_t)y * plane);
        }
#pragma unroll
        for (int z = 0; z < 8; ++z) s += v[z];
    }
    if (p.accumulate) s = *to + s;
    *to = s;
}

// ---------------------------------------------------------------------------------------------
// up.  A workgroup has a tile of rows and, a wave each, strips of 128 columns.  It first lays V's terms out in LDS, as the rows of the second product's
// left operand: first terms, second terms (third ones) of a row's ranks one behind the other, so that for up to 16 ranks two terms fill one matrix
// instruction's 32 k.  A wave turns its strip of the factor into matrix operands once, eight 16-column blocks, so that a lane ends up with eight
// columns of four rows: columns 8 c .. 8 c + 7 where C and the result are bf16, else 4 c .. 4 c + 3 and 64 + 4 c .. + 3, which makes every access of
// a row 16 (8) neighbouring bytes a lane and one draw a row either way.  (32 bytes a lane in two halves: each streamed store is half of a sector.)
// The next 16 rows of C are on their way while these are finished.
// GP: groups of eight ranks (2, 4, 8, 16: up to 16, 32, 64, 128 ranks; those beyond the rank are zeros).
// ---------------------------------------------------------------------------------------------
template <int GP, int TERMS> struct UpShape {
    static constexpr int NS = GP >= 4 ? GP / 4 : 1;                      // blocks of 32 k that the factor has
    static constexpr int STEPS = (TERMS * GP + 3) / 4;                   // and V's terms
    static constexpr int ROW = STEPS * 64 + 16;                          // bytes of a row in LDS (16 more: rows start in different banks)
    // How many times 16 rows of C are on their way while others are finished: what leaves the waves that run without (two where two a SIMD fit anyway: 2048 x
    // 8192, 64 ranks 19.6 -> 18.6 us; three instead of four waves a SIMD for it: 32896 x 640, 8 ranks 19.6 -> 23.8)
    template <bool C32> static constexpr int AHEAD = C32 ? (GP < 16 ? 1 : 0) : (GP == 8 ? 2 : 1);
};
template <bool C32> struct CRows { u32x4_t v[4][C32 ? 2 : 1]; };
template <int GP, int TERMS, bool DROP, bool C32>
struct UpStrip {
    using Sh = UpShape<GP, TERMS>;
    static constexpr bool O32 = TERMS == 3, WIDE = !C32 && !O32;
    static constexpr int CB = C32 ? 4 : 2;
    const UpArgs& p;
    const Tile& t;
    int c, g, n;
    bool in, in1;
    // the lane's columns: n .. n + 7, or n .. n + 3 and n + 64 .. n + 67
    __device__ __forceinline__ UpStrip(const UpArgs& args, const Tile& tile, int strip) : p(args), t(tile) {
        const int l = threadIdx.x & 63;
        c = l & 15;
        g = l >> 4;
        n = strip * 128 + (WIDE ? 8 : 4) * c;
        in = n < p.cols;
        in1 = WIDE ? in : n + 64 < p.cols;
    }
    // C of rows r0 + 4 g + e (past the end: the last row; past the columns: the first ones)
    __device__ __forceinline__ void load_c(CRows<C32>& q, int r0) const {
        const char* const c0 = static_cast<const char*>(p.c) + (int64_t)t.row0 * p.ldc * CB;
        const int at0 = (in ? n : 0) * CB, at1 = (in1 ? n + 64 : 0) * CB;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = r0 + 4 * g + e < t.rows ? r0 + 4 * g + e : t.rows - 1;
            const char* const row = c0 + r * p.ldc * CB;
            if constexpr (C32) {
                q.v[e][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + at0));
                q.v[e][1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + at1));
            } else if constexpr (WIDE) {
                q.v[e][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + at0));
            } else {
                const u32x2_t a = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(row + at0));
                const u32x2_t b = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(row + at1));
                q.v[e][0] = u32x4_t{a[0], a[1], b[0], b[1]};
            }
        }
    }
    // the strip of the factor, and its rows turned into matrix operands.  Up to 16 ranks both halves of the wave need the same eight rows a lane: each
    // loads four of them, and they swap.
    __device__ __forceinline__ void load_factor(u32x4_t (&f)[Sh::NS][8]) const {
        const __amdgpu_buffer_rsrc_t rf = make_rsrc(static_cast<const uint16_t*>(p.f) + t.id * p.stride, ((int64_t)(p.rank - 1) * p.ldf + p.cols) * 2);
#pragma unroll
        for (int s = 0; s < Sh::NS; ++s) {
            const int k = GP >= 4 ? 8 * (4 * s + g) : 8 * (g & 1) + 4 * (g >> 1);
            const bool ok = k < p.rank;
#pragma unroll
            for (int j = 0; j < (GP >= 4 ? 8 : 4); ++j) {
                const uint32_t at = (uint32_t)(((k + j) * p.ldf + n) * 2);
                if constexpr (WIDE) {
                    f[s][j] = buf_load16(rf, ok && in ? at : OOB_OFFSET);
                } else {
                    const u32x2_t a = __builtin_amdgcn_raw_buffer_load_b64(rf, (int)(ok && in ? at : OOB_OFFSET), 0, 0);
                    const u32x2_t b = __builtin_amdgcn_raw_buffer_load_b64(rf, (int)(ok && in1 ? at + 128 : OOB_OFFSET), 0, 0);
                    f[s][j] = u32x4_t{a[0], a[1], b[0], b[1]};
                }
            }
        }
    }
    __device__ __forceinline__ void turn(u32x4_t (&f)[Sh::NS][8]) const {
        if constexpr (GP < 4) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {                            // lanes 0 - 31 of both, lanes 32 - 63 of both
                    const u32x2_t x = __builtin_amdgcn_permlane32_swap(f[0][j][i], f[0][j][i], false, false);
                    f[0][j][i] = x[0];
                    f[0][4 + j][i] = x[1];
                }
        }
#pragma unroll
        for (int s = 0; s < Sh::NS; ++s) {
            u32x4_t o[8];
            transpose8(f[s], o);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[s][j] = o[j];
        }
    }
    __device__ __forceinline__ u32x4_t load_bias() const {
        u32x4_t bias = {0u, 0u, 0u, 0u};
        if (p.bias) {
            const char* const b = static_cast<const char*>(p.bias);
            if constexpr (WIDE) {
                bias = *reinterpret_cast<const u32x4_t*>(b + (in ? n : 0) * 2);
            } else {
                const u32x2_t q = *reinterpret_cast<const u32x2_t*>(b + (in ? n : 0) * 2), s = *reinterpret_cast<const u32x2_t*>(b + (in1 ? n + 64 : 0) * 2);
                bias = u32x4_t{q[0], q[1], s[0], s[1]};
            }
        }
        return bias;
    }
    __device__ __forceinline__ void store_bf16(void* base, int64_t ld, int64_t row, const float (&v)[8]) const {
        uint16_t* const to = static_cast<uint16_t*>(base) + row * ld + n;
        const u32x4_t o = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        if constexpr (WIDE) {
            if (in) __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(to));
        } else {
            if (in) __builtin_nontemporal_store(u32x2_t{o[0], o[1]}, reinterpret_cast<u32x2_t*>(to));
            if (in1) __builtin_nontemporal_store(u32x2_t{o[2], o[3]}, reinterpret_cast<u32x2_t*>(to + 64));
        }
    }
    // rows r0 .. r0 + 15 of the tile from V's terms at `low` (adapted) and their C
    __device__ __forceinline__ void rows16(const char* low, const u32x4_t (&f)[Sh::NS][8], const CRows<C32>& cv, const u32x4_t& bias, const Mask& m, int r0, bool adapted) const {
        f32x4_t acc[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (adapted) {
            const int r = r0 + c < t.rows ? r0 + c : t.rows - 1;
#pragma unroll
            for (int s = 0; s < Sh::STEPS; ++s) {
                const u32x4_t v = *reinterpret_cast<const u32x4_t*>(low + r * Sh::ROW + s * 64 + g * 16);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = mfma(v, f[s % Sh::NS][j], acc[j]);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = r0 + 4 * g + e;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (C32) v[j] = as_float(cv.v[e][j >> 2][j & 3]);
                else               v[j] = j & 1 ? bf16_hi(cv.v[e][0][j >> 1]) : bf16_lo(cv.v[e][0][j >> 1]);
            }
            if constexpr (DROP) {
                const uint32_t row = p.drop.row0 + (uint32_t)(t.row0 + r), group = p.drop.group0 + (uint32_t)(n >> 3);
                const u32x4_t bits = WIDE ? draw(m, group, row) : draw_shared(m, group, row, group + 8, row);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += keeps(m, bits, j) ? acc[j][e] : 0.0f;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += acc[j][e];
            }
            if (p.bias) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += j & 1 ? bf16_hi(bias[j >> 1]) : bf16_lo(bias[j >> 1]);
            }
            if (r >= t.rows) continue;
            const int64_t row = t.row0 + r;
            if (p.pre) store_bf16(p.pre, p.ldp, row, v);
            if (p.gelu) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = gelu_f(v[j]);
            }
            if constexpr (O32) {
                float* const to = static_cast<float*>(p.out) + row * p.ldo + n;
                if (in) __builtin_nontemporal_store(f32x4_t{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_t*>(to));
                if (in1) __builtin_nontemporal_store(f32x4_t{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4_t*>(to + 64));
            } else {
                store_bf16(p.out, p.ldo, row, v);
            }
        }
    }
};
// eight ranks' terms of row r, group q of V (already scaled), to LDS
template <int GP, int TERMS>
__device__ __forceinline__ void lay_terms(char* low, int r, int q, const float (&v)[8]) {
    using Sh = UpShape<GP, TERMS>;
    u32x4_t term[TERMS];
    split_terms(v, term);
#pragma unroll
    for (int s = 0; s < TERMS; ++s) *reinterpret_cast<u32x4_t*>(low + r * Sh::ROW + (s * GP + q) * 16) = term[s];
    if constexpr (Sh::STEPS * 4 > TERMS * GP) *reinterpret_cast<u32x4_t*>(low + r * Sh::ROW + (TERMS * GP + q) * 16) = u32x4_t{0u, 0u, 0u, 0u};
}

template <int GP, int TERMS, bool DROP, bool C32>
__global__ __launch_bounds__(384) void tp_adapter_up_kernel(const UpArgs p, const GradArgs fin) {
    using Strip = UpStrip<GP, TERMS, DROP, C32>;
    constexpr int AHEAD = UpShape<GP, TERMS>::template AHEAD<C32>;
    extern __shared__ __attribute__((aligned(16))) char low[];
    const int w = uni(threadIdx.x >> 6), strip = w < p.waves ? blockIdx.y * p.waves + w : 1 << 20;
    const bool mine = strip * 128 < p.cols;
    if (blockIdx.x >= (unsigned)p.tiles) {
        finish_share(fin, (blockIdx.x - p.tiles) * gridDim.y + blockIdx.y);
        return;
    }
    preload(p);
    Tile t;
    if (!find_tile(p.seg, blockIdx.x, p.tile, t)) return;
    const bool adapted = t.id >= 0;
    const Strip st(p, t, strip);
    u32x4_t f[UpShape<GP, TERMS>::NS][8];
    CRows<C32> cv[AHEAD ? AHEAD : 1];
    auto start_c = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) st.load_c(cv[i], 16 * i);
    };
    if (mine) {
        if (adapted) st.load_factor(f);
        start_c();
    }
    if (adapted) {
        // V's terms; eight ranks of a row a thread
        const float scale = (p.scale ? p.scale[t.id] : 1.0f) * (DROP ? p.drop.factor : 1.0f);
        for (int i = threadIdx.x; i < t.rows * GP; i += blockDim.x) {
            const int r = i / GP, q = i % GP;
            float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (8 * q < p.rank) {
                const int64_t at = (int64_t)(t.row0 + r) * p.rank + 8 * q;
                for (int z0 = 0; z0 < p.splits; z0 += 4) {               // (four planes on their way at a time)
                    f32x4_t a[4], b[4];
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        a[z] = b[z] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                        if (z0 + z < p.splits) {
                            const f32x4_t* src = reinterpret_cast<const f32x4_t*>(p.v + (z0 + z) * p.plane + at);
                            a[z] = src[0];
                            b[z] = src[1];
                        }
                    }
#pragma unroll
                    for (int z = 0; z < 4; ++z)
#pragma unroll
                        for (int k = 0; k < 4; ++k) { v[k] += a[z][k]; v[4 + k] += b[z][k]; }
                }
                if (p.v_out && blockIdx.y == 0) {
                    f32x4_t* const to = reinterpret_cast<f32x4_t*>(p.v_out + at);
                    to[0] = f32x4_t{v[0], v[1], v[2], v[3]};
                    to[1] = f32x4_t{v[4], v[5], v[6], v[7]};
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= scale;
            }
            lay_terms<GP, TERMS>(low, r, q, v);
        }
        if (mine) st.turn(f);
    }
    __syncthreads();
    if (!mine) return;
    Mask m;
    if constexpr (DROP) m = open_mask(p.drop);
    const u32x4_t bias = st.load_bias();
    if constexpr (AHEAD) {
        for (int r0 = 0; r0 < t.rows; r0 += 16 * AHEAD)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int r = r0 + 16 * i;
                if (r >= t.rows) return;
                const CRows<C32> now = cv[i];
                if (r + 16 * AHEAD < t.rows) st.load_c(cv[i], r + 16 * AHEAD);
                st.rows16(low, f, now, bias, m, r, adapted);
            }
    } else {
        for (int r0 = 0; r0 < t.rows; r0 += 16) {
            st.load_c(cv[0], r0);
            st.rows16(low, f, cv[0], bias, m, r0, adapted);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// few.  Both products of a tile of 16 rows in one launch, for segments of a few rows (a decoding batch): every workgroup of a tile forms V by itself, its waves
// sharing K, and goes on with its own strips.  The factor's first strip and C come in meanwhile.  Bound by latency: a launch, one trip for the
// segment, one for the operands; with many requests by the factors.  What is read more than once is A, once for every workgroup of
// a tile, from L2.
// ---------------------------------------------------------------------------------------------
constexpr int few_waves(int rb) { return rb <= 4 ? 8 : 4; }              // (as many as leave a wave its registers)
template <int RB> struct FewShape {                                      // RB: blocks of 16 ranks
    static constexpr int WAVES = few_waves(RB), SLOT = (1 + RB) * 2048, FIT = 163840 / (WAVES * SLOT);
    static constexpr int NS = RB == 1 ? 2 : FIT > 4 ? 4 : FIT;           // (up to 16 ranks, so that two workgroups share a CU where the registers allow it, below)
    static constexpr int PART = 16 * RB + 4, SUMS = WAVES * 16 * PART * 4;
    static constexpr int LOW = 16 * UpShape<2 * RB, 3>::ROW;             // behind the waves' sums, where the ring was
    static constexpr int BYTES = WAVES * NS * SLOT > SUMS + LOW ? WAVES * NS * SLOT : SUMS + LOW;
    static_assert(NS >= 1 && BYTES <= 163840);
};
// Up to 16 ranks and bf16 throughout the registers are held to what lets two workgroups share a CU (1000 single rows of 4096 x 4096 50 -> 35 us, one row 6.7 -> 6.5);
// elsewhere that would spill (32 ranks, 1000 rows 57 -> 63).  With an fp32 side up to 16 ranks take 134 to 152 registers: one workgroup a CU there,
// though the ring has two slots for them too.
constexpr int few_waves_a_simd(int rb, int terms, bool c32) { return rb == 1 && terms == 2 && !c32 ? 4 : 1; }
template <int RB, int TERMS, bool C32>
__global__ __launch_bounds__(64 * few_waves(RB), few_waves_a_simd(RB, TERMS, C32)) void tp_adapter_few_kernel(const DownArgs d, const UpArgs p) {
    constexpr int GP = 2 * RB;
    using Sh = FewShape<RB>;
    using Strip = UpStrip<GP, TERMS, false, C32>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int l = threadIdx.x & 63, c = l & 15, g = l >> 4, w = uni(threadIdx.x >> 6);
    preload(p);
    preload(d);
    Tile t;
    if (!find_tile(p.seg, blockIdx.x, 16, t)) return;
    const bool adapted = t.id >= 0;
    const int strips = (p.cols + 127) / 128, step = gridDim.y * Sh::WAVES;
    int strip = blockIdx.y * Sh::WAVES + w;
    constexpr int EARLY = RB == 2 ? 2 : 1;                               // strips whose factor and C come in early
    u32x4_t f[EARLY][UpShape<GP, TERMS>::NS][8], bias[EARLY];
    CRows<C32> cv[EARLY];
    char* const low = lds + Sh::SUMS;
#pragma unroll
    for (int s = 0; s < EARLY; ++s)
        if (strip + s * step < strips) {
            const Strip st(p, t, strip + s * step);
            if (adapted) st.load_factor(f[s]);
            st.load_c(cv[s], 0);
            bias[s] = st.load_bias();
        }
    if (adapted) {
        const float scale = p.scale ? p.scale[t.id] : 1.0f;
        f32x4_t acc[1][RB];
        const uint32_t ring = (uint32_t)(w * Sh::NS * Sh::SLOT);
        if (t.rows <= 8) down_sums<1, RB, Sh::NS, false, 1>(d, t, w, Sh::WAVES, ring, acc);
        else             down_sums<1, RB, Sh::NS, false, 2>(d, t, w, Sh::WAVES, ring, acc);
        __syncthreads();
        float* const part = reinterpret_cast<float*>(lds);
#pragma unroll
        for (int j = 0; j < RB; ++j) *reinterpret_cast<f32x4_t*>(part + (w * 16 + c) * Sh::PART + 16 * j + 4 * g) = acc[0][j];
        __syncthreads();
        for (int i = threadIdx.x; i < t.rows * GP; i += 64 * Sh::WAVES) {
            const int r = i / GP, q = i % GP;
            f32x4_t a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
            if (8 * q < p.rank) {                                // (sums of zeros beyond it, but NaN where X is not finite)
                a = waves_sum<Sh::PART, Sh::WAVES>(part, r, 2 * q);
                b = waves_sum<Sh::PART, Sh::WAVES>(part, r, 2 * q + 1);
                if (p.v_out && blockIdx.y == 0) {
                    f32x4_t* const to = reinterpret_cast<f32x4_t*>(p.v_out + (int64_t)(t.row0 + r) * p.rank + 8 * q);
                    to[0] = a;
                    to[1] = b;
                }
            }
            const float v[8] = {a[0] * scale, a[1] * scale, a[2] * scale, a[3] * scale, b[0] * scale, b[1] * scale, b[2] * scale, b[3] * scale};
            lay_terms<GP, TERMS>(low, r, q, v);
        }
        __syncthreads();
    }
    Mask none{};
#pragma unroll
    for (int s = 0; s < EARLY; ++s, strip += step) {
        if (strip >= strips) return;
        const Strip st(p, t, strip);
        if (adapted) st.turn(f[s]);
        st.rows16(low, f[s], cv[s], bias[s], none, 0, adapted);
    }
    for (; strip < strips; strip += step) {
        const Strip st(p, t, strip);
        if (adapted) st.load_factor(f[0]);
        st.load_c(cv[0], 0);
        if (adapted) st.turn(f[0]);
        st.rows16(low, f[0], cv[0], st.load_bias(), none, 0, adapted);
    }
}

// ---------------------------------------------------------------------------------------------
// grad.  A workgroup has a strip of 128 columns, 16 or 32 ranks and a share of an adapter's rows, counted in units of 32 rows of one segment; its four
// waves take the units in turn and their sums meet in LDS in order.  The factor's layout again leaves a lane with eight neighbouring columns.  With several
// shares their sums go to planes that are added in order later: nothing depends on which workgroup runs first.
// (32 ranks: two workgroups fit a CU.  All of a backward pass of 16384 x 4096 x 4096, 64 ranks 211 us, with 64 ranks a workgroup 228, with 16 237; 128 ranks
// 268 / 294 / 327; 731 rows of 1504 and 2496 columns, 64 ranks 25.1 / 28.5 / 23.7.)
// ---------------------------------------------------------------------------------------------
constexpr int GRAD_WAVES = 4;
template <int RB>
__global__ __launch_bounds__(64 * GRAD_WAVES) void tp_adapter_grad_kernel(const GradArgs p, const int strips0, const int strips) {
    __shared__ __attribute__((aligned(16))) float part[GRAD_WAVES][16][132];
    const int l = threadIdx.x & 63, c = l & 15, g = l >> 4, w = uni(threadIdx.x >> 6);
    const int chunks = (p.rank + 16 * RB - 1) / (16 * RB);
    // (the shares side by side: an XCD then has its own shares of the rows, and a CU strips of both pairs, of which one may draw a mask: 16384 rows of
    // 4096 and 4096 columns with dropout 52.2 us, 56.6 with the strips side by side)
    int x = blockIdx.x;
    const int share = x % p.shares; x /= p.shares;
    const int strip_all = x % strips; x /= strips;
    const int rank0 = (x % chunks) * 16 * RB, a = x / chunks;
    const int which = strip_all >= strips0, strip = which ? strip_all - strips0 : strip_all;
    const GradSide& q = p.side[which];
    const int n = strip * 128 + 8 * c;
    const bool in = n < q.cols;
    // units of this adapter, those of this share
    int total = 0;
    for (int first = 0; first < p.seg.n; first += 64) {
        int lo, len, id;
        segment(p.seg, first + l, lo, len, id);
        const int count = id == a ? (len + 31) / 32 : 0;
        total += __builtin_amdgcn_readlane(wave_sums(count), 63);
    }
    if (p.shares > 1 && share == 0 && strip_all == 0 && rank0 == 0 && threadIdx.x == 0) p.units[a] = total;
    const int u0 = (int)((int64_t)total * share / p.shares), u1 = (int)((int64_t)total * (share + 1) / p.shares);
    if (p.shares > 1 && u0 >= u1) return;
    Mask m;
    if (q.dropped) m = open_mask(p.drop);
    f32x4_t acc[RB][8];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // rows [row, row + have), have <= 32: lane's rows 8 g + j
    auto unit = [&](int row, int have) __attribute__((always_inline)) {
        const __amdgpu_buffer_rsrc_t rr = make_rsrc(static_cast<const uint16_t*>(q.r) + (int64_t)row * q.ldr, ((int64_t)(have - 1) * q.ldr + q.cols) * 2);
        u32x4_t rows[8], r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) rows[j] = buf_load16(rr, in ? (uint32_t)(((8 * g + j) * q.ldr + n) * 2) : OOB_OFFSET);
        uint32_t first[RB][8];
        auto plane = [&](int z, int i, int j) __attribute__((always_inline)) {
            const __amdgpu_buffer_rsrc_t rl = make_rsrc(q.l + z * q.plane + (int64_t)row * p.rank, z < q.splits ? (int64_t)have * p.rank * 4 : 0);
            const int k = rank0 + 16 * i + c;
            return __builtin_amdgcn_raw_buffer_load_b32(rl, k < p.rank ? ((8 * g + j) * p.rank + k) * 4 : (int)OOB_OFFSET, 0, 0);
        };
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) first[i][j] = plane(0, i, j);
        if (q.dropped) {                                         // (the draws need nothing that is under way)
            u32x4_t bits[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) bits[j] = draw(m, p.drop.group0 + (uint32_t)(n >> 3), p.drop.row0 + (uint32_t)(row + 8 * g + j));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 8; ++j) rows[j] = clear_dropped(m, bits[j], rows[j]);
        }
        float v[RB][8];
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = as_float(first[i][j]);
        constexpr int MORE = RB == 1 ? 4 : 2;                    // planes on their way at a time
        for (int z0 = 1; z0 < q.splits; z0 += MORE) {
            uint32_t next[MORE][RB][8];
#pragma unroll
            for (int z = 0; z < MORE; ++z)
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) next[z][i][j] = plane(z0 + z, i, j);
#pragma unroll
            for (int z = 0; z < MORE; ++z)
#pragma unroll
                for (int i = 0; i < RB; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] += as_float(next[z][i][j]);
        }
        transpose8(rows, r);
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            u32x4_t term[3];
            split_terms(v[i], term);
#pragma unroll
            for (int s = 0; s < 3; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = mfma(term[s], r[j], acc[i][j]);      // rank 16 i + 4 g + e, column 8 c + j
        }
    };
    int base = 0;
    for (int first = 0; first < p.seg.n && base < u1; first += 64) {
        int lo, len, id;
        segment(p.seg, first + l, lo, len, id);
        const int count = id == a ? (len + 31) / 32 : 0, sums = wave_sums(count);
        for (uint64_t some = __ballot(count > 0); some; some &= some - 1) {
            const int j = __builtin_ctzll(some);
            const int units = __builtin_amdgcn_readlane(count, j), before = base + __builtin_amdgcn_readlane(sums, j) - units;
            const int at = __builtin_amdgcn_readlane(lo, j), rows = __builtin_amdgcn_readlane(len, j);
            int u = before > u0 ? before : u0;
            u += (w - u) & (GRAD_WAVES - 1);                             // this wave's first one
            const int end = before + units < u1 ? before + units : u1;
            for (; u < end; u += GRAD_WAVES) {
                const int r = 32 * (u - before);
                unit(at + r, rows - r < 32 ? rows - r : 32);
            }
        }
        base += __builtin_amdgcn_readlane(sums, 63);
    }
    // (without rows 0, whatever the scale: that of a place in the pool which is not taken may be anything)
    const float scale = total ? (p.scale ? p.scale[a] : 1.0f) * (q.dropped ? p.drop.factor : 1.0f) : 0.0f;
#pragma unroll
    for (int i = 0; i < RB; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            *reinterpret_cast<f32x4_t*>(&part[w][4 * g + e][8 * c]) = f32x4_t{acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
            *reinterpret_cast<f32x4_t*>(&part[w][4 * g + e][8 * c + 4]) = f32x4_t{acc[i][4][e], acc[i][5][e], acc[i][6][e], acc[i][7][e]};
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = threadIdx.x + 256 * h, row = at >> 5, col = (at & 31) * 4;
            const int k = rank0 + 16 * i + row, cc = strip * 128 + col;
            if (k >= p.rank || cc >= q.cols) continue;
            f32x4_t s = *reinterpret_cast<const f32x4_t*>(&part[0][row][col]);
#pragma unroll
            for (int v = 1; v < GRAD_WAVES; ++v) s += *reinterpret_cast<const f32x4_t*>(&part[v][row][col]);
            s *= scale;
            if (p.shares > 1) {
                *reinterpret_cast<f32x4_t*>(q.part + (((int64_t)a * p.shares + share) * p.rank + k) * q.cols + cc) = s;
            } else {
                f32x4_t* const to = reinterpret_cast<f32x4_t*>(q.out + a * q.stride + k * q.ldo + cc);
                if (p.accumulate) s = *to + s;
                *to = s;
            }
        }
    }
}
__global__ __launch_bounds__(64) void tp_adapter_grad_finish_kernel(const GradArgs p) { finish_share(p, blockIdx.x); }

// Kernels with more LDS than a launch has by default: said once on every device (the same value every time)
template <class K>
hipError_t allow_lds(K kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
    if (hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes); e != hipSuccess) return e;
    done.fetch_or(bit, std::memory_order_relaxed);
    return hipSuccess;
}
template <int MT, int RB, bool DROP>
hipError_t down_as(const DownArgs& a, hipStream_t s) {
    using Sh = DownShape<MT, RB, DROP>;
    static std::atomic<uint64_t> done{0};
    if (hipError_t e = allow_lds(tp_adapter_down_kernel<MT, RB, DROP>, Sh::BYTES, done); e != hipSuccess) return e;
    return launch_kernel(tp_adapter_down_kernel<MT, RB, DROP>, dim3((unsigned)a.tiles, (unsigned)a.splits), dim3(64 * Sh::WAVES), Sh::BYTES, s, a);
}
template <int MT, int RB>
hipError_t down(const DownArgs& a, hipStream_t s) { return a.dropped ? down_as<MT, RB, true>(a, s) : down_as<MT, RB, false>(a, s); }
template <int MT>
hipError_t down_rank(const DownArgs& a, hipStream_t s) {
    if (a.rank <= 16) return down<MT, 1>(a, s);
    if (a.rank <= 32) return down<MT, 2>(a, s);
    if (a.rank <= 64) return down<MT, 4>(a, s);
    return down<MT, 8>(a, s);
}

template <int GP, int TERMS>
hipError_t up_as(const UpArgs& a, const GradArgs* fin, hipStream_t s) {
    const int strips = (a.cols + 127) / 128, strip_waves = up_waves(strips, a.tiles), y = (strips + strip_waves - 1) / strip_waves;
    // (a workgroup of one strip has as many waves as V's terms keep busy, up to four: all of a call, forward of 553 rows of 3968 to 432 columns, 64 ranks 17.8 us, 21.4
    // with one wave, 128 ranks 23.5 / 31.0; backward of 731 rows of 1504 and 2496 columns, 64 ranks 28.5 / 32.4,
    // 128 ranks 40.6 / 45.0, and 44.9 with up to six)
    const int waves = strip_waves > 1 ? strip_waves : a.tile * GP >= 256 ? 4 : (a.tile * GP + 63) / 64;
    UpArgs args = a;
    args.waves = strip_waves;
    // (planes to add: of the whole pool, shares and pool 256 together at most or as many as make two workgroups of *grad* a CU; the places of adapters without rows
    // add zeros.  128 workgroups for one adapter of 16384 x 4096 x 4096, 16 ranks; 131072 for a pool of 128 of 128 ranks)
    const int64_t more = fin ? ((int64_t)finish_blocks_each(*fin, 64 * waves) * fin->seg.pool * fin->sides + y - 1) / y : 0;
    const dim3 grid((unsigned)(a.tiles + more), (unsigned)y), block(64 * waves);
    const size_t lds = (size_t)a.tile * UpShape<GP, TERMS>::ROW;
    return launch_kernel(a.c_f32 ? (a.dropped ? tp_adapter_up_kernel<GP, TERMS, true, true> : tp_adapter_up_kernel<GP, TERMS, false, true>)
                                 : (a.dropped ? tp_adapter_up_kernel<GP, TERMS, true, false> : tp_adapter_up_kernel<GP, TERMS, false, false>), grid, block, lds, s, args,
                         fin ? *fin : GradArgs{});
}
template <int GP>
hipError_t up(const UpArgs& a, const GradArgs* fin, hipStream_t s) { return a.out_f32 ? up_as<GP, 3>(a, fin, s) : up_as<GP, 2>(a, fin, s); }

}  // namespace

hipError_t launch_down(const DownArgs& a, hipStream_t s) {
    if (a.tiles < 1) return hipSuccess;
    switch (a.tile) {
        case 16: return down_rank<1>(a, s);
        case 32: return down_rank<2>(a, s);
        case 64: return down_rank<4>(a, s);
        default: return hipErrorInvalidValue;
    }
}

template <int RB, int TERMS, bool C32>
static hipError_t few(const DownArgs& d, const UpArgs& u, hipStream_t s) {
    using Sh = FewShape<RB>;
    static std::atomic<uint64_t> done{0};
    if (hipError_t e = allow_lds(tp_adapter_few_kernel<RB, TERMS, C32>, Sh::BYTES, done); e != hipSuccess) return e;
    // workgroups of a tile: while there are CUs for them, as many as leave a wave one strip
    const int strips = (u.cols + 127) / 128, most = (strips + Sh::WAVES - 1) / Sh::WAVES, room = u.tiles < 256 ? 256 / u.tiles : 1;
    return launch_kernel(tp_adapter_few_kernel<RB, TERMS, C32>, dim3((unsigned)u.tiles, (unsigned)(most < room ? most : room)), dim3(64 * Sh::WAVES), Sh::BYTES, s,
                         d, u);
}
hipError_t launch_few(const DownArgs& d, const UpArgs& u, hipStream_t s) {
    if (d.dropped || u.dropped || u.tile != 16) return hipErrorInvalidValue;
    auto pick = [&](auto rb) {
        constexpr int RB = decltype(rb)::value;
        if (u.out_f32) return u.c_f32 ? few<RB, 3, true>(d, u, s) : few<RB, 3, false>(d, u, s);
        return u.c_f32 ? few<RB, 2, true>(d, u, s) : few<RB, 2, false>(d, u, s);
    };
    return u.rank <= 16 ? pick(std::integral_constant<int, 1>{}) : u.rank <= 32 ? pick(std::integral_constant<int, 2>{})
         : u.rank <= 64 ? pick(std::integral_constant<int, 4>{}) : pick(std::integral_constant<int, 8>{});
}

hipError_t launch_up(const UpArgs& a, const GradArgs* fin, hipStream_t s) {
    return a.rank <= 16 ? up<2>(a, fin, s) : a.rank <= 32 ? up<4>(a, fin, s) : a.rank <= 64 ? up<8>(a, fin, s) : up<16>(a, fin, s);
}

hipError_t launch_grad(const GradArgs& a, bool finish, hipStream_t s) {
    const int strips0 = (a.side[0].cols + 127) / 128, strips = strips0 + (a.sides > 1 ? (a.side[1].cols + 127) / 128 : 0);
    const int rb = a.rank <= 16 ? 1 : 2, chunks = (a.rank + 16 * rb - 1) / (16 * rb);
    const int64_t blocks = (int64_t)strips * chunks * a.shares * a.seg.pool;      // (the caller has looked at how many)
    if (hipError_t e = launch_kernel(rb == 1 ? tp_adapter_grad_kernel<1> : tp_adapter_grad_kernel<2>,
                                     dim3((unsigned)blocks), dim3(64 * GRAD_WAVES), 0, s, a, strips0, strips); e != hipSuccess || a.shares == 1 || !finish)
        return e;
    return launch_kernel(tp_adapter_grad_finish_kernel, dim3((unsigned)((int64_t)finish_blocks_each(a, 64) * a.seg.pool * a.sides)), dim3(64), 0, s, a);
}

}  // namespace tpl
