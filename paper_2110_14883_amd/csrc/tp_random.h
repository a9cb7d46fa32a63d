// The generator behind dropout, on the device: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011), a keyed bijection of a 128-bit counter.  The mask of a matrix is never stored: the eight columns 8 g .. 8 g + 7 of row R (numbers in
// the full matrix) share the draw of counter (g, R, offset) under key `seed`, 16 bits a column in ascending order, and a column is kept
// where its bits are at least `threshold`.  Every kernel here holds eight neighbouring columns of a row in one lane, so a lane draws
// for itself, and a block of the matrix draws what the whole matrix would.
// Ten rounds of two 32 x 32 -> 64 bit products: about 55 vector instructions a draw, 20 of them at a quarter of the rate.  (32 bits a column would
// take two draws; 16 put p on a grid of 1/65536 and leave it exact there, since the factor is 65536 / (65536 - threshold).)
#pragma once
#include "tp_device.h"

namespace tpl {

// What a kernel needs of it beside the position; the offset on the device is added when the kernel runs.
struct Mask {
    uint32_t key0, key1, off_lo, off_hi;
    uint32_t threshold;           // 0 .. 65536
};
__device__ __forceinline__ Mask open_mask(const DropArgs& d) {
    uint64_t off = d.offset;
    if (d.offset_dev) off += *d.offset_dev;
    return Mask{d.key0, d.key1, (uint32_t)off, (uint32_t)(off >> 32), d.threshold};
}
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
// the 128 bits of column group `group` of row `row`
__device__ __forceinline__ u32x4_t draw(const Mask& m, uint32_t group, uint32_t row) {
    uint32_t x0 = group, x1 = row, x2 = m.off_lo, x3 = m.off_hi, k0 = m.key0, k1 = m.key1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
        x0 = xor3((uint32_t)(b >> 32), x1, k0);
        x1 = (uint32_t)b;
        x2 = xor3((uint32_t)(a >> 32), x3, k1);
        x3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4_t{x0, x1, x2, x3};
}
// The same for a lane that holds four neighbouring columns in two places, lanes 2 j and 2 j + 1 the halves of one group in each: the even lane draws for
// the first place, the odd one for the second, and they hand each other the half that is its neighbour's.  Words 0, 1 are the bits of the
// first place's columns, 2, 3 of the second's.
__device__ __forceinline__ u32x4_t draw_shared(const Mask& m, uint32_t group0, uint32_t row0, uint32_t group1, uint32_t row1) {
    const bool odd = threadIdx.x & 1;
    const u32x4_t w = draw(m, odd ? group1 : group0, odd ? row1 : row0);
    const int a = odd ? w[0] : w[2], b = odd ? w[1] : w[3];
    const uint32_t x = (uint32_t)__builtin_amdgcn_mov_dpp(a, 0xB1, 0xF, 0xF, true), y = (uint32_t)__builtin_amdgcn_mov_dpp(b, 0xB1, 0xF, 0xF, true);   // lanes 1 0 3 2
    return u32x4_t{odd ? x : w[0], odd ? y : w[1], odd ? w[2] : x, odd ? w[3] : y};
}
__device__ __forceinline__ bool keeps(const Mask& m, const u32x4_t& bits, int e) {
    const uint32_t w = bits[e >> 1];
    return (e & 1 ? w >> 16 : w & 0xFFFFu) >= m.threshold;
}
// eight bf16 values with the dropped ones cleared (whatever they were; the factor is the caller's)
__device__ __forceinline__ u32x4_t clear_dropped(const Mask& m, const u32x4_t& bits, const u32x4_t& v) {
    u32x4_t o;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o[i] = v[i] & ((keeps(m, bits, 2 * i) ? 0xFFFFu : 0u) | (keeps(m, bits, 2 * i + 1) ? 0xFFFF0000u : 0u));
    return o;
}

}  // namespace tpl
