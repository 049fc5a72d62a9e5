// The 8-bit checkpoint format: blocks of 32 consecutive columns of a row (the last one of a row may be shorter), each with
// one exponent byte E and a signed byte a value.  A block's step is the smallest power of two 2^(E - 133) with which its
// largest magnitude rounds to at most 127; a value is its nearest whole multiple of the step, ties to even.  So a code is
// off by at most half a step, and a step is at most 1/64 of the block's largest magnitude, at least 1/127.5 of it.  A power
// of two keeps both directions exact in fp32 (no division, no rounding of a scale), and the codes a function of the values
// alone.  E = 255: the block holds an infinity or a NaN; it keeps those (code -128: NaN, +-127: the infinities), its finite
// values are lost (code 0).
#pragma once

#include "fs_common.h"

namespace fs {

constexpr int kPackBlock = 32;
constexpr int kPackLost = 255;                    // E of a block with an infinity or a NaN

// Codes are read and written by the 16-byte piece of the rows that they stand for: 4 or 8 at a time.
inline int codes_alignment(fs_dtype dtype) { return dtype == FS_F32 ? 4 : 8; }

inline int64_t pack_blocks(int64_t D) { return (D + kPackBlock - 1) / kPackBlock; }

// E of a block whose largest magnitude has these bits (a NaN counts as larger than all).  Adding 2^16 carries into the
// exponent from a significand of 255/128 on: magnitudes of 127.5 steps would round to 128.
__host__ __device__ inline int pack_exponent(uint32_t top_bits)
{
    if (top_bits >= 0x7F800000u) return kPackLost;
    const int E = (int)((top_bits + 0x10000u) >> 23);
    return E < 1 ? 1 : E > 254 ? 254 : E;         // 1: subnormal blocks too; 254: the largest floats, whose codes stop at 127
}

// 2^(E - 133) as a float: subnormal below E = 7.  E = 0 is never written and read as 1.
__host__ __device__ inline uint32_t pack_step_bits(int E)
{
    return E >= 7 ? (uint32_t)(E - 6) << 23 : 1u << (16 + (E < 1 ? 1 : E));
}

#ifdef __HIPCC__
__device__ __forceinline__ int pack_code(float v, int E)
{
    const float q = __builtin_amdgcn_fmed3f(rintf(__builtin_amdgcn_ldexpf(v, 133 - E)), -127.0f, 127.0f);
    return (int)q;
}

__device__ __forceinline__ int pack_code_lost(float v)
{
    return v != v ? -128 : __builtin_isinf(v) ? (v > 0.0f ? 127 : -127) : 0;
}

__device__ __forceinline__ uint32_t pack_four(const float* v, int E)
{
    int c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = pack_code(v[i], E);
    if (ballot(E == kPackLost) != 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = E == kPackLost ? pack_code_lost(v[i]) : c[i];
    }
    return (uint32_t)(c[0] & 255) | (uint32_t)(c[1] & 255) << 8 | (uint32_t)(c[2] & 255) << 16 | (uint32_t)c[3] << 24;
}

// Four values from their codes: in a block of finite values, in one that keeps its infinities and NaN alone.
__device__ __forceinline__ void unpack_four(uint32_t codes, float step, float* v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)((int32_t)(codes << (24 - 8 * i)) >> 24) * step;
}

__device__ __forceinline__ void unpack_four_lost(uint32_t codes, float* v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = (int32_t)(codes << (24 - 8 * i)) >> 24;
        v[i] = __uint_as_float(c == -128 ? 0x7FC00000u : c == 0 ? 0u : c > 0 ? 0x7F800000u : 0xFF800000u);
    }
}

// The N values (4 or 8) of a piece from its codes.  A block with an infinity or a NaN is a branch of the wave: as a selection
// a value it costs more than all the rest.
template <int N>
__device__ __forceinline__ void unpack_piece(uint32_t codes0, uint32_t codes1, int E, float* v)
{
    const float step = __uint_as_float(pack_step_bits(E));
    unpack_four(codes0, step, v);
    if constexpr (N == 8) unpack_four(codes1, step, v + 4);
    if (ballot(E == kPackLost) != 0) {
        if (E == kPackLost) {
            unpack_four_lost(codes0, v);
            if constexpr (N == 8) unpack_four_lost(codes1, v + 4);
        }
    }
}

// Largest magnitude, as bits, over the aligned group of LANES lanes (a power of two up to 8) that this lane is in; every
// lane of the group calls it.  Bits of magnitudes order as integers do, and a NaN's are above all others.
template <int LANES>
__device__ __forceinline__ uint32_t group_top(uint32_t m)
{
    auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    if constexpr (LANES >= 2) m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1 /* lane ^ 1 */, 0xf, 0xf, true));
    if constexpr (LANES >= 4) m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E /* lane ^ 2 */, 0xf, 0xf, true));
    if constexpr (LANES >= 8) m = larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141 /* lanes mirrored in 8 */, 0xf, 0xf, true));
    return m;
}
#endif  // __HIPCC__

}  // namespace fs
