// What the operators on the rows of a sequence share (norm, scan, pack8): 16-byte pieces of a row as fp32 and back, sums
// over the lanes of a row, the host's checks.
#pragma once

#include "fs_common.h"
#include "update_rules.h"

namespace fs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Elems with the rounding of pairs to bf16 in one instruction (nearest even, a NaN stays one) in place of five a value.
template <int DT>
struct Piece : Elems<DT> {
    static __device__ __forceinline__ u32x4 pack(const float* f)
    {
        if constexpr (DT == FS_BF16) {
            u32x4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[2 * i], f[2 * i + 1]}, bf16x2));
            return x;
        } else if constexpr (DT == FS_F16) {
            // The fp32 value is settled before it is rounded: folded into the operation before it, the rounding is of the unrounded
            // result, in some instances of a kernel and not in others.
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = f[i];
                asm("" : "+v"(v[i]));
            }
            return Elems<DT>::pack(v);
        } else {
            return Elems<DT>::pack(f);
        }
    }
};

// Sum over the aligned group of G lanes (4 .. 64) that the lane is in, in every lane of it, the same bits in each (every
// step adds the same two numbers).  All lanes of the wave call it.
template <int G>
__device__ __forceinline__ float group_sum(float v)
{
#define FS_DPP_ADD(ctrl) v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, 0xf, 0xf, true))
    if constexpr (G >= 2) FS_DPP_ADD(0xB1);       // lane ^ 1
    if constexpr (G >= 4) FS_DPP_ADD(0x4E);       // lane ^ 2
    if constexpr (G >= 8) FS_DPP_ADD(0x141);      // mirrored in 8: the other four
    if constexpr (G >= 16) FS_DPP_ADD(0x140);     // mirrored in 16: the other eight
    if constexpr (G >= 32) v += __shfl_xor(v, 16);
    if constexpr (G >= 64) v += __shfl_xor(v, 32);
#undef FS_DPP_ADD
    return v;
}

// A launch has fewer than 2^32 threads: the most workgroups of kBlock.  Longer batches go in several launches of whole rows.
constexpr int64_t kMostGrid = (1LL << 32) / kBlock - 1;

// Longest row of the norm and the recurrence, in 16-byte pieces (4 MB): the norm's launches over the columns stay under
// kMostGrid and its sums in fp32 of a use, the recurrence's tiles within 32-bit offsets.
constexpr int kMostPieces = (1 << 18) - 1;

inline bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// Sizes and type of n rows of D elements; *units = 16-byte pieces of a row.
inline fs_status check_seq_rows(int64_t n, int32_t D, fs_dtype dtype, int* units)
{
    const int es = dtype_bytes(dtype);
    if (es == 0) return FS_ERR_DTYPE;
    if (n < 0 || n >= (1LL << 31) || D < 1) return FS_ERR_SIZE;
    const int64_t row_bytes = (int64_t)D * es;
    if (row_bytes % 16 != 0) return FS_ERR_ALIGN;
    *units = (int)(row_bytes / 16);
    return FS_OK;
}

#define FS_DISPATCH_DTYPE(dtype, CALL)                                                  \
    switch (dtype) {                                                                    \
        case FS_F32: CALL(FS_F32); break;                                               \
        case FS_F16: CALL(FS_F16); break;                                               \
        default: CALL(FS_BF16); break;                                                  \
    }

}  // namespace fs
