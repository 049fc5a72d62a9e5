// fs_seq_pack8 / fs_seq_unpack8: rows of activations as 8-bit checkpoints (format: pack8.h) and back.
//
// HBM-bound, one pass: a 16-byte piece of a row to a lane, the block of 32 columns to 4 (16-bit types) or 8 (fp32) lanes,
// which find its largest magnitude by two or three DPP steps.  Measured (us, TB/s of the bytes): 4.2 M rows of 128 fp16 packed in
// 305 (5.4), unpacked in 287 (5.7); 2 M rows of 128 fp32 213 (6.0) and 175 (7.4, part of it out of the Infinity Cache).
#include "pack8.h"
#include "seq_rows.h"

namespace fs {

// Lane j of a block of columns: which row, which block, which piece of the row.
template <int LPB>
struct PackPlace {
    int64_t row;
    int block;
    int piece;
    bool in;
};

// Units of (row, block of columns) in order, LPB lanes each.  One 64-bit division a workgroup, the rest of the place in 32 bits.
template <int LPB>
__device__ __forceinline__ PackPlace<LPB> pack_place(int64_t n, int nb, int units)
{
    constexpr int kPer = kBlock / LPB;
    const int64_t first = (int64_t)blockIdx.x * kPer;
    const int64_t row0 = first / nb;
    const uint32_t at = (uint32_t)(first - row0 * nb) + threadIdx.x / LPB;
    PackPlace<LPB> p;
    p.row = row0 + at / (uint32_t)nb;
    p.block = (int)(at % (uint32_t)nb);
    p.piece = p.block * LPB + (int)(threadIdx.x % LPB);
    p.in = p.row < n && p.piece < units;
    return p;
}

template <int DT>
__global__ __launch_bounds__(kBlock) void pack8_kernel(const u32x4* __restrict__ x, int64_t n, int units, int nb,
                                                       uint32_t* __restrict__ codes, uint8_t* __restrict__ exps)
{
    constexpr int N = Piece<DT>::N, LPB = kPackBlock / N;
    const PackPlace<LPB> p = pack_place<LPB>(n, nb, units);
    float v[N];
    uint32_t top = 0;
    u32x4 raw = {0u, 0u, 0u, 0u};
    if (p.in) raw = load_stream(x + p.row * units + p.piece);
    Piece<DT>::unpack(raw, v);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        top = top > b ? top : b;
    }
    const int E = pack_exponent(group_top<LPB>(top));
    if (!p.in) return;
    uint32_t* to = codes + (p.row * units + p.piece) * (N / 4);
    if constexpr (N == 8) {
        const u32x2 c = {pack_four(v, E), pack_four(v + 4, E)};
        __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(to));
    } else {
        *to = pack_four(v, E);                          // (4 bytes a lane: streamed 229 us, 2 M rows of 128, through the caches 213)
    }
    if (threadIdx.x % LPB == 0) exps[p.row * nb + p.block] = (uint8_t)E;
}

template <int DT>
__global__ __launch_bounds__(kBlock) void unpack8_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ exps,
                                                         int64_t n, int units, int nb, u32x4* __restrict__ x)
{
    constexpr int N = Piece<DT>::N, LPB = kPackBlock / N;
    const PackPlace<LPB> p = pack_place<LPB>(n, nb, units);
    if (!p.in) return;
    const int E = exps[p.row * nb + p.block];
    const uint32_t* from = codes + (p.row * units + p.piece) * (N / 4);
    float v[N];
    unpack_piece<N>(from[0], N == 8 ? from[N / 8] : 0u, E, v);
    if constexpr (DT == FS_F16) {
        // 2^16 is a value of blocks with fp16's largest numbers in them; what was finite stays finite
        if (E != kPackLost) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = __builtin_amdgcn_fmed3f(v[i], -65504.0f, 65504.0f);
        }
    }
    store_stream(x + p.row * units + p.piece, Piece<DT>::pack(v));
}

namespace {
// Rows of one launch, and the grid for `rows` of them: (row, block of columns) by LPB lanes.
int64_t pack_launch_rows(int nb, int lpb) { return kMostGrid * (kBlock / lpb) / nb; }

dim3 pack_grid(int64_t rows, int nb, int lpb)
{
    const int64_t per = kBlock / lpb;
    return dim3((unsigned)((rows * nb + per - 1) / per));
}
}  // namespace

}  // namespace fs

extern "C" fs_status fs_seq_pack8(const void* x, int64_t n, int32_t D, fs_dtype dtype, int8_t* codes, uint8_t* exps, void* stream)
{
    using namespace fs;
    int units = 0;
    const fs_status st = check_seq_rows(n, D, dtype, &units);
    if (st != FS_OK) return st;
    if (n == 0) return FS_OK;
    if (!x || !codes || !exps) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(codes, codes_alignment(dtype))) return FS_ERR_ALIGN;
    const int nb = (int)pack_blocks(D);
    const int lpb = dtype == FS_F32 ? 8 : 4;
    const int64_t most = pack_launch_rows(nb, lpb);
    for (int64_t r0 = 0; r0 < n; r0 += most) {
        const int64_t rows = n - r0 < most ? n - r0 : most;
#define CALL(DT) FS_LAUNCH("pack8", pack8_kernel<DT>, pack_grid(rows, nb, lpb), dim3(kBlock), static_cast<hipStream_t>(stream),      \
                           static_cast<const u32x4*>(x) + r0 * units, rows, units, nb, reinterpret_cast<uint32_t*>(codes + r0 * D), exps + r0 * nb)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    }
    return FS_OK;
}

extern "C" fs_status fs_seq_unpack8(const int8_t* codes, const uint8_t* exps, int64_t n, int32_t D, fs_dtype dtype, void* x, void* stream)
{
    using namespace fs;
    int units = 0;
    const fs_status st = check_seq_rows(n, D, dtype, &units);
    if (st != FS_OK) return st;
    if (n == 0) return FS_OK;
    if (!x || !codes || !exps) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(codes, codes_alignment(dtype))) return FS_ERR_ALIGN;
    const int nb = (int)pack_blocks(D);
    const int lpb = dtype == FS_F32 ? 8 : 4;
    const int64_t most = pack_launch_rows(nb, lpb);
    for (int64_t r0 = 0; r0 < n; r0 += most) {
        const int64_t rows = n - r0 < most ? n - r0 : most;
#define CALL(DT) FS_LAUNCH("unpack8", unpack8_kernel<DT>, pack_grid(rows, nb, lpb), dim3(kBlock), static_cast<hipStream_t>(stream),  \
                           reinterpret_cast<const uint32_t*>(codes + r0 * D), exps + r0 * nb, rows, units, nb, static_cast<u32x4*>(x) + r0 * units)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    }
    return FS_OK;
}
