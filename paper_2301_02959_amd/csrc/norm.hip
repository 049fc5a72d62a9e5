// fs_seq_norm_fwd, fs_seq_norm_bwd, fs_seq_norm_bwd_packed: layer norm of the rows of a sequence and its gradients.
//
//   forward   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), y = (x - m) r gamma + beta
//   backward  u = (x - m) r, g = dy gamma:  dx = r (g - mean(g) - u mean(g u)), dgamma = sum over rows of dy u, dbeta = of dy
//
// HBM-bound: x read once and y written once; dy and x (or its checkpoint) read once and dx written once.  A row of up to
// 1024 pieces of 16 bytes lies in the registers of G lanes, P pieces a lane, so mean and squares are two passes over
// registers; longer rows are read three times by a workgroup each (kernels *_wide).  All sums are fp32.  The variance is taken
// about the rounded mean and corrected by what that mean is off (s1 below), so a row of equal values far from zero
// normalises to zeros.
// dgamma and dbeta: every lane keeps its columns' sums over the rows that its group walks, a workgroup adds its groups in
// LDS and writes one partial row, norm_grad_sum adds the partial rows in their order: no atomics, the same bits every run.
//
// Measured, 3.93 M rows of 256 bf16 (us, TB/s of what has to be read and written): forward 691 (5.8), with the checkpoint
// written too 884 (5.7), backward 1078 (5.6), from the checkpoint 890 (5.7).
#include "pack8.h"
#include "seq_rows.h"

namespace fs {

struct NormArgs {
    const u32x4* x;
    const uint32_t* x_codes;         // packed backward: x as a checkpoint
    const uint8_t* x_exps;
    const u32x4* dy;
    int64_t n;
    int units;                       // 16-byte pieces of a row
    int nb;                          // blocks of columns of a checkpoint's row
    float inv_D;
    float eps;
    const float* gamma;
    const float* beta;
    u32x4* y;
    float* mean;                     // forward: may be null
    float* rstd;
    uint32_t* codes;                 // forward: may be null
    uint8_t* exps;
    u32x4* dx;
    float* partial;                  // [workgroups][2][D]
    float* dgamma;
    float* dbeta;
};

template <int N>
__device__ __forceinline__ void load_floats(const float* p, float* v)
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(p + i);
        v[i] = q[0]; v[i + 1] = q[1]; v[i + 2] = q[2]; v[i + 3] = q[3];
    }
}

// Writes a piece's codes; all lanes of the block of columns call it (in = false: a lane past the row's end).
template <int DT, int G>
__device__ __forceinline__ void write_codes(const NormArgs& a, int64_t row, int piece, bool in, const float* v)
{
    constexpr int N = Piece<DT>::N, LPB = kPackBlock / N, L = LPB < G ? LPB : G;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t b = in ? __float_as_uint(v[i]) & 0x7FFFFFFFu : 0u;
        top = top > b ? top : b;
    }
    const int E = pack_exponent(group_top<L>(top));
    if (!in) return;
    uint32_t* to = a.codes + (row * a.units + piece) * (N / 4);
    if constexpr (N == 8) {
        const u32x2 c = {pack_four(v, E), pack_four(v + 4, E)};
        __builtin_nontemporal_store(c, reinterpret_cast<u32x2*>(to));
    } else {
        __builtin_nontemporal_store(pack_four(v, E), to);
    }
    if (piece % LPB == 0) a.exps[row * a.nb + piece / LPB] = (uint8_t)E;
}

// Sum over the workgroup, the same bits in every thread; `lds` holds kWavesPerBlock floats.
__device__ __forceinline__ float block_sum(float v, float* lds)
{
    v = group_sum<kWave>(v);
    __syncthreads();                       // lds may still be read from a previous call
    if (lane_id() == 0) lds[wave_id()] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWavesPerBlock; ++w) s += lds[w];
    return s;
}

// Sum over the G lanes of a row: a group of a wave, or the workgroup (whose threads all call it the same number of times).
template <int G>
__device__ __forceinline__ float row_sum(float v, float* lds)
{
    if constexpr (G <= kWave) return group_sum<G>(v);
    else return block_sum(v, lds);
}

// The mean with what it is off.  An infinite mean (of a row with an infinity) stays: what it is off would be a NaN.
__device__ __forceinline__ float corrected_mean(float mean, float off) { return __builtin_isinf(mean) ? mean : mean + off; }

// 1 / sqrt(v + eps); a variance that roundings have taken below zero counts as zero, one that is a NaN stays one (the larger of
// it and zero would be zero).
__device__ __forceinline__ float inverse_deviation(float var, float eps) { return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps); }

// A group of G lanes takes U rows, all their loads in flight at once.
template <int DT, int G, int P, int U, bool PACK>
__global__ __launch_bounds__(kBlock) void norm_fwd_kernel(NormArgs a)
{
    constexpr int N = Piece<DT>::N, kGroups = kBlock / G;
    __shared__ float lds[kWavesPerBlock];
    const int lig = threadIdx.x % G, group = threadIdx.x / G;
    const int64_t row0 = (int64_t)blockIdx.x * (kGroups * U) + group;
    u32x4 raw[U][P];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int64_t row = row0 + u * kGroups;
            const int piece = lig + p * G;
            raw[u][p] = u32x4{0u, 0u, 0u, 0u};
            if (row < a.n && piece < a.units) raw[u][p] = load_stream(a.x + row * a.units + piece);
        }
    float gamma[P][N], beta[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int piece = lig + p * G < a.units ? lig + p * G : 0;
        load_floats<N>(a.gamma + (int64_t)piece * N, gamma[p]);
        load_floats<N>(a.beta + (int64_t)piece * N, beta[p]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t row = row0 + u * kGroups;
        float c[P][N];
        float s = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            Piece<DT>::unpack(raw[u][p], c[p]);
            float t = 0.0f;                              // (a piece's sum of its own: shorter chains of roundings)
#pragma unroll
            for (int i = 0; i < N; ++i) t += c[p][i];
            s += t;
            if constexpr (PACK) write_codes<DT, G>(a, row, lig + p * G, row < a.n && lig + p * G < a.units, c[p]);
        }
        float mean = row_sum<G>(s, lds) * a.inv_D;
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool in = lig + p * G < a.units;
            float t1 = 0.0f, t2 = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                c[p][i] = in ? c[p][i] - mean : 0.0f;
                t1 += c[p][i];
                t2 = fmaf(c[p][i], c[p][i], t2);
            }
            s1 += t1;
            s2 += t2;
        }
        const float off = row_sum<G>(s1, lds) * a.inv_D;
        const float var = fmaf(-off, off, row_sum<G>(s2, lds) * a.inv_D);
        const float rstd = inverse_deviation(var, a.eps);
        if (row >= a.n) continue;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (lig + p * G >= a.units) continue;
            float y[N];
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = fmaf((c[p][i] - off) * rstd, gamma[p][i], beta[p][i]);
            store_stream(a.y + row * a.units + lig + p * G, Piece<DT>::pack(y));
        }
        if (lig == 0 && a.mean != nullptr) { a.mean[row] = corrected_mean(mean, off); a.rstd[row] = rstd; }
    }
}

// Rows of more than 1024 pieces, one workgroup a row; the second and third pass read what the first has brought into the L2.
template <int DT, bool PACK>
__global__ __launch_bounds__(kBlock) void norm_fwd_wide_kernel(NormArgs a)
{
    constexpr int N = Piece<DT>::N;
    __shared__ float lds[kWavesPerBlock];
    const int64_t row = blockIdx.x;
    const u32x4* x = a.x + row * a.units;
    float s = 0.0f;
    for (int p0 = 0; p0 < a.units; p0 += kBlock) {
        const int piece = p0 + (int)threadIdx.x;
        float c[N];
        u32x4 raw = {0u, 0u, 0u, 0u};
        if (piece < a.units) raw = x[piece];
        Piece<DT>::unpack(raw, c);
#pragma unroll
        for (int i = 0; i < N; ++i) s += c[i];
        if constexpr (PACK) write_codes<DT, kWave>(a, row, piece, piece < a.units, c);
    }
    float mean = block_sum(s, lds) * a.inv_D;
    float s1 = 0.0f, s2 = 0.0f;
    for (int piece = threadIdx.x; piece < a.units; piece += kBlock) {
        float c[N];
        Piece<DT>::unpack(x[piece], c);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = c[i] - mean;
            s1 += d;
            s2 = fmaf(d, d, s2);
        }
    }
    const float off = block_sum(s1, lds) * a.inv_D;
    const float var = fmaf(-off, off, block_sum(s2, lds) * a.inv_D);
    const float rstd = inverse_deviation(var, a.eps);
    for (int piece = threadIdx.x; piece < a.units; piece += kBlock) {
        float c[N], gamma[N], beta[N];
        Piece<DT>::unpack(x[piece], c);
        load_floats<N>(a.gamma + (int64_t)piece * N, gamma);
        load_floats<N>(a.beta + (int64_t)piece * N, beta);
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = fmaf((c[i] - mean - off) * rstd, gamma[i], beta[i]);
        store_stream(a.y + row * a.units + piece, Piece<DT>::pack(c));
    }
    if (threadIdx.x == 0 && a.mean != nullptr) { a.mean[row] = corrected_mean(mean, off); a.rstd[row] = rstd; }
}

// A piece of x for the backward pass, from the rows or from their checkpoint.
template <int DT, bool PACKED>
struct XPiece {
    u32x4 raw;                       // PACKED: the codes in [0], [1]; the exponent in [2]
    __device__ __forceinline__ void load(const NormArgs& a, int64_t row, int piece)
    {
        constexpr int N = Piece<DT>::N, LPB = kPackBlock / N;
        if constexpr (PACKED) {
            const uint32_t* from = a.x_codes + (row * a.units + piece) * (N / 4);
            if constexpr (N == 8) {
                const u32x2 c = load_stream(reinterpret_cast<const u32x2*>(from));
                raw[0] = c[0]; raw[1] = c[1];
            } else {
                raw[0] = load_stream(from);
            }
            raw[2] = a.x_exps[row * a.nb + piece / LPB];
        } else {
            raw = load_stream(a.x + row * a.units + piece);
        }
    }
    __device__ __forceinline__ void zero() { raw = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ void values(float* v) const
    {
        if constexpr (PACKED) {
            unpack_piece<Piece<DT>::N>(raw[0], raw[1], (int)raw[2], v);
        } else {
            Piece<DT>::unpack(raw, v);
        }
    }
};

// SMALL: few rows in one launch.  The first workgroup goes over all of them and writes dgamma and dbeta, the others write
// their rows of dx; what both read comes from the L2 the second time.  Where dx is dy the first one does everything (the
// others would write what it still has to read), in the same order.
template <int DT, int G, int P, int U, bool PACKED, bool SMALL>
__global__ __launch_bounds__(kBlock) void norm_bwd_kernel(NormArgs a)
{
    constexpr int N = Piece<DT>::N, kGroups = kBlock / G;
    __shared__ float lds[kGroups][2][G * N];
    __shared__ float sums[kWavesPerBlock];
    const bool adds = !SMALL || blockIdx.x == 0, writes = !SMALL || blockIdx.x != 0 || gridDim.x == 1;
    const int64_t first = SMALL && blockIdx.x > 0 ? blockIdx.x - 1 : blockIdx.x;
    const int64_t step = SMALL && adds ? 1 : gridDim.x;
    const int lig = threadIdx.x % G, group = threadIdx.x / G;
    float gamma[P][N], dg[P][N], db[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int piece = lig + p * G < a.units ? lig + p * G : 0;
        load_floats<N>(a.gamma + (int64_t)piece * N, gamma[p]);
#pragma unroll
        for (int i = 0; i < N; ++i) dg[p][i] = db[p][i] = 0.0f;
    }
    for (int64_t r0 = first * (kGroups * U); r0 < a.n; r0 += step * (kGroups * U)) {
        u32x4 dy_raw[U][P];
        XPiece<DT, PACKED> x_raw[U][P];
        float mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = r0 + u * kGroups + group;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int piece = lig + p * G;
                dy_raw[u][p] = u32x4{0u, 0u, 0u, 0u};
                x_raw[u][p].zero();
                if (row < a.n && piece < a.units) {
                    dy_raw[u][p] = load_stream(a.dy + row * a.units + piece);
                    x_raw[u][p].load(a, row, piece);
                }
            }
            mean[u] = rstd[u] = 0.0f;
            if (row < a.n) { mean[u] = a.mean[row]; rstd[u] = a.rstd[row]; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = r0 + u * kGroups + group;
            float w[P][N], g[P][N];                      // u of the formula, and dy gamma
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const bool in = row < a.n && lig + p * G < a.units;
                float dy[N], t1 = 0.0f, t2 = 0.0f;
                x_raw[u][p].values(w[p]);
                Piece<DT>::unpack(dy_raw[u][p], dy);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    w[p][i] = in ? (w[p][i] - mean[u]) * rstd[u] : 0.0f;
                    if (adds) {
                        dg[p][i] = fmaf(dy[i], w[p][i], dg[p][i]);
                        db[p][i] += dy[i];
                    }
                    g[p][i] = dy[i] * gamma[p][i];
                    t1 += g[p][i];
                    t2 = fmaf(g[p][i], w[p][i], t2);
                }
                s1 += t1;
                s2 += t2;
            }
            if (!writes) continue;
            const float m1 = row_sum<G>(s1, sums) * a.inv_D, m2 = row_sum<G>(s2, sums) * a.inv_D;
            if (row >= a.n) continue;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (lig + p * G >= a.units) continue;
                float dx[N];
#pragma unroll
                for (int i = 0; i < N; ++i) dx[i] = rstd[u] * fmaf(-w[p][i], m2, g[p][i] - m1);
                store_stream(a.dx + row * a.units + lig + p * G, Piece<DT>::pack(dx));
            }
        }
    }
    if (!adds) return;
    const int64_t D = (int64_t)a.units * N;
    float* to = a.partial + (int64_t)blockIdx.x * 2 * D;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            lds[group][0][lig * N + i] = dg[p][i];
            lds[group][1][lig * N + i] = db[p][i];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * G * N; c += kBlock) {
            const int which = c / (G * N), col = c % (G * N);
            float s = 0.0f;
#pragma unroll 4
            for (int k = 0; k < kGroups; ++k) s += lds[k][which][col];
            if (p * G * N + col >= D) continue;
            if constexpr (SMALL) (which == 0 ? a.dgamma : a.dbeta)[p * G * N + col] = s;
            else to[which * D + p * G * N + col] = s;
        }
    }
}

// dgamma and dbeta as the sums of the `rows` partial rows of 2 D columns: a workgroup has 32 columns, thread (i, c) adds rows
// i, i + 32, ... of its column c, 16 of them in flight; then the 32 sums are added in order.
constexpr int kSumCols = 32, kSumRows = 32;
__global__ __launch_bounds__(kSumCols * kSumRows) void norm_grad_sum_kernel(const float* __restrict__ partial, int rows, int64_t D,
                                                                           float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float lds[kSumRows][kSumCols];
    const int c = threadIdx.x % kSumCols, i = threadIdx.x / kSumCols;
    const int64_t col = (int64_t)blockIdx.x * kSumCols + c;
    float s = 0.0f;
    if (col < 2 * D) {
        const float* from = partial + col;
        for (int r0 = i; r0 < rows; r0 += kSumRows * 16) {
            float v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int r = r0 + j * kSumRows;
                v[j] = from[(int64_t)(r < rows ? r : i) * 2 * D];
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) s += r0 + j * kSumRows < rows ? v[j] : 0.0f;
        }
    }
    lds[i][c] = s;
    __syncthreads();
    if (i != 0 || col >= 2 * D) return;
    s = 0.0f;
#pragma unroll
    for (int j = 0; j < kSumRows; ++j) s += lds[j][c];
    if (col < D) dgamma[col] = s; else dbeta[col - D] = s;
}

// Rows of more than 1024 pieces: dx by a workgroup a row.
template <int DT, bool PACKED>
__global__ __launch_bounds__(kBlock) void norm_bwd_wide_kernel(NormArgs a)
{
    constexpr int N = Piece<DT>::N;
    __shared__ float lds[kWavesPerBlock];
    const int64_t row = blockIdx.x;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int piece = threadIdx.x; piece < a.units; piece += kBlock) {
        XPiece<DT, PACKED> xp;
        xp.load(a, row, piece);
        float x[N], dy[N], gamma[N];
        xp.values(x);
        Piece<DT>::unpack(a.dy[row * a.units + piece], dy);
        load_floats<N>(a.gamma + (int64_t)piece * N, gamma);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float g = dy[i] * gamma[i];
            s1 += g;
            s2 = fmaf(g, (x[i] - mean) * rstd, s2);
        }
    }
    const float m1 = block_sum(s1, lds) * a.inv_D, m2 = block_sum(s2, lds) * a.inv_D;
    for (int piece = threadIdx.x; piece < a.units; piece += kBlock) {
        XPiece<DT, PACKED> xp;
        xp.load(a, row, piece);
        float x[N], dy[N], gamma[N];
        xp.values(x);
        Piece<DT>::unpack(a.dy[row * a.units + piece], dy);
        load_floats<N>(a.gamma + (int64_t)piece * N, gamma);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = rstd * fmaf(-((x[i] - mean) * rstd), m2, dy[i] * gamma[i] - m1);
        store_stream(a.dx + row * a.units + piece, Piece<DT>::pack(x));
    }
}

// ... and the columns' sums over the rows r, r + gridDim.y, ... by workgroups of 256 pieces of columns.
template <int DT, bool PACKED>
__global__ __launch_bounds__(kBlock) void norm_cols_wide_kernel(NormArgs a)
{
    constexpr int N = Piece<DT>::N;
    const int piece = (int)blockIdx.x * kBlock + (int)threadIdx.x;
    if (piece >= a.units) return;
    float dg[N], db[N];
#pragma unroll
    for (int i = 0; i < N; ++i) dg[i] = db[i] = 0.0f;
    for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
        XPiece<DT, PACKED> xp;
        xp.load(a, row, piece);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float x[N], dy[N];
        xp.values(x);
        Piece<DT>::unpack(a.dy[row * a.units + piece], dy);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            dg[i] = fmaf(dy[i], (x[i] - mean) * rstd, dg[i]);
            db[i] += dy[i];
        }
    }
    const int64_t D = (int64_t)a.units * N;
    float* to = a.partial + (int64_t)blockIdx.y * 2 * D + (int64_t)piece * N;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        to[i] = dg[i];
        to[D + i] = db[i];
    }
}

namespace {

constexpr int kWidePieces = 4 * kBlock;      // longest row that lies in the registers of a workgroup: 4 pieces a thread
// Workgroups (= partial rows) of a large backward pass: two a CU (256, 512, 768, 1024: 1331, 1114, 1118, 1241 us for the
// 3.93 M rows, with two rows a group; with four and 512 1078).
constexpr int kBwdBlocks = 512;
constexpr int kWideChunks = 64;              // row chunks of the wide columns' sums
constexpr int kSmallRounds = 8;              // rounds of one workgroup over all rows that are worth a launch less (100 rows of 256: 6.9 us, with the second launch 10.8)

// Lanes (G) and pieces a lane (P) of a row as constants: CALL(G, P).  Up to 256 pieces a wave or a part of it has the row, up
// to 1024 the workgroup.  One piece a lane where a wave's instruction then takes whole rows one after the other; with three pieces a
// lane fewer lanes lie past the row's end, and rows of more instructions apart in time share more cache lines.  Bf16, 0.8 GB, us:
// forward rows of 40 pieces (64, 1) 313, (16, 3) 265; 150 (64, 4) 473, (64, 3) 292; 600 (256, 4) 342, (256, 3) 287; but 17
// (32, 1) 342, (8, 3) 476.
#define FS_DISPATCH_FWD_ROW(units, CALL)                                                \
    do {                                                                                \
        if ((units) > 768) { CALL(256, 4); }                                            \
        else if ((units) > 512) { CALL(256, 3); }                                       \
        else if ((units) > 256) { CALL(256, 2); }                                       \
        else if ((units) > 192) { CALL(64, 4); }                                        \
        else if ((units) > 128) { CALL(64, 3); }                                        \
        else if ((units) > 64) { CALL(64, 2); }                                         \
        else if ((units) > 48) { CALL(64, 1); }                                         \
        else if ((units) > 32) { CALL(16, 3); }                                         \
        else if ((units) > 16) { CALL(32, 1); }                                         \
        else if ((units) > 8) { CALL(16, 1); }                                          \
        else if ((units) > 4) { CALL(8, 1); }                                           \
        else { CALL(4, 1); }                                                            \
    } while (0)
// Backward fewer lanes a row still: what a lane does beside its columns (the sums over the lanes, the row's statistics and
// places) is shared by more of them.  From the checkpoint, bf16, 0.4 G values, us: 40 pieces (64, 1) 562, (16, 3) 346; 64 (64, 1) 377,
// (32, 2) 353; 65 (64, 2) 589, (32, 3) 413; 100 (64, 2) 408, (32, 4) 354; 513 (256, 4) 523, (256, 3) 449; from the rows 1 to 11 %.
// few: rows of 16-bit types from their checkpoint, which have the most to do for a byte: 9 pieces (16, 1) 600, (8, 2) 563; 24
// (32, 1) 463, (8, 3) 355; 32 (32, 1) 933, (16, 2) 890 (3.93 M rows).  From the rows 17 pieces (32, 1) 488, (16, 2) 540, and of fp32 from
// its checkpoint (32, 1) 432, (8, 3) 479.
#define FS_DISPATCH_BWD_ROW(units, few, CALL)                                           \
    do {                                                                                \
        if ((units) > 768) { CALL(256, 4); }                                            \
        else if ((units) > 512) { CALL(256, 3); }                                       \
        else if ((units) > 256) { CALL(256, 2); }                                       \
        else if ((units) > 128) { CALL(64, 4); }                                        \
        else if ((units) > 96) { CALL(32, 4); }                                         \
        else if ((units) > 64) { CALL(32, 3); }                                         \
        else if ((units) > 48) { CALL(32, 2); }                                         \
        else if ((units) > 32) { CALL(16, 3); }                                         \
        else if constexpr (few) {                                                       \
            if ((units) > 24) { CALL(16, 2); }                                          \
            else if ((units) > 16) { CALL(8, 3); }                                      \
            else if ((units) > 8) { CALL(8, 2); }                                       \
            else if ((units) > 4) { CALL(8, 1); }                                       \
            else { CALL(4, 1); }                                                        \
        } else {                                                                        \
            if ((units) > 16) { CALL(32, 1); }                                          \
            else if ((units) > 8) { CALL(16, 1); }                                      \
            else if ((units) > 4) { CALL(8, 1); }                                       \
            else { CALL(4, 1); }                                                        \
        }                                                                               \
    } while (0)

// Rows that a group has in flight.  Forward 2 (3.93 M rows of 256 bf16: 1, 2, 4, 8 rows 728, 691, 718, 718 us; rows of 1024 pieces 1, 2
// rows 339, 280).  Backward 4 of one piece a lane (3.93 M rows of 256: 2, 4 rows 1114, 1078), 2 of a workgroup with two pieces (300
// pieces: 1, 2 rows 544, 472), else 1 (80 pieces, three a lane: 1, 2 rows 411, 434).
constexpr int kFwdRows = 2;
constexpr int bwd_rows(int G, int P) { return P == 1 ? 4 : G > kWave && P == 2 ? 2 : 1; }

// Rows of a workgroup's round in the backward pass.
template <bool FEW>
int64_t bwd_round_of(int units)
{
#define CALL(G, P) return (int64_t)(kBlock / G) * bwd_rows(G, P)
    FS_DISPATCH_BWD_ROW(units, FEW, CALL);
#undef CALL
}

int64_t bwd_round(int units, bool few) { return few ? bwd_round_of<true>(units) : bwd_round_of<false>(units); }

int64_t bwd_blocks(int64_t n, int units, bool few)
{
    if (units > kWidePieces) return n < kWideChunks ? n : kWideChunks;
    const int64_t per = bwd_round(units, few), need = (n + per - 1) / per;
    return need < kBwdBlocks ? need : kBwdBlocks;
}

bool bwd_small(int64_t n, int units, bool few) { return units <= kWidePieces && n <= kSmallRounds * bwd_round(units, few); }

// The arguments from row r0 on, for `rows` rows.
template <int DT>
NormArgs part_of(NormArgs a, int64_t r0, int64_t rows)
{
    constexpr int N = Piece<DT>::N;
    const auto skip = [&](auto*& p, int64_t n) { if (p != nullptr) p += n; };
    skip(a.x, r0 * a.units); skip(a.dy, r0 * a.units); skip(a.y, r0 * a.units); skip(a.dx, r0 * a.units);
    skip(a.x_codes, r0 * a.units * (N / 4)); skip(a.codes, r0 * a.units * (N / 4));
    skip(a.x_exps, r0 * a.nb); skip(a.exps, r0 * a.nb);
    skip(a.mean, r0); skip(a.rstd, r0);
    a.n = rows;
    return a;
}

// Rows of a forward launch.
int64_t fwd_launch_rows(int units)
{
    if (units > kWidePieces) return kMostGrid;
#define CALL(G, P) return kMostGrid * ((kBlock / G) * kFwdRows)
    FS_DISPATCH_FWD_ROW(units, CALL);
#undef CALL
}

template <int DT>
fs_status norm_fwd_launch(const NormArgs& a, hipStream_t s)
{
    const int64_t most = fwd_launch_rows(a.units);
    if (a.n > most) {
        const fs_status rc = norm_fwd_launch<DT>(part_of<DT>(a, 0, most), s);
        return rc != FS_OK ? rc : norm_fwd_launch<DT>(part_of<DT>(a, most, a.n - most), s);
    }
    const bool pack = a.codes != nullptr;
    if (a.units > kWidePieces) {
        if (pack) FS_LAUNCH("norm_fwd_wide", (norm_fwd_wide_kernel<DT, true>), dim3((unsigned)a.n), dim3(kBlock), s, a);
        else FS_LAUNCH("norm_fwd_wide", (norm_fwd_wide_kernel<DT, false>), dim3((unsigned)a.n), dim3(kBlock), s, a);
        return FS_OK;
    }
#define CALL(G, P)                                                                                                        \
    do {                                                                                                                  \
        constexpr int U = kFwdRows;                                                                                       \
        const unsigned grid = (unsigned)((a.n + (kBlock / G) * U - 1) / ((kBlock / G) * U));                              \
        if (pack) FS_LAUNCH("norm_fwd", (norm_fwd_kernel<DT, G, P, U, true>), dim3(grid), dim3(kBlock), s, a);            \
        else FS_LAUNCH("norm_fwd", (norm_fwd_kernel<DT, G, P, U, false>), dim3(grid), dim3(kBlock), s, a);                \
    } while (0)
    FS_DISPATCH_FWD_ROW(a.units, CALL);
#undef CALL
    return FS_OK;
}

template <int DT, bool PACKED>
fs_status norm_bwd_launch(const NormArgs& a, hipStream_t s)
{
    constexpr bool few = PACKED && DT != FS_F32;
    const unsigned blocks = (unsigned)bwd_blocks(a.n, a.units, few);
    if (a.units > kWidePieces) {
        // the sums first: dx may be dy
        FS_LAUNCH("norm_cols_wide", (norm_cols_wide_kernel<DT, PACKED>), dim3((unsigned)((a.units + kBlock - 1) / kBlock), blocks),
                  dim3(kBlock), s, a);
        for (int64_t r0 = 0; r0 < a.n; r0 += kMostGrid) {
            const int64_t rows = a.n - r0 < kMostGrid ? a.n - r0 : kMostGrid;
            FS_LAUNCH("norm_bwd_wide", (norm_bwd_wide_kernel<DT, PACKED>), dim3((unsigned)rows), dim3(kBlock), s, part_of<DT>(a, r0, rows));
        }
        return FS_OK;
    }
#define CALL(G, P)                                                                                                        \
    do {                                                                                                                  \
        constexpr int U = bwd_rows(G, P);                                                                                 \
        if (bwd_small(a.n, a.units, few)) FS_LAUNCH("norm_bwd", (norm_bwd_kernel<DT, G, P, U, PACKED, true>), dim3(a.dx == a.dy ? 1 : blocks + 1), dim3(kBlock), s, a); \
        else FS_LAUNCH("norm_bwd", (norm_bwd_kernel<DT, G, P, U, PACKED, false>), dim3(blocks), dim3(kBlock), s, a);      \
    } while (0)
    FS_DISPATCH_BWD_ROW(a.units, few, CALL);
#undef CALL
    return FS_OK;
}

fs_status norm_bwd(NormArgs a, bool packed, int32_t D, fs_dtype dtype, float* dgamma, float* dbeta, void* workspace,
                   size_t* workspace_bytes, hipStream_t s)
{
    if (!workspace_bytes) return FS_ERR_NULL;
    const fs_status st = check_seq_rows(a.n, D, dtype, &a.units);
    if (st != FS_OK) return st;
    if (a.units > kMostPieces) return FS_ERR_SIZE;
    Carver ws(workspace);
    const bool few = packed && dtype != FS_F32;
    const int64_t blocks = bwd_blocks(a.n, a.units, few), other = bwd_blocks(a.n, a.units, !few);      // one size for both forms
    const int64_t held = blocks > other ? blocks : other;
    a.partial = ws.take<float>((size_t)(held > 0 ? held : 1) * 2 * (size_t)D);      // never nothing: a null workspace is a question
    if (!workspace) { *workspace_bytes = ws.used; return FS_OK; }
    if (*workspace_bytes < ws.used || misaligned(workspace, 256)) return FS_ERR_WORKSPACE;
    if (!a.gamma || !dgamma || !dbeta) return FS_ERR_NULL;
    if (a.n > 0 && (!a.dy || !a.mean || !a.rstd || !a.dx || (packed ? !a.x_codes || !a.x_exps : !a.x))) return FS_ERR_NULL;
    if (misaligned(a.dy, 16) || misaligned(a.x, 16) || misaligned(a.x_codes, codes_alignment(dtype)) || misaligned(a.dx, 16) ||
        misaligned(a.gamma, 16) || misaligned(dgamma, 4) || misaligned(dbeta, 4) || misaligned(a.mean, 4) || misaligned(a.rstd, 4))
        return FS_ERR_ALIGN;
    a.nb = (int)pack_blocks(D);
    a.inv_D = 1.0f / (float)D;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    if (a.n > 0) {
        fs_status rc = FS_OK;
        if (packed) {
#define CALL(DT) rc = norm_bwd_launch<DT, true>(a, s)
            FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
        } else {
#define CALL(DT) rc = norm_bwd_launch<DT, false>(a, s)
            FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
        }
        if (rc != FS_OK || bwd_small(a.n, a.units, few)) return rc;
    }
    FS_LAUNCH("norm_grad_sum", norm_grad_sum_kernel, dim3((unsigned)((2 * (int64_t)D + kSumCols - 1) / kSumCols)),
              dim3(kSumCols * kSumRows), s, a.partial, (int)blocks, (int64_t)D, dgamma, dbeta);
    return FS_OK;
}

}  // namespace
}  // namespace fs

extern "C" fs_status fs_seq_norm_fwd(
    const void* x, int64_t n, int32_t D, fs_dtype dtype, const float* gamma, const float* beta, float eps,
    void* y, float* mean, float* rstd, int8_t* codes, uint8_t* exps, void* stream)
{
    using namespace fs;
    NormArgs a = {};
    const fs_status st = check_seq_rows(n, D, dtype, &a.units);
    if (st != FS_OK) return st;
    if (a.units > kMostPieces) return FS_ERR_SIZE;
    if (!(eps > 0.0f) || __builtin_isinf(eps)) return FS_ERR_CONFIG;
    if (n == 0) return FS_OK;
    if (!x || !gamma || !beta || !y) return FS_ERR_NULL;
    if ((mean != nullptr) != (rstd != nullptr) || (codes != nullptr) != (exps != nullptr)) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(y, 16) || misaligned(gamma, 16) || misaligned(beta, 16) || misaligned(codes, codes_alignment(dtype)) ||
        misaligned(mean, 4) || misaligned(rstd, 4))
        return FS_ERR_ALIGN;
    a.x = static_cast<const u32x4*>(x); a.n = n;
    a.nb = (int)pack_blocks(D);
    a.inv_D = 1.0f / (float)D; a.eps = eps;
    a.gamma = gamma; a.beta = beta;
    a.y = static_cast<u32x4*>(y); a.mean = mean; a.rstd = rstd;
    a.codes = reinterpret_cast<uint32_t*>(codes); a.exps = exps;
#define CALL(DT) return norm_fwd_launch<DT>(a, static_cast<hipStream_t>(stream))
    FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
}

extern "C" fs_status fs_seq_norm_bwd(
    const void* dy, const void* x, const float* mean, const float* rstd, int64_t n, int32_t D, fs_dtype dtype,
    const float* gamma, void* dx, float* dgamma, float* dbeta,
    void* workspace, size_t* workspace_bytes, void* stream)
{
    using namespace fs;
    NormArgs a = {};
    a.dy = static_cast<const u32x4*>(dy); a.x = static_cast<const u32x4*>(x); a.n = n;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.gamma = gamma; a.dx = static_cast<u32x4*>(dx);
    return norm_bwd(a, false, D, dtype, dgamma, dbeta, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" fs_status fs_seq_norm_bwd_packed(
    const void* dy, const int8_t* codes, const uint8_t* exps, const float* mean, const float* rstd,
    int64_t n, int32_t D, fs_dtype dtype, const float* gamma, void* dx, float* dgamma, float* dbeta,
    void* workspace, size_t* workspace_bytes, void* stream)
{
    using namespace fs;
    NormArgs a = {};
    a.dy = static_cast<const u32x4*>(dy); a.n = n;
    a.x_codes = reinterpret_cast<const uint32_t*>(codes); a.x_exps = exps;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.gamma = gamma; a.dx = static_cast<u32x4*>(dx);
    return norm_bwd(a, true, D, dtype, dgamma, dbeta, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}
