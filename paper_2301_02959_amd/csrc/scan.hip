// fs_seq_scan_fwd, fs_seq_scan_bwd, fs_seq_scan_bwd_packed, fs_seq_scan_step: a gated linear recurrence along the sequences of
// a jagged batch.
//
//   forward   f = 1 / (1 + e^-gate), h_t = f_t h_(t-1) + (1 - f_t) x_t
//   backward  U_t = f_t G_t, G_t = dh_t + U_(t+1):  dx_t = (1 - f_t) G_t, dgate_t = G_t (h_(t-1) - x_t) f_t (1 - f_t)
//
// A workgroup walks one sequence for 64 pieces of columns.  States are fp32.
#include "pack8.h"
#include "seq_rows.h"

namespace fs {

struct ScanArgs {
    const u32x4* x;
    const u32x4* gate;
    const u32x4* h_in;               // backward: the forward pass's output
    const u32x4* dh;
    const uint32_t* codes[3];        // packed backward: x, gate, h as checkpoints
    const uint8_t* exps[3];
    int64_t n;
    int units;
    int nb;
    const int64_t* offsets;
    int64_t S;
    const float* h0;
    const float* dh_last;
    u32x4* h;
    float* h_last;
    u32x4* dx;
    u32x4* dgate;
    float* dh0;
    int32_t* status;
};

// f and 1 - f of a gate, each to the precision of e^-gate (1 - f is not taken from f, which is 1 for large gates).
__device__ __forceinline__ void gate_pair(float gate, float* f, float* o)
{
    const float e = __expf(-gate);
    *f = __builtin_amdgcn_rcpf(1.0f + e);
    *o = e > 1e30f ? 1.0f : e * *f;                     // e = infinity (a shut gate): f = 0, 1 - f = 1
}

template <int DT>
__device__ __forceinline__ void load_piece(const u32x4* p, int64_t at, float* v)
{
    Piece<DT>::unpack(p[at], v);
}

template <int DT, bool PACKED, int WHICH>
__device__ __forceinline__ void load_saved(const ScanArgs& a, int64_t row, int piece, float* v)
{
    constexpr int N = Piece<DT>::N, LPB = kPackBlock / N;
    if constexpr (PACKED) {
        const uint32_t* from = a.codes[WHICH] + (row * a.units + piece) * (N / 4);
        const int E = a.exps[WHICH][row * a.nb + piece / LPB];
        const float step = __uint_as_float(pack_step_bits(E));
        unpack_four(from[0], E, step, v);
        if constexpr (N == 8) unpack_four(from[1], E, step, v + 4);
    } else {
        const u32x4* p = WHICH == 0 ? a.x : WHICH == 1 ? a.gate : a.h_in;
        Piece<DT>::unpack(p[row * a.units + piece], v);
    }
}

// Rows [b, e) of sequence s, kept within [0, n) whatever the offsets say.
__device__ __forceinline__ void seq_bounds(const ScanArgs& a, int64_t s, int64_t* b, int64_t* e)
{
    *b = a.offsets[s];
    *e = a.offsets[s + 1];
    if (*b < 0 || *e > a.n || *b > *e || (s == 0 && *b != 0) || (s == a.S - 1 && *e != a.n)) {
        if (threadIdx.x == 0) report(a.status, FS_DEV_BAD_OFFSETS);
        *b = *b < 0 ? 0 : *b > a.n ? a.n : *b;
        *e = *e < *b ? *b : *e > a.n ? a.n : *e;
    }
}

template <int DT>
__global__ __launch_bounds__(kWave) void scan_fwd_kernel(ScanArgs a)
{
    constexpr int N = Piece<DT>::N;
    const int64_t s = blockIdx.x;
    int64_t b, e;
    seq_bounds(a, s, &b, &e);
    const int piece = (int)blockIdx.y * kWave + (int)threadIdx.x;
    if (piece >= a.units) return;
    const int64_t at = (s * a.units + piece) * N;
    float h[N];
#pragma unroll
    for (int i = 0; i < N; ++i) h[i] = a.h0 ? a.h0[at + i] : 0.0f;
    for (int64_t t = b; t < e; ++t) {
        float x[N], g[N];
        load_piece<DT>(a.x, t * a.units + piece, x);
        load_piece<DT>(a.gate, t * a.units + piece, g);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f, o;
            gate_pair(g[i], &f, &o);
            h[i] = fmaf(f, h[i], o * x[i]);
        }
        a.h[t * a.units + piece] = Piece<DT>::pack(h);
    }
    if (a.h_last)
#pragma unroll
        for (int i = 0; i < N; ++i) a.h_last[at + i] = h[i];
}

template <int DT, bool PACKED>
__global__ __launch_bounds__(kWave) void scan_bwd_kernel(ScanArgs a)
{
    constexpr int N = Piece<DT>::N;
    const int64_t s = blockIdx.x;
    int64_t b, e;
    seq_bounds(a, s, &b, &e);
    const int piece = (int)blockIdx.y * kWave + (int)threadIdx.x;
    if (piece >= a.units) return;
    const int64_t at = (s * a.units + piece) * N;
    float U[N];
#pragma unroll
    for (int i = 0; i < N; ++i) U[i] = a.dh_last ? a.dh_last[at + i] : 0.0f;
    for (int64_t t = e - 1; t >= b; --t) {
        float x[N], g[N], hb[N], dh[N], dx[N], dg[N];
        load_saved<DT, PACKED, 0>(a, t, piece, x);
        load_saved<DT, PACKED, 1>(a, t, piece, g);
        load_piece<DT>(a.dh, t * a.units + piece, dh);
        if (t > b) {
            load_saved<DT, PACKED, 2>(a, t - 1, piece, hb);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) hb[i] = a.h0 ? a.h0[at + i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f, o;
            gate_pair(g[i], &f, &o);
            const float G = dh[i] + U[i];
            dx[i] = o * G;
            dg[i] = dx[i] * f * (hb[i] - x[i]);
            U[i] = f * G;
        }
        a.dx[t * a.units + piece] = Piece<DT>::pack(dx);
        a.dgate[t * a.units + piece] = Piece<DT>::pack(dg);
    }
    if (a.dh0)
#pragma unroll
        for (int i = 0; i < N; ++i) a.dh0[at + i] = U[i];
}

// One token of every session: a 16-byte piece of x, gate and out to a lane, its states as fp32 beside it.
template <int DT>
__global__ __launch_bounds__(kBlock) void scan_step_kernel(const u32x4* __restrict__ x, const u32x4* __restrict__ gate,
                                                           const float* state, float* state_out, u32x4* __restrict__ h, int64_t pieces)
{
    constexpr int N = Piece<DT>::N;
    const int64_t at = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (at >= pieces) return;
    float xv[N], g[N], v[N];
    Piece<DT>::unpack(load_stream(x + at), xv);
    Piece<DT>::unpack(load_stream(gate + at), g);
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(state + at * N + i);
        v[i] = q[0]; v[i + 1] = q[1]; v[i + 2] = q[2]; v[i + 3] = q[3];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float f, o;
        gate_pair(g[i], &f, &o);
        v[i] = fmaf(f, v[i], o * xv[i]);
    }
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4*>(state_out + at * N + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
    h[at] = Piece<DT>::pack(v);
}

namespace {

// What both directions check before a workspace is asked for; *S = sequences.
fs_status check_scan(int64_t n, int32_t D, fs_dtype dtype, int32_t T, int32_t B, ScanArgs* a)
{
    const fs_status st = check_seq_rows(n, D, dtype, &a->units);
    if (st != FS_OK) return st;
    if (T < 1 || B < 1 || (int64_t)T * B >= (1LL << 31)) return FS_ERR_SIZE;
    a->S = (int64_t)T * B;
    a->n = n;
    a->nb = (int)pack_blocks(D);
    return FS_OK;
}

fs_status scan_bwd(ScanArgs a, bool packed, int32_t D, fs_dtype dtype, int32_t T, int32_t B, void* workspace,
                   size_t* workspace_bytes, hipStream_t s)
{
    if (!workspace_bytes) return FS_ERR_NULL;
    const fs_status st = check_scan(a.n, D, dtype, T, B, &a);
    if (st != FS_OK) return st;
    if (!workspace) { *workspace_bytes = 0; return FS_OK; }
    if (misaligned(workspace, 256)) return FS_ERR_WORKSPACE;
    if (!a.offsets) return FS_ERR_NULL;
    if (a.n > 0) {
        if (!a.dh || !a.dx || !a.dgate) return FS_ERR_NULL;
        if (!packed && (!a.x || !a.gate || !a.h_in)) return FS_ERR_NULL;
        for (int k = 0; packed && k < 3; ++k)
            if (!a.codes[k] || !a.exps[k]) return FS_ERR_NULL;
    }
    if (misaligned(a.dh, 16) || misaligned(a.x, 16) || misaligned(a.gate, 16) || misaligned(a.h_in, 16) || misaligned(a.dx, 16) ||
        misaligned(a.dgate, 16) || misaligned(a.codes[0], codes_alignment(dtype)) || misaligned(a.codes[1], codes_alignment(dtype)) || misaligned(a.codes[2], codes_alignment(dtype)) ||
        misaligned(a.h0, 16) || misaligned(a.dh_last, 16) || misaligned(a.dh0, 16) || misaligned(a.offsets, 8))
        return FS_ERR_ALIGN;
    const dim3 grid((unsigned)a.S, (unsigned)((a.units + kWave - 1) / kWave));
    if (packed) {
#define CALL(DT) FS_LAUNCH("scan_bwd", (scan_bwd_kernel<DT, true>), grid, dim3(kWave), s, a)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    } else {
#define CALL(DT) FS_LAUNCH("scan_bwd", (scan_bwd_kernel<DT, false>), grid, dim3(kWave), s, a)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    }
    return FS_OK;
}

}  // namespace
}  // namespace fs

extern "C" fs_status fs_seq_scan_fwd(
    const void* x, const void* gate, int64_t n, int32_t D, fs_dtype dtype, const int64_t* offsets, int32_t T, int32_t B,
    const float* h0, void* h, float* h_last,
    void* workspace, size_t* workspace_bytes, void* stream, int32_t* dev_status)
{
    using namespace fs;
    if (!workspace_bytes) return FS_ERR_NULL;
    ScanArgs a = {};
    const fs_status st = check_scan(n, D, dtype, T, B, &a);
    if (st != FS_OK) return st;
    if (!workspace) { *workspace_bytes = 0; return FS_OK; }
    if (misaligned(workspace, 256)) return FS_ERR_WORKSPACE;
    if (!offsets || (n > 0 && (!x || !gate || !h))) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(gate, 16) || misaligned(h, 16) || misaligned(h0, 16) || misaligned(h_last, 16) || misaligned(offsets, 8))
        return FS_ERR_ALIGN;
    a.x = static_cast<const u32x4*>(x); a.gate = static_cast<const u32x4*>(gate);
    a.offsets = offsets; a.h0 = h0; a.h = static_cast<u32x4*>(h); a.h_last = h_last; a.status = dev_status;
    const dim3 grid((unsigned)a.S, (unsigned)((a.units + kWave - 1) / kWave));
#define CALL(DT) FS_LAUNCH("scan_fwd", scan_fwd_kernel<DT>, grid, dim3(kWave), static_cast<hipStream_t>(stream), a)
    FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    return FS_OK;
}

extern "C" fs_status fs_seq_scan_bwd(
    const void* dh, const float* dh_last, const void* x, const void* gate, const void* h,
    int64_t n, int32_t D, fs_dtype dtype, const int64_t* offsets, int32_t T, int32_t B, const float* h0,
    void* dx, void* dgate, float* dh0,
    void* workspace, size_t* workspace_bytes, void* stream, int32_t* dev_status)
{
    using namespace fs;
    ScanArgs a = {};
    a.dh = static_cast<const u32x4*>(dh); a.dh_last = dh_last; a.n = n;
    a.x = static_cast<const u32x4*>(x); a.gate = static_cast<const u32x4*>(gate); a.h_in = static_cast<const u32x4*>(h);
    a.offsets = offsets; a.h0 = h0;
    a.dx = static_cast<u32x4*>(dx); a.dgate = static_cast<u32x4*>(dgate); a.dh0 = dh0; a.status = dev_status;
    return scan_bwd(a, false, D, dtype, T, B, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" fs_status fs_seq_scan_bwd_packed(
    const void* dh, const float* dh_last, const int8_t* x_codes, const uint8_t* x_exps,
    const int8_t* gate_codes, const uint8_t* gate_exps, const int8_t* h_codes, const uint8_t* h_exps,
    int64_t n, int32_t D, fs_dtype dtype, const int64_t* offsets, int32_t T, int32_t B, const float* h0,
    void* dx, void* dgate, float* dh0,
    void* workspace, size_t* workspace_bytes, void* stream, int32_t* dev_status)
{
    using namespace fs;
    ScanArgs a = {};
    a.dh = static_cast<const u32x4*>(dh); a.dh_last = dh_last; a.n = n;
    a.codes[0] = reinterpret_cast<const uint32_t*>(x_codes); a.exps[0] = x_exps;
    a.codes[1] = reinterpret_cast<const uint32_t*>(gate_codes); a.exps[1] = gate_exps;
    a.codes[2] = reinterpret_cast<const uint32_t*>(h_codes); a.exps[2] = h_exps;
    a.offsets = offsets; a.h0 = h0;
    a.dx = static_cast<u32x4*>(dx); a.dgate = static_cast<u32x4*>(dgate); a.dh0 = dh0; a.status = dev_status;
    return scan_bwd(a, true, D, dtype, T, B, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

extern "C" fs_status fs_seq_scan_step(
    const void* x, const void* gate, int64_t m, int32_t D, fs_dtype dtype, const float* state, float* state_out, void* h, void* stream)
{
    using namespace fs;
    int units = 0;
    const fs_status st = check_seq_rows(m, D, dtype, &units);
    if (st != FS_OK) return st;
    if (m == 0) return FS_OK;
    if (!x || !gate || !state || !state_out || !h) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(gate, 16) || misaligned(state, 16) || misaligned(state_out, 16) || misaligned(h, 16))
        return FS_ERR_ALIGN;
    const int64_t pieces = m * units, grid = (pieces + kBlock - 1) / kBlock;
    if (grid > 0x7FFFFFFF) return FS_ERR_SIZE;
#define CALL(DT) FS_LAUNCH("scan_step", scan_step_kernel<DT>, dim3((unsigned)grid), dim3(kBlock), static_cast<hipStream_t>(stream),  \
                           static_cast<const u32x4*>(x), static_cast<const u32x4*>(gate), state, state_out, static_cast<u32x4*>(h), pieces)
    FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    return FS_OK;
}
