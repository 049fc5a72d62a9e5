// fs_seq_scan_fwd, fs_seq_scan_bwd, fs_seq_scan_bwd_packed, fs_seq_scan_step: a gated linear recurrence along the sequences of
// a jagged batch.
//
//   forward   f = 1 / (1 + e^-gate), h_t = f_t h_(t-1) + (1 - f_t) x_t
//   backward  U_t = f_t G_t, G_t = dh_t + U_(t+1):  dx_t = (1 - f_t) G_t, dgate_t = G_t (h_(t-1) - x_t) f_t (1 - f_t)
//
// Both are v -> f v + b along the rows, and a stretch of rows is (A, B): v -> A v + B with A the product of its f; one that
// holds a sequence's first row (backwards: its last) does not depend on v at all.  So the rows are cut into tiles of equal
// size whatever the sequences' lengths: no sequence is too short to fill a wave or too long for one.  HBM-bound, every
// row is read once:
//   a group of G lanes has R consecutive rows of its columns in registers, as f and b, and folds them to (A, B);
//   a thread a column folds the groups of the workgroup, publishes the tile's (A, B), or its last state where a sequence
//   begins in the tile, looks back over the tiles before until it meets a state, goes forward from there over their pairs, and
//   publishes its own last state.  Going forward, a tile's state is A v + B of the state before it whoever computes it and
//   however far back the search went, so the bits do not depend on which tiles were done first;
//   the groups go over their registers a second time, from the state that reaches them, and write.
// Tiles are handed out in their order by a counter, so the tiles that a workgroup waits for are running or done, and every
// tile publishes whatever the data: every wait ends.  A published pair is one 8-byte word that is its own flag (relaxed
// atomics at the scope of the GPU, nothing else is passed on), cleared by a launch in front.
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
    const float* ends_in;            // forward: h0; backward: dh_last
    const float* h0;
    u32x4* h;
    float* ends_out;                 // forward: h_last; backward: dh0
    u32x4* dx;
    u32x4* dgate;
    int32_t* status;
    int64_t tiles;
    int64_t strides;                 // workgroups a block of columns; those past `tiles` only look after empty sequences
    int col_blocks;                  // blocks of G pieces of columns
    uint64_t* words;                 // [tiles][col_blocks][G * N]
    uint32_t* ticket;                // null: one tile, nothing to wait for
};

// f and 1 - f of a gate, each to the precision of e^-gate (1 - f is not taken from f, which is 1 for large gates).
__device__ __forceinline__ void gate_pair(float gate, float* f, float* o)
{
    const float e = __expf(-gate);
    *f = __builtin_amdgcn_rcpf(1.0f + e);
    *o = e > 1e30f ? 1.0f : e * *f;                     // e = infinity (a shut gate): f = 0, 1 - f = 1
}

// One of the three saved inputs of the backward pass at a row's piece, from the rows or from their checkpoint; 0: x, 1: gate, 2: h.
template <int DT, bool PACKED, int WHICH>
struct Saved {
    u32x4 raw;                       // PACKED: the codes in [0], [1]; the exponent in [2]
    __device__ __forceinline__ void zero() { raw = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ void load(const ScanArgs& a, int64_t row, int piece)
    {
        constexpr int N = Piece<DT>::N, LPB = kPackBlock / N;
        if constexpr (PACKED) {
            const uint32_t* from = a.codes[WHICH] + (row * a.units + piece) * (N / 4);
            if constexpr (N == 8) {
                const u32x2 c = *reinterpret_cast<const u32x2*>(from);
                raw[0] = c[0]; raw[1] = c[1];
            } else {
                raw[0] = *from;
            }
            raw[2] = a.exps[WHICH][row * a.nb + piece / LPB];
        } else {
            const u32x4* from = WHICH == 0 ? a.x : WHICH == 1 ? a.gate : a.h_in;
            raw = from[row * a.units + piece];
        }
    }
    __device__ __forceinline__ void values(float* v) const
    {
        if constexpr (PACKED) {
            const float step = __uint_as_float(pack_step_bits((int)raw[2]));
            unpack_four(raw[0], (int)raw[2], step, v);
            if constexpr (Piece<DT>::N == 8) unpack_four(raw[1], (int)raw[2], step, v + 4);
        } else {
            Piece<DT>::unpack(raw, v);
        }
    }
};

// G lanes a row, R rows a group.
template <int DT, int G_, int R_>
struct ScanShape {
    static constexpr int N = Piece<DT>::N, G = G_, R = R_;
    static constexpr int C = G * N;                     // columns of a workgroup
    static constexpr int Q = kBlock / G;                // groups
    static constexpr int T = Q * R;                     // rows of a tile
    static constexpr int P = kBlock / C;                // threads a column
    static_assert(T % 32 == 0 && 32 % R == 0 && C <= kBlock, "");
};

constexpr int kLookAhead = 4;                           // tiles that a thread looks back over at once

template <class Shape>
struct ScanShared {
    float A[Shape::Q][Shape::C];                        // the groups' pairs in the order of the walk; then B is what reaches them
    float B[Shape::Q][Shape::C];
    uint64_t seen[Shape::P * kLookAhead][Shape::C];     // the words of the tiles looked back over
    uint32_t firsts[Shape::T / 32], lasts[Shape::T / 32];   // rows of the tile where a sequence begins, ends
    int32_t first_of[Shape::T], last_of[Shape::T];      // ... and which one
    uint32_t ticket;
};

// Marks the first and last rows of the sequences in tile `row0` ..  Every thread calls it; contains barriers.  With bad
// offsets the marks are arbitrary but inside the tile.
template <class Shape>
__device__ __forceinline__ void mark_sequences(const ScanArgs& a, int64_t row0, ScanShared<Shape>* sh)
{
    for (int w = threadIdx.x; w < Shape::T / 32; w += kBlock) sh->firsts[w] = sh->lasts[w] = 0u;
    const int64_t row1 = row0 + Shape::T < a.n ? row0 + Shape::T : a.n;
    // the sequence that row0 - 1 is in and those after it, as far as they begin before row1
    int64_t s = row0 == 0 ? 0 : wave_table_of(a.offsets, (int)a.S, 1, row0 - 1);
    s += threadIdx.x;
    __syncthreads();
    for (bool more = true; more; s += kBlock) {
        int64_t b = row1, e = row1;
        if (s < a.S) { b = a.offsets[s]; e = a.offsets[s + 1]; }
        if (b < e) {
            if (b >= row0 && b < row1) {
                atomicOr(&sh->firsts[(b - row0) >> 5], 1u << ((b - row0) & 31));
                sh->first_of[b - row0] = (int32_t)s;
            }
            if (e > row0 && e <= row1) {
                atomicOr(&sh->lasts[(e - 1 - row0) >> 5], 1u << ((e - 1 - row0) & 31));
                sh->last_of[e - 1 - row0] = (int32_t)s;
            }
        }
        more = __syncthreads_or(threadIdx.x == kBlock - 1 && s < a.S && b < row1) != 0;
    }
}

// Marks of a group's R rows, bit r for row r.
template <class Shape>
__device__ __forceinline__ uint32_t group_marks(const uint32_t* marks, int group)
{
    const int at = group * Shape::R;
    return (marks[at >> 5] >> (at & 31)) & (uint32_t)((1ull << Shape::R) - 1ull);
}

constexpr uint64_t kNotReady = ~0ull;
constexpr uint32_t kIsState = 0xFF800000u;              // in place of A (which is not negative): B is the state after the tile

__device__ __forceinline__ uint64_t pair_word(float A, float B)
{
    return ((uint64_t)(A != A ? 0x7FC00000u : __float_as_uint(A)) << 32) | __float_as_uint(B);   // no NaN looks like kNotReady
}

__device__ __forceinline__ bool is_state(uint64_t word) { return (uint32_t)(word >> 32) == kIsState; }

__device__ __forceinline__ uint64_t state_word(float v) { return ((uint64_t)kIsState << 32) | __float_as_uint(v); }

// From the groups' pairs in sh->A and sh->B to the states that reach the groups, in sh->B.  k: the tile's number in the order
// of the walk; resets: bit q = a sequence begins in group q (in that order); open: the tile's first row goes on with a
// sequence of the tile before.  Every thread calls it; contains barriers.
template <class Shape>
__device__ __forceinline__ void carry_states(const ScanArgs& a, int64_t k, int cb, uint64_t resets, bool open, ScanShared<Shape>* sh)
{
    constexpr int C = Shape::C, Q = Shape::Q, P = Shape::P;
    const int c = threadIdx.x % C, part = threadIdx.x / C;
    float A = 1.0f, B = 0.0f;
    if (a.ticket != nullptr) {
        uint64_t* word = a.words + (k * a.col_blocks + cb) * C + c;
        const bool known = resets != 0 || !open;        // the state after the tile does not depend on what comes before
        if (part == 0) {
#pragma unroll 8
            for (int q = 0; q < Q; ++q) {
                const float qA = sh->A[q][c], qB = sh->B[q][c];
                const bool reset = (resets >> q) & 1;
                B = reset ? qB : fmaf(qA, B, qB);
                A *= qA;
            }
            __hip_atomic_store(word, known ? state_word(B) : pair_word(A, B), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        float v = 0.0f;                                 // the state that reaches the tile
        if (open) {
            const auto look = [&](int64_t p) {
                return p < 0 ? state_word(0.0f)
                             : __hip_atomic_load(a.words + (p * a.col_blocks + cb) * C + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            };
            const auto look_back = [&](int64_t nearest) {   // a window of tiles nearest, nearest - 1, ... into LDS, all ready
                uint64_t seen[kLookAhead];
#pragma unroll
                for (int u = 0; u < kLookAhead; ++u) seen[u] = look(nearest - part * kLookAhead - u);
#pragma unroll
                for (int u = 0; u < kLookAhead; ++u) {
                    while (seen[u] == kNotReady) {      // an older tile: it is running and waits for older ones only
                        __builtin_amdgcn_s_sleep(1);
                        seen[u] = look(nearest - part * kLookAhead - u);
                    }
                    sh->seen[part * kLookAhead + u][c] = seen[u];
                }
                __syncthreads();
            };
            // back, window by window, until there is a state in every column; then forward again from there
            constexpr int W = P * kLookAhead;
            int64_t window = 0;
            for (bool all = false; !all; ++window) {
                look_back(k - 1 - window * W);
                bool found = part != 0;
                for (int i = 0; i < W && !found; ++i) found = is_state(sh->seen[i][c]);
                all = __syncthreads_and(found) != 0;
            }
            for (--window;;) {
                if (part == 0) {
#pragma unroll
                    for (int i = W - 1; i >= 0; --i) {
                        const uint64_t w = sh->seen[i][c];
                        v = is_state(w) ? __uint_as_float((uint32_t)w) : fmaf(__uint_as_float((uint32_t)(w >> 32)), v, __uint_as_float((uint32_t)w));
                    }
                }
                if (window == 0) break;
                __syncthreads();
                look_back(k - 1 - --window * W);
            }
        }
        if (part == 0 && !known)
            __hip_atomic_store(word, state_word(fmaf(A, v, B)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        B = v;
    }
    if (part == 0) {
#pragma unroll 8
        for (int q = 0; q < Q; ++q) {
            const float qA = sh->A[q][c], qB = sh->B[q][c];
            sh->B[q][c] = B;
            B = ((resets >> q) & 1) ? qB : fmaf(qA, B, qB);
        }
    }
    __syncthreads();
}

// The states of empty sequences pass through, and the offsets are looked over: 256 sequences at a time, dealt to the workgroups.
template <class Shape>
__device__ __forceinline__ void empty_sequences(const ScanArgs& a, int64_t k, int cb)
{
    const int64_t cols = (int64_t)a.units * Shape::N;
    const int col = cb * Shape::C + 4 * lane_id();
    for (int64_t s0 = k * kBlock; s0 < a.S; s0 += a.strides * kBlock) {
        const int64_t s = s0 + threadIdx.x;
        bool empty = false;
        if (s < a.S) {
            const int64_t b = a.offsets[s], e = a.offsets[s + 1];
            empty = b == e;
            if (cb == 0 && (b < 0 || b > e || e > a.n || (s == 0 && b != 0) || (s == a.S - 1 && e != a.n))) report(a.status, FS_DEV_BAD_OFFSETS);
        }
        if (a.ends_out == nullptr) continue;
        for (uint64_t left = ballot(empty); left != 0; left &= left - 1) {
            const int64_t at = (s0 + (threadIdx.x & ~(kWave - 1)) + __builtin_ctzll(left)) * cols + col;
            if (4 * lane_id() < Shape::C && col < cols)
                *reinterpret_cast<f32x4*>(a.ends_out + at) = a.ends_in ? *reinterpret_cast<const f32x4*>(a.ends_in + at) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
}

// The workgroup's number: tiles go out in their order.
template <class Shape>
__device__ __forceinline__ uint32_t take_ticket(const ScanArgs& a, ScanShared<Shape>* sh)
{
    if (a.ticket == nullptr) return blockIdx.x;
    if (threadIdx.x == 0) sh->ticket = atomicAdd(a.ticket, 1u);
    __syncthreads();
    return sh->ticket;
}

__device__ __forceinline__ void load_four(const float* p, int64_t at, float* v)
{
    const f32x4 q = *reinterpret_cast<const f32x4*>(p + at);
    v[0] = q[0]; v[1] = q[1]; v[2] = q[2]; v[3] = q[3];
}

template <int N>
__device__ __forceinline__ void load_state(const float* p, int64_t at, float* v)
{
#pragma unroll
    for (int i = 0; i < N; i += 4) load_four(p, at + i, v + i);
}

template <int N>
__device__ __forceinline__ void store_state(float* p, int64_t at, const float* v)
{
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4*>(p + at + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

template <int DT, int G, int R>
__global__ __launch_bounds__(kBlock, 4) void scan_fwd_kernel(ScanArgs a)
{
    using Shape = ScanShape<DT, G, R>;
    constexpr int N = Shape::N;
    __shared__ ScanShared<Shape> sh;
    const uint32_t t = take_ticket(a, &sh);
    const int64_t k = t / (uint32_t)a.col_blocks;
    const int cb = (int)(t % (uint32_t)a.col_blocks);
    if (k < a.tiles) {
        const int lig = threadIdx.x % G, group = threadIdx.x / G;
        const int piece = cb * G + lig;
        const bool in = piece < a.units;
        const int64_t row0 = k * Shape::T, first = row0 + group * R;
        const int64_t cols = (int64_t)a.units * N, col = (int64_t)piece * N;
        u32x4 raw_x[R], raw_g[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            raw_x[r] = raw_g[r] = u32x4{0u, 0u, 0u, 0u};
            if (in && first + r < a.n) {
                raw_g[r] = load_stream(a.gate + (first + r) * a.units + piece);
                raw_x[r] = load_stream(a.x + (first + r) * a.units + piece);
            }
        }
        mark_sequences(a, row0, &sh);
        uint32_t firsts = group_marks<Shape>(sh.firsts, group);
        const uint32_t lasts = group_marks<Shape>(sh.lasts, group);
        float f[R][N], b[R][N];
        float A[N], B[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { A[i] = 1.0f; B[i] = 0.0f; }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[N];
            Piece<DT>::unpack(raw_g[r], f[r]);
            Piece<DT>::unpack(raw_x[r], x);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float o;
                gate_pair(f[r][i], &f[r][i], &o);
                b[r][i] = o * x[i];
            }
            if ((firsts >> r) & 1) {
                if (a.ends_in != nullptr && in) {
                    float h0[N];
                    load_state<N>(a.ends_in, (int64_t)sh.first_of[group * R + r] * cols + col, h0);
#pragma unroll
                    for (int i = 0; i < N; ++i) b[r][i] = fmaf(f[r][i], h0[i], b[r][i]);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) B[i] = 0.0f;                // nothing of the sequence before, a NaN either
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                A[i] *= f[r][i];
                B[i] = fmaf(f[r][i], B[i], b[r][i]);
            }
        }
        store_state<N>(&sh.A[group][0], lig * N, A);
        store_state<N>(&sh.B[group][0], lig * N, B);
        __syncthreads();
        uint64_t resets = 0;
        for (int q = 0; q < Shape::Q; ++q) resets |= (uint64_t)(group_marks<Shape>(sh.firsts, q) != 0) << q;
        const bool open = k > 0 && !(sh.firsts[0] & 1u);
        carry_states<Shape>(a, k, cb, resets, open, &sh);
        float h[N];
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] = sh.B[group][lig * N + i];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if ((firsts >> r) & 1) {
#pragma unroll
                for (int i = 0; i < N; ++i) h[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) h[i] = fmaf(f[r][i], h[i], b[r][i]);
            if (in && first + r < a.n) {
                store_stream(a.h + (first + r) * a.units + piece, Piece<DT>::pack(h));
                if (((lasts >> r) & 1) && a.ends_out != nullptr) store_state<N>(a.ends_out, (int64_t)sh.last_of[group * R + r] * cols + col, h);
            }
        }
    }
    empty_sequences<Shape>(a, k, cb);
}

template <int DT, int G, int R, bool PACKED>
__global__ __launch_bounds__(kBlock, 2) void scan_bwd_kernel(ScanArgs a)
{
    using Shape = ScanShape<DT, G, R>;
    constexpr int N = Shape::N, Q = Shape::Q;
    __shared__ ScanShared<Shape> sh;
    const uint32_t t = take_ticket(a, &sh);
    const int64_t k = t / (uint32_t)a.col_blocks;       // from the batch's end
    const int cb = (int)(t % (uint32_t)a.col_blocks);
    if (k < a.tiles) {
        const int lig = threadIdx.x % G, group = threadIdx.x / G, q = Q - 1 - group;
        const int piece = cb * G + lig;
        const bool in = piece < a.units;
        const int64_t row0 = (a.tiles - 1 - k) * Shape::T, first = row0 + group * R;
        const int64_t cols = (int64_t)a.units * N, col = (int64_t)piece * N;
        u32x4 raw_d[R];
        Saved<DT, PACKED, 0> x[R];
        Saved<DT, PACKED, 1> gate[R];
        Saved<DT, PACKED, 2> before[R];                 // h of the row before
#pragma unroll
        for (int r = 0; r < R; ++r) {
            raw_d[r] = u32x4{0u, 0u, 0u, 0u};
            gate[r].zero();
            x[r].zero();
            before[r].zero();
            if (in && first + r < a.n) {
                gate[r].load(a, first + r, piece);
                raw_d[r] = load_stream(a.dh + (first + r) * a.units + piece);
                x[r].load(a, first + r, piece);
                if (first + r > 0) before[r].load(a, first + r - 1, piece);
            }
        }
        mark_sequences(a, row0, &sh);
        const uint32_t firsts = group_marks<Shape>(sh.firsts, group), lasts = group_marks<Shape>(sh.lasts, group);
        float f[R][N], o[R][N], d[R][N];
        float A[N], B[N];
#pragma unroll
        for (int i = 0; i < N; ++i) { A[i] = 1.0f; B[i] = 0.0f; }
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            gate[r].values(f[r]);
            Piece<DT>::unpack(raw_d[r], d[r]);
#pragma unroll
            for (int i = 0; i < N; ++i) gate_pair(f[r][i], &f[r][i], &o[r][i]);
            if ((lasts >> r) & 1) {
                if (a.ends_in != nullptr && in) {
                    float end[N];
                    load_state<N>(a.ends_in, (int64_t)sh.last_of[group * R + r] * cols + col, end);
#pragma unroll
                    for (int i = 0; i < N; ++i) d[r][i] += end[i];
                }
#pragma unroll
                for (int i = 0; i < N; ++i) B[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                A[i] *= f[r][i];
                B[i] = f[r][i] * (d[r][i] + B[i]);
            }
        }
        store_state<N>(&sh.A[q][0], lig * N, A);
        store_state<N>(&sh.B[q][0], lig * N, B);
        __syncthreads();
        uint64_t resets = 0;
        for (int j = 0; j < Q; ++j) resets |= (uint64_t)(group_marks<Shape>(sh.lasts, Q - 1 - j) != 0) << j;
        const bool open = k > 0 && !(sh.lasts[Shape::T / 32 - 1] >> 31);
        carry_states<Shape>(a, k, cb, resets, open, &sh);
        float U[N];
#pragma unroll
        for (int i = 0; i < N; ++i) U[i] = sh.B[q][lig * N + i];
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            if ((lasts >> r) & 1) {
#pragma unroll
                for (int i = 0; i < N; ++i) U[i] = 0.0f;
            }
            float xv[N], hb[N], dx[N], dg[N];
            x[r].values(xv);
            before[r].values(hb);
            if ((firsts >> r) & 1) {
#pragma unroll
                for (int i = 0; i < N; ++i) hb[i] = 0.0f;
                if (a.h0 != nullptr && in) load_state<N>(a.h0, (int64_t)sh.first_of[group * R + r] * cols + col, hb);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float Gi = d[r][i] + U[i];
                dx[i] = o[r][i] * Gi;
                dg[i] = dx[i] * f[r][i] * (hb[i] - xv[i]);
                U[i] = f[r][i] * Gi;
            }
            if (in && first + r < a.n) {
                store_stream(a.dx + (first + r) * a.units + piece, Piece<DT>::pack(dx));
                store_stream(a.dgate + (first + r) * a.units + piece, Piece<DT>::pack(dg));
                if (((firsts >> r) & 1) && a.ends_out != nullptr) store_state<N>(a.ends_out, (int64_t)sh.first_of[group * R + r] * cols + col, U);
            }
        }
    }
    empty_sequences<Shape>(a, k, cb);
}

// All words not ready, no ticket taken.
__global__ __launch_bounds__(kBlock) void scan_clear_kernel(u32x4* __restrict__ words, int64_t pieces, uint32_t* __restrict__ ticket)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < pieces) words[i] = u32x4{~0u, ~0u, ~0u, ~0u};
    if (i == 0) *ticket = 0u;
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

// Lanes of a group: the whole row up to 16 pieces (in a power of two), longer rows in blocks of 16 or 8 pieces, whichever
// leaves fewer lanes idle.
int scan_lanes(int units)
{
    if (units <= 4) return 4;
    if (units <= 8) return 8;
    return (units + 15) / 16 * 16 <= (units + 7) / 8 * 8 ? 16 : 8;
}

// Values of a lane: R rows of a 16-byte piece.
constexpr int kFwdValues = 32, kBwdValues = 32;

// Everything that follows from the sizes; *a gets them, `words` the workspace's places.
fs_status plan_scan(int64_t n, int32_t D, fs_dtype dtype, int32_t T, int32_t B, int values, Carver* ws, ScanArgs* a, int* lanes)
{
    const fs_status st = check_seq_rows(n, D, dtype, &a->units);
    if (st != FS_OK) return st;
    if (T < 1 || B < 1 || (int64_t)T * B >= (1LL << 31)) return FS_ERR_SIZE;
    a->S = (int64_t)T * B;
    a->n = n;
    a->nb = (int)pack_blocks(D);
    const int N = dtype == FS_F32 ? 4 : 8;
    *lanes = scan_lanes(a->units);
    const int64_t rows = (int64_t)(kBlock / *lanes) * (values / N);
    a->col_blocks = (a->units + *lanes - 1) / *lanes;
    a->tiles = (n + rows - 1) / rows;
    const int64_t passes = (a->S + kBlock - 1) / kBlock;            // workgroups that the sequences alone would keep busy
    a->strides = a->tiles > passes ? a->tiles : passes < 1024 ? passes : a->tiles > 1024 ? a->tiles : 1024;
    if (a->strides * a->col_blocks > 0x7FFFFFFF) return FS_ERR_SIZE;
    if (a->tiles > 1) {
        a->words = ws->take<uint64_t>((size_t)a->tiles * (size_t)a->col_blocks * (size_t)(*lanes * N));
        a->ticket = ws->take<uint32_t>(1);
    }
    return FS_OK;
}

fs_status clear_words(const ScanArgs& a, int columns, hipStream_t s)
{
    if (a.tiles <= 1) return FS_OK;
    const int64_t pieces = a.tiles * a.col_blocks * columns / 2;
    const int64_t grid = (pieces + kBlock - 1) / kBlock;
    if (grid > 0x7FFFFFFF) return FS_ERR_SIZE;
    FS_LAUNCH("scan_clear", scan_clear_kernel, dim3((unsigned)grid), dim3(kBlock), s, reinterpret_cast<u32x4*>(a.words), pieces, a.ticket);
    return FS_OK;
}

#define FS_DISPATCH_LANES(lanes, CALL)                                                  \
    switch (lanes) {                                                                    \
        case 4: CALL(4); break;                                                         \
        case 8: CALL(8); break;                                                         \
        default: CALL(16); break;                                                       \
    }

template <int DT>
fs_status scan_fwd_launch(const ScanArgs& a, int lanes, hipStream_t s)
{
    const dim3 grid((unsigned)(a.strides * a.col_blocks));
#define CALL(G) FS_LAUNCH("scan_fwd", (scan_fwd_kernel<DT, G, kFwdValues / Piece<DT>::N>), grid, dim3(kBlock), s, a)
    FS_DISPATCH_LANES(lanes, CALL)
#undef CALL
    return FS_OK;
}

template <int DT, bool PACKED>
fs_status scan_bwd_launch(const ScanArgs& a, int lanes, hipStream_t s)
{
    const dim3 grid((unsigned)(a.strides * a.col_blocks));
#define CALL(G) FS_LAUNCH("scan_bwd", (scan_bwd_kernel<DT, G, kBwdValues / Piece<DT>::N, PACKED>), grid, dim3(kBlock), s, a)
    FS_DISPATCH_LANES(lanes, CALL)
#undef CALL
    return FS_OK;
}

fs_status scan_bwd(ScanArgs a, bool packed, int32_t D, fs_dtype dtype, int32_t T, int32_t B, void* workspace,
                   size_t* workspace_bytes, hipStream_t s)
{
    if (!workspace_bytes) return FS_ERR_NULL;
    Carver ws(workspace);
    int lanes = 0;
    fs_status st = plan_scan(a.n, D, dtype, T, B, kBwdValues, &ws, &a, &lanes);
    if (st != FS_OK) return st;
    if (!workspace) { *workspace_bytes = ws.used; return FS_OK; }
    if (*workspace_bytes < ws.used || misaligned(workspace, 256)) return FS_ERR_WORKSPACE;
    if (!a.offsets) return FS_ERR_NULL;
    if (a.n > 0) {
        if (!a.dh || !a.dx || !a.dgate) return FS_ERR_NULL;
        if (!packed && (!a.x || !a.gate || !a.h_in)) return FS_ERR_NULL;
        for (int i = 0; packed && i < 3; ++i)
            if (!a.codes[i] || !a.exps[i]) return FS_ERR_NULL;
    }
    if (misaligned(a.dh, 16) || misaligned(a.x, 16) || misaligned(a.gate, 16) || misaligned(a.h_in, 16) || misaligned(a.dx, 16) ||
        misaligned(a.dgate, 16) || misaligned(a.codes[0], codes_alignment(dtype)) || misaligned(a.codes[1], codes_alignment(dtype)) ||
        misaligned(a.codes[2], codes_alignment(dtype)) || misaligned(a.h0, 16) || misaligned(a.ends_in, 16) ||
        misaligned(a.ends_out, 16) || misaligned(a.offsets, 8))
        return FS_ERR_ALIGN;
    st = clear_words(a, lanes * (dtype == FS_F32 ? 4 : 8), s);
    if (st != FS_OK) return st;
    if (packed) {
#define CALL(DT) st = scan_bwd_launch<DT, true>(a, lanes, s)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    } else {
#define CALL(DT) st = scan_bwd_launch<DT, false>(a, lanes, s)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    }
    return st;
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
    Carver ws(workspace);
    int lanes = 0;
    fs_status st = plan_scan(n, D, dtype, T, B, kFwdValues, &ws, &a, &lanes);
    if (st != FS_OK) return st;
    if (!workspace) { *workspace_bytes = ws.used; return FS_OK; }
    if (*workspace_bytes < ws.used || misaligned(workspace, 256)) return FS_ERR_WORKSPACE;
    if (!offsets || (n > 0 && (!x || !gate || !h))) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(gate, 16) || misaligned(h, 16) || misaligned(h0, 16) || misaligned(h_last, 16) || misaligned(offsets, 8))
        return FS_ERR_ALIGN;
    a.x = static_cast<const u32x4*>(x); a.gate = static_cast<const u32x4*>(gate);
    a.offsets = offsets; a.ends_in = h0; a.h = static_cast<u32x4*>(h); a.ends_out = h_last; a.status = dev_status;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    st = clear_words(a, lanes * (dtype == FS_F32 ? 4 : 8), hs);
    if (st != FS_OK) return st;
#define CALL(DT) return scan_fwd_launch<DT>(a, lanes, hs)
    FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
}

extern "C" fs_status fs_seq_scan_bwd(
    const void* dh, const float* dh_last, const void* x, const void* gate, const void* h,
    int64_t n, int32_t D, fs_dtype dtype, const int64_t* offsets, int32_t T, int32_t B, const float* h0,
    void* dx, void* dgate, float* dh0,
    void* workspace, size_t* workspace_bytes, void* stream, int32_t* dev_status)
{
    using namespace fs;
    ScanArgs a = {};
    a.dh = static_cast<const u32x4*>(dh); a.ends_in = dh_last; a.n = n;
    a.x = static_cast<const u32x4*>(x); a.gate = static_cast<const u32x4*>(gate); a.h_in = static_cast<const u32x4*>(h);
    a.offsets = offsets; a.h0 = h0;
    a.dx = static_cast<u32x4*>(dx); a.dgate = static_cast<u32x4*>(dgate); a.ends_out = dh0; a.status = dev_status;
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
    a.dh = static_cast<const u32x4*>(dh); a.ends_in = dh_last; a.n = n;
    a.codes[0] = reinterpret_cast<const uint32_t*>(x_codes); a.exps[0] = x_exps;
    a.codes[1] = reinterpret_cast<const uint32_t*>(gate_codes); a.exps[1] = gate_exps;
    a.codes[2] = reinterpret_cast<const uint32_t*>(h_codes); a.exps[2] = h_exps;
    a.offsets = offsets; a.h0 = h0;
    a.dx = static_cast<u32x4*>(dx); a.dgate = static_cast<u32x4*>(dgate); a.ends_out = dh0; a.status = dev_status;
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
