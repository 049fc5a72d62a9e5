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
//   a thread a column folds the groups of the workgroup and publishes the tile's (A, B), or the state after it where a
//   sequence begins in the tile, and finds the state that reaches the tile from what the tiles before have published;
//   the groups go over their registers a second time, from the state that reaches them, and write.
// Tiles are handed out in their order by a counter, so the tiles that a workgroup waits for are running or done, and every
// tile publishes whatever the data: every wait ends.  A published pair is one 8-byte word that is its own flag (relaxed
// atomics at the scope of the GPU, nothing else is passed on), cleared by a launch in front.
//
// Measured (us, and the rate of what has to be read and written; a large copy runs at 6.2 TB/s, torch's own at 5.1): 4.2 M rows of 128
// in 32768 sequences, forward fp16 544 (5.9 TB/s), backward bf16 1098 (5.9); 80.5 k rows of 128 bf16 in 692 sequences 26 (2.4),
// which is the time of one tile from its number to its last store; 284 k rows of 64 fp32 in three sequences 63 (3.5): 1111 tiles
// for 768 places; 556 k rows of 256 fp16 backward from checkpoints 310 (4.2).  The traffic of the first two is the least possible
// within 4 % (the words; backward h of the row before every tile too); rows of 19 pieces and more that are no multiple of 8 have
// shorter tiles, whose words are up to 7.3 % of x forward and 14.5 % backward.  One workgroup a sequence instead took 1041, 1547, 559,
// 47950 and 5198.
#include <type_traits>

#include "pack8.h"
#include "seq_marks.h"
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
    int col_blocks;                  // blocks of `lanes` pieces of columns
    int lanes, groups;               // of a workgroup
    int by_lanes, by_columns;        // t / lanes and t / (columns of a workgroup) as (t * this) >> 16, t <= kBlock
    uint64_t* words;                 // [tiles + spans of kSpan tiles][col_blocks][columns of a workgroup]
    int32_t* tile_seq;               // [tiles + 1]: the sequence that the row before the tile is in
    uint32_t* ticket;                // null: one tile, nothing to wait for
};

// f and 1 - f of a gate, each to the precision of e^-gate (1 - f is not taken from f, which is 1 for large gates).  That is the
// exponential's own and up to |gate| roundings: its argument is a rounded product, and an exponent off by d takes e^d.
__device__ __forceinline__ void gate_pair(float gate, float* f, float* o)
{
    const float e = __builtin_amdgcn_exp2f(gate * -1.44269504f);
    *f = __builtin_amdgcn_rcpf(1.0f + e);
    *o = e > 1e30f ? 1.0f : e * *f;                     // e = infinity (a shut gate): f = 0, 1 - f = 1
}

// The same number, of which the compiler does not know that it has it already: it is worked out again where it is needed
// instead of kept in a register over the whole kernel (or, with no register left, in scratch memory, whose loads wait for
// the stores in flight: 9 % of the forward pass).
__device__ __forceinline__ uint32_t again(uint32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// p[at] by an offset of 32 bits in bytes (kMostPieces keeps them in range): a scalar base and one vector register.
template <typename T>
__device__ __forceinline__ T* piece_at(T* p, uint32_t at)
{
    using Byte = typename std::conditional<std::is_const<T>::value, const char, char>::type;
    return reinterpret_cast<T*>(reinterpret_cast<Byte*>(p) + (uint32_t)(at * sizeof(T)));
}

// Rows of whole cache lines are read once by one instruction each and streamed past the caches; of other rows a line belongs
// to two, and to instructions apart in time, so they go through the caches (us, streamed : cached: 4.2 M rows of 256 bytes
// forward 547 : 588, backward 1102 : 1192; of 272 bytes 725 : 677 and 1508 : 1387; of 48 bytes backward 538 : 283).
template <bool STREAM, typename T>
__device__ __forceinline__ T load_rows(const T* p)
{
    if constexpr (STREAM) return load_stream(p);
    else return *p;
}
template <bool STREAM, typename T>
__device__ __forceinline__ void store_rows(T* p, T v)
{
    if constexpr (STREAM) store_stream(p, v);
    else *p = v;
}

// One of the three saved inputs of the backward pass (0: x, 1: gate, 2: h) at a row's piece, from the rows or from their
// checkpoint.  base: a row, the same for the whole workgroup; at: row - base in pieces, plus the piece; block: row - base in
// blocks of columns, plus the block.
template <int DT, bool PACKED, int WHICH, bool STREAM>
struct Saved {
    u32x4 raw;                       // PACKED: the codes in [0], [1]; the exponent in [2]
    __device__ __forceinline__ void load(const ScanArgs& a, int64_t base, uint32_t at, uint32_t block)
    {
        constexpr int N = Piece<DT>::N;
        if constexpr (PACKED) {
            if constexpr (N == 8) {
                const u32x2 c = load_rows<STREAM>(piece_at(reinterpret_cast<const u32x2*>(a.codes[WHICH]) + base * a.units, at));
                raw[0] = c[0]; raw[1] = c[1];
            } else {
                raw[0] = load_rows<STREAM>(piece_at(a.codes[WHICH] + base * a.units, at));
            }
            raw[2] = (a.exps[WHICH] + base * a.nb)[block];
        } else {
            const u32x4* from = WHICH == 0 ? a.x : WHICH == 1 ? a.gate : a.h_in;
            raw = load_rows<STREAM>(piece_at(from + base * a.units, at));
        }
    }
    __device__ __forceinline__ void values(float* v) const
    {
        if constexpr (PACKED) {
            unpack_piece<Piece<DT>::N>(raw[0], raw[1], (int)raw[2], v);
        } else {
            Piece<DT>::unpack(raw, v);
        }
    }
};

// Most groups of a workgroup: all its threads have one from 16-bit rows of two pieces on (against 64 groups, 4.2 M rows of 8, 16 and 24
// bf16, us: forward 101 : 128, 117 : 139, 173 : 173).  fp32 groups have twice the rows: their marks' LDS would cost a workgroup a CU
// (rows of 12: 170 : 162).  Backward 154 : 221, 204 : 250, 283 : 292.
constexpr __host__ __device__ int most_groups(int N) { return N == 8 ? 128 : 64; }

// A workgroup's tile: G lanes a row and Q groups of R rows each.  G_ = 0: G is an argument.
template <int DT, int G_, int R_>
struct ScanShape {
    static constexpr int N = Piece<DT>::N, R = R_;
    static constexpr int kMostGroups = most_groups(N), kMostRows = kMostGroups * R, kMostCols = G_ > 0 ? G_ * N : kBlock;
    int G, Q;
    int C;                           // columns of the workgroup, at most kBlock
    int P;                           // threads a column
    int T;                           // rows
    int by_lanes, by_columns;        // (scalars all; the thread's places below are worked out where they are needed)
    static_assert(32 % R == 0, "");
    __device__ __forceinline__ explicit ScanShape(const ScanArgs& a)
    {
        if constexpr (G_ > 0) {
            G = G_; Q = kBlock / G_; C = G_ * N; P = kBlock / (G_ * N);
        } else {
            G = a.lanes; Q = a.groups; C = G * N; P = (kBlock * a.by_columns) >> 16;
            by_lanes = a.by_lanes; by_columns = a.by_columns;
        }
        T = Q * R;
    }
    // the thread's group (Q or more: none) and lane in it
    __device__ __forceinline__ int group() const
    {
        if constexpr (G_ > 0) return (int)(again(threadIdx.x) / (uint32_t)G_);
        return (int)(again(threadIdx.x) * (uint32_t)by_lanes) >> 16;
    }
    __device__ __forceinline__ int lane() const { return (int)threadIdx.x - group() * G; }
    // which of the threads of its column it is (P: none), and the column
    __device__ __forceinline__ int part() const
    {
        if constexpr (G_ > 0) return (int)(again(threadIdx.x) / (uint32_t)(G_ * N));
        return (int)(again(threadIdx.x) * (uint32_t)by_columns) >> 16;
    }
    __device__ __forceinline__ int col() const { return (int)threadIdx.x - part() * C; }
};

constexpr int kSpan = 8;                                // tiles of a span (see carry_states)
constexpr int kLookAhead = 4;                           // spans that a thread looks back over at once

template <class Shape>
struct ScanShared {
    float A[kBlock * Shape::N], B[kBlock * Shape::N];   // [Q][C] in the order of the walk: the groups' pairs, then what lies before each
    uint64_t tiles[(kSpan - 1) * Shape::kMostCols];     // [kSpan - 1][C]: the words of the span's tiles before
    uint64_t spans[kBlock * kLookAhead];                // [P * kLookAhead][C]: the words of the spans looked back over
    float reaches[kBlock];                              // [C]: the state that reaches the tile
    uint32_t firsts[Shape::kMostRows / 32], lasts[Shape::kMostRows / 32];       // rows of the tile where a sequence begins, ends
    int32_t first_of[Shape::kMostRows], last_of[Shape::kMostRows];              // ... and which one
    uint32_t ticket;
};

// The bounds of the 64 sequences from the one on that the row before the tile is in, one a lane of every wave.  Loaded in
// front of the rows: loads come back in their order, and behind the rows the marks would wait for all of them.
struct Bounds {
    int64_t s, b, e;
    __device__ __forceinline__ Bounds(const ScanArgs& a, int s0)
    {
        s = (int64_t)(s0 < 0 ? 0 : s0) + lane_id();     // (s0 is at most S - 1)
        b = e = a.n;
        if (s < a.S) { b = a.offsets[s]; e = a.offsets[s + 1]; }
    }
};

template <class Shape>
__device__ __forceinline__ void mark_first(ScanShared<Shape>* sh, int row, int32_t s)
{
    atomicOr(&sh->firsts[row >> 5], 1u << (row & 31));
    sh->first_of[row] = s;
}

template <class Shape>
__device__ __forceinline__ void mark_last(ScanShared<Shape>* sh, int row, int32_t s)
{
    atomicOr(&sh->lasts[row >> 5], 1u << (row & 31));
    sh->last_of[row] = s;
}

// Sequence s with rows b .. e - 1, of a tile of `rows` rows from row0 on.
template <class Shape>
__device__ __forceinline__ void mark_sequence(ScanShared<Shape>* sh, int64_t row0, int rows, int64_t s, int64_t b, int64_t e)
{
    if (b >= e) return;
    b -= row0;
    e -= row0;
    if (b >= 0 && b < rows) mark_first(sh, (int)b, (int32_t)s);
    if (e > 0 && e <= rows) mark_last(sh, (int)e - 1, (int32_t)s);
}

// Marks the first and last rows of the sequences in tile `number`, from row0 on; every thread calls it.  The first wave takes
// the 64 sequences of `mine`, which mostly is all; where there are more, all threads take the others, and where those are very
// many, each row finds its own: what a tile takes does not grow with the sequences without rows in it.  Contains barriers.
// With bad offsets the marks are arbitrary but inside the tile.
template <class Shape>
__device__ __forceinline__ void mark_sequences(const ScanArgs& a, const Shape& tile, const int32_t* tile_seq, int64_t number, int64_t row0,
                                               const Bounds& mine, ScanShared<Shape>* sh)
{
    const int rows = a.n - row0 < tile.T ? (int)(a.n - row0) : tile.T;
    if (wave_id() == 0) {
        const int lane = lane_id();
        if (lane < Shape::kMostRows / 32) sh->firsts[lane] = sh->lasts[lane] = 0u;
        mark_sequence(sh, row0, rows, mine.s, mine.b, mine.e);
    }
    const bool more = (ballot(mine.b - row0 < rows && mine.s < a.S) >> (kWave - 1)) != 0;     // the last lane's begins in the tile or before it
    __syncthreads();
    if (!more) return;
    const uint32_t first = tile_seq == nullptr ? 0u : (uint32_t)tile_seq[number];
    const uint32_t last = tile_seq == nullptr ? (uint32_t)(a.S - 1) : (uint32_t)tile_seq[number + 1];      // the last that begins in the tile
    const uint32_t count = last < first ? 0u : last - first + 1u;                                          // (0: bad offsets)
    if (mark_rounds(count) <= kMostMarkRounds) {
        for (int64_t s = (int64_t)first + kWave + threadIdx.x; s <= last; s += kBlock) mark_sequence(sh, row0, rows, s, a.offsets[s], a.offsets[s + 1]);
    } else {
        for (int row = threadIdx.x; row < rows; row += kBlock) {
            const int64_t at = row0 + row;
            const uint32_t s = sequence_of_row(first, count, at, [&](uint32_t i) { return a.offsets[i]; });
            if (a.offsets[s] == at) mark_first(sh, row, (int32_t)s);
            if (a.offsets[s + 1] == at + 1) mark_last(sh, row, (int32_t)s);
        }
    }
    __syncthreads();
}

// Marks of the thread's group, bit r for row r.
template <class Shape>
__device__ __forceinline__ uint32_t group_marks(const Shape& tile, const uint32_t* marks)
{
    const int group = tile.group(), at = group * Shape::R;
    return group < tile.Q ? (marks[at >> 5] >> (at & 31)) & (uint32_t)((1ull << Shape::R) - 1ull) : 0u;
}

template <class Shape>
__device__ __forceinline__ bool any_marks(const Shape& tile, const uint32_t* marks)
{
    uint32_t any = 0;
    for (int w = 0; w * 32 < tile.T; ++w) any |= marks[w];
    return __builtin_amdgcn_readfirstlane((int)any) != 0;
}

constexpr uint64_t kNotReady = ~0ull;
constexpr uint32_t kIsState = 0xFF800000u;              // in place of A (which is not negative): B is the state after the tile

__device__ __forceinline__ uint64_t pair_word(float A, float B)
{
    return ((uint64_t)(A != A ? 0x7FC00000u : __float_as_uint(A)) << 32) | __float_as_uint(B);   // no NaN looks like kNotReady
}

__device__ __forceinline__ bool is_state(uint64_t word) { return (uint32_t)(word >> 32) == kIsState; }

__device__ __forceinline__ uint64_t state_word(float v) { return ((uint64_t)kIsState << 32) | __float_as_uint(v); }

// A < 0 in a pair stands for a stretch in which a sequence begins: B is the state after it, whatever comes before.
__device__ __forceinline__ bool begins_in(float A) { return (int32_t)__float_as_uint(A) < 0; }
constexpr float kBegins = -1.0f;

// The state after the stretch (A, B) where v is the one before it.  (A NaN's sign may be set; its B is a NaN too.)
__device__ __forceinline__ float after(float A, float B, float v) { return begins_in(A) ? B : fmaf(A, v, B); }

// A word that is ready, waiting for it: an older workgroup's, which is running and waits for older ones only.
__device__ __forceinline__ uint64_t ready_word(const uint64_t* at)
{
    uint64_t w;
    while ((w = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) == kNotReady) __builtin_amdgcn_s_sleep(1);
    return w;
}

__device__ __forceinline__ void publish(uint64_t* at, uint64_t w) { __hip_atomic_store(at, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The state after the stretch of a word where v is the one before it.
__device__ __forceinline__ float after_word(uint64_t w, float v)
{
    const float B = __uint_as_float((uint32_t)w);
    return is_state(w) ? B : fmaf(__uint_as_float((uint32_t)(w >> 32)), v, B);
}

// From the groups' pairs in sh->A and sh->B to the pair of all that lies before each group in the tile, there, and the states
// that reach the tile, in sh->reaches.  k: the tile's number in the order of the walk; known: a sequence begins in the tile
// or with it, so the state after it does not depend on what comes before; open: the tile's first row goes on with a
// sequence of the tile before.  Every thread calls it; contains barriers.
//
// A tile's word is the state after it if that is known, else its pair.  An open tile takes the word of the tile before, which
// in a batch of short sequences mostly is a state; else those of its whole span of kSpan tiles, and where no state is among
// them either the words of the spans before, back to one with a state, and goes forward again from there.  The last tile of
// a span publishes the span's word: the state after it if that is known, else its pair, and the state once it is there.  So
// every state is the same chain of A v + B from the sequence's beginning, over whole spans and then over tiles, whoever works
// it out and however far the others are: the same bits on every run.  (Without spans, tile by tile: sequences of 20 k rows took 1.8
// times as long as short ones, 2 M rows of 128 bf16 526 us against 286.)
template <class Shape>
__device__ __forceinline__ void carry_states(const ScanArgs& a, const Shape& tile, int64_t k, int cb, bool known, bool open, ScanShared<Shape>* sh)
{
    const int C = tile.C, c = tile.col(), part = tile.part();
    const int64_t stride = (int64_t)a.col_blocks * C;   // words of a tile or a span
    uint64_t* const tiles = a.words + cb * C + c;
    const int64_t span = k / kSpan;
    const int in_span = (int)(k % kSpan);
    uint64_t* const spans = tiles + a.tiles * stride;
    const bool ends_span = in_span == kSpan - 1;
    float A = 1.0f, B = 0.0f;
    if (part == 0) {
#pragma unroll 8
        for (int q = 0; q < tile.Q; ++q) {
            const float qA = sh->A[q * C + c], qB = sh->B[q * C + c];
            sh->A[q * C + c] = A;
            sh->B[q * C + c] = B;
            B = after(qA, qB, B);
            A = begins_in(qA) ? kBegins : A * qA;
        }
        if (a.ticket != nullptr) {
            publish(tiles + k * stride, known ? state_word(B) : pair_word(A, B));
            if (known && ends_span) publish(spans + span * stride, state_word(B));
        }
    }
    float v = 0.0f;                                     // the state that reaches the tile
    if (open) {
        bool found = part != 0;
        bool all = false;
        if (in_span > 0) {
            // (words are states or pairs by the data alone, and the same in all columns but for a pair's values)
            if (part == 0) {
                const uint64_t w = ready_word(tiles + (k - 1) * stride);
                sh->tiles[(in_span - 1) * C + c] = w;
                found = is_state(w);
                v = after_word(w, 0.0f);
            }
            all = __syncthreads_and(found) != 0;
            if (!all) {
                for (int j = part; j < in_span - 1; j += tile.P)
                    if (part < tile.P) sh->tiles[j * C + c] = ready_word(tiles + (k - in_span + j) * stride);
                __syncthreads();
                if (part == 0) {
                    v = 0.0f;
                    for (int j = 0; j < in_span; ++j) {
                        const uint64_t w = sh->tiles[j * C + c];
                        found = found || is_state(w);
                        v = after_word(w, v);
                    }
                }
                all = __syncthreads_and(found) != 0;
            }
        }
        if (part == 0 && !known && ends_span && all) publish(spans + span * stride, state_word(fmaf(A, v, B)));
        if (!all) {
            float span_A = 1.0f, span_B = 0.0f;         // the tiles of the span before this one as a pair
            if (part == 0) {
                for (int j = 0; j < in_span; ++j) {
                    const uint64_t w = sh->tiles[j * C + c];
                    span_B = after_word(w, span_B);
                    span_A *= __uint_as_float((uint32_t)(w >> 32));
                }
                if (!known && ends_span) {
                    span_B = fmaf(A, span_B, B);
                    span_A *= A;
                    publish(spans + span * stride, pair_word(span_A, span_B));
                }
            }
            // back over the spans, first one and then kLookAhead a thread at once, until there is a state in every column
            int64_t window = 0;
            bool back = true;
            for (;;) {
                const int ahead = window == 0 ? 1 : kLookAhead, threads = window == 0 ? 1 : tile.P;
                const int W = ahead * threads;
                const int64_t nearest = window == 0 ? span - 1 : span - 2 - (window - 1) * W;
                if (part < threads) {
                    uint64_t w[kLookAhead];
#pragma unroll
                    for (int u = 0; u < kLookAhead; ++u) {
                        const int64_t p = nearest - part * ahead - u;
                        if (u < ahead) w[u] = p < 0 ? state_word(0.0f) : __hip_atomic_load(spans + p * stride, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
#pragma unroll
                    for (int u = 0; u < kLookAhead; ++u) {
                        if (u >= ahead) continue;
                        if (w[u] == kNotReady) w[u] = ready_word(spans + (nearest - part * ahead - u) * stride);
                        sh->spans[(part * ahead + u) * C + c] = w[u];
                    }
                }
                __syncthreads();
                if (back) {
                    found = part != 0;
                    for (int i = 0; i < W && !found; ++i) found = is_state(sh->spans[i * C + c]);
                    if (__syncthreads_and(found) == 0) {
                        ++window;
                        continue;
                    }
                    back = false;
                    v = 0.0f;
                }
                if (part == 0) {
#pragma unroll 4
                    for (int i = W - 1; i >= 0; --i) v = after_word(sh->spans[i * C + c], v);
                }
                if (window == 0) break;
                --window;
                __syncthreads();
            }
            if (part == 0) {
                if (!known && ends_span) publish(spans + span * stride, state_word(fmaf(span_A, v, span_B)));
                for (int j = 0; j < in_span; ++j) v = after_word(sh->tiles[j * C + c], v);
            }
        }
    }
    if (part == 0) sh->reaches[c] = v;
    __syncthreads();
}

// The states that reach the thread's group, q-th in the order of the walk.
template <class Shape>
__device__ __forceinline__ void group_states(const Shape& tile, int q, const ScanShared<Shape>& sh, float* v)
{
    constexpr int N = Shape::N;
    const int c = tile.lane() * N, at = (tile.group() < tile.Q ? q : 0) * tile.C + c;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = after(sh.A[at + i], sh.B[at + i], sh.reaches[c + i]);
}

// The thread's pair into its place.
template <class Shape>
__device__ __forceinline__ void store_pair(const Shape& tile, int q, bool begins, const float* A, const float* B, ScanShared<Shape>* sh)
{
    constexpr int N = Shape::N;
    if (tile.group() >= tile.Q) return;
    const int at = q * tile.C + tile.lane() * N;
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        *reinterpret_cast<f32x4*>(&sh->A[at + i]) = begins ? f32x4{kBegins, kBegins, kBegins, kBegins} : f32x4{A[i], A[i + 1], A[i + 2], A[i + 3]};
        *reinterpret_cast<f32x4*>(&sh->B[at + i]) = f32x4{B[i], B[i + 1], B[i + 2], B[i + 3]};
    }
}

// The states of empty sequences pass through, and the offsets are looked over: 256 sequences at a time, dealt to the workgroups.
template <class Shape>
__device__ __forceinline__ void empty_sequences(const ScanArgs& a, const Shape& tile, int64_t k, int cb)
{
    const int64_t cols = (int64_t)a.units * Shape::N;
    const int col = cb * tile.C + 4 * lane_id();
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
            if (4 * lane_id() < tile.C && col < cols)
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
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)sh->ticket);       // scalar, and so are the addresses made of it
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

// Where a lane's rows lie, as 32-bit offsets from the tile's first row.  Rows past n and pieces past the row's end are
// replaced by ones that are there: loads without a predicate go out one after the other, predicated ones wait for each
// other.  What is computed from the replacements is not stored and reaches no row that is.
template <class Shape>
struct Place {
    int piece, rows;                 // rows: of the group's R, those before n (none: not positive)
    uint32_t row_at;                 // the group's first row
    bool in;                         // the piece is in the row
    int64_t row0;
    uint32_t units, own, first;      // in pieces; own: the piece, or one that is there; first: the group's first row's
    __device__ __forceinline__ Place(const ScanArgs& a, const Shape& tile, int64_t number, int cb)
    {
        piece = cb * tile.G + tile.lane();
        in = piece < a.units;
        row0 = number * tile.T;
        row_at = (uint32_t)(tile.group() * Shape::R);
        const int64_t left = a.n - row0;
        rows = (left < tile.T ? (int)left : tile.T) - (int)row_at;
        units = (uint32_t)a.units;
        own = in ? (uint32_t)piece : units - 1u;
        first = row_at * units + own;
    }
    __device__ __forceinline__ uint32_t at(int r) const { return r < rows ? first + r * units : own; }
    __device__ __forceinline__ uint32_t row(int r) const { return r < rows ? row_at + r : 0u; }
    __device__ __forceinline__ bool stored(int r) const { return in && r < rows; }
};

// The lane's columns in the states of sequence `which[row]` of the tile's row r of the thread's group; -1: it has none.
template <class Shape>
__device__ __forceinline__ int64_t state_at(const ScanArgs& a, const Shape& tile, int cb, const int32_t* which, int r)
{
    const int group = tile.group(), piece = cb * tile.G + (int)threadIdx.x - group * tile.G;
    return piece < a.units ? ((int64_t)which[group * Shape::R + r] * a.units + piece) * Shape::N : -1;
}

template <int DT, int G, int R>
__global__ __launch_bounds__(kBlock, 3) void scan_fwd_kernel(ScanArgs a, const int32_t* __restrict__ tile_seq)
{
    using Shape = ScanShape<DT, G, R>;
    constexpr int N = Shape::N;
    __shared__ ScanShared<Shape> sh;
    const Shape tile(a);
    const uint32_t t = take_ticket(a, &sh);
    const int64_t k = t / (uint32_t)a.col_blocks;
    const int cb = (int)(t % (uint32_t)a.col_blocks);
    if (k < a.tiles) {
        const Place<Shape> p(a, tile, k, cb);
        const Bounds bounds(a, tile_seq == nullptr ? 0 : tile_seq[k]);          // (in every wave: without a branch it goes out first)
        const u32x4* from_x = a.x + p.row0 * a.units;
        const u32x4* from_g = a.gate + p.row0 * a.units;
        u32x4 raw_x[R], raw_g[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            raw_g[r] = load_rows<(G > 0)>(piece_at(from_g, p.at(r)));
            raw_x[r] = load_rows<(G > 0)>(piece_at(from_x, p.at(r)));
        }
        mark_sequences(a, tile, tile_seq, k, p.row0, bounds, &sh);
        const uint32_t firsts = group_marks(tile, sh.firsts);
        const uint32_t lasts = group_marks(tile, sh.lasts);
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
            const bool begins = (firsts >> r) & 1;
            if (ballot(begins) != 0) {                  // (few rows: a branch of the wave, not a selection a value)
                if (begins && a.ends_in != nullptr) {
                    const int64_t at = state_at(a, tile, cb, sh.first_of, r);
                    if (at >= 0) {
                        float h0[N];
                        load_state<N>(a.ends_in, at, h0);
#pragma unroll
                        for (int i = 0; i < N; ++i) b[r][i] = fmaf(f[r][i], h0[i], b[r][i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i) B[i] = begins ? 0.0f : B[i];        // nothing of the sequence before, a NaN either
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                A[i] *= f[r][i];
                B[i] = fmaf(f[r][i], B[i], b[r][i]);
            }
        }
        store_pair(tile, tile.group(), firsts != 0, A, B, &sh);
        __syncthreads();
        const bool open = k > 0 && !(__builtin_amdgcn_readfirstlane((int)sh.firsts[0]) & 1);
        carry_states(a, tile, k, cb, k == 0 || any_marks(tile, sh.firsts), open, &sh);
        float h[N];
        const Place<Shape> out(a, tile, k, cb);
        u32x4* to = a.h + out.row0 * a.units;
        group_states(tile, tile.group(), sh, h);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool begins = (firsts >> r) & 1;
            if (ballot(begins) != 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) h[i] = begins ? 0.0f : h[i];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) h[i] = fmaf(f[r][i], h[i], b[r][i]);
            if (out.stored(r)) store_rows<(G > 0)>(piece_at(to, out.first + r * out.units), Piece<DT>::pack(h));
            if (a.ends_out != nullptr && ((lasts >> r) & 1)) {
                const int64_t at = state_at(a, tile, cb, sh.last_of, r);
                if (at >= 0) store_state<N>(a.ends_out, at, h);
            }
        }
    }
    empty_sequences(a, tile, k, cb);
}

// (Three workgroups a CU, two took 1631 us instead of 1387 for 4.2 M rows of 136 bf16; 32 values of fp32 rows are 8 rows a lane and
// take the registers of two.)
template <int DT, int G, int R, bool PACKED>
__global__ __launch_bounds__(kBlock, DT == FS_F32 && !PACKED ? 2 : 3) void scan_bwd_kernel(ScanArgs a, const int32_t* __restrict__ tile_seq)
{
    using Shape = ScanShape<DT, G, R>;
    constexpr int N = Shape::N, LPB = kPackBlock / N;
    __shared__ ScanShared<Shape> sh;
    const Shape tile(a);
    const uint32_t t = take_ticket(a, &sh);
    const int64_t k = t / (uint32_t)a.col_blocks;       // from the batch's end
    const int cb = (int)(t % (uint32_t)a.col_blocks);
    if (k < a.tiles) {
        const Place<Shape> p(a, tile, a.tiles - 1 - k, cb);
        const Bounds bounds(a, tile_seq == nullptr ? 0 : tile_seq[a.tiles - 1 - k]);
        const u32x4* from_d = a.dh + p.row0 * a.units;
        u32x4 raw_d[R];
        Saved<DT, PACKED, 0, (G > 0)> x[R];
        Saved<DT, PACKED, 1, (G > 0)> gate[R];
        Saved<DT, PACKED, 2, (G > 0)> before[R];        // h of the row before
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {              // in the order of their use
            const uint32_t block = p.row(r) * (uint32_t)a.nb + p.own / LPB;
            gate[r].load(a, p.row0, p.at(r), block);
            raw_d[r] = load_rows<(G > 0)>(piece_at(from_d, p.at(r)));
        }
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            const uint32_t row = p.row(r), block = row * (uint32_t)a.nb + p.own / LPB;
            x[r].load(a, p.row0, p.at(r), block);
            const uint32_t up = p.row0 > 0 || row == 0 ? 0u : 1u;               // the batch's first row stands in for the one before it
            before[r].load(a, p.row0 > 0 ? p.row0 - 1 : 0, p.at(r) - up * p.units, block - up * (uint32_t)a.nb);
        }
        mark_sequences(a, tile, tile_seq, a.tiles - 1 - k, p.row0, bounds, &sh);
        const uint32_t firsts = group_marks(tile, sh.firsts), lasts = group_marks(tile, sh.lasts);
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
            const bool ends = (lasts >> r) & 1;
            if (ballot(ends) != 0) {
                if (ends && a.ends_in != nullptr) {
                    const int64_t at = state_at(a, tile, cb, sh.last_of, r);
                    if (at >= 0) {
                        float end[N];
                        load_state<N>(a.ends_in, at, end);
#pragma unroll
                        for (int i = 0; i < N; ++i) d[r][i] += end[i];
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i) B[i] = ends ? 0.0f : B[i];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                A[i] *= f[r][i];
                B[i] = f[r][i] * (d[r][i] + B[i]);
            }
        }
        store_pair(tile, tile.Q - 1 - tile.group(), lasts != 0, A, B, &sh);
        __syncthreads();
        const bool open = k > 0 && !((__builtin_amdgcn_readfirstlane((int)sh.lasts[(tile.T - 1) >> 5]) >> ((tile.T - 1) & 31)) & 1);
        carry_states(a, tile, k, cb, k == 0 || any_marks(tile, sh.lasts), open, &sh);
        float U[N];
        const Place<Shape> out(a, tile, a.tiles - 1 - k, cb);
        u32x4* to_x = a.dx + out.row0 * a.units;
        u32x4* to_g = a.dgate + out.row0 * a.units;
        group_states(tile, tile.Q - 1 - tile.group(), sh, U);
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            float xv[N], hb[N], dx[N], dg[N];
            x[r].values(xv);
            before[r].values(hb);
            const bool ends = (lasts >> r) & 1, begins = (firsts >> r) & 1;
            if (ballot(ends) != 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) U[i] = ends ? 0.0f : U[i];
            }
            if (ballot(begins) != 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) hb[i] = begins ? 0.0f : hb[i];
                if (begins && a.h0 != nullptr) {
                    const int64_t at = state_at(a, tile, cb, sh.first_of, r);
                    if (at >= 0) load_state<N>(a.h0, at, hb);
                }
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float Gi = d[r][i] + U[i];
                dx[i] = o[r][i] * Gi;
                dg[i] = dx[i] * f[r][i] * (hb[i] - xv[i]);
                U[i] = f[r][i] * Gi;
            }
            if (out.stored(r)) {
                store_rows<(G > 0)>(piece_at(to_x, out.first + r * out.units), Piece<DT>::pack(dx));
                store_rows<(G > 0)>(piece_at(to_g, out.first + r * out.units), Piece<DT>::pack(dg));
            }
            if (a.ends_out != nullptr && begins) {
                const int64_t at = state_at(a, tile, cb, sh.first_of, r);
                if (at >= 0) store_state<N>(a.ends_out, at, U);
            }
        }
    }
    empty_sequences(a, tile, k, cb);
}

// All words not ready, no ticket taken, and every tile's first sequence: the largest s with offsets[s] <= the row before it
// (bad offsets: some s in [0, S)); behind the last tile's the same for the batch's end.  A thread a tile bisects here, beside the writes of the others; in the tiles' own workgroups
// the search is a chain of loads in front of everything.
__global__ __launch_bounds__(kBlock) void scan_clear_kernel(ScanArgs a, int64_t pieces, int tile_rows)
{
    const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (i < pieces) reinterpret_cast<u32x4*>(a.words)[i] = u32x4{~0u, ~0u, ~0u, ~0u};
    if (i == 0) *a.ticket = 0u;
    if (i > a.tiles) return;
    const int64_t row = i < a.tiles ? i * tile_rows : a.n;
    int64_t lo = 0, hi = a.S;                            // offsets[lo] < row (taken as given for lo = 0) <= offsets[hi]
    while (hi - lo > 1) {
        const int64_t mid = lo + ((hi - lo) >> 1);
        if (a.offsets[mid] < row) lo = mid; else hi = mid;
    }
    a.tile_seq[i] = (int32_t)lo;
}

// One token of every session: a 16-byte piece of x, gate and h to a lane, its states as fp32 beside it.  (No pointer is
// restricted: h may be x, state_out state.)
template <int DT>
__global__ __launch_bounds__(kBlock) void scan_step_kernel(const u32x4* x, const u32x4* gate, const float* state,
                                                           float* state_out, u32x4* h, int64_t pieces)
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

// Lanes of a group: 16 or 8 for rows of as many pieces or a multiple of them (instances of their own: 3 % faster than with the
// lanes as an argument, and the tiles of long rows stay long); other rows whole up to 256 columns, longer ones in blocks of equal size.
int scan_lanes(int units, int N)
{
    if (units % 16 == 0) return 16;
    if (units % 8 == 0) return 8;
    const int most = kBlock / N, blocks = (units + most - 1) / most;
    return (units + blocks - 1) / blocks;
}

// Values of a lane, R rows of a 16-byte piece.  Forward f and b of 64 values are 128 registers of the 168 with which three
// workgroups share a CU (32 values, four workgroups: 867 us instead of 547 for 4.2 M rows of 128 fp16; 128 values, two: 753): longer
// tiles mean fewer words, counters and searches a row.  Backward five numbers a value are held, f, 1 - f, dh and, as they came, x
// and h: 32 values (64: 1208 us instead of 1100 in bf16, 1489 instead of 1024 for half as many rows of fp32; 16: 1720 and 1047).
constexpr int kFwdValues = 64, kBwdValues = 32;

// Everything that follows from the sizes; *a gets them, `words` the workspace's places.
fs_status plan_scan(int64_t n, int32_t D, fs_dtype dtype, int32_t T, int32_t B, int values, Carver* ws, ScanArgs* a)
{
    const fs_status st = check_seq_rows(n, D, dtype, &a->units);
    if (st != FS_OK) return st;
    if (T < 1 || B < 1 || (int64_t)T * B >= (1LL << 31)) return FS_ERR_SIZE;
    if (a->units > kMostPieces) return FS_ERR_SIZE;                 // a tile of at most 1024 rows has 32-bit offsets in bytes
    a->S = (int64_t)T * B;
    a->n = n;
    a->nb = (int)pack_blocks(D);
    const int N = dtype == FS_F32 ? 4 : 8;
    a->lanes = scan_lanes(a->units, N);
    a->groups = kBlock / a->lanes < most_groups(N) ? kBlock / a->lanes : most_groups(N);
    a->by_lanes = (65536 + a->lanes - 1) / a->lanes;
    a->by_columns = (65536 + a->lanes * N - 1) / (a->lanes * N);
    const int64_t rows = (int64_t)a->groups * (values / N);
    a->col_blocks = (a->units + a->lanes - 1) / a->lanes;
    a->tiles = (n + rows - 1) / rows;
    if (a->tiles * a->col_blocks > kMostGrid) return FS_ERR_SIZE;   // (over 240 GB in x: 14400 bytes of it a workgroup or more)
    // where the tiles are few, more workgroups share the sequences' passes of 256: up to 1024 of them, as many as a launch has room for
    const int64_t passes = (a->S + kBlock - 1) / kBlock, room = kMostGrid / a->col_blocks;
    const int64_t most = room < 1024 ? room : 1024, shared = passes < most ? passes : most;
    a->strides = a->tiles > shared ? a->tiles : shared;
    uint32_t* const ticket = ws->take<uint32_t>(1);                 // always: a workspace of no bytes could be null, which is a question
    if (a->tiles > 1) {
        a->words = ws->take<uint64_t>((size_t)(a->tiles + a->tiles / kSpan) * (size_t)a->col_blocks * (size_t)(a->lanes * N));
        a->tile_seq = ws->take<int32_t>((size_t)a->tiles + 1);
        a->ticket = ticket;
    }
    return FS_OK;
}

fs_status clear_words(const ScanArgs& a, int N, int values, hipStream_t s)
{
    if (a.tiles <= 1) return FS_OK;
    const int64_t pieces = (a.tiles + a.tiles / kSpan) * a.col_blocks * (a.lanes * N / 2);      // at least 2 a tile, of 2 tiles or more
    const int64_t grid = (pieces + kBlock - 1) / kBlock;                    // fewer than the tiles' workgroups, in plan_scan's bound
    FS_LAUNCH("scan_clear", scan_clear_kernel, dim3((unsigned)grid), dim3(kBlock), s, a, pieces, a.groups * (values / N));
    return FS_OK;
}

#define FS_DISPATCH_LANES(lanes, CALL)                                                  \
    switch (lanes) {                                                                    \
        case 8: CALL(8); break;                                                         \
        case 16: CALL(16); break;                                                       \
        default: CALL(0); break;                                                        \
    }

template <int DT>
fs_status scan_fwd_launch(const ScanArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.strides * a.col_blocks));
#define CALL(G) FS_LAUNCH("scan_fwd", (scan_fwd_kernel<DT, G, kFwdValues / Piece<DT>::N>), grid, dim3(kBlock), s, a, a.tile_seq)
    FS_DISPATCH_LANES(a.lanes, CALL)
#undef CALL
    return FS_OK;
}

template <int DT, bool PACKED>
fs_status scan_bwd_launch(const ScanArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.strides * a.col_blocks));
#define CALL(G) FS_LAUNCH("scan_bwd", (scan_bwd_kernel<DT, G, kBwdValues / Piece<DT>::N, PACKED>), grid, dim3(kBlock), s, a, a.tile_seq)
    FS_DISPATCH_LANES(a.lanes, CALL)
#undef CALL
    return FS_OK;
}

fs_status scan_bwd(ScanArgs a, bool packed, int32_t D, fs_dtype dtype, int32_t T, int32_t B, void* workspace,
                   size_t* workspace_bytes, hipStream_t s)
{
    if (!workspace_bytes) return FS_ERR_NULL;
    Carver ws(workspace);
    fs_status st = plan_scan(a.n, D, dtype, T, B, kBwdValues, &ws, &a);
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
    st = clear_words(a, dtype == FS_F32 ? 4 : 8, kBwdValues, s);
    if (st != FS_OK) return st;
    if (packed) {
#define CALL(DT) st = scan_bwd_launch<DT, true>(a, s)
        FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    } else {
#define CALL(DT) st = scan_bwd_launch<DT, false>(a, s)
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
    fs_status st = plan_scan(n, D, dtype, T, B, kFwdValues, &ws, &a);
    if (st != FS_OK) return st;
    if (!workspace) { *workspace_bytes = ws.used; return FS_OK; }
    if (*workspace_bytes < ws.used || misaligned(workspace, 256)) return FS_ERR_WORKSPACE;
    if (!offsets || (n > 0 && (!x || !gate || !h))) return FS_ERR_NULL;
    if (misaligned(x, 16) || misaligned(gate, 16) || misaligned(h, 16) || misaligned(h0, 16) || misaligned(h_last, 16) || misaligned(offsets, 8))
        return FS_ERR_ALIGN;
    a.x = static_cast<const u32x4*>(x); a.gate = static_cast<const u32x4*>(gate);
    a.offsets = offsets; a.ends_in = h0; a.h = static_cast<u32x4*>(h); a.ends_out = h_last; a.status = dev_status;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    st = clear_words(a, dtype == FS_F32 ? 4 : 8, kFwdValues, hs);
    if (st != FS_OK) return st;
#define CALL(DT) return scan_fwd_launch<DT>(a, hs)
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
    if (grid > kMostGrid) return FS_ERR_SIZE;                               // (64 GB a tensor)
#define CALL(DT) FS_LAUNCH("scan_step", scan_step_kernel<DT>, dim3((unsigned)grid), dim3(kBlock), static_cast<hipStream_t>(stream),  \
                           static_cast<const u32x4*>(x), static_cast<const u32x4*>(gate), state, state_out, static_cast<u32x4*>(h), pieces)
    FS_DISPATCH_DTYPE(dtype, CALL)
#undef CALL
    return FS_OK;
}
