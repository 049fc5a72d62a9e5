// Which sequences begin and end in a tile of rows, where many touch it: most of them without rows (scan.hip).
#pragma once

#include "fs_common.h"

namespace fs {

// Once the first wave has had the first kWave of the sequences that touch its tile, a workgroup looks at the others, kBlock at a
// time, and past so many rounds each row for its own sequence instead, by bisection.  (us, a round a time : bisection alone : the first
// wave alone, 64 a time: 500 k sequences of one row of 128 bf16 backward 144 : 177 : 145; 1.8 M rows of 16 bf16 in 500 k sequences of 0 to
// 7 66 : 97 : 72; 4000 rows of 128 in 40 gaps of 800, 1600, 3200 sequences without any 14.3, 15.7, - : 15.0, 15.0, 20.3 : 17.8, 22.2, 35.1, of
// 12800 - : 26 : 112; 1000 rows of 8 in 32768 sequences, one tile, - : 21 : 141; 2^20 sequences without any in front of 100 rows - : 9 : 5050.
// Four loads a thread in flight, 1024 a round: 148 for the first.)
constexpr uint32_t kMostMarkRounds = 8;

// Rounds over the sequences behind the first kWave of `count`.
__host__ __device__ inline uint32_t mark_rounds(uint32_t count)
{
    return count <= (uint32_t)kWave ? 0u : (count - (uint32_t)kWave + (uint32_t)kBlock - 1u) / (uint32_t)kBlock;
}

// The largest s in [first, first + count) with begin(s) <= row, where begin(first) is taken to be: log2(count) probes, inside
// that range whatever begin says.  (first + count <= 2^31)
template <typename Begin>
__host__ __device__ inline uint32_t sequence_of_row(uint32_t first, uint32_t count, int64_t row, Begin begin)
{
    uint32_t step = 1, at = 0;
    while (step < count - step) step <<= 1;
    for (; step > 0; step >>= 1)
        if (at + step < count && begin(first + at + step) <= row) at += step;
    return first + at;
}

}  // namespace fs
