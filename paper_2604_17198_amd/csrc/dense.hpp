// Dense rows of 32- and 16-bit floating point values: types, 16-byte words, reductions over a workgroup.
#pragma once
#include "common.hpp"

namespace nacho {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Elements of a 16-byte word, and the word.
template <typename T> struct Word {
    static constexpr int n = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
};

__device__ inline float wide(float v) { return v; }
__device__ inline float wide(bf16_t v) { return (float)v; }
__device__ inline float wide(f16_t v) { return (float)v; }

// How a row of `cols` elements splits at 16-byte boundaries: `head` elements before the first one (all of a row that
// does not reach it), `words` whole words, `tail` elements behind the last.  Rows of an odd number of elements start
// anywhere.
template <typename T> struct RowSplit {
    int head, words, tail;
    __device__ RowSplit(const T *row, int cols)
    {
        constexpr int n = Word<T>::n;
        const int past = (int)((16u - ((unsigned)(uintptr_t)row & 15u)) & 15u) / (int)sizeof(T);
        head = past < cols ? past : cols;
        words = (cols - head) / n;
        tail = cols - head - words * n;
    }
    // The element outside the words that a thread looks after (threads 0 .. 15 have one at most), or -1.
    __device__ int edge(int thread, int cols) const
    {
        if (thread < head) return thread;
        return thread >= 8 && thread < 8 + tail ? cols - tail + thread - 8 : -1;
    }
};

struct MaxOf {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct SumOf {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// One value over the lanes of a wavefront, the same bits in every lane.
template <typename Op> __device__ inline float wave_all(float v, Op op)
{
#pragma unroll
    for (int off = NACHO_WAVE / 2; off > 0; off >>= 1) v = op(v, __shfl_xor(v, off, NACHO_WAVE));
    return v;
}

// N values over the kThreads threads of a workgroup in a fixed order, the same bits in every thread.  `share`: LDS of
// N * kThreads / 64 floats, which the next call must not use before the threads have met again.
template <int kThreads, int N, typename... Ops> __device__ inline void group_all(float (&v)[N], float *share, Ops... ops)
{
    constexpr int kWaves = kThreads / NACHO_WAVE;
    const int wave = (int)threadIdx.x / NACHO_WAVE;
    int i = 0;
    ((v[i] = wave_all(v[i], ops), ++i), ...);
    if (kWaves == 1) return;
    if (lane_id() == 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) share[j * kWaves + wave] = v[j];
    }
    __syncthreads();
    i = 0;
    auto joined = [&](auto op) {
        float a = share[i * kWaves];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) a = op(a, share[i * kWaves + w]);
        v[i] = a;
        ++i;
    };
    (joined(ops), ...);
}

constexpr float kLog2e = 1.4426950408889634f, kInfinity = __builtin_inff();

// 2^x in one instruction (results below the smallest normal number are zero).
__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

}  // namespace nacho
