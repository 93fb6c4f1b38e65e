// Rows into 8 bits and back (kept.hpp has the arithmetic).  A thread has 16 columns, two threads a block, so that
// it writes 16 bytes of codes and reads the other half's largest value from the lane beside it.  Bound by memory: 16384 x 8192 bf16, 407 MB
// either way, 69 to 80 us to keep and 69 to 72 to restore, 5.1 to 5.9 TB/s (a copy of as many bytes 5.1 by the framework, 5.95 by the runtime).
// 16384 x 8192 floats, 675 MB: 118 and 180 us, 5.7 and 3.7 TB/s.  Rows that start anywhere, 16384 x 8191: bf16 106 and 116 us, floats 125 and 234.
#include "kept.hpp"
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kThreads = 256, kColumns = 16;

// A thread's row and first column: threads take a row's sixteens of columns (an even number of them) one after the other.
struct Part {
    int64_t row;
    int column;
    __device__ Part(int64_t group, int each_row)
    {
        // (one division of 64 bits a workgroup)
        const int64_t first = group * kThreads, row0 = first / each_row;
        const unsigned at = (unsigned)(first - row0 * each_row) + threadIdx.x, rows = at / (unsigned)each_row;
        row = row0 + rows;
        column = (int)(at - rows * (unsigned)each_row) * kColumns;
    }
};

template <typename T, bool kWords> __global__ void __launch_bounds__(kThreads) keep_kernel(KeepArgs a, int each_row)
{
    const Part part((int64_t)blockIdx.y * gridDim.x + blockIdx.x, each_row);
    const bool there = part.row < a.rows;
    const int width = there ? a.cols - part.column : 0;
    const T *from = static_cast<const T *>(a.x) + (there ? part.row : 0) * a.ldx + part.column;
    float v[kColumns];
    constexpr int n = Word<T>::n;
    if (width >= kColumns) {
        typename Word<T>::type w[kColumns / n];
#pragma unroll
        for (int i = 0; i < kColumns / n; ++i) {
            if constexpr (kWords) w[i] = *reinterpret_cast<const typename Word<T>::type *>(from + i * n);
            else __builtin_memcpy(&w[i], from + i * n, 16);
        }
#pragma unroll
        for (int i = 0; i < kColumns; ++i) v[i] = wide((T)w[i / n][i % n]);
    } else {
#pragma unroll
        for (int i = 0; i < kColumns; ++i) v[i] = i < width ? wide(from[i]) : 0.0f;
    }
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < kColumns; ++i) most = magnitude(v[i]) > most ? magnitude(v[i]) : most;
    const unsigned other = moved<0xb1>(most), exponent = exponent_of(other > most ? other : most);
    const float by = steps_per(exponent);
    unsigned codes[kColumns / 4];
#pragma unroll
    for (int i = 0; i < kColumns / 4; ++i) codes[i] = exponent == 255 ? 0 : four_codes(v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3], by);
    if (width <= 0) return;
    int8_t *to = a.kept.code + part.row * a.kept.ldc + part.column;
    if (width >= kColumns) {
        if constexpr (kWords) *reinterpret_cast<uint4 *>(to) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
        else __builtin_memcpy(to, codes, kColumns);
    } else {
#pragma unroll
        for (int i = 0; i < kColumns; ++i)
            if (i < width) to[i] = (int8_t)(codes[i / 4] >> (8 * (i % 4)));
    }
    if ((threadIdx.x & 1) == 0) a.kept.exponent[part.row * a.kept.lde + part.column / kBlock] = (uint8_t)exponent;
}

template <typename T, bool kWords> __global__ void __launch_bounds__(kThreads) restore_kernel(KeepArgs a, int each_row)
{
    const Part part((int64_t)blockIdx.y * gridDim.x + blockIdx.x, each_row);
    if (part.row >= a.rows || part.column >= a.cols) return;
    const int width = a.cols - part.column;
    const int8_t *from = a.kept.code + part.row * a.kept.ldc + part.column;
    const float step = step_of(a.kept.exponent[part.row * a.kept.lde + part.column / kBlock]);
    T *to = static_cast<T *>(a.out) + part.row * a.ldx + part.column;
    constexpr int n = Word<T>::n;
    if (width >= kColumns) {
        unsigned codes[kColumns / 4];
        if constexpr (kWords) *reinterpret_cast<uint4 *>(codes) = *reinterpret_cast<const uint4 *>(from);
        else __builtin_memcpy(codes, from, kColumns);
#pragma unroll
        for (int i = 0; i < kColumns; i += n) {
            typename Word<T>::type w;
#pragma unroll
            for (int e = 0; e < n; ++e) w[e] = (T)value_of(codes[(i + e) / 4], (i + e) % 4, step);
            if constexpr (kWords) *reinterpret_cast<typename Word<T>::type *>(to + i) = w;
            else __builtin_memcpy(to + i, &w, 16);
        }
    } else {
        for (int i = 0; i < width; ++i) to[i] = (T)((float)from[i] * step);
    }
}

template <typename F> hipError_t over_rows(const KeepArgs &a, F launch)
{
    const int64_t each_row = ((int64_t)a.cols + kBlock - 1) / kBlock * (kBlock / kColumns);
    const int64_t groups = (a.rows * each_row + kThreads - 1) / kThreads, row = groups < (1 << 22) ? groups : 1 << 22;
    if (groups == 0) return hipSuccess;
    if ((groups + row - 1) / row > 65535) return hipErrorNotSupported;
    launch(dim3((unsigned)row, (unsigned)((groups + row - 1) / row)), (int)each_row);
    return hipGetLastError();
}

template <typename F> void by_type(int dtype, F f)
{
    if (dtype == NACHO_F32) f((float)0);
    else if (dtype == NACHO_BF16) f((bf16_t)0.0f);
    else f((f16_t)0.0f);
}

// Whether all rows of both sides start at multiples of 16 bytes.
bool in_words(const KeepArgs &a, const void *rows, int elem)
{
    return (((uintptr_t)rows | (uintptr_t)(a.ldx * elem) | (uintptr_t)a.kept.code | (uintptr_t)a.kept.ldc) & 15) == 0;
}

}  // namespace

hipError_t launch_keep(int dtype, const KeepArgs &a, hipStream_t s)
{
    hipError_t rc = hipSuccess;
    const bool words = in_words(a, a.x, dtype == NACHO_F32 ? 4 : 2);
    by_type(dtype, [&](auto zero) {
        rc = over_rows(a, [&](dim3 grid, int each_row) {
            if (words) keep_kernel<decltype(zero), true><<<grid, kThreads, 0, s>>>(a, each_row);
            else keep_kernel<decltype(zero), false><<<grid, kThreads, 0, s>>>(a, each_row);
        });
    });
    return rc;
}

hipError_t launch_restore(int dtype, const KeepArgs &a, hipStream_t s)
{
    hipError_t rc = hipSuccess;
    const bool words = in_words(a, a.out, dtype == NACHO_F32 ? 4 : 2);
    by_type(dtype, [&](auto zero) {
        rc = over_rows(a, [&](dim3 grid, int each_row) {
            if (words) restore_kernel<decltype(zero), true><<<grid, kThreads, 0, s>>>(a, each_row);
            else restore_kernel<decltype(zero), false><<<grid, kThreads, 0, s>>>(a, each_row);
        });
    });
    return rc;
}

}  // namespace nacho
