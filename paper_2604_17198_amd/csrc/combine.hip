// The weighted sum of a token's rows, out_t = residual_t + sum_i gate_i y[slot_i], and its gradients
// grad_y[slot_i] = gate_i grad_out_t, grad_gate_i = <grad_out_t, y[slot_i]>.
//
// Bound by memory: every row of y is read (or written) once.  A workgroup has a token; a thread keeps its columns of the
// token's row in registers while it goes over the entries, so that this row is read once for four entries.
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kBatch = 4;              // entries whose rows are asked for together

// N consecutive elements, as one access.
template <typename T, int N> struct Part {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T> struct Part<T, 1> {
    typedef T type;
};
template <typename T, int N> __device__ inline void get(const T *at, float (&v)[N])
{
    const typename Part<T, N>::type p = *reinterpret_cast<const typename Part<T, N>::type *>(at);
    if constexpr (N == 1) v[0] = wide((T)p);
    else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = wide((T)p[e]);
    }
}
template <typename T, int N> __device__ inline void put(T *at, const float (&v)[N])
{
    typename Part<T, N>::type p;
    if constexpr (N == 1) p = (T)v[0];
    else {
#pragma unroll
        for (int e = 0; e < N; ++e) p[e] = (T)v[e];
    }
    *reinterpret_cast<typename Part<T, N>::type *>(at) = p;
}

template <typename T, int N, int kThreads>
__global__ void __launch_bounds__(kThreads) combine_kernel(CombineArgs a)
{
    const T *y = static_cast<const T *>(a.y), *residual = static_cast<const T *>(a.residual);
    T *out = static_cast<T *>(a.out);
    const int first = ((int)blockIdx.y * kThreads + (int)threadIdx.x) * N, step = (int)gridDim.y * kThreads * N;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const int begin = a.pos[t], end = a.pos[t + 1];
        for (int64_t c = first; c < a.cols; c += step) {
            float sum[N];
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] = 0.0f;
            for (int i = begin; i < end; i += kBatch) {
                float v[kBatch][N], g[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (i + b < end) {
                        get<T, N>(y + (int64_t)a.slot[i + b] * a.ldy + c, v[b]);
                        g[b] = a.gate ? a.gate[i + b] : 1.0f;
                    }
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (i + b < end) {
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[e] += g[b] * v[b][e];
                    }
            }
            if (residual) {
                float r[N];
                get<T, N>(residual + t * a.ldr + c, r);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += r[e];
            }
            put<T, N>(out + t * a.ldo + c, sum);
        }
    }
}

template <typename T, int N, int kThreads>
__global__ void __launch_bounds__(kThreads) combine_grad_kernel(CombineArgs a)
{
    __shared__ float share[kBatch * kThreads / NACHO_WAVE];
    const T *y = static_cast<const T *>(a.y), *grad_out = static_cast<const T *>(a.grad_out);
    T *grad_y = static_cast<T *>(a.grad_y);
    const int first = (int)threadIdx.x * N;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const int begin = a.pos[t], end = a.pos[t + 1];
        for (int i = begin; i < end; i += kBatch) {
            float dot[kBatch] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int64_t c = first; c < a.cols; c += kThreads * N) {
                float go[N];
                get<T, N>(grad_out + t * a.ldg + c, go);
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (i + b < end) {
                        const int64_t slot = a.slot[i + b];
                        if (a.grad_gate) {
                            float v[N];
                            get<T, N>(y + slot * a.ldy + c, v);
#pragma unroll
                            for (int e = 0; e < N; ++e) dot[b] += go[e] * v[e];
                        }
                        if (grad_y) {
                            const float g = a.gate ? a.gate[i + b] : 1.0f;
                            float v[N];
#pragma unroll
                            for (int e = 0; e < N; ++e) v[e] = g * go[e];
                            put<T, N>(grad_y + slot * a.ldgy + c, v);
                        }
                    }
            }
            if (a.grad_gate) {
                group_all<kThreads>(dot, share, SumOf(), SumOf(), SumOf(), SumOf());
                const int b = (int)threadIdx.x;
                if (b < kBatch && i + b < end) a.grad_gate[i + b] = b == 0 ? dot[0] : (b == 1 ? dot[1] : (b == 2 ? dot[2] : dot[3]));
                if (kThreads > NACHO_WAVE) __syncthreads();
            }
        }
    }
}

// The widest access that all rows allow: every one of the matrices starts and goes on at multiples of it, and so does
// the number of columns.
struct Widest {
    uintptr_t bits;
    explicit Widest(int64_t cols, int elem) : bits((uintptr_t)(cols * elem)) {}
    void with(const void *p, int64_t ld, int elem)
    {
        if (p) bits |= (uintptr_t)p | (uintptr_t)(ld * elem);
    }
};

template <typename F> void by_access(int dtype, uintptr_t bits, F f)
{
    using std::integral_constant;
    if (dtype == NACHO_F32) {
        if (bits % 16 == 0) f((float)0, integral_constant<int, 4>());
        else f((float)0, integral_constant<int, 1>());
    } else if (dtype == NACHO_BF16) {
        if (bits % 16 == 0) f((bf16_t)0.0f, integral_constant<int, 8>());
        else if (bits % 4 == 0) f((bf16_t)0.0f, integral_constant<int, 2>());
        else f((bf16_t)0.0f, integral_constant<int, 1>());
    } else {
        if (bits % 16 == 0) f((f16_t)0.0f, integral_constant<int, 8>());
        else if (bits % 4 == 0) f((f16_t)0.0f, integral_constant<int, 2>());
        else f((f16_t)0.0f, integral_constant<int, 1>());
    }
}

}  // namespace

hipError_t launch_combine(int dtype, const CombineArgs &a, hipStream_t s)
{
    if (a.tokens == 0 || a.cols == 0) return hipSuccess;
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    Widest w(a.cols, elem);
    w.with(a.y, a.ldy, elem);
    w.with(a.residual, a.ldr, elem);
    w.with(a.out, a.ldo, elem);
    by_access(dtype, w.bits, [&](auto zero, auto access) {
        constexpr int N = decltype(access)::value;
        typedef decltype(zero) T;
        const unsigned groups = (unsigned)(a.tokens < (1 << 20) ? a.tokens : 1 << 20);
        const int64_t parts = (a.cols + N - 1) / N;
        if (parts <= 128) combine_kernel<T, N, 64><<<dim3(groups, (unsigned)((parts + 63) / 64)), 64, 0, s>>>(a);
        else combine_kernel<T, N, 256><<<dim3(groups, (unsigned)(parts < 256 * 64 ? (parts + 255) / 256 : 64)), 256, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_combine_grad(int dtype, const CombineArgs &a, hipStream_t s)
{
    if (a.tokens == 0 || (!a.grad_y && !a.grad_gate)) return hipSuccess;
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    Widest w(a.cols, elem);
    if (a.grad_gate) w.with(a.y, a.ldy, elem);
    w.with(a.grad_out, a.ldg, elem);
    w.with(a.grad_y, a.ldgy, elem);
    by_access(dtype, w.bits, [&](auto zero, auto access) {
        constexpr int N = decltype(access)::value;
        typedef decltype(zero) T;
        const unsigned groups = (unsigned)(a.tokens < (1 << 20) ? a.tokens : 1 << 20);
        if ((a.cols + N - 1) / N <= 128) combine_grad_kernel<T, N, 64><<<dim3(groups), 64, 0, s>>>(a);
        else combine_grad_kernel<T, N, 256><<<dim3(groups), 256, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace nacho
