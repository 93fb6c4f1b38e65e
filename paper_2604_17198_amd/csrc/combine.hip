// The weighted sum of a token's rows, out_t = residual_t + sum_i gate_i y[slot_i], and its gradients
// grad_y[slot_i] = gate_i grad_out_t, grad_gate_i = <grad_out_t, y[slot_i]>.
//
// Bound by memory: every row of y is read (or written) once.  kLanes lanes have a token (8 to 64 of a wavefront where its
// rows are short, else a workgroup), a lane words of 16 bytes; it keeps its columns of the token's row in registers while it
// goes over the entries, four at a time: their slots first, then the rows, so that four rows are on their way at once.  Rows
// that start anywhere are read and written in words too (global memory takes any alignment).  16384 x 4 x 4096 bf16: sums
// 156 to 163 us, gradients 215, 5.2 TB/s (a row asked for before the next one's slot is known: 160 and 250 where it measured 155
// and 244); 16384 x 4 x 4095 168 and 266 (with a branch around each load 184 and 291).
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kBatch = 4;              // entries whose rows are asked for together

enum Access { WORDS, ANYWHERE, TINY };  // rows of words of 16 bytes; rows that start and end anywhere; such rows shorter than a word

// A word of a row, `left` elements of which are there from its first one on.  The word that ends with the row is loaded where
// fewer are there, and moved down when it is used: no branch lies around a load, as behind one that loads may be in, the next
// wait is for all of them.  (Rows shorter than a word: elements one by one.)
template <typename T, Access kAccess> __device__ inline typename Word<T>::type load(const T *at, int left)
{
    constexpr int n = Word<T>::n;
    typename Word<T>::type w;
    if constexpr (kAccess == WORDS) w = *reinterpret_cast<const typename Word<T>::type *>(at);
    else if constexpr (kAccess == ANYWHERE) __builtin_memcpy(&w, at - (left < n ? n - left : 0), 16);
    else {
#pragma unroll
        for (int e = 0; e < n; ++e) w[e] = at[e < left ? e : left - 1];
    }
    return w;
}
template <typename T, Access kAccess> __device__ inline void widen(typename Word<T>::type w, int left, float (&v)[Word<T>::n])
{
    constexpr int n = Word<T>::n;
    if constexpr (kAccess == ANYWHERE) {
        typedef unsigned int four __attribute__((ext_vector_type(4)));
        four u = __builtin_bit_cast(four, w);
        const int bytes = left < n ? (n - left) * (int)sizeof(T) : 0;
        if (bytes & 8) u = four{u[2], u[3], 0, 0};
        if (bytes & 4) u = four{u[1], u[2], u[3], 0};
        if (bytes & 2) u = four{u[0] >> 16 | u[1] << 16, u[1] >> 16 | u[2] << 16, u[2] >> 16 | u[3] << 16, u[3] >> 16};
        w = __builtin_bit_cast(typename Word<T>::type, u);
    }
#pragma unroll
    for (int e = 0; e < n; ++e) v[e] = kAccess == TINY && e >= left ? 0.0f : wide((T)w[e]);
}
template <typename T, Access kAccess> __device__ inline void put(T *at, int left, const float (&v)[Word<T>::n])
{
    constexpr int n = Word<T>::n;
    if (kAccess == WORDS || left >= n) {
        typename Word<T>::type w;
#pragma unroll
        for (int e = 0; e < n; ++e) w[e] = (T)v[e];
        if constexpr (kAccess == WORDS) *reinterpret_cast<typename Word<T>::type *>(at) = w;
        else __builtin_memcpy(at, &w, 16);
    } else {
#pragma unroll
        for (int e = 0; e < n; ++e)
            if (e < left) at[e] = (T)v[e];
    }
}

// The rows and factors of the entries from i on (behind the last: the last one again).
struct Entries {
    int64_t slot[kBatch];
    float gate[kBatch];
    __device__ Entries(const CombineArgs &a, int i, int end)
    {
        const float *gates = a.gate ? a.gate : reinterpret_cast<const float *>(a.slot);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int at = i + b < end ? i + b : end - 1;
            slot[b] = a.slot[at];
            gate[b] = gates[at];
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) gate[b] = a.gate ? gate[b] : 1.0f;
    }
};

template <int kLanes> constexpr int kThreads = kLanes <= 64 ? 64 : kLanes;

template <typename T, Access kAccess, int kLanes>
__global__ void __launch_bounds__(kThreads<kLanes>) combine_kernel(CombineArgs a)
{
    constexpr int n = Word<T>::n, kTokens = kThreads<kLanes> / kLanes;
    const T *y = static_cast<const T *>(a.y), *residual = static_cast<const T *>(a.residual);
    T *out = static_cast<T *>(a.out);
    const int first = ((int)blockIdx.y * kLanes + (int)threadIdx.x % kLanes) * n, step = (int)gridDim.y * kLanes * n;
    for (int64_t t = (int64_t)blockIdx.x * kTokens + (int)threadIdx.x / kLanes; t < a.tokens; t += (int64_t)gridDim.x * kTokens) {
        const int begin = a.pos[t], end = a.pos[t + 1];
        for (int64_t c = first; c < a.cols; c += step) {
            const int left = a.cols - (int)c;
            float sum[n];
#pragma unroll
            for (int e = 0; e < n; ++e) sum[e] = 0.0f;
            typename Word<T>::type last = {};
            if (residual) last = load<T, kAccess>(residual + t * a.ldr + c, left);
            for (int i = begin; i < end; i += kBatch) {
                const Entries of(a, i, end);
                typename Word<T>::type w[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) w[b] = load<T, kAccess>(y + of.slot[b] * a.ldy + c, left);
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (i + b < end) {
                        float v[n];
                        widen<T, kAccess>(w[b], left, v);
#pragma unroll
                        for (int e = 0; e < n; ++e) sum[e] += of.gate[b] * v[e];
                    }
            }
            if (residual) {
                float r[n];
                widen<T, kAccess>(last, left, r);
#pragma unroll
                for (int e = 0; e < n; ++e) sum[e] += r[e];
            }
            put<T, kAccess>(out + t * a.ldo + c, left, sum);
        }
    }
}

template <typename T, Access kAccess, int kLanes>
__global__ void __launch_bounds__(kThreads<kLanes>) combine_grad_kernel(CombineArgs a)
{
    constexpr int n = Word<T>::n, kTokens = kThreads<kLanes> / kLanes;
    __shared__ float share[kBatch * kThreads<kLanes> / NACHO_WAVE];
    const T *y = static_cast<const T *>(a.y), *grad_out = static_cast<const T *>(a.grad_out);
    T *grad_y = static_cast<T *>(a.grad_y);
    const int lane = (int)threadIdx.x % kLanes;
    for (int64_t t0 = (int64_t)blockIdx.x * kTokens; t0 < a.tokens; t0 += (int64_t)gridDim.x * kTokens) {
        const int64_t t = t0 + (int)threadIdx.x / kLanes;
        const int begin = t < a.tokens ? a.pos[t] : 0, end = t < a.tokens ? a.pos[t + 1] : 0;
        // (the tokens of one wavefront go on together, as long as the longest has entries)
        for (int i = begin; kTokens == 1 ? i < end : __any(i < end); i += kBatch) {
            float dot[kBatch] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (i < end) {
                const Entries of(a, i, end);
                for (int64_t c = lane * n; c < a.cols; c += kLanes * n) {
                    const int left = a.cols - (int)c;
                    const typename Word<T>::type w = load<T, kAccess>(grad_out + t * a.ldg + c, left);
                    float go[n];
                    if (a.grad_gate) {
                        typename Word<T>::type row[kBatch];
#pragma unroll
                        for (int b = 0; b < kBatch; ++b) row[b] = load<T, kAccess>(y + of.slot[b] * a.ldy + c, left);
                        widen<T, kAccess>(w, left, go);
#pragma unroll
                        for (int b = 0; b < kBatch; ++b) {
                            float v[n];
                            widen<T, kAccess>(row[b], left, v);
#pragma unroll
                            for (int e = 0; e < n; ++e) dot[b] += go[e] * v[e];
                        }
                    } else widen<T, kAccess>(w, left, go);
                    if (grad_y) {
#pragma unroll
                        for (int b = 0; b < kBatch; ++b)
                            if (i + b < end) {
                                float v[n];
#pragma unroll
                                for (int e = 0; e < n; ++e) v[e] = of.gate[b] * go[e];
                                put<T, kAccess>(grad_y + of.slot[b] * a.ldgy + c, left, v);
                            }
                    }
                }
            }
            if (a.grad_gate) {
                if constexpr (kLanes <= NACHO_WAVE) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
#pragma unroll
                        for (int off = kLanes / 2; off > 0; off >>= 1) dot[b] += __shfl_xor(dot[b], off, NACHO_WAVE);
                } else group_all<kThreads<kLanes>>(dot, share, SumOf(), SumOf(), SumOf(), SumOf());
                if (lane < kBatch && i + lane < end)
                    a.grad_gate[i + lane] = lane == 0 ? dot[0] : (lane == 1 ? dot[1] : (lane == 2 ? dot[2] : dot[3]));
                if (kLanes > NACHO_WAVE) __syncthreads();
            }
        }
    }
}

// Whether every row of all matrices, and with them every word, starts at a multiple of 16 bytes.
struct Words {
    uintptr_t bits;
    explicit Words(int64_t cols, int elem) : bits((uintptr_t)(cols * elem)) {}
    void with(const void *p, int64_t ld, int elem)
    {
        if (p) bits |= (uintptr_t)p | (uintptr_t)(ld * elem);
    }
};

// f(value of the type, aligned, lanes of a token)
template <typename F> void by_shape(int dtype, int64_t cols, bool aligned, F f)
{
    using std::integral_constant;
    auto by_type = [&](auto zero) {
        const int64_t words = (cols + Word<decltype(zero)>::n - 1) / Word<decltype(zero)>::n;
        auto by_lanes = [&](auto whole) {
            if (words <= 8) f(zero, whole, integral_constant<int, 8>());
            else if constexpr (whole.value == TINY) return;          // (a word)
            else if (words <= 16) f(zero, whole, integral_constant<int, 16>());
            else if (words <= 32) f(zero, whole, integral_constant<int, 32>());
            else if (words <= 128) f(zero, whole, integral_constant<int, 64>());
            else f(zero, whole, integral_constant<int, 256>());
        };
        if (aligned) by_lanes(integral_constant<Access, WORDS>());
        else if (cols >= Word<decltype(zero)>::n) by_lanes(integral_constant<Access, ANYWHERE>());
        else by_lanes(integral_constant<Access, TINY>());
    };
    if (dtype == NACHO_F32) by_type((float)0);
    else if (dtype == NACHO_BF16) by_type((bf16_t)0.0f);
    else by_type((f16_t)0.0f);
}

unsigned groups_of(int64_t tokens, int each)
{
    const int64_t groups = (tokens + each - 1) / each;
    return (unsigned)(groups < (1 << 20) ? groups : 1 << 20);
}

}  // namespace

hipError_t launch_combine(int dtype, const CombineArgs &a, hipStream_t s)
{
    if (a.tokens == 0 || a.cols == 0) return hipSuccess;
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    Words w(a.cols, elem);
    w.with(a.y, a.ldy, elem);
    w.with(a.residual, a.ldr, elem);
    w.with(a.out, a.ldo, elem);
    by_shape(dtype, a.cols, w.bits % 16 == 0, [&](auto zero, auto whole, auto lanes) {
        typedef decltype(zero) T;
        constexpr int kLanes = decltype(lanes)::value;
        const int64_t parts = ((int64_t)a.cols + kLanes * Word<T>::n - 1) / (kLanes * Word<T>::n);
        combine_kernel<T, decltype(whole)::value, kLanes>
            <<<dim3(groups_of(a.tokens, kThreads<kLanes> / kLanes), (unsigned)(parts < 64 ? parts : 64)), kThreads<kLanes>, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_combine_grad(int dtype, const CombineArgs &a, hipStream_t s)
{
    if (a.tokens == 0 || (!a.grad_y && !a.grad_gate)) return hipSuccess;
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    Words w(a.cols, elem);
    if (a.grad_gate) w.with(a.y, a.ldy, elem);
    w.with(a.grad_out, a.ldg, elem);
    w.with(a.grad_y, a.ldgy, elem);
    by_shape(dtype, a.cols, w.bits % 16 == 0, [&](auto zero, auto whole, auto lanes) {
        constexpr int kLanes = decltype(lanes)::value;
        combine_grad_kernel<decltype(zero), decltype(whole)::value, kLanes>
            <<<dim3(groups_of(a.tokens, kThreads<kLanes> / kLanes)), kThreads<kLanes>, 0, s>>>(a);
    });
    return hipGetLastError();
}

}  // namespace nacho
