// Distillation from a teacher's top logits, forward and backward.
//
// For every row i with teacher entries j in S_i (a CSR row: stored logits u_j), student logits z_v, temperature tau:
//   p_j = exp(u_j / tau) / sum over S_i,   q_v = exp(z_v / tau) / sum over all v
//   loss = w tau^2 sum_{j in S_i} p_j (log p_j - log q_j),   d loss / d z_v = w tau (q_v - p_v)
// With m the largest z and M the largest u of the row, e_j = exp((u_j - M) / tau), U = sum e_j, Z = sum exp((z_v - m) / tau):
//   sum p (log p - log q) = sum_j e_j ((u_j - M) - (z_j - m)) / (tau U) - log U + log Z
// so one pass over the row gives everything but the gradient.
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kThreads = 256;

// What the threads of a workgroup know of a row's teacher.
struct Teacher {
    float top, total;      // M, U
    bool held;             // an entry above -inf
};

// Whether row `row` has something to do; its entries and factor.
__device__ inline bool row_of(const DistillArgs &a, int64_t row, int &begin, int &end, float &w)
{
    begin = a.pos[row];
    end = a.pos[row + 1];
    w = a.weight ? a.weight[row] : 1.0f;
    return w != 0.0f && end > begin;
}

// The largest stored logit; not a number counts as +inf, so that it reaches the results.
template <int kThreads> __device__ inline float largest_entry(const DistillArgs &a, int begin, int end)
{
    float top = -kInfinity;
    for (int i = begin + (int)threadIdx.x; i < end; i += kThreads) {
        const float u = a.val[i];
        top = fmaxf(top, u != u ? kInfinity : u);
    }
    return top;
}

template <typename T> __device__ inline void put_word(T *to, bool same, const typename Word<T>::type &v)
{
    if (same) *reinterpret_cast<typename Word<T>::type *>(to) = v;
    else {
#pragma unroll
        for (int e = 0; e < Word<T>::n; ++e) to[e] = v[e];
    }
}

// The row of zeros of a row without loss.
template <typename T, int kThreads> __device__ inline void zero_row(T *g, int cols)
{
    const RowSplit<T> split(g, cols);
    const typename Word<T>::type none = (typename Word<T>::type)((T)0.0f);
    for (int i = (int)threadIdx.x; i < split.words; i += kThreads)
        reinterpret_cast<typename Word<T>::type *>(g + split.head)[i] = none;
    const int edge = split.edge((int)threadIdx.x, cols);
    if (edge >= 0) g[edge] = (T)0.0f;
}

// One workgroup a row: a pass over the logits with the running maximum and sum of every thread, then one that writes
// the gradient.
template <typename T>
__global__ void __launch_bounds__(kThreads) distill_row_kernel(DistillArgs a)
{
    typedef typename Word<T>::type word;
    __shared__ float share[3 * kThreads / NACHO_WAVE], share2[3 * kThreads / NACHO_WAVE];
    const int tid = (int)threadIdx.x, cols = a.cols;
    const float c = kLog2e / a.temperature;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        T *g = a.grad ? static_cast<T *>(a.grad) + row * a.ldg : nullptr;
        int begin, end;
        float w;
        bool active = row_of(a, row, begin, end, w);
        float top[2] = {-kInfinity, -kInfinity}, sum = 0.0f;
        const T *z = static_cast<const T *>(a.logits) + row * a.ldl;
        const RowSplit<T> split(z, cols);
        const word *words = reinterpret_cast<const word *>(z + split.head);
        const int edge = split.edge(tid, cols);
        if (active) {
            top[1] = largest_entry<kThreads>(a, begin, end);
            for (int i = tid; i < split.words; i += kThreads) {
                const word v = words[i];
                float m = wide(v[0]);
#pragma unroll
                for (int e = 1; e < Word<T>::n; ++e) m = fmaxf(m, wide(v[e]));
                if (m > top[0]) {
                    sum = sum * exp2_of((top[0] - m) * c);
                    top[0] = m;
                }
                if (top[0] == -kInfinity && m == -kInfinity) continue;
#pragma unroll
                for (int e = 0; e < Word<T>::n; ++e) sum += exp2_of((wide(v[e]) - top[0]) * c);
            }
            if (edge >= 0) {
                const float v = wide(z[edge]);
                if (v > top[0]) {
                    sum = sum * exp2_of((top[0] - v) * c);
                    top[0] = v;
                }
                if (v != -kInfinity) sum += exp2_of((v - top[0]) * c);
            }
            const float own_top = top[0];
            group_all<kThreads>(top, share, MaxOf(), MaxOf());
            if (own_top != top[0]) sum *= exp2_of((own_top - top[0]) * c);
            active = top[1] > -kInfinity;
        }
        if (!active) {
            if (tid == 0 && a.loss) a.loss[row] = 0.0f;
            if (tid == 0 && a.lse) a.lse[row] = 0.0f;
            if (g) zero_row<T, kThreads>(g, cols);
            __syncthreads();
            continue;
        }
        float s[3] = {sum, 0.0f, 0.0f};
        for (int i = begin + tid; i < end; i += kThreads) {
            const float u = a.val[i] - top[1], e = exp2_of(u * c);
            s[1] += e;
            if (!(e == 0.0f)) s[2] += e * (u - (wide(z[a.crd[i]]) - top[0]));
        }
        group_all<kThreads>(s, share2, SumOf(), SumOf(), SumOf());
        const float tau = a.temperature, log_z = logf(s[0]);
        if (tid == 0) {
            if (a.loss) a.loss[row] = w * tau * tau * (s[2] / (s[1] * tau) - logf(s[1]) + log_z);
            if (a.lse) a.lse[row] = top[0] / tau + log_z;
        }
        if (g) {
            const float q = w * tau / s[0], p = w * tau / s[1];
            const bool same = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
            for (int i = tid; i < split.words; i += kThreads) {
                word v = words[i];
#pragma unroll
                for (int e = 0; e < Word<T>::n; ++e) v[e] = (T)(q * exp2_of((wide(v[e]) - top[0]) * c));
                put_word(g + split.head + i * Word<T>::n, same, v);
            }
            if (edge >= 0) g[edge] = (T)(q * exp2_of((wide(z[edge]) - top[0]) * c));
            __syncthreads();               // (the stored columns again, now with the teacher's part)
            for (int i = begin + tid; i < end; i += kThreads) {
                const int j = a.crd[i];
                g[j] = (T)(q * exp2_of((wide(z[j]) - top[0]) * c) - p * exp2_of((a.val[i] - top[1]) * c));
            }
        }
        __syncthreads();
    }
}

// The gradient from what the forward call left.
template <typename T>
__global__ void __launch_bounds__(kThreads) distill_grad_kernel(DistillArgs a)
{
    typedef typename Word<T>::type word;
    __shared__ float share[kThreads / NACHO_WAVE], share2[kThreads / NACHO_WAVE];
    const int tid = (int)threadIdx.x, cols = a.cols;
    const float c = kLog2e / a.temperature, tau = a.temperature;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        T *g = static_cast<T *>(a.grad) + row * a.ldg;
        int begin, end;
        float w;
        bool active = row_of(a, row, begin, end, w);
        float top[1] = {-kInfinity};
        if (active) {
            top[0] = largest_entry<kThreads>(a, begin, end);
            group_all<kThreads>(top, share, MaxOf());
            active = top[0] > -kInfinity;
        }
        if (!active) {
            zero_row<T, kThreads>(g, cols);
            __syncthreads();
            continue;
        }
        float total[1] = {0.0f};
        for (int i = begin + tid; i < end; i += kThreads) total[0] += exp2_of((a.val[i] - top[0]) * c);
        group_all<kThreads>(total, share2, SumOf());
        const T *z = static_cast<const T *>(a.logits) + row * a.ldl;
        const RowSplit<T> split(z, cols);
        const word *words = reinterpret_cast<const word *>(z + split.head);
        const int edge = split.edge(tid, cols);
        const float base = a.lse_in[row] * tau, q = w * tau, p = w * tau / total[0];
        const bool same = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
        for (int i = tid; i < split.words; i += kThreads) {
            word v = words[i];
#pragma unroll
            for (int e = 0; e < Word<T>::n; ++e) v[e] = (T)(q * exp2_of((wide(v[e]) - base) * c));
            put_word(g + split.head + i * Word<T>::n, same, v);
        }
        if (edge >= 0) g[edge] = (T)(q * exp2_of((wide(z[edge]) - base) * c));
        __syncthreads();
        for (int i = begin + tid; i < end; i += kThreads) {
            const int j = a.crd[i];
            g[j] = (T)(q * exp2_of((wide(z[j]) - base) * c) - p * exp2_of((a.val[i] - top[0]) * c));
        }
        __syncthreads();
    }
}

unsigned row_groups(int64_t rows) { return (unsigned)(rows < (1 << 20) ? rows : 1 << 20); }

}  // namespace

hipError_t launch_distill(int dtype, const DistillArgs &a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    const dim3 grid(row_groups(a.rows));
    if (dtype == NACHO_F32) distill_row_kernel<float><<<grid, kThreads, 0, s>>>(a);
    else if (dtype == NACHO_BF16) distill_row_kernel<bf16_t><<<grid, kThreads, 0, s>>>(a);
    else distill_row_kernel<f16_t><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_distill_grad(int dtype, const DistillArgs &a, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    const dim3 grid(row_groups(a.rows));
    if (dtype == NACHO_F32) distill_grad_kernel<float><<<grid, kThreads, 0, s>>>(a);
    else if (dtype == NACHO_BF16) distill_grad_kernel<bf16_t><<<grid, kThreads, 0, s>>>(a);
    else distill_grad_kernel<f16_t><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace nacho
