// Distillation from a teacher's top logits, forward and backward.
//
// For every row i with teacher entries j in S_i (a CSR row: stored logits u_j), student logits z_v, temperature tau:
//   p_j = exp(u_j / tau) / sum over S_i,   q_v = exp(z_v / tau) / sum over all v
//   loss = w tau^2 sum_{j in S_i} p_j (log p_j - log q_j),   d loss / d z_v = w tau (q_v - p_v)
// With m the largest z and M the largest u of the row, e_j = exp((u_j - M) / tau), U = sum e_j, Z = sum exp((z_v - m) / tau):
//   sum p (log p - log q) = sum_j e_j ((u_j - M) - (z_j - m)) / (tau U) - log U + log Z
// so one pass over the row gives everything but the gradient.
//
// Bound by memory: the logits are read once and the gradient is written once.  A workgroup holds its words of 16 bytes in
// registers from the maximum over the sums to the gradient, a row at a time where a workgroup holds one (WHOLE: up to 512
// threads of 16 words in registers and 16 in LDS, 131072 values of 16 bits or 65536 floats).  Longer rows, and few long ones,
// are cut into parts: one launch leaves every part's maximum and sum (STATS), the next one joins them and writes its part of
// the gradient (APPLY).  The backward call knows the row's sum (GIVEN) and is cut likewise.
// 4096 x 65536 bf16 with gradients 229 us, 4.7 TB/s (logits read twice: 344); 4 x 131072 floats 4 + 5 us in two launches (a
// workgroup a row: 65 a call); 1021 x 100003 f16 statistics 39 us, join 9, gradients from the sums 73 to 75.
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

enum Stage { WHOLE, STATS, APPLY, GIVEN };

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

// Between two uses the words stay as they were loaded (the compiler would keep every element in 32 bits, twice the registers
// of 16-bit types: one workgroup a compute unit in place of two).
template <typename W, int kEach> __device__ inline void keep(W (&v)[kEach])
{
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        typedef unsigned int four __attribute__((ext_vector_type(4)));
        four bits = __builtin_bit_cast(four, v[i]);
        asm volatile("" : "+v"(bits));
        v[i] = __builtin_bit_cast(W, bits);
    }
}

template <typename T, int kThreads, int kEach, int kMore, Stage kStage>
__global__ void __launch_bounds__(kThreads, kThreads == 512 && kMore < 16 ? 4 : 1) distill_kernel(DistillArgs a, int part, int parts, int many)
{
    typedef typename Word<T>::type word;
    constexpr int n = Word<T>::n, kWaves = kThreads / NACHO_WAVE;
    __shared__ float share[2 * kWaves], share2[3 * kWaves];
    __shared__ word more[kMore > 0 ? kMore * kThreads : 1];           // a thread's words that its registers do not hold
    const int tid = (int)threadIdx.x;
    const float tau = a.temperature, c = kLog2e / tau;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x)
        for (int number = (int)blockIdx.y; number < many; number += (int)gridDim.y) {
            const int c0 = number * part, cols = a.cols - c0 < part ? a.cols - c0 : part;
            T *const g = kStage != STATS && a.grad ? static_cast<T *>(a.grad) + row * a.ldg + c0 : nullptr;
            const T *const z = static_cast<const T *>(a.logits) + row * a.ldl + c0;
            float *const left = a.partial + 2 * (row * parts + number);
            int begin, end;
            float w;
            bool active = row_of(a, row, begin, end, w);
            const RowSplit<T> split(z, cols);
            // (the same offset for every thread's words behind a base that the whole workgroup shares: few registers)
            const char *const words = reinterpret_cast<const char *>(z + split.head);
            const unsigned own = (unsigned)tid * 16u;
            auto word_at = [&](int i) -> const word & { return *reinterpret_cast<const word *>(words + (size_t)(i * kThreads) * 16 + own); };
            const int edge = split.edge(tid, cols);
            word v[kEach];
            float beside = -kInfinity;
            // (a row that has nothing to do is not read)
            const int there = active && (kStage == WHOLE || kStage == STATS || g) ? split.words : 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int at = tid + i * kThreads;
                v[i] = (word)((T)-kInfinity);
                if (at < there) v[i] = word_at(i);
            }
#pragma unroll
            for (int i = 0; i < kMore; ++i) {
                const int at = tid + (kEach + i) * kThreads;
                more[i * kThreads + tid] = at < there ? word_at(kEach + i) : (word)((T)-kInfinity);
            }
            if (edge >= 0 && active) beside = wide(z[edge]);
            // the largest logit (of the row, or of the part) and the largest stored one
            float top[2] = {-kInfinity, -kInfinity};
            if (active) {
                if (kStage != STATS) top[1] = largest_entry<kThreads>(a, begin, end);
                if (kStage == WHOLE || kStage == STATS) {
                    top[0] = beside;
#pragma unroll
                    for (int i = 0; i < kEach; ++i)
#pragma unroll
                        for (int e = 0; e < n; ++e) top[0] = fmaxf(top[0], wide((T)v[i][e]));
#pragma unroll 2
                    for (int i = 0; i < kMore; ++i) {
                        const word x = more[i * kThreads + tid];
#pragma unroll
                        for (int e = 0; e < n; ++e) top[0] = fmaxf(top[0], wide((T)x[e]));
                    }
                } else if (kStage == APPLY)
                    for (int i = tid; i < parts; i += kThreads) top[0] = fmaxf(top[0], a.partial[2 * (row * parts + i)]);
                group_all<kThreads>(top, share, MaxOf(), MaxOf());
                if (kStage == GIVEN) top[0] = a.lse_in[row] * tau;
                if (kStage != STATS) active = top[1] > -kInfinity;
            }
            if (!active) {
                if (kStage != STATS && kStage != GIVEN && tid == 0 && number == 0) a.loss[row] = a.lse[row] = 0.0f;
                if (g) {
                    const RowSplit<T> mine(g, cols);
                    for (int i = tid; i < mine.words; i += kThreads) reinterpret_cast<word *>(g + mine.head)[i] = (word)((T)0.0f);
                    const int last = mine.edge(tid, cols);
                    if (last >= 0) g[last] = (T)0.0f;
                }
                __syncthreads();
                continue;
            }
            keep(v);
            // Z, U, and the sum over the entries
            float s[3] = {0.0f, 0.0f, 0.0f};
            if (kStage == WHOLE || kStage == STATS) {
                // (a part of masked logits alone has nothing to add)
                const float from = kStage == STATS && top[0] == -kInfinity ? 0.0f : top[0];
                s[0] = edge >= 0 ? exp2_of((beside - from) * c) : 0.0f;
#pragma unroll
                for (int i = 0; i < kEach; ++i)
#pragma unroll
                    for (int e = 0; e < n; ++e) s[0] += exp2_of((wide((T)v[i][e]) - from) * c);
#pragma unroll 2
                for (int i = 0; i < kMore; ++i) {
                    const word x = more[i * kThreads + tid];
#pragma unroll
                    for (int e = 0; e < n; ++e) s[0] += exp2_of((wide((T)x[e]) - from) * c);
                }
            } else if (kStage == APPLY)
                for (int i = tid; i < parts; i += kThreads) {
                    const float m = a.partial[2 * (row * parts + i)], t = a.partial[2 * (row * parts + i) + 1];
                    s[0] += m == top[0] ? t : t * exp2_of((m - top[0]) * c);
                }
            if (kStage != STATS)
                for (int i = begin + tid; i < end; i += kThreads) {
                    const float u = a.val[i] - top[1], e = exp2_of(u * c);
                    s[1] += e;
                    if (kStage != GIVEN && number == 0 && !(e == 0.0f)) s[2] += e * (u - (wide(z[a.crd[i]]) - top[0]));
                }
            group_all<kThreads>(s, share2, SumOf(), SumOf(), SumOf());
            if (kStage == STATS) {
                if (tid == 0) {
                    left[0] = top[0];
                    left[1] = s[0];
                }
                __syncthreads();
                continue;
            }
            if (kStage != GIVEN && tid == 0 && number == 0) {
                const float log_z = logf(s[0]);
                // (one tau inside the sum: the square of a small one is zero)
                a.loss[row] = w * tau * (s[2] / s[1] + tau * (log_z - logf(s[1])));
                // (a row of masked logits alone has no distribution; joined parts have summed it to zero)
                a.lse[row] = top[0] == -kInfinity ? __builtin_nanf("") : top[0] / tau + log_z;
            }
            if (g) {
                keep(v);
                const float q = kStage == GIVEN ? w * tau : w * tau / s[0], p = w * tau / s[1];
                const bool same = (((uintptr_t)z ^ (uintptr_t)g) & 15u) == 0;
                char *const grads = reinterpret_cast<char *>(g + split.head);
                auto write = [&](int i, const word &from) {
                    if (tid + i * kThreads >= split.words) return;
                    word x;
#pragma unroll
                    for (int e = 0; e < n; ++e) x[e] = (T)(q * exp2_of((wide((T)from[e]) - top[0]) * c));
                    char *to = grads + (size_t)(i * kThreads) * 16 + own;
                    if (same && a.stream) __builtin_nontemporal_store(x, reinterpret_cast<word *>(to));
                    else if (same) *reinterpret_cast<word *>(to) = x;
                    else __builtin_memcpy(to, &x, sizeof(x));
                };
#pragma unroll
                for (int i = 0; i < kEach; ++i) write(i, v[i]);
#pragma unroll 2
                for (int i = 0; i < kMore; ++i) write(kEach + i, more[i * kThreads + tid]);
                if (edge >= 0) g[edge] = (T)(q * exp2_of((beside - top[0]) * c));
                __syncthreads();               // (the stored columns again, now with the teacher's part)
                for (int i = begin + tid; i < end; i += kThreads) {
                    const int j = a.crd[i] - c0;
                    if (j >= 0 && j < cols)
                        g[j] = (T)(q * exp2_of((wide(z[j]) - top[0]) * c) - p * exp2_of((a.val[i] - top[1]) * c));
                }
            }
            __syncthreads();
        }
}

template <typename T, int kThreads, int kEach, int kMore, Stage kStage> hipError_t run(const DistillArgs &a, int part, int parts, hipStream_t s, int wanted = 0)
{
    // (without a gradient the first part of a row, which writes its loss, is all that is wanted of the last launch)
    const int many = wanted > 0 ? wanted : parts;
    const dim3 grid((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20), (unsigned)(many < 4096 ? many : 4096));
    distill_kernel<T, kThreads, kEach, kMore, kStage><<<grid, kThreads, 0, s>>>(a, part, parts, many);
    return hipGetLastError();
}

// Words that a workgroup of a part has: 256 threads of kPartEach words.
constexpr int kPartEach = 4;
template <typename T> constexpr int kPart = 256 * kPartEach * Word<T>::n;

// Rows that no workgroup holds are cut into parts, and of those that need LDS too, which leave a compute unit one workgroup,
// the few, which would leave compute units idle, and many without a gradient, as nothing has to be held for it.  (us a call,
// held and in parts: 131072 bf16, 64 rows with gradients 23 and 14, 128 28 and 23, 192 30 and 34, 1024 145 and 181; without 64
// rows 14 and 13, 1024 80 and 54.  100000 bf16, 32 rows with 18 and 15; without 12 and 14, 512 27 and 28, 4096 197 and 174.
// Rows in registers are faster held whatever their number: 65536 bf16, 4 rows 12 and 15, without a gradient 4096 112 and 118.)
template <typename T> bool in_parts(int64_t rows, int64_t cols, bool grad)
{
    const int64_t words = cols / Word<T>::n;
    return words > 512 * 32 || (words > 512 * 16 && (grad ? rows <= 128 : rows >= 512));
}

template <typename T> hipError_t forward(const DistillArgs &a, hipStream_t s)
{
    const int64_t words = a.cols / Word<T>::n;
    if (in_parts<T>(a.rows, a.cols, a.grad != nullptr)) {
        const int parts = (int)(((int64_t)a.cols + kPart<T> - 1) / kPart<T>);
        const hipError_t rc = run<T, 256, kPartEach, 0, STATS>(a, kPart<T>, parts, s);
        if (rc != hipSuccess) return rc;
        nacho_host::profile_mark("distill_stats");
        return run<T, 256, kPartEach, 0, APPLY>(a, kPart<T>, parts, s, a.grad ? parts : 1);
    }
    const int part = a.cols > 0 ? a.cols : 1;
    if (words <= 64 * 4) return run<T, 64, 4, 0, WHOLE>(a, part, 1, s);
    if (words <= 256 * 4) return run<T, 256, 4, 0, WHOLE>(a, part, 1, s);
    if (words <= 256 * 8) return run<T, 256, 8, 0, WHOLE>(a, part, 1, s);
    if (words <= 512 * 8) return run<T, 512, 8, 0, WHOLE>(a, part, 1, s);
    if (words <= 512 * 16) return run<T, 512, 16, 0, WHOLE>(a, part, 1, s);
    // (9 words a thread in LDS, 74 KB, are the most that leave a compute unit two workgroups)
    if (words <= 512 * 25) return run<T, 512, 16, 9, WHOLE>(a, part, 1, s);
    return run<T, 512, 16, 16, WHOLE>(a, part, 1, s);
}

template <typename F> hipError_t by_type(int dtype, F f)
{
    if (dtype == NACHO_F32) return f((float)0);
    return dtype == NACHO_BF16 ? f((bf16_t)0.0f) : f((f16_t)0.0f);
}

}  // namespace

int64_t distill_partials(int dtype, int64_t rows, int64_t cols, bool grad)
{
    int64_t parts = 0;
    (void)by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        if (in_parts<T>(rows, cols, grad)) parts = (cols + kPart<T> - 1) / kPart<T>;
        return hipSuccess;
    });
    return 2 * rows * parts;
}

// Gradients that fill the last cache (256 MB) go past it: 1021 x 100003 f16 from the lse 65 us, through it 72; 4096 x 65536
// bf16 with the loss 220 and 226.  Smaller ones may be read from it by what comes next.
bool past_caches(int dtype, const DistillArgs &a) { return a.rows * a.cols > ((int64_t)1 << (dtype == NACHO_F32 ? 25 : 26)); }

hipError_t launch_distill(int dtype, const DistillArgs &args, hipStream_t s)
{
    if (args.rows == 0) return hipSuccess;
    DistillArgs a = args;
    a.stream = past_caches(dtype, a);
    return by_type(dtype, [&](auto zero) { return forward<decltype(zero)>(a, s); });
}

hipError_t launch_distill_grad(int dtype, const DistillArgs &args, hipStream_t s)
{
    if (args.rows == 0 || args.cols == 0) return hipSuccess;
    DistillArgs a = args;
    a.stream = past_caches(dtype, a);
    return by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const int parts = (int)(((int64_t)a.cols + kPart<T> - 1) / kPart<T>);
        return run<T, 256, kPartEach, 0, GIVEN>(a, kPart<T>, parts, s);
    });
}

}  // namespace nacho
