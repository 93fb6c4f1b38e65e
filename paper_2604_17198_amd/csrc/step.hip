// A whole layer of a mixture of experts for a few tokens, in two launches:
//
//   h_te  = act(up_e x_t + b_e),  or  act(gate_e x_t + b'_e) (up_e x_t + b_e)          for every expert e that token t chose
//   out_t = residual_t + sum_e g_te (down_e h_te + c_e)
//
// Few tokens read many weights: each weight that a token chose is read once and multiplied once with every token that chose it,
// and the time is that of reading them.  So a wavefront takes its stretch of 16 rows of weights from memory right into the
// registers that the matrix units read (16 rows x 64 bytes of k an instruction), and the tokens' rows the same way from the
// caches; wavefronts share out k, and their sums meet in LDS.
//
// The choice of experts is made by every workgroup of the first launch for itself: a wavefront a token, a round for each of the
// k largest.  That is less than a launch of its own would take.
#include "activation.hpp"
#include "products.hpp"

namespace nacho {

namespace {

constexpr int kWaves = 8, kThreads = kWaves * NACHO_WAVE;
constexpr int kTall = 16;              // rows of weights a workgroup
constexpr int kMostTokens = kMostStepTokens, kMostSlots = kMostTokens * kMostChoices;
constexpr uint16_t kNone = 0xffff;     // a choice that is not there

// 16 bytes of a row of k elements from element `from` on, zeros behind its end.
template <typename T, Access kAccess> __device__ inline v4u piece(const T *row, int from, int k)
{
    if constexpr (kAccess == WORDS) return from < k ? *reinterpret_cast<const v4u *>(row + from) : v4u{0, 0, 0, 0};
    else {
        const Ragged<T, kAccess == TINY> r(k, from);
        return r.placed(r.load(row + from));
    }
}

// The experts of a wavefront's tokens, into `choice`, and as bits.  `logits`: the wavefront's room for a token's.
template <typename T>
__device__ inline void choose_experts(const StepArgs &a, float *logits, uint16_t *choice, unsigned *bits, bool shares)
{
    const int lane = lane_id(), wave = (int)threadIdx.x / NACHO_WAVE, k = a.top_k, n = a.experts;
    const int each = (n + NACHO_WAVE - 1) / NACHO_WAVE, first = lane * each;       // a lane's experts, one after the other
    for (int t = wave; t < a.tokens; t += kWaves) {
        const bool kept = !a.keep || a.keep[t] != 0;
        const T *row = static_cast<const T *>(a.logits) + t * a.ldl;
        float top = -kInfinity;
        for (int i = 0; i < each; ++i) {
            const int e = first + i;
            const float v = kept && e < n ? wide(row[e]) : -kInfinity;
            logits[e] = v;
            top = fmaxf(top, v);
        }
        // the lane's largest logit that is left, of equal ones the first
        unsigned best = 0, gone = 0;
        int at = first;
        auto look = [&] {
            best = 0;
            for (int i = 0; i < each; ++i) {
                const unsigned key = gone >> i & 1 ? 0u : order_of(logits[first + i]);
                if (key > best) {
                    best = key;
                    at = first + i;
                }
            }
        };
        look();
        int held = 0;
        for (; held < k; ++held) {
            const unsigned most = group_max<NACHO_WAVE>(best);
            if (most == 0) break;
            const int who = __ffsll((long long)__ballot(best == most)) - 1, e = __builtin_amdgcn_readlane(at, who);
            if (lane == 0) {
                choice[t * k + held] = (uint16_t)e;
                atomicOr(&bits[e >> 5], 1u << (e & 31));
            }
            if (lane == who) {
                gone |= 1u << (e - first);
                look();
            }
        }
        if (lane >= held && lane < k) choice[t * k + lane] = kNone;
        wave_sync();
        if (shares) {
            top = group_reduce<NACHO_WAVE>(top, MaxOf());
            auto part = [&](float v) { return v == -kInfinity ? 0.0f : exp2_of((v - top) * kLog2e); };
            float sum = 0.0f;
            for (int i = 0; i < each; ++i) sum += part(logits[first + i]);
            sum = group_reduce<NACHO_WAVE>(sum, SumOf());
            const float mine = lane < held ? part(logits[choice[t * k + lane]]) : 0.0f;
            float whole = group_reduce<NACHO_WAVE>(mine, SumOf());
            whole = !a.normalise || sum != sum ? sum : whole;                      // (a NaN among the logits)
            if (lane < k) a.share[t * k + lane] = lane < held ? mine / whole : 0.0f;
        }
        wave_sync();
    }
}

// The slots (token x k + choice) that chose expert e, by tokens; how many they are.  All lanes of a wavefront.
__device__ inline int slots_of(const StepArgs &a, const uint16_t *choice, int e, int16_t *list)
{
    const int lane = lane_id(), k = a.top_k;
    int slot = -1;
    if (lane < a.tokens)
        for (int j = 0; j < k; ++j)
            if (choice[lane * k + j] == e) slot = lane * k + j;
    const unsigned long long who = __ballot(slot >= 0);
    const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0));
    if (slot >= 0) list[before] = (int16_t)slot;
    return __popcll((long long)who);
}

template <typename T, bool kGated, Access kAccess> __global__ void __launch_bounds__(kThreads) step_up_kernel(StepArgs a)
{
    __shared__ __attribute__((aligned(16))) char room[kWaves * kMostExperts * 4];
    __shared__ uint16_t choice[kMostSlots], active[kMostExperts];
    __shared__ unsigned bits[kMostExperts / 32];
    __shared__ int16_t list[kMostTokens];
    __shared__ int members;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid / NACHO_WAVE, k = a.top_k;
    if (tid < kMostExperts / 32) bits[tid] = 0;
    __syncthreads();
    choose_experts<T>(a, reinterpret_cast<float *>(room) + wave * kMostExperts, choice, bits, blockIdx.x == 0);
    __syncthreads();
    int count = 0;
    for (int w = 0; w < kMostExperts / 32; ++w) count += __popc(bits[w]);
    for (int e = tid; e < a.experts; e += kThreads)
        if (bits[e >> 5] >> (e & 31) & 1) {
            int place = __popc(bits[e >> 5] & ((1u << (e & 31)) - 1u));
            for (int w = 0; w < e >> 5; ++w) place += __popc(bits[w]);
            active[place] = (uint16_t)e;
        }
    __syncthreads();
    if (blockIdx.x == 0) {
        // what the second launch needs of the choice
        if (tid == 0) a.active[0] = count;
        for (int i = tid; i < count; i += kThreads) a.active[1 + i] = active[i];
        for (int i = tid; i < a.tokens * k; i += kThreads) a.choice[i] = choice[i];
        for (int i = tid; i < a.tiles; i += kThreads) a.arrived[i] = 0;
    }
    constexpr int n = Word<T>::n, kStep = 64 / (int)sizeof(T), kBatch = 4;
    const int tiles = (a.hidden + kTall - 1) / kTall, steps = (a.inner + kStep - 1) / kStep, pairs = (steps + 1) / 2;
    const int begin = pairs * wave / kWaves * 2, until = pairs * (wave + 1) / kWaves * 2, end = until < steps ? until : steps;
    v4f *const sums = reinterpret_cast<v4f *>(room);                               // [2][kWaves][64]
    for (int item = (int)blockIdx.x; item < count * tiles; item += (int)gridDim.x) {
        const int number = item / tiles, row0 = (item - number * tiles) * kTall, e = active[number];
        if (wave == 0) {
            const int m = slots_of(a, choice, e, list);
            if (lane == 0) members = m;
        }
        __syncthreads();
        const int m = members, row = row0 + lane % 16 < a.hidden ? row0 + lane % 16 : a.hidden - 1, off = lane / 16 * n;
        const T *up = static_cast<const T *>(a.up.w) + e * a.up.stride + row * a.up.ld;
        const T *gate = kGated ? static_cast<const T *>(a.gate.w) + e * a.gate.stride + row * a.gate.ld : up;
        auto groups_of = [&](auto most) {
            constexpr int kGroups = decltype(most)::value;
            v4f acc[kGroups][2];
            const T *x[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                acc[g][0] = acc[g][1] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                const int i = g * 16 + lane % 16;
                x[g] = static_cast<const T *>(a.x) + list[i < m ? i : m - 1] / k * a.ldx;
            }
            for (int s = begin; s < end; s += kBatch) {
                v4u p[kBatch], q[kBatch], r[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int from = s + i < end ? (s + i) * kStep + off : a.inner;
                    p[i] = piece<T, kAccess>(up, from, a.inner);
                    if (kGated) r[i] = piece<T, kAccess>(gate, from, a.inner);
                }
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (kGroups > 1 && g * 16 >= m) break;
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) q[i] = piece<T, kAccess>(x[g], s + i < end ? (s + i) * kStep + off : a.inner, a.inner);
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        acc[g][0] = matrix_step<T>(p[i], q[i], acc[g][0]);
                        if (kGated) acc[g][1] = matrix_step<T>(r[i], q[i], acc[g][1]);
                    }
                }
            }
            // 16 tokens at a time: a thread adds up the wavefronts' sums of one token and one row
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                if (g * 16 >= m) break;
                sums[wave * NACHO_WAVE + lane] = acc[g][0];
                if (kGated) sums[(kWaves + wave) * NACHO_WAVE + lane] = acc[g][1];
                __syncthreads();
                const int r = tid % kTall, token = tid / kTall, i = g * 16 + token, out = row0 + r;
                if (tid < 16 * kTall && i < m && out < a.hidden) {
                    const float *from = reinterpret_cast<const float *>(sums) + (token + r / 4 * 16) * 4 + r % 4;
                    float v[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int h = 0; h < 1 + kGated; ++h)
#pragma unroll
                        for (int w = 0; w < kWaves; ++w) v[h] += from[(h * kWaves + w) * NACHO_WAVE * 4];
                    if (a.up.bias) v[0] += wide(static_cast<const T *>(a.up.bias)[e * a.up.bias_stride + out]);
                    if (kGated) {
                        if (a.gate.bias) v[1] += wide(static_cast<const T *>(a.gate.bias)[e * a.gate.bias_stride + out]);
                        v[0] *= activated<T>(v[1], a.act);
                    } else v[0] = activated<T>(v[0], a.act);
                    static_cast<T *>(a.h)[list[i] * a.ldh + out] = (T)v[0];
                }
                __syncthreads();
            }
        };
        if (m <= 16) groups_of(std::integral_constant<int, 1>());
        else groups_of(std::integral_constant<int, kMostTokens / 16>());
    }
}

template <typename T, Access kAccess> __global__ void __launch_bounds__(kThreads) step_down_kernel(StepArgs a)
{
    constexpr int kSlab = kMostTokens * kTall, kGroups = kMostTokens / 16;
    __shared__ __attribute__((aligned(16))) float slab[kWaves][kSlab];             // [token][row] of every wavefront
    __shared__ float share[kMostSlots];
    __shared__ uint16_t choice[kMostSlots], active[kMostExperts];
    __shared__ int16_t lists[kWaves][kMostTokens];
    __shared__ int last;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid / NACHO_WAVE, k = a.top_k;
    const int tile = (int)blockIdx.x, part = (int)blockIdx.y, parts = (int)gridDim.y, row0 = tile * kTall, count = a.active[0];
    for (int i = tid; i < a.tokens * k; i += kThreads) {
        choice[i] = a.choice[i];
        share[i] = a.share[i];
    }
    for (int i = tid; i < count; i += kThreads) active[i] = (uint16_t)a.active[1 + i];
    for (int i = lane; i < a.tokens * kTall; i += NACHO_WAVE) slab[wave][i] = 0.0f;
    __syncthreads();
    // a unit of work: eight steps of k of one expert; a wavefront has consecutive ones
    constexpr int n = Word<T>::n, kStep = 64 / (int)sizeof(T), kBatch = 8;
    const int units = (a.hidden + kStep * kBatch - 1) / (kStep * kBatch), all = count * units;
    const int workers = parts * kWaves, worker = part * kWaves + wave;
    const int begin = (int)((int64_t)all * worker / workers), end = (int)((int64_t)all * (worker + 1) / workers);
    const int row = row0 + lane % 16 < a.outer ? row0 + lane % 16 : a.outer - 1, off = lane / 16 * n;
    int16_t *const list = lists[wave];
    int number = -1, m = 0;
    v4f acc[kGroups];
    auto add_up = [&] {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int i = g * 16 + lane % 16;
            if (i < m) {
                const int slot = list[i];
                v4f *to = reinterpret_cast<v4f *>(&slab[wave][slot / k * kTall + lane / 16 * 4]);
                const float by = share[slot];
                v4f v = *to;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += by * acc[g][j];
                *to = v;
            }
        }
    };
    for (int u = begin; u < end; ++u) {
        const int expert = u / units, from = (u - expert * units) * kBatch * kStep + off, e = active[expert];
        const T *down = static_cast<const T *>(a.down.w) + e * a.down.stride + row * a.down.ld;
        v4u p[kBatch], q[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) p[i] = piece<T, kAccess>(down, from + i * kStep, a.hidden);
        if (expert != number) {
            if (number >= 0) add_up();
            wave_sync();
            number = expert;
            m = slots_of(a, choice, e, list);
            wave_sync();
#pragma unroll
            for (int g = 0; g < kGroups; ++g) acc[g] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g * 16 >= m) break;
            const int i = g * 16 + lane % 16;
            const T *h = static_cast<const T *>(a.h) + list[i < m ? i : m - 1] * a.ldh;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) q[j] = piece<T, kAccess>(h, from + j * kStep, a.hidden);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) acc[g] = matrix_step<T>(p[j], q[j], acc[g]);
        }
    }
    if (number >= 0) add_up();
    __syncthreads();
    // the sum of the wavefronts' parts; of several workgroups the last one to be there adds up all of theirs
    auto finish = [&](int t, int r, float v) {
        const int out = row0 + r;
        if (a.down.bias)
            for (int j = 0; j < k; ++j)
                if (const int e = choice[t * k + j]; e != kNone)
                    v += share[t * k + j] * wide(static_cast<const T *>(a.down.bias)[e * a.down.bias_stride + out]);
        if (a.residual) v += wide(static_cast<const T *>(a.residual)[t * a.ldr + out]);
        static_cast<T *>(a.out)[t * a.ldo + out] = (T)v;
    };
    float *const mine = parts > 1 ? a.partial + ((int64_t)tile * parts + part) * a.tokens * kTall : nullptr;
    for (int i = tid; i < a.tokens * kTall; i += kThreads) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += slab[w][i];
        if (parts > 1) __hip_atomic_store(&mine[i], v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        else if (row0 + i % kTall < a.outer) finish(i / kTall, i % kTall, v);
    }
    if (parts == 1) return;
    // (Stores and loads of the sums are atomic ones, which go past the caches that a part of the chip has for itself; so it is enough that
    // every store is there before the workgroup is counted.  A fence would write back and drop these caches, once a wavefront: 64 tokens, 8
    // of 128 experts, 237 us with fences.)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) last = __hip_atomic_fetch_add(&a.arrived[tile], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    if (!last) return;
    for (int i = tid; i < a.tokens * kTall; i += kThreads) {
        float v = 0.0f;
        for (int p = 0; p < parts; ++p)
            v += __hip_atomic_load(&a.partial[((int64_t)tile * parts + p) * a.tokens * kTall + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (row0 + i % kTall < a.outer) finish(i / kTall, i % kTall, v);
    }
}

// The most experts that tokens can reach.
int64_t most_active(int64_t tokens, int64_t experts, int64_t top_k) { return tokens * top_k < experts ? tokens * top_k : experts; }

template <typename T, Access kAccess> hipError_t run_step(const StepArgs &a, hipStream_t s)
{
    const int64_t items = most_active(a.tokens, a.experts, a.top_k) * ((a.hidden + kTall - 1) / kTall);
    const unsigned groups = (unsigned)(items < 2 * kUnits ? items : 2 * kUnits);
    if (a.gate.w) step_up_kernel<T, true, kAccess><<<groups, kThreads, 0, s>>>(a);
    else step_up_kernel<T, false, kAccess><<<groups, kThreads, 0, s>>>(a);
    if (const hipError_t e = hipGetLastError()) return e;
    step_down_kernel<T, kAccess><<<dim3((unsigned)a.tiles, (unsigned)a.parts), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

void step_plan(int dtype, int64_t tokens, int64_t experts, int64_t top_k, int64_t hidden, int64_t outer, int32_t *tiles, int32_t *parts)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    *tiles = (int32_t)((outer + kTall - 1) / kTall);
    // workgroups for every compute unit, as long as each of their wavefronts has something to read
    const int64_t units = most_active(tokens, experts, top_k) * ((hidden * elem + 511) / 512), wanted = (2 * kUnits + *tiles - 1) / *tiles;
    const int64_t most = units / kWaves < 16 ? units / kWaves : 16;
    *parts = (int32_t)(wanted < most ? wanted : (most > 1 ? most : 1));
}

hipError_t launch_step(int dtype, const StepArgs &a, hipStream_t s)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    const bool words = in_words({{a.x, a.ldx}, {a.up.w, a.up.ld}, {a.up.w, a.up.stride}, {a.gate.w, a.gate.ld}, {a.gate.w, a.gate.stride}, {a.down.w, a.down.ld},
                                 {a.down.w, a.down.stride}, {a.x, a.inner}, {a.x, a.hidden}}, elem);
    const bool tiny = a.inner * elem < 16 || a.hidden * elem < 16;
    hipError_t rc = hipSuccess;
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        rc = words ? run_step<T, WORDS>(a, s) : tiny ? run_step<T, TINY>(a, s) : run_step<T, ANYWHERE>(a, s);
    });
    return rc;
}

}  // namespace nacho
