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
// The choice of experts is made by every workgroup of the first launch for itself, which takes less than a launch of its own.
//
// The rows between the products are rounded to the type because the matrix units take it, and because a second launch reads them: results in
// bf16 are off by 1.8e-3 (their own rounding is 1.7e-3), in f16 by 2.1e-4 (2.1e-4).
//
// Bound by the weights' bytes.  us a kernel: 64 tokens, 8 of 128 experts, gated, 2048 x 1024 x 2048 f16 (all 1.6 GB of weights) 175 and 82,
// 6.3 TB/s; 16 tokens, 2 of 32 experts, 2048 x 4096 x 2048 bf16 69 and 55; one token, 8 of 64 experts, gated, 2048 x 1024 x 2048, 101 MB that the
// last cache holds, 19 and 11.
#include "activation.hpp"
#include "choose.hpp"
#include "products.hpp"

namespace nacho {

namespace {

constexpr int kWaves = 8, kThreads = kWaves * NACHO_WAVE;
constexpr int kTall = 16;              // rows of weights that a wavefront multiplies at a time
constexpr int kMostTokens = kMostStepTokens, kMostSlots = kMostTokens * kMostChoices;
constexpr uint16_t kNone = 0xffff;     // a choice that is not there

// The experts of every token, ascending, into `choice`; how many tokens chose each; and the gates, of one workgroup.
template <typename T, int L, int I> __device__ inline void choose_experts(const StepArgs &a, uint16_t *choice, int *takers, bool shares)
{
    constexpr int kGroups = kThreads / L;
    const int tid = (int)threadIdx.x, group = tid / L, lane = tid % L, first = lane * I, n = a.experts, k = a.top_k;
    const T *logits = static_cast<const T *>(a.logits);
    const bool words = nacho::in_words<T, I>(logits, a.ldl);
    // (every lane of a wavefront stays in the loop: the lanes of a group ask each other)
    for (int t0 = 0; t0 < a.tokens; t0 += kGroups) {
        const int t = t0 + group;
        const bool there = t < a.tokens, live = there && (!a.keep || a.keep[t] != 0);
        float v[I];
        if (live) row_part<T, I>(logits + t * a.ldl, first, n, words, v);
        else {
#pragma unroll
            for (int i = 0; i < I; ++i) v[i] = -kInfinity;
        }
        const unsigned taken = choose<L, I>(v, k);
        // places of the lane's entries among the token's: those of the lanes before it come first
        const int own = __popc(taken), upto = group_scan<L>(own), held = __shfl(upto, L - 1, L);
        int place = t * k + upto - own;
        for (unsigned rest = taken; rest != 0; rest &= rest - 1, ++place) {
            const int e = first + __ffs((int)rest) - 1;
            choice[place] = (uint16_t)e;
            atomicAdd(&takers[e], 1);
        }
        for (int j = held + lane; there && j < k; j += L) choice[t * k + j] = kNone;
        if (!shares) continue;
        float e[I], top, sum, whole = 0.0f;
        exponentials<L, I>(v, e, top, sum);
#pragma unroll
        for (int i = 0; i < I; ++i) whole += taken >> i & 1 ? e[i] : 0.0f;
        whole = group_reduce<L>(whole, SumOf());
        whole = !a.normalise || sum != sum ? sum : whole;                          // (a NaN among the logits)
        place = t * k + upto - own;
        for (unsigned rest = taken; rest != 0; rest &= rest - 1, ++place) {
            const int at = __ffs((int)rest) - 1;
            float mine = e[0];
#pragma unroll
            for (int i = 1; i < I; ++i) mine = at == i ? e[i] : mine;
            a.share[place] = mine / whole;
        }
        for (int j = held + lane; there && j < k; j += L) a.share[t * k + j] = 0.0f;
    }
}

// The slots (token x k + choice) that chose expert e, by tokens.  All lanes of a wavefront.
__device__ inline int slots_of(const StepArgs &a, const uint16_t *choice, int e, uint16_t *list)
{
    const int lane = lane_id(), k = a.top_k;
    int slot = -1;
    if (lane < a.tokens)
        for (int j = 0; j < k; ++j)
            if (choice[lane * k + j] == e) slot = lane * k + j;
    const unsigned long long who = __ballot(slot >= 0);
    const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0));
    if (slot >= 0) list[before] = (uint16_t)slot;
    return __popcll((long long)who);
}

// The first product.  An item is 16 rows of an expert's weights, and belongs to a wavefront, or, where there are few items, to a
// workgroup whose wavefronts have a part of k each (kShared).
template <typename T, bool kGated, Access kAccess, bool kShared>
__global__ void __launch_bounds__(kThreads, 2) step_up_kernel(StepArgs a)
{
    constexpr int kMatrices = 1 + kGated;
    typedef Stretch<T, kAccess, 2> Part;
    constexpr int kBatch = Part::kBatch;
    __shared__ __attribute__((aligned(16))) v4f sums[kShared ? kMatrices * kWaves * NACHO_WAVE : 1];
    __shared__ uint16_t choice[kMostSlots], active[kMostExperts], lists[kWaves][kMostTokens];
    __shared__ int takers[kMostExperts], counts[kThreads / NACHO_WAVE];
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / NACHO_WAVE), k = a.top_k;
    for (int e = tid; e < a.experts; e += kThreads) takers[e] = 0;
    __syncthreads();
    if (a.experts <= 64) choose_experts<T, 16, 4>(a, choice, takers, blockIdx.x == 0);
    else if (a.experts <= 256) choose_experts<T, 16, 16>(a, choice, takers, blockIdx.x == 0);
    else choose_experts<T, 64, 16>(a, choice, takers, blockIdx.x == 0);
    __syncthreads();
    // the experts that a token chose, ascending
    int count = 0;
    for (int e0 = 0; e0 < a.experts; e0 += kThreads) {
        const int e = e0 + tid;
        const unsigned long long chosen = __ballot(e < a.experts && takers[e] > 0);
        if (lane == 0) counts[wave] = __popcll((long long)chosen);
        __syncthreads();
        int place = count + __builtin_amdgcn_mbcnt_hi((unsigned)(chosen >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)chosen, 0));
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) place += counts[w];
            count += counts[w];
        }
        if (e < a.experts && takers[e] > 0) active[place] = (uint16_t)e;
        __syncthreads();
    }
    if (blockIdx.x == 0) {
        // what the second launch needs of the choice
        if (tid == 0) a.active[0] = count;
        for (int i = tid; i < count; i += kThreads) a.active[1 + i] = active[i];
        for (int i = tid; i < a.tokens * k; i += kThreads) a.choice[i] = choice[i];
        for (int i = tid; i < a.tiles; i += kThreads) a.arrived[i] = 0;
        int before = 0;
        for (int i = 0; i < count; i += NACHO_WAVE) {
            const int mine = i + lane < count ? takers[active[i + lane]] : 0, upto = before + wave_inclusive_scan(mine);
            if (wave == 0 && i + lane < count) a.first[i + lane] = upto - mine;
            for (int j = wave; j < NACHO_WAVE && i + j < count; j += kWaves)
                slots_of(a, choice, active[i + j], a.order + __builtin_amdgcn_readlane(upto - mine, j));
            before = __builtin_amdgcn_readlane(upto, NACHO_WAVE - 1);
        }
        if (tid == 0) a.first[count] = before;
    }
    const int tiles = (a.hidden + kTall - 1) / kTall, stretches = (a.inner + Part::kLong - 1) / Part::kLong, items = count * tiles;
    const int begin = kShared ? stretches * wave / kWaves : 0, end = kShared ? stretches * (wave + 1) / kWaves : stretches;
    uint16_t *const list = lists[wave];
    const int step = (int)gridDim.x * (kShared ? 1 : kWaves);
    for (int item = kShared ? (int)blockIdx.x : (int)blockIdx.x + (int)gridDim.x * wave; item < items; item += step) {
        const int number = item / tiles, row0 = (item - number * tiles) * kTall, e = __builtin_amdgcn_readfirstlane(active[number]);
        const int row = row0 + lane % 16 < a.hidden ? row0 + lane % 16 : a.hidden - 1;
        const T *rows[kMatrices];
        rows[0] = static_cast<const T *>(a.up.w) + e * a.up.stride + row * a.up.ld;
        if constexpr (kGated) rows[1] = static_cast<const T *>(a.gate.w) + e * a.gate.stride + row * a.gate.ld;
        auto groups_of = [&](auto most) {
            constexpr int kGroups = decltype(most)::value;
            struct Loaded {
                typename Part::Loaded p[kMatrices][kBatch], q[kBatch];
            } one, two;
            v4f acc[kGroups][kMatrices];
            int token[kGroups];
            int m = 0;
            auto fetch_rows = [&](Loaded &to, int s) {
#pragma unroll
                for (int h = 0; h < kMatrices; ++h)
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) to.p[h][i] = Part::load(rows[h], Part::from(s, i), a.inner);
            };
            auto fetch_x = [&](Loaded &to, int s, int g) {
                const T *x = static_cast<const T *>(a.x) + token[g] * a.ldx;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) to.q[i] = Part::load(x, Part::from(s, i), a.inner);
            };
            auto multiply = [&](Loaded &of, int s) {
                v4u p[kMatrices][kBatch];
                Part::by_end(s, a.inner, [&](auto whole) {
#pragma unroll
                    for (int h = 0; h < kMatrices; ++h)
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) p[h][i] = Part::value(of.p[h][i], rows[h], Part::from(s, i), a.inner, whole);
                });
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (g > 0) {
                        if (g * 16 >= m) break;
                        fetch_x(of, s, g);
                    }
                    const T *x = static_cast<const T *>(a.x) + token[g] * a.ldx;
                    v4u q[kBatch];
                    Part::by_end(s, a.inner, [&](auto whole) {
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) q[i] = Part::value(of.q[i], x, Part::from(s, i), a.inner, whole);
                    });
#pragma unroll
                    for (int i = 0; i < kBatch; ++i)
#pragma unroll
                        for (int h = 0; h < kMatrices; ++h) acc[g][h] = matrix_step<T>(p[h][i], q[i], acc[g][h]);
                }
            };
            // (weights first: they have the longest way)
            // (every wavefront starts somewhere else along k: rows are often a power of two apart, and so would be what is read at a time)
            const int turn = kShared ? 0 : item % stretches;
            auto at = [&](int s) {
                const int t = (s < end ? s : end - 1) + turn;      // (behind the last stretch it is loaded again: no branch around a load)
                return kShared || t < stretches ? t : t - stretches;
            };
            if (begin < end) fetch_rows(one, at(begin));
            m = slots_of(a, choice, e, list);
            wave_sync();
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int i = g * 16 + lane % 16;
                token[g] = list[i < m ? i : m - 1] / k;
#pragma unroll
                for (int h = 0; h < kMatrices; ++h) acc[g][h] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            }
            if (begin < end) fetch_x(one, at(begin), 0);
            for (int s = begin; s < end; s += 2) {
                fetch_rows(two, at(s + 1));
                fetch_x(two, at(s + 1), 0);
                multiply(one, at(s));
                fetch_rows(one, at(s + 2));
                fetch_x(one, at(s + 2), 0);
                if (s + 1 < end) multiply(two, at(s + 1));
            }
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                if (g * 16 >= m) break;
                if constexpr (kShared) {
                    __syncthreads();
#pragma unroll
                    for (int h = 0; h < kMatrices; ++h) sums[(h * kWaves + wave) * NACHO_WAVE + lane] = acc[g][h];
                    __syncthreads();
                    if (wave != 0) continue;
#pragma unroll
                    for (int h = 0; h < kMatrices; ++h) {
                        acc[g][h] = sums[h * kWaves * NACHO_WAVE + lane];
#pragma unroll
                        for (int w = 1; w < kWaves; ++w) acc[g][h] += sums[(h * kWaves + w) * NACHO_WAVE + lane];
                    }
                }
                // a lane has four rows of one token
                const int i = g * 16 + lane % 16, out = row0 + lane / 16 * 4;
                if (i >= m || out >= a.ldh) continue;
                typedef T four __attribute__((ext_vector_type(4)));
                four v;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float z[kMatrices];
#pragma unroll
                    for (int h = 0; h < kMatrices; ++h) {
                        const nacho_dense &d = h == 0 ? a.up : a.gate;
                        z[h] = acc[g][h][j];
                        if (d.bias && out + j < a.hidden) z[h] += wide(static_cast<const T *>(d.bias)[e * d.bias_stride + out + j]);
                    }
                    const float h = kGated ? activated<T>(z[kMatrices - 1], a.act) * z[0] : activated<T>(z[0], a.act);
                    v[j] = (T)(out + j < a.hidden ? h : 0.0f);
                }
                // (rows are whole words of 8 elements, with zeros behind the last)
                *reinterpret_cast<four *>(static_cast<T *>(a.h) + list[i] * a.ldh + out) = v;
            }
            wave_sync();
        };
        if (__builtin_amdgcn_readfirstlane(takers[e]) <= 16) groups_of(std::integral_constant<int, 1>());
        else groups_of(std::integral_constant<int, kMostTokens / 16>());
    }
}

// The second product and the weighted sum.  A workgroup has 16 rows of every chosen expert's weights, or a part of their k (with
// others, `parts` of them); its wavefronts share out what it has, a stretch of k of an expert at a time, and keep sums of their own
// for every token in LDS.
template <typename T, Access kAccess> __global__ void __launch_bounds__(kThreads, 2) step_down_kernel(StepArgs a)
{
    typedef Stretch<T, kAccess, kAccess == WORDS ? 4 : 2> Part;
    typedef Stretch<T, WORDS, Part::kBatch> Whole;                                 // (the rows between the products)
    constexpr int kSlab = kMostTokens * kTall, kGroups = kMostTokens / 16, kBatch = Part::kBatch;
    __shared__ __attribute__((aligned(16))) float slab[kWaves][kSlab];             // [token][row] of every wavefront
    __shared__ float share[kMostSlots];
    __shared__ uint16_t order[kMostSlots], active[kMostExperts];
    __shared__ int firsts[kMostExperts + 1], last;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / NACHO_WAVE), k = a.top_k;
    const int tile = (int)blockIdx.x, part = (int)blockIdx.y, parts = (int)gridDim.y, row0 = tile * kTall, count = a.active[0];
    const int slots = a.tokens * k, most = slots < a.experts ? slots : a.experts;
    for (int i = tid; i < slots; i += kThreads) {
        order[i] = a.order[i];
        share[i] = a.share[i];
    }
    // (as many as there can be: nothing waits for how many there are)
    for (int i = tid; i <= most; i += kThreads) {
        firsts[i] = a.first[i];
        if (i < most) active[i] = (uint16_t)a.active[1 + i];
    }
    for (int i = lane; i < a.tokens * kTall; i += NACHO_WAVE) slab[wave][i] = 0.0f;
    __syncthreads();
    const int units = (a.hidden + Part::kLong - 1) / Part::kLong, all = count * units;
    const int workers = parts * kWaves, worker = part * kWaves + wave;
    const int begin = (int)((int64_t)all * worker / workers), end = (int)((int64_t)all * (worker + 1) / workers);
    const int row = row0 + lane % 16 < a.outer ? row0 + lane % 16 : a.outer - 1;
    struct Unit {
        int expert, stretch;       // (the expert by its number among the chosen ones)
    };
    struct Loaded {
        Unit at;
        const T *row;
        typename Part::Loaded p[kBatch];
        v4u q[kBatch];
    } one, two;
    v4f acc[kGroups];
    auto slot_of = [&](int expert, int g) {
        const int first = firsts[expert], m = firsts[expert + 1] - first, i = g * 16 + lane % 16;
        return order[first + (i < m ? i : m - 1)];
    };
    auto row_of = [&](int expert, int g) { return static_cast<const T *>(a.h) + slot_of(expert, g) * a.ldh; };
    auto fetch = [&](Loaded &to, Unit at) {
        to.at = at;
        const int e = __builtin_amdgcn_readfirstlane(active[at.expert]);
        to.row = static_cast<const T *>(a.down.w) + e * a.down.stride + row * a.down.ld;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) to.p[i] = Part::load(to.row, Part::from(at.stretch, i), a.hidden);
        const T *h = row_of(at.expert, 0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) to.q[i] = Whole::load(h, Part::from(at.stretch, i), (int)a.ldh);
    };
    auto add_up = [&](int expert) {
        const int m = __builtin_amdgcn_readfirstlane(firsts[expert + 1] - firsts[expert]);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g * 16 >= m) break;
            if (g * 16 + lane % 16 < m) {
                const int slot = slot_of(expert, g);
                v4f *to = reinterpret_cast<v4f *>(&slab[wave][slot / k * kTall + lane / 16 * 4]);
                const float by = share[slot];
                v4f v = *to;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += by * acc[g][j];
                *to = v;
            }
        }
    };
    int number = -1;
    auto multiply = [&](Loaded &of) {
        const Unit at = of.at;
        if (at.expert != number) {
            if (number >= 0) add_up(number);
            number = at.expert;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) acc[g] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int m = __builtin_amdgcn_readfirstlane(firsts[number + 1] - firsts[number]);
        v4u p[kBatch];
        Part::by_end(at.stretch, a.hidden, [&](auto whole) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) p[i] = Part::value(of.p[i], of.row, Part::from(at.stretch, i), a.hidden, whole);
        });
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g > 0) {
                if (g * 16 >= m) break;
                const T *h = row_of(number, g);
#pragma unroll
                for (int i = 0; i < kBatch; ++i) of.q[i] = Whole::load(h, Part::from(at.stretch, i), (int)a.ldh);
            }
            Part::by_end(at.stretch, a.hidden, [&](auto whole) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) of.q[i] = Whole::value(of.q[i], nullptr, Part::from(at.stretch, i), (int)a.ldh, whole);
            });
#pragma unroll
            for (int i = 0; i < kBatch; ++i) acc[g] = matrix_step<T>(p[i], of.q[i], acc[g]);
        }
    };
    if (begin < end) {
        auto behind = [&](Unit at) { return at.stretch + 1 < units ? Unit{at.expert, at.stretch + 1} : Unit{at.expert + 1, 0}; };
        Unit at{begin / units, 0};
        at.stretch = begin - at.expert * units;
        fetch(one, at);
        for (int u = begin; u < end; u += 2) {
            // (behind the last unit it is loaded again: no branch around a load)
            if (u + 1 < end) at = behind(at);
            fetch(two, at);
            multiply(one);
            if (u + 2 < end) at = behind(at);
            fetch(one, at);
            if (u + 1 < end) multiply(two);
        }
        add_up(number);
    }
    __syncthreads();
    // the sum of the wavefronts' parts; of several workgroups the last one to be there adds up all of theirs
    auto finish = [&](int t, int r, float v) {
        const int out = row0 + r;
        if (a.down.bias)
            for (int j = 0; j < k; ++j)
                if (const int e = a.choice[t * k + j]; e != kNone)
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

// Below this number of items (of 16 rows) a workgroup has one at a time.  (2048 x 1024 bf16 gated, us a call with one a workgroup and with
// one a wavefront, a graph's start included: 256 items 24 and 41, 512 items 34 and 55, 1024 items 52 and 56, 2048 items 76 and 72, 4096
// items 103 and 99.)
constexpr int64_t kSharedBelow = 2048;

// The most experts that tokens can reach.
int64_t most_active(int64_t tokens, int64_t experts, int64_t top_k) { return tokens * top_k < experts ? tokens * top_k : experts; }

template <typename T, Access kAccess> hipError_t run_step(const StepArgs &a, hipStream_t s)
{
    const int64_t items = most_active(a.tokens, a.experts, a.top_k) * ((a.hidden + kTall - 1) / kTall);
    const bool shared = items < kSharedBelow;
    const int64_t groups = shared ? items : (items + kWaves - 1) / kWaves;
    auto up = [&](auto gated, auto together) {
        step_up_kernel<T, decltype(gated)::value, kAccess, decltype(together)::value>
            <<<(unsigned)(groups < 2 * kUnits ? groups : 2 * kUnits), kThreads, 0, s>>>(a);
    };
    auto up_of = [&](auto gated) { shared ? up(gated, std::true_type()) : up(gated, std::false_type()); };
    a.gate.w ? up_of(std::true_type()) : up_of(std::false_type());
    if (const hipError_t e = hipGetLastError()) return e;
    step_down_kernel<T, kAccess><<<dim3((unsigned)a.tiles, (unsigned)a.parts), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

void step_plan(int dtype, int64_t tokens, int64_t experts, int64_t top_k, int64_t hidden, int64_t outer, int32_t *tiles, int32_t *parts)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    *tiles = (int32_t)((outer + kTall - 1) / kTall);
    // workgroups for every compute unit, as long as each of their wavefronts has something to read (2048 x 4096 x 2048 bf16, us a call so and
    // with one workgroup for 16 rows: 1 token, 2 experts 35 and 37; 64 tokens, 32 experts 189 and 244; with twice as many parts 1 token 35.5)
    const int64_t units = most_active(tokens, experts, top_k) * ((hidden * elem + 255) / 256), wanted = (kUnits + *tiles - 1) / *tiles;
    const int64_t each = units / (2 * kWaves), most = each < 16 ? each : 16;
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
        const Access access = stretch_access(words, tiny, elem, a.x, a.up.w, a.gate.w, a.down.w);
        rc = access == WORDS ? run_step<T, WORDS>(a, s) : access == TINY ? run_step<T, TINY>(a, s) : run_step<T, ANYWHERE>(a, s);
    });
    return rc;
}

}  // namespace nacho
