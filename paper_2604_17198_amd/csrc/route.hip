// The routing matrix of a mixture of experts: top-k of every token's logits, gates, the transposed order, counts and the
// balance loss; and the gradient of the logits.
//
// L lanes hold a token's logits, I consecutive experts a lane, so that an expert's running sums stay in one lane's
// registers over all tokens of a group of lanes.  Three kernels: every workgroup chooses for a stretch of consecutive
// tokens and leaves its counts by expert; one wavefront an expert turns these into the entries before every workgroup;
// every workgroup then knows where its entries lie in both orders.  Few tokens are one workgroup's, in one launch (16 x 64
// bf16: 15.6 us a call, in three launches 22).  All sums are in a fixed order.
//
// Bound by instructions: 65536 x 128 floats, 8 each, 23 to 25 us to choose (the logits are 6 us of memory), 9 for
// the scan, 9 to place, and 21 to 22 for the gradient, which waits for a token's entries before it can weigh them (11 us of memory).
#include "choose.hpp"
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 64;             // tokens whose entries are placed at a time

// I consecutive elements of a row into it, those behind `n` left out.
template <typename T, int I> __device__ inline void put_row_part(T *row, int at, int n, bool words, const float (&v)[I])
{
    constexpr int kBytes = I * (int)sizeof(T) < 16 ? I * (int)sizeof(T) : 16, kEach = kBytes / (int)sizeof(T);
    typedef T part __attribute__((ext_vector_type(kEach)));
    if (words && at + I <= n) {
#pragma unroll
        for (int i = 0; i < I; i += kEach) {
            part p;
#pragma unroll
            for (int e = 0; e < kEach; ++e) p[e] = (T)v[i + e];
            *reinterpret_cast<part *>(row + at + i) = p;
        }
    } else {
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (at + i < n) row[at + i] = (T)v[i];
    }
}

// A workgroup's stretch of tokens: their experts and gates, and its counts and sums by expert.
template <typename T, int L, int I> __device__ inline void choose_stretch(const RouteArgs &a, const RouteScratch &w)
{
    constexpr int kGroups = kThreads / L, kSlots = L * I;
    __shared__ int hist[kSlots];
    __shared__ float shares[kGroups][kSlots + 1];
    __shared__ int totals[2];
    const int tid = (int)threadIdx.x, group = tid / L, lane = tid % L, first = lane * I, n = a.experts, k = a.top_k;
    for (int i = tid; i < kSlots; i += kThreads) hist[i] = 0;
    if (tid < 2) totals[tid] = 0;
    __syncthreads();
    const int64_t begin = (int64_t)blockIdx.x * w.per_group;
    const int64_t end = begin + w.per_group < a.tokens ? begin + w.per_group : a.tokens;
    const T *logits = static_cast<const T *>(a.logits);
    const bool words = in_words<T, I>(logits, a.ldl);
    float share[I];
#pragma unroll
    for (int i = 0; i < I; ++i) share[i] = 0.0f;
    int entries = 0, routed = 0;
    // (every lane of a wavefront stays in the loop: the lanes of a group ask each other; the next token is on its way)
    auto fetch = [&](int64_t t, float (&to)[I]) {
        const bool kept = t < end && (!a.keep || a.keep[t] != 0);
        if (kept) row_part<T, I>(logits + t * a.ldl, first, n, words, to);
        else {
#pragma unroll
            for (int i = 0; i < I; ++i) to[i] = -kInfinity;
        }
        return kept;
    };
    float ahead[I];
    bool kept_ahead = fetch(begin + group, ahead);
    for (int64_t t0 = begin; t0 < end; t0 += kGroups) {
        const int64_t t = t0 + group;
        const bool live = kept_ahead;
        float v[I], e[I], top, sum;
#pragma unroll
        for (int i = 0; i < I; ++i) v[i] = ahead[i];
        kept_ahead = fetch(t + kGroups, ahead);
        exponentials<L, I>(v, e, top, sum);
        const unsigned taken = choose<L, I>(v, k);
        // places of the lane's entries among the token's: those of the lanes before it come first
        const int own = __popc(taken);
        const int upto = group_scan<L>(own), before = upto - own;
        const int held = __shfl(upto, L - 1, L);
        float whole = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) whole += taken >> i & 1 ? e[i] : 0.0f;
        whole = group_reduce<L>(whole, SumOf());
        if (a.normalise) whole = sum != sum ? sum : whole;     // (a NaN among the logits)
        const float by = 1.0f / (a.normalise ? whole : sum), part = 1.0f / sum;
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (live && sum != 0.0f) share[i] += e[i] * part;
        // (most lanes have no entry or one: a turn for every entry of the lane that has most)
        int place = before;
        for (unsigned rest = taken; rest != 0; rest &= rest - 1) {
            const int at = __ffs((int)rest) - 1;
            float mine = e[0];
#pragma unroll
            for (int i = 1; i < I; ++i) mine = at == i ? e[i] : mine;
            w.choice[t * k + place] = (uint16_t)(first + at);
            w.gate[t * k + place] = mine * by;
            atomicAdd(&hist[first + at], 1);
            ++place;
        }
        if (t < end && lane == 0) {
            w.held[t] = (uint8_t)held;
            a.out.lse[t] = !live || sum == 0.0f ? 0.0f : top + logf(sum);
            entries += held;
            routed += held > 0;
        }
    }
#pragma unroll
    for (int i = 0; i < I; ++i) shares[group][first + i] = share[i];
    if (lane == 0) {
        atomicAdd(&totals[0], entries);
        atomicAdd(&totals[1], routed);
    }
    __syncthreads();
    for (int e = tid; e < n; e += kThreads) {
        float total = 0.0f;
        for (int g = 0; g < kGroups; ++g) total += shares[g][e];
        w.share[(int64_t)blockIdx.x * n + e] = total;
        w.hist[(int64_t)blockIdx.x * n + e] = hist[e];
    }
    if (tid == 0) {
        w.entries[blockIdx.x] = totals[0];
        w.routed[blockIdx.x] = totals[1];
    }
}

// One wavefront an expert, and one for the tokens: what the workgroups left becomes what lies before each of them; the
// totals go to counts, pos and routed.  A lane has consecutive workgroups, all asked for at once.
constexpr int kMostGroups = 1024;
__global__ void __launch_bounds__(NACHO_WAVE) route_scan_kernel(RouteArgs a, RouteScratch w)
{
    constexpr int kMost = kMostGroups / NACHO_WAVE;
    const int e = (int)blockIdx.x, n = a.experts, lane = lane_id(), groups = (int)w.groups;
    const int each = (groups + NACHO_WAVE - 1) / NACHO_WAVE, first = lane * each;
    int32_t *const from = e < n ? w.hist + e : w.entries;
    const int64_t step = e < n ? n : 1;
    int v[kMost], routed = 0, own = 0;
    float share = 0.0f, s[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int g = first + i;
        v[i] = 0;
        s[i] = 0.0f;
        if (i < each && g < groups) {
            v[i] = from[g * step];
            if (e < n) s[i] = w.share[(int64_t)g * n + e];
            else routed += w.routed[g];
        }
    }
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        own += v[i];
        share += s[i];
    }
    const int upto = wave_inclusive_scan(own);
    int before = upto - own;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int g = first + i;
        if (i < each && g < groups) from[g * step] = before;
        before += v[i];
    }
    share = wave_sum(share);
    routed = wave_sum(routed);
    const int total = __shfl(upto, NACHO_WAVE - 1, NACHO_WAVE);
    if (lane == 0) {
        if (e < n) {
            a.out.counts[e] = total;
            w.share[e] = share;
        } else {
            a.out.pos[a.tokens] = total;
            a.out.routed[0] = routed;
        }
    }
}

// Where the entries of a workgroup's stretch lie, when the counts and what lies before the workgroup are known.
__device__ inline void place_stretch(const RouteArgs &a, const RouteScratch &w)
{
    __shared__ int base[kMostExperts];                 // where the workgroup's next entry of an expert goes
    __shared__ unsigned bits[kMostExperts][kChunk / 32];
    __shared__ int scan[kThreads / NACHO_WAVE];
    __shared__ int before[kChunk + 1];
    __shared__ float sums[kThreads / NACHO_WAVE];
    const int tid = (int)threadIdx.x, n = a.experts, k = a.top_k, lane = lane_id(), wave = tid / NACHO_WAVE;
    const int64_t begin = (int64_t)blockIdx.x * w.per_group;
    const int64_t end = begin + w.per_group < a.tokens ? begin + w.per_group : a.tokens;
    const int entries = a.out.pos[a.tokens];
    // expert_pos: prefix sums of the counts, a thread 4 consecutive experts
    constexpr int kEach = kMostExperts / kThreads;
    int c[kEach], own = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        c[i] = tid * kEach + i < n ? a.out.counts[tid * kEach + i] : 0;
        own += c[i];
    }
    const int upto = wave_inclusive_scan(own);
    if (lane == NACHO_WAVE - 1) scan[wave] = upto;
    __syncthreads();
    int at = upto - own;
    for (int i = 0; i < wave; ++i) at += scan[i];
    float balance = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = tid * kEach + i;
        if (e < n) {
            base[e] = at + w.hist[(int64_t)blockIdx.x * n + e];
            if (blockIdx.x == 0) {
                a.out.expert_pos[e] = at;
                balance += (float)c[i] * w.share[e];
            }
        }
        at += c[i];
    }
    if (blockIdx.x == 0) {
        balance = wave_sum(balance);
        if (lane == 0) sums[wave] = balance;
        __syncthreads();
        if (tid == 0) {
            float total = 0.0f;
            for (int i = 0; i < kThreads / NACHO_WAVE; ++i) total += sums[i];
            const int routed = a.out.routed[0];
            a.out.expert_pos[n] = entries;
            a.out.balance[0] = total * ((float)n / ((float)(entries > 0 ? entries : 1) * (float)(routed > 0 ? routed : 1)));
        }
    }
    int first = w.entries[blockIdx.x];                 // the workgroup's next entry
    for (int64_t t0 = begin; t0 < end; t0 += kChunk) {
        const int many = (int)(end - t0 < kChunk ? end - t0 : kChunk);
        for (int i = tid; i < n * (kChunk / 32); i += kThreads) (&bits[0][0])[i] = 0;
        if (wave == 0) {
            const int held = lane < many ? w.held[t0 + lane] : 0;
            const int sum = wave_inclusive_scan(held);
            before[lane + 1] = sum;
            if (lane == 0) before[0] = 0;
            if (lane < many) a.out.pos[t0 + lane] = first + sum - held;
        }
        __syncthreads();
        for (int i = tid; i < many * k; i += kThreads) {
            const int t = i / k, r = i - t * k;
            if (r < before[t + 1] - before[t]) atomicOr(&bits[w.choice[t0 * k + i]][t / 32], 1u << (t % 32));
        }
        __syncthreads();
        for (int i = tid; i < many * k; i += kThreads) {
            const int t = i / k, r = i - t * k;
            if (r < before[t + 1] - before[t]) {
                const int e = w.choice[t0 * k + i], entry = first + before[t] + r;
                int place = base[e];
                if (t >= 32) place += __popc(bits[e][0]);
                place += __popc(bits[e][t / 32] & ((1u << (t % 32)) - 1u));
                a.out.expert[entry] = e;
                a.out.gate[entry] = w.gate[t0 * k + i];
                a.out.slot[entry] = place;
                a.out.token[place] = (int32_t)(t0 + t);
            }
        }
        first += before[many];
        __syncthreads();
        for (int e = tid; e < n; e += kThreads) base[e] += __popc(bits[e][0]) + __popc(bits[e][1]);
        __syncthreads();
    }
    // the places behind the last entry, shared out
    const int64_t room = a.tokens * k;
    for (int64_t i = entries + (int64_t)blockIdx.x * kThreads + tid; i < room; i += (int64_t)gridDim.x * kThreads) {
        a.out.expert[i] = -1;
        a.out.gate[i] = 0.0f;
        a.out.slot[i] = -1;
        a.out.token[i] = -1;
    }
}

template <typename T, int L, int I>
__global__ void __launch_bounds__(kThreads) route_choose_kernel(RouteArgs a, RouteScratch w) { choose_stretch<T, L, I>(a, w); }
__global__ void __launch_bounds__(kThreads) route_place_kernel(RouteArgs a, RouteScratch w) { place_stretch(a, w); }

// Tokens of one workgroup: nothing lies before it, and one launch does (16 tokens of 64 experts: 22 us a call with three).
template <typename T, int L, int I>
__global__ void __launch_bounds__(kThreads) route_few_kernel(RouteArgs a, RouteScratch w)
{
    choose_stretch<T, L, I>(a, w);
    __syncthreads();
    for (int e = (int)threadIdx.x; e < a.experts; e += kThreads) {
        a.out.counts[e] = w.hist[e];
        w.hist[e] = 0;
    }
    if (threadIdx.x == 0) {
        a.out.pos[a.tokens] = w.entries[0];
        a.out.routed[0] = w.routed[0];
        w.entries[0] = 0;
    }
    __syncthreads();
    place_stretch(a, w);
}

template <typename T, int L, int I>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(RouteGradArgs a)
{
    constexpr int kGroups = kThreads / L;
    __shared__ float added[kGroups][L * I];                    // what the gates add to every expert of a group's token
    const int tid = (int)threadIdx.x, group = tid / L, lane = tid % L, first = lane * I, n = a.experts;
    const T *logits = static_cast<const T *>(a.logits);
    T *grad = static_cast<T *>(a.grad);
    const bool words = in_words<T, I>(logits, a.ldl), words_out = in_words<T, I>(grad, a.ldg);
    // the balance loss by an expert's probability
    const int entries = a.routing.pos[a.tokens], routed = a.routing.routed[0];
    const float unit = a.balance * ((float)n / ((float)(entries > 0 ? entries : 1) * (float)(routed > 0 ? routed : 1)));
    float c[I];
#pragma unroll
    for (int i = 0; i < I; ++i) c[i] = first + i < n ? unit * (float)a.routing.counts[first + i] : 0.0f;
    // a token's logits and the place of its entries are on their way while the one before it is worked on (also of tokens
    // that store nothing, whose result does not take them)
    auto fetch = [&](int64_t t, float (&to)[I], int &at, int &held) {
        at = held = 0;
        if (t < a.tokens) {
            row_part<T, I>(logits + t * a.ldl, first, n, words, to);
            at = a.routing.pos[t];
            held = a.routing.pos[t + 1] - at;
        } else {
#pragma unroll
            for (int i = 0; i < I; ++i) to[i] = -kInfinity;
        }
    };
    const int64_t step = (int64_t)gridDim.x * kGroups;
    float ahead[I];
    int at_ahead, held_ahead;
    fetch((int64_t)blockIdx.x * kGroups + group, ahead, at_ahead, held_ahead);
    for (int64_t t0 = (int64_t)blockIdx.x * kGroups; t0 < a.tokens; t0 += step) {
        const int64_t t = t0 + group;
        const int at = at_ahead, held = held_ahead;
        float v[I], p[I], top, sum, mean = 0.0f, inner = 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) v[i] = ahead[i];
        // a lane has every L-th entry of the token, the first of them in registers
        float g = 0.0f, dg = 0.0f;
        int to = -1;
        if (a.grad_gate && lane < held) {
            g = a.routing.gate[at + lane];
            dg = a.grad_gate[at + lane];
            to = a.routing.expert[at + lane];
        }
        fetch(t + step, ahead, at_ahead, held_ahead);
#pragma unroll
        for (int i = 0; i < I; ++i) added[group][first + i] = 0.0f;
        // (not by the lse of the forward call: next to large logits it has no room for the sum)
        exponentials<L, I>(v, p, top, sum);
        const float part = sum != 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            p[i] *= part;
            mean += p[i] * c[i];
        }
        mean = group_reduce<L>(mean, SumOf());
        inner = g * dg;
        if (a.grad_gate)
            for (int j = lane + L; j < held; j += L) inner += a.routing.gate[at + j] * a.grad_gate[at + j];
        inner = group_reduce<L>(inner, SumOf());
        wave_sync();
        if (to >= 0) added[group][to] = g * (a.normalise ? dg - inner : dg);
        if (a.grad_gate)
            for (int j = lane + L; j < held; j += L) {
                const float more = a.routing.gate[at + j], by = a.grad_gate[at + j];
                added[group][a.routing.expert[at + j]] = more * (a.normalise ? by - inner : by);
            }
        wave_sync();
        const float less = mean + (a.normalise ? 0.0f : inner);
        float d[I];
#pragma unroll
        for (int i = 0; i < I; ++i) d[i] = held > 0 ? added[group][first + i] + p[i] * (c[i] - less) : 0.0f;
        if (t < a.tokens) put_row_part<T, I>(grad + t * a.ldg, first, n, words_out, d);
        wave_sync();
    }
}

// Lanes and experts a lane for n experts, as a call of f(L, I).
template <typename F> void by_experts(int n, F f)
{
    using std::integral_constant;
    if (n <= 16) f(integral_constant<int, 4>(), integral_constant<int, 4>());
    else if (n <= 32) f(integral_constant<int, 4>(), integral_constant<int, 8>());
    else if (n <= 64) f(integral_constant<int, 8>(), integral_constant<int, 8>());
    else if (n <= 128) f(integral_constant<int, 16>(), integral_constant<int, 8>());
    else if (n <= 256) f(integral_constant<int, 32>(), integral_constant<int, 8>());
    else if (n <= 512) f(integral_constant<int, 64>(), integral_constant<int, 8>());
    else f(integral_constant<int, 64>(), integral_constant<int, 16>());
}
template <typename F> void by_type(int dtype, F f)
{
    if (dtype == NACHO_F32) f((float)0);
    else if (dtype == NACHO_BF16) f((bf16_t)0.0f);
    else f((f16_t)0.0f);
}

}  // namespace

void route_plan(int64_t tokens, int32_t, int64_t *groups, int64_t *per_group)
{
    // up to 1024 workgroups (four a compute unit), whole chunks of tokens each
    const int64_t chunks = (tokens + kChunk - 1) / kChunk, each = (chunks + kMostGroups - 1) / kMostGroups;
    *per_group = (each > 0 ? each : 1) * kChunk;
    *groups = (tokens + *per_group - 1) / *per_group;
    if (*groups < 1) *groups = 1;
}

hipError_t launch_route(int dtype, const RouteArgs &a, const RouteScratch &w, hipStream_t s)
{
    if (w.groups == 1) {
        by_type(dtype, [&](auto zero) {
            by_experts(a.experts, [&](auto lanes, auto items) {
                route_few_kernel<decltype(zero), decltype(lanes)::value, decltype(items)::value><<<dim3(1), kThreads, 0, s>>>(a, w);
            });
        });
        const hipError_t rc = hipGetLastError();
        if (rc == hipSuccess) nacho_host::profile_mark("route");
        return rc;
    }
    by_type(dtype, [&](auto zero) {
        by_experts(a.experts, [&](auto lanes, auto items) {
            route_choose_kernel<decltype(zero), decltype(lanes)::value, decltype(items)::value>
                <<<dim3((unsigned)w.groups), kThreads, 0, s>>>(a, w);
        });
    });
    hipError_t rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    nacho_host::profile_mark("route_choose");
    route_scan_kernel<<<dim3((unsigned)a.experts + 1), NACHO_WAVE, 0, s>>>(a, w);
    rc = hipGetLastError();
    if (rc != hipSuccess) return rc;
    nacho_host::profile_mark("route_scan");
    route_place_kernel<<<dim3((unsigned)w.groups), kThreads, 0, s>>>(a, w);
    rc = hipGetLastError();
    if (rc == hipSuccess) nacho_host::profile_mark("route_place");
    return rc;
}

hipError_t launch_route_grad(int dtype, const RouteGradArgs &a, hipStream_t s)
{
    if (a.tokens == 0) return hipSuccess;
    by_type(dtype, [&](auto zero) {
        by_experts(a.experts, [&](auto lanes, auto items) {
            constexpr int L = decltype(lanes)::value;
            const int64_t tiles = (a.tokens + kThreads / L - 1) / (kThreads / L);
            route_grad_kernel<decltype(zero), L, decltype(items)::value>
                <<<dim3((unsigned)(tiles < 2048 ? tiles : 2048)), kThreads, 0, s>>>(a);
        });
    });
    return hipGetLastError();
}

}  // namespace nacho
