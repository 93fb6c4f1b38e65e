// The choice of a token's experts: L lanes of a wavefront hold its logits, I consecutive experts a lane.
#pragma once
#include "dense.hpp"

namespace nacho {

// I consecutive elements of a row from element `at`, those behind `n` are -inf.
template <typename T, int I> __device__ inline void row_part(const T *row, int at, int n, bool words, float (&v)[I])
{
    constexpr int kBytes = I * (int)sizeof(T) < 16 ? I * (int)sizeof(T) : 16, kEach = kBytes / (int)sizeof(T);
    typedef T part __attribute__((ext_vector_type(kEach)));
    if (words && at + I <= n) {
#pragma unroll
        for (int i = 0; i < I; i += kEach) {
            const part p = *reinterpret_cast<const part *>(row + at + i);
#pragma unroll
            for (int e = 0; e < kEach; ++e) v[i + e] = wide((T)p[e]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < I; ++i) v[i] = at + i < n ? wide(row[at + i]) : -kInfinity;
    }
}
// Whether rows `ld` apart can be read in words of 16 bytes (or of a lane's I elements, if these are fewer).
template <typename T, int I> __host__ __device__ inline bool in_words(const void *base, int64_t ld)
{
    constexpr int kBytes = I * (int)sizeof(T) < 16 ? I * (int)sizeof(T) : 16;
    return ((uintptr_t)base & (kBytes - 1)) == 0 && (ld * (int64_t)sizeof(T)) % kBytes == 0;
}

// The softmax of a token's logits: exp(v - top) of a lane's experts, and their sum over the group.
template <int L, int I> __device__ inline void exponentials(const float (&v)[I], float (&e)[I], float &top, float &sum)
{
    top = v[0];
#pragma unroll
    for (int i = 1; i < I; ++i) top = fmaxf(top, v[i]);
    top = group_reduce<L>(top, MaxOf());
    sum = 0.0f;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        e[i] = v[i] == -kInfinity ? 0.0f : exp2_of((v[i] - top) * kLog2e);
        sum += e[i];
    }
    sum = group_reduce<L>(sum, SumOf());
}

// Prefix sum over the lanes of a group, the lane's own included: inside 16 lanes, then with what the sixteens before hold.
template <int L> __device__ inline int group_scan(int v)
{
    const int lane = lane_id(), own = lane % (L < 16 ? L : 16);
    auto add = [&](unsigned from, int off) { v += own >= off ? (int)from : 0; };
    if constexpr (L > 1) add(moved<0x111>((unsigned)v), 1);              // from the lane 1, 2, 4, 8 before in 16 lanes
    if constexpr (L > 2) add(moved<0x112>((unsigned)v), 2);
    if constexpr (L > 4) add(moved<0x114>((unsigned)v), 4);
    if constexpr (L > 8) add(moved<0x118>((unsigned)v), 8);
    if constexpr (L > 16) {
        const int before = __shfl(v, (lane & ~31) + 15, NACHO_WAVE);
        v += lane & 16 ? before : 0;
    }
    if constexpr (L > 32) {
        const int before = __shfl(v, 31, NACHO_WAVE);
        v += lane & 32 ? before : 0;
    }
    return v;
}
// How many lanes of the group say yes.
template <int L> __device__ inline int group_count(bool yes)
{
    const unsigned long long all = __ballot(yes);
    if constexpr (L == NACHO_WAVE) return __popcll((long long)all);
    else {
        const int lane = lane_id();
        unsigned low = (unsigned)all, high = (unsigned)(all >> 32);
        asm volatile("" : "+s"(low), "+s"(high));      // (or the compiler makes one shift of 64 bits by a lane's own amount of it)
        const unsigned half = (lane < 32 ? low : high) >> ((unsigned)(lane / L * L) & 31u);
        return __popc(L == 32 ? half : half & ((1u << (L % 32)) - 1u));
    }
}

// The k largest of a group's experts, as bits of the lanes' own.  Every lane sorts its keys (a network, two instructions a
// pair); in a round the lanes whose first one is the group's largest drop it, until k are dropped: the last of them is the
// threshold.  What lies above it is chosen, and of what equals it as many as are left, the lowest indices first.
template <int L, int I> __device__ inline unsigned choose(const float (&v)[I], int k)
{
    unsigned key[I], sorted[I];
#pragma unroll
    for (int i = 0; i < I; ++i) sorted[i] = key[i] = order_of(v[i]);
    // (Batcher's merges of odd and even places)
#pragma unroll
    for (int p = 1; p < I; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < I; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < I && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                        const unsigned x = sorted[i + j], y = sorted[i + j + q];
                        sorted[i + j] = x > y ? x : y;
                        sorted[i + j + q] = x > y ? y : x;
                    }
    unsigned threshold = 0;
    int dropped = 0, left = 0;                 // left: of those at the threshold
    for (int r = 0; r < k; ++r) {
        const unsigned best = group_max<L>(sorted[0]);
        const bool mine = sorted[0] == best;
        if (dropped < k) {
            if (best != threshold) left = k - dropped;
            threshold = best;
        }
        dropped += group_count<L>(mine);
#pragma unroll
        for (int i = 0; i + 1 < I; ++i) {
            unsigned next = sorted[i + 1];
            asm volatile("" : "+v"(next));     // (or it becomes a choice of the place, and that a chain of choices)
            sorted[i] = mine ? next : sorted[i];
        }
        sorted[I - 1] = mine ? 0u : sorted[I - 1];
    }
    unsigned above = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        above |= key[i] > threshold ? 1u << i : 0u;
        equal |= key[i] == threshold ? 1u << i : 0u;
    }
    if (threshold == 0) return above;          // (fewer than k may be chosen)
    const int own = __popc(equal);
    int room = left - (group_scan<L>(own) - own);
    for (unsigned rest = equal; rest != 0 && room > 0; rest &= rest - 1, --room) above |= rest & (0u - rest);
    return above;
}

}  // namespace nacho
