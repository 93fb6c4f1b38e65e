// The logits of a few rows against a large vocabulary (see xent.hip): the vocabulary's weights are what is read, once, and the time is
// that of reading them.  A wavefront takes 16 or 64 words of the vocabulary at a time from memory right into the registers that the
// matrix units read, and the rows of x the same way from the caches; for the loss it keeps the largest logit of each row and the sum of
// exponentials under it over all words that it has.
#include "xent.hpp"

namespace nacho {

namespace {

constexpr int kWaves = 4, kThreads = kWaves * NACHO_WAVE;

// The rows that count, which are so few that every workgroup lists them for itself: what xent_rows_kernel does for many.  One workgroup
// leaves what the kernels behind need.  Returns how many there are.
struct RowList {
    int row[kFewRows], label[kFewRows];
};
template <typename Label> __device__ inline int list_rows(const XentArgs &a, RowList &list, float &scale)
{
    const int lane = lane_id();
    int64_t label = -1;
    float weight = 0.0f;
    if (lane < a.rows) {
        label = (int64_t)static_cast<const Label *>(a.label)[lane];
        weight = a.weight ? a.weight[lane] : 1.0f;
    }
    const bool held = lane < a.rows && label >= 0 && label < a.vocabulary && weight != 0.0f;
    const unsigned long long who = __ballot(held);
    const int slot = __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0)), count = __popcll((long long)who);
    if (held) {
        list.row[slot] = lane;
        list.label[slot] = (int)label;
    }
    wave_sync();
    int by = 0;
    if (a.scale) by = a.half ? scale_exponent(wave_all(held ? fabsf(weight) : 0.0f, MaxOf())) : 0;
    scale = ldexpf(1.0f, by);
    if (blockIdx.x == 0 && threadIdx.x < NACHO_WAVE) {
        if (lane == 0) {
            a.bounds[0] = 0;
            a.bounds[1] = count;
            if (a.scale) {
                a.scale[0] = scale;
                a.scale[1] = ldexpf(1.0f, -by);
            }
        }
        if (held) {
            a.token[slot] = lane;
            a.slot_label[slot] = (int)label;
        } else if (lane < a.rows && a.loss) a.loss[lane] = a.lse[lane] = 0.0f;
        if (a.slot_of && lane < a.rows) a.slot_of[lane] = held ? slot : -1;
    }
    return count;
}

template <typename T, int kGroups, int kTiles, int kSteps, bool kGradient>
__global__ void __launch_bounds__(kThreads) xent_few_kernel(XentArgs a, int first, int words, int64_t ldg)
{
    typedef Stretch<T, WORDS, kSteps> Part;
    constexpr int kBatch = Part::kBatch, kWords = 16 * kTiles;
    const int lane = lane_id(), lane_row = lane % 16, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / NACHO_WAVE);
    __shared__ RowList lists[kWaves];
    RowList &list = lists[wave];
    float scale;
    const int held = __builtin_amdgcn_readfirstlane(a.label_bytes == 8 ? list_rows<int64_t>(a, list, scale) : list_rows<int32_t>(a, list, scale));
    if (held == 0) return;
    int slot[kGroups], label[kGroups];
    const T *x[kGroups];
    float lse[kGroups], factor[kGroups], top[kGroups], sum[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        slot[g] = g * 16 + lane_row;
        const int there = slot[g] < held ? slot[g] : held - 1;
        const int row = list.row[there];
        x[g] = static_cast<const T *>(a.x) + row * a.ldx;
        label[g] = list.label[there] - first;
        if constexpr (kGradient) {
            lse[g] = a.lse[row];
            factor[g] = (a.weight ? a.weight[row] : 1.0f) * scale;
        }
        top[g] = -kInfinity;
        sum[g] = 0.0f;
    }
    const int tiles = (words + kWords - 1) / kWords, stretches = (a.inner + Part::kLong - 1) / Part::kLong, k = a.inner;
    const T *const head = static_cast<const T *>(a.head) + (int64_t)first * a.ldh;
    struct Loaded {
        typename Part::Loaded p[kTiles][kBatch], q[kBatch];
    } one, two;
    for (int tile = (int)blockIdx.x * kWaves + wave; tile < tiles; tile += (int)gridDim.x * kWaves) {
        const T *rows[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            const int row = tile * kWords + i * 16 + lane % 16;
            rows[i] = head + (row < words ? row : words - 1) * a.ldh;
        }
        v4f acc[kGroups][kTiles];
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
            for (int i = 0; i < kTiles; ++i) acc[g][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        auto fetch_x = [&](Loaded &to, int s, int g) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) to.q[b] = Part::load(x[g], Part::from(s, b), k);
        };
        auto fetch = [&](Loaded &to, int s) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int b = 0; b < kBatch; ++b) to.p[i][b] = Part::load(rows[i], Part::from(s, b), k);
            fetch_x(to, s, 0);
        };
        auto multiply = [&](Loaded &of, int s) {
            Part::by_end(s, k, [&](auto whole) {
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) of.p[i][b] = Part::value(of.p[i][b], rows[i], Part::from(s, b), k, whole);
            });
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                if (g > 0) {
                    if (g * 16 >= held) break;
                    fetch_x(of, s, g);
                }
                Part::by_end(s, k, [&](auto whole) {
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) of.q[b] = Part::value(of.q[b], x[g], Part::from(s, b), k, whole);
                });
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
#pragma unroll
                    for (int i = 0; i < kTiles; ++i) acc[g][i] = matrix_step<T>(of.p[i][b], of.q[b], acc[g][i]);
            }
        };
        // every wavefront starts somewhere else along k
        const int turn = tile % stretches;
        auto at = [&](int s) {
            const int t = (s < stretches ? s : stretches - 1) + turn;      // (behind the last stretch it is loaded again: no branch around a load)
            return t < stretches ? t : t - stretches;
        };
        fetch(one, at(0));
        for (int s = 0; s < stretches; s += 2) {
            fetch(two, at(s + 1));
            multiply(one, at(s));
            fetch(one, at(s + 2));
            if (s + 1 < stretches) multiply(two, at(s + 1));
        }
        // a lane has four words of every 16 for one row
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g * 16 >= held) break;
            const int word0 = tile * kWords + lane / 16 * 4;
            if constexpr (kGradient) {
                typedef T four __attribute__((ext_vector_type(4)));
                T *const out = static_cast<T *>(a.g) + slot[g] * ldg;
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    const int word = word0 + i * 16;
                    four v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float q = exp2_of((acc[g][i][e] - lse[g]) * kLog2e) - (label[g] == word + e ? 1.0f : 0.0f);
                        v[e] = (T)(word + e < words ? q * factor[g] : 0.0f);
                    }
                    // (rows of g are whole words of 8 elements)
                    if (slot[g] < held && word < (words + 7) / 8 * 8) *reinterpret_cast<four *>(out + word) = v;
                }
            } else {
                float most = top[g];
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int word = word0 + i * 16 + e;
                        if (word >= words) acc[g][i][e] = -kInfinity;
                        most = fmaxf(most, acc[g][i][e]);
                        if (label[g] == word && slot[g] < held) a.at_label[slot[g]] = acc[g][i][e];
                    }
                const float base = most == -kInfinity ? 0.0f : most;
                float all = top[g] == most ? sum[g] : sum[g] * exp2_of((top[g] - base) * kLog2e);
#pragma unroll
                for (int i = 0; i < kTiles; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) all += exp2_of((acc[g][i][e] - base) * kLog2e);
                top[g] = most;
                sum[g] = all;
            }
        }
    }
    if constexpr (!kGradient) {
        __shared__ float2 share[kWaves][kGroups * 16];
        auto join = [](float &t, float &s, float t2, float s2) {
            const float most = fmaxf(t, t2);
            s = (t == most ? s : s * exp2_of((t - most) * kLog2e)) + (t2 == most ? s2 : s2 * exp2_of((t2 - most) * kLog2e));
            t = most;
        };
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            join(top[g], sum[g], __shfl_xor(top[g], 16, NACHO_WAVE), __shfl_xor(sum[g], 16, NACHO_WAVE));
            join(top[g], sum[g], __shfl_xor(top[g], 32, NACHO_WAVE), __shfl_xor(sum[g], 32, NACHO_WAVE));
            if (lane < 16) share[wave][g * 16 + lane] = make_float2(top[g], sum[g]);
        }
        __syncthreads();
        for (int i = (int)threadIdx.x; i < kGroups * 16 && i < held; i += kThreads) {
            float t = share[0][i].x, s = share[0][i].y;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) join(t, s, share[w][i].x, share[w][i].y);
            a.partial[(int64_t)blockIdx.x * a.rows + i] = make_float2(t, s);
        }
    }
}

// Groups of 16 rows, and words that a wavefront has at a time: 16 as long as more would leave compute units without any.
int groups_of(int64_t rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }
int words_at_a_time(int64_t rows, int64_t vocabulary)
{
    const int most = groups_of(rows) == 1 ? 32 : 64;
    return vocabulary < most * kWaves * kUnits ? 16 : most;
}

}  // namespace

int64_t xent_few_groups(int64_t rows, int64_t vocabulary)
{
    const int64_t each = words_at_a_time(rows, vocabulary) * kWaves, groups = (vocabulary + each - 1) / each;
    return groups < 4 * kUnits ? groups : 4 * kUnits;
}

hipError_t launch_xent_few(int dtype, const XentArgs &a, int64_t first, int64_t words, int64_t ldg, hipStream_t s)
{
    const unsigned grid = (unsigned)xent_few_groups(a.rows, words);
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        auto run = [&](auto groups, auto tiles, auto steps) {
            constexpr int kGroups = decltype(groups)::value, kTiles = decltype(tiles)::value, kSteps = decltype(steps)::value;
            if (a.g) xent_few_kernel<T, kGroups, kTiles, kSteps, true><<<grid, kThreads, 0, s>>>(a, (int)first, (int)words, ldg);
            else xent_few_kernel<T, kGroups, kTiles, kSteps, false><<<grid, kThreads, 0, s>>>(a, (int)first, (int)words, ldg);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        const bool single = words_at_a_time(a.rows, words) == 16;
        switch (groups_of(a.rows)) {
        case 1: single ? run(one, one, two) : run(one, two, four); break;
        case 2: single ? run(two, one, two) : run(two, four, two); break;
        default: single ? run(four, one, two) : run(four, four, two);
        }
    });
    return hipGetLastError();
}

}  // namespace nacho
