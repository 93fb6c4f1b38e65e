// The logits of a few rows against a large vocabulary (see xent.hip): the vocabulary's weights are what is read, once, and the time is
// that of reading them.  A wavefront takes 16 or 32 words of the vocabulary at a time from memory right into the registers that the
// matrix units read, and the rows of x the same way from the caches; for the loss it keeps the largest logit of each row and the sum of
// exponentials under it over all words that it has.  3 rows against 131072 x 2048 bf16: 88 us a kernel, 6.1 TB/s (by tiles 119 us).
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

template <typename T, Access kAccess, int kTiles, int kSteps, bool kGradient>
__global__ void __launch_bounds__(kThreads) xent_few_kernel(XentArgs a, int first, int words, int64_t ldg)
{
    typedef Stretch<T, kAccess, kSteps> Part;
    constexpr int kBatch = Part::kBatch, kWords = 16 * kTiles;
    const int lane = lane_id(), slot = lane % 16, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / NACHO_WAVE);
    __shared__ RowList lists[kWaves];
    RowList &list = lists[wave];
    float scale;
    const int held = __builtin_amdgcn_readfirstlane(a.label_bytes == 8 ? list_rows<int64_t>(a, list, scale) : list_rows<int32_t>(a, list, scale));
    if (held == 0) return;
    // (lanes without a row have the last one, whose results are not stored)
    const int there = slot < held ? slot : held - 1, own = list.row[there], label = list.label[there] - first;
    const T *const x = static_cast<const T *>(a.x) + own * a.ldx;
    float lse = 0.0f, factor = 0.0f, top = -kInfinity, sum = 0.0f;
    if constexpr (kGradient) {
        lse = a.lse[own];
        factor = (a.weight ? a.weight[own] : 1.0f) * scale;
    }
    const int tiles = (words + kWords - 1) / kWords, stretches = (a.inner + Part::kLong - 1) / Part::kLong, k = a.inner;
    const T *const head = static_cast<const T *>(a.head) + (int64_t)first * a.ldh;
    struct Loaded {
        typename Part::Loaded p[kTiles][kBatch], q[kBatch];
    } one, two;
    for (int tile = (int)blockIdx.x * kWaves + wave; tile < tiles; tile += (int)gridDim.x * kWaves) {
        const T *rows[kTiles];
        v4f acc[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            const int row = tile * kWords + i * 16 + lane % 16;
            rows[i] = head + (row < words ? row : words - 1) * a.ldh;
            acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        auto fetch = [&](Loaded &to, int s) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int b = 0; b < kBatch; ++b) to.p[i][b] = Part::load(rows[i], Part::from(s, b), k);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) to.q[b] = Part::load(x, Part::from(s, b), k);
        };
        auto multiply = [&](Loaded &of, int s) {
            Part::by_end(s, k, [&](auto whole) {
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    of.q[b] = Part::value(of.q[b], x, Part::from(s, b), k, whole);
#pragma unroll
                    for (int i = 0; i < kTiles; ++i) of.p[i][b] = Part::value(of.p[i][b], rows[i], Part::from(s, b), k, whole);
                }
            });
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
#pragma unroll
                for (int i = 0; i < kTiles; ++i) acc[i] = matrix_step<T>(of.p[i][b], of.q[b], acc[i]);
        };
        // every wavefront starts somewhere else along k: rows are often a power of two apart, and so would be what is read at a time
        // (3 rows against 131072 x 2048 bf16: 120 us a call without, 95 with; against 131072 x 2000 103 and 103)
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
        const int word0 = tile * kWords + lane / 16 * 4;
        if constexpr (kGradient) {
            typedef T four __attribute__((ext_vector_type(4)));
            T *const out = static_cast<T *>(a.g) + slot * ldg;
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const int word = word0 + i * 16;
                four v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float q = exp2_of((acc[i][e] - lse) * kLog2e) - (label == word + e ? 1.0f : 0.0f);
                    v[e] = (T)(word + e < words ? q * factor : 0.0f);
                }
                // (rows of g are whole words of 8 elements)
                if (slot < held && word < (words + 7) / 8 * 8) *reinterpret_cast<four *>(out + word) = v;
            }
        } else {
            float most = top;
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int word = word0 + i * 16 + e;
                    if (word >= words) acc[i][e] = -kInfinity;
                    most = fmaxf(most, acc[i][e]);
                    if (label == word && slot < held) a.at_label[slot] = acc[i][e];
                }
            const float base = most == -kInfinity ? 0.0f : most;
            float all = top == most ? sum : sum * exp2_of((top - base) * kLog2e);
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) all += exp2_of((acc[i][e] - base) * kLog2e);
            top = most;
            sum = all;
        }
    }
    if constexpr (!kGradient) {
        __shared__ float2 share[kWaves][16];
        auto join = [](float &t, float &s, float t2, float s2) {
            const float most = fmaxf(t, t2);
            s = (t == most ? s : s * exp2_of((t - most) * kLog2e)) + (t2 == most ? s2 : s2 * exp2_of((t2 - most) * kLog2e));
            t = most;
        };
        join(top, sum, __shfl_xor(top, 16, NACHO_WAVE), __shfl_xor(sum, 16, NACHO_WAVE));
        join(top, sum, __shfl_xor(top, 32, NACHO_WAVE), __shfl_xor(sum, 32, NACHO_WAVE));
        if (lane < 16) share[wave][lane] = make_float2(top, sum);
        __syncthreads();
        if ((int)threadIdx.x < held) {
            float t = share[0][threadIdx.x].x, s = share[0][threadIdx.x].y;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) join(t, s, share[w][threadIdx.x].x, share[w][threadIdx.x].y);
            a.partial[(int64_t)blockIdx.x * a.rows + threadIdx.x] = make_float2(t, s);
        }
    }
}

// Gradients of the vocabulary's weights: 16 words are one product of g^T with the rows of x, which a wavefront keeps (kAcross columns of them,
// zeros behind the last) and takes through the words.  Bound by writing: a lane ends with a word of 16 bytes of a row, so results need no LDS.
// (The tiles of columns that make up such a word take every other four columns.)  Rows that start at multiples of 64 bytes leave by stores that
// no cache keeps, the 64 bytes that an instruction has of a row at once; other rows' lines would be written in parts.  (Loss and gradients, us a
// pass so, otherwise, and with the tiles of many rows: 1 row, 65536 x 2048 bf16 220, 231 and 246, 16 rows 238, 253 and 258; 2 rows, 50622 x 3867
// f32 1255, 782 and 824.  65536 x 2048 bf16 is 268 MB in about 45 us.)
// (2 rows, 50622 x 3867 f32: 128 columns 811 us, 256 776; 16 rows, 65536 x 2048 bf16 258 and 261)
template <typename T> constexpr int kAcross = sizeof(T) == 4 ? 256 : 128;
template <typename T, bool kWhole>
__global__ void __launch_bounds__(kThreads) xent_few_head_kernel(XentArgs a, int first, int words, int64_t ldg, int chunks, int each)
{
    typedef typename Word<T>::type word;
    constexpr int n = Word<T>::n, kGroup = n / 4, kTiles = kAcross<T> / 16;
    const int lane = lane_id(), number = (int)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x / NACHO_WAVE);
    const int c0 = number % chunks * kAcross<T>, tiles = (words + 15) / 16, row0 = lane / 16 * n;
    const int held = a.rows > 0 ? a.bounds[1] : 0;
    if (number / chunks >= each) return;
    const float by = a.scale[1];
    v4u p[kTiles];
    word q[2];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) p[i] = v4u{0, 0, 0, 0};
    auto fetch = [&](word &to, int tile) {
        const int at = tile * 16 + lane % 16, there = at < words ? at : words - 1;
#pragma unroll
        for (int e = 0; e < n; ++e) to[e] = row0 + e < held ? static_cast<const T *>(a.g)[(row0 + e) * ldg + there] : (T)0.0f;
    };
    q[0] = q[1] = __builtin_bit_cast(word, p[0]);
    if (row0 < held) {
#pragma unroll
        for (int e = 0; e < n; ++e) {
            if (row0 + e >= held) break;
            const T *const x = static_cast<const T *>(a.x) + a.token[row0 + e] * a.ldx;
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const int m = lane % 16, c = c0 + i / kGroup * 16 * kGroup + m / 4 * n + i % kGroup * 4 + m % 4;
                word v = __builtin_bit_cast(word, p[i]);
                v[e] = c < a.inner ? x[c] : (T)0.0f;
                p[i] = __builtin_bit_cast(v4u, v);
            }
        }
        fetch(q[0], number / chunks);
    }
    for (int tile = number / chunks; tile < tiles; tile += each) {
        if (row0 < held && tile + each < tiles) fetch(q[1], tile + each);
        v4f acc[kTiles];
#pragma unroll
        for (int i = 0; i < kTiles; ++i) acc[i] = matrix_step<T>(p[i], __builtin_bit_cast(v4u, q[0]), v4f{0.0f, 0.0f, 0.0f, 0.0f});
        const int at = tile * 16 + lane % 16;
        T *const out = static_cast<T *>(a.grad_head) + (int64_t)(first + at) * a.ldgh;
        if (at < words) {
#pragma unroll
            for (int j = 0; j < kTiles / kGroup; ++j) {
                const int c = c0 + j * 16 * kGroup + lane / 16 * n;
                word v;
#pragma unroll
                for (int e = 0; e < n; ++e) v[e] = (T)(acc[j * kGroup + e / 4][e % 4] * by);
                if (kWhole && c + n <= a.inner) __builtin_nontemporal_store(v, reinterpret_cast<word *>(out + c));
                else if (c + n <= a.inner) __builtin_memcpy(out + c, &v, 16);
                else {
#pragma unroll
                    for (int e = 0; e < n; ++e)
                        if (c + e < a.inner) out[c + e] = v[e];
                }
            }
        }
        q[0] = q[1];
    }
}

// Words that a wavefront has at a time: 16 as long as 32 would leave a quarter of the compute units without any.  (16 rows bf16, us a call
// with 16 and with 32: 8000 x 1024 21 and 25, 16000 x 1024 21 and 25, 32000 x 1024 29 and 26, 65536 x 1024 47 and 41, 65536 x 2048 74 and
// 62, a graph's start included.)
int words_at_a_time(int64_t vocabulary) { return vocabulary < 24 * kWaves * kUnits ? 16 : 32; }

}  // namespace

int64_t xent_few_groups(int64_t vocabulary)
{
    const int64_t each = words_at_a_time(vocabulary) * kWaves, groups = (vocabulary + each - 1) / each;
    return groups < 4 * kUnits ? groups : 4 * kUnits;
}

hipError_t launch_xent_few(int dtype, const XentArgs &a, int64_t first, int64_t words, int64_t ldg, bool in_words, hipStream_t s)
{
    const unsigned grid = (unsigned)xent_few_groups(words);
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        auto run = [&](auto access, auto tiles, auto steps) {
            constexpr Access kAccess = decltype(access)::value;
            constexpr int kTiles = decltype(tiles)::value, kSteps = decltype(steps)::value;
            if (a.g) xent_few_kernel<T, kAccess, kTiles, kSteps, true><<<grid, kThreads, 0, s>>>(a, (int)first, (int)words, ldg);
            else xent_few_kernel<T, kAccess, kTiles, kSteps, false><<<grid, kThreads, 0, s>>>(a, (int)first, (int)words, ldg);
        };
        auto of = [&](auto access) {
            if (words_at_a_time(words) == 16) run(access, std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
            else run(access, std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
        };
        typedef std::integral_constant<Access, WORDS> Words;
        typedef std::integral_constant<Access, sizeof(T) == 4 ? ANYWHERE : WORDS> Anywhere;
        in_words ? of(Words()) : of(Anywhere());
    });
    return hipGetLastError();
}

hipError_t launch_xent_few_head(int dtype, const XentArgs &a, int64_t first, int64_t words, int64_t ldg, hipStream_t s)
{
    const bool whole = ((uintptr_t)a.grad_head | (uintptr_t)(a.ldgh * a.elem)) % 64 == 0;
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        // (8 wavefronts a compute unit write as fast as 16 and fetch the rows of x half as often: 1 row, 65536 x 2048 bf16, 220 and 223 us)
        const int64_t chunks = (a.inner + kAcross<T> - 1) / kAcross<T>, tiles = (words + 15) / 16, most = 8 * kUnits / chunks;
        const int64_t each = tiles < most ? tiles : most > 1 ? most : 1;
        auto run = [&](auto streams) {
            xent_few_head_kernel<T, decltype(streams)::value>
                <<<(unsigned)((chunks * each + kWaves - 1) / kWaves), kThreads, 0, s>>>(a, (int)first, (int)words, ldg, (int)chunks, (int)each);
        };
        whole ? run(std::true_type()) : run(std::false_type());
    });
    return hipGetLastError();
}

}  // namespace nacho
