// Softmax cross entropy of rows against a large vocabulary, from the rows x and the vocabulary's weights W, without keeping the
// logits z_iv = <x_i, W_v>:
//
//   lse_i = log sum_v exp z_iv        loss_i = w_i (lse_i - z_i,label)
//   g_iv  = w_i (exp(z_iv - lse_i) - [v = label_i])        grad_x = g W        grad_W = g^T x
//
// Three products on the tiles of products.hpp.  The loss: a tile of logits leaves the matrix units as the largest one of each row
// and the sum of exponentials under it; a small kernel joins the tiles of a row.  The gradient makes the logits again, in pieces of
// the vocabulary whose g (rounded to the type, which the matrix units take) fits a fixed room, from where both products read it.
// grad_x then is a sum over pieces, and over stretches of the vocabulary where there are too few tiles for the chip, held in 32 bits.
//
// Rows that do not count (no label in the vocabulary, weight 0) are left out before the first product: it reads the others by a list.
//
// g is rounded to the type because the matrix units take it: gradients in bf16 are off by 2.4e-3 (a result's own rounding is 1.7e-3), in f16 by
// 3.0e-4 (2.1e-4).  Second products for what the rounding leaves would take as long as grad_x and grad_W, 2 ms more than the 3.9 below.
//
// Bound by the matrix units: 4096 x 65536 x 2048 bf16, loss and gradients, 3.93 ms a pass for 4 products of 1.1 TFLOP, 1120 TFLOP/s.  (Kernels
// alone, the least and the median of nine: the loss 909 and 937 us, 1210 TFLOP/s; the pieces' g 2 x 479 and 2 x 496, grad_x 2 x 436 and 2 x 460,
// grad_W 2 x 543 and 2 x 570; what lists and joins them 74 and 77.)  Few rows by the weights: xent_few.hip.
#include "xent.hpp"

namespace nacho {

namespace {

constexpr int kRowThreads = 1024;

template <typename Label> __device__ inline bool row_counts(const XentArgs &a, int64_t i)
{
    const Label label = static_cast<const Label *>(a.label)[i];
    return label >= 0 && label < (Label)a.vocabulary && (!a.weight || a.weight[i] != 0.0f);
}

// How many rows count, and the largest weight of one, by workgroups of xent_rows_kernel.
template <typename Label> __global__ void __launch_bounds__(kRowThreads) xent_count_kernel(XentArgs a, int each)
{
    constexpr int kWaves = kRowThreads / NACHO_WAVE;
    __shared__ int counts[kWaves];
    __shared__ float share[kWaves];
    const int tid = (int)threadIdx.x, wave = tid / NACHO_WAVE;
    const int64_t begin = (int64_t)blockIdx.x * each * kRowThreads, behind = begin + (int64_t)each * kRowThreads, end = behind < a.rows ? behind : a.rows;
    int count = 0;
    float most = 0.0f;
#pragma unroll 4
    for (int64_t i = begin + tid; i < end; i += kRowThreads) {
        const bool held = row_counts<Label>(a, i);
        count += held;
        if (a.scale && a.weight) most = held ? fmaxf(most, fabsf(a.weight[i])) : most;
    }
    count = wave_sum(count);
    most = wave_all(most, MaxOf());
    if (lane_id() == 0) {
        counts[wave] = count;
        share[wave] = most;
    }
    __syncthreads();
    if (tid != 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        count += counts[w];
        most = fmaxf(most, share[w]);
    }
    a.counts[blockIdx.x] = count;
    a.most[blockIdx.x] = most;
}

// The list of the rows that count, ascending, and by it their labels (and weights and lse, for the gradient).  Every workgroup has
// `each` x kRowThreads rows, and knows how many count before them from xent_count_kernel or, where there is no a.counts, counts them
// itself.  The loss's call clears the results of the other rows.
template <typename Label> __global__ void __launch_bounds__(kRowThreads) xent_rows_kernel(XentArgs a, int each)
{
    constexpr int kWaves = kRowThreads / NACHO_WAVE;
    __shared__ int counts[kWaves];
    __shared__ float share[kWaves];
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid / NACHO_WAVE;
    const int64_t begin = (int64_t)blockIdx.x * each * kRowThreads;
    int before = 0;
    if (a.counts) before = tid < (int)blockIdx.x ? a.counts[tid] : 0;
    else {
#pragma unroll 4
        for (int64_t i = tid; i < begin; i += kRowThreads) before += row_counts<Label>(a, i);
    }
    before = wave_sum(before);
    if (lane == 0) counts[wave] = before;
    __syncthreads();
    before = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) before += counts[w];
    __syncthreads();
    for (int64_t first = begin; first < begin + (int64_t)each * kRowThreads && first < a.rows; first += kRowThreads) {
        const int64_t i = first + tid;
        const bool held = i < a.rows && row_counts<Label>(a, i);
        const unsigned long long who = __ballot(held);
        if (lane == 0) counts[wave] = __popcll((long long)who);
        __syncthreads();
        int slot = before + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0));
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            slot += w < wave ? counts[w] : 0;
            before += counts[w];
        }
        __syncthreads();
        if (held) {
            a.token[slot] = (int32_t)i;
            a.slot_label[slot] = (int32_t)static_cast<const Label *>(a.label)[i];
            if (a.slot_lse) {
                a.slot_lse[slot] = a.lse[i];
                a.factor[slot] = a.weight ? a.weight[i] : 1.0f;
            }
        } else if (i < a.rows && a.loss) a.loss[i] = a.lse[i] = 0.0f;
        if (a.slot_of && i < a.rows) a.slot_of[i] = held ? slot : -1;
    }
    if (blockIdx.x == gridDim.x - 1 && tid == 0) {
        a.bounds[0] = 0;
        a.bounds[1] = before;
    }
    if (!a.scale || blockIdx.x != 0) return;
    float most = 0.0f;
    if (a.counts) most = tid < (int)gridDim.x ? a.most[tid] : 0.0f;
    else if (a.weight) {
        for (int64_t j = tid; j < a.rows; j += kRowThreads) most = row_counts<Label>(a, j) ? fmaxf(most, fabsf(a.weight[j])) : most;
    }
    most = wave_all(most, MaxOf());
    if (lane == 0) share[wave] = most;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, share[w]);
        if (!a.weight) most = 1.0f;
        const int by = a.half ? scale_exponent(most) : 0;
        a.scale[0] = ldexpf(1.0f, by);
        a.scale[1] = ldexpf(1.0f, -by);
    }
}

// The loss: of every row of a tile the largest logit and the sum of exponentials under it; and the label's logit, from the tile
// that has it.
struct Statistics {
    static constexpr bool kParts = false;
    static constexpr unsigned parts() { return 1; }
    const int32_t *label;
    float2 *partial;               // [tiles of columns][rows], of the piece
    int64_t rows;
    float *at_label;
    int32_t first;                 // the piece's first word of the vocabulary
    template <typename Tile>
    __device__ void end(const ProductArgs &a, const Place &at, v4f (&acc)[Tile::kFragM][Tile::kFragN], char *stage0, char *) const
    {
        const int lane = lane_id(), c0 = at.n0 + at.wn + lane / 16 * 4;
        float2 *const share = reinterpret_cast<float2 *>(stage0);                  // [wavefronts along n][rows]
        const bool whole = at.n0 + at.wn + Tile::kTileN <= a.n;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Tile::kFragM; ++i) {
            if (!whole) {
#pragma unroll
                for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] = c0 + j * 16 + e < a.n ? acc[i][j][e] : -kInfinity;
            }
            float top = -kInfinity;
#pragma unroll
            for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, acc[i][j][e]);
            top = fmaxf(top, __shfl_xor(top, 16, NACHO_WAVE));
            top = fmaxf(top, __shfl_xor(top, 32, NACHO_WAVE));
            const float base = top == -kInfinity ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += exp2_of((acc[i][j][e] - base) * kLog2e);
            sum += __shfl_xor(sum, 16, NACHO_WAVE);
            sum += __shfl_xor(sum, 32, NACHO_WAVE);
            const int r = at.wm + i * 16 + lane % 16;
            const unsigned m = (unsigned)at.m0 + r;
            const bool there = m < (unsigned)at.m_end;
            const int c = there ? label[m] - first - c0 : -1;
            if (__any(c >= 0 && c < Tile::kTileN)) {
#pragma unroll
                for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c == j * 16 + e) at_label[m] = acc[i][j][e];
            }
            if (lane < 16) share[at.wn / Tile::kTileN * Tile::kTall + r] = make_float2(top, sum);
        }
        __syncthreads();
        for (int r = (int)threadIdx.x; r < Tile::kTall; r += Tile::kThreads) {
            const unsigned m = (unsigned)at.m0 + r;
            if (m >= (unsigned)at.m_end) break;
            float top = -kInfinity, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < Tile::kColumns; ++w) top = fmaxf(top, share[w * Tile::kTall + r].x);
#pragma unroll
            for (int w = 0; w < Tile::kColumns; ++w) {
                const float2 part = share[w * Tile::kTall + r];
                sum += part.x == top ? part.y : part.y * exp2_of((part.x - top) * kLog2e);
            }
            partial[at.n0 / Tile::kWide * rows + m] = make_float2(top, sum);
        }
    }
};

// The tiles of a row: 16 rows a workgroup, 64 threads each.
constexpr int kJoinRows = 16, kJoinParts = 64;
__global__ void __launch_bounds__(kJoinRows *kJoinParts) xent_join_kernel(XentArgs a, int tiles)
{
    __shared__ float2 share[kJoinParts][kJoinRows];
    const int r = (int)threadIdx.x % kJoinRows, part = (int)threadIdx.x / kJoinRows;
    const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kJoinRows, m = first + r, held = a.bounds[1];
    if (first >= held) return;
    auto join = [](float2 x, float2 y) {
        const float top = fmaxf(x.x, y.x);
        const float sx = x.x == top ? x.y : x.y * exp2_of((x.x - top) * kLog2e), sy = y.x == top ? y.y : y.y * exp2_of((y.x - top) * kLog2e);
        return make_float2(top, sx + sy);
    };
    float2 v = make_float2(-kInfinity, 0.0f);
    if (m < held) {
        constexpr int kBatch = 16;
        for (int t = part; t < tiles; t += kBatch * kJoinParts) {
            float2 next[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) next[i] = a.partial[(int64_t)(t + i * kJoinParts < tiles ? t + i * kJoinParts : t) * a.rows + m];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (t + i * kJoinParts < tiles) v = join(v, next[i]);
        }
    }
    share[part][r] = v;
    __syncthreads();
    for (int half = kJoinParts / 2; half > 0; half /= 2) {
        if (part < half) share[part][r] = join(share[part][r], share[part + half][r]);
        __syncthreads();
    }
    if (part != 0 || m >= held) return;
    v = share[0][r];
    // (a row of nothing but -inf has no distribution)
    const float lse = v.x == -kInfinity ? __builtin_nanf("") : v.x + logf(v.y);
    const int64_t t = a.token[m];
    a.lse[t] = lse;
    a.loss[t] = (a.weight ? a.weight[t] : 1.0f) * (lse - a.at_label[m]);
}

// The gradient of a piece's logits, as rows of the type.
struct Gradient {
    static constexpr bool kParts = false;
    static constexpr unsigned parts() { return 1; }
    const int32_t *label;
    const float *lse, *factor, *scale;
    int32_t first;                 // the piece's first word of the vocabulary
    template <typename Tile>
    __device__ void end(const ProductArgs &a, const Place &at, v4f (&acc)[Tile::kFragM][Tile::kFragN], char *stage0, char *stage1) const
    {
        typedef typename Tile::type T;
        const int lane = lane_id(), c0 = at.n0 + at.wn + lane / 16 * 4;
        const float by = scale[0];
        float l[Tile::kFragM], w[Tile::kFragM];
        int c[Tile::kFragM];
#pragma unroll
        for (int i = 0; i < Tile::kFragM; ++i) {
            const unsigned m = (unsigned)at.m0 + at.wm + i * 16 + lane % 16;
            const unsigned row = m < (unsigned)at.m_end ? m : (unsigned)at.m_end - 1;
            l[i] = lse[row];
            w[i] = factor[row] * by;
            c[i] = label[row] - first - c0;
        }
#pragma unroll
        for (int i = 0; i < Tile::kFragM; ++i) {
#pragma unroll
            for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = exp2_of((acc[i][j][e] - l[i]) * kLog2e);
            if (__any(c[i] >= 0 && c[i] < Tile::kTileN)) {
#pragma unroll
                for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] -= c[i] == j * 16 + e ? 1.0f : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < Tile::kFragN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] *= w[i];
        }
        // (rows of g are whole words of 8 elements: zeros behind the piece's last one)
        T *const out = static_cast<T *>(a.out);
        Tile::each_row(a, at, acc, stage0, stage1, [&](unsigned m, int n, int width, float (&v)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < width ? v[e] : 0.0f;
            Tile::put(out + (int64_t)m * a.ldo + n, v, 8);
        });
    }
};

// Eight results of a row that starts anywhere.
template <typename T> __device__ inline void put_anywhere(T *to, const float (&v)[8], int width)
{
    typename Word<T>::type w[8 / Word<T>::n];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e / Word<T>::n][e % Word<T>::n] = (T)v[e];
    if (width >= 8) __builtin_memcpy(to, w, sizeof w);
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < width) to[e] = w[e / Word<T>::n][e % Word<T>::n];
    }
}

// Gradients of the rows: sums in 32 bits by stretches of the vocabulary, or, where there is one, the result itself.
struct RowGradients {
    static constexpr bool kParts = true;
    unsigned parts() const { return stretches.most; }
    __device__ int k_part(int live) const { return sums ? stretches.of(live) : stretches.words; }
    Stretches stretches;
    float *sums;                   // [stretches][rows that count][ld], or NULL
    int64_t ld;
    bool first;                    // (the sums hold nothing yet)
    const int32_t *token;
    const float *scale;
    int32_t inner;                 // columns of the result (the product may have a few more)
    template <typename Tile>
    __device__ void end(const ProductArgs &a, const Place &at, v4f (&acc)[Tile::kFragM][Tile::kFragN], char *stage0, char *stage1) const
    {
        typedef typename Tile::type T;
        if (sums) {
            float *const to = sums + (int64_t)at.stretch * at.m_end * ld;
            Tile::each_row(a, at, acc, stage0, stage1, [&](unsigned m, int n, int, float (&v)[8]) {
                v4f *const p = reinterpret_cast<v4f *>(to + (int64_t)m * ld + n);
                v4f lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
                if (!first) {
                    lo += p[0];
                    hi += p[1];
                }
                p[0] = lo;
                p[1] = hi;
            });
        } else {
            const float by = scale[1];
            T *const out = static_cast<T *>(a.out);
            Tile::each_row(a, at, acc, stage0, stage1, [&](unsigned m, int n, int, float (&v)[8]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= by;
                put_anywhere(out + (int64_t)token[m] * a.ldo + n, v, inner - n);
            });
        }
    }
};

// Gradients of the vocabulary's weights, without the scale.
struct HeadGradients {
    static constexpr bool kParts = false;
    static constexpr unsigned parts() { return 1; }
    const float *scale;
    int32_t last, inner;           // words of the piece, columns (rows of g, and the product, may have a few more)
    template <typename Tile>
    __device__ void end(const ProductArgs &a, const Place &at, v4f (&acc)[Tile::kFragM][Tile::kFragN], char *stage0, char *stage1) const
    {
        typedef typename Tile::type T;
        const float by = scale[1];
        T *const out = static_cast<T *>(a.out);
        Place mine = at;
        mine.m_end = last;
        Tile::each_row(a, mine, acc, stage0, stage1, [&](unsigned m, int n, int, float (&v)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= by;
            put_anywhere(out + (int64_t)m * a.ldo + n, v, inner - n);
        });
    }
};

// A row's gradient from its sums, zeros for a row that does not count (without sums: these alone).  A workgroup has 256 columns of a
// row, a wavefront every fourth stretch of them.  (16 rows, 32 stretches of 512 columns: a thread with all stretches of 4 columns took 6 us
// more a call; with 2 stretches both take the same.)
constexpr int kSumColumns = 256;
template <typename T> __global__ void __launch_bounds__(256) xent_row_gradients_kernel(XentArgs a, Stretches parts, int64_t ld, int chunks)
{
    constexpr int kWaves = 256 / NACHO_WAVE, kBatch = 8;
    __shared__ v4f share[kWaves][NACHO_WAVE];
    const int64_t number = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, t = number / chunks;
    if (t >= a.rows) return;
    const int slot = a.slot_of[t], lane = lane_id(), wave = (int)threadIdx.x / NACHO_WAVE;
    if (slot >= 0 && !a.sums) return;
    const int c = (int)(number - t * chunks) * kSumColumns + lane * 4;
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (slot >= 0) {
        const int live = a.bounds[1], k_part = parts.of(live), stretches = (parts.words + k_part - 1) / k_part;
        const int64_t part_stride = live * ld;
        const float *from = a.sums + slot * ld + (c < ld ? c : 0);
        for (int p = wave; p < stretches; p += kBatch * kWaves) {
            v4f next[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                next[i] = *reinterpret_cast<const v4f *>(from + (int64_t)(p + i * kWaves < stretches ? p + i * kWaves : p) * part_stride);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (p + i * kWaves < stretches) v += next[i];
        }
        share[wave][lane] = v;
        __syncthreads();
        v = share[0][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += share[w][lane];
    }
    if (wave != 0 || c >= a.inner) return;
    const float by = a.scale[1];
    T *const out = static_cast<T *>(a.grad_x) + t * a.ldgx + c;
    if (c + 4 <= a.inner) {
        typedef T four __attribute__((ext_vector_type(4)));
        const four w = {(T)(v[0] * by), (T)(v[1] * by), (T)(v[2] * by), (T)(v[3] * by)};
        __builtin_memcpy(out, &w, sizeof w);
    } else {
        for (int e = 0; c + e < a.inner; ++e) out[e] = (T)(v[e] * by);
    }
}

// Rows (by a list, or all of them) whose words of 16 bytes start anywhere, as rows of whole words with zeros behind their end.
template <typename T>
__global__ void __launch_bounds__(256) xent_pad_kernel(const void *from, int64_t ld, int cols, const int32_t *list, const int32_t *held, int64_t rows,
                                                       void *to, int64_t ldp)
{
    const int words = (int)(ldp / Word<T>::n);
    const int64_t most = held ? (int64_t)*held : rows, each = (int64_t)gridDim.x * (256 / NACHO_WAVE);
    for (int64_t r = (int64_t)blockIdx.x * (256 / NACHO_WAVE) + (int)threadIdx.x / NACHO_WAVE; r < most; r += each) {
        const T *row = static_cast<const T *>(from) + (list ? (int64_t)list[r] : r) * ld;
        for (int w = lane_id(); w < words; w += NACHO_WAVE) {
            const Ragged<T, false> word(cols, w * Word<T>::n);
            *reinterpret_cast<v4u *>(static_cast<T *>(to) + r * ldp + w * Word<T>::n) = word.placed(word.load(row + w * Word<T>::n));
        }
    }
}

int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }

// Rows for the choice of tiles: one group, whose last tile counts as a whole one of 128 from 33 rows of 16 bits on (tiles of 32 rows would
// read the vocabulary's weights several times).  (Loss and gradients, us a pass with whole tiles and without, a graph's start included, bf16:
// 40 x 65536 x 2048 292 and 322, 500 x 65536 x 1024 362 and 381, 2000 x 32000 x 1024 549 and 583.  f32, whose time is the matrix units':
// 64 x 32000 x 1024 328 and 240, 300 x 30001 x 777 827 and 725.)
int64_t counted(int elem, int64_t rows) { return elem == 2 && rows > 32 ? (rows + 127) / 128 * 128 : rows; }

// The rows that count and a piece of the vocabulary as the products read them: where they lie, or from the workspace as rows of whole
// words.
struct Sides {
    const void *x, *head;
    int64_t ldx, ldh;
    const int32_t *token;          // rows of x, or NULL: they lie one after the other
    int32_t inner;
    Access access;
};
Access access_of_rows(const XentArgs &a)
{
    const bool words = a.ldx < 0x7fffffff && a.ldh < 0x7fffffff && in_words({{a.x, a.ldx}, {a.head, a.ldh}, {a.x, a.inner}}, a.elem);
    return words ? WORDS : a.inner * a.elem < 16 ? TINY : ANYWHERE;
}
template <typename T>
hipError_t pad(const void *from, int64_t ld, const XentArgs &a, const int32_t *list, const int32_t *held, int64_t rows, void *to, hipStream_t s)
{
    const int64_t groups = (rows + 3) / 4;
    xent_pad_kernel<T><<<(unsigned)(groups < 8 * kUnits ? groups : 8 * kUnits), 256, 0, s>>>(from, ld, a.inner, list, held, rows, to, padded(a.inner));
    return hipGetLastError();
}
// (the rows of x are copied with the first piece)
template <typename T> hipError_t sides_of(const XentArgs &a, int64_t first, int64_t words, Sides *v, hipStream_t s)
{
    const void *head = static_cast<const T *>(a.head) + first * a.ldh;
    *v = Sides{a.x, head, a.ldx, a.ldh, a.token, a.inner, access_of_rows(a)};
    if (!a.padded_x) return hipSuccess;
    *v = Sides{a.padded_x, a.padded_head, padded(a.inner), padded(a.inner), nullptr, (int32_t)padded(a.inner), WORDS};
    if (first == 0)
        if (const hipError_t e = pad<T>(a.x, a.ldx, a, a.token, a.bounds + 1, a.rows, a.padded_x, s)) return e;
    return pad<T>(head, a.ldh, a, nullptr, nullptr, words, a.padded_head, s);
}

ProductArgs logits_of(const XentArgs &a, const Sides &v, int64_t words)
{
    ProductArgs p{};
    p.bounds = a.bounds;
    p.token = v.token;
    p.experts = 1;
    p.n = (int32_t)words;
    p.k = v.inner;
    p.slots = counted(a.elem, a.rows);
    p.q = v.x;
    p.ldq = v.ldx;
    p.p = v.head;
    p.ldp = v.ldh;
    return p;
}

// Few rows of words of 16 bytes go without LDS.  (65536 x 2048 bf16, us a call without LDS and by tiles, a graph's start included: 1 row 58
// and 79, 16 rows 62 and 79, 48 rows 85 and 85, 64 rows 92 and 84; x 1024: 16 rows 41 and 41, 24 rows 44 and 41.  Rows of 16
// bits that start anywhere go by tiles all the same: 16 rows against 100003 x 999, 66 us by tiles, 86 without LDS.  Such rows of floats, which
// memory has no narrower access for, go without as long as the rows of x fit the nearest cache: 16 rows x 20000 x 501 24 us without LDS and 34
// by tiles, 4 rows x 50622 x 3867 192 and 202, 16 rows x 50622 x 1999 126 and 119.)
bool few_rows(const XentArgs &a)
{
    const Access access = access_of_rows(a);
    return a.rows <= kFewRows && (access == WORDS || (access == ANYWHERE && a.elem == 4 && a.rows * a.inner <= 1 << 14));
}

// (the narrowest tiles there can be)
int64_t tiles_of_loss(int elem, int64_t rows, int64_t vocabulary)
{
    const int64_t wide = elem == 2 ? 128 : tiny_tiles(rows, 1, vocabulary) ? 32 : 64;
    return (vocabulary + wide - 1) / wide;
}

// How the rows are listed: `groups` workgroups of `each` x kRowThreads rows.  Workgroups that each count all rows before theirs read as many as
// the square of the rows; from kCountedFrom on a launch of its own counts them first, kRowThreads numbers at most.  (Loss and gradients against
// 8 x 8, us a pass so and without: 16384 rows 184 and 185, 32768 336 and 344, 131072 1240 and 1327, 16 million 168 and 535 ms.)
constexpr int64_t kCountedFrom = 1 << 15;
struct Lists {
    int64_t groups;
    int32_t each;
    explicit Lists(int64_t rows)
    {
        const int64_t chunks = rows > 0 ? (rows + kRowThreads - 1) / kRowThreads : 1;
        each = rows >= kCountedFrom ? (int32_t)((chunks + kRowThreads - 1) / kRowThreads) : 1;
        groups = (chunks + each - 1) / each;
    }
};
template <typename Label> hipError_t list_rows_of(const XentArgs &a, hipStream_t s)
{
    const Lists lists(a.rows);
    if (a.counts) {
        xent_count_kernel<Label><<<(unsigned)lists.groups, kRowThreads, 0, s>>>(a, lists.each);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    xent_rows_kernel<Label><<<(unsigned)lists.groups, kRowThreads, 0, s>>>(a, lists.each);
    return hipGetLastError();
}
hipError_t list_rows(const XentArgs &a, hipStream_t s)
{
    return a.label_bytes == 8 ? list_rows_of<int64_t>(a, s) : list_rows_of<int32_t>(a, s);
}

}  // namespace

int64_t xent_counts(int64_t rows) { return rows >= kCountedFrom ? Lists(rows).groups : 0; }

int64_t xent_partials(int elem, int64_t rows, int64_t vocabulary)
{
    const int64_t few = rows <= kFewRows ? xent_few_groups(vocabulary) : 0, tiles = tiles_of_loss(elem, rows, vocabulary);
    return (few > tiles ? few : tiles) * rows;
}

// Whether the products read copies of the rows and of the vocabulary's weights.  Rows that start anywhere take up to twice the time in the
// products; the copies are two passes over the weights a call.  (Loss and gradients, us a pass with copies and without, bf16, 32003 x 1001
// and 100003 x 499: 200 rows 217 and 197, 347 and 330; 300 rows 291 and 295, 464 and 427; 400 rows 284 and 315, 493 and 511; 1500 rows 557
// and 773.  4000 rows, 50001 x 1999: 3575 and 5374.)
bool xent_pads(const XentArgs &a) { return a.elem == 2 && a.rows >= kPaddedFrom && access_of_rows(a) == ANYWHERE; }

// The pieces of the vocabulary: g of one takes at most 256 MiB (which the last cache holds), or 256 words of it; and so do its weights
// where they are copied.  The loss's call, which has no g, goes by these alone.  (Loss and gradients, bf16, us with 128, 256 and 512 MiB:
// 4096 x 65536 x 2048 3740, 3850 and 3876; 16384 x 32000 x 1024 4743, 4258 and 4300.)
XentPlan xent_plan(int elem, int64_t rows, int64_t vocabulary, int64_t inner, bool pads, bool gradient)
{
    constexpr int64_t kRoom = 256 << 20;
    XentPlan p;
    const int64_t by_g = rows > 0 && gradient ? kRoom / (rows * elem) / 256 * 256 : vocabulary;
    const int64_t by_copy = pads ? kRoom / (padded(inner) * elem) / 256 * 256 : vocabulary;
    const int64_t most = by_g < by_copy ? by_g : by_copy, least = most > 256 ? most : 256;
    p.pieces = (vocabulary + least - 1) / least;
    p.words = p.pieces > 1 ? ((vocabulary + p.pieces - 1) / p.pieces + 255) / 256 * 256 : vocabulary;
    if (p.pieces > 1 && elem == 2 && inner >= 256) {
        // As many words as fill whole rounds of grad_W's workgroups, if there is room and its rounds and those of g, which go through the
        // rows and the rows' elements, are shorter together.  (Loss and gradients, bf16, us so and with equal pieces: 3000 x 100000 x 2048
        // 4735 and 4965, 8192 x 50000 x 1024 3403 and 3665; where they are as long, 4096 x 128000 x 1024, 4260 and 4189.)
        const int64_t wide = (inner + 255) / 256, tall = (rows + 255) / 256;
        auto rounds = [&](int64_t words) {
            const int64_t tiles = (words + 255) / 256;
            return (tiles * wide + kUnits - 1) / kUnits * rows + (tiles * tall + kUnits - 1) / kUnits * inner;
        };
        auto all = [&](int64_t words) { return vocabulary / words * rounds(words) + rounds(vocabulary % words); };
        int64_t unit = 256;
        while (unit < 256 * kUnits && unit / 256 * wide % kUnits) unit *= 2;
        const int64_t words = (p.words + unit - 1) / unit * unit;
        if (words <= most && all(words) < all(p.words)) p.words = words;
    }
    p.pieces = (vocabulary + p.words - 1) / p.words;
    p.ldg = padded(p.words);
    // stretches of a piece, where its rows alone are too few tiles for the chip (loss and gradients, us a pass with stretches and without,
    // bf16: 64 x 32000 x 1024 112 and 281, 500 x 65536 x 1024 362 and 653; 4096 x 65536 x 2048, with twice the pieces' 128 tiles, 3850 and 4087)
    const bool large = rows >= 256 && inner >= 256;
    const int64_t tall = rows <= 32 ? 32 : elem == 4 ? 64 : large ? 256 : 128, wide = rows <= 32 ? 128 : elem == 4 ? 64 : large ? 256 : 128;
    const int64_t tiles = ((rows + tall - 1) / tall) * ((inner + wide - 1) / wide);
    int64_t wanted = tiles > 0 ? 2 * kUnits / tiles : 1;
    if (elem == 2 && large && tiles > 0 && (tiles < kUnits || p.pieces > 1)) {
        // (A compute unit has one such tile at a time.)  As few stretches as fill whole rounds of workgroups; or else about two rounds, or,
        // where these leave a tenth of the chip without work, up to four.  (us so and with two rounds whatever they fill: 500 x 65536 x 1024
        // 362 and 405, 2000 x 32000 x 1024 549 and 589, 16384 x 32000 x 1024 4258 and 4363.)
        auto empty = [&](int64_t n) { return 1000 - 1000 * n * tiles / ((n * tiles + kUnits - 1) / kUnits * kUnits); };      // of a thousand
        const int64_t two = wanted > 1 ? wanted : 1;
        wanted = two;
        if (empty(two) > 100)
            for (int64_t n = 1; n * tiles <= 4 * kUnits; ++n) wanted = empty(n) < empty(wanted) ? n : wanted;
        for (int64_t n = two; n >= 1; --n) wanted = empty(n) <= 20 ? n : wanted;
    }
    p.shortest = large ? 1024 : 256;
    const int64_t longest = (p.words + p.shortest - 1) / p.shortest;
    p.stretches = wanted < longest ? wanted : longest;
    if (p.stretches < 1) p.stretches = 1;
    p.k_part = ((p.words + p.stretches - 1) / p.stretches + 127) / 128 * 128;
    p.stretches = (p.words + p.k_part - 1) / p.k_part;
    p.lds = padded(inner);
    p.sums = p.pieces > 1 || p.stretches > 1;
    return p;
}

hipError_t launch_xent(int dtype, const XentArgs &a, const XentPlan &plan, hipStream_t s)
{
    if (a.rows == 0) return hipSuccess;
    hipError_t rc = few_rows(a) ? hipSuccess : list_rows(a, s);
    if (rc != hipSuccess) return rc;
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        int64_t parts = 0;
        if (few_rows(a)) {
            parts = xent_few_groups(a.vocabulary);
            rc = launch_xent_few(dtype, a, 0, a.vocabulary, 0, access_of_rows(a) == WORDS, s);
        } else {
            for (int64_t first = 0; first < a.vocabulary; first += plan.words) {
                const int64_t words = a.vocabulary - first < plan.words ? a.vocabulary - first : plan.words;
                Sides v;
                rc = sides_of<T>(a, first, words, &v, s);
                if (rc != hipSuccess) return;
                const ProductArgs p = logits_of(a, v, words);
                const int wide = wide_of(shape_of<T, FORWARD>(p, v.access));
                rc = by_size<T, FORWARD>(p, Statistics{a.slot_label, a.partial + parts * a.rows, a.rows, a.at_label, (int32_t)first}, v.access, s);
                if (rc != hipSuccess) return;
                parts += (words + wide - 1) / wide;
            }
        }
        if (rc != hipSuccess) return;
        // (a launch holds 2^32 threads along its first dimension)
        const int64_t groups = (a.rows + kJoinRows - 1) / kJoinRows, row = groups < (1 << 20) ? groups : 1 << 20;
        xent_join_kernel<<<dim3((unsigned)row, (unsigned)((groups + row - 1) / row)), kJoinRows * kJoinParts, 0, s>>>(a, (int)parts);
        rc = hipGetLastError();
    });
    return rc;
}

hipError_t launch_xent_grad(int dtype, const XentArgs &a, const XentPlan &plan, hipStream_t s)
{
    hipError_t rc = few_rows(a) ? hipSuccess : list_rows(a, s);
    if (rc != hipSuccess) return rc;
    const int elem = a.elem;
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        Stretches stretches = {};
        for (int64_t first = 0; first < a.vocabulary; first += plan.words) {
            const int64_t words = a.vocabulary - first < plan.words ? a.vocabulary - first : plan.words;
            Sides v;
            rc = sides_of<T>(a, first, words, &v, s);
            if (rc != hipSuccess) return;
            ProductArgs p = logits_of(a, v, words);
            p.out = a.g;
            p.ldo = plan.ldg;
            rc = few_rows(a) ? launch_xent_few(dtype, a, first, words, plan.ldg, access_of_rows(a) == WORDS, s)
                             : by_size<T, FORWARD>(p, Gradient{a.slot_label, a.slot_lse, a.factor, a.scale, (int32_t)first}, v.access, s);
            if (rc != hipSuccess) return;
            if (a.grad_x) {
                p = ProductArgs{};
                p.bounds = a.bounds;
                p.experts = 1;
                p.n = v.inner;
                p.k = (int32_t)words;
                p.slots = counted(a.elem, a.rows);
                p.q = a.g;
                p.ldq = plan.ldg;
                p.p = v.head;
                p.ldp = v.ldh;
                p.out = a.grad_x;
                p.ldo = a.ldgx;
                const Access access = v.access == WORDS && plan.ldg < 0x7fffffff ? WORDS : access_of<ROWS>(p, elem);
                if (first == 0)
                    stretches = Stretches{(int32_t)plan.stretches, (int32_t)plan.k_part, tall_of(shape_of<T, ROWS>(p, access, plan.stretches)),
                                          (int32_t)plan.words, (int32_t)plan.shortest, a.rows};
                const RowGradients f{stretches, plan.sums ? a.sums : nullptr, plan.lds, first == 0, a.token, a.scale, a.inner};
                rc = by_size<T, ROWS>(p, f, access, s);
                if (rc != hipSuccess) return;
            }
            if (a.grad_head && a.rows <= kFewRows) {
                rc = launch_xent_few_head(dtype, a, first, words, plan.ldg, s);
                if (rc != hipSuccess) return;
            } else if (a.grad_head) {
                p = ProductArgs{};
                p.bounds = a.bounds;
                p.token = v.token;
                p.experts = 1;
                p.n = v.inner;
                p.slots = counted(a.elem, a.rows);
                p.q = a.g;
                p.ldq = plan.ldg;
                p.p = v.x;
                p.ldp = v.ldx;
                p.out = static_cast<T *>(a.grad_head) + first * a.ldgh;
                p.ldo = a.ldgh;
                const bool in = v.access == WORDS && plan.ldg < 0x7fffffff;
                p.m = (int32_t)(in ? padded(words) : words);
                rc = by_size<T, WEIGHTS>(p, HeadGradients{a.scale, (int32_t)words, a.inner}, in ? WORDS : access_of<WEIGHTS>(p, elem), s);
                if (rc != hipSuccess) return;
            }
        }
        if (a.grad_x && a.rows > 0) {
            XentArgs b = a;
            if (!plan.sums) b.sums = nullptr;
            const int64_t chunks = (a.inner + kSumColumns - 1) / kSumColumns, all = a.rows * chunks, row = all < (1 << 22) ? all : 1 << 22;
            xent_row_gradients_kernel<T><<<dim3((unsigned)row, (unsigned)((all + row - 1) / row)), 256, 0, s>>>(
                b, stretches, plan.lds, (int)chunks);
            rc = hipGetLastError();
        }
    });
    return rc;
}

}  // namespace nacho
