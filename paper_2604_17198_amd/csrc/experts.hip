// The products of a mixture of experts: one dense layer over the ragged groups of rows that a routing leaves.
//
//   forward   y_s = act(x_token(s) W_e^T + b_e)       rows    grad_x_s = g_s W_e       weights  grad_W_e = sum_s g_s^T x_token(s)
//
// The tiles are those of products.hpp; here is what becomes of their results, and the slopes on the way back.
//
// Bound by the matrix units for many slots an expert (16384 bf16 slots of 16 experts, 2048 x 8192: 612 to 657 us a call by the
// card, 837 to 898 TFLOP/s of the 1211 of a library's product of 8192^3), by the weights for few (16 of 32 experts, 2048 x 4096:
// 44 to 55 us a call for 213 MB; 32 us a kernel where the last cache still has most of them).
#include "activation.hpp"
#include "kept.hpp"
#include "products.hpp"

namespace nacho {

namespace {

constexpr int kThreads = 256;

// Results as rows of the type: with the bias and after the activation (the forward form), or as they are.
struct Rows {
    static constexpr bool kParts = false;
    static constexpr unsigned parts() { return 1; }
    template <typename Tile>
    __device__ void end(const ProductArgs &a, const Place &at, v4f (&acc)[Tile::kFragM][Tile::kFragN], char *stage0, char *stage1) const
    {
        typedef typename Tile::type T;
        T *const out = static_cast<T *>(a.out) + (Tile::form == WEIGHTS ? (int64_t)at.expert * a.out_stride : 0);
        float bias[8];
        if constexpr (Tile::form == FORWARD) bias_of<T, Tile::kTileN / 8>(a, at, bias);
        Tile::each_row(a, at, acc, stage0, stage1, [&](unsigned m, int n, int width, float (&v)[8]) {
            if constexpr (Tile::form == FORWARD) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += bias[e];
                if (a.pre) Tile::put(static_cast<T *>(a.pre) + (int64_t)m * a.ldpre + n, v, width);
                if (a.act != NACHO_ACT_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = activated<T>(v[e], a.act);
                }
            }
            Tile::put(out + (int64_t)m * a.ldo + n, v, width);
        });
    }
};

// grad_z = grad_y act'(pre), rounded to the type that the matrix units take (pre is kept in it as well, which halves what is
// written and read of it), and the sums of its rows before that rounding, over tiles of kSlopeRows rows of an expert: a workgroup
// has a tile and 16 words of 16 bytes of its columns, 16 threads along them and 16 along the rows.  Bound by memory: 16384 x 4096
// bf16, gelu, 88 us, 4.6 TB/s.
constexpr int kSlopeRows = 64;
template <typename T, Access kAccess, bool kKept>
__global__ void __launch_bounds__(kThreads) experts_slope_kernel(SlopeArgs a, int tiles_n)
{
    constexpr int n = Word<T>::n;
    typedef typename Word<T>::type word;
    __shared__ float share[16][16 * n + 1];
    const int number = (int)(blockIdx.y * gridDim.x + blockIdx.x), tile = number / tiles_n;
    const int tx = (int)threadIdx.x % 16, ty = (int)threadIdx.x / 16, c0 = (number - tile * tiles_n) * 16 * n, c = c0 + tx * n, width = a.cols - c;
    int expert, row, end;
    if (!find_tile<kSlopeRows>(a, tile, expert, row, end)) return;
    const T *gy = static_cast<const T *>(a.grad_y) + c, *pre = static_cast<const T *>(a.pre) + c;
    T *gz = static_cast<T *>(a.grad_z) + c;
    auto get = [&](const T *from) {
        if constexpr (kAccess == WORDS) return width > 0 ? *reinterpret_cast<const v4u *>(from) : v4u{0, 0, 0, 0};
        else {
            const Ragged<T, kAccess == TINY> last(a.cols, c);
            return last.placed(last.load(from));
        }
    };
    float sum[n];
#pragma unroll
    for (int e = 0; e < n; ++e) sum[e] = 0.0f;
    constexpr int kRows = kSlopeRows / 16;
    v4u g[kRows], z[kKept ? 1 : kRows];
    unsigned codes[kKept ? kRows : 1][n / 4], exponent[kKept ? kRows : 1];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const unsigned m = (unsigned)row + ty + i * 16;
        g[i] = v4u{0, 0, 0, 0};
        if constexpr (kKept) {
#pragma unroll
            for (int e = 0; e < n / 4; ++e) codes[i][e] = 0;
            exponent[i] = 0;
        } else z[i] = v4u{0, 0, 0, 0};
        if (m < (unsigned)end) {
            g[i] = get(gy + (int64_t)m * a.ldgy);
            if constexpr (kKept) {
                const int8_t *from = a.kept.code + (int64_t)m * a.kept.ldc + c;
                if (width >= n) __builtin_memcpy(codes[i], from, n);
                else {
#pragma unroll
                    for (int e = 0; e < n; ++e) codes[i][e / 4] |= e < width ? (unsigned)(uint8_t)from[e] << (8 * (e % 4)) : 0u;
                }
                if (width > 0) exponent[i] = a.kept.exponent[(int64_t)m * a.kept.lde + c / kBlock];
            } else if (a.act != NACHO_ACT_NONE) z[i] = get(pre + (int64_t)m * a.ldpre);
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const unsigned m = (unsigned)row + ty + i * 16;
        word v = __builtin_bit_cast(word, g[i]);
        // (what the sums take is not rounded to the type yet; behind the last row it is zero)
        if (a.act != NACHO_ACT_NONE) {
            float at[n];
            if constexpr (kKept) {
                const float step = step_of(exponent[i]);
#pragma unroll
                for (int e = 0; e < n; ++e) at[e] = value_of(codes[i][e / 4], e % 4, step);
            } else {
                const word rows = __builtin_bit_cast(word, z[i]);
#pragma unroll
                for (int e = 0; e < n; ++e) at[e] = wide((T)rows[e]);
            }
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float x = wide((T)v[e]) * slope_at<T>(at[e], a.act);
                v[e] = (T)x;
                sum[e] += x;
            }
        } else {
#pragma unroll
            for (int e = 0; e < n; ++e) sum[e] += wide((T)v[e]);
        }
        if (m < (unsigned)end && a.grad_z) {
            T *to = gz + (int64_t)m * a.ldgz;
            if (width >= n) {
                if constexpr (kAccess == WORDS) *reinterpret_cast<word *>(to) = v;
                else __builtin_memcpy(to, &v, 16);
            } else {
#pragma unroll
                for (int e = 0; e < n; ++e)
                    if (e < width) to[e] = v[e];
            }
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int e = 0; e < n; ++e) share[ty][tx * n + e] = sum[e];
    __syncthreads();
    for (int i = (int)threadIdx.x; i < 16 * n; i += kThreads)
        if (c0 + i < a.cols) {
            float total = 0.0f;
#pragma unroll
            for (int y = 0; y < 16; ++y) total += share[y][i];
            a.sums[(int64_t)tile * a.cols + c0 + i] = total;
        }
}

// The sums of an expert's tiles, one after the other.
template <typename T> __global__ void __launch_bounds__(kThreads) experts_bias_kernel(SlopeArgs a, int tiles_n)
{
    const int expert = (int)blockIdx.x / tiles_n, c = ((int)blockIdx.x - expert * tiles_n) * kThreads + (int)threadIdx.x;
    auto tiles_at = [&](int e) { return tiles_of<kSlopeRows>(bound_of(a, e + 1) - bound_of(a, e)); };
    int first = 0;
    for (int e0 = 0; e0 < expert; e0 += NACHO_WAVE) first += e0 + lane_id() < expert ? tiles_at(e0 + lane_id()) : 0;
    first = wave_sum(first);
    const int tiles = tiles_at(expert);
    if (c >= a.cols) return;
    float total = 0.0f;
    constexpr int kBatch = 8;
    for (int t = 0; t < tiles; t += kBatch) {
        float part[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) part[i] = a.sums[(int64_t)(first + (t + i < tiles ? t + i : tiles - 1)) * a.cols + c];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) total += t + i < tiles ? part[i] : 0.0f;
    }
    (static_cast<T *>(a.grad_bias) + (int64_t)expert * a.bias_stride)[c] = (T)total;
}

}  // namespace

hipError_t launch_experts_forward(int dtype, const ProductArgs &a, hipStream_t s) { return launch<FORWARD>(dtype, a, Rows(), s); }
hipError_t launch_experts_rows(int dtype, const ProductArgs &a, hipStream_t s) { return launch<ROWS>(dtype, a, Rows(), s); }
hipError_t launch_experts_weights(int dtype, const ProductArgs &a, hipStream_t s) { return launch<WEIGHTS>(dtype, a, Rows(), s); }

// Tiles of rows of the sums: as many as the slots fill, and a part of one for every expert that may have any.
int64_t experts_slope_tiles(int64_t slots, int64_t experts) { return slots / kSlopeRows + (slots < experts ? slots : experts); }

hipError_t launch_experts_slope(int dtype, const SlopeArgs &a, hipStream_t s)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    const bool words = in_words({{a.grad_y, a.ldgy}, {a.act && !a.kept.code ? a.pre : nullptr, a.ldpre}, {a.grad_z, a.ldgz}, {a.grad_y, a.cols}}, elem);
    hipError_t rc = hipSuccess;
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const int64_t tiles_n = (a.cols + 16 * Word<T>::n - 1) / (16 * Word<T>::n);
        const int64_t tiles = experts_slope_tiles(a.slots, a.experts) * tiles_n, row = tiles < (1 << 22) ? tiles : 1 << 22;
        const int64_t sums = (int64_t)a.experts * ((a.cols + kThreads - 1) / kThreads);
        if (tiles > 0x7fffffff - (1 << 22) || sums > (1 << 24) - 1) {
            rc = hipErrorNotSupported;
            return;
        }
        if (tiles > 0) {
            const dim3 grid((unsigned)row, (unsigned)((tiles + row - 1) / row));
            auto run = [&](auto kept) {
                constexpr bool kKept = decltype(kept)::value;
                if (words) experts_slope_kernel<T, WORDS, kKept><<<grid, kThreads, 0, s>>>(a, (int)tiles_n);
                else if (a.cols >= Word<T>::n) experts_slope_kernel<T, ANYWHERE, kKept><<<grid, kThreads, 0, s>>>(a, (int)tiles_n);
                else experts_slope_kernel<T, TINY, kKept><<<grid, kThreads, 0, s>>>(a, (int)tiles_n);
            };
            if (a.kept.code) run(std::true_type());
            else run(std::false_type());
            rc = hipGetLastError();
        }
        if (rc == hipSuccess && a.grad_bias) {
            experts_bias_kernel<T><<<dim3((unsigned)sums), kThreads, 0, s>>>(a, (int)((a.cols + kThreads - 1) / kThreads));
            rc = hipGetLastError();
        }
    });
    return rc;
}

}  // namespace nacho
