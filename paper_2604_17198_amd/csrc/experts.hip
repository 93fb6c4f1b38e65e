// The products of a mixture of experts: one dense layer over the ragged groups of rows that a routing leaves.
//
//   forward   y_s = act(x_token(s) W_e^T + b_e)       rows    grad_x_s = g_s W_e       weights  grad_W_e = sum_s g_s^T x_token(s)
//
// All three are out[m][n] = sum_k Q(m, k) P(n, k); they differ in which side's rows run along k in memory.  A workgroup
// computes a tile of kM x kN results on the matrix units, from tiles of Q and P that pass through LDS.  A side whose
// rows run along k lies there as rows of k, and a lane reads 16 bytes of its row; a side whose columns run along k lies
// there as rows of n (or m) for every k, and is transposed by the LDS on the way to the registers (16-bit types), or
// read an element at a time (floats).  P is the first operand of the matrix instruction, so that a lane ends with four
// consecutive columns of a result row.
//
// Which expert a tile belongs to is found by its workgroup from expert_pos alone (a prefix sum of the experts' tiles
// over the lanes), so nothing about the routing is read on the host.
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / NACHO_WAVE;
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));

enum Form { FORWARD, ROWS, WEIGHTS };

// acc += (16 x 64 bytes of k) (64 bytes of k x 16); a lane's 16 bytes are consecutive k of row lane % 16, the lanes'
// fours of 16 lie one after the other.  (The order of k inside a step does not matter as long as both sides agree.)
template <typename T> __device__ inline v4f matrix_step(v4u p, v4u q, v4f acc)
{
    typedef typename Word<T>::type word;
    if constexpr (sizeof(T) == 4) {
        const word a = __builtin_bit_cast(word, p), b = __builtin_bit_cast(word, q);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
        return acc;
    } else if constexpr (__is_same(T, bf16_t)) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(word, p), __builtin_bit_cast(word, q), acc, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(word, p), __builtin_bit_cast(word, q), acc, 0, 0, 0);
    }
}

// (Phi by the complement of the error function: next to one, 1 + erf has no digits left for a negative argument)
__device__ inline float normal_below(float z) { return 0.5f * erfcf(-0.70710678118654752f * z); }
__device__ inline float activated(float z, int act)
{
    if (act == NACHO_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == NACHO_ACT_GELU) return z * normal_below(z);
    if (act == NACHO_ACT_SILU) return z / (1.0f + expf(-z));
    return z;
}
// (Next to its root a slope is a difference of nearly equal numbers: of rows of floats it is taken in 64 bits, so that
// its error is a rounding's there too.)
template <typename T> __device__ inline float slope_at(float v, int act)
{
    typedef std::conditional_t<sizeof(T) == 4, double, float> Real;
    const Real z = (Real)v;
    if (act == NACHO_ACT_RELU) return v > 0.0f ? 1.0f : (v != v ? v : 0.0f);
    if (act == NACHO_ACT_GELU) {
        const Real root = (Real)0.70710678118654752440, peak = (Real)0.39894228040143267794;
        if constexpr (sizeof(T) == 4) return (float)(0.5 * erfc(-root * z) + z * peak * exp(-0.5 * z * z));
        else return 0.5f * erfcf(-root * z) + z * peak * expf(-0.5f * z * z);
    }
    if (act == NACHO_ACT_SILU) {
        Real q;
        if constexpr (sizeof(T) == 4) q = 1.0 / (1.0 + exp(-z));
        else q = 1.0f / (1.0f + expf(-z));
        return (float)(q * ((Real)1 + z * ((Real)1 - q)));
    }
    return 1.0f;
}

// The first slot of expert e (a list that runs past the slots ends there).
template <typename Args> __device__ inline int bound_of(const Args &a, int e)
{
    const int at = a.bounds[e];
    return at < (int)a.slots ? at : (int)a.slots;
}

// The expert and the first row of tile `tile` of kM rows, the experts' tiles one after the other; false behind the last.
template <int kM> __device__ inline bool find_tile(const ProductArgs &a, int tile, int &expert, int &row, int &end)
{
    const int lane = lane_id(), experts = a.experts;
    int before = 0;
    for (int e0 = 0; e0 < experts; e0 += NACHO_WAVE) {
        const int e = e0 + lane;
        int first = 0, last = 0;
        if (e < experts) {
            first = bound_of(a, e);
            last = bound_of(a, e + 1);
        }
        const int tiles = (last - first + kM - 1) / kM, upto = before + wave_inclusive_scan(tiles);
        const unsigned long long past = __ballot(upto > tile);
        if (past != 0) {
            const int at = __ffsll((long long)past) - 1;
            expert = e0 + at;
            end = __builtin_amdgcn_readlane(last, at);
            row = __builtin_amdgcn_readlane(first, at) + (tile - __builtin_amdgcn_readlane(upto - tiles, at)) * kM;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, NACHO_WAVE - 1);
    }
    return false;
}

// A side of the product: kRows rows (of Q or P), kStep bytes of k of each.
constexpr int kStep = 128, kUnits = kStep / 16;        // 16-byte words of k a row
template <typename T> constexpr int kDepth = kStep / (int)sizeof(T);

// Rows that run along k.  A thread loads the words `unit` of the rows tid / kUnits + i * 32.
template <typename T, int kRows, bool kWords> struct AlongK {
    static constexpr int kLoads = kRows * kUnits / kThreads, kBytes = kRows * kStep;
    const T *row[kLoads];
    v4u word[kLoads];
    int unit, at;

    template <typename Row> __device__ void start(Row address)
    {
        unit = (int)threadIdx.x % kUnits;
        at = (int)threadIdx.x / kUnits;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) row[i] = address(at + i * (kThreads / kUnits));
    }
    __device__ void load(int k0, int k)
    {
        constexpr int n = Word<T>::n;
        const int first = k0 + unit * n;
        if constexpr (kWords) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) word[i] = first < k ? *reinterpret_cast<const v4u *>(row[i] + first) : v4u{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                typename Word<T>::type v;
#pragma unroll
                for (int e = 0; e < n; ++e) v[e] = first + e < k ? row[i][first + e] : (T)0.0f;
                word[i] = __builtin_bit_cast(v4u, v);
            }
        }
    }
    // (8 rows' words of one column of the tile lie in all 8 columns: the 8 lanes that the LDS serves at a time read
    // different banks)
    __device__ void store(char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = at + i * (kThreads / kUnits);
            *reinterpret_cast<v4u *>(lds + r * kStep + ((unit ^ (r & 7)) << 4)) = word[i];
        }
    }
    // The lane's 16 bytes of rows r0 .. r0 + 15 in step `step` of 64 bytes.
    static __device__ v4u fragment(const char *lds, int r0, int step)
    {
        const int lane = lane_id(), r = r0 + lane % 16, u = step * 4 + lane / 16;
        return *reinterpret_cast<const v4u *>(lds + r * kStep + ((u ^ (r & 7)) << 4));
    }
};

// Columns that run along k: for every k a row of kRows elements.
template <typename T, int kRows, bool kWords> struct AcrossK {
    static constexpr int kRowBytes = kRows * (int)sizeof(T), kRowWords = kRowBytes / 16;
    static constexpr int kLoads = kDepth<T> * kRowWords / kThreads, kBytes = kDepth<T> * kRowBytes;
    v4u word[kLoads];

    // address(k): the row of k; `most`: elements of it from the tile's first one on.
    template <typename Row> __device__ void load(Row address, int k0, int k, int most)
    {
        constexpr int n = Word<T>::n;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = (int)threadIdx.x + i * kThreads, kk = k0 + u / kRowWords, first = u % kRowWords * n;
            word[i] = v4u{0, 0, 0, 0};
            if (kk < k && first < most) {
                const T *from = address(kk) + first;
                if constexpr (kWords) word[i] = *reinterpret_cast<const v4u *>(from);
                else {
                    typename Word<T>::type v;
#pragma unroll
                    for (int e = 0; e < n; ++e) v[e] = first + e < most ? from[e] : (T)0.0f;
                    word[i] = __builtin_bit_cast(v4u, v);
                }
            }
        }
    }
    // Where word w of the row of k lies: rows that are read together by one instruction lie in different banks, 32
    // bytes (16-bit types: rows k .. k + 3 of two fours of eight) or 64 bytes (floats: rows 4 apart) of each.
    static __device__ int place(int k, int w)
    {
        const int turn = sizeof(T) == 2 ? ((k & 3) | (k >> 1 & 4)) << 1 : (k >> 2 & 3) << 2;
        return k * kRowBytes + ((w ^ turn) << 4);
    }
    __device__ void store(char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = (int)threadIdx.x + i * kThreads;
            *reinterpret_cast<v4u *>(lds + place(u / kRowWords, u % kRowWords)) = word[i];
        }
    }
    static __device__ v4u fragment(const char *lds, int r0, int step)
    {
        const int lane = lane_id(), four = lane / 16, i = lane % 16;
        if constexpr (sizeof(T) == 2) {
            // the LDS hands 16 lanes four rows of 16 elements transposed: lane i gets column i of rows k .. k + 3
            v4s part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = step * 32 + four * 8 + h * 4 + i / 4, byte = (r0 + (i % 4) * 4) * 2;
                const char *at = lds + place(k, byte >> 4) + (byte & 15);
                part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)at);
            }
            typedef short v8s __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(v4u, (v8s)__builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v4u v;
            const int byte = (r0 + i) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = step * 16 + four * 4 + j;
                v[j] = *reinterpret_cast<const unsigned *>(lds + place(k, byte >> 4) + (byte & 15));
            }
            return v;
        }
    }
};

// One tile of kM x kN results; kWavesM x kWavesN wavefronts share it.
template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, bool kWords>
__global__ void __launch_bounds__(kThreads) experts_kernel(ProductArgs a, int tiles_n)
{
    static_assert(kWavesM * kWavesN == kWaves, "four wavefronts");
    constexpr int kTileM = kM / kWavesM, kTileN = kN / kWavesN, kFragM = kTileM / 16, kFragN = kTileN / 16;
    constexpr bool kAcrossQ = kForm == WEIGHTS, kAcrossP = kForm != FORWARD;
    typedef std::conditional_t<kAcrossQ, AcrossK<T, kM, kWords>, AlongK<T, kM, kWords>> SideQ;
    typedef std::conditional_t<kAcrossP, AcrossK<T, kN, kWords>, AlongK<T, kN, kWords>> SideP;
    __shared__ __attribute__((aligned(16))) char lds[2][SideQ::kBytes + SideP::kBytes];
    const int number = (int)(blockIdx.y * gridDim.x + blockIdx.x), tile = number / tiles_n, n0 = (number - tile * tiles_n) * kN;
    int expert, m0, m_end, k_begin = 0, k = a.k;
    if (kForm == WEIGHTS) {
        const int tiles_m = (a.m + kM - 1) / kM;
        expert = tile / tiles_m;
        if (expert >= a.experts) return;
        m0 = (tile - expert * tiles_m) * kM;
        m_end = a.m;
        k_begin = bound_of(a, expert);
        k = bound_of(a, expert + 1) - k_begin;
    } else if (!find_tile<kM>(a, tile, expert, m0, m_end)) return;
    const T *const q = static_cast<const T *>(a.q);
    const T *const p = static_cast<const T *>(a.p) + (int64_t)expert * a.p_stride;
    SideQ side_q;
    SideP side_p;
    // rows behind the last: the last one again, whose results are not stored
    if constexpr (!kAcrossQ)
        side_q.start([&](int r) {
            const int row = m0 + r < m_end ? m0 + r : m_end - 1;
            return q + (int64_t)(kForm == FORWARD && a.token ? a.token[row] : row) * a.ldq;
        });
    if constexpr (!kAcrossP) side_p.start([&](int r) { return p + (int64_t)(n0 + r < a.n ? n0 + r : a.n - 1) * a.ldp; });
    auto load = [&](int k0) {
        if constexpr (kAcrossQ)
            side_q.load([&](int kk) { return q + (int64_t)(k_begin + kk) * a.ldq + m0; }, k0, k, a.m - m0);
        else side_q.load(k0, k);
        if constexpr (kForm == ROWS) side_p.load([&](int kk) { return p + (int64_t)kk * a.ldp + n0; }, k0, k, a.n - n0);
        else if constexpr (kForm == WEIGHTS)
            side_p.load([&](int kk) {
                const int s = k_begin + kk;
                return p + (int64_t)(a.token ? a.token[s] : s) * a.ldp + n0;
            }, k0, k, a.n - n0);
        else side_p.load(k0, k);
    };
    const int wave = (int)threadIdx.x / NACHO_WAVE, lane = lane_id();
    const int wm = wave / kWavesN * kTileM, wn = wave % kWavesN * kTileN;
    v4f acc[kFragM][kFragN];
#pragma unroll
    for (int i = 0; i < kFragM; ++i)
#pragma unroll
        for (int j = 0; j < kFragN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    if (k > 0) {
        load(0);
        side_q.store(lds[0]);
        side_p.store(lds[0] + SideQ::kBytes);
        __syncthreads();
        int buffer = 0;
        for (int k0 = 0; k0 < k; k0 += kDepth<T>) {
            const bool more = k0 + kDepth<T> < k;
            if (more) load(k0 + kDepth<T>);
#pragma unroll
            for (int step = 0; step < kStep / 64; ++step) {
                v4u fp[kFragN];
#pragma unroll
                for (int j = 0; j < kFragN; ++j) fp[j] = SideP::fragment(lds[buffer] + SideQ::kBytes, wn + j * 16, step);
#pragma unroll
                for (int i = 0; i < kFragM; ++i) {
                    const v4u fq = SideQ::fragment(lds[buffer], wm + i * 16, step);
#pragma unroll
                    for (int j = 0; j < kFragN; ++j) acc[i][j] = matrix_step<T>(fp[j], fq, acc[i][j]);
                }
            }
            if (more) {
                side_q.store(lds[buffer ^ 1]);
                side_p.store(lds[buffer ^ 1] + SideQ::kBytes);
            }
            __syncthreads();
            buffer ^= 1;
        }
    }
    // a lane has four consecutive columns of result row lane % 16 of every 16 x 16
    T *const out = static_cast<T *>(a.out) + (kForm == WEIGHTS ? (int64_t)expert * a.out_stride : 0);
    typedef T four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < kFragM; ++i) {
        const int m = m0 + wm + i * 16 + lane % 16;
        if (m >= m_end) continue;
#pragma unroll
        for (int j = 0; j < kFragN; ++j) {
            const int n = n0 + wn + j * 16 + lane / 16 * 4;
            v4f v = acc[i][j];
            if (kForm == FORWARD && a.bias) {
                const T *b = static_cast<const T *>(a.bias) + (int64_t)expert * a.bias_stride + n;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += n + e < a.n ? wide(b[e]) : 0.0f;
            }
            auto put = [&](T *to, const v4f &x) {
                if (kWords && n + 4 <= a.n) {
                    four w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = (T)x[e];
                    *reinterpret_cast<four *>(to) = w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n + e < a.n) to[e] = (T)x[e];
                }
            };
            if (kForm == FORWARD) {
                if (a.pre) put(static_cast<T *>(a.pre) + (int64_t)m * a.ldpre + n, v);
                if (a.act != NACHO_ACT_NONE) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = activated(v[e], a.act);
                }
            }
            put(out + (int64_t)m * a.ldo + n, v);
        }
    }
}

// grad_z = grad_y act'(pre), a thread N consecutive elements at a time.
template <typename T, int N>
__global__ void __launch_bounds__(kThreads) experts_slope_kernel(SlopeArgs a)
{
    typedef T part __attribute__((ext_vector_type(N)));
    const int rows = bound_of(a, a.experts), parts = (a.cols + N - 1) / N;
    const T *gy = static_cast<const T *>(a.grad_y), *pre = static_cast<const T *>(a.pre);
    T *gz = static_cast<T *>(a.grad_z);
    for (int row = (int)blockIdx.x; row < rows; row += (int)gridDim.x)
        for (int c = (int)threadIdx.x; c < parts; c += kThreads) {
            const part g = *reinterpret_cast<const part *>(gy + (int64_t)row * a.ldgy + c * N);
            const part z = *reinterpret_cast<const part *>(pre + (int64_t)row * a.ldpre + c * N);
            part v;
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = (T)(wide((T)g[e]) * slope_at<T>(wide((T)z[e]), a.act));
            *reinterpret_cast<part *>(gz + (int64_t)row * a.ldgz + c * N) = v;
        }
}

// Sums of an expert's rows of grad_z (or of grad_y act'(pre)): 16 threads along N columns each, 16 along the rows.
template <typename T, int N>
__global__ void __launch_bounds__(kThreads) experts_bias_kernel(SlopeArgs a, int tiles)
{
    typedef T part __attribute__((ext_vector_type(N)));
    __shared__ float sums[16][16 * N + 1];
    const int expert = (int)blockIdx.x / tiles, tx = (int)threadIdx.x % 16, ty = (int)threadIdx.x / 16;
    const int c0 = ((int)blockIdx.x - expert * tiles) * 16 * N, c = c0 + tx * N;
    const int begin = bound_of(a, expert), end = bound_of(a, expert + 1);
    const T *gz = static_cast<const T *>(a.grad_z ? a.grad_z : a.grad_y), *pre = static_cast<const T *>(a.pre);
    const int64_t ld = a.grad_z ? a.ldgz : a.ldgy;
    const bool slope = !a.grad_z && a.act != NACHO_ACT_NONE;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.0f;
    if (c < a.cols)
        for (int row = begin + ty; row < end; row += 16) {
            const part g = *reinterpret_cast<const part *>(gz + (int64_t)row * ld + c);
            if (slope) {
                const part z = *reinterpret_cast<const part *>(pre + (int64_t)row * a.ldpre + c);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += wide((T)(wide((T)g[e]) * slope_at<T>(wide((T)z[e]), a.act)));
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] += wide((T)g[e]);
            }
        }
#pragma unroll
    for (int e = 0; e < N; ++e) sums[ty][tx * N + e] = sum[e];
    __syncthreads();
    for (int i = (int)threadIdx.x; i < 16 * N; i += kThreads)
        if (c0 + i < a.cols) {
            float total = 0.0f;
#pragma unroll
            for (int y = 0; y < 16; ++y) total += sums[y][i];
            (static_cast<T *>(a.grad_bias) + (int64_t)expert * a.bias_stride)[c0 + i] = (T)total;
        }
}

template <typename F> void by_type(int dtype, F f)
{
    if (dtype == NACHO_F32) f((float)0);
    else if (dtype == NACHO_BF16) f((bf16_t)0.0f);
    else f((f16_t)0.0f);
}

// Whether all rows of these matrices start at multiples of 16 bytes.
bool in_words(std::initializer_list<std::pair<const void *, int64_t>> all, int elem)
{
    uintptr_t bits = 0;
    for (const auto &m : all)
        if (m.first) bits |= (uintptr_t)m.first | (uintptr_t)(m.second * elem);
    return bits % 16 == 0;
}

template <Form kForm> hipError_t launch(int dtype, const ProductArgs &a, hipStream_t s)
{
    constexpr int kM = 128, kN = 128;
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    const int tiles_n = (a.n + kN - 1) / kN;
    // tiles of rows: as many as the slots fill, and a part of one for every expert that may have any
    const int64_t tiles_m = kForm == WEIGHTS ? (int64_t)a.experts * ((a.m + kM - 1) / kM)
                                             : a.slots / kM + (a.slots < a.experts ? a.slots : a.experts);
    if (tiles_m == 0) return hipSuccess;
    // (a launch holds 2^32 threads along its first dimension)
    const int64_t tiles = tiles_m * tiles_n, wide_grid = tiles < (1 << 22) ? tiles : 1 << 22;
    if (tiles > 0x7fffffff - (1 << 22)) return hipErrorNotSupported;
    const bool words = in_words({{a.q, a.ldq}, {a.p, a.ldp}, {a.p, a.p_stride}, {a.out, a.ldo}, {a.out, a.out_stride}, {a.pre, a.ldpre},
                                 {a.q, kForm == WEIGHTS ? 0 : a.k}, {a.q, kForm == WEIGHTS ? a.m : 0}, {a.q, kForm == FORWARD ? 0 : a.n}}, elem);
    const dim3 grid((unsigned)wide_grid, (unsigned)((tiles + wide_grid - 1) / wide_grid));
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        if (words) experts_kernel<T, kForm, kM, kN, 2, 2, true><<<grid, kThreads, 0, s>>>(a, tiles_n);
        else experts_kernel<T, kForm, kM, kN, 2, 2, false><<<grid, kThreads, 0, s>>>(a, tiles_n);
    });
    return hipGetLastError();
}

}  // namespace

hipError_t launch_experts_forward(int dtype, const ProductArgs &a, hipStream_t s) { return launch<FORWARD>(dtype, a, s); }
hipError_t launch_experts_rows(int dtype, const ProductArgs &a, hipStream_t s) { return launch<ROWS>(dtype, a, s); }
hipError_t launch_experts_weights(int dtype, const ProductArgs &a, hipStream_t s) { return launch<WEIGHTS>(dtype, a, s); }

hipError_t launch_experts_slope(int dtype, const SlopeArgs &a, hipStream_t s)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    const bool words = in_words({{a.grad_y, a.ldgy}, {a.pre, a.ldpre}, {a.grad_z, a.ldgz}, {a.grad_y, a.cols}}, elem);
    by_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        auto run = [&](auto each) {
            constexpr int N = decltype(each)::value;
            if (a.grad_z && a.slots > 0)
                experts_slope_kernel<T, N><<<dim3((unsigned)(a.slots < 8192 ? a.slots : 8192)), kThreads, 0, s>>>(a);
            if (a.grad_bias) {
                const int tiles = (a.cols + 16 * N - 1) / (16 * N);
                experts_bias_kernel<T, N><<<dim3((unsigned)(tiles * a.experts)), kThreads, 0, s>>>(a, tiles);
            }
        };
        if (words) run(std::integral_constant<int, Word<T>::n>());
        else run(std::integral_constant<int, 1>());
    });
    return hipGetLastError();
}

}  // namespace nacho
