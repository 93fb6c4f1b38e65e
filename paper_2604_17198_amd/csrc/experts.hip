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
//
// Bound by the matrix units for many slots an expert (16384 bf16 slots of 16 experts, 2048 x 8192: 612 to 657 us a call by the
// card, 837 to 898 TFLOP/s of the 1211 of a library's product of 8192^3), by the weights for few (16 of 32 experts, 2048 x 4096:
// 44 to 55 us a call for 213 MB; 32 us a kernel where the last cache still has most of them).
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

constexpr int kThreads = 256;
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));

enum Form { FORWARD, ROWS, WEIGHTS };
enum Access { WORDS, ANYWHERE, TINY };  // rows of words of 16 bytes; rows that start and end anywhere; such rows shorter than a word

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

// Activations and their slopes.  Rows of floats take the library's functions, and slopes in 64 bits: next to its root a
// slope is a difference of nearly equal numbers.  For rows of 16 bits the normal distribution comes from a polynomial (in the
// form of Abramowitz and Stegun 7.1.26, fitted here): erfc(x) exp(x^2) = t P(t) with t = 1 / (1 + 0.38 x), relative error below
// 4e-7 for all x >= 0 in 32 bits, a hundredth of what the rounding to the type takes; and it shares its exponential with the
// density.  (16384 x 4096 bf16, slopes of gelu: 143 us with erfcf, bound by its instructions.)
struct Normal {
    float below, density;
    __device__ explicit Normal(float z)
    {
        const float t = __builtin_amdgcn_rcpf(1.0f + 2.687005769e-01f * fabsf(z)), e = exp2_of(-0.5f * kLog2e * z * z);
        const float c[9] = {2.144118706e-01f, 2.139049757e-01f, 2.040023426e-01f, 1.382982534e-01f, 2.308058125e-01f,
                            -1.625332754e-01f, 3.647579072e-01f, -2.626970734e-01f, 5.904920688e-02f};
        float p = c[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = p * t + c[i];
        const float tail = 0.5f * t * p * e;
        below = z < 0.0f ? tail : 1.0f - tail;
        density = 0.3989422804014327f * e;
    }
};
template <typename T> __device__ inline float activated(float z, int act)
{
    if (act == NACHO_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == NACHO_ACT_GELU) {
        // (by the complement of the error function: next to one, 1 + erf has no digits left for a negative argument)
        if constexpr (sizeof(T) == 4) return z * 0.5f * erfcf(-0.70710678118654752f * z);
        else return z * Normal(z).below;
    }
    if (act == NACHO_ACT_SILU) {
        if constexpr (sizeof(T) == 4) return z / (1.0f + expf(-z));
        else return z * __builtin_amdgcn_rcpf(1.0f + exp2_of(-kLog2e * z));
    }
    return z;
}
// (A row past its type's range is kept as an infinity: its slope is that of any number so far out, 0 or 1, where the formulas'
// products of zero and infinity would make a NaN.)
template <typename T> __device__ inline float slope_at(float z, int act)
{
    if (act == NACHO_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if constexpr (sizeof(T) == 4) {
        const double v = z;
        if (act == NACHO_ACT_GELU) {
            const double density = 0.39894228040143267794 * exp(-0.5 * v * v);
            return (float)(0.5 * erfc(-0.70710678118654752440 * v) + (density == 0.0 ? 0.0 : v * density));
        }
        if (act == NACHO_ACT_SILU) {
            const double q = 1.0 / (1.0 + exp(-v)), both = q * (1.0 - q);
            return (float)(both == 0.0 ? q : q + v * both);
        }
    } else {
        if (act == NACHO_ACT_GELU) {
            const Normal at(z);
            return at.below + (at.density == 0.0f ? 0.0f : z * at.density);
        }
        if (act == NACHO_ACT_SILU) {
            const float q = __builtin_amdgcn_rcpf(1.0f + exp2_of(-kLog2e * z)), both = q * (1.0f - q);
            return both == 0.0f ? q : q + z * both;
        }
    }
    return 1.0f;
}

// The first slot of expert e (a list that runs past the slots ends there).
template <typename Args> __device__ inline int bound_of(const Args &a, int e)
{
    const int at = a.bounds[e];
    return at < (int)a.slots ? at : (int)a.slots;
}

// Tiles of kM rows that `rows` < 2^31 make (unsigned: the sum passes 31 bits where an expert has nearly all there can be).
template <int kM> __device__ inline int tiles_of(int rows) { return rows > 0 ? (int)(((unsigned)rows + (kM - 1)) / kM) : 0; }

// The expert and the first row of tile `tile` of kM rows, the experts' tiles one after the other; false behind the last.
template <int kM, typename Args> __device__ inline bool find_tile(const Args &a, int tile, int &expert, int &row, int &end)
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
        const int tiles = tiles_of<kM>(last - first), upto = before + wave_inclusive_scan(tiles);
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

// Which tile of rows (the experts' one after the other) and which columns a workgroup computes.  Workgroups are dealt out to
// the chip's eight parts one by one, each of which has a cache; 32 of a part's that run at a time get 4 x 8 neighbouring
// tiles, which need 12 stretches of Q and P between them.  (16384 slots of 16 experts, 2048 x 8192, bf16, us: weights 662, in
// the order of rows 687; of 32 experts, 1024 x 4096, forward 205 and 217.)
template <int kN> __device__ inline void place_tile(int tiles_m, int tiles_n, int &tile, int &n0)
{
    constexpr int kRound = 256, kParts = 8, kTall = 4;
    int number = (int)(blockIdx.y * gridDim.x + blockIdx.x);
    if ((number | (kRound - 1)) < tiles_m * tiles_n)
        number = (number & ~(kRound - 1)) | (number % kParts) * (kRound / kParts) | (number % kRound) / kParts;
    const int band = number / (kTall * tiles_n), in_band = number - band * kTall * tiles_n;
    const int rows = tiles_m - band * kTall < kTall ? tiles_m - band * kTall : kTall;
    tile = tiles_m;                    // (behind the last tile)
    n0 = 0;
    if (rows <= 0) return;
    const int column = in_band / rows;
    tile = band * kTall + in_band - column * rows;
    n0 = column * kN;
}

// A side of the product: kRows rows (of Q or P), kStep bytes of k of each, loaded by kThreads threads.
template <typename T, int kStep> constexpr int kDepth = kStep / (int)sizeof(T);

// 16 bytes from every lane's own address to LDS, one lane's behind the other's from `to` on (the same for the whole
// wavefront); not there before wait_loads has counted it.
__device__ inline void load_to_lds(const void *from, char *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
// Waits until the wavefront's loads and LDS reads are there, then for the workgroup.  (The builtin: the compiler counts
// the loads to LDS too, and waits again for those it does not see waited for.)
__device__ inline void wait_loads()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x70);          // vmcnt 0, lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The address of row `row` of rows `ld` < 2^31 elements apart: one instruction where it is needed (the compiler would
// keep running addresses of every row in registers that the results need).
template <typename T> __device__ inline const T *at_row(const T *base, int row, int64_t ld)
{
    asm volatile("" : "+v"(row));
    return base + (uint64_t)(unsigned)row * (unsigned)ld;
}

// Words of rows that no 16-byte boundary fits: 16 bytes from any element's address, in one instruction (global memory takes
// any alignment).  Of a row's last elements, fewer than a word, and behind them, the word that ends with the row is loaded, and
// moved down when it is stored to LDS, so that nothing waits for it before.  There is no branch on the way: behind one that loads
// may be in, the next wait is for all loads (16384 bf16 slots of 16 experts, 1023 x 1025, both gradients: 441 us with branches,
// 210 without).  Rows shorter than a word (kTiny): elements one by one.
template <typename T, bool kTiny> struct Ragged {
    int there, back;           // elements from the word's first one on; places that the loaded word lies before it
    // `before`: elements of the row before the word; `length`: the row's, at least one.
    __device__ Ragged(int length, int before)
    {
        constexpr int n = Word<T>::n;
        there = length - before < n ? length - before : n;
        back = n - there;
    }
    __device__ v4u load(const T *from) const
    {
        constexpr int n = Word<T>::n;
        v4u word;
        if constexpr (!kTiny) __builtin_memcpy(&word, from - back, 16);
        else {
            typename Word<T>::type v;
#pragma unroll
            for (int e = 0; e < n; ++e) v[e] = from[e < there ? e : there - 1];
            word = __builtin_bit_cast(v4u, v);
        }
        return word;
    }
    // The word with zeros behind the row.
    __device__ v4u placed(v4u w) const
    {
        constexpr int n = Word<T>::n;
        if constexpr (kTiny) {
            typename Word<T>::type v = __builtin_bit_cast(typename Word<T>::type, w);
#pragma unroll
            for (int e = 0; e < n; ++e) v[e] = e < there ? v[e] : (T)0.0f;
            return __builtin_bit_cast(v4u, v);
        }
        const int bytes = back * (int)sizeof(T);
        if (bytes & 8) w = v4u{w[2], w[3], 0, 0};
        if (bytes & 4) w = v4u{w[1], w[2], w[3], 0};
        if (bytes & 2) w = v4u{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
        return there > 0 ? w : v4u{0, 0, 0, 0};
    }
};

// Rows that run along k.  A thread loads words of 16 bytes, the same one of several rows.
template <typename T, int kRows, int kStep, int kThreads, Access kAccess, int kSets> struct AlongK {
    static constexpr int kUnits = kStep / 16, kApart = kThreads / kUnits;
    static constexpr int kLoads = kRows / kApart, kBytes = kRows * kStep;
    static_assert(kLoads * kApart == kRows, "a whole number of rows a thread");
    const T *base;
    int64_t ld;
    int row[kLoads];
    v4u word[kSets][kLoads];
    int first[kSets], end;
    int unit, at;

    // number(r): which row of the matrix is row r of the tile.
    template <typename Row> __device__ void start(const T *matrix, int64_t apart, Row number)
    {
        base = matrix;
        ld = apart;
        unit = (int)threadIdx.x % kUnits;
        at = (int)threadIdx.x / kUnits;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) row[i] = number(at + i * kApart);
    }
    template <typename Set> __device__ void load(Set set, int k0, int k)
    {
        constexpr int n = Word<T>::n;
        const int from = k0 + unit * n;
        first[set.value] = from;
        end = k;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const T *at = base + row[i] * ld + from;
            if constexpr (kAccess == WORDS) word[set.value][i] = from < k ? *reinterpret_cast<const v4u *>(at) : v4u{0, 0, 0, 0};
            else word[set.value][i] = Ragged<T, kAccess == TINY>(k, from).load(at);
        }
    }
    // Asks for the words k0 .. of all rows (whole words).  What a lane loads lies behind what the lane before it loads,
    // so the lanes share out the words of a row in the order in which they lie.
    __device__ void ask(int k0, char *lds) const
    {
        static_assert(kApart % 8 == 0, "the same turn for all rows of a thread");
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / NACHO_WAVE);
        const int first = k0 + (unit ^ turn(at)) * Word<T>::n;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(at_row(base, row[i], ld) + first, lds + (i * kThreads + wave * NACHO_WAVE) * 16);
    }
    // Where word u of row r lies: the same word of 8 consecutive rows, which the LDS serves at a time, in 8 different
    // sixteens of bytes of 128.
    static __device__ int turn(int r) { return kUnits == 8 ? r & 7 : r >> 1 & 3; }
    static __device__ int place(int r, int u) { return r * kStep + ((u ^ turn(r)) << 4); }
    template <typename Set> __device__ void store(Set set, char *lds) const
    {
        const Ragged<T, kAccess == TINY> last(end, first[set.value]);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const v4u w = word[set.value][i];
            *reinterpret_cast<v4u *>(lds + place(at + i * kApart, unit)) = kAccess == WORDS ? w : last.placed(w);
        }
    }
    // Where a lane's fragments of the rows from r0 on (a multiple of 16) start; and its 16 bytes of rows 16 number ..
    // from there in step `step` of 64 bytes.
    static __device__ int lane_base(int r0) { return r0 * kStep + lane_id() % 16 * kStep; }
    static __device__ v4u fragment(const char *lds, int base, int number, int step)
    {
        const int u = (step * 4 + lane_id() / 16) ^ turn(lane_id() % 16);
        return *reinterpret_cast<const v4u *>(lds + base + number * 16 * kStep + (u << 4));
    }
};

// Columns that run along k: for every k a row of kRows elements.
template <typename T, int kRows, int kStep, int kThreads, Access kAccess, int kSets> struct AcrossK {
    static constexpr int kRowBytes = kRows * (int)sizeof(T), kRowWords = kRowBytes / 16;
    static constexpr int kLoads = kDepth<T, kStep> * kRowWords / kThreads, kBytes = kDepth<T, kStep> * kRowBytes;
    static_assert(kRowWords >= 16 && kLoads * kThreads == kDepth<T, kStep> * kRowWords, "rows that the turns fit into");
    v4u word[kSets][kLoads];
    Ragged<T, kAccess == TINY> last = Ragged<T, kAccess == TINY>(1, 0);
    int rows[kSets];  // rows of k from the thread's first one on

    // address(i, k): the row of k (of the thread's i-th word); `length`: its elements, `before`: those before the tile's first.
    template <typename Set, typename Row> __device__ void load(Set set, Row address, int k0, int k, int length, int before)
    {
        constexpr int n = Word<T>::n;
        static_assert(kThreads % kRowWords == 0, "the same word of all rows of a thread");
        const int first = before + (int)threadIdx.x % kRowWords * n;
        if constexpr (kAccess != WORDS) last = Ragged<T, kAccess == TINY>(length, first);
        rows[set.value] = k - k0 - row_of_load(0);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const unsigned kk = (unsigned)k0 + row_of_load(i);
            const T *from = address(i, kk < (unsigned)k ? (int)kk : k - 1);
            if constexpr (kAccess == WORDS) word[set.value][i] = *reinterpret_cast<const v4u *>(from + (first < length ? first : length - n));
            else word[set.value][i] = last.load(from + first);
        }
    }
    // Asks for the rows of k0 ..; address(i, kk): the row of kk, which is k0 or more by i threads' words.  (Words behind
    // the last: the last one again, whose results are not stored.)
    static __device__ int row_of_load(int i) { return (int)threadIdx.x / kRowWords + i * (kThreads / kRowWords); }
    template <typename Row> __device__ void ask(Row address, int k0, int most, char *lds) const
    {
        constexpr int n = Word<T>::n;
        constexpr bool kSame = kThreads / kRowWords % 16 == 0;           // (the same turn for all rows of a thread)
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / NACHO_WAVE);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int first = ((int)threadIdx.x % kRowWords ^ turn(row_of_load(kSame ? 0 : i))) * n;
            load_to_lds(address(i, k0 + row_of_load(i)) + (first < most ? first : most - n), lds + (i * kThreads + wave * NACHO_WAVE) * 16);
        }
    }
    // Where word w of the row of k lies: rows that are read together by one instruction lie in different banks, 32
    // bytes (16-bit types: rows k .. k + 3 of two fours of eight) or 64 bytes (floats: rows 4 apart) of each.
    static __device__ int turn(int k) { return sizeof(T) == 2 ? ((k & 3) | (k >> 1 & 4)) << 1 : (k >> 2 & 3) << 2; }
    static __device__ int place(int k, int w) { return k * kRowBytes + ((w ^ turn(k)) << 4); }
    template <typename Set> __device__ void store(Set set, char *lds) const
    {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int u = (int)threadIdx.x + i * kThreads;
            const v4u w = kAccess == WORDS ? word[set.value][i] : last.placed(word[set.value][i]), zero = {0, 0, 0, 0};
            *reinterpret_cast<v4u *>(lds + place(u / kRowWords, u % kRowWords)) = row_of_load(i) - row_of_load(0) < rows[set.value] ? w : zero;
        }
    }
    static __device__ int lane_base(int r0) { return r0 * (int)sizeof(T); }
    static __device__ v4u fragment(const char *lds, int base, int number, int step)
    {
        const int lane = lane_id(), four = lane / 16, i = lane % 16;
        if constexpr (sizeof(T) == 2) {
            // the LDS hands 16 lanes four rows of 16 elements transposed: lane i gets column i of rows k .. k + 3
            v4s part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = four * 8 + i / 4, byte = base + number * 32 + i % 4 * 8;       // (h and step turn nothing)
                const char *at = lds + (step * 32 + h * 4) * kRowBytes + place(k, byte >> 4) + (byte & 15);
                part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)at);
            }
            typedef short v8s __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(v4u, (v8s)__builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v4u v;
            const int byte = base + number * 64 + i * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = step * 16 + four * 4 + j;
                v[j] = *reinterpret_cast<const unsigned *>(lds + place(k, byte >> 4) + (byte & 15));
            }
            return v;
        }
    }
};

template <typename F, int... i> __device__ inline void unrolled(F f, std::integer_sequence<int, i...>)
{
    (f(std::integral_constant<int, i>()), ...);
}
template <int n, typename F> __device__ inline void unrolled(F f) { unrolled(f, std::make_integer_sequence<int, n>()); }

// One tile of kM x kN results; kWavesM x kWavesN wavefronts share it.
template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess> struct Tile {
    static constexpr int kThreads = kWavesM * kWavesN * NACHO_WAVE;
    static constexpr int kTileM = kM / kWavesM, kTileN = kN / kWavesN, kFragM = kTileM / 16, kFragN = kTileN / 16;
    // steps of k that a thread has in registers on their way to LDS, where rows do not go there by themselves
    static constexpr int kSets = kAccess == ANYWHERE && kM * kN <= 64 * 64 ? 2 : 1;
    static constexpr bool kAcrossQ = kForm == WEIGHTS, kAcrossP = kForm != FORWARD;
    typedef std::conditional_t<kAcrossQ, AcrossK<T, kM, kStep, kThreads, kAccess, kSets>, AlongK<T, kM, kStep, kThreads, kAccess, kSets>> SideQ;
    typedef std::conditional_t<kAcrossP, AcrossK<T, kN, kStep, kThreads, kAccess, kSets>, AlongK<T, kN, kStep, kThreads, kAccess, kSets>> SideP;
    static constexpr int kBytes = SideQ::kBytes + SideP::kBytes;
    // (The stages are arguments that do not overlap: so the compiler knows that reads of one do not wait for loads to the
    // other, also those reads that transpose.)
    static __device__ void compute(const ProductArgs &a, int tiles_m, int tiles_n, char *__restrict stage0, char *__restrict stage1);
};

template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess>
__global__ void __launch_bounds__(kWavesM * kWavesN * NACHO_WAVE) experts_kernel(ProductArgs a, int tiles_m, int tiles_n)
{
    typedef Tile<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess> Work;
    __shared__ __attribute__((aligned(16))) char stage0[Work::kBytes], stage1[Work::kBytes];
    Work::compute(a, tiles_m, tiles_n, stage0, stage1);
}

template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess>
__device__ inline void Tile<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess>::compute(const ProductArgs &a, int tiles_m, int tiles_n,
                                                                                        char *__restrict stage0, char *__restrict stage1)
{
    auto stage = [&](auto i) -> char * {
        if constexpr (decltype(i)::value == 0) return stage0;
        else return stage1;
    };
    int tile, n0;
    place_tile<kN>(tiles_m, tiles_n, tile, n0);
    int expert, m0, m_end, k_begin = 0, k = a.k;
    if (kForm == WEIGHTS) {
        const int tiles = (a.m + kM - 1) / kM;
        expert = tile / tiles;
        if (expert >= a.experts) return;
        m0 = (tile - expert * tiles) * kM;
        m_end = a.m;
        k_begin = bound_of(a, expert);
        k = bound_of(a, expert + 1) - k_begin;
    } else if (!find_tile<kM>(a, tile, expert, m0, m_end) || n0 >= a.n) return;
    // (sums of a row, or a step of k, and what a tile has may pass 31 bits behind the last one: compared in 32)
    const T *const q = static_cast<const T *>(a.q);
    const T *const p = static_cast<const T *>(a.p) + (int64_t)expert * a.p_stride;
    SideQ side_q;
    SideP side_p;
    // rows behind the last: the last one again, whose results are not stored
    if constexpr (!kAcrossQ)
        side_q.start(q, a.ldq, [&](int r) {
            const int row = (unsigned)m0 + r < (unsigned)m_end ? m0 + r : m_end - 1;
            return kForm == FORWARD && a.token ? a.token[row] : row;
        });
    if constexpr (!kAcrossP) side_p.start(p, a.ldp, [&](int r) { return n0 + r < a.n ? n0 + r : a.n - 1; });
    // Rows of x that the words of the next step of k come from: asked for a step ahead, or every step would wait for them
    // before it can ask for the words.
    int slot[kForm == WEIGHTS ? SideP::kLoads : 1], found[kForm == WEIGHTS ? SideP::kLoads : 1];
    auto look_up = [&](int k0) {
        if constexpr (kForm == WEIGHTS) {
#pragma unroll
            for (int l = 0; l < SideP::kLoads; ++l) {
                const unsigned kk = (unsigned)k0 + SideP::row_of_load(l);
                slot[l] = k_begin + (kk < (unsigned)k ? (int)kk : k - 1);
            }
            if constexpr (kAccess != WORDS) {
                // (without a branch, see Ragged)
                const int *list = a.token ? a.token : a.bounds;
#pragma unroll
                for (int l = 0; l < SideP::kLoads; ++l) found[l] = list[a.token ? slot[l] : 0];
            } else if (a.token) {
#pragma unroll
                for (int l = 0; l < SideP::kLoads; ++l) slot[l] = a.token[slot[l]];
            }
        }
    };
    auto load = [&](auto set, int k0) {
        if constexpr (kAcrossQ)
            side_q.load(set, [&](int, int kk) { return q + (int64_t)(k_begin + kk) * a.ldq; }, k0, k, a.m, m0);
        else side_q.load(set, k0, k);
        if constexpr (kForm == ROWS) side_p.load(set, [&](int, int kk) { return p + (int64_t)kk * a.ldp; }, k0, k, a.n, n0);
        else if constexpr (kForm == WEIGHTS) {
            side_p.load(set, [&](int l, int) { return p + (int64_t)(kAccess != WORDS && a.token ? found[l] : slot[l]) * a.ldp; }, k0, k, a.n, n0);
            look_up(kDepth<T, kStep> < k - k0 ? k0 + kDepth<T, kStep> : k0);
        } else side_p.load(set, k0, k);
    };
    const int wave = (int)threadIdx.x / NACHO_WAVE, lane = lane_id();
    const int wm = wave / kWavesN * kTileM, wn = wave % kWavesN * kTileN;
    const bool busy = __builtin_amdgcn_readfirstlane((unsigned)m0 + wm < (unsigned)m_end && n0 + wn < a.n ? 1 : 0) != 0;
    v4f acc[kFragM][kFragN];
#pragma unroll
    for (int i = 0; i < kFragM; ++i)
#pragma unroll
        for (int j = 0; j < kFragN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    int base_q = SideQ::lane_base(wm), base_p = SideP::lane_base(wn);
    // A wavefront multiplies two of its rows of fragments at a time (or its only one); what the next ones need is read before.
    constexpr int kPart = kFragM > 1 ? 2 : 1, kParts = kFragM / kPart, kSteps = kStep / 64;
    static_assert(kFragM % kPart == 0 && kSteps % 2 == 0, "registers of P and of Q in turn");
    v4u fp[2][kFragN], fq[2][kPart];
    auto read_p = [&](const char *lds, auto step) {
        constexpr int s = decltype(step)::value;
#pragma unroll
        for (int j = 0; j < kFragN; ++j) fp[s % 2][j] = SideP::fragment(lds + SideQ::kBytes, base_p, j, s);
    };
    auto read_q = [&](const char *lds, auto step, auto part) {
        constexpr int s = decltype(step)::value, h = decltype(part)::value;
#pragma unroll
        for (int i = 0; i < kPart; ++i) fq[(s * kParts + h) % 2][i] = SideQ::fragment(lds, base_q, h * kPart + i, s);
    };
    // (nothing moves across: what is read before it is on its way while it runs)
    auto multiply = [&](auto step, auto part) {
        constexpr int s = decltype(step)::value, h = decltype(part)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kPart; ++i)
#pragma unroll
            for (int j = 0; j < kFragN; ++j)
                acc[h * kPart + i][j] = matrix_step<T>(fp[s % 2][j], fq[(s * kParts + h) % 2][i], acc[h * kPart + i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    const std::integral_constant<int, 0> zero;
    const std::integral_constant<int, 1> one;
    // A step of k that is there, without one behind it.
    auto multiply_all = [&](const char *lds) {
        unrolled<kSteps>([&](auto step) {
            read_p(lds, step);
            unrolled<kParts>([&](auto part) {
                read_q(lds, step, part);
                multiply(step, part);
            });
        });
    };
    constexpr int kDeep = kDepth<T, kStep>;
    int done = 0;
    if (k > 0) look_up(0);
    if constexpr (kAccess == WORDS) {
        // Whole steps of k.  One is on its way to LDS while the one before it is multiplied; and while the matrix units
        // have one half of a wavefront's tile, the registers of the next half are read.
        const int steps = k / kDeep;
        // (i: of stage t)
        auto ask = [&](int t, auto i) {
            char *lds = stage(i);
            if constexpr (kAcrossQ) side_q.ask([&](int, int kk) { return at_row(q + m0, k_begin + kk, a.ldq); }, t * kDeep, a.m - m0, lds);
            else side_q.ask(t * kDeep, lds);
            if constexpr (kForm == WEIGHTS)
                side_p.ask([&](int l, int) { return at_row(p + n0, slot[l], a.ldp); }, t * kDeep, a.n - n0, lds + SideQ::kBytes);
            else if constexpr (kForm == ROWS)
                side_p.ask([&](int, int kk) { return at_row(p + n0, kk, a.ldp); }, t * kDeep, a.n - n0, lds + SideQ::kBytes);
            else side_p.ask(t * kDeep, lds + SideQ::kBytes);
            look_up((t + 1) * kDeep);
        };
        // (Behind the last step the next one's registers are read all the same, and not used: a wait that is not there on
        // every path would have the compiler wait for all loads before it reads.)
        auto body = [&](int t, auto which) {
            // (or the compiler keeps the address of every fragment in a register of its own)
            asm volatile("" : "+v"(base_q), "+v"(base_p));
            const std::integral_constant<int, 1 - decltype(which)::value> other;
            unrolled<kSteps>([&](auto step) {
                constexpr int s = decltype(step)::value;
                unrolled<kParts>([&](auto part) {
                    constexpr int h = decltype(part)::value;
                    if constexpr (h + 1 < kParts) {
                        read_q(stage(which), step, std::integral_constant<int, h + 1>());
                    } else if constexpr (s + 1 < kSteps) {
                        const std::integral_constant<int, s + 1> behind;
                        read_p(stage(which), behind);
                        read_q(stage(which), behind, zero);
                    } else {
                        wait_loads();
                        if (kForm == WEIGHTS && t + 2 < steps) ask(t + 2, which);
                        read_p(stage(other), zero);
                        read_q(stage(other), zero, zero);
                    }
                    multiply(step, part);
                    // (behind the part: its matrix instructions run while the loads are asked for; 16384 slots, 2048 x 8192, us, before and after:
                    // forward 579 and 566, rows 661 and 616.  The weights' product has no registers left for that.)
                    if constexpr (kForm != WEIGHTS && h + 1 == kParts && s + 1 == kSteps)
                        if (t + 2 < steps) ask(t + 2, which);
                });
            });
        };
        // Wavefronts whose rows or columns all lie behind the last only load: the others of their SIMD then have the matrix unit
        // for themselves.
        if (steps > 0) {
            ask(0, zero);
            wait_loads();
            if (steps > 1) ask(1, one);
            int t = 0;
            if (busy) {
                read_p(stage0, zero);
                read_q(stage0, zero, zero);
                for (; t + 2 <= steps; t += 2) {
                    body(t, zero);
                    body(t + 1, one);
                }
                if (t < steps) body(t, zero);
            } else {
                auto pass = [&](int at, auto which) {
                    wait_loads();
                    if (at + 2 < steps) ask(at + 2, which);
                };
                for (; t + 2 <= steps; t += 2) {
                    pass(t, zero);
                    pass(t + 1, one);
                }
                if (t < steps) pass(t, zero);
            }
        }
        done = steps * kDeep;
        __syncthreads();
    }
    auto store = [&](auto set, char *lds) {
        side_q.store(set, lds);
        side_p.store(set, lds + SideQ::kBytes);
    };
    if constexpr (kAccess == WORDS) {
        // what is left of a step
        if (done < k) {
            load(zero, done);
            store(zero, stage0);
            __syncthreads();
            // (a loop of one turn: with the product in line the tiles of 256 x 256 need two registers more than there are)
            for (int left = k - done; left > 0; left -= kDeep)
                if (busy) multiply_all(stage0);
        }
    } else if (k > 0) {
        // The next steps (two of them if there are registers) are on their way while one is multiplied.  (Behind the last step
        // it is loaded again: a load that is not there on every path would have the compiler wait for all of them.)
        const int steps = (k - 1) / kDeep + 1;
        auto at = [&](int t) { return (t < steps ? t : steps - 1) * kDeep; };
        load(zero, 0);
        if constexpr (kSets == 2) load(one, at(1));
        store(zero, stage0);
        __syncthreads();
        auto body = [&](int t, auto which) {
            const std::integral_constant<int, (int)decltype(which)::value % kSets> set;
            const std::integral_constant<int, 1 - (int)decltype(which)::value> other;
            load(set, at(t + kSets));
            if (busy) multiply_all(stage(which));
            store(std::integral_constant<int, (int)decltype(other)::value % kSets>(), stage(other));
            __syncthreads();
        };
        int t = 0;
        for (; t + 2 <= steps; t += 2) {
            body(t, zero);
            body(t + 1, one);
        }
        if (t < steps) body(t, zero);
    }
    // A lane has four consecutive columns of result row lane % 16 of every 16 x 16.  A wavefront takes its tile through its
    // part of LDS, so that lanes that store side by side have neighbouring parts of a row, eight columns each.
    __syncthreads();
    constexpr int kRowBytes = kTileN * 4, kLanes = kTileN / 8, kPerWave = 2 * kBytes / (kThreads / NACHO_WAVE) / 1024 * 1024;
    constexpr int kPhase = kPerWave / (16 * kRowBytes) < kFragM ? kPerWave / (16 * kRowBytes) : kFragM;
    static_assert(kFragM % kPhase == 0 && kBytes % kPerWave == 0, "a wavefront's part lies in one stage");
    char *const mine = (wave < kBytes / kPerWave ? stage0 : stage1) + wave % (kBytes / kPerWave) * kPerWave;
    T *const out = static_cast<T *>(a.out) + (kForm == WEIGHTS ? (int64_t)expert * a.out_stride : 0);
    const int n = n0 + wn + lane % kLanes * 8, width = a.n - n;
    float bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
    if (kForm == FORWARD && a.bias) {
        const T *b = static_cast<const T *>(a.bias) + (int64_t)expert * a.bias_stride + n;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < width) bias[e] = wide(b[e]);
    }
    auto put = [&](T *to, const float (&v)[8]) {
        constexpr int kWord = Word<T>::n;
#pragma unroll
        for (int h = 0; h < 8; h += kWord) {
            if (h + kWord <= width) {
                typename Word<T>::type w;
#pragma unroll
                for (int e = 0; e < kWord; ++e) w[e] = (T)v[h + e];
                if constexpr (kAccess == WORDS) *reinterpret_cast<typename Word<T>::type *>(to + h) = w;
                else __builtin_memcpy(to + h, &w, 16);
            } else {
#pragma unroll
                for (int e = 0; e < kWord; ++e)
                    if (h + e < width) to[h + e] = (T)v[h + e];
            }
        }
    };
    unrolled<kFragM / kPhase>([&](auto phase) {
        constexpr int i0 = decltype(phase)::value * kPhase;
#pragma unroll
        for (int i = 0; i < kPhase; ++i)
#pragma unroll
            for (int j = 0; j < kFragN; ++j) {
                const int r = lane % 16, unit = (j * 4 + lane / 16) ^ (r & 7);
                *reinterpret_cast<v4f *>(mine + (i * 16 + r) * kRowBytes + unit * 16) = acc[i0 + i][j];
            }
        wave_sync();
#pragma unroll 1
        for (int r = lane / kLanes; r < kPhase * 16; r += NACHO_WAVE / kLanes) {
            const unsigned m = (unsigned)m0 + wm + i0 * 16 + r;
            if (m >= (unsigned)m_end || width <= 0) break;
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4f part = *reinterpret_cast<const v4f *>(mine + r * kRowBytes + (((lane % kLanes * 2 + h) ^ (r & 7)) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[h * 4 + e] = part[e] + bias[h * 4 + e];
            }
            if (kForm == FORWARD) {
                if (a.pre) put(static_cast<T *>(a.pre) + (int64_t)m * a.ldpre + n, v);
                if (a.act != NACHO_ACT_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = activated<T>(v[e], a.act);
                }
            }
            put(out + (int64_t)m * a.ldo + n, v);
        }
        wave_sync();
    });
}

// grad_z = grad_y act'(pre), rounded to the type that the matrix units take (pre is kept in it as well, which halves what is
// written and read of it), and the sums of its rows before that rounding, over tiles of kSlopeRows rows of an expert: a workgroup
// has a tile and 16 words of 16 bytes of its columns, 16 threads along them and 16 along the rows.  Bound by memory: 16384 x 4096
// bf16, gelu, 88 us, 4.6 TB/s.
constexpr int kSlopeRows = 64;
template <typename T, Access kAccess>
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
    v4u g[kRows], z[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const unsigned m = (unsigned)row + ty + i * 16;
        g[i] = z[i] = v4u{0, 0, 0, 0};
        if (m < (unsigned)end) {
            g[i] = get(gy + (int64_t)m * a.ldgy);
            if (a.act != NACHO_ACT_NONE) z[i] = get(pre + (int64_t)m * a.ldpre);
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const unsigned m = (unsigned)row + ty + i * 16;
        word v = __builtin_bit_cast(word, g[i]);
        // (what the sums take is not rounded to the type yet; behind the last row it is zero)
        if (a.act != NACHO_ACT_NONE) {
            const word at = __builtin_bit_cast(word, z[i]);
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float x = wide((T)v[e]) * slope_at<T>(wide((T)at[e]), a.act);
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

template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, Access kAccess, int kStep = 128>
hipError_t run(const ProductArgs &a, hipStream_t s)
{
    const int tiles_n = (a.n + kN - 1) / kN;
    // tiles of rows: as many as the slots fill, and a part of one for every expert that may have any
    const int64_t tiles_m = kForm == WEIGHTS ? (int64_t)a.experts * ((a.m + kM - 1) / kM)
                                             : a.slots / kM + (a.slots < a.experts ? a.slots : a.experts);
    if (tiles_m == 0) return hipSuccess;
    // (a launch holds 2^32 threads along its first dimension)
    const int64_t tiles = tiles_m * tiles_n, row = tiles < (1 << 22) ? tiles : 1 << 22;
    if (tiles > 0x7fffffff - (1 << 22)) return hipErrorNotSupported;
    experts_kernel<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess>
        <<<dim3((unsigned)row, (unsigned)((tiles + row - 1) / row)), kWavesM * kWavesN * NACHO_WAVE, 0, s>>>(a, (int)tiles_m, tiles_n);
    return hipGetLastError();
}

constexpr int64_t kUnits = 256;        // compute units

// Tiles of 256 x 256 need half the LDS reads of tiles of 128 x 128 for the same results, but leave more of a tile empty
// and fill the chip only if there are many of them.  16384 slots bf16, us with 256 and with 128, in equal groups and in groups
// whose sizes are as 0.6 of a normal logarithm (in brackets): 64 experts (256 slots each), 1024 x 4096, forward 185 and 215 (227
// and 256), rows 151 and 192 (233 and 233), 2048 x 8192 670 and 779 (813 and 896), 543 and 689 (715 and 867); 128 experts (128
// each), 1024 x 4096, 305 and 269 (340 and 312), 236 and 228 (343 and 266).  The weights' product, whatever the slots: 16 to 128
// experts 165 and 200 to 393 and 502 (179 and 202, 476 and 540); with fewer tiles than compute units (2 experts, 8192 slots) 117
// and 82.
// Tiles of 32 x 128 for few slots an expert, where the weights are what is read, and where larger ones would leave compute
// units without one.  1024 x 4096 bf16, us with 32 and with 128: 32 experts of 32 slots forward 46 and 49 (59 and 50), of 48 58
// and 51 (71 and 68); rows, for the number of larger tiles, 8 experts of 192 slots (96 tiles) 38 and 52 (39 and 52), 32 of 64 (128)
// 59 and 64 (92 and 69), 32 of 96 (192) 87 and 72 (96 and 75).  Rows that start anywhere gain more: 1023 x 4097, 32 experts of 48
// forward 0.91 of the time (0.92), of 64 0.94 (1.07), of 96 1.17 (1.24).  Their steps are of 256 bytes: 8 tokens, 2 of 32 experts,
// 49 us a call, with 128 bytes 53.
// Floats need four times as many matrix instructions for what is loaded: tiles of 64 x 64, which are as many again.  3000 slots
// of 7 experts, 777 x 499, us: weights 73 (64 x 128: 95), forward 42 (32 x 128: 45), rows 44 (50); with two steps on their way
// in registers 54, 43 and 42.  512 x 2048, 32 experts of 64 and 128 slots, us with 32, 64 and 128: rows 51, 52 and 141, 87, 81 and 149.
template <typename T, Form kForm> hipError_t by_size(const ProductArgs &a, Access access, hipStream_t s)
{
    const int64_t each = a.slots / a.experts, n128 = (a.n + 127) / 128;
    const bool words = access == WORDS;
    if (access == TINY) return run<T, kForm, kForm == WEIGHTS ? 128 : 32, 128, kForm == WEIGHTS ? 2 : 1, kForm == WEIGHTS ? 2 : 4, TINY>(a, s);
    if constexpr (kForm == WEIGHTS) {
        const int64_t tiles = (int64_t)a.experts * ((a.m + 255) / 256) * ((a.n + 255) / 256);
        if constexpr (sizeof(T) == 2) {
            if (words && a.m >= 256 && a.n >= 256 && tiles >= kUnits) return run<T, kForm, 256, 256, 2, 4, WORDS>(a, s);
        } else if (tiles < kUnits) {
            return words ? run<T, kForm, 64, 64, 2, 2, WORDS>(a, s) : run<T, kForm, 64, 64, 2, 2, ANYWHERE>(a, s);
        }
        return words ? run<T, kForm, 128, 128, 2, 2, WORDS>(a, s) : run<T, kForm, 128, 128, 2, 2, ANYWHERE>(a, s);
    } else {
        if constexpr (sizeof(T) == 2) {
            if (words && each >= 256 && a.n >= 256 && a.slots / 256 * ((a.n + 255) / 256) >= kUnits)
                return run<T, kForm, 256, 256, 2, 4, WORDS>(a, s);
        }
        const int64_t few = words && sizeof(T) == 2 ? 32 : 64, most = sizeof(T) == 2 ? kUnits / 2 : 2 * kUnits - 1;
        const bool small = each <= few || a.slots / 128 * n128 <= most;
        if constexpr (sizeof(T) == 4) {
            if (small && each > 64) return words ? run<T, kForm, 64, 64, 2, 2, WORDS>(a, s) : run<T, kForm, 64, 64, 2, 2, ANYWHERE>(a, s);
        }
        if (small)
            return words ? run<T, kForm, 32, 128, 1, 4, WORDS, 256>(a, s) : run<T, kForm, 32, 128, 1, 4, ANYWHERE>(a, s);
        return words ? run<T, kForm, 128, 128, 2, 2, WORDS>(a, s) : run<T, kForm, 128, 128, 2, 2, ANYWHERE>(a, s);
    }
}

template <Form kForm> hipError_t launch(int dtype, const ProductArgs &a, hipStream_t s)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    // (words of 16 bytes; addresses of rows are one product of 32 bits)
    const bool words = a.ldq < 0x7fffffff && a.ldp < 0x7fffffff &&
                       in_words({{a.q, a.ldq}, {a.p, a.ldp}, {a.p, a.p_stride}, {a.out, a.ldo}, {a.out, a.out_stride}, {a.pre, a.ldpre},
                                 {a.q, kForm == WEIGHTS ? 0 : a.k}, {a.q, kForm == WEIGHTS ? a.m : 0}, {a.q, a.n}}, elem);
    // the shorter rows that are read
    const int64_t along = kForm == WEIGHTS ? a.m : a.k, other = kForm == FORWARD ? a.k : a.n, least = along < other ? along : other;
    const Access access = words ? WORDS : least * elem < 16 ? TINY : ANYWHERE;
    hipError_t rc = hipSuccess;
    by_type(dtype, [&](auto zero) { rc = by_size<decltype(zero), kForm>(a, access, s); });
    return rc;
}

}  // namespace

hipError_t launch_experts_forward(int dtype, const ProductArgs &a, hipStream_t s) { return launch<FORWARD>(dtype, a, s); }
hipError_t launch_experts_rows(int dtype, const ProductArgs &a, hipStream_t s) { return launch<ROWS>(dtype, a, s); }
hipError_t launch_experts_weights(int dtype, const ProductArgs &a, hipStream_t s) { return launch<WEIGHTS>(dtype, a, s); }

// Tiles of rows of the sums: as many as the slots fill, and a part of one for every expert that may have any.
int64_t experts_slope_tiles(int64_t slots, int64_t experts) { return slots / kSlopeRows + (slots < experts ? slots : experts); }

hipError_t launch_experts_slope(int dtype, const SlopeArgs &a, hipStream_t s)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    const bool words = in_words({{a.grad_y, a.ldgy}, {a.act ? a.pre : nullptr, a.ldpre}, {a.grad_z, a.ldgz}, {a.grad_y, a.cols}}, elem);
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
            if (words) experts_slope_kernel<T, WORDS><<<grid, kThreads, 0, s>>>(a, (int)tiles_n);
            else if (a.cols >= Word<T>::n) experts_slope_kernel<T, ANYWHERE><<<grid, kThreads, 0, s>>>(a, (int)tiles_n);
            else experts_slope_kernel<T, TINY><<<grid, kThreads, 0, s>>>(a, (int)tiles_n);
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
