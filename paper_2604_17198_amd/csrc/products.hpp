// Products of ragged groups of rows on the matrix units: tiles of out[m][n] = sum_k Q(m, k) P(n, k), of which every file that
// needs them makes its own kernels.
//
//   forward   m: rows of Q, n: rows of P, both run along k        rows    P's columns run along k        weights  both sides' do
//
// A workgroup computes a tile of kM x kN results on the matrix units, from tiles of Q and P that pass through LDS.  A side whose
// rows run along k lies there as rows of k, and a lane reads 16 bytes of its row; a side whose columns run along k lies there as
// rows of n (or m) for every k, and is transposed by the LDS on the way to the registers (16-bit types), or read an element at a
// time (floats).  P is the first operand of the matrix instruction, so that a lane ends with four consecutive columns of a result
// row.  What becomes of the results is the kernel's last argument (a Finish).
//
// Which group (expert) a tile belongs to is found by its workgroup from the groups' bounds alone (a prefix sum of their tiles
// over the lanes), so nothing about them is read on the host.
#pragma once
#include "kernels.hpp"
#include "model.hpp"

namespace nacho {

namespace {

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
template <int kN> __device__ inline void place_tile(int number, int tiles_m, int tiles_n, int &tile, int &n0)
{
    constexpr int kRound = 256, kParts = 8, kTall = 4;
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

// Rows of k elements that go from memory right into the registers that the matrix units read, in stretches of kBatch x 64 bytes: a lane
// has 16 of every 64.  Loads have no branch around them (behind one the compiler waits for all loads): past the row's end its last word is
// loaded, and made zeros when it is used, if the stretch is not whole.
// Rows of 16 bits that start anywhere: 16 bytes from a multiple of 4, which take half the time of 16 bytes from between two, and the
// word's last element; a word that starts between is put together from both.  (The first row of all starts at a multiple of 4.  53 tokens,
// 3 of 11 experts, 2131 x 2384 x 1121 f16, us a call so and with words from between two: 127 and 151.)
template <typename T, Access kAccess, int kSteps> struct Stretch {
    static constexpr int kBatch = kAccess == TINY ? 1 : kSteps, n = Word<T>::n, kStep = 64 / (int)sizeof(T), kLong = kBatch * kStep;
    static constexpr bool kHalves = kAccess == ANYWHERE && sizeof(T) == 2;
    struct Joined {
        v4u word;
        unsigned last;
    };
    typedef std::conditional_t<kHalves, Joined, v4u> Loaded;
    // f(whole): the two kinds of stretches apart.
    template <typename F> static __device__ void by_end(int stretch, int k, F f)
    {
        if ((stretch + 1) * kLong <= k) f(std::true_type());
        else f(std::false_type());
    }
    static __device__ int from(int stretch, int i) { return stretch * kLong + i * kStep + lane_id() / 16 * n; }
    static __device__ Loaded load(const T *row, int at, int k)
    {
        if constexpr (kAccess == WORDS) return *reinterpret_cast<const v4u *>(row + (at < k ? at : k - n));
        else {
            const Ragged<T, kAccess == TINY> r(k, at);
            if constexpr (kHalves) {
                typedef unsigned words __attribute__((ext_vector_type(4), aligned(4)));
                const T *const first = row + at - r.back;
                return {*reinterpret_cast<const words *>((uintptr_t)first & ~(uintptr_t)3), *reinterpret_cast<const unsigned short *>(first + n - 1)};
            } else return r.load(row + at);
        }
    }
    // What was loaded, with zeros behind the row's end (whole: it does not end in the stretch).
    template <typename Whole> static __device__ v4u value(const Loaded &v, const T *row, int at, int k, Whole)
    {
        constexpr bool whole = Whole::value;
        if constexpr (kAccess == WORDS) return whole || at < k ? v : v4u{0, 0, 0, 0};
        else {
            v4u w;
            if constexpr (kHalves) {
                const T *first = row;                                              // (words of a whole stretch all start as the row does)
                if (!whole) first += at - Ragged<T, false>(k, at).back;
                const unsigned by = (unsigned)((uintptr_t)first & 2) * 8;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_alignbit(e < 3 ? v.word[e + 1] : v.last, v.word[e], by);
            } else w = v;
            return whole ? w : Ragged<T, kAccess == TINY>(k, at).placed(w);
        }
    }
};
// How matrices whose first rows are these are read so.  (16-bit arrays that start at an odd element, which Joined's words cannot be cut from: all of
// them element by element.  16 tokens, 2 of 32 experts, 2048 x 4096 x 2048 bf16, us a step with x at a multiple of 16 bytes, of 4 and of 2: 126, 207
// and 609.)
template <typename... Rows> Access stretch_access(bool words, bool tiny, int elem, Rows... rows)
{
    const uintptr_t bits = ((uintptr_t)rows | ...);
    return words ? WORDS : tiny || (elem == 2 && (bits & 2) != 0) ? TINY : ANYWHERE;
}

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

// What a Finish knows of a tile: its group, its first row and the one behind the group's last, its first column; the first of the
// wavefront's rows and columns in it; the stretch of k that it sums.
struct Place {
    int expert, m0, m_end, n0, wm, wn, stretch;
};

// One tile of kM x kN results; kWavesM x kWavesN wavefronts share it.
template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess> struct Tile {
    typedef T type;
    static constexpr Form form = kForm;
    static constexpr Access access = kAccess;
    static constexpr int kTall = kM, kWide = kN, kRows = kWavesM, kColumns = kWavesN;
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
    template <typename Finish>
    static __device__ void compute(const ProductArgs &a, const Finish &finish, int tiles_m, int tiles_n, char *__restrict stage0,
                                   char *__restrict stage1);
    // For a Finish: row(m, n, width, v) for every row m of the tile and eight columns from n on that a lane has of it (width: the
    // columns from n to the last; where there is none the lane is called only if kAll, so that the four lanes of 32 columns can ask
    // each other).
    template <bool kAll = false, typename Row>
    static __device__ void each_row(const ProductArgs &a, const Place &at, const v4f (&acc)[kFragM][kFragN], char *stage0, char *stage1, Row row);
    // Eight results of a row.
    static __device__ void put(T *to, const float (&v)[8], int width)
    {
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
    }
};

template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess, typename Finish>
__global__ void __launch_bounds__(kWavesM * kWavesN * NACHO_WAVE) product_kernel(ProductArgs a, Finish finish, int tiles_m, int tiles_n)
{
    typedef Tile<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess> Work;
    __shared__ __attribute__((aligned(16))) char stage0[Work::kBytes], stage1[Work::kBytes];
    Work::compute(a, finish, tiles_m, tiles_n, stage0, stage1);
}

template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess>
template <typename Finish>
__device__ inline void Tile<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess>::compute(const ProductArgs &a, const Finish &finish, int tiles_m,
                                                                                        int tiles_n, char *__restrict stage0,
                                                                                        char *__restrict stage1)
{
    auto stage = [&](auto i) -> char * {
        if constexpr (decltype(i)::value == 0) return stage0;
        else return stage1;
    };
    int tile, n0;
    // (of one group only the rows that are there are dealt out: tiles without any, among the others, cost 400 us instead of 275 where 1213 of
    // 2021 rows are, 100003 x 1024 f16)
    if (kForm != WEIGHTS && a.experts == 1) tiles_m = tiles_of<kM>(bound_of(a, 1) - bound_of(a, 0));
    int number = (int)(blockIdx.y * gridDim.x + blockIdx.x), stretch = 0;
    if constexpr (Finish::kParts) {
        // (the launch's third dimension has stretches of k; fewer rows leave room for more of them)
        const int tiles = tiles_m * tiles_n;
        if (tiles == 0) return;
        number += (int)(blockIdx.z * gridDim.y * gridDim.x);
        stretch = number / tiles;
        number -= stretch * tiles;
    }
    place_tile<kN>(number, tiles_m, tiles_n, tile, n0);
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
    const T *q = static_cast<const T *>(a.q);
    const T *p = static_cast<const T *>(a.p) + (int64_t)expert * a.p_stride;
    if constexpr (Finish::kParts) {
        static_assert(kForm == ROWS, "k along the rows of Q");
        const int part = finish.k_part(m_end);
        const int64_t first = (int64_t)stretch * part;
        if (first >= k) return;
        q += first;
        p += first * a.ldp;
        k = k - (int)first < part ? k - (int)first : part;
    }
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
    const int wave = (int)threadIdx.x / NACHO_WAVE;
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
    finish.template end<Tile>(a, Place{expert, m0, m_end, n0, wm, wn, stretch}, acc, stage0, stage1);
}

// A lane has four consecutive columns of result row lane % 16 of every 16 x 16.  A wavefront takes its tile through its
// part of LDS, so that lanes that store side by side have neighbouring parts of a row, eight columns each.
template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, int kStep, Access kAccess>
template <bool kAll, typename Row>
__device__ inline void Tile<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess>::each_row(const ProductArgs &a, const Place &at,
                                                                                         const v4f (&acc)[kFragM][kFragN], char *stage0,
                                                                                         char *stage1, Row row)
{
    const int wave = (int)threadIdx.x / NACHO_WAVE, lane = lane_id();
    __syncthreads();
    constexpr int kRowBytes = kTileN * 4, kLanes = kTileN / 8, kPerWave = 2 * kBytes / (kThreads / NACHO_WAVE) / 1024 * 1024;
    constexpr int kPhase = kPerWave / (16 * kRowBytes) < kFragM ? kPerWave / (16 * kRowBytes) : kFragM;
    static_assert(kFragM % kPhase == 0 && kBytes % kPerWave == 0, "a wavefront's part lies in one stage");
    char *const mine = (wave < kBytes / kPerWave ? stage0 : stage1) + wave % (kBytes / kPerWave) * kPerWave;
    const int n = at.n0 + at.wn + lane % kLanes * 8, width = a.n - n;
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
            const unsigned m = (unsigned)at.m0 + at.wm + i0 * 16 + r;
            if (m >= (unsigned)at.m_end || (!kAll && width <= 0)) break;
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4f part = *reinterpret_cast<const v4f *>(mine + r * kRowBytes + (((lane % kLanes * 2 + h) ^ (r & 7)) << 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) v[h * 4 + e] = part[e];
            }
            row(m, n, width, v);
        }
        wave_sync();
    });
}

// A group's bias at the lane's eight columns (the forward form).
template <typename T, int kLanes> __device__ inline void bias_of(const ProductArgs &a, const Place &at, float (&bias)[8])
{
    const int n = at.n0 + at.wn + lane_id() % kLanes * 8, width = a.n - n;
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.0f;
    if (a.bias) {
        const T *b = static_cast<const T *>(a.bias) + (int64_t)at.expert * a.bias_stride + n;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < width) bias[e] = wide(b[e]);
    }
}

template <typename F> void by_type(int dtype, F f)
{
    if (dtype == NACHO_F32) f((float)0);
    else if (dtype == NACHO_BF16) f((bf16_t)0.0f);
    else f((f16_t)0.0f);
}

// Whether all rows of these matrices start at multiples of 16 bytes.
inline bool in_words(std::initializer_list<std::pair<const void *, int64_t>> all, int elem)
{
    uintptr_t bits = 0;
    for (const auto &m : all)
        if (m.first) bits |= (uintptr_t)m.first | (uintptr_t)(m.second * elem);
    return bits % 16 == 0;
}

template <typename T, Form kForm, int kM, int kN, int kWavesM, int kWavesN, Access kAccess, int kStep = 128, typename Finish>
hipError_t run(const ProductArgs &a, const Finish &finish, hipStream_t s)
{
    const int tiles_n = (a.n + kN - 1) / kN;
    // tiles of rows: as many as the slots fill, and a part of one for every expert that may have any
    const int64_t tiles_m = kForm == WEIGHTS ? (int64_t)a.experts * ((a.m + kM - 1) / kM)
                             : a.experts == 1 ? (a.slots + kM - 1) / kM
                                             : a.slots / kM + (a.slots < a.experts ? a.slots : a.experts);
    if (tiles_m == 0) return hipSuccess;
    // (a launch holds 2^32 threads along its first dimension)
    const int64_t tiles = tiles_m * tiles_n, row = tiles < (1 << 22) ? tiles : 1 << 22;
    if (tiles > 0x7fffffff - (1 << 22)) return hipErrorNotSupported;
    product_kernel<T, kForm, kM, kN, kWavesM, kWavesN, kStep, kAccess, Finish>
        <<<dim3((unsigned)row, (unsigned)((tiles + row - 1) / row), finish.parts()), kWavesM * kWavesN * NACHO_WAVE, 0, s>>>(
            a, finish, (int)tiles_m, tiles_n);
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
// Where forward products of floats leave compute units without one of the larger tiles, tiles are of 32 x 32: a stage then takes a
// wavefront half the time, and more of them are at work.  (us a call with 32 x 32 and without: loss of 21 rows, 1567 x 2275 56 and 76, of
// 100 rows, 2000 x 4095 87 and 119, of 300 rows, 1300 x 4000 95 and 103, of 600 rows, 3000 x 1024 73 and 56; experts in training, 64 tokens,
// 2 of 4, 2000 x 1000 92 and 113.  With stages of 128 bytes 58, 91, 97 and 62.)
enum Shape { TILES_256, TILES_128, TILES_64, TILES_32, TILES_32_32 };
// Rows and columns of these tiles (of rows shorter than a word: 128 x 128 for the weights, 32 x 128).
constexpr int tall_of(Shape s) { return s == TILES_256 ? 256 : s == TILES_128 ? 128 : s == TILES_64 ? 64 : 32; }
constexpr int wide_of(Shape s) { return s == TILES_256 ? 256 : s == TILES_64 ? 64 : s == TILES_32_32 ? 32 : 128; }
// Whether floats go by tiles of 32 x 32: every expert that can have slots has tiles of its own, and a tile with no more than 16 rows, whose
// other rows are the last one again, counts half.  (Experts that all have a slot or more, us a launch with 32 x 32 and without, 4096 x 2048: 4 of 4
// slots 38 and 50, of 24 44 and 50, of 64 63 and 50; 2 of 64 43 and 49; 7 of 8 52 and 55, 8 of 8 (on the line) 65 and 60, 9 of 8 96 and 88, 12 of
// 8 98 and 96; 4096 x 4096: 7 of 8 98 and 109, 8 of 8 123 and 124, 10 of 8 202 and 181, 16 of 8 230 and 206; 1024 x 1024, 48 of 4 56 and 52; 1000 x
// 1001, 64 of 8 65 and 57.  Well past the line neither side is ahead: 64 of 4, 2048 x 500 64 and 61, x 1001 121 and 113, x 1024 124 and 142, x 2048
// 231 and 257, x 4096 438 and 404.)
inline bool tiny_tiles(int64_t slots, int64_t experts, int64_t n)
{
    const int64_t active = slots < experts ? slots : experts;
    return active == 0 || active * (((slots + active - 1) / active + 15) / 16) * ((n + 31) / 32) <= 4 * kUnits;
}
// `parts`: stretches of k that workgroups share a tile's sum by.
template <typename T, Form kForm> Shape shape_of(const ProductArgs &a, Access access, int64_t parts = 1)
{
    const int64_t each = a.slots / a.experts, n128 = (a.n + 127) / 128;
    const bool words = access == WORDS;
    if (access == TINY) return kForm == WEIGHTS ? TILES_128 : TILES_32;
    if constexpr (kForm == WEIGHTS) {
        const int64_t tiles = (int64_t)a.experts * ((a.m + 255) / 256) * ((a.n + 255) / 256);
        if (sizeof(T) == 2) return words && a.m >= 256 && a.n >= 256 && tiles >= kUnits ? TILES_256 : TILES_128;
        return tiles < kUnits ? TILES_64 : TILES_128;
    } else {
        if (sizeof(T) == 2 && words && each >= 256 && a.n >= 256 && a.slots / 256 * ((a.n + 255) / 256) * parts >= kUnits) return TILES_256;
        const int64_t few = words && sizeof(T) == 2 ? 32 : 64, most = sizeof(T) == 2 ? kUnits / 2 : 2 * kUnits - 1;
        const bool small = each <= few || a.slots / 128 * n128 * parts <= most;
        if (kForm == FORWARD && sizeof(T) == 4 && tiny_tiles(a.slots, a.experts, a.n)) return TILES_32_32;
        return !small ? TILES_128 : sizeof(T) == 4 && each > 64 ? TILES_64 : TILES_32;
    }
}

template <typename T, Form kForm, typename Finish> hipError_t by_size(const ProductArgs &a, const Finish &f, Access access, hipStream_t s)
{
    const Shape shape = shape_of<T, kForm>(a, access, f.parts());
    const bool words = access == WORDS;
    if (access == TINY) return run<T, kForm, kForm == WEIGHTS ? 128 : 32, 128, kForm == WEIGHTS ? 2 : 1, kForm == WEIGHTS ? 2 : 4, TINY>(a, f, s);
    if constexpr (sizeof(T) == 2) {
        if (shape == TILES_256) return run<T, kForm, 256, 256, 2, 4, WORDS>(a, f, s);
    } else if (shape == TILES_64) return words ? run<T, kForm, 64, 64, 2, 2, WORDS>(a, f, s) : run<T, kForm, 64, 64, 2, 2, ANYWHERE>(a, f, s);
    if constexpr (kForm != WEIGHTS) {
        if constexpr (sizeof(T) == 4 && kForm == FORWARD)
            if (shape == TILES_32_32)
                return words ? run<T, kForm, 32, 32, 2, 1, WORDS, 256>(a, f, s) : run<T, kForm, 32, 32, 2, 1, ANYWHERE, 256>(a, f, s);
        if (shape == TILES_32)
            return words ? run<T, kForm, 32, 128, 1, 4, WORDS, 256>(a, f, s) : run<T, kForm, 32, 128, 1, 4, ANYWHERE>(a, f, s);
    }
    return words ? run<T, kForm, 128, 128, 2, 2, WORDS>(a, f, s) : run<T, kForm, 128, 128, 2, 2, ANYWHERE>(a, f, s);
}

// How rows that no 16-byte boundary fits are read, by the shorter ones.
template <Form kForm> Access access_of(const ProductArgs &a, int elem)
{
    const int64_t along = kForm == WEIGHTS ? a.m : a.k, other = kForm == FORWARD ? a.k : a.n, least = along < other ? along : other;
    return least * elem < 16 ? TINY : ANYWHERE;
}

template <Form kForm, typename Finish> hipError_t launch(int dtype, const ProductArgs &a, const Finish &f, hipStream_t s)
{
    const int elem = dtype == NACHO_F32 ? 4 : 2;
    // (words of 16 bytes; addresses of rows are one product of 32 bits)
    const bool words = a.ldq < 0x7fffffff && a.ldp < 0x7fffffff &&
                       in_words({{a.q, a.ldq}, {a.p, a.ldp}, {a.p, a.p_stride}, {a.out, a.ldo}, {a.out, a.out_stride}, {a.pre, a.ldpre},
                                 {a.q, kForm == WEIGHTS ? 0 : a.k}, {a.q, kForm == WEIGHTS ? a.m : 0}, {a.q, a.n}}, elem);
    const Access access = words ? WORDS : access_of<kForm>(a, elem);
    hipError_t rc = hipSuccess;
    by_type(dtype, [&](auto zero) { rc = by_size<decltype(zero), kForm>(a, f, access, s); });
    return rc;
}

}  // namespace

}  // namespace nacho
