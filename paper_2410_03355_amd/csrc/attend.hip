// Attention of draft trees, and of single tokens, over a paged cache (lantern_attend_trees).
//
// Row i of a sequence (0: the token before the candidates, 1 + j: candidate j) sees the cached tokens and, of the sequence's
// own rows, itself and its ancestors:  o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale * q . k_j - m).
//
// One wavefront takes 16 or 32 rows (QT tiles of 16; the query heads of a key head are rows of one matrix) through a run of
// cached tokens, one pass, with the running maximum and sum of the softmax.  Scores and weights keep to registers:
//   S^T = K Q^T    A: 16 tokens by 32 of the head's elements, B: the same elements of 16 rows
//   O^T = V^T P^T  A: 16 elements by 32 tokens, B: the same tokens of 16 rows
// The result of an instruction has a row's scores of four tokens in each lane, and the second product wants a row's weights of
// eight tokens in each lane.  Which token stands in which row of A is free: with token CH * (i / 4) + 4 t + i % 4 in row i of
// tile t, lane group g ends with the scores of tokens CH * g .. CH * g + CH - 1, and those are the ones it has to hold of P, so
// no value changes its lane.  Values are cached as [D][token] for the same reason: CH tokens of one element are 16 bytes.
//
// The four wavefronts of a workgroup take the same rows, or two sets of them, and every fourth (second) tile of tokens each, and join through LDS; where sequences, heads and
// row tiles are too few to fill the device a sequence is split over workgroups as well, whose parts a second kernel joins.
//
// Measured (kernel time; 8-bit cache, bf16, unless said): 8 single tokens of 32 heads on 4 of 128 behind 4099 to 32768 tokens 32 us and 5 for the join,
// 4.7 TB/s, where a large copy reaches 5.1; 64 trees of 61 rows, 20 heads of 64 over 120 to 690 tokens 45.7 us, bound by latency and issue (half of
// the vector instructions are prologue, own rows and join); 4 trees of 33 rows, 32 heads on 8 of 128 behind 2000 to 16001 tokens 57 + 5 us, 315
// TFLOP/s: vector units 46 k and matrix units 24 k of 136 k cycles, 1.4 wavefronts to a SIMD on the average, which wait for a third of their
// time; one token over 577 tokens 9 us, five loads one after the other.
//
// Registers.  The bounds at the kernel let two workgroups to a CU (bf16 up to 64 elements: three).  Two instances pay with scratch memory: bf16 over 8
// bits, D = 128, two tiles of rows 6 registers, and fp32, D = 128, two tiles 39 over 16 bits and 106 over 8 bits (D = 96 over 8 bits: 1).
#include <hip/hip_runtime.h>
#include <float.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cache_args.h"
#include "device_utils.h"
#include "lds_limit.h"
#include "rotation.h"

namespace lantern {

constexpr int MOST_ROWS = LANTERN_MAX_TREE + 1;   // of a sequence
// Of the lambdas: into their one caller before anything else is done with them, so that what they are handed stays in registers.
#define INLINE __attribute__((always_inline))
constexpr float LAZY = 8.f;      // a row's maximum moves up only when a score passes it by 8: weights stay under 2^8

struct F32x8 {
    float x[8];
};
template <typename T> struct Frag;
template <> struct Frag<bf16> { typedef bf16x8 type; };
template <> struct Frag<float> { typedef F32x8 type; };

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// fp32: eight steps of four elements, lane group g giving element j of its eight to step j.
__device__ __forceinline__ f32x4 mma(const F32x8& a, const F32x8& b, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x[j], b.x[j], c, 0, 0, 0);
    return c;
}

// Eight cached values as an operand; both types of a cache are exact in both types of an operand.
// (bf16: times a power of two, for nothing).
template <typename T>
__device__ __forceinline__ typename Frag<T>::type from_e4m3(unsigned lo, unsigned hi, float by = 1.f);
template <>
__device__ __forceinline__ bf16x8 from_e4m3<bf16>(unsigned lo, unsigned hi, float by) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <>
__device__ __forceinline__ F32x8 from_e4m3<float>(unsigned lo, unsigned hi, float) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, true);
    const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, true);
    return F32x8{{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]}};
}
template <typename T>
__device__ __forceinline__ typename Frag<T>::type from_bf16(u32x4 w);
template <>
__device__ __forceinline__ bf16x8 from_bf16<bf16>(u32x4 w) { return __builtin_bit_cast(bf16x8, w); }
template <>
__device__ __forceinline__ F32x8 from_bf16<float>(u32x4 w) {
    F32x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.x[2 * i] = __uint_as_float(w[i] << 16);
        r.x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
    return r;
}
__device__ __forceinline__ void set(bf16x8& f, int i, float x) { f[i] = (bf16)x; }
__device__ __forceinline__ void set(F32x8& f, int i, float x) { f.x[i] = x; }

__device__ __forceinline__ bf16 element_of(const bf16x8& f, int i) { return f[i]; }
__device__ __forceinline__ float element_of(const F32x8& f, int i) { return f.x[i]; }
__device__ __forceinline__ bf16x8 zeros(const bf16x8&) { return __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u}); }
__device__ __forceinline__ F32x8 zeros(const F32x8&) { return F32x8{}; }
// All eight finite: no exponent of ones only.
__device__ __forceinline__ bool finite(const bf16x8& f) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const u32x4 w = __builtin_bit_cast(u32x4, f);
    u16x2 top = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
    return max(top[0], top[1]) < 0x7F80u;
}
__device__ __forceinline__ bool finite(const F32x8& f) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f.x[i]) & 0x7FFFFFFFu);
    return top < 0x7F800000u;
}

__device__ __forceinline__ float get(const bf16x8& f, int i) { return (float)f[i]; }
__device__ __forceinline__ float get(const F32x8& f, int i) { return f.x[i]; }

// Eight elements in a row of a dense tensor.
__device__ __forceinline__ bf16x8 load8(const bf16* x, bool wide) {
    if (wide) return *reinterpret_cast<const bf16x8*>(x);
    return bf16x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ F32x8 load8(const float* x, bool wide) {
    if (wide) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(x), b = *reinterpret_cast<const f32x4*>(x + 4);
        return F32x8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
    }
    return F32x8{{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}};
}

// Over the four lane groups: the swaps leave a value's partner of 16, then of 32 lanes on in the other register.
__device__ __forceinline__ float over_groups_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float over_groups_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A tile of cached tokens: 4 * CH of them, of which lane group g holds the values of CH.
//
// Neighbouring lanes of a product want neighbouring tokens of the keys and neighbouring elements of the values, and those lie
// 32 .. 256 bytes apart in a page: a load in that order costs the address unit one access per lane (48 to 51 per instruction were counted,
// and the unit was busy all the time).  So a wavefront brings its tile to LDS in the order of memory, 16 bytes to a lane, and the
// products read it from there.  Two or four wavefronts that share a tile wait for each other twice a tile and were slower.  Rows of LDS end
// with 16 bytes more, and keys stand in the order of the product's rows, so that 16 lanes meet 16 different groups of banks.
template <bool EIGHT, int D>
struct Tile {
    static constexpr int CH = EIGHT ? 16 : 8;          // 16 bytes of an element's values
    static constexpr int TOKENS = 4 * CH;
    static constexpr int SIZE = EIGHT ? 1 : 2;
    static constexpr int CHUNKS = 4 * D;               // of 16 bytes, of its keys as of its values
    static constexpr int PER_TOKEN = D * SIZE / 16;    // of them a token's key
    static constexpr int PARTS = TOKENS / 16;          // most pages that it lies on
    static constexpr int KROW = D * SIZE + 16, VROW = 64 + 16;
    static constexpr int KBYTES = TOKENS * KROW, VBYTES = D * VROW;
    // Whether 64 chunks in a row lie on one page, however small
    static constexpr bool WHOLE = 16 * D * SIZE % 1024 == 0;

    // Where the eight elements of step s (of 32) begin in a lane group: a load of 16 bytes brings two steps of 8-bit keys.
    __device__ static __forceinline__ int element(int s, int g) {
        if (EIGHT && s < D / 64 * 2) return s / 2 * 64 + g * 16 + s % 2 * 8;
        return s * 32 + g * 8;
    }
    // Row of a token's key in LDS: tile t of 16, row i of that, for token CH * (i / 4) + 4 t + i % 4.
    __device__ static __forceinline__ int row_of(int token) { return token % CH / 4 * 16 + token / CH * 4 + token % 4; }
};

// What one wavefront keeps of its QT * 16 rows: lane col of every group holds row col of a tile.
template <typename T, int D, int QT>
struct Rows {
    typedef typename Frag<T>::type Operand;
    static constexpr int DT = D / 16, STEPS = D / 32;
    // bf16 weights are summed as they are rounded, by the same instructions: a row of ones above the values.  fp32: in the lanes.
    static constexpr bool ONES = sizeof(T) == 2;
    Operand q[QT][STEPS];
    f32x4 o[QT][DT], sums[QT];
    float m[QT];                   // running maximum, the same in all groups

    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            m[qt] = neg_inf_f();
            sums[qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ float sum(int qt) const {
        return ONES ? sums[qt][0] : over_groups_sum((sums[qt][0] + sums[qt][1]) + (sums[qt][2] + sums[qt][3]));
    }

    // Scores of 32 tokens -> weights.  f > 0: the scores' scale in this lane; vs: what the weights are multiplied by for the second product.
    // Tokens that are not seen have a score of -inf.  EARLIER: there are weights that have been summed and wait for the second product.  The
    // maximum is a whole number, upwards: a step of it is a power of two, by which earlier weights, bf16 ones too, are moved exactly.
    // With bf16 operands a weight is rounded to bf16, which the matrix instructions take, at most half a step of 2^-8 of it, and the sum takes
    // it as rounded, so what all weights are off by alike cancels.  1.6e-3 of an output (relative, over listed calls) where the output's own rounding
    // is 1.7e-3, 2.3e-3 together; a second operand for what the rounding leaves would be half as many matrix instructions again.
    template <bool EARLIER>
    __device__ __forceinline__ void weigh(const f32x4 (&s)[QT][2], float f, float vs, Operand (&p)[QT], Operand (&earlier)[QT]) {
        float top[QT];
        bool up = false;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            float x = s[qt][0][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) x = fmaxf(x, s[qt][j / 4][j % 4]);
            top[qt] = x * f;
            up |= top[qt] > m[qt] + LAZY;
        }
        if (__any(up)) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const float to = fmaxf(m[qt], ceilf(over_groups_max(top[qt])));
                const float by = to == m[qt] ? 1.f : ldexpf(1.f, (int)fmaxf(m[qt] - to, -1000.f));
                m[qt] = to;
                sums[qt] *= by;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[qt][dt] *= by;
                if constexpr (EARLIER) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) set(earlier[qt], j, get(earlier[qt], j) * by);
                }
            }
        }
        const bool scaled = __any(vs != 1.f);
        Operand one;
#pragma unroll
        for (int i = 0; i < 8; ++i) set(one, i, 1.f);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const float less = m[qt] == neg_inf_f() ? 0.f : -m[qt];
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][j / 4][j % 4], f, less));
#pragma unroll
            for (int j = 0; j < 8; ++j) set(p[qt], j, w[j]);
            if constexpr (ONES) {
                sums[qt] = mma(one, p[qt], sums[qt]);
            } else {
                sums[qt][0] += w[0] + w[1];
                sums[qt][1] += w[2] + w[3];
                sums[qt][2] += w[4] + w[5];
                sums[qt][3] += w[6] + w[7];
            }
            if (scaled) {      // bf16: rounded once all the same, from fp32
#pragma unroll
                for (int j = 0; j < 8; ++j) set(p[qt], j, w[j] * vs);
            }
        }
    }
};

// What other lanes of the wavefront have written to LDS is there.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// LDS of a workgroup: a place for each wavefront's tile, which keys and then values go through; own rows, as many as a tile has tokens:
// their keys like a tile's, their values turned over; what the rows see.  In the end the wavefronts' parts.
template <typename T, bool EIGHT, int D, int QT>
struct Shared {
    typedef Tile<EIGHT, D> Tokens;
    static constexpr int TILE = Tokens::KBYTES > Tokens::VBYTES ? Tokens::KBYTES : Tokens::VBYTES;
    static constexpr int OWN_KROW = D * (int)sizeof(T) + 16, OWN_VROW = Tokens::TOKENS + 16 / (int)sizeof(T);
    static constexpr int OWN_K = Tokens::TOKENS * OWN_KROW, OWN_V = (int)sizeof(T) * D * OWN_VROW;
    static constexpr int FIXED = NW * TILE + OWN_K + OWN_V;
    static constexpr int PART = 16 * QT * (D + 4);                  // floats of a wavefront's part
    static constexpr int JOIN = NW * PART * (int)sizeof(float);
    __host__ __device__ static constexpr int bytes(int rows) {      // seen, present; jump, lost where rows are over 64
        const int words = (rows + 31) / 32;
        const int all = FIXED + (int)sizeof(int) * (rows * words + words + (rows > WAVE ? 2 * rows : 0));
        return all > JOIN ? all : JOIN;
    }
};

// Parts of the B sequences where there are `parts` > B: all are of as many tiles of tokens, the last of a sequence of what is left, and
// a sequence has one at least.  With tiles T_b and size = T / (parts - B), sum ceil(T_b / size) <= parts; the least such size lies between
// that and T / parts, and a wavefront that has a sequence to a lane finds it by halves (4 trees behind 2000 to 16001 tokens: 56 tiles instead
// of 72).  Every wavefront finds its part from the lengths by itself.
struct Parts {
    int size;      // tiles
    __device__ __forceinline__ static int tiles_of(const AttendArgs& a, int b, int tokens) {
        const int n = b < a.B ? a.lengths[b] : 0;
        return n < 0 || (int64_t)n > (int64_t)a.width << a.page_shift ? 0 : (n + tokens - 1) / tokens;
    }
    __device__ __forceinline__ Parts(const AttendArgs& a, int tokens) {
        const int lane = threadIdx.x & (WAVE - 1);
        int low = 0, high = 0;      // two sums: up to 512 sequences of 2^25 tiles
        for (int b = lane; b < a.B; b += WAVE) {
            const int t = tiles_of(a, b, tokens);
            low += t & 0xFFFF;
            high += t >> 16;
        }
        low = __builtin_amdgcn_readlane(wave_scan_i<OpSum>(low, 0), WAVE - 1);
        high = __builtin_amdgcn_readlane(wave_scan_i<OpSum>(high, 0), WAVE - 1);
        const double all = (double)high * 65536.0 + (double)low;
        size = ((int)(all * a.per_part) + NW) / NW * NW;      // per_part: 1 / (parts - B), a little more
        if (a.B <= WAVE) {
            const int mine = tiles_of(a, lane, tokens), low_rounds = max(1, (int)(all * a.per_all));      // per_all: 1 / (parts * NW), a little less
            for (int from = low_rounds, to = size / NW; from < to;) {
                const int mid = (from + to) / 2;
                size = mid * NW;
                const int n = __builtin_amdgcn_readlane(wave_scan_i<OpSum>(lane < a.B ? count(mine) : 0, 0), WAVE - 1);
                if (n <= a.parts) to = mid;
                else from = mid + 1;
                size = to * NW;
            }
        }
    }
    __device__ __forceinline__ int count(int tiles) const { return tiles <= size ? 1 : (int)((unsigned)(tiles + size - 1) / (unsigned)size); }
};

// ABREAST wavefronts of a workgroup take QT * 16 rows each, side by side; the TEAMS that there are of such take a sequence's tiles of cached
// tokens in turn.
template <typename T, bool EIGHT, int D, int QT, int ABREAST>
__global__ __launch_bounds__(NT, sizeof(T) == 2 && D <= 64 ? 3 : 2) void attend_trees_kernel(AttendArgs a) {
    typedef Rows<T, D, QT> Mine;
    typedef Tile<EIGHT, D> Tokens;
    typedef Shared<T, EIGHT, D, QT> Lds;
    typedef typename Frag<T>::type Operand;
    constexpr int CH = Tokens::CH, TOKENS = Tokens::TOKENS, STEPS = D / 32, DT = D / 16, SIZE = Tokens::SIZE, HALVES = CH / 8;
    constexpr int ROW = Lds::OWN_VROW, PARTS = Tokens::PARTS;
    constexpr int TEAMS = NW / ABREAST;
    constexpr int PER = Tokens::CHUNKS / WAVE;      // chunks of a tile to a lane
    extern __shared__ __attribute__((aligned(16))) char shared[];
    __shared__ float wave_m[NW][16 * QT], wave_l[NW][16 * QT];

    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), col = lane & 15, g = lane >> 4;
    const int rows_of = a.M + 1, words = (rows_of + 31) / 32, R = rows_of * a.group, heads = a.cache.heads;
    char* const own_keys = shared + NW * Lds::TILE;
    T* const staged = reinterpret_cast<T*>(own_keys + Lds::OWN_K);
    unsigned* const seen = reinterpret_cast<unsigned*>(shared + Lds::FIXED);
    unsigned* const present = seen + rows_of * words;
    int *const jump = reinterpret_cast<int*>(present + words), *const lost = jump + rows_of;
    // The row tiles of one part of a sequence and head read the same tokens: they get numbers 8 apart, which one XCD serves.
    const int chunk = a.by_tiles.of(blockIdx.x >> 3);
    const int item = chunk * 8 + (int)(blockIdx.x & 7);
    const int beside = wave % ABREAST, team = wave / ABREAST;
    const int group_row = ((int)(blockIdx.x >> 3) - chunk * a.row_tiles) * (16 * QT * ABREAST), first_row = group_row + beside * 16 * QT;
    const int part = a.by_heads.of(item), h = item - part * heads;
    if (part >= a.parts) return;
    int b = part, nth = 0, size = INT_MAX;      // the sequence, its part, and how many tiles that has
    bool whole = true;
    if (a.parts > a.B) {
        const Parts parts(a, TOKENS);
        size = parts.size;
        b = -1;
        for (int base = 0, before = 0; base < a.B; base += WAVE) {
            const int n = base + lane < a.B ? parts.count(Parts::tiles_of(a, base + lane, TOKENS)) : 0;
            const int upto = before + wave_scan_i<OpSum>(n, 0);
            const uint64_t mine = __ballot(part >= upto - n && part < upto);
            if (mine) {
                const int at = __ffsll((long long)mine) - 1;
                b = base + at;
                nth = part - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(n, at));
                const int of = __builtin_amdgcn_readlane(n, at);
                whole = of == 1;
                if (nth == 0 && h == 0 && group_row == 0 && threadIdx.x == 0) a.cut[b] = make_int2(part, of);      // for the join
                break;
            }
            before = __builtin_amdgcn_readlane(upto, WAVE - 1);
        }
        if (b < 0) return;      // fewer parts than there is room for
    }
    const int told = a.lengths[b], page = 1 << a.page_shift;
    const bool absent = told < 0, too_long = (int64_t)told > (int64_t)a.width << a.page_shift;
    const int length = absent || too_long ? 0 : told;
    const int tiles = (length + TOKENS - 1) / TOKENS;
    const int begin = (whole ? 0 : nth * size) + team, end = ABREAST > 1 && first_row >= R ? 0 : whole ? tiles : min(tiles, (nth + 1) * size);
    const bool has_tree = whole || (nth + 1) * size >= tiles;

    // ---- the rows: B of the first product
    Mine mine;
    int node[QT];      // the sequence's row that a row of the matrix belongs to
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) node[qt] = a.by_group.of(min(first_row + qt * 16 + col, R - 1));
    auto rows = [&](bool wide) INLINE {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const int head = h * a.group + min(first_row + qt * 16 + col, R - 1) - node[qt] * a.group;
            const T* x = static_cast<const T*>(a.q) + b * a.sq.seq + node[qt] * a.sq.row + head * a.sq.head;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) mine.q[qt][s] = load8(x + Tokens::element(s, g), wide);
        }
    };
    if (a.wide) rows(true);
    else rows(false);
    mine.begin();

    // ---- where the cached tokens are
    const int last = begin < end ? begin + (end - 1 - begin) / TEAMS * TEAMS : begin;      // this wavefront's last tile
    const int32_t* const table = a.table + (int64_t)b * a.width;
    const unsigned page_bytes = (unsigned)heads * page * D * SIZE;      // 65535 heads at most: under 2^31
    const char* const kbase = static_cast<const char*>(a.cache.k) + (int64_t)h * page * D * SIZE;
    const char* const vbase = static_cast<const char*>(a.cache.v) + (int64_t)h * page * D * SIZE;
    // This lane's chunks of a tile: page of the tile's, place in it, place in LDS; each a lane's own part and, where a load's 64 chunks
    // are whole tokens (elements) of one page, one that the wavefront shares.
    constexpr bool LINEAR = Tokens::WHOLE && WAVE % Tokens::PER_TOKEN == 0;
    const int row_chunks = page * SIZE >= 64 ? 2 : page * SIZE >= 32 ? 1 : 0;      // log2 of an element's chunks on one page
    struct Chunk {
        int part, from, to, token;
    };
    auto key_chunk = [&](int j) INLINE {
        constexpr int AT_ONCE = WAVE / Tokens::PER_TOKEN;      // tokens to a load
        if constexpr (LINEAR) {
            const int first = j * AT_ONCE, mine = lane / Tokens::PER_TOKEN;
            return Chunk{first >> a.page_shift, (first & (page - 1)) * (D * SIZE) + lane * 16,
                         (Tokens::row_of(first + mine) * Tokens::KROW) + lane % Tokens::PER_TOKEN * 16, first};
        } else {
            const int c = lane + j * WAVE, token = c / Tokens::PER_TOKEN, ch = c % Tokens::PER_TOKEN;
            return Chunk{token >> a.page_shift, (token & (page - 1)) * (D * SIZE) + ch * 16, Tokens::row_of(token) * Tokens::KROW + ch * 16, token};
        }
    };
    auto value_chunk = [&](int j) INLINE {
        if constexpr (LINEAR) {
            const int first = j * (WAVE >> row_chunks), d = first % D, part = first / D;
            const int mine = lane >> row_chunks, gi = lane & ((1 << row_chunks) - 1);
            return Chunk{part, d * page * SIZE + (mine * page * SIZE + gi * 16),
                         d * Tokens::VROW + (part << row_chunks) * 16 + (mine * Tokens::VROW + gi * 16), ((part << row_chunks) + gi) * CH};
        } else {
            const int x = (lane + j * WAVE) >> row_chunks, gi = lane & ((1 << row_chunks) - 1), part = x / D, d = x % D;
            return Chunk{part, d * page * SIZE + gi * 16, d * Tokens::VROW + ((part << row_chunks) + gi) * 16, ((part << row_chunks) + gi) * CH};
        }
    };
    // Pages of a tile, in the lanes of one load that is asked for a tile ahead and without waiting for the length.
    auto ask_ids = [&](int tile) INLINE { return table[min((tile * TOKENS >> a.page_shift) + lane % PARTS, a.width - 1)]; };
    auto good = [&](int id) INLINE { return (unsigned)id < (unsigned)a.cache.pages; };
    // One of the up to four of a tile.  A page behind the end is not looked at (page 0 is read in its place, and its tokens are not
    // seen); nor is one that is no page.
    struct Pages {
        uint64_t a, b, c, d;
        __device__ __forceinline__ uint64_t operator[](int i) const {
            const uint64_t p = a, q = b, r = c, s = d;      // values first: a choice of members is one of addresses, in scratch memory
            const uint64_t low = i & 1 ? q : p, high = i & 1 ? s : r;
            return i & 2 ? high : low;
        }
    };
    auto pages_of = [&](int tile, int ids) INLINE {
        auto at = [&](int i) INLINE {
            const int id = __builtin_amdgcn_readlane(ids, i);
            return good(id) && tile * TOKENS + (i << a.page_shift) < length ? (uint64_t)(unsigned)id * page_bytes : (uint64_t)0;
        };
        Pages x = {at(0), 0, 0, 0};
        if (PARTS > 1 && page < TOKENS) {
            x.b = at(1);
            if (PARTS > 2) x.c = at(2), x.d = at(3);
        }
        return x;
    };
    struct Scales {
        float k, v;      // of this lane's scores and values
        bool bad;        // the page is none
    };
    u32x4 coming[PER];      // keys or values of a tile on their way
    auto ask_keys = [&](int tile, const Pages& x) INLINE {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            coming[j] = *reinterpret_cast<const u32x4*>(kbase + x[key_chunk(j).part] + (tile * TOKENS & (page - 1)) * (D * SIZE) + key_chunk(j).from);
    };
    auto ask_values = [&](int tile, const Pages& x) INLINE {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            coming[j] = *reinterpret_cast<const u32x4*>(vbase + x[value_chunk(j).part] + (tile * TOKENS & (page - 1)) * SIZE + value_chunk(j).from);
    };
    auto put_keys = [&](char* to) INLINE {
#pragma unroll
        for (int j = 0; j < PER; ++j) *reinterpret_cast<u32x4*>(to + key_chunk(j).to) = coming[j];
    };
    // Nothing of the values behind the sequence's end: those slots hold anything, NaN too.
    auto put_values = [&](char* to, int tile) INLINE {
        if ((tile + 1) * TOKENS > length) {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int keep = length - tile * TOKENS - value_chunk(j).token;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int in = min(4, max(0, keep * SIZE - 4 * w));     // bytes of this word
                    coming[j][w] &= in == 4 ? 0xFFFFFFFFu : (1u << 8 * in) - 1u;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) *reinterpret_cast<u32x4*>(to + value_chunk(j).to) = coming[j];
    };
    const float *const k_scale = a.cache.k_scale + h, *const v_scale = a.cache.v_scale + h;
    const int own_part = g * CH >> a.page_shift;
    auto ask_scales = [&](int tile, int ids) INLINE {      // a lane group's scores are those of its values' tokens
        int id = __builtin_amdgcn_readlane(ids, 0);
        if (PARTS > 1 && page < TOKENS) {
#pragma unroll
            for (int i = 1; i < PARTS; ++i) {
                const int other = __builtin_amdgcn_readlane(ids, i);
                id = own_part == i ? other : id;
            }
        }
        const bool seen_here = tile * TOKENS + g * CH < length;
        Scales s = {1.f, 1.f, !good(id) && seen_here};
        if constexpr (EIGHT) {
            const uint64_t at = (uint64_t)(good(id) && seen_here ? (unsigned)id : 0u) * (unsigned)heads;
            s.k = k_scale[at];
            s.v = v_scale[at];
        }
        return s;
    };
    auto tile_after = [&](int tile) INLINE { return min(tile + TEAMS, last); };
    int ids = ask_ids(begin);
    Scales scales = {1.f, 1.f, false};

    // ---- the sequence's own rows
    const T* const own_k = static_cast<const T*>(a.k) + b * a.sk.seq + h * a.sk.head;
    const T* const own_v = static_cast<const T*>(a.v) + b * a.sv.seq + h * a.sv.head;
    auto parent_of = [&](int i, int* bad) INLINE {      // row of the token before row i
        if (i == 0) return 0;
        const int p = a.parent ? a.parent[(int64_t)b * a.M + i - 1] : i - 2;
        if (p >= -1 && p < i - 1) return p + 1;
        *bad = 1;
        return 0;
    };
    // Own rows on their way to LDS, 8 elements to a thread: keys in the order of the product's rows, values turned over; where one is not
    // finite, such values are taken out by another pass.  Neighbouring threads have neighbouring elements of a key, and the same elements of neighbouring values: what
    // they write then lies next to each other.
    constexpr int OWN = TOKENS * (D / 8), OWN_PER = (OWN + NT - 1) / NT;
    struct Taken {
        Operand k[OWN_PER], v[OWN_PER];
    };
    auto take = [&](int base, bool wide) INLINE {
        Taken t;
#pragma unroll
        for (int n = 0; n < OWN_PER; ++n) {
            const int e = min((int)threadIdx.x + n * NT, OWN - 1);
            t.k[n] = load8(own_k + min(base + e / (D / 8), rows_of - 1) * a.sk.row + e % (D / 8) * 8, wide);
            t.v[n] = load8(own_v + min(base + e % TOKENS, rows_of - 1) * a.sv.row + e / TOKENS * 8, wide);
        }
        return t;
    };
    auto stage = [&](const Taken& t, int base) INLINE {      // returns whether a value is not finite
        bool odd = false;
#pragma unroll
        for (int n = 0; n < OWN_PER; ++n) {
            const int e = min((int)threadIdx.x + n * NT, OWN - 1), i = e % TOKENS, d = e / TOKENS * 8;
            *reinterpret_cast<Operand*>(own_keys + Tokens::row_of(e / (D / 8)) * Lds::OWN_KROW + e % (D / 8) * 8 * (int)sizeof(T)) = t.k[n];
            const Operand v = base + i < rows_of ? t.v[n] : zeros(t.v[n]);
            odd |= !finite(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) staged[(d + j) * ROW + i] = element_of(v, j);
        }
        return odd;
    };
    auto clean = [&]() INLINE {      // seldom: 0 for what is not finite of this thread's values
#pragma unroll 1
        for (int e = threadIdx.x; e < OWN; e += NT)
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                T& x = staged[(e / TOKENS * 8 + j) * ROW + e % TOKENS];
                if (!(fabsf((float)x) < __builtin_huge_valf())) x = (T)0.f;
            }
        __syncthreads();
    };
    Taken taken;
    const int i = threadIdx.x;
    int bad = absent, up = 0;
    if (has_tree) {
        taken = a.wide ? take(0, true) : take(0, false);
        if (i < rows_of) up = parent_of(i, &bad);
    }
    Pages at = {0, 0, 0, 0};
    if (begin < end) {
        at = pages_of(begin, ids);
        scales = ask_scales(begin, ids);
        ids = ask_ids(tile_after(begin));
        ask_keys(begin, at);
    }
    // Ancestors of every row, itself included, as bits: doubling along the parents
    bool odd = false;
    if (has_tree) {
        odd = stage(taken, 0);
        if (rows_of <= WAVE) {      // one wavefront, a row to a lane
            if (wave == 0) {
                unsigned lo = i < 32 ? 1u << i : 0u, hi = i < 32 ? 0u : 1u << (i - 32);
                while (__any(up != 0)) {
                    lo |= __shfl(lo, up);
                    hi |= __shfl(hi, up);
                    bad |= __shfl(bad, up);
                    up = __shfl(up, up);
                }
                if (i < rows_of) {
                    seen[i * words] = lo | 1u;
                    if (words > 1) seen[i * words + 1] = hi;
                }
            }
        } else {
            if (i < rows_of) {
                jump[i] = up;
                lost[i] = bad;
                for (int w = 0; w < words; ++w) seen[i * words + w] = w == i / 32 ? 1u << i % 32 : 0u;
            }
            __syncthreads();
            for (int more = 1; more;) {
                unsigned got[MOST_ROWS / 32];
                int above = 0;
                if (i < rows_of) {
                    above = jump[i];
#pragma unroll
                    for (int w = 0; w < MOST_ROWS / 32; ++w)
                        if (w < words) got[w] = seen[above * words + w];
                    bad = lost[above];
                    up = jump[above];
                }
                more = __syncthreads_or(above != 0);
                if (i < rows_of) {
#pragma unroll
                    for (int w = 0; w < MOST_ROWS / 32; ++w)
                        if (w < words) seen[i * words + w] |= got[w];
                    lost[i] |= bad;
                    jump[i] = up;
                }
                __syncthreads();
            }
            if (i < rows_of) bad = lost[i];
        }
        const uint64_t alive = __ballot(i < rows_of && !bad);
        if (lane < 2 && 2 * wave + lane < words) present[2 * wave + lane] = (unsigned)(alive >> 32 * lane);
        odd = __syncthreads_or(odd);
        if (odd) clean();
    }

    // ---- cached tokens, a half of a tile (8 tokens of every lane group) at a time
    f32x4 s[QT][2];
    Operand p[QT];
    auto scores = [&](const char* keys, int half) INLINE {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const char* row = keys + ((2 * half + t) * 16 + col) * Tokens::KROW;
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) s[qt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (EIGHT) {
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(row + j * 64 + g * 16);
                    const Operand k = from_e4m3<T>(w[0], w[1]), l = from_e4m3<T>(w[2], w[3]);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(k, mine.q[qt][2 * j], s[qt][t]);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(l, mine.q[qt][2 * j + 1], s[qt][t]);
                }
                if constexpr (D % 64 != 0) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(row + D / 64 * 64 + g * 8);
                    const Operand k = from_e4m3<T>(w[0], w[1]);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(k, mine.q[qt][STEPS - 1], s[qt][t]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const Operand k = from_bf16<T>(*reinterpret_cast<const u32x4*>(row + j * 64 + g * 16));
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(k, mine.q[qt][j], s[qt][t]);
                }
            }
        }
    };
    auto outputs = [&](const char* values, int half, float two) INLINE {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const char* at = values + (dt * 16 + col) * Tokens::VROW + g * 16;
            Operand v;
            if constexpr (EIGHT) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(at + half * 8);
                v = from_e4m3<T>(w[0], w[1], two);
            } else {
                v = from_bf16<T>(*reinterpret_cast<const u32x4*>(at));
            }
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) mine.o[qt][dt] = mma(v, p[qt], mine.o[qt][dt]);
        }
    };
    char* const place = shared + wave * Lds::TILE;
    for (int tile = begin; tile < end; tile += TEAMS) {
        float f = a.scale * scales.k, vs = scales.v, two = 1.f;
        f = f < FLT_MIN ? FLT_MIN : f;                   // -inf * f stays -inf
        if (scales.bad) f = __builtin_nanf("");          // what the page should have held is not known: the rows become NaN
        if constexpr (EIGHT && sizeof(T) == 2) {         // the scale's power of two goes to the values as they are converted
            two = __uint_as_float(__float_as_uint(vs) & 0x7F800000u);
            vs = __uint_as_float((__float_as_uint(vs) & 0x7FFFFFu) | 0x3F800000u);
        }
        const int keep = length - tile * TOKENS - g * CH;
        if (keep <= 0) f = vs = two = 1.f;
        // No branch around a load: where two ways meet, the compiler's wait is the longer of theirs.  The last round asks for its own
        // tile again.
        wave_sync();
        put_keys(place);
        wave_sync();
        ask_values(tile, at);
        Operand weights[HALVES][QT];
        auto weigh_half = [&](auto of) INLINE {
            constexpr int half = of;
            scores(place, half);
            if ((tile + 1) * TOKENS > length) {
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (8 * half + j >= keep) s[qt][j / 4][j % 4] = neg_inf_f();
            }
            mine.template weigh<half != 0>(s, f, vs, weights[half], weights[0]);
        };
        weigh_half(std::integral_constant<int, 0>());
        if constexpr (HALVES == 2) weigh_half(std::integral_constant<int, 1>());
        wave_sync();
        put_values(place, tile);
        wave_sync();
        const int to = tile_after(tile);
        at = pages_of(to, ids);
        scales = ask_scales(to, ids);
        ids = ask_ids(tile_after(to));
        ask_keys(to, at);
#pragma unroll
        for (int half = 0; half < HALVES; ++half) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) p[qt] = weights[half][qt];
            outputs(place, half, two);
        }
    }

    // ---- the sequence's own rows, a half of what is staged to a wavefront, from the last on: it has the fewest cached tiles
    bool gone[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) gone[qt] = has_tree && !(present[node[qt] >> 5] >> (node[qt] & 31) & 1);
    for (int base = 0, turn = 0; has_tree && base < rows_of; base += TOKENS) {
        if (base > 0) {
            taken = a.wide ? take(base, true) : take(base, false);
            __syncthreads();
            odd = __syncthreads_or(stage(taken, base));
            if (odd) clean();
        }
#pragma unroll 1
        for (int half = 0; half < HALVES; ++half, ++turn) {
            if (turn % TEAMS != TEAMS - 1 - team || (ABREAST > 1 && first_row >= R)) continue;
            const int at = base + g * CH + half * 8;      // the first of this lane group's 8
            unsigned vis[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
                vis[qt] = gone[qt] || at >= rows_of ? 0u : seen[node[qt] * words + (at >> 5)] >> (at & 31);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const char* row = own_keys + ((2 * half + t) * 16 + col) * Lds::OWN_KROW;
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const Operand k = *reinterpret_cast<const Operand*>(row + Tokens::element(j, g) * (int)sizeof(T));
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(k, mine.q[qt][j], s[qt][t]);
                }
            }
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(vis[qt] >> j & 1)) s[qt][j / 4][j % 4] = neg_inf_f();
            mine.template weigh<false>(s, a.scale < FLT_MIN ? FLT_MIN : a.scale, 1.f, p, p);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const Operand v = load8(staged + (dt * 16 + col) * ROW + g * CH + half * 8, true);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) mine.o[qt][dt] = mma(v, p[qt], mine.o[qt][dt]);
            }
            if (odd) {
                // A value that is not finite may touch the rows that see it alone, and 0 * NaN is NaN: such values have been taken
                // out, and here the rows that see one become NaN.
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    Operand what;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float x = at + c < rows_of ? (float)own_v[(at + c) * a.sv.row + dt * 16 + col] : 0.f;
                        set(what, c, fabsf(x) < __builtin_huge_valf() ? 0.f : 1.f);
                    }
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) {
                        Operand sees;
#pragma unroll
                        for (int c = 0; c < 8; ++c) set(sees, c, vis[qt] >> c & 1 ? 1.f : 0.f);
                        const f32x4 hit = mma(what, sees, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (hit[r] > 0.f) mine.o[qt][dt][r] = __builtin_nanf("");
                    }
                }
            }
        }
    }

    // ---- the wavefronts' parts, each [rows][D + 4], through LDS: 4 elements of a row to a thread
    constexpr int PART = Lds::PART, ROWS = 16 * QT;
    float* const joined = reinterpret_cast<float*>(shared);
    __syncthreads();      // nobody reads tiles and own rows any more
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const float l = mine.sum(qt);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            *reinterpret_cast<f32x4*>(&joined[wave * PART + (qt * 16 + col) * (D + 4) + dt * 16 + g * 4]) = mine.o[qt][dt];
        if (g == 0) {
            // a row that is not there: no weight, and none of other parts' either
            wave_m[wave][qt * 16 + col] = gone[qt] ? __builtin_huge_valf() : mine.m[qt];
            wave_l[wave][qt * 16 + col] = gone[qt] ? 0.f : too_long && has_tree ? __builtin_nanf("") : l;
        }
    }
    __syncthreads();
    const int64_t rows_all = (int64_t)a.parts * heads * R;
    constexpr int UNITS = ABREAST * ROWS * (D / 4);
#pragma unroll
    for (int n = 0; n < (UNITS + NT - 1) / NT; ++n) {
        const int e = threadIdx.x + n * NT, d = e % (D / 4) * 4, rr = e / (D / 4) % ROWS, with = e / (D / 4) / ROWS, row = group_row + e / (D / 4);
        if (e >= UNITS || row >= R) continue;
        float m[TEAMS], high = neg_inf_f(), all = 0.f;
#pragma unroll
        for (int w = 0; w < TEAMS; ++w) {
            m[w] = wave_m[w * ABREAST + with][rr];
            high = fmaxf(high, m[w]);
        }
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < TEAMS; ++w) {
            const float by = m[w] == high ? 1.f : __builtin_amdgcn_exp2f(m[w] - high);
            sum += by * *reinterpret_cast<const f32x4*>(&joined[(w * ABREAST + with) * PART + rr * (D + 4) + d]);
            all += by * wave_l[w * ABREAST + with][rr];
        }
        const bool none = all == 0.f;       // nothing seen with a weight, or no row
        if (whole) {
            const int of = a.by_group.of(row), head = h * a.group + row - of * a.group;
            typedef typename Vec<T, 4>::type Four;
            const float per_all = 1.f / all;
            Four four;
#pragma unroll
            for (int j = 0; j < 4; ++j) four[j] = (T)(none ? 0.f : sum[j] * per_all);
            *reinterpret_cast<Four*>(static_cast<T*>(a.out) + (((int64_t)b * rows_of + of) * a.q_heads + head) * D + d) = four;
        } else {
            const int64_t at = (int64_t)item * R + row;
            *reinterpret_cast<f32x4*>(a.part + at * D + d) = none ? f32x4{0.f, 0.f, 0.f, 0.f} : sum;
            if (d == 0) {
                a.part[rows_all * D + at] = high;
                a.part[rows_all * (D + 1) + at] = all;
            }
        }
    }
}

// The parts of a sequence's rows joined.  A workgroup takes 64 pieces of 4 elements of the rows of one sequence and head, a piece to a lane,
// and its wavefronts every fourth part.  Sequences of one part have been written already.
template <typename T>
__global__ __launch_bounds__(NT) void attend_join_kernel(AttendArgs a) {
    __shared__ f32x4 sums[NW][WAVE];
    __shared__ float highs[NW][WAVE], alls[NW][WAVE];
    const int lane = threadIdx.x & (WAVE - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), heads = a.cache.heads, D = a.cache.D, rows_of = a.M + 1, R = rows_of * a.group;
    const int b = blockIdx.x, h = blockIdx.y;
    const int first = a.cut[b].x, n = a.cut[b].y;
    if (n == 1) return;
    const int64_t rows_all = (int64_t)a.parts * heads * R;
    const float *const pm = a.part + rows_all * D, *const pl = pm + rows_all;
    const int per_row = D / 4, units = R * per_row, unit = blockIdx.z * WAVE + lane;
    const int row = min(unit, units - 1) / per_row, d = min(unit, units - 1) % per_row * 4;
    float high = neg_inf_f(), all = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    bool gone = false;
    auto take = [&](float m, float l, f32x4 o) INLINE {
        gone |= m == __builtin_huge_valf() && l == 0.f;
        const float to = fmaxf(high, m), was = high == to ? 1.f : __builtin_amdgcn_exp2f(high - to), by = m == to ? 1.f : __builtin_amdgcn_exp2f(m - to);
        high = to;
        all = all * was + l * by;
        sum = sum * was + o * by;
    };
    constexpr int AHEAD = 4;
    for (int i = wave; i < n; i += AHEAD * NW) {
        float m[AHEAD], l[AHEAD];
        f32x4 o[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {      // past the end the last one again, without a weight
            const int64_t at = ((int64_t)(first + min(i + j * NW, n - 1)) * heads + h) * R + row;
            m[j] = pm[at];
            l[j] = pl[at];
            o[j] = *reinterpret_cast<const f32x4*>(a.part + at * D + d);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (i + j * NW < n) take(m[j], l[j], o[j]);
    }
    highs[wave][lane] = gone ? __builtin_huge_valf() : high;
    alls[wave][lane] = gone ? 0.f : all;
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave > 0 || unit >= units) return;
    for (int w = 1; w < NW; ++w) take(highs[w][lane], alls[w][lane], sums[w][lane]);
    const bool none = gone || all == 0.f;
    const int node = a.by_group.of(row), head = h * a.group + row - node * a.group;
    typedef typename Vec<T, 4>::type Four;
    const float per_all = 1.f / all;
    Four four;
#pragma unroll
    for (int j = 0; j < 4; ++j) four[j] = (T)(none ? 0.f : sum[j] * per_all);
    *reinterpret_cast<Four*>(static_cast<T*>(a.out) + (((int64_t)b * rows_of + node) * a.q_heads + head) * D + d) = four;
}

AttendPlan plan_attend(int dtype, int B, int M, int q_heads, const lantern_cache& c, int width) {
    AttendPlan p;
    const int64_t R = (int64_t)(M + 1) * (q_heads / c.heads);
    // Workgroups that are counted on to be resident on the 256 CUs: what the kernel's bound on registers lets in.  That is what fits with two tiles of
    // rows from D = 64 on, but for fp32 over 8 bits with D = 96 and 128, whose 82 and 108 KiB of LDS leave one to a CU, and D = 128 with trees of
    // about 160 rows and more over 8 bits (fp32: over 16).  With D = 32, and with one tile at D = 64 (bf16, and fp32 over 16 bits), four and more fit.
    const int64_t room = dtype == LANTERN_BF16 && c.D <= 64 ? 768 : 512;
    const int64_t tokens = (int64_t)width * c.page_tokens, tile = c.dtype == LANTERN_E4M3 ? 64 : 32;
    const int64_t useful = std::max<int64_t>(1, tokens / (tile * NW * 2));    // parts of two tiles to a wavefront at least
    // Tiles of 16 rows that a wavefront takes together: each conversion of a tile of tokens serves all of them.  Four (D <= 64, 246 registers)
    // were no faster where they had all their use: 64 trees of 61 rows 55.1 us against 53.8 with two, one tree 14.8 against 11.3.  One, where
    // all workgroups are counted to fit at once and sequences are not cut: a wavefront has less to do (one tree of 61 rows behind 640 tokens 9.9 us against 11.0, 8
    // of 33 11.6 against 13.1, but 26 of 33 23.4 against 21.7, and long sequences behind 33 rows 32 against 27).  Also in fp32, bound by its
    // products, where one leaves a sixth less of empty rows (20 trees of 33 rows 50 us against 61, of 66 97 against 102, but 132 rows 191
    // against 192 and less with shorter heads).
    const int64_t ones = (R + 15) / 16, twos = (R + 31) / 32;
    const bool one = R <= 16 || (useful == 1 && B * c.heads * ones <= room) || (dtype == LANTERN_F32 && 6 * ones <= 10 * twos);
    p.row_group = one ? 1 : 2;
    const int64_t tiles = one ? ones : twos;
    // Where workgroups of one set of such tiles are more than fit at once, two wavefronts take two sets side by side: half the workgroups,
    // which bring own rows, tree and arguments for twice the work.  20 heads, trees of 61 rows: 64 sequences 45.5 us against 52.5, 39 30.5
    // against 32.9, 20 21.3 against 22.8, but one 15.4 against 11.1.  fp32 is bound by its products and loses (32 sequences 97 against 87).
    p.abreast = dtype == LANTERN_BF16 && !one && tiles > 1 && B * c.heads * tiles > room ? 2 : 1;
    p.row_tiles = (int)((tiles + p.abreast - 1) / p.abreast);
    // Where sequences, heads and row tiles make fewer workgroups than fit, sequences are cut.
    const int64_t groups = (int64_t)c.heads * p.row_tiles;
    const int64_t parts = std::min(room / groups, B * useful);
    p.parts = (int)(parts >= 2 * (int64_t)B ? parts : B);
    p.workspace = p.parts == B ? 0 : (size_t)p.parts * c.heads * R * (c.D + 2) * sizeof(float) + B * sizeof(int2);
    return p;
}

template <typename T, bool EIGHT, int D, int QT, int ABREAST>
static hipError_t launch(const AttendArgs& a, hipStream_t stream) {
    hipError_t e = allow_lds<attend_trees_kernel<T, EIGHT, D, QT, ABREAST>>(Shared<T, EIGHT, D, QT>::bytes(MOST_ROWS));
    if (e != hipSuccess) return e;
    const int64_t items = (int64_t)a.parts * a.cache.heads;
    const int R = (a.M + 1) * a.group;
    const int blocks = (int)((items + 7) / 8 * 8 * a.row_tiles);
    const int lds = Shared<T, EIGHT, D, QT>::bytes(a.M + 1);
    hipLaunchKernelGGL((attend_trees_kernel<T, EIGHT, D, QT, ABREAST>), dim3(blocks), dim3(NT), lds, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.parts == a.B) return e;
    hipLaunchKernelGGL((attend_join_kernel<T>), dim3(a.B, a.cache.heads, (R * (D / 4) + WAVE - 1) / WAVE), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

template <typename T, bool EIGHT, int D>
static hipError_t launch_rows(const AttendArgs& a, int row_group, int abreast, hipStream_t stream) {
    if (row_group == 1) return launch<T, EIGHT, D, 1, 1>(a, stream);
    if constexpr (sizeof(T) == 2) {
        if (abreast == 2) return launch<T, EIGHT, D, 2, 2>(a, stream);
    }
    return launch<T, EIGHT, D, 2, 1>(a, stream);
}

template <typename T, bool EIGHT>
static hipError_t launch_width(const AttendArgs& a, int row_group, int abreast, hipStream_t stream) {
    switch (a.cache.D) {
        case 32: return launch_rows<T, EIGHT, 32>(a, row_group, abreast, stream);
        case 64: return launch_rows<T, EIGHT, 64>(a, row_group, abreast, stream);
        case 96: return launch_rows<T, EIGHT, 96>(a, row_group, abreast, stream);
        case 128: return launch_rows<T, EIGHT, 128>(a, row_group, abreast, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_attend_trees(const AttendArgs& a, int dtype, int row_group, int abreast, hipStream_t stream) {
    const bool eight = a.cache.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? launch_width<float, true>(a, row_group, abreast, stream) : launch_width<float, false>(a, row_group, abreast, stream);
    return eight ? launch_width<bf16, true>(a, row_group, abreast, stream) : launch_width<bf16, false>(a, row_group, abreast, stream);
}

template <typename T, bool EIGHT, int D>
static hipError_t prepare_rows() {
    hipError_t e = allow_lds<attend_trees_kernel<T, EIGHT, D, 1, 1>>(Shared<T, EIGHT, D, 1>::bytes(MOST_ROWS));
    if (e == hipSuccess) e = allow_lds<attend_trees_kernel<T, EIGHT, D, 2, 1>>(Shared<T, EIGHT, D, 2>::bytes(MOST_ROWS));
    if constexpr (sizeof(T) == 2) {
        if (e == hipSuccess) e = allow_lds<attend_trees_kernel<T, EIGHT, D, 2, 2>>(Shared<T, EIGHT, D, 2>::bytes(MOST_ROWS));
    }
    return e;
}

template <typename T, bool EIGHT>
static hipError_t prepare_width(int D) {
    switch (D) {
        case 32: return prepare_rows<T, EIGHT, 32>();
        case 64: return prepare_rows<T, EIGHT, 64>();
        case 96: return prepare_rows<T, EIGHT, 96>();
        case 128: return prepare_rows<T, EIGHT, 128>();
    }
    return hipSuccess;      // a cache that is not read here
}

hipError_t prepare_attend(int dtype, const lantern_cache& c) {
    hipFuncAttributes attr;   // the runtime loads all of a file's kernels together
    const hipError_t e = hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&attend_join_kernel<bf16>));
    if (e != hipSuccess) return e;
    const bool eight = c.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? prepare_width<float, true>(c.D) : prepare_width<float, false>(c.D);
    return eight ? prepare_width<bf16, true>(c.D) : prepare_width<bf16, false>(c.D);
}

}  // namespace lantern
