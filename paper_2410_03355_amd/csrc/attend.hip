// Attention of draft trees, and of single tokens, over a paged cache (lantern_attend_trees).
//
// Row i of a sequence (0: the token before the candidates, 1 + j: candidate j) sees the cached tokens and, of the sequence's
// own rows, itself and its ancestors:  o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale * q . k_j - m).
//
// One wavefront takes up to 64 rows (QT tiles of 16; the query heads of a key head are rows of one matrix) through a run of
// cached tokens, one pass, with the running maximum and sum of the softmax.  Both products keep to registers:
//   S^T = K Q^T    A: 16 tokens by 32 of the head's elements, B: the same elements of 16 rows
//   O^T = V^T P^T  A: 16 elements by 32 tokens, B: the same tokens of 16 rows
// The result of an instruction has a row's scores of four tokens in each lane, and the second product wants a row's weights of
// eight tokens in each lane.  Which token stands in which row of A is free: with token CH * (i / 4) + 4 t + i % 4 in row i of
// tile t, lane group g ends with the scores of tokens CH * g .. CH * g + CH - 1, and those are the ones it has to hold of P, so
// no value changes its lane.  Values are cached as [D][token] for the same reason: CH tokens of one element are 16 bytes.
//
// The four wavefronts of a workgroup take every fourth tile of tokens each and join through LDS; where sequences, heads and
// row tiles are too few to fill the device a sequence is split over workgroups as well, whose parts a second kernel joins.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include <algorithm>

#include "cache_args.h"
#include "device_utils.h"
#include "rotation.h"

namespace lantern {

constexpr int MOST_ROWS = LANTERN_MAX_TREE + 1;   // of a sequence
constexpr int WORDS = MOST_ROWS / 32;
constexpr float LAZY = 8.f;      // a row's maximum moves up only when a score passes it by 2^8: weights stay under 2^8

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
template <typename T>
__device__ __forceinline__ typename Frag<T>::type from_e4m3(unsigned lo, unsigned hi);
template <>
__device__ __forceinline__ bf16x8 from_e4m3<bf16>(unsigned lo, unsigned hi) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <>
__device__ __forceinline__ F32x8 from_e4m3<float>(unsigned lo, unsigned hi) {
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

__device__ __forceinline__ float over_groups_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float over_groups_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A tile of cached tokens on its way: keys as the first product's A, values as the second's.
template <bool EIGHT, int D>
struct Tile {
    static constexpr int CH = EIGHT ? 16 : 8;          // tokens to a lane group
    static constexpr int TOKENS = 4 * CH;
    static constexpr int SUB = CH / 4;                 // tiles of 16 tokens
    static constexpr int KW = EIGHT ? D / 16 : D / 8;  // words of a token's key in a lane
    unsigned k[SUB][KW];
    u32x4 v[D / 16];
    float f, vs;                                       // scale of this lane's scores, and of its values

    // Where the eight elements of step s (of 32) begin in a lane group: a load of 16 bytes brings two steps of 8-bit keys.
    __device__ static __forceinline__ int element(int s, int g) {
        if (EIGHT && s < D / 64 * 2) return s / 2 * 64 + g * 16 + s % 2 * 8;
        return s * 32 + g * 8;
    }

    template <typename T>
    __device__ __forceinline__ typename Frag<T>::type key(int t, int s) const {
        if constexpr (EIGHT) return from_e4m3<T>(k[t][2 * s], k[t][2 * s + 1]);
        else return from_bf16<T>(u32x4{k[t][4 * s], k[t][4 * s + 1], k[t][4 * s + 2], k[t][4 * s + 3]});
    }
    template <typename T>
    __device__ __forceinline__ typename Frag<T>::type value(int dt, int p) const {
        if constexpr (EIGHT) return from_e4m3<T>(v[dt][2 * p], v[dt][2 * p + 1]);
        else return from_bf16<T>(v[dt]);
    }
    // Nothing of the values from the lane's `keep`-th on: the slots behind a sequence's end hold anything, NaN too.
    __device__ __forceinline__ void cut_values(int keep) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int in = min(4, max(0, (keep * (EIGHT ? 1 : 2)) - 4 * w));     // bytes of this word
            const unsigned mask = in == 4 ? 0xFFFFFFFFu : (1u << 8 * in) - 1u;
#pragma unroll
            for (int dt = 0; dt < D / 16; ++dt) v[dt][w] &= mask;
        }
    }
};

// Pages of a tile, asked for one tile ahead of its tokens.
struct PageIds {
    int k, v;
};

template <typename T, bool EIGHT, int D, int QT>
__global__ __launch_bounds__(NT, 1) void attend_trees_kernel(AttendArgs a) {
    typedef Tile<EIGHT, D> Tokens;
    typedef typename Frag<T>::type Operand;
    constexpr int CH = Tokens::CH, TOKENS = Tokens::TOKENS, SUB = Tokens::SUB, STEPS = D / 32, DT = D / 16;
    constexpr int RED = 16 * (D + 4);                      // floats of one wavefront's part of 16 rows
    constexpr int SHARED = NW * RED > MOST_ROWS * WORDS ? NW * RED : MOST_ROWS * WORDS;
    __shared__ __attribute__((aligned(16))) float shared[SHARED];   // first the rows' ancestors, then the wavefronts' parts
    __shared__ int jump[MOST_ROWS], lost[MOST_ROWS];
    __shared__ float wave_m[NW][16 * QT], wave_l[NW][16 * QT];

    const int lane = threadIdx.x & (WAVE - 1), wave = threadIdx.x / WAVE, col = lane & 15, g = lane >> 4;
    const int rows_of = a.M + 1, R = rows_of * a.group, heads = a.cache.heads;
    // The row tiles of one part of a sequence and head read the same tokens: they get numbers 8 apart, which one XCD serves.
    const int parts = a.B * heads * a.splits, per = 8 * a.row_tiles;
    const int part = (int)blockIdx.x / per * 8 + (int)blockIdx.x % 8, row_tile = (int)blockIdx.x % per / 8;
    if (part >= parts) return;
    const int split = part % a.splits, bh = part / a.splits, b = bh / heads, h = bh % heads;
    const int first_row = row_tile * 16 * QT;
    const int told = a.lengths[b], page = 1 << a.page_shift;
    const bool absent = told < 0, too_long = (int64_t)told > (int64_t)a.width << a.page_shift;
    const int length = absent || too_long ? 0 : told;
    const bool has_tree = split == a.splits - 1;

    // ---- ancestors of every row, itself included, as bits: doubling along the parents
    unsigned* seen = reinterpret_cast<unsigned*>(shared);
    if (has_tree) {
        const int i = threadIdx.x;
        if (i < rows_of) {
            int up = 0, bad = absent;
            if (i > 0) {
                const int p = a.parent ? a.parent[(int64_t)b * a.M + i - 1] : i - 2;
                if (p < -1 || p >= i - 1) bad = 1;
                else up = p + 1;
            }
            for (int w = 0; w < WORDS; ++w) seen[i * WORDS + w] = w == i / 32 ? 1u << i % 32 : 0u;
            jump[i] = up;
            lost[i] = bad;
        }
        __syncthreads();
        for (;;) {
            unsigned got[WORDS];
            int to = 0, bad = 0;
            if (i < rows_of) {
                const int j = jump[i];
                for (int w = 0; w < WORDS; ++w) got[w] = seen[j * WORDS + w];
                bad = lost[j];
                to = jump[j];
            }
            const int more = __syncthreads_or(i < rows_of && jump[i] != 0);
            if (i < rows_of) {
                for (int w = 0; w < WORDS; ++w) seen[i * WORDS + w] |= got[w];
                lost[i] |= bad;
                jump[i] = to;
            }
            __syncthreads();
            if (!more) break;
        }
    }

    // ---- the rows: B of the first product
    Operand q[QT][STEPS];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int r = min(first_row + qt * 16 + col, R - 1), node = r / a.group, head = h * a.group + r % a.group;
        const T* x = static_cast<const T*>(a.q) + b * a.sq.seq + node * a.sq.row + head * a.sq.head;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q[qt][s] = load8(x + Tokens::element(s, g), a.wide);
    }
    f32x4 o[QT][DT];
    float m[QT], l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        m[qt] = neg_inf_f();
        l[qt] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Scores -> weights of one tile.  s: the scores, f: their scale (>= 0) in this lane, vs: the values'.  vis[qt]: bit c, whether
    // the row sees token c of the lane's CH.
    auto weigh = [&](f32x4 (&s)[QT][SUB], float f, float vs, const unsigned (&vis)[QT], bool masked, Operand (&p)[QT][CH / 8]) {
        float top[QT];
        bool up = false;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            float x = neg_inf_f();
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (masked && !(vis[qt] >> (4 * t + r) & 1)) s[qt][t][r] = neg_inf_f();
                    x = fmaxf(x, s[qt][t][r]);
                }
            top[qt] = x == neg_inf_f() ? x : x * f;
            up |= top[qt] > m[qt] + LAZY;
        }
        if (__any(up)) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const float to = fmaxf(m[qt], over_groups_max(top[qt]));
                const float by = to == m[qt] ? 1.f : __builtin_amdgcn_exp2f(m[qt] - to);
                m[qt] = to;
                l[qt] *= by;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[qt][dt] *= by;
            }
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const float less = m[qt] == neg_inf_f() ? 0.f : -m[qt];
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[qt][t][r], f, less));
                    if (masked && !(vis[qt] >> (4 * t + r) & 1)) w = 0.f;
                    l[qt] += w;
                    // bf16: a weight times its value's scale is rounded once, by 2^-9 of it at most, as an output is
                    set(p[qt][t / 2], t % 2 * 4 + r, EIGHT ? w * vs : w);
                }
        }
    };

    // ---- cached tokens
    const int tiles = (length + TOKENS - 1) / TOKENS;
    const int begin = (int)((int64_t)tiles * split / a.splits) + wave, end = (int)((int64_t)tiles * (split + 1) / a.splits);
    const int32_t* table = a.table + (int64_t)b * a.width;
    const int last_page = (length - 1) >> a.page_shift;
    const int64_t page_bytes = (int64_t)heads * page * D * (EIGHT ? 1 : 2);
    const char* kbase = static_cast<const char*>(a.cache.k) + (int64_t)h * page * D * (EIGHT ? 1 : 2);
    const char* vbase = static_cast<const char*>(a.cache.v) + (int64_t)h * page * D * (EIGHT ? 1 : 2);

    auto pages_of = [&](int tile) {      // a group behind the end is given the last page, whose tokens are then not seen
        const int kt = tile * TOKENS + col / 4 * CH, vt = tile * TOKENS + g * CH;
        return PageIds{table[min(kt >> a.page_shift, last_page)], table[min(vt >> a.page_shift, last_page)]};
    };
    auto bring = [&](int tile, PageIds id, Tokens& x) {
        const bool good_k = id.k >= 0 && id.k < a.cache.pages, good_v = id.v >= 0 && id.v < a.cache.pages;
        const int kpage = good_k ? id.k : 0, vpage = good_v ? id.v : 0;
        const int kslot = ((tile * TOKENS + col / 4 * CH) & (page - 1)) + col % 4, vslot = (tile * TOKENS + g * CH) & (page - 1);
        const char* kp = kbase + kpage * page_bytes + (int64_t)kslot * D * (EIGHT ? 1 : 2);
        const char* vp = vbase + vpage * page_bytes + vslot * (EIGHT ? 1 : 2);
#pragma unroll
        for (int t = 0; t < SUB; ++t) {
            const char* kr = kp + t * 4 * D * (EIGHT ? 1 : 2);
            if constexpr (EIGHT) {
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(kr + j * 64 + g * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.k[t][4 * j + i] = w[i];
                }
                if constexpr (D % 64 != 0) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(kr + D / 64 * 64 + g * 8);
                    x.k[t][D / 64 * 4] = w[0];
                    x.k[t][D / 64 * 4 + 1] = w[1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const u32x4 w = *reinterpret_cast<const u32x4*>(kr + j * 64 + g * 16);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.k[t][4 * j + i] = w[i];
                }
            }
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            x.v[dt] = *reinterpret_cast<const u32x4*>(vp + (int64_t)(dt * 16 + col) * page * (EIGHT ? 1 : 2));
        x.f = a.scale;
        x.vs = 1.f;
        if constexpr (EIGHT) {      // lane group g's scores are those of its values' tokens
            x.f *= a.cache.k_scale[(int64_t)vpage * heads + h];
            x.vs = a.cache.v_scale[(int64_t)vpage * heads + h];
        }
        if (!good_v) x.f = __builtin_nanf("");      // what a bad page should have held is not known: the rows become NaN
    };

    Tokens now, next;
    PageIds ids = {0, 0};
    if (begin < end) {
        bring(begin, pages_of(begin), now);
        if (begin + NW < end) ids = pages_of(begin + NW);
    }
    for (int tile = begin; tile < end; tile += NW) {
        if (tile + NW < end) {
            bring(tile + NW, ids, next);
            if (tile + 2 * NW < end) ids = pages_of(tile + 2 * NW);
        }
        const bool masked = (tile + 1) * TOKENS > length;
        unsigned vis[QT];
        if (masked) {
            const int keep = min(CH, max(0, length - tile * TOKENS - g * CH));
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) vis[qt] = (1u << keep) - 1u;
            now.cut_values(keep);
            if (keep == 0) now.f = 0.f, now.vs = 0.f;
        } else {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) vis[qt] = ~0u;
        }
        f32x4 s[QT][SUB];
#pragma unroll
        for (int t = 0; t < SUB; ++t) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) s[qt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const Operand k = now.template key<T>(t, j);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(k, q[qt][j], s[qt][t]);
            }
        }
        Operand p[QT][CH / 8];
        if (masked) weigh(s, now.f, now.vs, vis, true, p);
        else weigh(s, now.f, now.vs, vis, false, p);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < CH / 8; ++i) {
                const Operand v = now.template value<T>(dt, i);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) o[qt][dt] = mma(v, p[qt][i], o[qt][dt]);
            }
        now = next;
    }

    // ---- the sequence's own rows, from the last wavefront on: it has the fewest cached tiles
    bool gone[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) gone[qt] = false;
    if (has_tree) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) gone[qt] = lost[min(first_row + qt * 16 + col, R - 1) / a.group] != 0;
        const T* kx = static_cast<const T*>(a.k) + b * a.sk.seq + h * a.sk.head;
        const T* vx = static_cast<const T*>(a.v) + b * a.sv.seq + h * a.sv.head;
        for (int base = (NW - 1 - wave) * TOKENS; base < rows_of; base += NW * TOKENS) {
            unsigned vis[QT], there = 0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int i = base + g * CH + c;
                if (i < rows_of && !lost[i]) there |= 1u << c;
            }
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const int node = min(first_row + qt * 16 + col, R - 1) / a.group;
                vis[qt] = gone[qt] ? 0u : seen[node * WORDS + (base + g * CH) / 32] >> (g * CH) % 32 & there;
            }
            f32x4 s[QT][SUB];
#pragma unroll
            for (int t = 0; t < SUB; ++t) {
                const int i = min(base + col / 4 * CH + 4 * t + col % 4, rows_of - 1);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) s[qt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < STEPS; ++j) {
                    const Operand k = load8(kx + i * a.sk.row + Tokens::element(j, g), a.wide);
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) s[qt][t] = mma(k, q[qt][j], s[qt][t]);
                }
            }
            Operand p[QT][CH / 8];
            weigh(s, a.scale, 1.f, vis, true, p);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < CH / 8; ++i) {
                    Operand v, odd;
                    bool any_odd = false;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const int j = base + g * CH + i * 8 + c;
                        float x = there >> (8 * i + c) & 1 ? (float)vx[j * a.sv.row + dt * 16 + col] : 0.f;
                        const bool fine = fabsf(x) < __builtin_huge_valf();
                        any_odd |= !fine;
                        set(odd, c, fine ? 0.f : 1.f);
                        set(v, c, fine ? x : 0.f);
                    }
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt) o[qt][dt] = mma(v, p[qt][i], o[qt][dt]);
                    if (__any(any_odd)) {
                        // A value that is not finite may touch the rows that see it alone, and 0 * NaN is NaN: such values are taken
                        // out, and the rows that see one become NaN.
#pragma unroll
                        for (int qt = 0; qt < QT; ++qt) {
                            Operand sees;
#pragma unroll
                            for (int c = 0; c < 8; ++c) set(sees, c, vis[qt] >> (8 * i + c) & 1 ? 1.f : 0.f);
                            const f32x4 hit = mma(odd, sees, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (hit[r] > 0.f) o[qt][dt][r] = __builtin_nanf("");
                        }
                    }
                }
        }
    }

    // ---- join of the four wavefronts
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        l[qt] = over_groups_sum(l[qt]);
        if (too_long && has_tree) l[qt] = __builtin_nanf("");
        // a row that is not there: no weight, and none of other parts' either
        if (gone[qt]) m[qt] = __builtin_huge_valf(), l[qt] = 0.f;
        if (g == 0) {
            wave_m[wave][qt * 16 + col] = m[qt];
            wave_l[wave][qt * 16 + col] = l[qt];
        }
    }
    __syncthreads();      // and nobody reads the ancestors any more
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int i = qt * 16 + col;
        const float top = fmaxf(fmaxf(wave_m[0][i], wave_m[1][i]), fmaxf(wave_m[2][i], wave_m[3][i]));
        const float by = gone[qt] ? 0.f : m[qt] == top ? 1.f : __builtin_amdgcn_exp2f(m[qt] - top);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const f32x4 x = gone[qt] ? f32x4{0.f, 0.f, 0.f, 0.f} : o[qt][dt] * by;
            *reinterpret_cast<f32x4*>(&shared[wave * RED + col * (D + 4) + dt * 16 + g * 4]) = x;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * (D / 4); e += NT) {
            const int rr = e / (D / 4), d = e % (D / 4) * 4, row = first_row + qt * 16 + rr;
            if (row >= R) continue;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            float all = 0.f, high = neg_inf_f();
#pragma unroll
            for (int w = 0; w < NW; ++w) high = fmaxf(high, wave_m[w][qt * 16 + rr]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                sum += *reinterpret_cast<const f32x4*>(&shared[w * RED + rr * (D + 4) + d]);
                const float mw = wave_m[w][qt * 16 + rr];
                all += wave_l[w][qt * 16 + rr] * (mw == high ? 1.f : __builtin_amdgcn_exp2f(mw - high));
            }
            if (a.splits == 1) {
                const int node = row / a.group, head = h * a.group + row % a.group;
                T* out = static_cast<T*>(a.out) + (((int64_t)b * rows_of + node) * a.q_heads + head) * D + d;
                const float per_all = 1.f / all;
#pragma unroll
                for (int j = 0; j < 4; ++j) out[j] = (T)(all == 0.f ? 0.f : sum[j] * per_all);
            } else {
                const int64_t rows_all = (int64_t)a.B * heads * R, at = split * rows_all + (int64_t)bh * R + row;
                *reinterpret_cast<f32x4*>(a.part + at * D + d) = sum;
                if (d == 0) {
                    a.part[a.splits * rows_all * D + at] = high;
                    a.part[a.splits * rows_all * (D + 1) + at] = all;
                }
            }
        }
        __syncthreads();
    }
}

// The parts of a sequence's rows joined: D / 4 threads to a row.
template <typename T>
__global__ __launch_bounds__(NT) void attend_join_kernel(AttendArgs a) {
    const int D = a.cache.D, per_row = D / 4, rows_of = a.M + 1, R = rows_of * a.group, heads = a.cache.heads;
    const int64_t rows_all = (int64_t)a.B * heads * R, at = (int64_t)blockIdx.x * NT + threadIdx.x, row = at / per_row;
    if (row >= rows_all) return;
    const int d = (int)(at % per_row) * 4;
    const float *pm = a.part + a.splits * rows_all * D, *pl = pm + a.splits * rows_all;
    float high = neg_inf_f();
    for (int s = 0; s < a.splits; ++s) high = fmaxf(high, pm[s * rows_all + row]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float all = 0.f;
    bool gone = false;
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const float ms = pm[s * rows_all + row], ls = pl[s * rows_all + row], by = ms == high ? 1.f : __builtin_amdgcn_exp2f(ms - high);
        gone |= ms == __builtin_huge_valf() && ls == 0.f;
        all += by * ls;
        sum += by * *reinterpret_cast<const f32x4*>(a.part + (s * rows_all + row) * D + d);
    }
    const int r = (int)(row % R), bh = (int)(row / R), node = r / a.group, head = bh % heads * a.group + r % a.group;
    T* out = static_cast<T*>(a.out) + (((int64_t)(bh / heads) * rows_of + node) * a.q_heads + head) * D + d;
    const float per_all = 1.f / all;
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = (T)(gone || all == 0.f ? 0.f : sum[j] * per_all);
}

AttendPlan plan_attend(int dtype, int B, int M, int q_heads, const lantern_cache& c, int width) {
    AttendPlan p;
    const int64_t R = (int64_t)(M + 1) * (q_heads / c.heads);
    // fp32 operands take twice the registers: two tiles of rows
    const int most = dtype == LANTERN_F32 ? 2 : 4;
    p.query_tiles = R <= 16 ? 1 : R <= 32 || most == 2 ? 2 : 4;
    p.row_tiles = (int)((R + 16 * p.query_tiles - 1) / (16 * p.query_tiles));
    // Workgroups for twice the 256 CUs, as long as each wavefront has two tiles of tokens.
    const int64_t groups = (int64_t)B * c.heads * p.row_tiles, tokens = (int64_t)width * c.page_tokens;
    const int64_t tile = c.dtype == LANTERN_E4M3 ? 64 : 32;
    const int64_t useful = std::max<int64_t>(1, tokens / (tile * NW * 2));
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({64, useful, 512 / std::max<int64_t>(1, groups)}));
    p.workspace = p.splits == 1 ? 0 : (size_t)p.splits * B * c.heads * R * (c.D + 2) * sizeof(float);
    return p;
}

template <typename T, bool EIGHT, int D, int QT>
static hipError_t launch(const AttendArgs& a, hipStream_t stream) {
    const int64_t parts = (int64_t)a.B * a.cache.heads * a.splits;
    const int blocks = (int)((parts + 7) / 8 * 8 * a.row_tiles);
    hipLaunchKernelGGL((attend_trees_kernel<T, EIGHT, D, QT>), dim3(blocks), dim3(NT), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t threads = (int64_t)a.B * a.q_heads * (a.M + 1) * (D / 4);
    hipLaunchKernelGGL((attend_join_kernel<T>), dim3((unsigned)((threads + NT - 1) / NT)), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

template <typename T, bool EIGHT, int D>
static hipError_t launch_tiles(const AttendArgs& a, int query_tiles, hipStream_t stream) {
    if (query_tiles == 1) return launch<T, EIGHT, D, 1>(a, stream);
    if (query_tiles == 2) return launch<T, EIGHT, D, 2>(a, stream);
    if constexpr (sizeof(T) == 2) return launch<T, EIGHT, D, 4>(a, stream);
    return hipErrorInvalidValue;
}

template <typename T, bool EIGHT>
static hipError_t launch_width(const AttendArgs& a, int query_tiles, hipStream_t stream) {
    switch (a.cache.D) {
        case 32: return launch_tiles<T, EIGHT, 32>(a, query_tiles, stream);
        case 64: return launch_tiles<T, EIGHT, 64>(a, query_tiles, stream);
        case 96: return launch_tiles<T, EIGHT, 96>(a, query_tiles, stream);
        case 128: return launch_tiles<T, EIGHT, 128>(a, query_tiles, stream);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_attend_trees(const AttendArgs& a, int dtype, int query_tiles, hipStream_t stream) {
    const bool eight = a.cache.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? launch_width<float, true>(a, query_tiles, stream) : launch_width<float, false>(a, query_tiles, stream);
    return eight ? launch_width<bf16, true>(a, query_tiles, stream) : launch_width<bf16, false>(a, query_tiles, stream);
}

hipError_t prepare_attend(int, const lantern_cache&) {
    hipFuncAttributes attr;   // the runtime loads all of a file's kernels together
    return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&attend_join_kernel<bf16>));
}

}  // namespace lantern
