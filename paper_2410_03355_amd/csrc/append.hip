// Appending rows of keys and values to a paged cache (lantern_append_cache), the keys' rotation applied on the way.
//
// Two kernels.  Few rows (the accepted candidates of a step, single tokens): a wavefront to a page, head and side, keys or values, in
// registers.  Whole pages (prompts): a workgroup to a page, side and some heads; a key's angles are formed once for all of these.
// Keys go out as rows [token][D], from registers; values turned over, [D][token], which is how the matrix instructions of attend.hip
// take them: through LDS.
//
// Measured: accepted paths of 64 trees, 20 heads of 64, 8 bits 8.7 us, bound by loads one after the other (path, page, row, old scale); 16
// prompts of about 1000 tokens, 8 heads of 128, 8 bits 39 us, 2.3 TB/s; with one kernel for both 18 and 66.  The latter are bound by waiting: wavefronts
// wait for 54 % of their time, on loads and for each other, and the vector units work 36 % of it, since 174 registers (a thread's rows of a page, keys
// and values in one kernel) leave two workgroups to a CU.  On pages of 128 tokens (256 and 98 more, one workgroup to a CU) the same takes 80 us.
//
// 8-bit pages: value = code * scale.  The scale is the smallest power of two s with largest <= 448 s.  A code has four
// significant bits under any scale, so nothing is lost against largest / 448 but part of one of e4m3's fifteen binades;
// and when later rows raise a page's scale, the codes it has are divided by a power of two, which is exact but for those that
// fall among the subnormal ones.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cache_args.h"
#include "device_utils.h"
#include "lds_limit.h"
#include "rotation.h"

namespace lantern {

constexpr float LARGEST = 448.f;     // of e4m3
constexpr unsigned NAN_CODE = 0x7F;

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < __builtin_huge_valf(); }

// The smallest power of two s >= 2^-126 with largest <= 448 s (448 = 0.875 * 2^9).
__device__ __forceinline__ float scale_for(float largest) {
    int e;
    const float m = frexpf(largest, &e);
    return largest > 0.f ? ldexpf(1.f, max(-126, e - 9 + (m > 0.875f))) : ldexpf(1.f, -126);
}

struct Quantiser {
    float scale, per;      // per: 1 / scale, exact, or 0 where the scale is no power of two (a cache filled by others)
    bool odd;              // not all values are finite
    __device__ __forceinline__ Quantiser(float s, bool o) : scale(s), per((__float_as_uint(s) & 0x7FFFFFu) ? 0.f : 1.f / s), odd(o) {}
    // Four codes.  Finite values are within 448 scales, so they need no limit; what is not finite becomes NaN, the 8-bit type having no
    // infinity.
    __device__ __forceinline__ unsigned codes(const float (&x)[4]) const {
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = per != 0.f ? x[i] * per : x[i] / scale;
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
        unsigned r = (unsigned)w;
        if (odd)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!finite(x[i])) r = (r & ~(0xFFu << 8 * i)) | NAN_CODE << 8 * i;
        return r;
    }
};

// A code under a new scale: `by` = old scale / new scale.
__device__ __forceinline__ uint8_t recode(uint8_t c, float by) {
    const float x = __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * by;
    return x == x ? (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(x, -LARGEST), LARGEST), 0.f, 0, false) & 0xFF)
                  : (uint8_t)NAN_CODE;
}

// What a sequence appends and where.  Every wavefront of a sequence checks all of it and comes to the same end: the sequence is written whole
// or not at all.
struct Where {
    int start, n, page, slot, rows, first;   // rows first .. of the appended n go to the page's slots from `slot` on; rows 0: nothing here
    int64_t id;
    __device__ __forceinline__ Where(const AppendArgs& a, int b, int nth_page, bool reports) : start(a.lengths[b]), rows(0) {
        const int lane = threadIdx.x & (WAVE - 1);
        if (start < 0) {                       // no sequence here
            if (reports) a.out_lengths[b] = start;
            return;
        }
        const int most = a.T - (a.path ? 1 : 0), told = a.count ? a.count[b] : most;
        bool bad = told < 0 || told > most;      // a count may be anything: looked at before it is added to
        n = bad ? 0 : told + a.T - most;
        bad |= (int64_t)start + n > (int64_t)a.width << a.page_shift;
        if (!bad && n > 0) {
            const int first_page = start >> a.page_shift, pages = ((start + n - 1) >> a.page_shift) - first_page + 1;
            for (int i = lane; i < pages; i += WAVE) {
                const int p = a.table[(int64_t)b * a.width + first_page + i];
                bad |= p < 0 || p >= a.cache.pages;
            }
            if (a.path)
                for (int i = lane; i < told; i += WAVE) {
                    const int node = a.path[(int64_t)b * (a.T - 1) + i];
                    bad |= node < 0 || node >= a.T - 1;
                }
        }
        bad = __any(bad);
        if (reports) a.out_lengths[b] = bad ? -2 : start + n;
        const int w = (start >> a.page_shift) + nth_page;
        if (bad || (int64_t)w << a.page_shift >= (int64_t)start + n) return;
        const int lo = max(start, w << a.page_shift), hi = (int)min((int64_t)start + n, (int64_t)(w + 1) << a.page_shift);
        rows = max(0, hi - lo);
        slot = lo - (w << a.page_shift);
        first = lo - start;
        id = rows > 0 ? a.table[(int64_t)b * a.width + w] : 0;
    }
    __device__ __forceinline__ int row_of(const AppendArgs& a, int b, int r) const {
        const int nth = first + r;
        return a.path && nth > 0 ? a.path[(int64_t)b * (a.T - 1) + nth - 1] + 1 : nth;
    }
};

// The largest magnitude as bits, which order like it; from ODD on a value is not finite.
constexpr int ODD = 0x7F800000;
__device__ __forceinline__ int largest_of(const float (&p)[4], const float (&q)[4], int largest) {
#pragma unroll
    for (int j = 0; j < 4; ++j) largest = max(largest, max(__float_as_int(p[j]) & 0x7FFFFFFF, __float_as_int(q[j]) & 0x7FFFFFFF));
    return largest;
}
// The same of the finite ones.
__device__ __forceinline__ int largest_finite(const float (&p)[4], const float (&q)[4], int largest) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int a = __float_as_int(p[j]) & 0x7FFFFFFF, b = __float_as_int(q[j]) & 0x7FFFFFFF;
        largest = max(largest, max(a < ODD ? a : 0, b < ODD ? b : 0));
    }
    return largest;
}
__device__ __forceinline__ int wave_max_i(int x) { return __builtin_amdgcn_readlane(wave_scan_i<OpMax>(x, 0), WAVE - 1); }

// A unit's values into a row of keys.  RUNS: both its runs are four values in a row at multiples of four.
template <bool EIGHT, typename U>
__device__ __forceinline__ void write_key(void* row, const U& unit, const Quantiser& to, bool runs, const float (&p)[4], const float (&q)[4]) {
    if constexpr (EIGHT) {
        uint8_t* out = static_cast<uint8_t*>(row);
        if (runs) {
            const float a[4] = {p[0], unit.inter ? q[0] : p[1], unit.inter ? p[1] : p[2], unit.inter ? q[1] : p[3]};
            const float b[4] = {unit.inter ? p[2] : q[0], unit.inter ? q[2] : q[1], unit.inter ? p[3] : q[2], q[3]};
            *reinterpret_cast<unsigned*>(out + unit.o1) = to.codes(a);
            *reinterpret_cast<unsigned*>(out + unit.o2) = to.codes(b);
        } else {
            const unsigned a = to.codes(p), b = to.codes(q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j < unit.n1) out[unit.inter ? unit.o1 + 2 * j : unit.o1 + j] = (uint8_t)(a >> 8 * j);
                if (j < unit.n2) out[unit.inter ? unit.o1 + 2 * j + 1 : unit.o2 + j] = (uint8_t)(b >> 8 * j);
            }
        }
    } else {
        if (runs) {
            RotationUnit<float, 4, true> whole;
            whole.inter = unit.inter;
            whole.o1 = unit.o1, whole.o2 = unit.o2, whole.n1 = whole.n2 = 4;
            whole.store(static_cast<bf16*>(row), p, q);
        } else {
            RotationUnit<float, 4, false> some;
            some.inter = unit.inter;
            some.o1 = unit.o1, some.o2 = unit.o2, some.n1 = unit.n1, some.n2 = unit.n2;
            some.store(static_cast<bf16*>(row), p, q);
        }
    }
}

// The new scale of a page that holds `slot` tokens already; where it grows, their codes are rounded to it, by the threads of a team.
__device__ __forceinline__ float rescale(uint8_t* out, float was, int largest, int slot, int D, int page_shift, bool values, int member, int team) {
    const float need = scale_for(__int_as_float(largest)), scale = slot ? fmaxf(was, need) : need;
    if (slot && !(was == scale)) {
        const float by = was / scale;
        if (values)
            for (int i = member; i < D * slot; i += team) {
                uint8_t* c = out + ((int64_t)(i / slot) << page_shift) + i % slot;
                *c = recode(*c, by);
            }
        else
            for (int i = member; i < D * slot; i += team) out[i] = recode(out[i], by);
    }
    return scale;
}

// ---- few rows

template <typename T, bool EIGHT>
__global__ __launch_bounds__(NT) void append_rows_kernel(AppendArgs a) {
    const int lane = threadIdx.x & (WAVE - 1), heads = a.cache.heads, D = a.cache.D;
    const int item = blockIdx.x * NW + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), place = item / heads, h = item % heads;
    if (place >= 2 * a.B * a.touched) return;
    const bool values = place & 1;
    const int b = (place >> 1) / a.touched, nth_page = (place >> 1) % a.touched;
    const Where w(a, b, nth_page, nth_page == 0 && h == 0 && !values && lane == 0);
    if (w.rows == 0) return;
    const Strided s = values ? a.sv : a.sk;
    const T* const x = static_cast<const T*>(values ? a.v : a.k) + b * s.seq + h * s.head;
    const int pairs = values ? 0 : a.pairs, units = rotation_units<4>(pairs, D);
    const bool wide = values ? a.wide_v : a.wide_k;
    typedef RotationUnit<T, 4, false> Unit;
    auto bring = [&](int i, Unit& unit, int* r, float (&p)[4], float (&q)[4]) {
        *r = i / units;
        const int u = i % units, row = w.row_of(a, b, *r);
        unit.place(u, pairs, D, a.rot.interleaved != 0);
        if (wide) {
            RotationUnit<T, 4, true> whole;
            whole.inter = unit.inter;
            whole.o1 = unit.o1, whole.o2 = unit.o2, whole.n1 = whole.n2 = 4;
            whole.load(x + row * s.row, p, q);
        } else {
            unit.load(x + row * s.row, p, q);
        }
        if (unit.turned) {
            unit.angles(a.rot, a.rot.positions + ((int64_t)b * a.T + row) * a.rot.axes, u, false);
            unit.turn(p, q);
        }
    };
    const int all = w.rows * units, block_bytes = D << a.page_shift;
    const int64_t block = w.id * heads + h;
    Unit unit;
    int r = 0;
    float p[4], q[4], scale = 1.f;
    bool odd = false;
    if (lane < all) bring(lane, unit, &r, p, q);
    uint8_t* const bytes = static_cast<uint8_t*>(values ? a.cache.v : a.cache.k) + block * block_bytes * (EIGHT ? 1 : 2);
    if constexpr (EIGHT) {
        float* const scales = values ? a.cache.v_scale : a.cache.k_scale;
        int largest = lane < all ? largest_of(p, q, 0) : 0;
        for (int i = lane + WAVE; i < all; i += WAVE) {      // more than a wavefront holds: turned again for writing
            Unit other;
            int of;
            float c[4], d[4];
            bring(i, other, &of, c, d);
            largest = largest_of(c, d, largest);
        }
        largest = wave_max_i(largest);
        odd = largest >= ODD;
        if (odd) {
            largest = 0;
            for (int i = lane; i < all; i += WAVE) {
                Unit other;
                int of;
                float c[4], d[4];
                bring(i, other, &of, c, d);
                largest = largest_finite(c, d, largest);
            }
            largest = wave_max_i(largest);
        }
        const float was = w.slot ? scales[block] : 0.f;
        scale = rescale(bytes, was, largest, w.slot, D, a.page_shift, values, lane, WAVE);
        if (lane == 0) scales[block] = scale;
    }
    const Quantiser to(scale, odd);
    for (int i = lane; i < all; i += WAVE) {
        if (i > lane) bring(i, unit, &r, p, q);
        const int slot = w.slot + r;
        if (!values) {
            write_key<EIGHT>(bytes + (int64_t)slot * D * (EIGHT ? 1 : 2), unit, to, wide && unit.n1 == 4 && unit.n2 == 4, p, q);
            continue;
        }
        const unsigned cp = EIGHT ? to.codes(p) : 0u, cq = EIGHT ? to.codes(q) : 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {      // D is a multiple of 8: units of values are whole
            const int64_t at = ((int64_t)(unit.o1 + j) << a.page_shift) + slot, next = at + ((int64_t)4 << a.page_shift);
            if constexpr (EIGHT) {
                bytes[at] = (uint8_t)(cp >> 8 * j);
                bytes[next] = (uint8_t)(cq >> 8 * j);
            } else {
                reinterpret_cast<bf16*>(bytes)[at] = (bf16)p[j];
                reinterpret_cast<bf16*>(bytes)[next] = (bf16)q[j];
            }
        }
    }
}

// ---- whole pages, of rows one after the other (no path).  The rows of the next head are asked for before this one's are worked on.

__device__ __forceinline__ int block_max(int x, int* waves) {
    x = wave_max_i(x);
    __syncthreads();      // what was there has been read
    if ((threadIdx.x & (WAVE - 1)) == 0) waves[threadIdx.x / WAVE] = x;
    __syncthreads();
    return max(max(waves[0], waves[1]), max(waves[2], waves[3]));
}

// A thread has one unit of EACH rows at most, NT / units apart.
template <typename T, bool EIGHT, int EACH, bool WIDE>
__device__ __forceinline__ void append_keys(const AppendArgs& a, const Where& w, int b, int h, int last, int* waves) {
    const int D = a.cache.D, units = rotation_units<4>(a.pairs, D), at_once = NT / units;
    const int u = threadIdx.x % units, mine = threadIdx.x / units;      // threads from at_once * units on have nothing
    RotationUnit<T, 4, WIDE> unit;
    unit.place(u, a.pairs, D, a.rot.interleaved != 0);
    float c[EACH][4], s[EACH][4];
    if (unit.turned) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int row = w.first + min(mine + e * at_once, w.rows - 1);
            unit.angles(a.rot, a.rot.positions + ((int64_t)b * a.T + row) * a.rot.axes, u, false);
#pragma unroll
            for (int j = 0; j < 4; ++j) c[e][j] = unit.c[j], s[e][j] = unit.s[j];
        }
    }
    T p[EACH][4], q[EACH][4];
    auto ask = [&](int head) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int64_t row = w.first + min(mine + e * at_once, w.rows - 1);
            unit.load_as(static_cast<const T*>(a.k) + b * a.sk.seq + head * a.sk.head + row * a.sk.row, p[e], q[e]);
        }
    };
    ask(h);
    for (; h < last; ++h) {
        const int64_t block = w.id * a.cache.heads + h;
        float x[EACH][4], y[EACH][4], scale = 1.f;
        int largest = 0;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[e][j] = (float)p[e][j], y[e][j] = (float)q[e][j];
                unit.c[j] = c[e][j], unit.s[j] = s[e][j];
            }
            unit.turn(x[e], y[e]);
            largest = largest_of(x[e], y[e], largest);
        }
        ask(min(h + 1, last - 1));
        uint8_t* const bytes = static_cast<uint8_t*>(a.cache.k) + (block << a.page_shift) * D * (EIGHT ? 1 : 2);
        if constexpr (EIGHT) {
            const float was = w.slot ? a.cache.k_scale[block] : 0.f;
            largest = block_max(largest, waves);      // and every thread has read the scale
            odd = largest >= ODD;
            if (odd) {
                largest = 0;
#pragma unroll
                for (int e = 0; e < EACH; ++e) largest = largest_finite(x[e], y[e], largest);
                largest = block_max(largest, waves);
            }
            scale = rescale(bytes, was, largest, w.slot, D, a.page_shift, false, threadIdx.x, NT);
            if (threadIdx.x == 0) a.cache.k_scale[block] = scale;
        }
        const Quantiser to(scale, odd);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int r = mine + e * at_once;
            if (mine < at_once && r < w.rows)
                write_key<EIGHT>(bytes + (int64_t)(w.slot + r) * D * (EIGHT ? 1 : 2), unit, to, WIDE, x[e], y[e]);
        }
    }
}

template <typename T, bool EIGHT>
__device__ __forceinline__ void append_values(const AppendArgs& a, const Where& w, int b, int h, int last, int* waves, T* lds) {
    typedef typename Vec<T, 4>::type Four;
    constexpr int MOST = 4;      // pieces of 8 elements that a thread asks for ahead: all of a page's up to 64 tokens of 128
    const int D = a.cache.D, per_row = D / 8, all = w.rows * per_row, stride = D + 4;
    Four p[MOST], q[MOST];
    auto load = [&](int head, int i, Four& x, Four& y) {
        const T* const from = static_cast<const T*>(a.v) + b * a.sv.seq + head * a.sv.head + (int64_t)(w.first + i / per_row) * a.sv.row + i % per_row * 8;
        if (a.wide_v) {
            x = *reinterpret_cast<const Four*>(from);
            y = *reinterpret_cast<const Four*>(from + 4);
        } else {
            x = Four{from[0], from[1], from[2], from[3]};
            y = Four{from[4], from[5], from[6], from[7]};
        }
    };
    auto ask = [&](int head) {
#pragma unroll
        for (int e = 0; e < MOST; ++e) load(head, min((int)threadIdx.x + e * NT, all - 1), p[e], q[e]);
    };
    ask(h);
    for (; h < last; ++h) {
        const int64_t block = w.id * a.cache.heads + h;
        uint8_t* const bytes = static_cast<uint8_t*>(a.cache.v) + (block << a.page_shift) * D * (EIGHT ? 1 : 2);
        const float was = EIGHT && w.slot ? a.cache.v_scale[block] : 0.f;
        float scale = 1.f;
        int largest = 0;
        bool odd = false;
        __syncthreads();      // the head before has been written
        auto put = [&](int i, const Four& x, const Four& y) {
            T* const to = lds + i / per_row * stride + i % per_row * 8;
            *reinterpret_cast<Four*>(to) = x;
            *reinterpret_cast<Four*>(to + 4) = y;
            if constexpr (EIGHT) {
                const float c[4] = {(float)x[0], (float)x[1], (float)x[2], (float)x[3]}, e[4] = {(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
                largest = largest_of(c, e, largest);
            }
        };
#pragma unroll
        for (int e = 0; e < MOST; ++e) put(min((int)threadIdx.x + e * NT, all - 1), p[e], q[e]);
        for (int i = threadIdx.x + MOST * NT; i < all; i += NT) {
            Four x, y;
            load(h, i, x, y);
            put(i, x, y);
        }
        ask(min(h + 1, last - 1));
        if constexpr (EIGHT) {
            largest = block_max(largest, waves);      // and the rows are there
            odd = largest >= ODD;
            if (odd) {
                largest = 0;
                for (int i = threadIdx.x; i < all; i += NT) {
                    const T* const x = lds + i / per_row * stride + i % per_row * 8;
                    const float c[4] = {(float)x[0], (float)x[1], (float)x[2], (float)x[3]}, e[4] = {(float)x[4], (float)x[5], (float)x[6], (float)x[7]};
                    largest = largest_finite(c, e, largest);
                }
                largest = block_max(largest, waves);
            }
            scale = rescale(bytes, was, largest, w.slot, D, a.page_shift, true, threadIdx.x, NT);
            if (threadIdx.x == 0) a.cache.v_scale[block] = scale;
        } else {
            __syncthreads();
        }
        const Quantiser to(scale, odd);
        // 16 bytes of an element at a time; a piece that is not all new is written token by token
        constexpr int AT_ONCE = EIGHT ? 16 : 8;
        const int g0 = w.slot / AT_ONCE, groups = (w.slot + w.rows + AT_ONCE - 1) / AT_ONCE - g0;
        for (int i = threadIdx.x; i < D * groups; i += NT) {
            const int d = i / groups, at = (g0 + i % groups) * AT_ONCE;
            u32x4 out;
            const bool whole = at >= w.slot && at + AT_ONCE <= w.slot + w.rows;
            float v[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) v[j] = (float)lds[min(max(at + j - w.slot, 0), w.rows - 1) * stride + d];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (EIGHT) {
                    const float four[4] = {v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
                    out[k] = to.codes(four);
                } else {
                    out[k] = __builtin_bit_cast(unsigned, bf16x2{(bf16)v[2 * k], (bf16)v[2 * k + 1]});
                }
            }
            const int64_t place = ((int64_t)d << a.page_shift) + at;
            if (whole) {
                *reinterpret_cast<u32x4*>(bytes + place * (EIGHT ? 1 : 2)) = out;
            } else {
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    if (at + j < w.slot || at + j >= w.slot + w.rows) continue;
                    if constexpr (EIGHT) bytes[place + j] = (uint8_t)(out[j / 4] >> 8 * (j % 4));
                    else reinterpret_cast<uint16_t*>(bytes)[place + j] = (uint16_t)(out[j / 2] >> 16 * (j % 2));
                }
            }
        }
    }
}

template <typename T, bool EIGHT, int EACH>
__global__ __launch_bounds__(NT) void append_pages_kernel(AppendArgs a, int heads_each) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ int waves[NW];
    const int b = blockIdx.x / a.touched, nth_page = blockIdx.x % a.touched, h = blockIdx.y * heads_each, last = min(a.cache.heads, h + heads_each);
    const bool values = blockIdx.z != 0;
    const Where w(a, b, nth_page, nth_page == 0 && h == 0 && !values && threadIdx.x == 0);
    if (w.rows == 0) return;
    if (values) append_values<T, EIGHT>(a, w, b, h, last, waves, reinterpret_cast<T*>(lds));
    else if (a.wide_k) append_keys<T, EIGHT, EACH, true>(a, w, b, h, last, waves);
    else append_keys<T, EIGHT, EACH, false>(a, w, b, h, last, waves);
}

template <typename T>
static size_t lds_bytes(const lantern_cache& c) { return sizeof(T) * c.page_tokens * (c.D + 4); }

template <typename T, bool EIGHT, int EACH>
static hipError_t launch_pages(const AppendArgs& a, hipStream_t stream) {
    if ((int64_t)a.B * a.touched > MOST_GROUPS) return hipErrorInvalidConfiguration;
    const size_t lds = lds_bytes<T>(a.cache);
    const hipError_t e = allow_lds<append_pages_kernel<T, EIGHT, EACH>>(lds);
    if (e != hipSuccess) return e;
    // Several heads to a workgroup, for whose keys the angles are formed once, while there are four workgroups and more to a CU (of which the forms
    // for pages of 64 tokens of 128 and for 128 tokens have two and one resident at once).
    const int64_t places = 2 * (int64_t)a.B * a.touched;
    const int each = (int)std::max<int64_t>(1, std::min<int64_t>(a.cache.heads, places * a.cache.heads / 1024));
    hipLaunchKernelGGL((append_pages_kernel<T, EIGHT, EACH>), dim3(a.B * a.touched, (a.cache.heads + each - 1) / each, 2), dim3(NT), lds, stream, a,
                       each);
    return hipGetLastError();
}

template <typename T, bool EIGHT>
static hipError_t launch(const AppendArgs& a, hipStream_t stream) {
    const int units = std::max(rotation_units<4>(a.pairs, a.cache.D), a.cache.D / 8);
    // A wavefront holds 64 units: up to four times that in rows, and the accepted candidates of a tree, which are few
    if (a.path || (int64_t)a.T * units <= 4 * WAVE) {
        const int64_t items = 2 * (int64_t)a.B * a.touched * a.cache.heads;
        if (items > MOST_GROUPS * NW) return hipErrorInvalidConfiguration;
        hipLaunchKernelGGL((append_rows_kernel<T, EIGHT>), dim3((unsigned)((items + NW - 1) / NW)), dim3(NT), 0, stream, a);
        return hipGetLastError();
    }
    const int rows = NT / rotation_units<4>(a.pairs, a.cache.D), each = (a.cache.page_tokens + rows - 1) / rows;      // 9 at most: pages of 128, 17 units
    if (each <= 2) return launch_pages<T, EIGHT, 2>(a, stream);
    if (each <= 4) return launch_pages<T, EIGHT, 4>(a, stream);
    return launch_pages<T, EIGHT, 9>(a, stream);
}

hipError_t launch_append_cache(const AppendArgs& a, int dtype, hipStream_t stream) {
    const bool eight = a.cache.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
    return eight ? launch<bf16, true>(a, stream) : launch<bf16, false>(a, stream);
}

template <typename T, bool EIGHT>
static hipError_t prepare(const lantern_cache& c) {
    hipFuncAttributes attr;   // the runtime loads all of a file's kernels together
    hipError_t e = hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&append_rows_kernel<T, EIGHT>));
    const size_t lds = lds_bytes<T>(c);
    if (e == hipSuccess) e = allow_lds<append_pages_kernel<T, EIGHT, 2>>(lds);
    if (e == hipSuccess) e = allow_lds<append_pages_kernel<T, EIGHT, 4>>(lds);
    if (e == hipSuccess) e = allow_lds<append_pages_kernel<T, EIGHT, 9>>(lds);
    return e;
}

hipError_t prepare_append(int dtype, const lantern_cache& c) {
    const bool eight = c.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? prepare<float, true>(c) : prepare<float, false>(c);
    return eight ? prepare<bf16, true>(c) : prepare<bf16, false>(c);
}

}  // namespace lantern
