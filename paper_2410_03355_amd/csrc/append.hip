// Appending rows of keys and values to a paged cache (lantern_append_cache), the keys' rotation applied on the way.
//
// One workgroup per page that a sequence's rows reach, head, and keys or values.  It brings the rows to LDS in fp32
// (rotated there: a key is rounded once, to the cache's type), finds their largest magnitude, and writes them: keys as rows
// [token][D], values turned over, [D][token], which is how the matrix instructions of attend.hip take them.
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
    __device__ __forceinline__ explicit Quantiser(float s) : scale(s), per((__float_as_uint(s) & 0x7FFFFFu) ? 0.f : 1.f / s) {}
    __device__ __forceinline__ float shrink(float x) const {
        const float y = per != 0.f ? x * per : x / scale;
        return fminf(fmaxf(y, -LARGEST), LARGEST);
    }
    // Four codes; what is not finite becomes NaN, the 8-bit type having no infinity.
    __device__ __forceinline__ unsigned codes(const float x[4]) const {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(shrink(x[0]), shrink(x[1]), 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(shrink(x[2]), shrink(x[3]), w, true);
        unsigned r = (unsigned)w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (!finite(x[i])) r = (r & ~(0xFFu << 8 * i)) | NAN_CODE << 8 * i;
        return r;
    }
    __device__ __forceinline__ uint8_t code(float x) const {
        const float four[4] = {x, 0.f, 0.f, 0.f};
        return (uint8_t)codes(four);
    }
};

// A code under a new scale: `by` = old scale / new scale.
__device__ __forceinline__ uint8_t recode(uint8_t c, float by) {
    const float x = __builtin_amdgcn_cvt_f32_fp8((int)c, 0) * by;
    return x == x ? (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(x, -LARGEST), LARGEST), 0.f, 0, false) & 0xFF)
                  : (uint8_t)NAN_CODE;
}

// Rows of the page to LDS [rows][D + 1] in fp32; returns the largest finite magnitude this thread has seen.
template <typename T, bool WIDE>
__device__ __forceinline__ float bring(const AppendArgs& a, const T* x, int64_t row_stride, int b, int first, int rows, int pairs,
                                       float* lds) {
    const int D = a.cache.D, units = rotation_units<4>(pairs, D);
    float largest = 0.f;
    for (int i = threadIdx.x; i < rows * units; i += NT) {
        const int r = i / units, u = i % units, nth = first + r;
        const int row = a.path && nth > 0 ? a.path[(int64_t)b * (a.T - 1) + nth - 1] + 1 : nth;
        RotationUnit<T, 4, WIDE> unit;
        float p[4], q[4];
        unit.place(u, pairs, D, a.rot.interleaved != 0);
        unit.load(x + row * row_stride, p, q);
        if (unit.turned) {
            unit.angles(a.rot, a.rot.positions + ((int64_t)b * a.T + row) * a.rot.axes, u, false);
            unit.turn(p, q);
        }
        RotationUnit<T, 4, false> plain;      // LDS rows of D + 1 floats are not aligned
        plain.place(u, pairs, D, a.rot.interleaved != 0);
        plain.store(lds + r * (D + 1), p, q);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (finite(p[j])) largest = fmaxf(largest, fabsf(p[j]));
            if (finite(q[j])) largest = fmaxf(largest, fabsf(q[j]));
        }
    }
    return largest;
}

template <typename T, bool EIGHT>
__global__ __launch_bounds__(NT) void append_cache_kernel(AppendArgs a) {
    extern __shared__ float lds[];
    __shared__ float wave_largest[NW];
    const int b = blockIdx.x / a.touched, nth_page = blockIdx.x % a.touched, h = blockIdx.y;
    const bool values = blockIdx.z != 0;
    const bool reports = nth_page == 0 && h == 0 && !values && threadIdx.x == 0;
    const int start = a.lengths[b];
    if (start < 0) {                       // no sequence here
        if (reports) a.out_lengths[b] = start;
        return;
    }
    // Every workgroup of a sequence checks all of it and comes to the same end: it is written whole or not at all.
    const int told = a.count ? a.count[b] : a.T - (a.path ? 1 : 0);
    const int n = a.path ? told + 1 : told;
    bool bad = told < 0 || n > a.T || (int64_t)start + n > (int64_t)a.width << a.page_shift;
    if (!bad && n > 0) {
        const int first_page = start >> a.page_shift, pages = ((start + n - 1) >> a.page_shift) - first_page + 1;
        for (int i = threadIdx.x; i < pages; i += NT) {
            const int id = a.table[(int64_t)b * a.width + first_page + i];
            bad |= id < 0 || id >= a.cache.pages;
        }
        if (a.path)
            for (int i = threadIdx.x; i < told; i += NT) {
                const int node = a.path[(int64_t)b * (a.T - 1) + i];
                bad |= node < 0 || node >= a.T - 1;
            }
    }
    bad = __syncthreads_or(bad);
    if (reports) a.out_lengths[b] = bad ? -2 : start + n;
    if (bad) return;
    const int w = (start >> a.page_shift) + nth_page;
    if ((int64_t)w << a.page_shift >= (int64_t)start + n) return;
    const int lo = max(start, w << a.page_shift), hi = (int)min((int64_t)start + n, (int64_t)(w + 1) << a.page_shift);
    if (lo >= hi) return;
    const int rows = hi - lo, slot = lo - (w << a.page_shift);     // slot: where they begin in the page, and how many tokens are before them
    const int D = a.cache.D, heads = a.cache.heads;
    const int64_t id = a.table[(int64_t)b * a.width + w], block = id * heads + h;

    float largest;
    if (values) {
        const T* x = static_cast<const T*>(a.v) + b * a.sv.seq + h * a.sv.head;
        largest = a.wide_v ? bring<T, true>(a, x, a.sv.row, b, lo - start, rows, 0, lds) : bring<T, false>(a, x, a.sv.row, b, lo - start, rows, 0, lds);
    } else {
        const T* x = static_cast<const T*>(a.k) + b * a.sk.seq + h * a.sk.head;
        largest = a.wide_k ? bring<T, true>(a, x, a.sk.row, b, lo - start, rows, a.pairs, lds)
                           : bring<T, false>(a, x, a.sk.row, b, lo - start, rows, a.pairs, lds);
    }
    if constexpr (EIGHT) {
        largest = wave_max(largest);
        if ((threadIdx.x & (WAVE - 1)) == 0) wave_largest[threadIdx.x / WAVE] = largest;
    }
    __syncthreads();

    if constexpr (EIGHT) {
        uint8_t* out = static_cast<uint8_t*>(values ? a.cache.v : a.cache.k) + (block << a.page_shift) * D;
        float* scales = values ? a.cache.v_scale : a.cache.k_scale;
        const float need = scale_for(fmaxf(fmaxf(wave_largest[0], wave_largest[1]), fmaxf(wave_largest[2], wave_largest[3])));
        const float was = scales[block], scale = slot ? fmaxf(was, need) : need;
        const Quantiser to(scale);
        if (slot && !(was == scale)) {
            const float by = was / scale;
            if (values)
                for (int i = threadIdx.x; i < D * slot; i += NT) {
                    uint8_t* c = out + ((int64_t)(i / slot) << a.page_shift) + i % slot;
                    *c = recode(*c, by);
                }
            else
                for (int i = threadIdx.x; i < D * slot; i += NT) out[i] = recode(out[i], by);
        }
        if (values) {
            // four tokens of a column at a time; a group that is not all new is written byte by byte
            const int g0 = slot / 4, groups = (slot + rows + 3) / 4 - g0;
            for (int i = threadIdx.x; i < D * groups; i += NT) {
                const int d = i / groups, at = (g0 + i % groups) * 4;
                uint8_t* c = out + ((int64_t)d << a.page_shift) + at;
                float x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = at + j - slot;
                    x[j] = r >= 0 && r < rows ? lds[r * (D + 1) + d] : 0.f;
                }
                const unsigned four = to.codes(x);
                if (at >= slot && at + 4 <= slot + rows)
                    *reinterpret_cast<unsigned*>(c) = four;
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at + j >= slot && at + j < slot + rows) c[j] = (uint8_t)(four >> 8 * j);
            }
        } else {
            for (int i = threadIdx.x; i < rows * (D / 4); i += NT) {
                const int r = i / (D / 4), d = i % (D / 4) * 4;
                const float x[4] = {lds[r * (D + 1) + d], lds[r * (D + 1) + d + 1], lds[r * (D + 1) + d + 2], lds[r * (D + 1) + d + 3]};
                *reinterpret_cast<unsigned*>(out + (slot + r) * D + d) = to.codes(x);
            }
        }
        __syncthreads();      // every thread has read the old scale
        if (threadIdx.x == 0) scales[block] = scale;
    } else {
        bf16* out = static_cast<bf16*>(values ? a.cache.v : a.cache.k) + (block << a.page_shift) * D;
        if (values) {
            for (int i = threadIdx.x; i < D * rows; i += NT) {
                const int d = i / rows, r = i % rows;
                out[((int64_t)d << a.page_shift) + slot + r] = (bf16)lds[r * (D + 1) + d];
            }
        } else {
            for (int i = threadIdx.x; i < rows * (D / 2); i += NT) {
                const int r = i / (D / 2), d = i % (D / 2) * 2;
                const bf16x2 two = {(bf16)lds[r * (D + 1) + d], (bf16)lds[r * (D + 1) + d + 1]};
                *reinterpret_cast<bf16x2*>(out + (slot + r) * D + d) = two;
            }
        }
    }
}

static size_t lds_bytes(const lantern_cache& c) { return sizeof(float) * c.page_tokens * (c.D + 1); }

template <typename T, bool EIGHT>
static hipError_t launch(const AppendArgs& a, hipStream_t stream) {
    const size_t lds = lds_bytes(a.cache);
    const hipError_t e = allow_lds<append_cache_kernel<T, EIGHT>>(lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((append_cache_kernel<T, EIGHT>), dim3(a.B * a.touched, a.cache.heads, 2), dim3(NT), lds, stream, a);
    return hipGetLastError();
}

hipError_t launch_append_cache(const AppendArgs& a, int dtype, hipStream_t stream) {
    const bool eight = a.cache.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
    return eight ? launch<bf16, true>(a, stream) : launch<bf16, false>(a, stream);
}

template <typename T, bool EIGHT>
static hipError_t prepare(const lantern_cache& c) {
    hipFuncAttributes attr;
    const hipError_t e = hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&append_cache_kernel<T, EIGHT>));
    return e != hipSuccess ? e : allow_lds<append_cache_kernel<T, EIGHT>>(lds_bytes(c));
}

hipError_t prepare_append(int dtype, const lantern_cache& c) {
    const bool eight = c.dtype == LANTERN_E4M3;
    if (dtype == LANTERN_F32) return eight ? prepare<float, true>(c) : prepare<float, false>(c);
    return eight ? prepare<bf16, true>(c) : prepare<bf16, false>(c);
}

}  // namespace lantern
