// Rotation of a head's pairs by positions with several axes, and the types around it.
//
// Pair j belongs to the axis whose run of pairs holds j; it is turned by phi = position on that axis * freqs[j]:
//   y1 = x1 cos phi - x2 sin phi,  y2 = x1 sin phi + x2 cos phi
// The pair is (x[2j], x[2j+1]) (interleaved) or (x[j], x[j+P]), P pairs in all; elements from 2P on stay as they are.
// The angle is formed in fp64 and so are cosine and sine, which are then rounded once: a position of 10^5 in fp32 would
// leave an error of 2^-24 * 10^5 in the angle.  They serve all heads of a token.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lantern.h"

namespace lantern {

typedef __bf16 bf16;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <typename T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N)));
};

// cos and sin of position * freq: the product in fp64, less k quarter turns (pi / 2 in two parts, the fused steps exact but for
// their last), then the Taylor sums to y^13 and y^12 with |y| <= pi / 4: their errors, y^15 / 15! and y^14 / 14!, are under 2^-40, and the
// results rounded to fp32 once.  Some 25 fp64 operations.
__device__ __forceinline__ void angle(int32_t position, float freq, float* c, float* s) {
    constexpr double QUARTERS = 0.63661977236758134308, HALF_PI = 1.5707963267948966192, HALF_PI_LOW = 6.1232339957367660359e-17;
    const double x = (double)position * (double)freq;
    const double k = rint(x * QUARTERS);
    const double y = __builtin_fma(-k, HALF_PI_LOW, __builtin_fma(-k, HALF_PI, x)), z = y * y;
    double sn = 1.0 / 6227020800.0, cs = 1.0 / 479001600.0;
    sn = __builtin_fma(sn, z, -1.0 / 39916800.0);
    sn = __builtin_fma(sn, z, 1.0 / 362880.0);
    sn = __builtin_fma(sn, z, -1.0 / 5040.0);
    sn = __builtin_fma(sn, z, 1.0 / 120.0);
    sn = __builtin_fma(sn, z, -1.0 / 6.0);
    sn = __builtin_fma(sn * z, y, y);
    cs = __builtin_fma(cs, z, -1.0 / 3628800.0);
    cs = __builtin_fma(cs, z, 1.0 / 40320.0);
    cs = __builtin_fma(cs, z, -1.0 / 720.0);
    cs = __builtin_fma(cs, z, 1.0 / 24.0);
    cs = __builtin_fma(cs, z, -0.5);
    cs = __builtin_fma(cs, z, 1.0);
    const int turn = (int)(k - 4.0 * floor(k * 0.25));      // 0 .. 3
    const float a = (float)(turn & 1 ? sn : cs), b = (float)(turn & 1 ? cs : sn);
    *c = turn == 1 || turn == 2 ? -a : a;
    *s = turn & 2 ? -b : b;
}

__device__ __forceinline__ int axis_of(const lantern_rotation& r, int j) {
    int a = 0, end = r.pairs[0];
    for (; j >= end && a < r.axes - 1; end += r.pairs[a]) ++a;
    return a;
}

// A head's elements in units of 2 * NP: unit u < ceil(P / NP) holds pairs u * NP .. of the P, the units after those the
// elements from 2P on.
template <int NP>
__host__ __device__ __forceinline__ int rotation_units(int P, int D) {
    return (P + NP - 1) / NP + (D - 2 * P + 2 * NP - 1) / (2 * NP);
}

// One unit: where its two runs of up to NP values begin.  WIDE: P % NP == 0 and D % (2 * NP) == 0 or D % NP == 0 as the
// caller has checked, so that every run is whole, and every run's address a multiple of its size.
template <typename T, int NP, bool WIDE>
struct RotationUnit {
    bool turned, inter;
    int o1, o2, n1, n2;       // runs x[o1 ..], x[o2 ..] of n1, n2 values (interleaved: pairs in a row from o1)
    float c[NP], s[NP];

    __device__ __forceinline__ void place(int u, int P, int D, bool interleaved) {
        const int lead = (P + NP - 1) / NP;
        turned = u < lead;
        inter = interleaved && turned;
        if (turned) {
            n1 = n2 = min(NP, P - u * NP);
            o1 = interleaved ? 2 * u * NP : u * NP;
            o2 = interleaved ? o1 + NP : o1 + P;
        } else {
            o1 = 2 * P + (u - lead) * 2 * NP;
            o2 = o1 + NP;
            n1 = min(NP, D - o1);
            n2 = min(NP, max(0, D - o2));
        }
    }
    __device__ __forceinline__ void angles(const lantern_rotation& r, const int32_t* position, int u, bool inverse) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int j = min(u * NP + i, max(0, r.pairs[0] + r.pairs[1] + r.pairs[2] + r.pairs[3] - 1));
            angle(position[axis_of(r, j)], r.freqs[j], &c[i], &s[i]);
            if (inverse) s[i] = -s[i];
        }
    }
    // The values x[..] of the unit: first and second of pair i in a[i], b[i]; of a unit that is not turned, its runs.
    __device__ __forceinline__ void load(const T* x, float a[NP], float b[NP]) const {
        if constexpr (WIDE) {
            typedef typename Vec<T, NP>::type V;
            const V p = n1 ? *reinterpret_cast<const V*>(x + o1) : V{};
            const V q = n2 ? *reinterpret_cast<const V*>(x + o2) : V{};
            float all[2 * NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                all[i] = (float)p[i];
                all[NP + i] = (float)q[i];
            }
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                a[i] = inter ? all[2 * i] : all[i];
                b[i] = inter ? all[2 * i + 1] : all[NP + i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                a[i] = i < n1 ? (float)x[inter ? o1 + 2 * i : o1 + i] : 0.f;
                b[i] = i < n2 ? (float)x[inter ? o1 + 2 * i + 1 : o2 + i] : 0.f;
            }
        }
    }
    // The same in the values' own type, for later.
    __device__ __forceinline__ void load_as(const T* x, T a[NP], T b[NP]) const {
        if constexpr (WIDE) {
            typedef typename Vec<T, NP>::type V;
            const V p = *reinterpret_cast<const V*>(x + o1), q = *reinterpret_cast<const V*>(x + o2);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                a[i] = inter ? (2 * i < NP ? p[2 * i % NP] : q[2 * i % NP]) : p[i];
                b[i] = inter ? (2 * i < NP ? p[(2 * i + 1) % NP] : q[(2 * i + 1) % NP]) : q[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                a[i] = i < n1 ? x[inter ? o1 + 2 * i : o1 + i] : (T)0.f;
                b[i] = i < n2 ? x[inter ? o1 + 2 * i + 1 : o2 + i] : (T)0.f;
            }
        }
    }
    __device__ __forceinline__ void turn(float a[NP], float b[NP]) const {
        if (!turned) return;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const float y = a[i] * c[i] - b[i] * s[i], z = a[i] * s[i] + b[i] * c[i];
            a[i] = y;
            b[i] = z;
        }
    }
    template <typename O>
    __device__ __forceinline__ void store(O* x, const float a[NP], const float b[NP]) const {
        if constexpr (WIDE) {
            typedef typename Vec<O, NP>::type V;
            V p, q;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                p[i] = (O)(inter ? (i % 2 ? b[i / 2] : a[i / 2]) : a[i]);
                q[i] = (O)(inter ? (i % 2 ? b[NP / 2 + i / 2] : a[NP / 2 + i / 2]) : b[i]);
            }
            if (n1) *reinterpret_cast<V*>(x + o1) = p;
            if (n2) *reinterpret_cast<V*>(x + o2) = q;
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                if (i < n1) x[inter ? o1 + 2 * i : o1 + i] = (O)a[i];
                if (i < n2) x[inter ? o1 + 2 * i + 1 : o2 + i] = (O)b[i];
            }
        }
    }
};

}  // namespace lantern
