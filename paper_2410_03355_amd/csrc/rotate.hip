// Rotary positions with several axes (lantern_rotate_axes): queries and keys of N tokens in one launch.
//
// Every value is read once and written once.  A thread owns one unit of a token's head (rotation.h), forms its cosines and
// sines once and goes through the heads of its block with them.  36864 tokens of 24 bf16 heads of 128 take 100 us, 4.5 TB/s of a copy's 5.1;
// with one head loaded at a time 108.  Few tokens are bound by the launch (61 tokens 5.7 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cache_args.h"
#include "device_utils.h"
#include "rotation.h"

namespace lantern {

constexpr int AT_ONCE = 4;      // heads loaded together: an output may be its input, so no load passes a store

template <typename T, int NP, bool WIDE>
__global__ __launch_bounds__(NT) void rotate_axes_kernel(RotateArgs a) {
    const int units = rotation_units<NP>(a.pairs, a.D);
    const int per_block = NT / units;      // D <= 1024: at most 130 units
    const int64_t token = (int64_t)blockIdx.x * per_block + threadIdx.x / units;
    if ((int)threadIdx.x >= per_block * units || token >= a.N) return;
    const int u = threadIdx.x % units;
    RotationUnit<T, NP, WIDE> unit;
    unit.place(u, a.pairs, a.D, a.rot.interleaved != 0);
    if (unit.turned) unit.angles(a.rot, a.rot.positions + token * a.rot.axes, u, a.inverse != 0);
    const int heads = a.q_heads + a.k_heads;
    const int first = blockIdx.y * a.heads_per_block, last = min(heads, first + a.heads_per_block);
    auto in = [&](int h) {
        return h < a.q_heads ? static_cast<const T*>(a.q) + token * a.sq.row + h * a.sq.head
                             : static_cast<const T*>(a.k) + token * a.sk.row + (h - a.q_heads) * a.sk.head;
    };
    auto out = [&](int h) {
        return h < a.q_heads ? static_cast<T*>(a.out_q) + token * a.soq.row + h * a.soq.head
                             : static_cast<T*>(a.out_k) + token * a.sok.row + (h - a.q_heads) * a.sok.head;
    };
    for (int h = first; h < last; h += AT_ONCE) {      // the last heads again where fewer are left: loaded, not written
        float p[AT_ONCE][NP], q[AT_ONCE][NP];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) unit.load(in(min(h + i, last - 1)), p[i], q[i]);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (h + i >= last) break;
            unit.turn(p[i], q[i]);
            unit.store(out(h + i), p[i], q[i]);
        }
    }
}

template <typename T, int NP, bool WIDE>
static hipError_t launch(RotateArgs a, hipStream_t stream) {
    const int per_block = NT / rotation_units<NP>(a.pairs, a.D);
    const int blocks = (int)(((int64_t)a.N + per_block - 1) / per_block), heads = a.q_heads + a.k_heads;
    // Few tokens: their heads are spread over blocks until there are some 8 wavefronts for each of the 256 CUs.
    if (blocks > MOST_GROUPS) return hipErrorInvalidConfiguration;
    const int chunks = std::max(1, std::min(heads, 512 / std::max(1, blocks)));
    a.heads_per_block = (heads + chunks - 1) / chunks;
    hipLaunchKernelGGL((rotate_axes_kernel<T, NP, WIDE>), dim3(blocks, (heads + a.heads_per_block - 1) / a.heads_per_block), dim3(NT), 0,
                       stream, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_type(const RotateArgs& a, hipStream_t stream) {
    if (!a.wide) return launch<T, 4, false>(a, stream);
    // 16-byte loads of bf16 where the pairs come in eights, else of 8 bytes
    if (sizeof(T) == 2 && a.pairs % 8 == 0) return launch<T, sizeof(T) == 2 ? 8 : 4, true>(a, stream);
    return launch<T, 4, true>(a, stream);
}

hipError_t launch_rotate_axes(const RotateArgs& a, int dtype, hipStream_t stream) {
    return dtype == LANTERN_F32 ? launch_type<float>(a, stream) : launch_type<bf16>(a, stream);
}

hipError_t prepare_rotate(int dtype) {
    hipFuncAttributes attr;   // the runtime loads all of a file's kernels together
    return hipFuncGetAttributes(&attr, dtype == LANTERN_F32 ? reinterpret_cast<const void*>(&rotate_axes_kernel<float, 4, true>)
                                                            : reinterpret_cast<const void*>(&rotate_axes_kernel<bf16, 4, true>));
}

}  // namespace lantern
