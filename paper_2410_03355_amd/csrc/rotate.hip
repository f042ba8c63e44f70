// Rotary positions with several axes (lantern_rotate_axes): queries and keys of N tokens in one launch.
//
// Every value is read once and written once.  A thread owns one unit of a token's head (rotation.h), forms its cosines and
// sines once and goes through the heads of its block with them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "cache_args.h"
#include "device_utils.h"
#include "rotation.h"

namespace lantern {

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
#pragma unroll 4
    for (int h = first; h < last; ++h) {
        const bool of_q = h < a.q_heads;
        const int hh = of_q ? h : h - a.q_heads;
        const T* x = static_cast<const T*>(of_q ? a.q : a.k) + (of_q ? token * a.sq.row + hh * a.sq.head : token * a.sk.row + hh * a.sk.head);
        T* y = static_cast<T*>(of_q ? a.out_q : a.out_k) + (of_q ? token * a.soq.row + hh * a.soq.head : token * a.sok.row + hh * a.sok.head);
        float p[NP], q[NP];
        unit.load(x, p, q);
        unit.turn(p, q);
        unit.store(y, p, q);
    }
}

template <typename T, int NP, bool WIDE>
static hipError_t launch(RotateArgs a, hipStream_t stream) {
    const int per_block = NT / rotation_units<NP>(a.pairs, a.D);
    const int blocks = (int)(((int64_t)a.N + per_block - 1) / per_block), heads = a.q_heads + a.k_heads;
    // Few tokens: their heads are spread over blocks until there are some 8 wavefronts for each of the 256 CUs.
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
