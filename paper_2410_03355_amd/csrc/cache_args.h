// Arguments of the kernels around a tree step (rotate.hip, append.hip, attend.hip), as api.hip hands them over after its checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lantern.h"

namespace lantern {

constexpr int64_t MOST_GROUPS = (1 << 24) - 1;      // workgroups of 256 along a grid's x: a launch has less than 2^32 threads there

struct Strided {            // elements from one sequence, row and head to the next; a head's elements are dense
    int64_t seq, row, head;
};

struct RotateArgs {
    lantern_rotation rot;
    int pairs;              // of all axes
    int N, D, q_heads, k_heads, inverse;
    int heads_per_block;
    bool wide;              // vector loads and stores
    const void *q, *k;
    void *out_q, *out_k;
    Strided sq, sk, soq, sok;
};

struct AppendArgs {
    lantern_cache cache;
    lantern_rotation rot;
    int pairs;              // 0: keys are stored as they are
    int page_shift;
    const int32_t *table, *lengths;
    int width, B, T, touched;   // touched: most pages that one sequence's rows reach
    bool wide_k, wide_v;
    const void *k, *v;
    Strided sk, sv;
    const int32_t *path, *count;
    int32_t* out_lengths;
};

// Division by a number that the host knows, for 0 <= n < 2^31 (Granlund and Montgomery 1994, division by invariant integers).  With 2^(l-1) < d <= 2^l and mul = floor(2^32 (2^l - d) / d) + 1 the
// quotient is (umulhi(n, mul) + n) >> l.
struct Divisor {
    unsigned mul;
    int shift;
    Divisor() = default;
    explicit Divisor(unsigned d) : shift(0) {
        while ((1ull << shift) < d) ++shift;
        mul = (unsigned)((((1ull << shift) - d) << 32) / d + 1);
    }
    __device__ __forceinline__ int of(int n) const { return (int)((__umulhi((unsigned)n, mul) + (unsigned)n) >> shift); }
};

struct AttendArgs {
    lantern_cache cache;
    int page_shift;
    const int32_t *table, *lengths, *parent;
    int width, B, M, q_heads, group;   // group: query heads to a key head
    bool wide;              // 16-byte loads of queries, keys and values
    const void *q, *k, *v;
    Strided sq, sk, sv;
    float scale;            // of the scores, times log2(e)
    void* out;              // [B, M + 1, q_heads, D]
    int parts, row_tiles;   // parts of all sequences, B or more; sets of rows, one to a workgroup
    double per_part, per_all;   // 1 / (parts - B), a little more; 1 / (4 * parts), a little less
    float* part;            // where they are more: outputs [parts, heads, rows, D], then maxima and sums [parts, heads, rows]
    int2* cut;              // behind them: a sequence's first part and how many it has
    Divisor by_tiles, by_heads, by_group;
};

struct AttendPlan {
    int parts, row_tiles, row_group, abreast;
    size_t workspace;
};
AttendPlan plan_attend(int dtype, int B, int M, int q_heads, const lantern_cache& c, int width);

hipError_t launch_rotate_axes(const RotateArgs& a, int dtype, hipStream_t stream);
hipError_t launch_append_cache(const AppendArgs& a, int dtype, hipStream_t stream);
hipError_t launch_attend_trees(const AttendArgs& a, int dtype, int row_group, int abreast, hipStream_t stream);
hipError_t prepare_rotate(int dtype);
hipError_t prepare_append(int dtype, const lantern_cache& c);
hipError_t prepare_attend(int dtype, const lantern_cache& c);

}  // namespace lantern
