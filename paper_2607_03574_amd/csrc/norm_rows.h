// What the norms' kernels share: a row's values in the registers of 16, 64 or 256 threads, and their sums.
#pragma once
#include <type_traits>

#include "ops.h"
#include "ops_types.h"

namespace ndvm {
namespace ops {
namespace {

// Sums over the L threads of a row (thread t of it; the row's own words of LDS);
// every one of them gets them.  All threads of the workgroup call it together.
template <int L> __device__ inline void row_sum2(float &u, float &v, int t, float *lds) {
#pragma unroll
    for (int s = (L < 64 ? L : 64) / 2; s > 0; s >>= 1) {
        u += __shfl_xor(u, s);
        v += __shfl_xor(v, s);
    }
    if (L > 64) {
        __syncthreads();
        if (t % 64 == 0) {
            lds[t / 64] = u;
            lds[L / 64 + t / 64] = v;
        }
        __syncthreads();
        u = v = 0;
#pragma unroll
        for (int w = 0; w < L / 64; ++w) {
            u += lds[w];
            v += lds[L / 64 + w];
        }
    }
}
template <int L> __device__ inline float row_sum(float v, int t, float *lds) {
    float none = 0;
    row_sum2<L>(v, none, t, lds);
    return v;
}

// Calls f(L, NV) with the fewest threads a row that hold n columns in at most 32
// registers' worth each; false if none do.
template <class T, class F> bool with_shape(int64_t n, F f) {
    constexpr int V = kVec<T>;
    const int64_t v = ceil_div(n, V);
    constexpr int64_t most = 32 / V;        // vectors a thread
    using std::integral_constant;
#define NDVM_SHAPE(L, NV) \
    if constexpr (NV <= most) \
        if (v <= int64_t(L) * NV) return f(integral_constant<int, L>(), integral_constant<int, NV>()), true;
    NDVM_SHAPE(16, 1)
    NDVM_SHAPE(16, 2)
    NDVM_SHAPE(64, 1)
    NDVM_SHAPE(64, 2)
    NDVM_SHAPE(64, 4)
    NDVM_SHAPE(64, 8)
    NDVM_SHAPE(256, 2)
    NDVM_SHAPE(256, 4)
    NDVM_SHAPE(256, 8)
#undef NDVM_SHAPE
    return false;
}

}  // namespace
}  // namespace ops
}  // namespace ndvm
