// Operators of a sequence encoder (layer norm, linear attention with decay,
// gated feed-forward): what their kernels' files and the C entry points share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/ndvm.h"

namespace ndvm {
namespace ops {

constexpr int64_t kCus = 256;    // compute units a launch is sized to fill
// Workgroups of 256 threads along one axis of a launch, whose threads are counted in 32 bits.
constexpr int64_t kMostGroups = (1 << 24) - 1;
// The last cache holds 256 MB.  Calls that read and write more than this in all, or streams whose states
// are together more than that, mark data that they touch once as passing through.
constexpr int64_t kPassingTraffic = int64_t(192) << 20, kPassingStates = int64_t(128) << 20;

inline size_t type_bytes(int dtype) { return dtype == NDVM_F32 ? 4 : 2; }
__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t round256(size_t b) { return (b + 255) / 256 * 256; }

// ---- layer norm
struct NormArgs {
    const void *x, *weight, *bias;
    void *y;
    float *mean, *rstd;
    int64_t rows, n, ld_x, ld_y;
    float eps;
};
hipError_t launch_norm(int dtype, const NormArgs &a, hipStream_t stream);

struct NormGradArgs {
    const void *dy, *x, *weight;
    const float *mean, *rstd;
    void *dx, *dweight, *dbias;
    float *part;                // [groups][2][n] partial sums of dweight and dbias
    int64_t rows, n, ld_dy, ld_x, ld_dx;
};
constexpr int64_t kMostNormGrad = int64_t(1) << 27;     // values of a row
size_t norm_grad_bytes(int64_t rows, int64_t n);
hipError_t launch_norm_grad(int dtype, const NormGradArgs &a, hipStream_t stream);

// ---- linear attention: out_i = sum_{j<=i} lambda^(i-j) (a_i . b_j) c_j over the
// tokens of a sequence taken in order (or, reversed, from the last to the first)
struct Heads {
    const void *p;
    int64_t seq, tok, head;     // strides in elements
    int group;                  // head h of the launch reads head h / group
};
struct AttendArgs {
    Heads a, b, c, out;         // widths da, da, dc, dc
    const float *log_decay;     // [heads]
    const int64_t *offsets;     // [n_seq + 1], or null: n_tokens / n_seq tokens each
    const float *state_in;      // [n_seq, heads, da, dc] (or transposed), or null
    float *state_out;           // as state_in, or null
    float *segments;            // a state for each segment and head: what the segment adds, then what enters it
    int64_t n_seq, n_tokens, heads, da, dc;
    int64_t seg_len, n_segments;    // tokens of a segment (a multiple of kSegStep); ids of the launch
    float scale_pair, scale_add, scale_read;    // of a pair's product, of what the state takes, of what is read from it
    int reversed;
    int state_transposed;       // state_in and state_out are [dc, da]
    int out_f32;                // `out` is float whatever the type
    int shared_segments;        // `segments` are those of a sum with b and c exchanged (widths up to 128)
};
// Sums over the same sequences and heads, cut alike, that one launch forms together.
constexpr int kMostSets = 3;
struct AttendSets {
    AttendArgs set[kMostSets];
    int count;
};
constexpr int64_t kSegStep = 64, kMostPartsDim = 128, kMostHeadDim = 256, kMostHeads = 65535, kMostTokens = 1 << 30;
struct Cut {
    int64_t seg_len, n_segments;    // more segments than sequences: sequences are cut
    int64_t state;                  // floats of a segment's and head's state
};
// sets: how many sums a launch forms together
Cut attend_cut(int dtype, int64_t n_seq, int64_t n_tokens, int64_t heads, int64_t da, int64_t dc, bool packed, int sets);
// What enters each segment of sums of the same widths, where there are more segments than sequences.
hipError_t launch_attend_segments(int dtype, const AttendSets &s, hipStream_t stream);
// The outputs, and the states that the sequences end with.
hipError_t launch_attend(int dtype, const AttendSets &s, hipStream_t stream);
// sums of `group` consecutive heads of float [heads][tokens][d] into `out` [.., heads / group, d], two at most
struct FoldHeadsArgs {
    const float *part;
    Heads out;
    int64_t n_seq, n_tokens, heads, d;
    bool packed;
};
struct FoldHeadsSets {
    FoldHeadsArgs set[2];
    int count;
};
hipError_t launch_fold_heads(int dtype, const FoldHeadsSets &s, hipStream_t stream);

struct StepArgs {
    Heads q, k, v, o;           // seq and head strides
    const float *log_decay;
    float *state;               // [n_slots, heads, dk, dv]
    const int64_t *slots;       // [n_seq], or null: slot i
    int64_t n_seq, n_slots, heads, dk, dv;
    float scale;
};
hipError_t launch_step(int dtype, const StepArgs &a, hipStream_t stream);

// ---- gated feed-forward
// Widths and row counts up to this (offsets inside a tile of 256 rows stay below 2^31 bytes).
constexpr int64_t kMostFfnWidth = 1 << 21, kMostFfnRows = 1 << 22;
struct FfnArgs {
    int dtype, act;
    const void *x, *wg, *wu, *dh;
    int64_t rows, n_in, n_out, ld_x, ld_wg, ld_wu, ld_dh;
    void *h;
    int64_t ld_h;
    void *dx, *dwg, *dwu;
    int64_t ld_dx, ld_dwg, ld_dwu;
    void *ws;
};
size_t ffn_bytes(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool grad);
hipError_t launch_ffn(const FfnArgs &a, hipStream_t stream);
hipError_t launch_ffn_grad(const FfnArgs &a, hipStream_t stream);

}  // namespace ops
}  // namespace ndvm
