// Root-mean-square norm over the last axis with the addition of a residual, its gradient, and
// rows in 8 bits with a scale each.
//   h = x + r (rounded to the tensors' type: what the residual carries on is what is normalised)
//   y = h rstd w,  rstd = 1 / sqrt(mean(h^2) + eps)
//   g = dy w,  dx = dr = rstd (g - hh mean(g hh)) + dh,  hh = h rstd,  dw = sum_rows dy hh
//   8 bits (e4m3, largest value 448): scale = max(max |y|, 448 2^-126) / 448, y8 = y / scale
// Bound by memory, like the layer norm: a row stays in the registers of the threads that loaded it, so the sum
// of squares, the largest value and the result come from one read.
#include <algorithm>

#include "norm_rows.h"

namespace ndvm {
namespace ops {
namespace {

enum Out { kNorm, kNorm8, kRows8 };     // y; y in 8 bits; x itself in 8 bits

// The largest of the L threads of a row; NaN where one of them has it.
__device__ inline float larger(float m, float a) { return a > m || a != a ? a : m; }
template <int L> __device__ inline float row_largest(float m, int t, float *lds) {
#pragma unroll
    for (int s = (L < 64 ? L : 64) / 2; s > 0; s >>= 1) m = larger(m, __shfl_xor(m, s));
    if (L > 64) {
        __syncthreads();
        if (t % 64 == 0) lds[t / 64] = m;
        __syncthreads();
        m = 0;
#pragma unroll
        for (int w = 0; w < L / 64; ++w) m = larger(m, lds[w]);
    }
    return m;
}
__device__ inline float scale_of_row(float largest) { return larger(448.0f * 0x1p-126f, largest) / 448.0f; }

// V values to e4m3, [0, count) of them to p.
template <int V> __device__ inline void store_8bit(uint8_t *p, const float (&v)[V], int64_t count) {
    typedef uint32_t words __attribute__((ext_vector_type(V / 4), aligned(1)));
    words w;
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        w[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], low, true));
    }
    if (count >= V) {
        *reinterpret_cast<words *>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < count) p[i] = uint8_t(w[i / 4] >> (i % 4 * 8));
}

// x, or x + r as it is rounded.
template <class T> __device__ inline vec<T> joined(const T *x, const T *r, int64_t count) {
    vec<T> v = load_vec(x, count);
    if (r) {
        const vec<T> more = load_vec(r, count);
#pragma unroll
        for (int j = 0; j < kVec<T>; ++j) v[j] = T(float(v[j]) + float(more[j]));
    }
    return v;
}

// L threads a row, NV vectors a thread.
template <class T, int L, int NV, Out OUT, bool PASSING> __global__ void __launch_bounds__(256) rms_rows(RmsArgs a) {
    constexpr int V = kVec<T>, R = 256 / L;
    __shared__ float lds[8];
    const int lane = threadIdx.x % L;
    const T *w = static_cast<const T *>(a.weight);
    for (int64_t row = int64_t(blockIdx.x) * R + threadIdx.x / L; row < a.rows; row += int64_t(gridDim.x) * R) {
        const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
        const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ld_r : nullptr;
        vec<T> h[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
            h[i] = joined(x + c, r ? r + c : nullptr, a.n - c);
        }
        float rstd = 1.0f;
        if constexpr (OUT != kRows8) {
            float sq = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) sq += float(h[i][j]) * float(h[i][j]);
            rstd = 1.0f / sqrtf(row_sum<L>(sq, lane, lds) / float(a.n) + a.eps);
            if (r) {
                T *to = static_cast<T *>(a.h) + row * a.ld_h;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int64_t c = int64_t(i * L + lane) * V;
                    if (c < a.n) store_vec<PASSING>(to + c, h[i], a.n - c);
                }
            }
        }
        float y[NV][V], most = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
            vec<T> wv = T(1.0f);
            if (OUT != kRows8 && w && c < a.n) wv = load_vec(w + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                y[i][j] = OUT == kRows8 ? float(h[i][j]) : float(h[i][j]) * rstd * float(wv[j]);
                if (OUT != kNorm && c + j < a.n) most = larger(most, fabsf(y[i][j]));
            }
            if constexpr (OUT == kNorm) {
                if (c >= a.n) continue;
                vec<T> out;
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] = T(y[i][j]);
                store_vec<PASSING>(static_cast<T *>(a.y) + row * a.ld_y + c, out, a.n - c);
            }
        }
        if constexpr (OUT != kNorm) {
            const float scale = scale_of_row(row_largest<L>(most, lane, lds)), inverse = 1.0f / scale;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t c = int64_t(i * L + lane) * V;
                if (c >= a.n) continue;
#pragma unroll
                for (int j = 0; j < V; ++j) y[i][j] *= inverse;
                store_8bit<V>(static_cast<uint8_t *>(a.y) + row * a.ld_y + c, y[i], a.n - c);
            }
            if (lane == 0) a.scale[row] = scale;
        }
        if (OUT == kNorm && lane == 0 && a.rstd) a.rstd[row] = rstd;
    }
}

// A row of any length: 256 threads, two or three reads of it.  (The later ones are of h as it was stored, by the thread that stored
// it: x or the residual may be what h took the place of.)
template <class T, Out OUT> __global__ void __launch_bounds__(256) rms_long(RmsArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float lds[8];
    const T *w = static_cast<const T *>(a.weight);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
        const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.ld_r : nullptr;
        T *const held = r ? static_cast<T *>(a.h) + row * a.ld_h : nullptr;
        float rstd = 1.0f;
        if constexpr (OUT != kRows8) {
            float sq = 0;
            for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
                const vec<T> h = joined(x + c, r ? r + c : nullptr, a.n - c);
#pragma unroll
                for (int j = 0; j < V; ++j) sq += float(h[j]) * float(h[j]);
                if (r) store_vec(held + c, h, a.n - c);
            }
            rstd = 1.0f / sqrtf(row_sum<256>(sq, threadIdx.x, lds) / float(a.n) + a.eps);
        }
        const auto result = [&](int64_t c, float (&y)[V]) {
            const vec<T> h = load_vec((r ? held : x) + c, a.n - c);
            vec<T> wv = T(1.0f);
            if (OUT != kRows8 && w) wv = load_vec(w + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = OUT == kRows8 ? float(h[j]) : float(h[j]) * rstd * float(wv[j]);
        };
        float y[V], scale = 1.0f;
        if constexpr (OUT != kNorm) {
            float most = 0;
            for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
                result(c, y);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < a.n) most = larger(most, fabsf(y[j]));
            }
            scale = scale_of_row(row_largest<256>(most, threadIdx.x, lds));
            if (threadIdx.x == 0) a.scale[row] = scale;
        }
        const float inverse = 1.0f / scale;
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            result(c, y);
            if constexpr (OUT == kNorm) {
                vec<T> out;
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] = T(y[j]);
                store_vec(static_cast<T *>(a.y) + row * a.ld_y + c, out, a.n - c);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] *= inverse;
                store_8bit<V>(static_cast<uint8_t *>(a.y) + row * a.ld_y + c, y, a.n - c);
            }
        }
        if (OUT == kNorm && threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
    }
}

// ---- gradient
constexpr int kGradThreads = 512;
constexpr int64_t kGradGroups = 256;        // workgroups that keep partial sums
constexpr int64_t kLongCols = 256, kLongGroups = 64;

// L threads a row, NV vectors a thread.  A thread has the same columns in every row, so its sums for dweight stay
// in registers over all rows of the workgroup; a partial sum a workgroup goes to memory, and a second launch adds
// them up in order.
template <class T, int L, int NV, bool SUMS, bool PASSING>
__global__ void __launch_bounds__(kGradThreads) rms_grad_rows(RmsGradArgs a) {
    constexpr int V = kVec<T>, R = kGradThreads / L;
    __shared__ float lds[2 * (L / 64) * R + 1];
    __shared__ float fold[SUMS && L < kGradThreads ? L * NV * V : 1];
    const int lane = threadIdx.x % L, sub = threadIdx.x / L;
    const T *w = static_cast<const T *>(a.weight);
    float dw[NV][V];
    vec<T> wv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t c = int64_t(i * L + lane) * V;
        wv[i] = T(1.0f);
        if (w) wv[i] = load_vec(w + c, a.n - c);
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = 0;
    }
    const int64_t step = int64_t(gridDim.x) * R;
    // A row is read while the one before it is worked on, where the registers hold two.
    constexpr bool AHEAD = NV <= 4;
    vec<T> hv[NV], gv[NV], rv[NV], next_h[NV], next_g[NV], next_r[NV];
    float rstd = 0, next_rstd = 0;
    const auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        if (row >= a.rows) return;
        const T *h = static_cast<const T *>(a.h) + row * a.ld_h;
        const T *dy = static_cast<const T *>(a.dy) + row * a.ld_dy;
        next_rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
            next_h[i] = load_vec(h + c, a.n - c);
            next_g[i] = load_vec(dy + c, a.n - c);      // 0 beyond the row: adds nothing anywhere
            if (a.dx && a.dh) next_r[i] = load_vec(static_cast<const T *>(a.dh) + row * a.ld_dh + c, a.n - c);
        }
    };
    if (AHEAD) fetch(int64_t(blockIdx.x) * R + sub);
    // a workgroup's threads take the same number of turns (they meet at barriers)
    for (int64_t base = int64_t(blockIdx.x) * R; base < a.rows; base += step) {
        const int64_t row = base + sub;
        const bool on = row < a.rows;
        if (!AHEAD) fetch(row);
        rstd = next_rstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            hv[i] = next_h[i];
            gv[i] = next_g[i];
            rv[i] = next_r[i];
        }
        if (AHEAD) fetch(row + step);
        float along = 0;
        if (on) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float hh = float(hv[i][j]) * rstd, dy = float(gv[i][j]);
                    if (SUMS) dw[i][j] += dy * hh;
                    along += dy * float(wv[i][j]) * hh;
                }
        }
        if (a.dx) {
            along = row_sum<L>(along, lane, lds + 2 * (L / 64) * sub);
            if (on) {
                const float m = along / float(a.n);
                T *dx = static_cast<T *>(a.dx) + row * a.ld_dx;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int64_t c = int64_t(i * L + lane) * V;
                    if (c >= a.n) continue;
                    vec<T> out;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float d = rstd * (float(gv[i][j]) * float(wv[i][j]) - float(hv[i][j]) * rstd * m);
                        out[j] = T(a.dh ? d + float(rv[i][j]) : d);
                    }
                    store_vec<PASSING>(dx + c, out, a.n - c);
                }
            }
        }
    }
    if (!SUMS) return;
    float *part = a.part + int64_t(blockIdx.x) * a.n;
    for (int r = 0; r < R; ++r) {
        __syncthreads();
        if (sub != r) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = (i * L + lane) * V + j;
                const float v = (r ? fold[c] : 0.0f) + dw[i][j];
                if (r < R - 1) fold[c] = v;
                else if (c < a.n) part[c] = v;
            }
    }
}

// Rows of any length: 256 threads a row, two reads.
template <class T> __global__ void __launch_bounds__(256) rms_grad_long(RmsGradArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float lds[8];
    const T *w = static_cast<const T *>(a.weight);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *h = static_cast<const T *>(a.h) + row * a.ld_h;
        const T *dy = static_cast<const T *>(a.dy) + row * a.ld_dy;
        const T *dh = a.dh ? static_cast<const T *>(a.dh) + row * a.ld_dh : nullptr;
        T *dx = static_cast<T *>(a.dx) + row * a.ld_dx;
        const float rstd = a.rstd[row];
        float along = 0;
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> hv = load_vec(h + c, a.n - c), gv = load_vec(dy + c, a.n - c);
            vec<T> wv = T(1.0f);
            if (w) wv = load_vec(w + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) along += float(gv[j]) * float(wv[j]) * (float(hv[j]) * rstd);
        }
        const float m = row_sum<256>(along, threadIdx.x, lds) / float(a.n);
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> hv = load_vec(h + c, a.n - c), gv = load_vec(dy + c, a.n - c);
            vec<T> wv = T(1.0f), rv = T(0.0f), out;
            if (w) wv = load_vec(w + c, a.n - c);
            if (dh) rv = load_vec(dh + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = rstd * (float(gv[j]) * float(wv[j]) - float(hv[j]) * rstd * m);
                out[j] = T(dh ? d + float(rv[j]) : d);
            }
            store_vec(dx + c, out, a.n - c);
        }
    }
}
// ... and their column sums: a thread a column, a workgroup every gridDim.y-th row.
template <class T> __global__ void __launch_bounds__(kLongCols) rms_grad_columns(RmsGradArgs a) {
    const int64_t c = int64_t(blockIdx.x) * kLongCols + threadIdx.x;
    if (c >= a.n) return;
    float dw = 0;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y)
        dw += float(static_cast<const T *>(a.dy)[row * a.ld_dy + c]) * (float(static_cast<const T *>(a.h)[row * a.ld_h + c]) * a.rstd[row]);
    a.part[int64_t(blockIdx.y) * a.n + c] = dw;
}

// dweight from the workgroups' sums, in order: 32 columns a workgroup, 8 threads a column, each every eighth sum.
template <class T> __global__ void __launch_bounds__(256) rms_grad_fold(RmsGradArgs a, int groups) {
    __shared__ float lds[8][32];
    const int64_t c = int64_t(blockIdx.x) * 32 + threadIdx.x % 32;
    const int s = threadIdx.x / 32;
    float v = 0;
    if (c < a.n)
#pragma unroll 8
        for (int g = s; g < groups; g += 8) v += a.part[int64_t(g) * a.n + c];
    lds[s][threadIdx.x % 32] = v;
    __syncthreads();
    if (s || c >= a.n) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) v += lds[i][threadIdx.x];
    static_cast<T *>(a.dweight)[c] = T(v);
}

int64_t grad_groups(int64_t rows) { return std::min<int64_t>(std::max<int64_t>(rows, 1), kGradGroups); }

template <class T, Out OUT> void launch(const RmsArgs &a, hipStream_t stream) {
    const bool held = with_shape<T>(a.n, [&](auto l, auto nv) {
        constexpr int L = decltype(l)::value, NV = decltype(nv)::value;
        const dim3 grid(uint32_t(std::min<int64_t>(ceil_div(a.rows, 256 / L), 1 << 20)));
        const int64_t moved = a.rows * a.n * ((a.residual ? 3 : 1) * int64_t(sizeof(T)) + (OUT == kNorm ? int64_t(sizeof(T)) : 1));
        if (moved >= kPassingTraffic) rms_rows<T, L, NV, OUT, true><<<grid, 256, 0, stream>>>(a);
        else rms_rows<T, L, NV, OUT, false><<<grid, 256, 0, stream>>>(a);
    });
    if (!held) rms_long<T, OUT><<<dim3(uint32_t(std::min<int64_t>(a.rows, 1 << 20))), 256, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_rms(int dtype, const RmsArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        if (!a.scale) launch<T, kNorm>(a, stream);
        else if (a.rows_only) launch<T, kRows8>(a, stream);
        else launch<T, kNorm8>(a, stream);
        return hipGetLastError();
    });
}

size_t rms_grad_bytes(int64_t rows, int64_t n) { return size_t(grad_groups(rows)) * size_t(n) * sizeof(float); }

hipError_t launch_rms_grad(int dtype, const RmsGradArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const bool sums = a.dweight;
        int64_t groups = 0;
        const bool held = with_shape<T>(a.n, [&](auto l, auto nv) {
            constexpr int L = decltype(l)::value, NV = decltype(nv)::value;
            constexpr int R = kGradThreads / L;
            groups = std::min(ceil_div(a.rows, R), sums ? kGradGroups : int64_t(1) << 20);
            if (groups == 0) return;
            const bool passing = (a.dh ? 4 : 3) * a.rows * a.n * int64_t(sizeof(T)) >= kPassingTraffic;
            const dim3 grid(static_cast<uint32_t>(groups));
            if (sums && passing) rms_grad_rows<T, L, NV, true, true><<<grid, kGradThreads, 0, stream>>>(a);
            else if (sums) rms_grad_rows<T, L, NV, true, false><<<grid, kGradThreads, 0, stream>>>(a);
            else if (passing) rms_grad_rows<T, L, NV, false, true><<<grid, kGradThreads, 0, stream>>>(a);
            else rms_grad_rows<T, L, NV, false, false><<<grid, kGradThreads, 0, stream>>>(a);
        });
        if (!held) {
            if (a.dx && a.rows) rms_grad_long<T><<<dim3(uint32_t(std::min<int64_t>(a.rows, 1 << 20))), 256, 0, stream>>>(a);
            groups = std::min(a.rows, kLongGroups);
            if (groups && sums)
                rms_grad_columns<T><<<dim3(uint32_t(ceil_div(a.n, kLongCols)), uint32_t(groups)), kLongCols, 0, stream>>>(a);
        }
        if (sums) rms_grad_fold<T><<<dim3(uint32_t(ceil_div(a.n, 32))), 256, 0, stream>>>(a, int(groups));
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
