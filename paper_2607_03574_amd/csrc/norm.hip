// Layer norm over the last axis, and its gradient.
//   y = xh w + b,  xh = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//   g = dy w,  dx = rstd (g - mean(g) - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy
// Both are bound by memory: about ten operations an element, read once and
// written once.  A row stays in the registers of the threads that loaded it
// (16, 64 or 256 of them, by its length), so mean, squares and result come
// from one read; rows too long for that are read again, from cache.
// Measured: 32768 x 2048 bf16 49 us a call, the kernel 45 (6.0 TB/s; a copy that moves as much, part of it in the
// last cache, 7.2, a larger one 5.5); its gradient at 16384 x 2048 49 us, the kernel 42 (4.8 TB/s) and the
// sum of its partial sums 5.
#include <algorithm>

#include "norm_rows.h"

namespace ndvm {
namespace ops {
namespace {

// L threads a row, NV vectors a thread.
template <class T, int L, int NV, bool PASSING> __global__ void __launch_bounds__(256) norm_rows(NormArgs a) {
    constexpr int V = kVec<T>, R = 256 / L;
    __shared__ float lds[8];
    const int lane = threadIdx.x % L;
    const T *w = static_cast<const T *>(a.weight), *b = static_cast<const T *>(a.bias);
    for (int64_t row = int64_t(blockIdx.x) * R + threadIdx.x / L; row < a.rows; row += int64_t(gridDim.x) * R) {
        const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
        T *y = static_cast<T *>(a.y) + row * a.ld_y;
        vec<T> xv[NV];
        float sum = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
            xv[i] = load_vec(x + c, a.n - c);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) sum += float(xv[i][j]);
        const float mean = row_sum<L>(sum, lane, lds) / float(a.n);
        float sq = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = float(xv[i][j]) - mean;
                if (c + j < a.n) sq += d * d;
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<L>(sq, lane, lds) / float(a.n) + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
            if (c >= a.n) continue;
            vec<T> wv = T(1.0f), bv = T(0.0f), out;
            if (w) wv = load_vec(w + c, a.n - c);
            if (b) bv = load_vec(b + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = T((float(xv[i][j]) - mean) * rstd * float(wv[j]) + float(bv[j]));
            store_vec<PASSING>(y + c, out, a.n - c);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// A row of any length: 256 threads, three reads of it.
template <class T> __global__ void __launch_bounds__(256) norm_long(NormArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float lds[8];
    const T *w = static_cast<const T *>(a.weight), *b = static_cast<const T *>(a.bias);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
        T *y = static_cast<T *>(a.y) + row * a.ld_y;
        float sum = 0, sq = 0;
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> xv = load_vec(x + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) sum += float(xv[j]);
        }
        const float mean = row_sum<256>(sum, threadIdx.x, lds) / float(a.n);
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> xv = load_vec(x + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = float(xv[j]) - mean;
                if (c + j < a.n) sq += d * d;
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<256>(sq, threadIdx.x, lds) / float(a.n) + a.eps);
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> xv = load_vec(x + c, a.n - c);
            vec<T> wv = T(1.0f), bv = T(0.0f), out;
            if (w) wv = load_vec(w + c, a.n - c);
            if (b) bv = load_vec(b + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) out[j] = T((float(xv[j]) - mean) * rstd * float(wv[j]) + float(bv[j]));
            store_vec(y + c, out, a.n - c);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// ---- gradient
constexpr int kGradThreads = 512;
constexpr int64_t kGradGroups = 256;        // workgroups that keep partial sums
constexpr int64_t kLongCols = 256, kLongGroups = 64;

// L threads a row, NV vectors a thread.  A thread has the same columns in every
// row, so its sums for dweight and dbias stay in registers over all rows of the
// workgroup; at the end the workgroup's rows of threads are added in order and
// one partial sum a workgroup goes to memory (no atomics: the sum's order is fixed).
template <class T, int L, int NV, bool SUMS, bool PASSING>
__global__ void __launch_bounds__(kGradThreads) norm_grad_rows(NormGradArgs a) {
    constexpr int V = kVec<T>, R = kGradThreads / L;
    __shared__ float lds[2 * (L / 64) * R + 1];
    __shared__ float fold[SUMS && L < kGradThreads ? L * NV * V : 1];
    const int lane = threadIdx.x % L, sub = threadIdx.x / L;
    const T *w = static_cast<const T *>(a.weight);
    float dw[NV][V], db[NV][V];
    vec<T> wv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t c = int64_t(i * L + lane) * V;
        wv[i] = T(1.0f);
        if (w) wv[i] = load_vec(w + c, a.n - c);
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = 0;
    }
    const int64_t step = int64_t(gridDim.x) * R;
    // A row is read while the one before it is worked on, where the registers hold two.
    constexpr bool AHEAD = NV <= 4;
    vec<T> xv[NV], gv[NV], next_x[NV], next_g[NV];
    float mean = 0, rstd = 0, next_mean = 0, next_rstd = 0;
    const auto fetch = [&](int64_t row) __attribute__((always_inline)) {
        if (row >= a.rows) return;
        const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
        const T *dy = static_cast<const T *>(a.dy) + row * a.ld_dy;
        next_mean = a.mean[row];
        next_rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = int64_t(i * L + lane) * V;
            next_x[i] = load_vec(x + c, a.n - c);
            next_g[i] = load_vec(dy + c, a.n - c);      // 0 beyond the row: adds nothing anywhere
        }
    };
    if (AHEAD) fetch(int64_t(blockIdx.x) * R + sub);
    // a workgroup's threads take the same number of turns (they meet at barriers)
    for (int64_t base = int64_t(blockIdx.x) * R; base < a.rows; base += step) {
        const int64_t row = base + sub;
        const bool on = row < a.rows;
        if (!AHEAD) fetch(row);
        mean = next_mean;
        rstd = next_rstd;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            xv[i] = next_x[i];
            gv[i] = next_g[i];
        }
        if (AHEAD) fetch(row + step);
        float s1 = 0, s2 = 0;
        if (on) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float xh = (float(xv[i][j]) - mean) * rstd, dy1 = float(gv[i][j]);
                    if (SUMS) {
                        dw[i][j] += dy1 * xh;
                        db[i][j] += dy1;
                    }
                    const float g = dy1 * float(wv[i][j]);
                    s1 += g;
                    s2 += g * xh;
                }
        }
        if (a.dx) {
            row_sum2<L>(s1, s2, lane, lds + 2 * (L / 64) * sub);
            if (on) {
                const float m1 = s1 / float(a.n), m2 = s2 / float(a.n);
                T *dx = static_cast<T *>(a.dx) + row * a.ld_dx;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int64_t c = int64_t(i * L + lane) * V;
                    if (c >= a.n) continue;
                    vec<T> out;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float xh = (float(xv[i][j]) - mean) * rstd;
                        out[j] = T(rstd * (float(gv[i][j]) * float(wv[i][j]) - m1 - xh * m2));
                    }
                    store_vec<PASSING>(dx + c, out, a.n - c);
                }
            }
        }
    }
    if (!SUMS) return;
    float *part = a.part + int64_t(blockIdx.x) * 2 * a.n;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&s)[NV][V] = which ? db : dw;
        for (int r = 0; r < R; ++r) {
            __syncthreads();
            if (sub != r) continue;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int c = (i * L + lane) * V + j;
                    const float v = (r ? fold[c] : 0.0f) + s[i][j];
                    if (r < R - 1) fold[c] = v;
                    else if (c < a.n) part[int64_t(which) * a.n + c] = v;
                }
        }
    }
}

// Rows of any length: 256 threads a row, two reads.
template <class T> __global__ void __launch_bounds__(256) norm_grad_long(NormGradArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float lds[8];
    const T *w = static_cast<const T *>(a.weight);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.ld_x;
        const T *dy = static_cast<const T *>(a.dy) + row * a.ld_dy;
        T *dx = static_cast<T *>(a.dx) + row * a.ld_dx;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0, s2 = 0;
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> xv = load_vec(x + c, a.n - c), gv = load_vec(dy + c, a.n - c);
            vec<T> wv = T(1.0f);
            if (w) wv = load_vec(w + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float g = float(gv[j]) * float(wv[j]);
                s1 += g;
                s2 += g * (float(xv[j]) - mean) * rstd;
            }
        }
        row_sum2<256>(s1, s2, threadIdx.x, lds);
        const float m1 = s1 / float(a.n), m2 = s2 / float(a.n);
        for (int64_t c = threadIdx.x * V; c < a.n; c += 256 * V) {
            const vec<T> xv = load_vec(x + c, a.n - c), gv = load_vec(dy + c, a.n - c);
            vec<T> wv = T(1.0f), out;
            if (w) wv = load_vec(w + c, a.n - c);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float xh = (float(xv[j]) - mean) * rstd;
                out[j] = T(rstd * (float(gv[j]) * float(wv[j]) - m1 - xh * m2));
            }
            store_vec(dx + c, out, a.n - c);
        }
    }
}
// ... and their column sums: a thread a column, a workgroup every gridDim.y-th row.
template <class T> __global__ void __launch_bounds__(kLongCols) norm_grad_columns(NormGradArgs a) {
    const int64_t c = int64_t(blockIdx.x) * kLongCols + threadIdx.x;
    if (c >= a.n) return;
    float dw = 0, db = 0;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float dy = float(static_cast<const T *>(a.dy)[row * a.ld_dy + c]);
        dw += dy * (float(static_cast<const T *>(a.x)[row * a.ld_x + c]) - a.mean[row]) * a.rstd[row];
        db += dy;
    }
    float *part = a.part + int64_t(blockIdx.y) * 2 * a.n;
    part[c] = dw;
    part[a.n + c] = db;
}

// dweight and dbias from the workgroups' sums, in order: 32 columns a workgroup,
// 8 threads a column, each every eighth sum.
template <class T> __global__ void __launch_bounds__(256) norm_grad_fold(NormGradArgs a, int groups) {
    __shared__ float lds[8][32];
    const int64_t c = int64_t(blockIdx.x) * 32 + threadIdx.x % 32;      // column of [2][n]
    const int s = threadIdx.x / 32;
    float v = 0;
    if (c < 2 * a.n)
#pragma unroll 8
        for (int g = s; g < groups; g += 8) v += a.part[int64_t(g) * 2 * a.n + c];
    lds[s][threadIdx.x % 32] = v;
    __syncthreads();
    if (s || c >= 2 * a.n) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) v += lds[i][threadIdx.x];
    if (c < a.n) {
        if (a.dweight) static_cast<T *>(a.dweight)[c] = T(v);
    } else if (a.dbias) {
        static_cast<T *>(a.dbias)[c - a.n] = T(v);
    }
}

int64_t grad_groups(int64_t rows) { return std::min<int64_t>(std::max<int64_t>(rows, 1), kGradGroups); }

}  // namespace

hipError_t launch_norm(int dtype, const NormArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const bool held = with_shape<T>(a.n, [&](auto l, auto nv) {
            constexpr int L = decltype(l)::value, NV = decltype(nv)::value;
            const int64_t blocks = std::min<int64_t>(ceil_div(a.rows, 256 / L), 1 << 20);
            // results that pass the caches by leave them to what is read: 32768 x 2048 bf16 46 us, through them 55
            if (2 * a.rows * a.n * int64_t(sizeof(T)) >= kPassingTraffic) norm_rows<T, L, NV, true><<<dim3(uint32_t(blocks)), 256, 0, stream>>>(a);
            else norm_rows<T, L, NV, false><<<dim3(uint32_t(blocks)), 256, 0, stream>>>(a);
        });
        if (!held) norm_long<T><<<dim3(uint32_t(std::min<int64_t>(a.rows, 1 << 20))), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

size_t norm_grad_bytes(int64_t rows, int64_t n) { return size_t(grad_groups(rows)) * 2 * size_t(n) * sizeof(float); }

hipError_t launch_norm_grad(int dtype, const NormGradArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const bool sums = a.dweight || a.dbias;
        int64_t groups = 0;
        const bool held = with_shape<T>(a.n, [&](auto l, auto nv) {
            constexpr int L = decltype(l)::value, NV = decltype(nv)::value;
            constexpr int R = kGradThreads / L;
            groups = std::min(ceil_div(a.rows, R), sums ? kGradGroups : int64_t(1) << 20);
            if (groups == 0) return;
            const bool passing = 3 * a.rows * a.n * int64_t(sizeof(T)) >= kPassingTraffic;      // 16384 x 2048 bf16: 47 us, else 50
            const dim3 grid(static_cast<uint32_t>(groups));
            if (sums && passing) norm_grad_rows<T, L, NV, true, true><<<grid, kGradThreads, 0, stream>>>(a);
            else if (sums) norm_grad_rows<T, L, NV, true, false><<<grid, kGradThreads, 0, stream>>>(a);
            else if (passing) norm_grad_rows<T, L, NV, false, true><<<grid, kGradThreads, 0, stream>>>(a);
            else norm_grad_rows<T, L, NV, false, false><<<grid, kGradThreads, 0, stream>>>(a);
        });
        if (!held) {
            if (a.dx && a.rows) norm_grad_long<T><<<dim3(uint32_t(std::min<int64_t>(a.rows, 1 << 20))), 256, 0, stream>>>(a);
            groups = std::min(a.rows, kLongGroups);
            if (groups && sums)
                norm_grad_columns<T><<<dim3(uint32_t(ceil_div(a.n, kLongCols)), uint32_t(groups)), kLongCols, 0, stream>>>(a);
        }
        if (sums) norm_grad_fold<T><<<dim3(uint32_t(ceil_div(2 * a.n, 32))), 256, 0, stream>>>(a, int(groups));
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
