// Matrix products of the projections, feed-forward and plain: C[m][n] = sum_k A[n][k] B[m][k] in tiles, from operands
// whose rows run along the sum or along C, with what is done to a result before it leaves its tile.
// 16-bit types are multiplied as they are.  product() has a float as three bf16 (8 + 8 +
// 8 bits, exactly) and adds up the six products down to 2^-14 of the largest in float: what
// is left out, the second part times the third and less, is below 2^-21 of a term (parts are cut, not
// rounded: a second part can be 2^-7 of the value, a third 2^-15, and what is left out has the term's
// sign), 2^-24 on average; bf16 products are 16 times the rate of float ones.  Norm-wise error 3 to 4 10^-7.
#pragma once
#include <algorithm>
#include <type_traits>

#include "ffn_cut.h"
#include "ops.h"
#include "ops_types.h"

namespace ndvm {
namespace ops {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
template <class T> struct Oct;
template <> struct Oct<bf16> { typedef bf16x8 type; };
template <> struct Oct<f16> { typedef f16x8 type; };

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Parts of a value in an operand: itself, or a float's three bf16.
template <class T> struct Parts {       // 16-bit types
    typedef T type;
    static constexpr int count = 1;
    static __device__ inline void split(float v, T *to) { to[0] = T(v); }
};
template <> struct Parts<float> {
    typedef bf16 type;
    static constexpr int count = 3;
    // cut, not rounded: each part takes the next 8 bits, and nothing overflows
    static __device__ inline void split(float v, bf16 *to) {
        const auto top = [](float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); };
        const float a = top(v);
        const float r = fabsf(v) <= 3.402823466e38f ? v - a : 0.0f;
        const float b = top(r);
        to[0] = bf16(v == v ? a : v);
        to[1] = bf16(b);
        to[2] = bf16(r - b);
    }
};

// ---- activations: value and derivative.  __expf rounds its argument's product with log2 e, and rcp is off by a unit: silu and
// sigmoid are off by (1 + |g|) 2^-21 of themselves at most, of a float result too.
template <int ACT> __device__ inline void act_both(float g, float &f, float &d) {
    if constexpr (ACT == NDVM_ACT_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
        f = g * s;
        d = s * (1.0f + g * (1.0f - s));
    } else if constexpr (ACT == NDVM_ACT_GELU) {
        const float p = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
        f = g * p;
        d = p + g * 0.39894228040143268f * __expf(-0.5f * g * g);
    } else if constexpr (ACT == NDVM_ACT_SIGMOID) {
        f = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
        d = f * (1.0f - f);
    } else if constexpr (ACT == NDVM_ACT_RELU) {
        f = g > 0.0f ? g : g != g ? g : 0.0f;
        d = g > 0.0f ? 1.0f : 0.0f;
    } else {
        f = g;
        d = 1.0f;
    }
}
// ... of what is stored in 16 bits: the normal distribution at -x <= 0 is exp(-x^2 / 2) t P(t), t = 1 / (1 + 0.36 x), P fitted to
// it with weights 1 / itself: off by 9.2e-7 of the value at most up to x = 13, where it leaves float's range; the exponent is rounded
// twice, which is up to (x^2 + 14) 2^-24 more (emulated, 1.8e-6 of the value in all up to 5, 7.2e-6 up to 13).  (erff, for both
// signs' ranges, was 60 instructions of a value: 8192 x 2048 x 8192 of 8-bit rows 234 us with it, 200 without.)
template <class T, int ACT> __device__ inline void act_of(float g, float &f, float &d) {
    if constexpr (ACT == NDVM_ACT_GELU && sizeof(T) == 2) {
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.36f * fabsf(g)), e = __expf(-0.5f * g * g);
        float q = 0.047056444f;
        q = q * t - 0.17976522f;
        q = q * t + 0.18095469f;
        q = q * t + 0.026548903f;
        q = q * t + 0.1397194f;
        q = q * t + 0.14177243f;
        q = q * t + 0.14371304f;
        q = q * t * e;
        const float p = g > 0.0f ? 1.0f - q : q;
        f = g * p;
        d = p + g * 0.39894228040143268f * e;
    } else {
        act_both<ACT>(g, f, d);
    }
}
// Calls f with the activation as a constant: the branch is taken once, not for every value.
template <class F> __device__ __attribute__((always_inline)) inline void with_act(int act, F f) {
    using std::integral_constant;
    if (act == NDVM_ACT_SILU) f(integral_constant<int, NDVM_ACT_SILU>());
    else if (act == NDVM_ACT_GELU) f(integral_constant<int, NDVM_ACT_GELU>());
    else if (act == NDVM_ACT_SIGMOID) f(integral_constant<int, NDVM_ACT_SIGMOID>());
    else f(integral_constant<int, NDVM_ACT_RELU>());
}

// ... of a product that may have none.
template <class F> __device__ __attribute__((always_inline)) inline void with_act_or_none(int act, F f) {
    if (act == NDVM_ACT_NONE) f(std::integral_constant<int, NDVM_ACT_NONE>());
    else with_act(act, f);
}

// ---- operands laid out: a copy in parts, rows of `pad` values (zeros beyond the source's)
struct PackArgs {
    const void *from[3];
    void *to[3];
    int64_t rows[3], ld[3], plane[3];   // plane: elements between a value's parts
    int64_t cols, pad;                  // pad: a multiple of 64
};
// A thread eight values; blockIdx.y: which of the copies.
template <class T> __global__ void __launch_bounds__(256) pack(PackArgs a) {
    typedef typename Parts<T>::type P;
    typedef P p8 __attribute__((ext_vector_type(8)));
    constexpr int N = Parts<T>::count, V = kVec<T>;
    const int w = blockIdx.y;
    const int64_t per = a.pad / 8;
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < a.rows[w] * per; at += int64_t(gridDim.x) * 256) {
        const int64_t r = at / per, c = at % per * 8;
        const T *from = static_cast<const T *>(a.from[w]) + r * a.ld[w] + c;
        p8 part[N];
#pragma unroll
        for (int j = 0; j < 8 / V; ++j) {
            vec<T> v = T(0.0f);
            if (c + j * V < a.cols) v = load_vec(from + j * V, a.cols - c - j * V);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                P q[N];
                Parts<T>::split(float(v[i]), q);
#pragma unroll
                for (int k = 0; k < N; ++k) part[k][j * V + i] = q[k];
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) *reinterpret_cast<p8 *>(static_cast<P *>(a.to[w]) + k * a.plane[w] + r * a.pad + c) = part[k];
    }
}

// ---- the product
struct Operand {
    const void *p;
    int64_t rows, ld, plane;
};
struct ProductArgs {
    Operand a, a2, b;           // a2: gated, the second weight; plain, what follows `a` along the sum from k2 on
    int64_t k, k2;              // the sum's length, a multiple of 8 (of 64 where an operand runs along C)
    int64_t tiles_n, tiles_m;
    int splits;                 // workgroups that share a tile's sum
    float *part;                // with splits: [splits][m][n], what each sums up (gated: [splits][m][2][pad_n])
    int act;
    // plain: rows m < split go to out + m * ld, those from split2 to m2 to out2 + (m - split2) * ld2
    void *out, *out2;
    int64_t ld, ld2, n, m, split, split2, m2;
    // linear: y = act(x w^T + bias) + residual; either may be null
    const void *bias, *residual;
    int64_t ld_r;
    const float *x_scale, *w_scale;     // of 8-bit rows of x and of w, or null
    // gradient
    const void *dh;             // of h, or of y

    int64_t ld_dh;
    void *p;                    // [m][dg du], or [m][dz], each padded with zeros to pad_n, in parts
    int64_t ld_p, plane_p;
    int64_t pad_n;              // n_out padded to a multiple of 64
    unsigned *largest;          // gradient in half: see scale_of
    int again;
    float *sums;                // [every 64 rows][pad_n]: their sums of dz in float, as it is before it is rounded; or null
};
enum Kind { kGated, kGatedGrad, kPlain, kLinear, kLinearGrad };
constexpr bool of_two(Kind k) { return k == kGated || k == kGatedGrad; }
constexpr bool with_slope(Kind k) { return k == kGatedGrad || k == kLinearGrad; }

#ifdef __HIP_DEVICE_COMPILE__
typedef short s16x4 __attribute__((ext_vector_type(4)));
// Lane 4 r + x of 16 names four values of row r; lane i gets column i of the four rows.
template <class O> __device__ inline O read_transposed(const char *p, const char *q) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const auto four = [](const char *at) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at)); };
    return __builtin_bit_cast(O, s16x8(__builtin_shufflevector(four(p), four(q), 0, 1, 2, 3, 4, 5, 6, 7)));
}
#endif

// dg and du are rounded to the tensors' type: in two parts the two products that take them would be twice the
// work (4096 x 1024 x 4096 bf16: 124 us of 204).  A half has not the range for that: dh u act' of halves can pass
// 65504, and small ones fall below 2^-24.  So the first pass over a gradient in half notes the largest value of
// dg and du that is finite (`largest`, its bits; a maximum does not depend on the order of the atomics); where that is
// not between 1 and 2^15, a second pass writes them again times a power of two that brings it there, and
// the products are divided by it.  A value is then off by at most 2^-11 of itself or 2^-25 of the largest.
// Calls within the range pay for a clear and for a pass that returns: 4096 x 1024 x 4096 249 us,
// 241 without them; out of it 301.
__device__ inline float scale_of(const ProductArgs &A) {
    if (!A.largest) return 1.0f;        // operands that were halves before
    const unsigned bits = *A.largest;
    const int e = int(bits >> 23) - 127;
    return bits == 0 || (e >= 0 && e < 15) ? 1.0f : __uint_as_float(unsigned(min(14 - e, 100) + 127) << 23);
}
template <class T> __device__ inline float unscaled(const ProductArgs &A) {
    if constexpr (std::is_same<T, f16>::value) return 1.0f / scale_of(A);
    return 1.0f;
}
// Whether a pass over dg and du has to write anything.
template <class T, Kind KIND> __device__ inline bool nothing_to_do(const ProductArgs &A) {
    if constexpr (std::is_same<T, f16>::value && with_slope(KIND)) return A.again && scale_of(A) == 1.0f;
    return false;
}
__device__ inline void note_largest(const ProductArgs &A, float top) {
    if (A.again) return;
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    const unsigned bits = __float_as_uint(top);
    if (threadIdx.x % 64 == 0 && bits > __hip_atomic_load(A.largest, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(A.largest, bits);
}
__global__ void clear_largest(unsigned *p) { *p = 0; }

// What becomes of eight columns (n on) of a row of g and u: h, or dg and du.  top: the largest of these so far.
template <class T, Kind KIND, int ACT> __device__ __attribute__((always_inline)) inline void gated_out(const ProductArgs &A, int64_t m, int64_t n, const float (&g)[8], const float (&u)[8], float scale, float &top) {
    constexpr bool RANGED = std::is_same<T, f16>::value && KIND == kGatedGrad;
    typedef typename Parts<T>::type P;
    constexpr int PARTS = Parts<T>::count;
    typedef T eight __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    typedef P eight_p __attribute__((ext_vector_type(8)));
    if constexpr (KIND == kGated) {
        T *row = static_cast<T *>(A.out) + m * A.ld;
        eight v;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float value, slope;
            act_both<ACT>(g[r], value, slope);
            v[r] = T(value * u[r]);
        }
        if (n + 8 <= A.n) *reinterpret_cast<eight *>(row + n) = v;
        else
            for (int r = 0; r < 8; ++r)
                if (n + r < A.n) row[n + r] = v[r];
    } else {
        if (n >= A.pad_n) return;
        const T *row = static_cast<const T *>(A.dh) + m * A.ld_dh + n;
        eight dh = T(0.0f);
        if (n + 8 <= A.n) dh = *reinterpret_cast<const eight *>(row);
        else
            for (int r = 0; r < 8; ++r)
                if (n + r < A.n) dh[r] = row[r];
        eight_p vg[PARTS], vu[PARTS];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float value, slope;
            act_both<ACT>(g[r], value, slope);
            P pg[PARTS], pu[PARTS];
            // what lies beyond the operands is 0, whatever act does there
            const bool there = n + r < A.n;
            float dg = there ? float(dh[r]) * u[r] * slope : 0.0f, du = there ? float(dh[r]) * value : 0.0f;
            if constexpr (RANGED) {
                const float a = fabsf(dg), b = fabsf(du);
                top = fmaxf(top, fmaxf(a <= 3.402823466e38f ? a : 0.0f, b <= 3.402823466e38f ? b : 0.0f));
                dg *= scale;
                du *= scale;
            }
            Parts<T>::split(dg, pg);
            Parts<T>::split(du, pu);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) {
                vg[q][r] = pg[q];
                vu[q][r] = pu[q];
            }
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            P *p = static_cast<P *>(A.p) + q * A.plane_p + m * A.ld_p + n;
            *reinterpret_cast<eight_p *>(p) = vg[q];
            *reinterpret_cast<eight_p *>(p + A.pad_n) = vu[q];
        }
    }
}

// ... of a row of x w^T: y, or dz = dy act'(z), which is left in z too, in float.
template <class T, Kind KIND, int ACT> __device__ __attribute__((always_inline)) inline void linear_out(const ProductArgs &A, int64_t m, int64_t n, float (&z)[8], float scale, float &top) {
    constexpr bool RANGED = std::is_same<T, f16>::value && KIND == kLinearGrad;
    typedef typename Parts<T>::type P;
    constexpr int PARTS = Parts<T>::count;
    typedef T eight __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    typedef P eight_p __attribute__((ext_vector_type(8)));
    const bool all = n + 8 <= A.n;
    const auto read = [&](const void *row) __attribute__((always_inline)) {
        eight v = T(0.0f);
        const T *p = static_cast<const T *>(row) + n;
        if (all) v = *reinterpret_cast<const eight *>(p);
        else
            for (int r = 0; r < 8; ++r)
                if (n + r < A.n) v[r] = p[r];
        return v;
    };
    eight bias = T(0.0f);
    if (A.bias) bias = read(A.bias);
    if constexpr (KIND == kLinear) {
        float x_scale = 1.0f, w_scale[8];
        if (A.x_scale) {
            x_scale = A.x_scale[m];
            typedef float eight_f __attribute__((ext_vector_type(8), aligned(4)));
            if (all) {
                const eight_f all_of_them = *reinterpret_cast<const eight_f *>(A.w_scale + n);
#pragma unroll
                for (int r = 0; r < 8; ++r) w_scale[r] = all_of_them[r];
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r) w_scale[r] = A.w_scale[min(n + r, A.n - 1)];
            }
        }
        eight more = T(0.0f), v;
        if (A.residual) more = read(static_cast<const T *>(A.residual) + m * A.ld_r);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float value, slope;
            const float sum = A.x_scale ? z[r] * x_scale * w_scale[r] : z[r];
            act_of<T, ACT>(A.bias ? sum + float(bias[r]) : sum, value, slope);
            v[r] = T(A.residual ? value + float(more[r]) : value);
        }
        T *row = static_cast<T *>(A.out) + m * A.ld;
        if (all) *reinterpret_cast<eight *>(row + n) = v;
        else
            for (int r = 0; r < 8; ++r)
                if (n + r < A.n) row[n + r] = v[r];
    } else {
        if (n >= A.pad_n) return;
        const eight dy = read(static_cast<const T *>(A.dh) + m * A.ld_dh);
        eight_p v[PARTS];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            float value, slope;
            act_of<T, ACT>(z[r] + float(bias[r]), value, slope);
            // what lies beyond the operands is 0, whatever act does there
            float dz = n + r < A.n ? float(dy[r]) * slope : 0.0f;
            z[r] = dz;
            if constexpr (RANGED) {
                const float a = fabsf(dz);
                top = fmaxf(top, a <= 3.402823466e38f ? a : 0.0f);
                dz *= scale;
            }
            P p[PARTS];
            Parts<T>::split(dz, p);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) v[q][r] = p[q];
        }
#pragma unroll
        for (int q = 0; q < PARTS; ++q) *reinterpret_cast<eight_p *>(static_cast<P *>(A.p) + q * A.plane_p + m * A.ld_p + n) = v[q];
    }
}

#ifdef __HIP_DEVICE_COMPILE__
// ROWS rows of COLS columns of a linear product, from the wave's own LDS (rows of COLS + 4 floats) to memory: eight
// columns a lane, so that whole rows are read and written, and one copy of the code for all of a wave's accumulators.
// Of a gradient, each lane's sums of dz lie behind the stage: in registers they are spilled beside the accumulators.
template <Kind KIND, int ROWS, int COLS> constexpr int kStage = ROWS * (COLS + 4) + (KIND == kLinearGrad ? 512 : 0);
template <class T, Kind KIND, int ROWS, int COLS> struct Leaving {
    const ProductArgs &A;
    const int part;
    float *stage;
    float scale;
    bool summed;
    __device__ inline f32x4 *own() const { return reinterpret_cast<f32x4 *>(stage + ROWS * (COLS + 4)) + threadIdx.x % 64; }
    __device__ inline Leaving(const ProductArgs &a, int p, float *s) : A(a), part(p), stage(s) {
        scale = std::is_same<T, f16>::value && KIND == kLinearGrad && a.again && a.splits == 1 ? scale_of(a) : 1.0f;
        summed = KIND == kLinearGrad && a.sums && a.splits == 1 && !a.again;
        if (summed) own()[0] = own()[64] = 0;
    }
    // m0, n0: where they lie in C
    __device__ __attribute__((always_inline)) inline void rows(int64_t m0, int64_t n0, float &top) const {
        constexpr int PER = COLS / 8;
        static_assert(64 % PER == 0, "a lane has the same columns in every row");
        asm volatile("" ::: "memory");      // other lanes' values: a wave's accesses to LDS are in order
#pragma unroll 1
        for (int at = threadIdx.x % 64; at < ROWS * PER; at += 64) {
            const f32x4 *from = reinterpret_cast<const f32x4 *>(stage + at / PER * (COLS + 4) + at % PER * 8);
            const f32x4 u = from[0], v = from[1];
            const int64_t m = m0 + at / PER, n = n0 + at % PER * 8;
            if (m >= A.m || n >= (KIND == kLinear && A.splits == 1 ? A.n : A.pad_n)) continue;
            if (A.splits > 1) {
                f32x4 *to = reinterpret_cast<f32x4 *>(A.part + (int64_t(part) * A.m + m) * A.pad_n + n);
                to[0] = u;
                to[1] = v;
                continue;
            }
            float z[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
            with_act_or_none(A.act, [&](auto act) __attribute__((always_inline)) { linear_out<T, KIND, decltype(act)::value>(A, m, n, z, scale, top); });
            if (summed) {
                own()[0] += f32x4{z[0], z[1], z[2], z[3]};
                own()[64] += f32x4{z[4], z[5], z[6], z[7]};
            }
        }
        asm volatile("" ::: "memory");
    }
    // The wave's 64 rows m0 on, added up.
    __device__ inline void sums(int64_t m0, int64_t n0) const {
        constexpr int PER = COLS / 8;
        if (!summed) return;
        f32x4 u = own()[0], v = own()[64];
#pragma unroll
        for (int s = PER; s < 64; s <<= 1)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                u[r] += __shfl_xor(u[r], s);
                v[r] += __shfl_xor(v[r], s);
            }
        const int l = threadIdx.x % 64;
        const int64_t n = n0 + l % PER * 8;
        if (l >= PER || m0 >= A.m || n >= A.pad_n) return;
        f32x4 *to = reinterpret_cast<f32x4 *>(A.sums + m0 / 64 * A.pad_n + n);
        to[0] = u;
        to[1] = v;
    }
};
__device__ inline void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
#endif

// BA columns n by BB rows m a workgroup; NA x NB waves.  ALONG_B: the rows of B run along
// C (B[k][m]); those of A do in a plain product (A[k][n]).
// An LDS tile of an operand is 32 long along the sum: rows of 32 values, or 32 rows along C,
// in granules of 16 bytes.  Along the sum granule i of row r lies at place i ^ (r / 4 % 4), along
// C at i ^ 2 (r % 4 + r / 8 % 2 * 4) (such rows are read two granules at a time), so that the 16 rows
// an instruction reads are in different banks.  The loads go to LDS directly and choose
// their source accordingly; what is out of range reads as 0.
// Four tiles are in LDS: while one is multiplied, from registers, the next is read into
// registers and three more are on their way, so neither latency is waited for (8192 x 2048 x
// 8192: 492 us with two tiles of 64 read as they are multiplied).
#ifdef __HIP_DEVICE_COMPILE__       // the host's pass does not know the types of the loads to LDS
template <class T, int BA, int BB, int NA, int NB, Kind KIND, bool ALONG_B>
__device__ __attribute__((always_inline)) inline void product_tile(const ProductArgs &A, int64_t id, char *buffer0, char *buffer1, char *buffer2, char *buffer3) {
    typedef typename Parts<T>::type P;
    typedef typename Oct<P>::type oct;
    constexpr int PARTS = Parts<T>::count, PAIRS = PARTS == 1 ? 1 : 6, W = NA * NB;
    constexpr int WA = BA / NA, WB = BB / NB, TA = WA / 16, TB = WB / 16;
    constexpr bool GATED = of_two(KIND), ALONG_A = KIND == kPlain;
    constexpr int COLS = GATED ? BA / 2 : BA;       // columns of C a tile has

    // Tiles in an order that keeps an XCD (workgroup % 8) on neighbouring ones: its share
    // of the tiles, in bands of 8 tile rows.
    const int64_t tiles = A.tiles_n * A.tiles_m;
    {
        const int64_t total = tiles * A.splits, x = id % 8, per = total / 8, more = total % 8;
        id = x * per + min(x, more) + id / 8;
    }
    const int part = int(id / tiles);
    id %= tiles;
    const int64_t band = id / (8 * A.tiles_n), in = id % (8 * A.tiles_n);
    const int64_t tall = min(int64_t(8), A.tiles_m - band * 8);
    const int64_t m0 = (band * 8 + in % tall) * BB, n0 = in / tall * COLS;

    const int l = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lm = l % 16, lg = l / 16, wa = wave / NB, wb = wave % NB;
    constexpr unsigned kNowhere = 0x80000000u;
    const auto rsrc = [](const void *p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, 0x7fffffff, 0x00020000); };
    const auto f = [](int row) { return row % 4 + row / 8 % 2 * 4; };

    // Wave-wide loads of 1 KB.  Along the sum: 16 rows of 4 granules.
    constexpr int LA = BA / 16 / W, LB = BB / 16 / W;
    const int sub = l / 4, granule = (l % 4) ^ (sub / 4);
    // Along C: rows of R / 8 granules, 512 / R rows a load.
    // A load's rows are 512 W / R after those of the load before, which is a multiple of 16: the same f.
    const auto along_row = [&](int R) { return wave * (512 / R) + l / (R / 8); };
    const auto along_col = [&](int R) { return ((l % (R / 8)) ^ 2 * f(along_row(R))) * 8; };
    static_assert(512 * W / BA % 16 == 0 && 512 * W / BB % 16 == 0, "");
    unsigned at_a[LA], at_b[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        if constexpr (ALONG_A) {
            const int col = along_col(BA);
            at_a[i] = n0 + col < A.n ? unsigned(along_row(BA) * A.a.ld + col) * 2 : kNowhere;
        } else {
            const int row = (wave + W * i) * 16 + sub;
            const bool second = GATED && row % WA >= WA / 2;
            const int r = GATED ? row / WA * (WA / 2) + row % (WA / 2) : row;
            at_a[i] = n0 + r < A.a.rows ? unsigned(r * (second ? A.a2.ld : A.a.ld) + granule * 8) * 2 : kNowhere;
        }
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        if constexpr (ALONG_B) {
            const int col = along_col(BB);
            at_b[i] = m0 + col < A.m ? unsigned(along_row(BB) * A.b.ld + col) * 2 : kNowhere;
        } else {
            const int row = (wave + W * i) * 16 + sub;
            at_b[i] = m0 + row < A.b.rows ? unsigned(row * A.b.ld + granule * 8) * 2 : kNowhere;
        }
    }
    const int steps = int((A.k + kStep - 1) / kStep);
    // this workgroup's share of the sum
    const int first = int(int64_t(steps) * PAIRS * part / A.splits), total = int(int64_t(steps) * PAIRS * (part + 1) / A.splits);
    // Where the next tiles to load begin: moved on from step to step, or worked out again where there are
    // pairs of parts (small products first: the large ones' sum is then rounded in a sixth of the steps;
    // 1289 x 2668 x 1028 5.0e-7 of the result, largest first 1.2e-6).  No branches: the accumulators would be moved about at each.
    const P *next_a = nullptr, *next_a2 = nullptr, *next_b = nullptr;
    int left = 0;               // of the sum, from there to the end of these operands
    int rows_a = 0, rows_b = 0; // rows there are from there on, for operands along C
    int at = first;             // the step
    const auto find = [&]() __attribute__((always_inline)) {
        constexpr int pair_a[6] = {2, 0, 1, 1, 0, 0}, pair_b[6] = {0, 2, 1, 0, 1, 0};     // small products first
        int pa = 0, pb = 0;
        int64_t k0 = int64_t(at) * kStep;
        if (PAIRS > 1) {
            const int pair = at / steps;
            k0 = int64_t(at % steps) * kStep;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i)
                if (i == pair) pa = pair_a[i], pb = pair_b[i];
        }
        const bool after = ALONG_A && k0 >= A.k2;
        const Operand &o = after ? A.a2 : A.a;
        const int64_t k1 = after ? k0 - A.k2 : k0;
        next_a = static_cast<const P *>(o.p) + pa * o.plane + (ALONG_A ? k1 * o.ld + n0 : n0 * o.ld + k0);
        if (GATED) next_a2 = static_cast<const P *>(A.a2.p) + pa * A.a2.plane + n0 * A.a2.ld + k0;
        next_b = static_cast<const P *>(A.b.p) + pb * A.b.plane + (ALONG_B ? k0 * A.b.ld + m0 : m0 * A.b.ld + k0);
        left = int((ALONG_A && !after ? A.k2 : A.k) - k0);
        rows_a = int(min(o.rows - k1, int64_t(1) << 30));
        rows_b = int(min(A.b.rows - k0, int64_t(1) << 30));
    };
    const unsigned apart_a = ALONG_A ? unsigned(512 * W / BA * A.a.ld) * 2 : 0, apart_b = ALONG_B ? unsigned(512 * W / BB * A.b.ld) * 2 : 0;
    // The next tile into `to`: always LA + LB loads a wave (past the end they fetch nothing).
    const auto load = [&](char *to) __attribute__((always_inline)) {
        if (PAIRS > 1) find();
        const bool some = at < total && granule * 8 < left;
        const int have_a = at < total ? rows_a : 0, have_b = at < total ? rows_b : 0;
        const auto r = rsrc(next_a), r2 = GATED ? rsrc(next_a2) : r, rb = rsrc(next_b);
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const bool second = GATED && (wave + W * i) * 16 % WA >= WA / 2;
            const bool there = ALONG_A ? along_row(BA) < have_a - 512 * W / BA * i : some;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second ? r2 : r, (__attribute__((address_space(3))) void *)(to + (wave + W * i) * 1024), 16,
                                                     there ? at_a[i] : kNowhere, apart_a * i, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const bool there = ALONG_B ? along_row(BB) < have_b - 512 * W / BB * i : some;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (__attribute__((address_space(3))) void *)(to + BA * 64 + (wave + W * i) * 1024), 16,
                                                     there ? at_b[i] : kNowhere, apart_b * i, 0, 0);
        }
        ++at;
        if (PAIRS > 1) return;
        left -= kStep;
        next_a += ALONG_A ? kStep * A.a.ld : kStep;
        if (GATED) next_a2 += kStep;
        next_b += ALONG_B ? kStep * A.b.ld : kStep;
        rows_a -= kStep;
        rows_b -= kStep;
        if (ALONG_A && !ALONG_B) {      // on to what follows along the sum
            const bool wrap = left <= 0;
            next_a = wrap ? static_cast<const P *>(A.a2.p) + n0 : next_a;
            rows_a = wrap ? int(A.a2.rows) : rows_a;
            left = wrap ? int(A.k - A.k2) : left;
        }
    };

    f32x4 acc[TA][TB];
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = 0;
    const int tr_row = 8 * lg + lm / 4;     // (+ 4: the same f)
    // One set of A's registers: a tile's is free for the next step's once its row of products is
    // under way.  Two of B's.
    oct fa[TA], fb[2][TB];
    // Where a lane's values of the first 16 rows of an operand's tile lie: along the sum, in tiles of
    // even and of odd number (gated: rows of a pair of tiles are in the order that leaves a lane with eight
    // columns side by side); along C, the row and the granule's place, to be crossed with the columns'.
    // Kept from the compiler's sight, or it works out the address of every read of every buffer
    // ahead of the loop, which has no registers for them.
    struct Places {
        int a0, a1, b;
    };
    const auto places = [&]() __attribute__((always_inline)) {
        const int row_a = lm / 4 * 8 + lm % 4, row_b = lm, crossed = (lm % 4 / 2 ^ 2 * f(tr_row)) * 16;
        Places p;
        if constexpr (ALONG_A) p = Places{crossed, tr_row * BA * 2 + lm % 2 * 8, crossed};
        else p = Places{(wa * WA + row_a) * 64 + (lg ^ row_a / 4 % 4) * 16, (wa * WA + row_a + 4) * 64 + (lg ^ (row_a + 4) / 4 % 4) * 16, 0};
        if constexpr (ALONG_B) p.b = tr_row * BB * 2 + lm % 2 * 8;
        else p.b = (wb * WB + row_b) * 64 + (lg ^ row_b / 4 % 4) * 16;
        asm volatile("" : "+v"(p.a0), "+v"(p.a1), "+v"(p.b));
        return p;
    };
    const auto read_a = [&](const char *from, int i, const Places &p) __attribute__((always_inline)) {
        if constexpr (ALONG_A) {
            const char *at = from + p.a1 + ((wa * WA + i * 16) * 2 ^ p.a0);
            fa[i] = read_transposed<oct>(at, at + 4 * BA * 2);
        } else {
            fa[i] = *reinterpret_cast<const oct *>(from + (i % 2 ? p.a1 : p.a0) + i / 2 * (32 * 64));
        }
    };
    const auto read_b = [&](const char *from, oct &to, int j, const Places &p) __attribute__((always_inline)) {
        if constexpr (ALONG_B) {
            const char *at = from + BA * 64 + p.b + ((wb * WB + j * 16) * 2 ^ p.a0);
            to = read_transposed<oct>(at, at + 4 * BB * 2);
        } else {
            to = *reinterpret_cast<const oct *>(from + BA * 64 + p.b + j * (16 * 64));
        }
    };
    constexpr int LOADS = LA + LB;
    static_assert(3 * LOADS < 16, "");
    const auto wait = [&](auto loads) __attribute__((always_inline)) {
        // this wave's older loads have landed and its reads are done; after the barrier everybody's
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);      // multiplications stay on their side
        __builtin_amdgcn_s_waitcnt(0x0070 | decltype(loads)::value);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    using std::integral_constant;
    // A step: its operands are in registers (B's in set `now`); the next tile is in `next`; the tile
    // four on takes its own place, `to`
    const auto step = [&](const char *next, char *to, auto now) __attribute__((always_inline)) {
        constexpr int n = decltype(now)::value;
        wait(integral_constant<int, 2 * LOADS>());
        load(to);
        const Places place = places();
        static_assert(TB <= TA, "");
#pragma unroll
        for (int i = 0; i < TA; ++i) {
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = mfma(fa[i], fb[n][j], acc[i][j]);
            if (i < TB) read_b(next, fb[1 - n][i], i, place);
            read_a(next, i, place);
        }
        // loads and reads among the multiplications, none of which waits for them
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, TB, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, (LOADS + TB - 1) / TB, 0);
            if (ALONG_A) __builtin_amdgcn_sched_group_barrier(0x002, 1 + ALONG_B, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, (ALONG_A ? 2 : 1) + (ALONG_B ? 2 : 1), 0);
        }
#pragma unroll
        for (int i = TB; i < TA; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, TB, 0);
            if (ALONG_A) __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, ALONG_A ? 2 : 1, 0);
        }
    };
    if (first < total) {
        find();
        load(buffer0);
        load(buffer1);
        load(buffer2);
        load(buffer3);
        wait(integral_constant<int, 3 * LOADS>());
        const Places place = places();
#pragma unroll
        for (int i = 0; i < TA; ++i) {
            if (i < TB) read_b(buffer0, fb[0][i], i, place);
            read_a(buffer0, i, place);
        }
        const integral_constant<int, 0> even;
        const integral_constant<int, 1> odd;
        for (int s = first; s < total; s += 4) {    // steps past the end add zeros
            step(buffer1, buffer0, even);
            step(buffer2, buffer1, odd);
            step(buffer3, buffer2, even);
            step(buffer0, buffer3, odd);
        }
        // the loads past the end fetch nothing, but write zeros to LDS, which has to be this workgroup's still
        __builtin_amdgcn_s_waitcnt(0x0f70);
    }

    const float unscale = KIND == kPlain ? unscaled<T>(A) : 1.0f;
    // lane l, register r of tile (i, j): row m = l % 16 of j; column 4 (l / 16) + r of i, or, where both
    // operands run along the sum, 8 (l / 16) + 4 (i % 2) + r of the pair of tiles
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int64_t m = m0 + wb * WB + j * 16 + lm;
        if constexpr (KIND == kPlain) {
            typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            if (A.splits > 1) {
                typedef float four_f __attribute__((ext_vector_type(4), aligned(4)));
                if (m >= A.m) continue;
                float *row = A.part + (int64_t(part) * A.m + m) * A.n;
#pragma unroll
                for (int i = 0; i < TA; ++i) {
                    const int64_t n = n0 + wa * WA + i * 16 + lg * 4;
                    if (n + 4 <= A.n) *reinterpret_cast<four_f *>(row + n) = acc[i][j];
                    else
                        for (int r = 0; r < 4; ++r)
                            if (n + r < A.n) row[n + r] = acc[i][j][r];
                }
                continue;
            }
            T *row = nullptr;
            if (m < A.split) row = static_cast<T *>(A.out) + m * A.ld;
            else if (m >= A.split2 && m < A.m2) row = static_cast<T *>(A.out2) + (m - A.split2) * A.ld2;
            if (!row) continue;
#pragma unroll
            for (int i = 0; i < TA; ++i) {
                const int64_t n = n0 + wa * WA + i * 16 + lg * 4;
                four v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = T(acc[i][j][r] * unscale);
                if (n + 4 <= A.n) *reinterpret_cast<four *>(row + n) = v;
                else
                    for (int r = 0; r < 4; ++r)
                        if (n + r < A.n) row[n + r] = v[r];
            }
        }
    }
    if constexpr (KIND == kLinear || KIND == kLinearGrad) {
        constexpr int STAGE = kStage<KIND, 16, WA>;
        static_assert(STAGE * 4 * W / 4 <= (BA + BB) * kStep * 2, "");
        float *stage = reinterpret_cast<float *>(wave % 4 == 0 ? buffer0 : wave % 4 == 1 ? buffer1 : wave % 4 == 2 ? buffer2 : buffer3) + wave / 4 * STAGE;
        meet();     // the buffers are everybody's until here
        float top = 0;
        Leaving<T, KIND, 16, WA> leaving(A, part, stage);
#pragma unroll 1
        for (int j = 0; j < TB; ++j) {
#pragma unroll
            for (int c = 0; c < TB; ++c)
                if (c == j)
#pragma unroll
                    for (int i = 0; i < TA; ++i) *reinterpret_cast<f32x4 *>(stage + lm * (WA + 4) + i / 2 * 32 + lg * 8 + i % 2 * 4) = acc[i][c];
            leaving.rows(m0 + wb * WB + j * 16, n0 + wa * WA, top);
        }
        if constexpr (KIND == kLinearGrad) {
            static_assert(WB == 64, "");
            leaving.sums(m0 + wb * WB, n0 + wa * WA);
        }
        if (std::is_same<T, f16>::value && KIND == kLinearGrad && A.splits == 1) note_largest(A, top);
    }
    if constexpr (GATED) {
        if (A.splits > 1) {
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                const int64_t m = m0 + wb * WB + j * 16 + lm;
                if (m >= A.m) continue;
#pragma unroll
                for (int i = 0; i < TA / 2; ++i) {
                    const int64_t n = n0 + wa * (WA / 2) + i / 2 * 32 + lg * 8 + i % 2 * 4;
                    if (n >= A.pad_n) continue;
                    float *to = A.part + (int64_t(part) * A.m + m) * 2 * A.pad_n + n;
                    *reinterpret_cast<f32x4 *>(to) = acc[i][j];
                    *reinterpret_cast<f32x4 *>(to + A.pad_n) = acc[i + TA / 2][j];
                }
            }
            return;
        }
        constexpr bool RANGED = std::is_same<T, f16>::value && KIND == kGatedGrad;
        const float scale = RANGED && A.again ? scale_of(A) : 1.0f;
        float top = 0;
        with_act(A.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                const int64_t m = m0 + wb * WB + j * 16 + lm;
                if (m >= A.m) continue;
#pragma unroll
                for (int i = 0; i < TA / 2; i += 2) {
                    float g[8], u[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        g[r] = acc[i + r / 4][j][r % 4];
                        u[r] = acc[i + r / 4 + TA / 2][j][r % 4];
                    }
                    gated_out<T, KIND, decltype(act)::value>(A, m, n0 + wa * (WA / 2) + i * 16 + lg * 8, g, u, scale, top);
                }
            }
        });
        if (RANGED) note_largest(A, top);
    }
}
#endif

template <class T, int BA, int BB, int NA, int NB, Kind KIND>
__global__ void __launch_bounds__(64 * NA * NB) product(ProductArgs A) {
#ifdef __HIP_DEVICE_COMPILE__
    // separate arrays, so that the compiler sees that loads into one leave reads of the others alone
    constexpr int SIZE = (BA + BB) * kStep * 2;
    __shared__ __align__(1024) char buffer0[SIZE], buffer1[SIZE], buffer2[SIZE], buffer3[SIZE];
    if (nothing_to_do<T, KIND>(A)) return;
    product_tile<T, BA, BB, NA, NB, KIND, false>(A, blockIdx.x, buffer0, buffer1, buffer2, buffer3);
#endif
}

// Two plain products in one launch: dx = [dg du] [Wg; Wu], and [dWg; dWu] = [dg du]^T x.
template <class T, int BA, int BB, int NA, int NB>
__global__ void __launch_bounds__(64 * NA * NB) product_pair(ProductArgs A, ProductArgs B) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int SIZE = (BA + BB) * kStep * 2;
    __shared__ __align__(1024) char buffer0[SIZE], buffer1[SIZE], buffer2[SIZE], buffer3[SIZE];
    const int64_t of_a = A.tiles_n * A.tiles_m * A.splits;
    if (int64_t(blockIdx.x) < of_a) product_tile<T, BA, BB, NA, NB, kPlain, false>(A, blockIdx.x, buffer0, buffer1, buffer2, buffer3);
    else product_tile<T, BA, BB, NA, NB, kPlain, true>(B, blockIdx.x - of_a, buffer0, buffer1, buffer2, buffer3);
#endif
}

// The sums of a plain product that was split, added up in order.  A thread four columns.
template <class T> __global__ void __launch_bounds__(256) fold_splits(ProductArgs A) {
    typedef float four_f __attribute__((ext_vector_type(4), aligned(4)));
    const int64_t per = (A.n + 3) / 4, at = int64_t(blockIdx.x) * 256 + threadIdx.x, m = at / per, n = at % per * 4;
    if (m >= A.m) return;
    T *row = nullptr;
    if (m < A.split) row = static_cast<T *>(A.out) + m * A.ld;
    else if (m >= A.split2 && m < A.m2) row = static_cast<T *>(A.out2) + (m - A.split2) * A.ld2;
    if (!row) return;
    const float unscale = unscaled<T>(A);
    const float *p = A.part + m * A.n + n;
    if (n + 4 <= A.n) {
        f32x4 sum = *reinterpret_cast<const four_f *>(p);
        for (int i = 1; i < A.splits; ++i) sum += *reinterpret_cast<const four_f *>(p + i * A.m * A.n);
        typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        four v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = T(sum[r] * unscale);
        *reinterpret_cast<four *>(row + n) = v;
    } else {
        for (int r = 0; n + r < A.n; ++r) {
            float sum = p[r];
            for (int i = 1; i < A.splits; ++i) sum += p[i * A.m * A.n + r];
            row[n + r] = T(sum * unscale);
        }
    }
}

// ... of a gated product.  A thread eight columns.
template <class T, Kind KIND> __global__ void __launch_bounds__(256) fold_gated(ProductArgs A) {
#ifdef __HIP_DEVICE_COMPILE__
    if (nothing_to_do<T, KIND>(A)) return;
    constexpr bool RANGED = std::is_same<T, f16>::value && KIND == kGatedGrad;
    const float scale = RANGED && A.again ? scale_of(A) : 1.0f;
    float top = 0;
    const int64_t per = A.pad_n / 8, at = int64_t(blockIdx.x) * 256 + threadIdx.x, m = at / per, n = at % per * 8;
    if (m < A.m) {
        f32x4 sum[4] = {};
        for (int i = 0; i < A.splits; ++i) {
            const f32x4 *p = reinterpret_cast<const f32x4 *>(A.part + (i * A.m + m) * 2 * A.pad_n + n), *q = p + A.pad_n / 4;
            sum[0] += p[0];
            sum[1] += p[1];
            sum[2] += q[0];
            sum[3] += q[1];
        }
        with_act(A.act, [&](auto act) __attribute__((always_inline)) {
            float g[8], u[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                g[r] = sum[r / 4][r % 4];
                u[r] = sum[2 + r / 4][r % 4];
            }
            gated_out<T, KIND, decltype(act)::value>(A, m, n, g, u, scale, top);
        });
    }
    if (RANGED) note_largest(A, top);
#endif
}

// ... of a linear one.
__device__ inline void split_sums(const ProductArgs &A, int64_t m, int64_t n, float (&z)[8]) {
    f32x4 sum[2] = {};
    for (int i = 0; i < A.splits; ++i) {
        const f32x4 *p = reinterpret_cast<const f32x4 *>(A.part + (i * A.m + m) * A.pad_n + n);
        sum[0] += p[0];
        sum[1] += p[1];
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) z[r] = sum[r / 4][r % 4];
}
template <class T> __global__ void __launch_bounds__(256) fold_linear(ProductArgs A) {
#ifdef __HIP_DEVICE_COMPILE__
    float top = 0, z[8];
    const int64_t per = A.pad_n / 8, at = int64_t(blockIdx.x) * 256 + threadIdx.x, m = at / per, n = at % per * 8;
    if (m >= A.m || n >= A.n) return;
    split_sums(A, m, n, z);
    with_act_or_none(A.act, [&](auto act) __attribute__((always_inline)) { linear_out<T, kLinear, decltype(act)::value>(A, m, n, z, 1.0f, top); });
#endif
}
// ... and of its gradient's: 64 rows of 64 columns a workgroup, eight lanes a row.
template <class T> __global__ void __launch_bounds__(512) fold_linear_grad(ProductArgs A) {
#ifdef __HIP_DEVICE_COMPILE__
    if (nothing_to_do<T, kLinearGrad>(A)) return;
    constexpr bool RANGED = std::is_same<T, f16>::value;
    __shared__ float lds[8][64];
    const float scale = RANGED && A.again ? scale_of(A) : 1.0f;
    float top = 0, z[8] = {};
    const int l = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t per = A.pad_n / 64, m0 = blockIdx.x / per * 64, n0 = blockIdx.x % per * 64, n = n0 + l % 8 * 8, m = m0 + wave * 8 + l / 8;
    if (m < A.m) {
        split_sums(A, m, n, z);
        with_act_or_none(A.act, [&](auto act) __attribute__((always_inline)) { linear_out<T, kLinearGrad, decltype(act)::value>(A, m, n, z, scale, top); });
    }
    if (RANGED) note_largest(A, top);
    if (!A.sums || A.again) return;
#pragma unroll
    for (int s = 8; s < 64; s <<= 1)
#pragma unroll
        for (int r = 0; r < 8; ++r) z[r] += __shfl_xor(z[r], s);
    if (l < 8)
#pragma unroll
        for (int r = 0; r < 8; ++r) lds[wave][l * 8 + r] = z[r];
    __syncthreads();
    if (wave) return;
    float sum = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) sum += lds[w][l];
    A.sums[m0 / 64 * A.pad_n + n0 + l] = sum;
#endif
}

template <class T, int BA, int BB, int NA, int NB, Kind KIND> void launch_tiles(ProductArgs a, int64_t n, int64_t m, hipStream_t stream) {
    a.tiles_n = ceil_div(n, of_two(KIND) ? BA / 2 : BA);
    a.tiles_m = ceil_div(m, BB);
    const int64_t wgs = a.tiles_n * a.tiles_m * a.splits;
    if (wgs) product<T, BA, BB, NA, NB, KIND><<<dim3(uint32_t(wgs)), 64 * NA * NB, 0, stream>>>(a);
}

template <class T, Kind KIND> void launch_product(const Gated &c, ProductArgs a, int64_t n, int64_t m, hipStream_t stream) {
    constexpr bool RANGED = std::is_same<T, f16>::value && with_slope(KIND);
    if (RANGED) clear_largest<<<1, 1, 0, stream>>>(a.largest);
    a.splits = int(c.splits);
    const auto sums = [&]() {
        if (c.bb == 256) launch_tiles<T, 256, 256, 2, 4, KIND>(a, n, m, stream);
        else if (c.ba == 256) launch_tiles<T, 256, 128, 4, 2, KIND>(a, n, m, stream);
        else launch_tiles<T, 128, 128, 2, 2, KIND>(a, n, m, stream);
    };
    const auto fold = [&]() {
        const dim3 grid(uint32_t(ceil_div(a.pad_n / 8 * a.m, 256)));
        if constexpr (of_two(KIND)) fold_gated<T, KIND><<<grid, 256, 0, stream>>>(a);
        else if constexpr (KIND == kLinear) fold_linear<T><<<grid, 256, 0, stream>>>(a);
        else fold_linear_grad<T><<<dim3(uint32_t(a.pad_n / 64 * ceil_div(a.m, 64))), 512, 0, stream>>>(a);
    };
    sums();
    if (c.splits > 1) fold();
    if (!RANGED) return;
    a.again = 1;        // split sums are still there
    if (c.splits > 1) fold();
    else sums();
}

template <class T, int BT, int NA, int NB> void launch_pair(ProductArgs a, ProductArgs b, hipStream_t stream) {
    for (ProductArgs *q : {&a, &b}) {
        q->tiles_n = ceil_div(q->n, BT);
        q->tiles_m = ceil_div(q->m, BT);
    }
    const int64_t wgs = a.tiles_n * a.tiles_m * a.splits + b.tiles_n * b.tiles_m * b.splits;
    if (wgs) product_pair<T, BT, BT, NA, NB><<<dim3(uint32_t(wgs)), 64 * NA * NB, 0, stream>>>(a, b);
    for (const ProductArgs *q : {&a, &b})
        if (q->splits > 1 && q->m && q->n) fold_splits<T><<<dim3(uint32_t(ceil_div(ceil_div(q->n, 4) * q->m, 256))), 256, 0, stream>>>(*q);
}

int64_t pad64(int64_t n) { return ceil_div(n, 64) * 64; }

// An operand that product() reads as it is: rows of 16-byte granules.
bool direct(int dtype, const void *p, int64_t ld, int64_t k) {
    return dtype != NDVM_F32 && ld <= kMostFfnWidth && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && k % 8 == 0;
}

// Workspace of a call: the parts that it may need, one after the other.
struct Space {
    char *base;
    size_t used = 0;
    int64_t plane = 0;
    explicit Space(void *p) : base(static_cast<char *>(p)) {}
    void *take(int dtype, int64_t rows, int64_t cols) {
        plane = rows * cols;
        void *p = base ? base + used : nullptr;
        used += round256(size_t(plane) * (dtype == NDVM_F32 ? 6 : 2));
        return p;
    }
    float *take_floats(int64_t n) {
        void *p = base ? base + used : nullptr;
        used += round256(size_t(n) * 4);
        return static_cast<float *>(p);
    }
};

char *aligned(void *p) { return reinterpret_cast<char *>(round256(reinterpret_cast<size_t>(p))); }

}  // namespace
}  // namespace ops
}  // namespace ndvm
