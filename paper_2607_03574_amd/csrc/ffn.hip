// Gated feed-forward projections and their gradient.
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u
//   dg = dh u act'(g),  du = dh act(g),  dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x
// Matrix products throughout: bound by the matrix instructions for many rows, by
// reading the weights for few.  One kernel, product(), computes C[m][n] = sum_k A[n][k]
// B[m][k] from operands whose rows run along the sum or along C:
//  - forward: a tile holds the same columns of both weights, so act(g) u is formed in
//    the accumulators and g and u never reach memory;
//  - gradient: g and u are formed again the same way (reading them back would cost their
//    rounding; the two products are a third of the work), and dg, du leave the tile as
//    one operand [rows][2 n_out] of dx = [dg du] [Wg; Wu] and [dWg; dWu] = [dg du]^T x.
//    Operands that run along C are turned by the transposing reads from LDS: nothing is
//    transposed in memory.
// Few rows have a kernel of their own, few(), that reads weights straight into the
// matrix instructions' registers.
// 16-bit types are multiplied as they are.  product() has a float as three bf16 (8 + 8 +
// 8 bits, exactly) and adds up the six products down to 2^-14 of the largest in float: what
// is left out, the second part times the third and less, is below 2^-21 of a term (parts are cut, not
// rounded: a second part can be 2^-7 of the value, a third 2^-15, and what is left out has the term's
// sign), 2^-24 on average; bf16 products are 16 times the rate of float ones.  Norm-wise error 3 to 4 10^-7.
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

// ---- activations: value and derivative
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
    } else {
        f = g > 0.0f ? g : g != g ? g : 0.0f;
        d = g > 0.0f ? 1.0f : 0.0f;
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
    // gated gradient
    const void *dh;
    int64_t ld_dh;
    void *p;                    // [m][dg du], each padded with zeros to pad_n, in parts
    int64_t ld_p, plane_p;
    int64_t pad_n;              // n_out padded to a multiple of 64
    unsigned *largest;          // gradient in half: see scale_of
    int again;
};
enum Kind { kGated, kGatedGrad, kPlain };

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
    if constexpr (std::is_same<T, f16>::value && KIND == kGatedGrad) return A.again && scale_of(A) == 1.0f;
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
    constexpr bool GATED = KIND != kPlain, ALONG_A = !GATED;
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
            const bool second = row % WA >= WA / 2;
            const int r = row / WA * (WA / 2) + row % (WA / 2);
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
    // lane l, register r of tile (i, j): row m = l % 16 of j; column 4 (l / 16) + r of i, or,
    // gated, 8 (l / 16) + 4 (i % 2) + r of the pair of tiles
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

// ---- few rows: the weights are read once, straight into registers, by workgroups of 16
// columns whose four waves share the sum; x comes from cache.  TB: rows in 16s.  Values are
// loaded as 16 bytes of a row at any address, so nothing is laid out first; a float is multiplied as it is
// (16 x 16 x 4: step r of the instruction takes value r of each lane's four).
template <class T, int TB> __global__ void __launch_bounds__(256) few(FfnArgs A) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int V = kVec<T>, K = 4 * V, U = TB > 2 ? 2 : 4;     // values of the sum a wave takes at a time; times in flight
    __shared__ f32x4 sums[4][2][TB][64];
    const int l = threadIdx.x % 64, wave = threadIdx.x / 64, lm = l % 16, lg = l / 16;
    const int64_t n0 = int64_t(blockIdx.x) * 16, n = min(n0 + lm, A.n_out - 1);
    const T *g = static_cast<const T *>(A.wg) + n * A.ld_wg, *u = static_cast<const T *>(A.wu) + n * A.ld_wu, *x[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) x[j] = static_cast<const T *>(A.x) + min(int64_t(j * 16 + lm), A.rows - 1) * A.ld_x;
    f32x4 acc[2][TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[0][j] = acc[1][j] = 0;
    const auto multiply = [](vec<T> a, vec<T> b, f32x4 c) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
            return c;
        } else {
            return mfma(__builtin_bit_cast(typename Oct<T>::type, a), __builtin_bit_cast(typename Oct<T>::type, b), c);
        }
    };
    for (int64_t k0 = wave * K; k0 < A.n_in; k0 += 4 * K * U) {
        vec<T> vg[U], vu[U], vx[U][TB];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t k = k0 + i * 4 * K + lg * V;
            vg[i] = vu[i] = T(0.0f);
#pragma unroll
            for (int j = 0; j < TB; ++j) vx[i][j] = T(0.0f);
            if (k < A.n_in) {
                vg[i] = load_vec(g + k, A.n_in - k);
                vu[i] = load_vec(u + k, A.n_in - k);
#pragma unroll
                for (int j = 0; j < TB; ++j) vx[i][j] = load_vec(x[j] + k, A.n_in - k);
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                acc[0][j] = multiply(vg[i], vx[i][j], acc[0][j]);
                acc[1][j] = multiply(vu[i], vx[i][j], acc[1][j]);
            }
    }
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        sums[wave][0][j][l] = acc[0][j];
        sums[wave][1][j][l] = acc[1][j];
    }
    __syncthreads();
    // wave j sums up rows 16 j on: lane l has row l % 16, columns 4 (l / 16) on
    if (wave >= TB) return;
    f32x4 sg = sums[0][0][wave][l], su = sums[0][1][wave][l];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        sg += sums[w][0][wave][l];
        su += sums[w][1][wave][l];
    }
    const int64_t m = wave * 16 + lm, c = n0 + lg * 4;
    if (m >= A.rows) return;
    T *row = static_cast<T *>(A.h) + m * A.ld_h;
    with_act(A.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float value, slope;
            act_both<decltype(act)::value>(sg[r], value, slope);
            if (c + r < A.n_out) row[c + r] = T(value * su[r]);
        }
    });
#endif
}

template <class T, int BA, int BB, int NA, int NB, Kind KIND> void launch_tiles(ProductArgs a, int64_t n, int64_t m, hipStream_t stream) {
    a.tiles_n = ceil_div(n, BA / 2);
    a.tiles_m = ceil_div(m, BB);
    const int64_t wgs = a.tiles_n * a.tiles_m * a.splits;
    if (wgs) product<T, BA, BB, NA, NB, KIND><<<dim3(uint32_t(wgs)), 64 * NA * NB, 0, stream>>>(a);
}

template <class T, Kind KIND> void launch_product(const Gated &c, ProductArgs a, int64_t n, int64_t m, hipStream_t stream) {
    constexpr bool RANGED = std::is_same<T, f16>::value && KIND == kGatedGrad;
    if (RANGED) clear_largest<<<1, 1, 0, stream>>>(a.largest);
    a.splits = int(c.splits);
    const auto sums = [&]() {
        if (c.bb == 256) launch_tiles<T, 256, 256, 2, 4, KIND>(a, n, m, stream);
        else if (c.ba == 256) launch_tiles<T, 256, 128, 4, 2, KIND>(a, n, m, stream);
        else launch_tiles<T, 128, 128, 2, 2, KIND>(a, n, m, stream);
    };
    const auto fold = [&]() { fold_gated<T, KIND><<<dim3(uint32_t(ceil_div(a.pad_n / 8 * a.m, 256))), 256, 0, stream>>>(a); };
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

constexpr int64_t kFewRows = 64;

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

}  // namespace

size_t ffn_bytes(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool grad) {
    if (!grad && rows <= kFewRows) return 0;
    // room for copies of x and both weights, whether or not the call's pointers and strides need them
    Space s(nullptr);
    s.take(dtype, rows, pad64(n_in));
    s.take(dtype, n_out, pad64(n_in));
    s.take(dtype, n_out, pad64(n_in));
    const Gated g = gated_cut(dtype, rows, n_in, n_out);
    if (g.splits > 1) s.take_floats(g.splits * rows * 2 * pad64(n_out));
    if (grad) {
        s.take(dtype, rows, 2 * pad64(n_out));
        if (dtype == NDVM_F16) s.take_floats(1);
        const Pieces c = pieces(dtype, rows, n_in, n_out);
        if (c.dx > 1) s.take_floats(c.dx * rows * n_in);
        if (c.dw > 1) s.take_floats(c.dw * 2 * pad64(n_out) * n_in);
    }
    return s.used + 256;
}

namespace {

struct Operands {
    Operand x, wg, wu;
    int64_t k;
};
// x and the weights as product() reads them: themselves, or padded copies.  (The weights one after the
// other along a sum have one row stride.)
template <class T> Operands operands(const FfnArgs &a, Space &s, hipStream_t stream) {
    Operands o;
    if (direct(a.dtype, a.x, a.ld_x, a.n_in) && direct(a.dtype, a.wg, a.ld_wg, a.n_in) && direct(a.dtype, a.wu, a.ld_wu, a.n_in) &&
        (!a.dx || a.ld_wg == a.ld_wu)) {
        o.x = Operand{a.x, a.rows, a.ld_x, 0};
        o.wg = Operand{a.wg, a.n_out, a.ld_wg, 0};
        o.wu = Operand{a.wu, a.n_out, a.ld_wu, 0};
        o.k = a.n_in;
        return o;
    }
    PackArgs p{};
    p.cols = a.n_in;
    p.pad = o.k = pad64(a.n_in);
    const auto copy = [&](int i, const void *from, int64_t rows, int64_t ld) {
        p.from[i] = from;
        p.to[i] = s.take(a.dtype, rows, p.pad);
        p.rows[i] = rows;
        p.ld[i] = ld;
        p.plane[i] = s.plane;
        return Operand{p.to[i], rows, p.pad, s.plane};
    };
    o.x = copy(0, a.x, a.rows, a.ld_x);
    o.wg = copy(1, a.wg, a.n_out, a.ld_wg);
    o.wu = copy(2, a.wu, a.n_out, a.ld_wu);
    const int64_t most = std::max(a.rows, a.n_out) * (p.pad / 8);
    pack<T><<<dim3(uint32_t(std::min(ceil_div(most, 256), kMostGroups)), 3), 256, 0, stream>>>(p);
    return o;
}

char *aligned(void *p) { return reinterpret_cast<char *>(round256(reinterpret_cast<size_t>(p))); }

// Also takes the room for the sums of a product that is split.
ProductArgs gated(const FfnArgs &a, const Operands &o, const Gated &c, Space &s) {
    ProductArgs p{};
    p.pad_n = pad64(a.n_out);
    if (c.splits > 1) p.part = s.take_floats(c.splits * a.rows * 2 * p.pad_n);
    p.a = o.wg;
    p.a2 = o.wu;
    p.b = o.x;
    p.k = o.k;
    p.act = a.act;
    p.n = a.n_out;
    p.m = a.rows;
    return p;
}

template <class T> void ffn(const FfnArgs &a, hipStream_t stream) {
    if (a.rows <= kFewRows) {
        const dim3 grid(uint32_t(ceil_div(a.n_out, 16)));
        if (a.rows <= 16) few<T, 1><<<grid, 256, 0, stream>>>(a);
        else if (a.rows <= 32) few<T, 2><<<grid, 256, 0, stream>>>(a);
        else few<T, 4><<<grid, 256, 0, stream>>>(a);
        return;
    }
    Space s(aligned(a.ws));
    const Gated g = gated_cut(a.dtype, a.rows, a.n_in, a.n_out);
    const Operands o = operands<T>(a, s, stream);
    ProductArgs p = gated(a, o, g, s);
    p.out = a.h;
    p.ld = a.ld_h;
    launch_product<T, kGated>(g, p, a.n_out, a.rows, stream);
}

template <class T> void ffn_grad(const FfnArgs &a, hipStream_t stream) {
    Space s(aligned(a.ws));
    const Operands o = operands<T>(a, s, stream);
    const int64_t pad_n = pad64(a.n_out);
    const Gated g = gated_cut(a.dtype, a.rows, a.n_in, a.n_out);
    ProductArgs p = gated(a, o, g, s);
    p.dh = a.dh;
    p.ld_dh = a.ld_dh;
    p.p = s.take(a.dtype, a.rows, 2 * pad_n);
    p.ld_p = 2 * pad_n;
    p.plane_p = s.plane;
    if (std::is_same<T, f16>::value) p.largest = reinterpret_cast<unsigned *>(s.take_floats(1));
    launch_product<T, kGatedGrad>(g, p, pad_n, a.rows, stream);
    const Operand both{p.p, a.rows, 2 * pad_n, p.plane_p};
    const Pieces c = pieces(a.dtype, a.rows, a.n_in, a.n_out);
    ProductArgs dx{}, dw{};
    dx.splits = dw.splits = 1;
    dx.largest = dw.largest = p.largest;
    if (a.dx) {     // n: x's columns; the sum: the rows of both weights
        dx.a = o.wg;
        dx.a2 = o.wu;
        dx.k2 = pad_n;
        dx.b = both;
        dx.k = 2 * pad_n;
        dx.out = a.dx;
        dx.ld = a.ld_dx;
        dx.n = a.n_in;
        dx.m = dx.split = dx.split2 = dx.m2 = a.rows;
        dx.splits = int(c.dx);
        if (c.dx > 1) dx.part = s.take_floats(c.dx * a.rows * a.n_in);
    }
    if (a.dwg) {    // m: the columns of [dg du]; the sum: rows
        dw.a = dw.a2 = o.x;
        dw.k = dw.k2 = pad64(a.rows);
        dw.b = both;
        dw.out = a.dwg;
        dw.ld = a.ld_dwg;
        dw.out2 = a.dwu;
        dw.ld2 = a.ld_dwu;
        dw.n = a.n_in;
        dw.m = 2 * pad_n;
        dw.split = a.n_out;
        dw.split2 = pad_n;
        dw.m2 = pad_n + a.n_out;
        dw.splits = int(c.dw);
        if (c.dw > 1) dw.part = s.take_floats(c.dw * dw.m * a.n_in);
    }
    if (c.tile == 256) launch_pair<T, 256, 2, 4>(dx, dw, stream);
    else launch_pair<T, 128, 2, 2>(dx, dw, stream);
}

}  // namespace

hipError_t launch_ffn(const FfnArgs &a, hipStream_t stream) {
    return with_type(a.dtype, [&](auto zero) {
        ffn<decltype(zero)>(a, stream);
        return hipGetLastError();
    });
}
hipError_t launch_ffn_grad(const FfnArgs &a, hipStream_t stream) {
    return with_type(a.dtype, [&](auto zero) {
        ffn_grad<decltype(zero)>(a, stream);
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
