// Gated feed-forward projections and their gradient.
//   g = x Wg^T,  u = x Wu^T,  h = act(g) u
//   dg = dh u act'(g),  du = dh act(g),  dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x
// Matrix products throughout: bound by the matrix instructions for many rows, by
// reading the weights for few.  One kernel, product(), computes all of them from
// operands whose rows run along the sum:  C[m][n] = sum_k A[n][k] B[m][k].
//  - forward: a tile holds the same columns of both weights, so act(g) u is formed in
//    the accumulators and g and u never reach memory;
//  - gradient: g and u are formed again the same way (reading them back would cost their
//    rounding; the two products are a third of the work), and dg, du leave the tile in
//    both orders, [rows][2 n_out] and transposed, as operands of
//    dx = [dg du] [Wg; Wu] and [dWg; dWu] = [dg du]^T x;
//  - x and the weights are transposed once for those two.
// 16-bit types are multiplied as they are.  A float is split exactly into three bf16
// (8 + 8 + 8 bits) and the six products down to 2^-16 of the largest are added up in
// float: what is left out is below 2^-23 of a term, and bf16 products are 16 times
// the rate of float ones.
#include <algorithm>

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

[[maybe_unused]] constexpr int kStep = 64;      // of the sum, per LDS tile

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
__device__ inline void act_both(int act, float g, float &f, float &d) {
    if (act == NDVM_ACT_SILU) {
        const float s = 1.0f / (1.0f + __expf(-g));
        f = g * s;
        d = s * (1.0f + g * (1.0f - s));
    } else if (act == NDVM_ACT_GELU) {
        const float p = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
        f = g * p;
        d = p + g * 0.39894228040143268f * __expf(-0.5f * g * g);
    } else if (act == NDVM_ACT_SIGMOID) {
        f = 1.0f / (1.0f + __expf(-g));
        d = f * (1.0f - f);
    } else {
        f = g > 0.0f ? g : g != g ? g : 0.0f;
        d = g > 0.0f ? 1.0f : 0.0f;
    }
}

// ---- operands laid out: a copy with rows padded to `ld_to` zeros, or the transpose
struct PackArgs {
    const void *from;
    void *to;
    int64_t rows, cols, ld;     // of `from`
    int64_t ld_to, pad;         // row length of `to`; columns written (the source's and zeros)
    int64_t plane;              // elements between a value's parts
};
template <class T, bool TRANSPOSE> __global__ void __launch_bounds__(256) pack(PackArgs a) {
    typedef typename Parts<T>::type P;
    constexpr int N = Parts<T>::count;
    __shared__ T tile[64][65];
    const int64_t r0 = int64_t(blockIdx.x) * 64, c0 = int64_t(blockIdx.y) * 64;
    const int x = threadIdx.x % 64;
    for (int y = threadIdx.x / 64; y < 64; y += 4) {
        const int64_t r = r0 + y, c = c0 + x;
        tile[y][x] = r < a.rows && c < a.cols ? static_cast<const T *>(a.from)[r * a.ld + c] : T(0.0f);
    }
    __syncthreads();
    const int64_t out_rows = TRANSPOSE ? a.cols : a.rows;
    for (int y = threadIdx.x / 64; y < 64; y += 4) {
        const int64_t r = (TRANSPOSE ? c0 : r0) + y, c = (TRANSPOSE ? r0 : c0) + x;
        if (r >= out_rows || c >= a.pad) continue;
        P part[N];
        const T v = TRANSPOSE ? tile[x][y] : tile[y][x];
        Parts<T>::split(float(v), part);
#pragma unroll
        for (int i = 0; i < N; ++i) static_cast<P *>(a.to)[i * a.plane + r * a.ld_to + c] = part[i];
    }
}
template <class T, bool TRANSPOSE> void launch_pack(const PackArgs &a, hipStream_t stream) {
    // the grid covers the padded columns too
    const int64_t rows = TRANSPOSE ? a.pad : a.rows, cols = TRANSPOSE ? a.cols : a.pad;
    if (rows && cols) pack<T, TRANSPOSE><<<dim3(uint32_t(ceil_div(rows, 64)), uint32_t(ceil_div(cols, 64))), 256, 0, stream>>>(a);
}

// ---- the product
struct Operand {
    const void *p;
    int64_t rows, ld, plane;
};
struct ProductArgs {
    Operand a, a2, b;           // a2: the second weight of a gated product
    int64_t k;                  // a multiple of 8
    int64_t tiles_n, tiles_m;
    int act;
    // plain: rows m < split go to out + m * ld, the others from split2 on to out2 + (m - split2) * ld2
    void *out, *out2;
    int64_t ld, ld2, n, m, split, split2, m2;
    // gated gradient
    const void *dh;
    int64_t ld_dh;
    void *p, *pt;               // [dg du] and its transpose, in parts
    int64_t pad_n, ld_p, plane_p, pad_m, ld_pt, plane_pt;
};
enum Kind { kGated, kGatedGrad, kPlain };

// BA rows of A by BB rows of B a workgroup; NA x NB waves.
// LDS rows are 64 values (128 bytes, 8 granules of 16); granule i of row r lies at place
// i ^ (r % 8), so a wave's reads of 16 rows touch all banks evenly.  The loads go to LDS
// directly and choose their source accordingly; values out of range read as 0.
template <class T, int BA, int BB, int NA, int NB, Kind KIND>
__global__ void __launch_bounds__(64 * NA * NB) product(ProductArgs A) {
#ifdef __HIP_DEVICE_COMPILE__       // the host's pass does not know the types of the loads to LDS
    typedef typename Parts<T>::type P;
    typedef typename Oct<P>::type oct;
    constexpr int PARTS = Parts<T>::count, PAIRS = PARTS == 1 ? 1 : 6, W = NA * NB;
    constexpr int WA = BA / NA, WB = BB / NB, TA = WA / 16, TB = WB / 16;
    constexpr bool GATED = KIND != kPlain;
    constexpr int COLS = GATED ? BA / 2 : BA;       // columns of C a tile has
    // two arrays, so that the compiler sees that loads into one leave reads of the other alone
    __shared__ __align__(1024) char buffer0[(BA + BB) * kStep * 2], buffer1[(BA + BB) * kStep * 2];

    // Tiles in an order that keeps an XCD (workgroup % 8) on neighbouring ones: its share
    // of the tiles, in bands of 8 tile rows.
    int64_t id = blockIdx.x;
    {
        const int64_t total = A.tiles_n * A.tiles_m, x = id % 8, per = total / 8, more = total % 8;
        id = x * per + min(x, more) + id / 8;
    }
    const int64_t band = id / (8 * A.tiles_n), in = id % (8 * A.tiles_n);
    const int64_t tall = min(int64_t(8), A.tiles_m - band * 8);
    const int64_t m0 = (band * 8 + in % tall) * BB, n0 = in / tall * COLS;

    const int l = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lm = l % 16, lg = l / 16, wa = wave / NB, wb = wave % NB;
    constexpr unsigned kNowhere = 0x80000000u;
    const auto rsrc = [](const void *p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, 0x7fffffff, 0x00020000); };

    // Wave-wide loads of 8 rows: which rows, and where a lane's granule of them is.
    constexpr int LA = BA / 8 / W, LB = BB / 8 / W;
    const int sub = l / 8, granule = (l % 8) ^ sub;
    unsigned at_a[LA], at_b[LB];
    const P *base_a = static_cast<const P *>(A.a.p) + n0 * A.a.ld, *base_b = static_cast<const P *>(A.b.p) + m0 * A.b.ld;
    const P *base_a2 = GATED ? static_cast<const P *>(A.a2.p) + n0 * A.a2.ld : nullptr;
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int row = (wave + W * i) * 8 + sub;
        const bool second = GATED && row % WA >= WA / 2;
        const int r = GATED ? row / WA * (WA / 2) + row % (WA / 2) : row;
        at_a[i] = n0 + r < A.a.rows ? unsigned(r * (second ? A.a2.ld : A.a.ld) + granule * 8) * 2 : kNowhere;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int row = (wave + W * i) * 8 + sub;
        at_b[i] = m0 + row < A.b.rows ? unsigned(row * A.b.ld + granule * 8) * 2 : kNowhere;
    }
    const int64_t steps = ceil_div(A.k, kStep);
    // pairs of parts, largest products first
    constexpr int pair_a[6] = {0, 0, 1, 1, 0, 2}, pair_b[6] = {0, 1, 0, 1, 2, 0};
    const auto load = [&](int64_t s, char *to) __attribute__((always_inline)) {
        int64_t k0 = s * kStep;
        int pa = 0, pb = 0;
        if (PAIRS > 1) {
            const int pair = int(s / steps);
            k0 = s % steps * kStep;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i)
                if (i == pair) pa = pair_a[i], pb = pair_b[i];
        }
        const bool some = k0 + granule * 8 < A.k;
        const auto ra = rsrc(base_a + pa * A.a.plane + k0), rb = rsrc(base_b + pb * A.b.plane + k0);
        const auto ra2 = GATED ? rsrc(base_a2 + pa * A.a2.plane + k0) : ra;
#pragma unroll
        for (int i = 0; i < LA; ++i) {
            const int first = (wave + W * i) * 8;
            const bool second = GATED && first % WA >= WA / 2;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(second ? ra2 : ra, (__attribute__((address_space(3))) void *)(to + first * 128), 16,
                                                     some ? at_a[i] : kNowhere, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < LB; ++i) {
            const int first = (wave + W * i) * 8;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (__attribute__((address_space(3))) void *)(to + (BA + first) * 128), 16,
                                                     some ? at_b[i] : kNowhere, 0, 0, 0);
        }
    };

    f32x4 acc[TA][TB];
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = 0;
    const int64_t total = steps * PAIRS;
    const auto step = [&](int64_t s, const char *from, char *next) __attribute__((always_inline)) {
        // every wave's loads of this buffer have landed, and none reads the other one
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (s + 1 < total) load(s + 1, next);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            oct fa[TA], fb[TB];
            const int place = ((kk * 4 + lg) ^ (lm % 8)) * 16;
#pragma unroll
            for (int i = 0; i < TA; ++i) fa[i] = *reinterpret_cast<const oct *>(from + (wa * WA + i * 16 + lm) * 128 + place);
#pragma unroll
            for (int j = 0; j < TB; ++j) fb[j] = *reinterpret_cast<const oct *>(from + (BA + wb * WB + j * 16 + lm) * 128 + place);
#pragma unroll
            for (int i = 0; i < TA; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = mfma(fa[i], fb[j], acc[i][j]);
        }
    };
    if (total > 0) load(0, buffer0);
    for (int64_t s = 0; s < total; s += 2) {
        step(s, buffer0, buffer1);
        if (s + 1 < total) step(s + 1, buffer1, buffer0);
    }

    // lane l, register r of tile (i, j): column n = 4 (l / 16) + r, row m = l % 16
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef P four_p __attribute__((ext_vector_type(4), aligned(8)));
#pragma unroll
    for (int j = 0; j < TB; ++j) {
        const int64_t m = m0 + wb * WB + j * 16 + lm;
        if constexpr (KIND == kPlain) {
            T *row = nullptr;
            if (m < A.split) row = static_cast<T *>(A.out) + m * A.ld;
            else if (m >= A.split2 && m < A.m2) row = static_cast<T *>(A.out2) + (m - A.split2) * A.ld2;
            if (!row) continue;
#pragma unroll
            for (int i = 0; i < TA; ++i) {
                const int64_t n = n0 + wa * WA + i * 16 + lg * 4;
                four v;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = T(acc[i][j][r]);
                if (n + 4 <= A.n) *reinterpret_cast<four *>(row + n) = v;
                else
                    for (int r = 0; r < 4; ++r)
                        if (n + r < A.n) row[n + r] = v[r];
            }
        } else {
#pragma unroll
            for (int i = 0; i < TA / 2; ++i) {
                const int64_t n = n0 + wa * (WA / 2) + i * 16 + lg * 4;
                if constexpr (KIND == kGated) {
                    if (m >= A.m) continue;
                    T *row = static_cast<T *>(A.out) + m * A.ld;
                    four v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float f, d;
                        act_both(A.act, acc[i][j][r], f, d);
                        v[r] = T(f * acc[i + TA / 2][j][r]);
                    }
                    if (n + 4 <= A.n) *reinterpret_cast<four *>(row + n) = v;
                    else
                        for (int r = 0; r < 4; ++r)
                            if (n + r < A.n) row[n + r] = v[r];
                } else {
                    if (n >= A.pad_n || m >= A.pad_m) continue;
                    const T *row = static_cast<const T *>(A.dh) + m * A.ld_dh;
                    four_p vg[PARTS], vu[PARTS];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float dh = m < A.m && n + r < A.n ? float(row[n + r]) : 0.0f;
                        float f, d;
                        act_both(A.act, acc[i][j][r], f, d);
                        P pg[PARTS], pu[PARTS];
                        // what lies beyond the operands is 0, whatever act does there
                        const bool there = m < A.m && n + r < A.n;
                        Parts<T>::split(there ? dh * acc[i + TA / 2][j][r] * d : 0.0f, pg);
                        Parts<T>::split(there ? dh * f : 0.0f, pu);
#pragma unroll
                        for (int q = 0; q < PARTS; ++q) {
                            vg[q][r] = pg[q];
                            vu[q][r] = pu[q];
                            P *pt = static_cast<P *>(A.pt) + q * A.plane_pt + m;
                            pt[(n + r) * A.ld_pt] = pg[q];
                            pt[(A.pad_n + n + r) * A.ld_pt] = pu[q];
                        }
                    }
                    if (m >= A.m) continue;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        P *p = static_cast<P *>(A.p) + q * A.plane_p + m * A.ld_p + n;
                        *reinterpret_cast<four_p *>(p) = vg[q];
                        *reinterpret_cast<four_p *>(p + A.pad_n) = vu[q];
                    }
                }
            }
        }
    }
#endif
}

template <class T, int BA, int BB, int NA, int NB, Kind KIND> void launch_tiles(ProductArgs a, int64_t n, int64_t m, hipStream_t stream) {
    a.tiles_n = ceil_div(n, KIND == kPlain ? BA : BA / 2);
    a.tiles_m = ceil_div(m, BB);
    if (a.tiles_n * a.tiles_m == 0) return;
    product<T, BA, BB, NA, NB, KIND><<<dim3(uint32_t(a.tiles_n * a.tiles_m)), 64 * NA * NB, 0, stream>>>(a);
}
template <class T, Kind KIND> void launch_product(const ProductArgs &a, int64_t n, int64_t m, hipStream_t stream) {
    if (ceil_div(n, KIND == kPlain ? 256 : 128) * ceil_div(m, 256) >= 2 * kCus) launch_tiles<T, 256, 256, 2, 4, KIND>(a, n, m, stream);
    else launch_tiles<T, 128, 128, 2, 2, KIND>(a, n, m, stream);
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
};

}  // namespace

size_t ffn_bytes(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool grad) {
    // room for copies of x and both weights, whether or not the call's pointers and strides need them
    Space s(nullptr);
    s.take(dtype, rows, pad64(n_in));
    s.take(dtype, 2 * n_out, pad64(n_in));
    if (grad) {
        s.take(dtype, n_in, pad64(rows));
        s.take(dtype, n_in, 2 * pad64(n_out));
        s.take(dtype, rows, 2 * pad64(n_out));
        s.take(dtype, 2 * pad64(n_out), pad64(rows));
    }
    return s.used + 256;
}

namespace {

template <class T> struct Operands {
    Operand x, wg, wu;
    int64_t k;
};
// x and the weights as product() reads them: themselves, or padded copies.
template <class T> Operands<T> operands(const FfnArgs &a, Space &s, hipStream_t stream) {
    const int64_t pad = pad64(a.n_in);
    Operands<T> o;
    const bool as_is = direct(a.dtype, a.x, a.ld_x, a.n_in) && direct(a.dtype, a.wg, a.ld_wg, a.n_in) && direct(a.dtype, a.wu, a.ld_wu, a.n_in);
    if (as_is) {
        o.x = Operand{a.x, a.rows, a.ld_x, 0};
        o.wg = Operand{a.wg, a.n_out, a.ld_wg, 0};
        o.wu = Operand{a.wu, a.n_out, a.ld_wu, 0};
        o.k = a.n_in;
        return o;
    }
    const auto copy = [&](const void *from, int64_t rows, int64_t ld) {
        void *to = s.take(a.dtype, rows, pad);
        launch_pack<T, false>(PackArgs{from, to, rows, a.n_in, ld, pad, pad, s.plane}, stream);
        return Operand{to, rows, pad, s.plane};
    };
    o.x = copy(a.x, a.rows, a.ld_x);
    o.wg = copy(a.wg, a.n_out, a.ld_wg);
    o.wu = copy(a.wu, a.n_out, a.ld_wu);
    o.k = pad;
    return o;
}

char *aligned(void *p) { return reinterpret_cast<char *>(round256(reinterpret_cast<size_t>(p))); }

template <class T> void ffn(const FfnArgs &a, hipStream_t stream) {
    Space s(aligned(a.ws));
    const Operands<T> o = operands<T>(a, s, stream);
    ProductArgs p{};
    p.a = o.wg;
    p.a2 = o.wu;
    p.b = o.x;
    p.k = o.k;
    p.act = a.act;
    p.out = a.h;
    p.ld = a.ld_h;
    p.n = a.n_out;
    p.m = a.rows;
    launch_product<T, kGated>(p, a.n_out, a.rows, stream);
}

template <class T> void ffn_grad(const FfnArgs &a, hipStream_t stream) {
    typedef typename Parts<T>::type P;
    Space s(aligned(a.ws));
    const Operands<T> o = operands<T>(a, s, stream);
    const int64_t pad_n = pad64(a.n_out), pad_m = pad64(a.rows);
    ProductArgs p{};
    p.a = o.wg;
    p.a2 = o.wu;
    p.b = o.x;
    p.k = o.k;
    p.act = a.act;
    p.n = a.n_out;
    p.m = a.rows;
    p.dh = a.dh;
    p.ld_dh = a.ld_dh;
    p.pad_n = pad_n;
    p.pad_m = pad_m;
    p.p = s.take(a.dtype, a.rows, 2 * pad_n);
    p.ld_p = 2 * pad_n;
    p.plane_p = s.plane;
    p.pt = s.take(a.dtype, 2 * pad_n, pad_m);
    p.ld_pt = pad_m;
    p.plane_pt = s.plane;
    launch_product<T, kGatedGrad>(p, pad_n, pad_m, stream);
    if (a.dx) {
        P *wt = static_cast<P *>(s.take(a.dtype, a.n_in, 2 * pad_n));
        const int64_t plane = s.plane;
        launch_pack<T, true>(PackArgs{a.wg, wt, a.n_out, a.n_in, a.ld_wg, 2 * pad_n, pad_n, plane}, stream);
        launch_pack<T, true>(PackArgs{a.wu, wt + pad_n, a.n_out, a.n_in, a.ld_wu, 2 * pad_n, pad_n, plane}, stream);
        ProductArgs q{};
        q.a = Operand{wt, a.n_in, 2 * pad_n, plane};
        q.b = Operand{p.p, a.rows, 2 * pad_n, p.plane_p};
        q.k = 2 * pad_n;
        q.out = a.dx;
        q.ld = a.ld_dx;
        q.n = a.n_in;
        q.split = a.rows;
        q.split2 = q.m2 = a.rows;
        launch_product<T, kPlain>(q, a.n_in, a.rows, stream);
    }
    if (a.dwg) {
        void *xt = s.take(a.dtype, a.n_in, pad_m);
        const int64_t plane = s.plane;
        launch_pack<T, true>(PackArgs{a.x, xt, a.rows, a.n_in, a.ld_x, pad_m, pad_m, plane}, stream);
        ProductArgs q{};
        q.a = Operand{xt, a.n_in, pad_m, plane};
        q.b = Operand{p.pt, 2 * pad_n, pad_m, p.plane_pt};
        q.k = pad_m;
        q.out = a.dwg;
        q.ld = a.ld_dwg;
        q.out2 = a.dwu;
        q.ld2 = a.ld_dwu;
        q.n = a.n_in;
        q.split = a.n_out;
        q.split2 = pad_n;
        q.m2 = pad_n + a.n_out;
        launch_product<T, kPlain>(q, a.n_in, 2 * pad_n, stream);
    }
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
