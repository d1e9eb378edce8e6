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
#include "product.h"

namespace ndvm {
namespace ops {
namespace {

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

constexpr int64_t kFewRows = 64;

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
