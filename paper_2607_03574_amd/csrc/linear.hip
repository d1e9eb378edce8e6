// Projections with bias, activation and residual, and their gradient.
//   z = x W^T + b,  y = act(z) + r
//   dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum_rows dz,  dr = dy
// Matrix products (product.h): bound by the matrix instructions for many rows, by reading the
// weights for few.  Bias, activation and residual are applied to a tile's accumulators, so z never
// reaches memory; the gradient forms it again the same way where there is an activation, and writes dz
// once, as the operand of both of its other products.  Few rows have a kernel of their own.
// Rows in 8 bits (e4m3, a scale a row of x and of W) are multiplied as they are, on the matrix
// instructions of twice the 16-bit rate; z = (x8 W8^T) scale_x scale_W is formed in the accumulators too.
// These instructions line up eight products at a time at the largest of them and cut what lies below 2^-13 of
// its power of two, before they are added in float (measured): an error of some 10^-5 in norm, 7 2^-13 of the
// magnitudes' sum at most.  That is little beside a 16-bit result's own rounding (2^-9 or 2^-11 in bf16 and half)
// but not beside a float's, which this form therefore does not give; few rows are multiplied as bf16, exactly.
#include "product.h"

namespace ndvm {
namespace ops {
namespace {

typedef uint8_t byte;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

#ifdef __HIP_DEVICE_COMPILE__
__device__ inline bf16x8 wide(uint32_t a, uint32_t b) {
    typedef bf16 two __attribute__((ext_vector_type(2)));
    const auto pair = [](uint32_t v, auto high) { return __builtin_bit_cast(two, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.0f, decltype(high)::value)); };
    const std::false_type low;
    const std::true_type high;
    const two p = pair(a, low), q = pair(a, high), r = pair(b, low), s = pair(b, high);
    return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
#endif

// ---- few rows: the weights are read once, straight into registers, by workgroups of 16
// columns whose NW waves share the sum; x comes from cache.  TB: rows in 16s.  Values are
// loaded as 16 bytes of a row at any address, so nothing is laid out first; a float is multiplied as it is
// (16 x 16 x 4: step r of the instruction takes value r of each lane's four).  E: an operand's element.
template <class E, class T, int TB, int NW> __global__ void __launch_bounds__(64 * NW) few(LinearArgs A) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int V = kVec<E>, K = 4 * V, U = TB > 2 ? 2 : 4;     // values of the sum a wave takes at a time; times in flight
    __shared__ f32x4 sums[NW][TB][64];
    const int l = threadIdx.x % 64, wave = threadIdx.x / 64, lm = l % 16, lg = l / 16;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const E *w = static_cast<const E *>(A.w) + min(n0 + lm, A.n_out - 1) * A.ld_w, *x[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) x[j] = static_cast<const E *>(A.x) + min(int64_t(j * 16 + lm), A.rows - 1) * A.ld_x;
    f32x4 acc[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[j] = 0;
    const auto multiply = [](vec<E> a, vec<E> b, f32x4 c) {
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int r = 0; r < 4; ++r) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[r], b[r], c, 0, 0, 0);
            return c;
        } else if constexpr (sizeof(E) == 1) {
            // as bf16, which holds every e4m3 value
            const u32x4 p = __builtin_bit_cast(u32x4, a), q = __builtin_bit_cast(u32x4, b);
#pragma unroll
            for (int i = 0; i < 2; ++i) c = mfma(wide(p[2 * i], p[2 * i + 1]), wide(q[2 * i], q[2 * i + 1]), c);
            return c;
        } else {
            return mfma(__builtin_bit_cast(typename Oct<E>::type, a), __builtin_bit_cast(typename Oct<E>::type, b), c);
        }
    };
    for (int64_t k0 = wave * K; k0 < A.n_in; k0 += NW * K * U) {
        vec<E> vw[U], vx[U][TB];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t k = k0 + i * NW * K + lg * V;
            vw[i] = E(0);
#pragma unroll
            for (int j = 0; j < TB; ++j) vx[i][j] = E(0);
            if (k < A.n_in) {
                vw[i] = load_vec(w + k, A.n_in - k);
#pragma unroll
                for (int j = 0; j < TB; ++j) vx[i][j] = load_vec(x[j] + k, A.n_in - k);
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[j] = multiply(vw[i], vx[i][j], acc[j]);
    }
#pragma unroll
    for (int j = 0; j < TB; ++j) sums[wave][j][l] = acc[j];
    __syncthreads();
    // wave j sums up rows 16 j on: lane l has row l % 16, columns 4 (l / 16) on
    if (wave >= TB) return;
    f32x4 z = sums[0][wave][l];
#pragma unroll
    for (int i = 1; i < NW; ++i) z += sums[i][wave][l];
    const int64_t m = wave * 16 + lm, c = n0 + lg * 4;
    if (m >= A.rows) return;
    T *row = static_cast<T *>(A.y) + m * A.ld_y;
    const T *bias = static_cast<const T *>(A.bias), *more = A.residual ? static_cast<const T *>(A.residual) + m * A.ld_r : nullptr;
    const float x_scale = sizeof(E) == 1 ? A.x_scale[m] : 1.0f;
    with_act_or_none(A.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (c + r >= A.n_out) continue;
            float value, slope, sum = z[r];
            if (sizeof(E) == 1) sum = sum * x_scale * A.w_scale[c + r];
            if (bias) sum += float(bias[c + r]);
            act_of<T, decltype(act)::value>(sum, value, slope);
            if (more) value += float(more[c + r]);
            row[c + r] = T(value);
        }
    });
#endif
}

template <class E, class T> void launch_few(const LinearArgs &a, hipStream_t stream) {
    const dim3 grid(uint32_t(ceil_div(a.n_out, 16)));
    if (a.rows <= 16) few<E, T, 1, 16><<<grid, 1024, 0, stream>>>(a);
    else if (a.rows <= 32) few<E, T, 2, 16><<<grid, 1024, 0, stream>>>(a);
    else few<E, T, 4, 8><<<grid, 512, 0, stream>>>(a);
}

// ---- 8 bits: the product of product.h for rows of bytes along the sum, on the 32 x 32 x 64 instruction.
// An LDS tile is 64 bytes long along the sum, in granules of 16; lane l of an operand has granules 2 (l / 32) and
// the next of row l % 32.  Granule i of a row of x lies at place i ^ (row / 2 % 4); rows of W are read in the
// order that leaves a lane with 16 columns side by side, and lie at i ^ (row / 2 % 2 + row / 16 % 2 * 2): eight lanes
// read all banks in both.
struct Product8Args {
    ProductArgs out;            // tiles, splits, n, m, epilogue
    const byte *x, *w;          // rows of 16-byte granules
    int64_t ld_x, ld_w, k;      // k: a multiple of 16
};
#ifdef __HIP_DEVICE_COMPILE__
__device__ inline f32x16 mfma8(i32x8 a, i32x8 b, f32x16 c) { return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0); }
#endif

template <class T, int BA, int BB, int NA, int NB> __global__ void __launch_bounds__(64 * NA * NB) product8(Product8Args A) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int kStep8 = 64;      // bytes of the sum, per LDS tile
    constexpr int W = NA * NB, WA = BA / NA, WB = BB / NB, TA = WA / 32, TB = WB / 32;
    constexpr int SIZE = (BA + BB) * kStep8;
    __shared__ __align__(1024) char buffer0[SIZE], buffer1[SIZE], buffer2[SIZE], buffer3[SIZE];
    const ProductArgs &O = A.out;
    // tiles as in product(): an XCD (workgroup % 8) on neighbouring ones, in bands of 8 tile rows
    const int64_t tiles = O.tiles_n * O.tiles_m;
    int64_t id = blockIdx.x;
    {
        const int64_t total = tiles * O.splits, x = id % 8, per = total / 8, more = total % 8;
        id = x * per + min(x, more) + id / 8;
    }
    const int part = int(id / tiles);
    id %= tiles;
    const int64_t band = id / (8 * O.tiles_n), in = id % (8 * O.tiles_n);
    const int64_t tall = min(int64_t(8), O.tiles_m - band * 8);
    const int64_t m0 = (band * 8 + in % tall) * BB, n0 = in / tall * BA;

    const int l = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lr = l % 32, lh = l / 32, wa = wave / NB, wb = wave % NB;
    constexpr unsigned kNowhere = 0x80000000u;
    const auto rsrc = [](const void *p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, 0x7fffffff, 0x00020000); };
    // Wave-wide loads of 1 KB: 16 rows of 4 granules.
    constexpr int LA = BA / 16 / W, LB = BB / 16 / W, LOADS = LA + LB;
    static_assert(W % 2 == 0, "rows of a load and of the next have the same places");
    const int sub = l / 4, granule_a = (l % 4) ^ (sub / 2 % 2 + wave % 2 * 2), granule_b = (l % 4) ^ (sub / 2 % 4);
    unsigned at_a[LA], at_b[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int row = (wave + W * i) * 16 + sub;
        at_a[i] = n0 + row < O.n ? unsigned(row * A.ld_w + granule_a * 16) : kNowhere;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int row = (wave + W * i) * 16 + sub;
        at_b[i] = m0 + row < O.m ? unsigned(row * A.ld_x + granule_b * 16) : kNowhere;
    }
    const int steps = int((A.k + kStep8 - 1) / kStep8);
    const int first = int(int64_t(steps) * part / O.splits), total = int(int64_t(steps) * (part + 1) / O.splits);
    const byte *next_a = A.w + n0 * A.ld_w + int64_t(first) * kStep8, *next_b = A.x + m0 * A.ld_x + int64_t(first) * kStep8;
    int64_t left = A.k - int64_t(first) * kStep8;
    int at = first;
    // The next tile into `to`: always LA + LB loads a wave (past the end they fetch nothing).
    const auto load = [&](char *to) __attribute__((always_inline)) {
        const bool some_a = at < total && granule_a * 16 < left, some_b = at < total && granule_b * 16 < left;
        const auto ra = rsrc(next_a), rb = rsrc(next_b);
#pragma unroll
        for (int i = 0; i < LA; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (__attribute__((address_space(3))) void *)(to + (wave + W * i) * 1024), 16,
                                                     some_a ? at_a[i] : kNowhere, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < LB; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (__attribute__((address_space(3))) void *)(to + BA * 64 + (wave + W * i) * 1024), 16,
                                                     some_b ? at_b[i] : kNowhere, 0, 0, 0);
        ++at;
        left -= kStep8;
        next_a += kStep8;
        next_b += kStep8;
    };
    f32x16 acc[TA][TB];
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = 0;
    // One set of A's registers, two of B's, as in product().
    i32x8 fa[TA], fb[2][TB];
    const auto both = [](const char *p, const char *q) __attribute__((always_inline)) {
        const u32x4 u = *reinterpret_cast<const u32x4 *>(p), v = *reinterpret_cast<const u32x4 *>(q);
        return __builtin_bit_cast(i32x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    struct Places {
        int a, b;
    };
    // kept from the compiler's sight, as in product()
    const auto places = [&]() __attribute__((always_inline)) {
        const int row_a = lr / 4 % 2 * 16 + lr / 8 * 4 + lr % 4;
        Places p{(wa * WA + row_a) * 64 + (2 * lh ^ (row_a / 2 % 2 + row_a / 16 % 2 * 2)) * 16, (wb * WB + lr) * 64 + (2 * lh ^ (lr / 2 % 4)) * 16};
        asm volatile("" : "+v"(p.a), "+v"(p.b));
        return p;
    };
    // granules 2 h and 2 h + 1 are neighbours, or one before the other: their places differ in the lowest bit
    const auto read_a = [&](const char *from, int i, const Places &p) __attribute__((always_inline)) {
        fa[i] = both(from + p.a + i * 2048, from + (p.a ^ 16) + i * 2048);
    };
    const auto read_b = [&](const char *from, i32x8 &to, int j, const Places &p) __attribute__((always_inline)) {
        to = both(from + BA * 64 + p.b + j * 2048, from + BA * 64 + (p.b ^ 16) + j * 2048);
    };
    static_assert(3 * LOADS < 16, "");
    const auto wait = [&](auto loads) __attribute__((always_inline)) {
        // this wave's older loads have landed and its reads are done; after the barrier everybody's
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | decltype(loads)::value);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    };
    using std::integral_constant;
    const auto step = [&](const char *next, char *to, auto now) __attribute__((always_inline)) {
        constexpr int n = decltype(now)::value;
        wait(integral_constant<int, 2 * LOADS>());
        load(to);
        const Places place = places();
        static_assert(TB <= TA, "");
#pragma unroll
        for (int i = 0; i < TA; ++i) {
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = mfma8(fa[i], fb[n][j], acc[i][j]);
            if (i < TB) read_b(next, fb[1 - n][i], i, place);
            read_a(next, i, place);
        }
        // loads and reads among the multiplications, none of which waits for them
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, TB, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, (LOADS + TB - 1) / TB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        }
#pragma unroll
        for (int i = TB; i < TA; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, TB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    };
    if (first < total) {
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
        // the loads past the end write zeros to LDS, which has to be this workgroup's still
        __builtin_amdgcn_s_waitcnt(0x0f70);
    }
    // lane l, register r of tile (i, j): row m = l % 32 of j, column 16 (l / 32) + r of i; two tiles side by side at a time
    static_assert(32 * 68 * 4 * W / 4 <= SIZE && TA % 2 == 0, "");
    float *stage = reinterpret_cast<float *>(wave % 4 == 0 ? buffer0 : wave % 4 == 1 ? buffer1 : wave % 4 == 2 ? buffer2 : buffer3) + wave / 4 * (32 * 68);
    meet();     // the buffers are everybody's until here
    float top = 0;
    Leaving<T, kLinear, 32, 64> leaving(O, part, stage);
#pragma unroll 1
    for (int t = 0; t < TA / 2 * TB; ++t) {
#pragma unroll
        for (int c = 0; c < TA / 2 * TB; ++c)
            if (c == t)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16 &v = acc[c / TB * 2 + i][c % TB];
                        *reinterpret_cast<f32x4 *>(stage + lr * 68 + i * 32 + lh * 16 + q * 4) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                    }
        leaving.rows(m0 + wb * WB + t % TB * 32, n0 + wa * WA + t / TB * 64, top);
    }
#endif
}

// Rows of bytes laid out: whole granules, zeros beyond a row's end.  blockIdx.y: which of the two operands.
struct Pack8Args {
    const byte *from[2];
    byte *to[2];
    int64_t rows[2], ld[2];
    int64_t cols, pad;
};
__global__ void __launch_bounds__(256) pack8(Pack8Args a) {
    const int w = blockIdx.y;
    const int64_t per = a.pad / 16;
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < a.rows[w] * per; at += int64_t(gridDim.x) * 256) {
        const int64_t r = at / per, c = at % per * 16;
        vec<byte> v = byte(0);
        if (c < a.cols) v = load_vec(a.from[w] + r * a.ld[w] + c, a.cols - c);
        *reinterpret_cast<vec<byte> *>(a.to[w] + r * a.pad + c) = v;
    }
}

// ---- db: sums of dz over the rows, in float before dz is rounded for the products.  With an activation the product that forms
// dz leaves the sums of every 64 rows (4096 x 1024 x 4096 bf16, silu: db is 1.66e-3 off in norm, its own rounding; as a sum of dz
// as it is rounded 2.32e-3); without one dz is dy as it came, whose sums are taken in parts of `groups` workgroups, a
// thread eight columns of every eighth row of its workgroup's.  A launch adds the parts up in order.
struct ColumnArgs {
    const void *dy;             // [rows][ld]
    int64_t rows, n, ld;
    float *part;                // [groups][pad]
    int64_t pad;
    void *to;
};
constexpr int64_t kColumnGroups = 64;
template <class T> __global__ void __launch_bounds__(256) column_sums(ColumnArgs a) {
    typedef T eight __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    __shared__ float lds[8][256];
    const int x = threadIdx.x % 32, s = threadIdx.x / 32;
    const int64_t c = int64_t(blockIdx.x) * 256 + x * 8;
    const int have = int(min(max(a.n - c, int64_t(0)), int64_t(8)));
    float sum[8] = {};
    for (int64_t row = int64_t(blockIdx.y) * 8 + s; row < a.rows; row += int64_t(gridDim.y) * 8) {
        const T *p = static_cast<const T *>(a.dy) + row * a.ld + c;
        eight v = T(0.0f);
        if (have == 8) v = *reinterpret_cast<const eight *>(p);
        else
            for (int r = 0; r < 8; ++r)
                if (r < have) v[r] = p[r];
#pragma unroll
        for (int r = 0; r < 8; ++r) sum[r] += float(v[r]);
    }
#pragma unroll
    for (int r = 0; r < 8; ++r) lds[s][x * 8 + r] = sum[r];
    __syncthreads();
    const int64_t col = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (col >= a.n) return;
    float v = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += lds[i][threadIdx.x];
    a.part[int64_t(blockIdx.y) * a.pad + col] = v;
}
template <class T> __global__ void __launch_bounds__(256) column_fold(ColumnArgs a, int groups) {
    __shared__ float lds[8][32];
    const int64_t c = int64_t(blockIdx.x) * 32 + threadIdx.x % 32;
    const int s = threadIdx.x / 32;
    float v = 0;
    if (c < a.n)
#pragma unroll 8
        for (int g = s; g < groups; g += 8) v += a.part[int64_t(g) * a.pad + c];
    lds[s][threadIdx.x % 32] = v;
    __syncthreads();
    if (s || c >= a.n) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) v += lds[i][threadIdx.x];
    static_cast<T *>(a.to)[c] = T(v);
}
// what db takes of the workspace: sums of every 64 rows, or of as many groups as there are
int64_t column_floats(int64_t rows, int64_t n_out) { return std::max(kColumnGroups, ceil_div(rows, 64)) * pad64(n_out); }

constexpr int64_t kFewRows = 64;

}  // namespace

size_t linear_bytes(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, bool grad) {
    if (!grad && rows <= kFewRows) return 0;
    // room for copies of the operands, whether or not the call's pointers and strides need them
    Space s(nullptr);
    const bool formed = !grad || act != NDVM_ACT_NONE;      // whether z is
    s.take(dtype, rows, pad64(n_in));
    s.take(dtype, n_out, pad64(n_in));
    const Gated g = linear_cut(dtype, rows, n_in, n_out);
    if (formed && g.splits > 1) s.take_floats(g.splits * rows * pad64(n_out));
    if (grad) {
        s.take(dtype, rows, pad64(n_out));
        s.take_floats(1);
        const Pieces c = linear_pieces(dtype, rows, n_in, n_out);
        if (c.dx > 1) s.take_floats(c.dx * rows * n_in);
        if (c.dw > 1) s.take_floats(c.dw * pad64(n_out) * n_in);
        s.take_floats(column_floats(rows, n_out));
    }
    return s.used + 256;
}

size_t linear_8bit_bytes(int64_t rows, int64_t n_in, int64_t n_out) {
    if (rows <= kFewRows) return 0;
    const Gated g = linear_cut(NDVM_BF16, rows, ceil_div(n_in, 2), n_out);
    return size_t(rows + n_out) * size_t(pad64(n_in)) + (g.splits > 1 ? size_t(g.splits * rows) * size_t(pad64(n_out)) * 4 : 0) + 1024;
}

namespace {

// x and W as product() reads them: themselves, or padded copies.
struct Operands {
    Operand x, w;
    int64_t k;
};
template <class T> Operands operands(const LinearArgs &a, Space &s, hipStream_t stream) {
    Operands o;
    if (direct(a.dtype, a.x, a.ld_x, a.n_in) && direct(a.dtype, a.w, a.ld_w, a.n_in)) {
        o.x = Operand{a.x, a.rows, a.ld_x, 0};
        o.w = Operand{a.w, a.n_out, a.ld_w, 0};
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
    o.w = copy(1, a.w, a.n_out, a.ld_w);
    pack<T><<<dim3(uint32_t(std::min(ceil_div(std::max(a.rows, a.n_out) * (p.pad / 8), 256), kMostGroups)), 2), 256, 0, stream>>>(p);
    return o;
}

ProductArgs formed(const LinearArgs &a, const Operands &o, const Gated &c, Space &s) {
    ProductArgs p{};
    p.pad_n = pad64(a.n_out);
    if (c.splits > 1) p.part = s.take_floats(c.splits * a.rows * p.pad_n);
    p.a = p.a2 = o.w;
    p.b = o.x;
    p.k = p.k2 = o.k;
    p.act = a.act;
    p.bias = a.bias;
    p.n = a.n_out;
    p.m = a.rows;
    return p;
}

template <class T> void linear(const LinearArgs &a, hipStream_t stream) {
    if (a.rows <= kFewRows) return launch_few<T, T>(a, stream);
    Space s(aligned(a.ws));
    const Gated g = linear_cut(a.dtype, a.rows, a.n_in, a.n_out);
    const Operands o = operands<T>(a, s, stream);
    ProductArgs p = formed(a, o, g, s);
    p.residual = a.residual;
    p.ld_r = a.ld_r;
    p.out = a.y;
    p.ld = a.ld_y;
    launch_product<T, kLinear>(g, p, a.n_out, a.rows, stream);
}

template <class T, int BA, int BB, int NA, int NB> void launch_tiles8(Product8Args a, hipStream_t stream) {
    a.out.tiles_n = ceil_div(a.out.n, BA);
    a.out.tiles_m = ceil_div(a.out.m, BB);
    product8<T, BA, BB, NA, NB><<<dim3(uint32_t(a.out.tiles_n * a.out.tiles_m * a.out.splits)), 64 * NA * NB, 0, stream>>>(a);
}

template <class T> void linear_8bit(const LinearArgs &a, hipStream_t stream) {
    if (a.rows <= kFewRows) return launch_few<byte, T>(a, stream);
    char *ws = aligned(a.ws);
    const Gated g = linear_cut(NDVM_BF16, a.rows, ceil_div(a.n_in, 2), a.n_out);
    Product8Args p{};
    p.x = static_cast<const byte *>(a.x);
    p.w = static_cast<const byte *>(a.w);
    p.ld_x = a.ld_x;
    p.ld_w = a.ld_w;
    p.k = a.n_in;
    const auto granules = [&](const void *q, int64_t ld) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % 16 == 0 && ld <= 2 * kMostFfnWidth; };
    if (a.n_in % 16 || !granules(a.x, a.ld_x) || !granules(a.w, a.ld_w)) {
        Pack8Args c{};
        c.cols = a.n_in;
        c.pad = p.k = p.ld_x = p.ld_w = pad64(a.n_in);
        c.from[0] = p.x;
        c.from[1] = p.w;
        c.to[0] = reinterpret_cast<byte *>(ws);
        c.to[1] = reinterpret_cast<byte *>(ws += round256(size_t(a.rows) * size_t(c.pad)));
        ws += round256(size_t(a.n_out) * size_t(c.pad));
        c.rows[0] = a.rows;
        c.rows[1] = a.n_out;
        c.ld[0] = a.ld_x;
        c.ld[1] = a.ld_w;
        p.x = c.to[0];
        p.w = c.to[1];
        pack8<<<dim3(uint32_t(std::min(ceil_div(std::max(a.rows, a.n_out) * (c.pad / 16), 256), kMostGroups)), 2), 256, 0, stream>>>(c);
    }
    p.out.splits = int(g.splits);
    p.out.part = reinterpret_cast<float *>(ws);
    p.out.pad_n = pad64(a.n_out);
    p.out.n = a.n_out;
    p.out.m = a.rows;
    p.out.act = a.act;
    p.out.bias = a.bias;
    p.out.residual = a.residual;
    p.out.ld_r = a.ld_r;
    p.out.x_scale = a.x_scale;
    p.out.w_scale = a.w_scale;
    p.out.out = a.y;
    p.out.ld = a.ld_y;
    if (g.bb == 256) launch_tiles8<T, 256, 256, 2, 4>(p, stream);
    else if (g.ba == 256) launch_tiles8<T, 256, 128, 4, 2>(p, stream);
    else launch_tiles8<T, 128, 128, 2, 2>(p, stream);
    if (g.splits > 1) fold_linear<T><<<dim3(uint32_t(ceil_div(p.out.pad_n / 8 * p.out.m, 256))), 256, 0, stream>>>(p.out);
}

template <class T> void linear_grad(const LinearArgs &a, hipStream_t stream) {
    Space s(aligned(a.ws));
    const int64_t pad_n = pad64(a.n_out);
    const Operands o = operands<T>(a, s, stream);
    Operand dz{a.dy, a.rows, a.ld_dy, 0};
    unsigned *largest = nullptr;
    ColumnArgs c{};
    if (a.db) c.part = s.take_floats(column_floats(a.rows, a.n_out));
    if (a.act != NDVM_ACT_NONE) {
        const Gated g = linear_cut(a.dtype, a.rows, a.n_in, a.n_out);
        ProductArgs p = formed(a, o, g, s);
        p.dh = a.dy;
        p.ld_dh = a.ld_dy;
        p.p = s.take(a.dtype, a.rows, pad_n);
        p.ld_p = pad_n;
        p.plane_p = s.plane;
        p.sums = c.part;
        if (std::is_same<T, f16>::value) p.largest = largest = reinterpret_cast<unsigned *>(s.take_floats(1));
        if (a.rows) launch_product<T, kLinearGrad>(g, p, pad_n, a.rows, stream);
        dz = Operand{p.p, a.rows, pad_n, p.plane_p};
        // without rows nothing notes the largest: there is nothing to scale
        if (a.rows == 0) largest = nullptr;
    } else if ((a.dx || a.dw) && !(direct(a.dtype, a.dy, a.ld_dy, a.n_out) && a.n_out == pad_n)) {
        PackArgs p{};
        p.cols = a.n_out;
        p.pad = pad_n;
        p.from[0] = a.dy;
        p.to[0] = s.take(a.dtype, a.rows, pad_n);
        p.rows[0] = a.rows;
        p.ld[0] = a.ld_dy;
        p.plane[0] = s.plane;
        if (a.rows) pack<T><<<dim3(uint32_t(std::min(ceil_div(a.rows * (pad_n / 8), 256), kMostGroups))), 256, 0, stream>>>(p);
        dz = Operand{p.to[0], a.rows, pad_n, s.plane};
    }
    const Pieces cut = linear_pieces(a.dtype, a.rows, a.n_in, a.n_out);
    ProductArgs dx{}, dw{};
    dx.splits = dw.splits = 1;
    dx.largest = dw.largest = largest;
    if (a.dx) {     // n: x's columns; the sum: the rows of W
        dx.a = dx.a2 = o.w;
        dx.b = dz;
        dx.k = dx.k2 = pad_n;
        dx.out = a.dx;
        dx.ld = a.ld_dx;
        dx.n = a.n_in;
        dx.m = dx.split = dx.split2 = dx.m2 = a.rows;
        dx.splits = int(cut.dx);
        if (cut.dx > 1) dx.part = s.take_floats(cut.dx * a.rows * a.n_in);
    }
    if (a.dw) {     // m: the columns of dz; the sum: rows
        dw.a = dw.a2 = o.x;
        dw.k = dw.k2 = pad64(a.rows);
        dw.b = dz;
        dw.out = a.dw;
        dw.ld = a.ld_dw;
        dw.n = a.n_in;
        dw.m = dw.split2 = dw.m2 = pad_n;
        dw.split = a.n_out;
        dw.splits = int(cut.dw);
        if (cut.dw > 1) dw.part = s.take_floats(cut.dw * dw.m * a.n_in);
    }
    if (cut.tile == 256) launch_pair<T, 256, 2, 4>(dx, dw, stream);
    else launch_pair<T, 128, 2, 2>(dx, dw, stream);
    if (!a.db) return;
    c.dy = a.dy;
    c.ld = a.ld_dy;
    c.rows = a.rows;
    c.n = a.n_out;
    c.pad = pad_n;
    c.to = a.db;
    int64_t groups = ceil_div(a.rows, 64);
    if (a.act == NDVM_ACT_NONE) {
        groups = std::min(groups, kColumnGroups);
        if (groups) column_sums<T><<<dim3(uint32_t(ceil_div(a.n_out, 256)), uint32_t(groups)), 256, 0, stream>>>(c);
    }
    column_fold<T><<<dim3(uint32_t(ceil_div(a.n_out, 32))), 256, 0, stream>>>(c, int(groups));
}

}  // namespace

hipError_t launch_linear(const LinearArgs &a, hipStream_t stream) {
    return with_type(a.dtype, [&](auto zero) {
        linear<decltype(zero)>(a, stream);
        return hipGetLastError();
    });
}
hipError_t launch_linear_8bit(const LinearArgs &a, hipStream_t stream) {
    if (a.dtype == NDVM_BF16) linear_8bit<bf16>(a, stream);
    else linear_8bit<f16>(a, stream);
    return hipGetLastError();
}
hipError_t launch_linear_grad(const LinearArgs &a, hipStream_t stream) {
    return with_type(a.dtype, [&](auto zero) {
        linear_grad<decltype(zero)>(a, stream);
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
