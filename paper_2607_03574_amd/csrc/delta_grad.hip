// Gradient of attention by the gated delta rule.  (Formulas: delta_parts.h.)
// Launches: the chunks' records; where few sequences are long, their segments; the walk forwards, which leaves m and the state
// before each block of 64 tokens, beside the walk backwards, which leaves dv, e and the state's gradient after each block;
// then every block by itself.  With u = b m, x = b e, and within a block
//   Pd_ij = s L_ij do_i.u_j (j <= i),  Ad_ij = -L_ij x_i.u_j (j < i)
//   dq = diag(s exp G) do S^T + Pd K
//   dk = diag(exp(G_last - G)) U D^T - diag(exp G) X S^T + (Ad + Ad^T) K + Pd^T Q
//   db_i = e_i.m_i
//   dg_t = exp(G_last) <D, S> + sum_{j<t} f_j + sum_{i>=t} (y_i - z_i) + sum_{i>=t>j} (Pd_ij q_i.k_j + Ad_ij k_i.k_j)
// f, y, z: the products of k's, q's and k's rows with those of the first terms above.  What decays between two tokens counts
// for every t between them: no difference of large sums.
#include "delta_walk.h"

namespace ndvm {
namespace ops {
namespace {

// z: 0 forwards, 1 backwards.  (8 x 2048 tokens x 16 heads of 128 bf16: 343 us for both, 850 MB written.)
template <class T, int DK, Walk WALK> __global__ void __launch_bounds__(256, (kResident<T, DK>)) delta_grad_walk(DeltaArgs a) {
    __shared__ __align__(16) char lds[kWalkLds<T, DK, true, kReadBack>];
    const uint32_t id = blockIdx.x / uint32_t(a.heads);
    const int64_t h = blockIdx.x - id * uint32_t(a.heads);
    const int tile = int(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const Piece g = find_piece(a, id, a.seg_len, !a.segments);
    if (g.count == 0 || (blockIdx.z && blockIdx.y * 64 >= a.dv)) return;
    if (blockIdx.z == 0) {
        if (a.m || WALK == kSums) walk<T, DK, WALK>(a, lds, g, blockIdx.x, h, tile);
    } else {
        walk_back<T, DK, WALK>(a, lds, g, blockIdx.x, h, tile);
    }
}

template <int DK> __global__ void __launch_bounds__(256) delta_grad_carry(DeltaArgs a) {
    __shared__ __align__(16) char lds[kCarryLds<DK>];
    const uint32_t seq = blockIdx.x / uint32_t(a.heads);
    const int64_t h = blockIdx.x - seq * uint32_t(a.heads);
    const int tile = int(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if (blockIdx.z == 0) {
        if (a.m) carry<DK, false>(a, lds, seq, h, tile);
    } else {
        carry<DK, true>(a, lds, seq, h, tile);
    }
}

// A block's LDS: 32 columns of u, x and do as parts, later the pairs' matrices; the rows of q, later of k.
template <class T> constexpr int kSlab = 64 * 64;      // bytes of 32 columns of a part
template <class T> constexpr int kPair = 64 * 128;     // of a part of a pairs' matrix, [j][i]
template <class T> constexpr int kSlabs = (2 * kResultParts<T> + kInputParts<T>) * kSlab<T>;
// two lots of columns, where there is room
template <class T, int DK> constexpr int kLots = kInputParts<T> * DK <= 512 ? 2 : 1;
template <class T, int DK> constexpr int kArea = std::max(kLots<T, DK> * kSlabs<T>, 2 * kResultParts<T> * kPair<T>);

// Over the 16 lanes of a row, in all of them.
__device__ inline float sum_of_16(float v) {
#ifdef __HIP_DEVICE_COMPILE__
    const auto turn = [&](auto by) __attribute__((always_inline)) {
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + decltype(by)::value, 0xf, 0xf, false));     // row_ror
    };
    turn(std::integral_constant<int, 8>());
    turn(std::integral_constant<int, 4>());
    turn(std::integral_constant<int, 2>());
    turn(std::integral_constant<int, 1>());
#endif
    return v;
}

// Bound by waiting: 8 x 2048 tokens x 16 heads of 128 bf16 428 us, 1.0 GB read at 2.4 TB/s, one workgroup of eight waves a compute
// unit (four waves with twice the widths, 500 registers: 728; two workgroups of 128 registers: 1,113, they spill).
// W waves and a block: a wave has 64 tokens x 16 NT widths of dq and dk, and 16 rows x 16 PT columns of the pairs' matrices.
template <int DK> constexpr int kBlockWaves = DK >= 128 ? 8 : 4;
// waves on a matrix unit
template <class T, int DK> constexpr int kBlockResident = DK >= 128 || kInputParts<T> == 1 ? 2 : 1;
template <class T, int DK> __global__ void __launch_bounds__(64 * kBlockWaves<DK>, (kBlockResident<T, DK>)) delta_blocks(DeltaArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int W = kBlockWaves<DK>, THREADS = 64 * W, PT = 16 / W;
    constexpr int PARTS = kInputParts<T>, HELD = kResultParts<T>, NT = DK <= 16 * W ? 1 : DK / (16 * W), G = DK / 8, ROWS = 64 * G * 16;
    constexpr int LOADS = 64 * G / THREADS, SLAB = kSlab<T>, PAIR = kPair<T>;
    __shared__ __align__(16) char area[kArea<T, DK>], rows[PARTS * ROWS];
    __shared__ double sum[64], row_sum[W / 4][64], col_sum[4][64];
    __shared__ float betas[64], rise[64], fall[64], dots[W][3][64], between[W];
    const uint32_t id = blockIdx.x / uint32_t(a.heads);
    const int64_t h = blockIdx.x - id * uint32_t(a.heads);
    const Piece g = find_piece(a, id, kDeltaBlock);
    if (g.count == 0) return;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int len = int(g.len);
    const int w0 = wave * 16 * NT;
    const bool has = w0 < DK;
    const int row_tile = wave % 4, col_tile = wave / 4 * PT;
    const auto width = [&](int n) { return NT == 1 ? w0 + lm : w0 + 32 * (n / 2) + 8 * (lm / 4) + 4 * (n % 2) + lm % 4; };

    // (what is not there is read at another place, and is 0 when it is put)
    Eight<T> held[LOADS];
    const auto fetch_rows = [&](const Heads &x) __attribute__((always_inline)) {
        const T *p = at_token<T>(x, a, g, g.begin, h);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * THREADS + threadIdx.x, row = at / G, gr = at % G;
            get_eight(held[i], p, row < len && gr * 8 < a.dkp ? (uint32_t(row) * uint32_t(x.tok) + gr * 8) * sizeof(T) : 0);
        }
    };
    const auto put_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * THREADS + threadIdx.x, row = at / G, gr = at % G;
            const bool in = row < len && gr * 8 < a.dkp;
            bf16x8 p[PARTS];
            parts_of(held[i], p);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8 *>(rows + q * ROWS + (row * G + (gr ^ turned<G>(row))) * 16) = in ? p[q] : bf16x8(bf16(0.0f));
        }
    };
    fetch_rows(a.q);
    // over 32 columns of v after the other: do S^T, X S^T, U D^T, do U^T, X U^T, e.m and <D, S>
    // (of eight waves, four bring u and x, the others do)
    const int srow = threadIdx.x % 256 / 4, sgr = threadIdx.x % 4;
    const bool of_states = W == 4 || threadIdx.x < 256, of_do = W == 4 || threadIdx.x >= 256;
    const int64_t at_row = (h * a.n_tokens + g.first + g.begin) * a.dvp;
    const T *const dop = at_token<T>(a.d_o, a, g, g.begin, h);
    const float beta = srow < len ? float(*at_token<T>(a.beta, a, g, g.begin + srow, h)) : 0.0f;
    const float *const sp = a.states + (int64_t(id) * a.heads + h) * a.dk * a.dvp, *const dp = a.d_states + (int64_t(id) * a.heads + h) * a.dk * a.dvp;
    Eight<float> m, e, S[NT], D[NT];
    Eight<T> o;
    const int dvp = int(a.dvp);
    const auto fetch = [&](int c) __attribute__((always_inline)) {
        const bool in = srow < len && c + sgr * 8 < dvp;
        const uint32_t off = in ? (uint32_t(srow) * uint32_t(dvp) + c + sgr * 8) * 4 : 0;
        if (of_states) {
            get_eight(m, a.m + at_row, off);
            get_eight(e, a.e + at_row, off);
        }
        if (of_do) get_eight(o, dop, in ? (uint32_t(srow) * uint32_t(a.d_o.tok) + c + sgr * 8) * sizeof(T) : 0);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t at = width(n) < a.dk && c + 8 * lg < dvp ? (uint32_t(width(n)) * uint32_t(dvp) + c + 8 * lg) * 4 : 0;
            get_eight(S[n], sp, at);
            get_eight(D[n], dp, at);
        }
    };
    fetch(0);
    put_rows();
    if (wave == 0) {
        double log_a = 0.0;
        float beta = 0.0f;
        if (l < len) {
            beta = float(*at_token<T>(a.beta, a, g, g.begin + l, h));
            log_a = log_decay(*at_token<T>(a.g, a, g, g.begin + l, h));
        }
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const double before = __shfl_up(log_a, s);
            if (l >= s) log_a += before;
        }
        sum[l] = log_a;
        betas[l] = beta;
        rise[l] = expf(float(log_a));
        fall[l] = expf(float(__shfl(log_a, 63) - log_a));
    }

    f32x4 a1[4][NT], a2[4][NT], a3[4][NT], pd[PT], ad[PT];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        pd[i % PT] = ad[i % PT] = 0;
#pragma unroll
        for (int n = 0; n < NT; ++n) a1[i][n] = a2[i][n] = a3[i][n] = 0;
    }
    float db = 0.0f, ds = 0.0f;
    const auto put = [&](int c) __attribute__((always_inline)) {
        char *const of_u = area + c / 32 % kLots<T, DK> * kSlabs<T>, *const of_x = of_u + HELD * SLAB, *const of_o = of_x + HELD * SLAB;
        const bool in = srow < len && c + sgr * 8 < dvp;
        const int at = srow * 64 + (sgr ^ turned<4>(srow)) * 16;
        if (of_states) {
            bf16x8 u[HELD], x[HELD];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float mi = in ? value(m, i) : 0.0f, ei = in ? value(e, i) : 0.0f;
                db += ei * mi;
                split(beta * mi, u, i);
                split(beta * ei, x, i);
            }
#pragma unroll
            for (int q = 0; q < HELD; ++q) {
                *reinterpret_cast<bf16x8 *>(of_u + q * SLAB + at) = u[q];
                *reinterpret_cast<bf16x8 *>(of_x + q * SLAB + at) = x[q];
            }
        }
        if (of_do) {
            bf16x8 p[PARTS];
            parts_of(o, p);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8 *>(of_o + q * SLAB + at) = in ? p[q] : bf16x8(bf16(0.0f));
        }
    };
    put(0);
    __syncthreads();
    for (int c = 0; c < dvp; c += 32) {
        const char *const of_u = area + c / 32 % kLots<T, DK> * kSlabs<T>, *const of_x = of_u + HELD * SLAB, *const of_o = of_x + HELD * SLAB;
        bf16x8 s[NT][HELD], d[NT][HELD];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const bool in = width(n) < a.dk && c + 8 * lg < dvp;
            float sd = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sd += value(S[n], i) * value(D[n], i);
            ds += in ? sd : 0.0f;
            parts_of(S[n], s[n]);
            parts_of(D[n], d[n]);
#pragma unroll
            for (int q = 0; q < HELD; ++q)
                if (!in) s[n][q] = d[n][q] = bf16x8(bf16(0.0f));
        }
        if (c + 32 < dvp) fetch(c + 32);
        const auto operand = [&](const char *from, int tile, auto &x) __attribute__((always_inline)) {
            const int row = 16 * tile + lm;
            constexpr int N = sizeof(x) / sizeof(bf16x8);
#pragma unroll
            for (int q = 0; q < N; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(from + q * SLAB + row * 64 + (lg ^ turned<4>(row)) * 16);
        };
        bf16x8 own_o[PARTS], own_x[HELD];
        operand(of_o, row_tile, own_o);
        operand(of_x, row_tile, own_x);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            bf16x8 u[HELD], x[HELD], p[PARTS];
            operand(of_u, t, u);
            if (has) {
                operand(of_x, t, x);
                operand(of_o, t, p);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    a1[t][n] = multiply<HELD - 1>(p, s[n], a1[t][n]);
                    a2[t][n] = multiply<HELD - 1>(x, s[n], a2[t][n]);
                    a3[t][n] = multiply<HELD - 1>(u, d[n], a3[t][n]);
                }
            }
            if (t / PT * PT == col_tile && t <= row_tile) {
                pd[t % PT] = multiply<HELD - 1>(own_o, u, pd[t % PT]);
                ad[t % PT] = multiply<HELD - 1>(own_x, u, ad[t % PT]);
            }
        }
        if (kLots<T, DK> == 1) __syncthreads();
        if (c + 32 < dvp) put(c + 32);
        __syncthreads();
    }
    fetch_rows(a.k);
    // Pd and Ad, transposed, where the columns of v lay
#pragma unroll
    for (int t = 0; t < PT; ++t) {
        const int j = 16 * (col_tile + t) + lm;
        const double gj = sum[j];
        bf16x4 p[HELD], x[HELD];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * row_tile + 4 * lg + r;
            const float decay = j <= i ? expf(float(sum[i] - gj)) : 0.0f;
            pd[t][r] = j <= i ? a.scale * decay * pd[t][r] : 0.0f;
            ad[t][r] = j < i ? -decay * ad[t][r] : 0.0f;
            split(pd[t][r], p, r);
            split(ad[t][r], x, r);
        }
        const int at = j * 128 + ((2 * row_tile + lg / 2) ^ turned<8>(j)) * 16 + lg % 2 * 8;
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            *reinterpret_cast<bf16x4 *>(area + q * PAIR + at) = p[q];
            *reinterpret_cast<bf16x4 *>(area + (HELD + q) * PAIR + at) = x[q];
        }
    }
    __syncthreads();
    // operands of the pairs' matrices: 16 rows j, 32 columns i as they lie; or 16 rows i, 32 columns j
    const auto down = [&](const char *from, int tile, int step, bf16x8(&x)[HELD]) __attribute__((always_inline)) {
        const int row = 16 * tile + lm;
#pragma unroll
        for (int q = 0; q < HELD; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(from + q * PAIR + row * 128 + ((4 * step + lg) ^ turned<8>(row)) * 16);
    };
    const auto across = [&](const char *from, int tile, int step, bf16x8(&x)[HELD]) __attribute__((always_inline)) {
        const int row = 32 * step + 8 * lg + lm / 4, gr = 2 * tile + lm % 4 / 2;
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            const char *p = from + q * PAIR + lm % 2 * 8;
            const bf16x4 lo = read_transposed(p + row * 128 + (gr ^ turned<8>(row)) * 16);
            const bf16x4 hi = read_transposed(p + (row + 4) * 128 + (gr ^ turned<8>(row + 4)) * 16);
            x[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };
    // 32 rows of q or k, the wave's widths, as the right operand
    const auto widths = [&](int step, int n, bf16x8(&x)[PARTS]) __attribute__((always_inline)) {
        const int row = 32 * step + 8 * lg + lm / 4;
        const int gr = NT == 1 ? w0 / 8 + lm % 4 / 2 : w0 / 8 + 4 * (n / 2) + lm % 4, off = NT == 1 ? lm % 2 * 8 : n % 2 * 8;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            const char *p = rows + q * ROWS + off;
            const bf16x4 lo = read_transposed(p + (row * G + (gr ^ turned<G>(row))) * 16);
            const bf16x4 hi = read_transposed(p + ((row + 4) * G + (gr ^ turned<G>(row + 4))) * 16);
            x[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };
    // a value of q or k
    const auto value_at = [&](int row, int w) __attribute__((always_inline)) {
        const char *p = rows + (row * G + ((w / 8) ^ turned<G>(row))) * 16 + w % 8 * 2;
        float v = float(*reinterpret_cast<const bf16 *>(p));
#pragma unroll
        for (int q = 1; q < PARTS; ++q) v += float(*reinterpret_cast<const bf16 *>(p + q * ROWS));
        return v;
    };
    // over the widths of the wave: the products of a token's row and what it gets
    const auto dot = [&](int which, int t, const f32x4(&x)[NT], const f32x4(&y)[NT], auto both) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int token = 16 * t + 4 * lg + r;
            float v = 0.0f, w = 0.0f;
            if (has)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const float at = value_at(token, width(n));
                    v += at * x[n][r];
                    if constexpr (decltype(both)::value) w += at * y[n][r];
                }
            v = sum_of_16(v);
            if (lm == 0) dots[wave][which][token] = v;
            if constexpr (decltype(both)::value) {
                w = sum_of_16(w);
                if (lm == 0) dots[wave][which + 1][token] = w;
            }
        }
    };
    f32x4 out[4][NT];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            out[t][n] = 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * lg + r;
                a1[t][n][r] *= rise[i] * a.scale;
                a2[t][n][r] *= rise[i];
                a3[t][n][r] *= fall[i];
            }
        }
        dot(0, t, a1[t], a1[t], std::false_type());
    }
    if (has) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            bf16x8 y[NT][PARTS];
#pragma unroll
            for (int n = 0; n < NT; ++n) widths(step, n, y[n]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (32 * step + 31 < 16 * t) continue;      // all of its i lie before j
                bf16x8 p[HELD];
                down(area, t, step, p);
#pragma unroll
                for (int n = 0; n < NT; ++n) out[t][n] = multiply<HELD - 1>(p, y[n], out[t][n]);
            }
        }
    }
    __syncthreads();
    put_rows();
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        dot(1, t, a2[t], a3[t], std::true_type());
#pragma unroll
        for (int n = 0; n < NT; ++n) out[t][n] += a3[t][n] - a2[t][n];
    }
    if (has) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            bf16x8 y[NT][PARTS];
#pragma unroll
            for (int n = 0; n < NT; ++n) widths(step, n, y[n]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                bf16x8 p[HELD];
                if (32 * step <= 16 * t + 15) {
                    across(area, t, step, p);
#pragma unroll
                    for (int n = 0; n < NT; ++n) a1[t][n] = multiply<HELD - 1>(p, y[n], a1[t][n]);
                    across(area + HELD * PAIR, t, step, p);
#pragma unroll
                    for (int n = 0; n < NT; ++n) out[t][n] = multiply<HELD - 1>(p, y[n], out[t][n]);
                }
                if (32 * step + 31 >= 16 * t) {
                    down(area + HELD * PAIR, t, step, p);
#pragma unroll
                    for (int n = 0; n < NT; ++n) out[t][n] = multiply<HELD - 1>(p, y[n], out[t][n]);
                }
            }
        }
    }
    // what pairs add to dg: q k^T and k k^T of the wave's rows
    {
        f32x4 qk[PT], kk[PT];
#pragma unroll
        for (int t = 0; t < PT; ++t) qk[t] = kk[t] = 0;
        const auto operand = [&](int tile, int ks, bf16x8(&x)[PARTS]) __attribute__((always_inline)) {
            const int row = 16 * tile + lm;
#pragma unroll
            for (int q = 0; q < PARTS; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(rows + q * ROWS + (row * G + ((4 * ks + lg) ^ turned<G>(row))) * 16);
        };
        const int row = 16 * row_tile + lm;
        const T *const qp = at_token<T>(a.q, a, g, g.begin, h);
#pragma unroll
        for (int ks = 0; ks < DK / 32; ++ks) {
            bf16x8 q[PARTS], k[PARTS];
            const bool in = row < len && ks * 32 + 8 * lg < a.dkp;
            Eight<T> eight;
            get_eight(eight, qp, in ? (uint32_t(row) * uint32_t(a.q.tok) + ks * 32 + 8 * lg) * sizeof(T) : 0);
            parts_of(eight, q);
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
                if (!in) q[i] = bf16x8(bf16(0.0f));
            operand(row_tile, ks, k);
#pragma unroll
            for (int t = 0; t < PT; ++t) {
                if (col_tile + t > row_tile) continue;
                bf16x8 x[PARTS];
                operand(col_tile + t, ks, x);
                qk[t] = multiply<HELD - 1>(q, x, qk[t]);
                kk[t] = multiply<HELD - 1>(k, x, kk[t]);
            }
        }
        double of_row[4] = {0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < PT; ++t) {
            double of_col = 0;
            const int j = 16 * (col_tile + t) + lm;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * row_tile + 4 * lg + r;
                const double w = j < i ? double(pd[t][r] * qk[t][r] + ad[t][r] * kk[t][r]) : 0.0;
                of_row[r] += w;
                of_col += w;
            }
            of_col += __shfl_xor(of_col, 16);
            of_col += __shfl_xor(of_col, 32);
            if (lg == 0) col_sum[row_tile][j] = of_col;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int s = 1; s < 16; s <<= 1) of_row[r] += __shfl_xor(of_row[r], s);
            if (lm == 0) row_sum[wave / 4][16 * row_tile + 4 * lg + r] = of_row[r];
        }
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) ds += __shfl_xor(ds, s);
    if (l == 0) between[wave] = ds;
    __syncthreads();
    if (wave == 0 && a.dg.p) {
        float y = 0, z = 0, f = 0;
        double pairs = 0, whole = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            y += dots[w][0][l];
            z += dots[w][1][l];
            f += dots[w][2][l];
            whole += between[w];
            if (w < W / 4) pairs += row_sum[w][l];
            if (w < 4) pairs -= col_sum[w][l];
        }
        whole *= rise[63];
        double after = double(y) - double(z) + pairs, before = f;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const double x = __shfl_down(after, s), y2 = __shfl_up(before, s);
            if (l + s < 64) after += x;
            if (l >= s) before += y2;
        }
        if (l < len) *const_cast<T *>(at_token<T>(a.dg, a, g, g.begin + l, h)) = T(float(whole + (before - f) + after));
    }
    db += __shfl_xor(db, 1);
    db += __shfl_xor(db, 2);
    if (a.dbeta.p && of_states && sgr == 0 && srow < len) *const_cast<T *>(at_token<T>(a.dbeta, a, g, g.begin + srow, h)) = T(db);
    if (!has) return;
    // (the piece of memory that the block's rows lie in: what is beyond it is not stored)
    const auto rows_to = [&](auto *p, uint32_t step, const f32x4(&x)[4][NT]) __attribute__((always_inline)) {
        typedef std::remove_pointer_t<decltype(p)> V;
        if (len == 1) step = 256;       // (rows need not be apart where there is one)
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(same(p), 0, ((len - 1) * step + uint32_t(a.dk)) * sizeof(V), 0x00020000);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (width(n) >= a.dk) continue;
            const uint32_t at = (4 * lg * step + width(n)) * sizeof(V);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t off = at + (16 * t + r) * step * uint32_t(sizeof(V));
                    const V v = V(x[t][n][r]);
                    if constexpr (sizeof(V) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), rsrc, off, 0, 0);
                    else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), rsrc, off, 0, 0);
                }
        }
    };
    const auto store = [&](const Heads &to, float *part, const f32x4(&x)[4][NT]) __attribute__((always_inline)) {
        if (!to.p) return;
        if (part) rows_to(part + (h * a.n_tokens + g.first + g.begin) * a.dk, uint32_t(a.dk), x);
        else rows_to(const_cast<T *>(at_token<T>(to, a, g, g.begin, h)), uint32_t(to.tok), x);
    };
    store(a.dq, a.dq_part, a1);
    store(a.dk_out, a.dk_part, out);
#endif
}

// What heads that share q and k give them, added up; rows of no sequence stay as they are.  y: heads of q and k; z: dq, dk.
template <class T> __global__ void __launch_bounds__(256) delta_fold(DeltaArgs a) {
    const Heads &to = blockIdx.z ? a.dk_out : a.dq;
    const float *part = blockIdx.z ? a.dk_part : a.dq_part;
    if (!to.p) return;
    const int64_t begin = a.offsets ? token_at(a, 0) : 0, end = a.offsets ? token_at(a, a.n_seq) : a.n_tokens, per = a.n_tokens / a.n_seq;
    for (int64_t at = begin * a.dk + int64_t(blockIdx.x) * 256 + threadIdx.x; at < end * a.dk; at += int64_t(gridDim.x) * 256) {
        const int64_t token = at / a.dk, d = at - token * a.dk;
        float s = 0;
        for (int i = 0; i < to.group; ++i) s += part[((int64_t(blockIdx.y) * to.group + i) * a.n_tokens) * a.dk + at];
        const int64_t row = a.offsets ? token * to.tok : token / per * to.seq + token % per * to.tok;
        static_cast<T *>(const_cast<void *>(to.p))[row + blockIdx.y * to.head + d] = T(s);
    }
}

// need: whether anything but dv and the initial state's gradient is wanted
template <class T> size_t lay_out(DeltaArgs &a, Space s, bool need) {
    const int64_t states = a.heads * a.dk * a.dv * 4;
    a.dkp = padded(a.dk);
    a.dvp = padded(a.dv);
    a.record = kRecordGrad;
    if (a.dk % 8) {
        s.take(a.k_rows, a.n_tokens * (a.heads / a.k.group) * a.dkp * int64_t(sizeof(T)));
        s.take(a.q_rows, a.n_tokens * (a.heads / a.k.group) * a.dkp * int64_t(sizeof(T)));
    }
    if (a.dv % 8) s.take(a.d_rows, a.n_tokens * a.heads * a.dvp * int64_t(sizeof(T)));
    s.take(a.chunks, piece_ids(a, kDeltaChunk) * a.heads * a.record);
    if (cut(a)) {
        s.take(a.segments, a.n_segments * states);
        s.take(a.d_segments, a.n_segments * states);
        s.take(a.moves, a.n_segments * a.heads * a.dk * a.dkp * 4);
        s.take(a.moves_t, a.n_segments * a.heads * a.dk * a.dkp * 4);
    }
    if (!need) return s.used + 256;
    const int64_t blocks = piece_ids(a, kDeltaBlock);
    s.take(a.states, blocks * a.heads * a.dk * a.dvp * 4);
    s.take(a.d_states, blocks * a.heads * a.dk * a.dvp * 4);
    s.take(a.m, a.heads * a.n_tokens * a.dvp * 4);
    s.take(a.e, a.heads * a.n_tokens * a.dvp * 4);
    if (a.k.group > 1) {
        s.take(a.dq_part, a.heads * a.n_tokens * a.dk * 4);
        s.take(a.dk_part, a.heads * a.n_tokens * a.dk * 4);
    }
    return s.used + 256;
}

template <class T> void delta_grad(DeltaArgs a, hipStream_t stream) {
    const bool need = a.dq.p || a.dk_out.p || a.dg.p || a.dbeta.p;
    lay_out<T>(a, Space(a.ws), need);
    pad_rows<T>(a, a.k, a.k_rows, a.dk, stream);
    pad_rows<T>(a, a.q, a.q_rows, a.dk, stream);
    pad_rows<T>(a, a.d_o, a.d_rows, a.dv, stream);
    const int64_t pairs = piece_ids(a, kDeltaChunk) * a.heads;
    if (a.n_tokens) delta_prepare<T, true><<<dim3(uint32_t(ceil_div(pairs, 4))), 256, 0, stream>>>(a, pairs);
    with_width(a.dk, [&](auto d) {
        constexpr int DK = decltype(d)::value;
        const auto grid = [&](int64_t ids, int64_t tiles) { return dim3(uint32_t(ids * a.heads), uint32_t(ceil_div(tiles, 4)), 2); };
        const int64_t of_v = ceil_div(a.dv, 16), of_k = ceil_div(a.dk, 16);
        if (a.segments) {
            delta_grad_walk<T, DK, kSums><<<grid(a.n_segments, of_v + of_k), 256, 0, stream>>>(a);
            delta_grad_carry<DK><<<grid(a.n_seq, of_v), 256, 0, stream>>>(a);
        }
        delta_grad_walk<T, DK, kKept><<<grid(a.n_segments, of_v), 256, 0, stream>>>(a);
        if (need && a.n_tokens) delta_blocks<T, DK><<<dim3(uint32_t(piece_ids(a, kDeltaBlock) * a.heads)), 64 * kBlockWaves<DK>, 0, stream>>>(a);
    });
    if (a.dq_part && (a.dq.p || a.dk_out.p) && a.n_tokens) {
        const int64_t groups = std::min(ceil_div(a.n_tokens * a.dk, 256), kMostGroups);
        delta_fold<T><<<dim3(uint32_t(groups), uint32_t(a.heads / a.k.group), 2), 256, 0, stream>>>(a);
    }
}

}  // namespace

size_t delta_grad_bytes(int dtype, const DeltaArgs &a) {
    DeltaArgs b = a;
    return dtype == NDVM_F32 ? lay_out<float>(b, Space(nullptr), true) : lay_out<bf16>(b, Space(nullptr), true);
}

hipError_t launch_delta_grad(int dtype, DeltaArgs a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        delta_grad<decltype(zero)>(a, stream);
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
