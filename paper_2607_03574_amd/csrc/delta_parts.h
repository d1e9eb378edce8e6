// What the kernels of the gated delta rule share: pieces of sequences, values as bf16 parts, and the
// record that is kept for a chunk of 32 tokens and a head.
//   S_t = a_t S_{t-1} + k_t^T u_t,  u_t = b_t (v_t - a_t k_t S_{t-1}),  o_t = s q_t S_t,  a_t = exp(g_t)
// Over a chunk, with G the running sum of g in it, L_ij = exp(G_i - G_j) and S what entered it:
//   (I + A) M = X = V - diag(exp G) K S,  U = diag(b) M,  A_ij = L_ij k_i.k_j b_j for j < i
//   O = s (diag(exp G) Q S + P U),  P_ij = L_ij q_i.k_j for j <= i
//   S' = exp(G_last) S + sum_j exp(G_last - G_j) k_j^T u_j
// The gradient, with D that of S', do that of O, and A_ij = A'_ij b_j:
//   dU = s P^T do + diag(exp(G_last - G)) K D,  E = (I + diag(b) A')^-T dU,  dV = dX = diag(b) E,  db_i = e_i.m_i
//   dS = exp(G_last) D + Q^T diag(s exp G) do - K^T diag(exp G) dX
// Both inverses come from B = (I + A)^-1 A': they are I - B diag(b) and I - diag(b) B.
// All sums and states are in float; products are made of bf16 parts on the bf16 matrix instructions (16 times the
// rate of the float ones): 16-bit inputs are one part (bfloat16) or two (half), floats three; what the state is made
// of is three parts, products whose places add up to 2 at most: 2^-21 of a term is left out at most, 2^-24 on
// average.  What only reaches a 16-bit result is two parts, so that the result is off by its own rounding alone.
#pragma once
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "ops_types.h"

namespace ndvm {
namespace ops {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> constexpr int kInputParts = sizeof(T) == 4 ? 3 : std::is_same<T, f16>::value ? 2 : 1;
// of what reaches a result only
template <class T> constexpr int kResultParts = sizeof(T) == 4 ? 3 : 2;
constexpr int kStateParts = 3;

#ifdef __HIP_DEVICE_COMPILE__
__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
// Lane 4 r + x of 16 names four values of row r; lane i gets column i of the four rows.
__device__ inline bf16x4 read_transposed(const char *p) {
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p)));
}
#endif
// The upper 8 bits of v's significand.
__device__ inline float upper(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
// v as N parts, the last one rounded, into place `at` of vectors.
template <int N, class V> __device__ inline void split(float v, V (&to)[N], int at) {
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        const float up = upper(v);
        to[i][at] = bf16(up);
        v -= up;
    }
    to[N - 1][at] = bf16(v);
}
#ifdef __HIP_DEVICE_COMPILE__
// c + x y of parts whose places add up to ORDER at most, small ones first.
template <int ORDER, int NX, int NY> __device__ inline f32x4 multiply(const bf16x8 (&x)[NX], const bf16x8 (&y)[NY], f32x4 c) {
#pragma unroll
    for (int o = ORDER; o >= 0; --o)
#pragma unroll
        for (int i = 0; i < NX; ++i)
            if (o - i >= 0 && o - i < NY) c = mfma(x[i], y[o - i], c);
    return c;
}
#endif

// Eight values of a row, as they are.
template <class T> struct Eight {
    vec<T> v[8 / kVec<T>];
};
template <class T> __device__ inline float value(const Eight<T> &e, int i) { return float(e.v[i / kVec<T>][i % kVec<T>]); }
template <class T, int N> __device__ inline void parts_of(const Eight<T> &e, bf16x8 (&to)[N]) {
    if constexpr (std::is_same<T, bf16>::value && N == 1) {
        to[0] = __builtin_bit_cast(bf16x8, e.v[0]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) split(value(e, i), to, i);
    }
}
// Where a lane's value lies: bytes behind an address that is the same for the wave.
#ifdef __HIP_DEVICE_COMPILE__
#define GLOBAL __attribute__((address_space(1)))
#else
#define GLOBAL
#endif
template <class V> __device__ inline V get(const void *base, uint32_t off) {
    return *(const GLOBAL V *)((const GLOBAL char *)base + off);
}
template <class V> __device__ inline void set(void *base, uint32_t off, V v) { *(GLOBAL V *)((GLOBAL char *)base + off) = v; }
#undef GLOBAL
// v, known from here on only: an offset that the compiler takes out of a loop it no longer sees to be 32 bits wide, and adds it to
// the address in vector registers, once for every access.
__device__ inline uint32_t here(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}
template <class T> __device__ inline void get_eight(Eight<T> &e, const void *base, uint32_t off) {
#pragma unroll
    for (int i = 0; i < 8 / kVec<T>; ++i) e.v[i] = get<vec<T>>(base, off + i * 16);
}
__device__ inline bool finite(float v) { return fabsf(v) <= 3.402823466e38f; }

// Sequences cut into pieces of `len` tokens (packed ones: a power of two).  Those of equal length have equally many;
// packed ones have ids from offsets[s] / len + s on, which leaves room for all of theirs: the spare ids have no tokens.
struct Piece {
    int64_t seq, first, tokens;     // sequence, its first token, its length
    int64_t begin, len;             // the piece's place in the sequence
    int64_t index, count;           // of the sequence's pieces; count 0: a spare id
};
__device__ inline int64_t token_at(const DeltaArgs &a, int64_t s) { return min(max(a.offsets[s], int64_t(0)), a.n_tokens); }
__device__ inline int shift_of(int64_t len) { return 63 - __builtin_clzll(len); }
// The id of a sequence's first piece.
__device__ inline int64_t first_piece(const DeltaArgs &a, int64_t seq, int64_t len) {
    if (a.offsets) return (token_at(a, seq) >> shift_of(len)) + seq;
    return seq * ((a.n_tokens / a.n_seq + len - 1) / len);
}
// 64 lanes of a wave look for it together.  whole: pieces are sequences.
__device__ inline Piece find_piece(const DeltaArgs &a, uint32_t id, int64_t len, bool whole = false) {
    Piece g;
    if (!a.offsets) {
        g.tokens = uint32_t(a.n_tokens) / uint32_t(a.n_seq);
        const uint32_t per = whole ? 1 : uint32_t((g.tokens + len - 1) / len);
        g.seq = id / per;
        g.index = id % per;
        g.first = g.seq * g.tokens;
        g.count = per;
    } else {
        const int shift = shift_of(len);
        uint32_t lo = id, base = id;
        if (!whole) {
            // the last sequence whose ids begin at or before id
            uint32_t hi = uint32_t(a.n_seq);
            lo = base = 0;
            while (hi - lo > 1) {
                const uint32_t step = (hi - lo + 63) / 64, s = lo + (threadIdx.x % 64) * step;
                const uint32_t mine = s < hi ? uint32_t(token_at(a, s) >> shift) + s : 0xffffffffu;
                const int n = max(__popcll(__ballot(mine <= id)), 1);
                base = __shfl(mine, n - 1);
                lo += (n - 1) * step;
                hi = min(lo + step, hi);
            }
            if (a.n_seq == 1) base = uint32_t(token_at(a, 0) >> shift);
            lo = __builtin_amdgcn_readfirstlane(lo);
            base = __builtin_amdgcn_readfirstlane(base);
        }
        g.seq = lo;
        g.index = int64_t(id) - base;
        g.first = token_at(a, lo);
        g.tokens = max(token_at(a, int64_t(lo) + 1) - g.first, int64_t(0));
        g.count = whole ? 1 : (g.tokens + len - 1) >> shift;
    }
    // the same for the wave, and below 2^31: in scalar registers
    const auto same = [](int64_t v) { return int64_t(__builtin_amdgcn_readfirstlane(int(v))); };
    g.seq = same(g.seq);
    g.first = same(g.first);
    g.tokens = same(g.tokens);
    g.index = same(g.index);
    g.count = same(g.count);
    g.begin = whole ? 0 : g.index * len;
    g.len = whole ? g.tokens : min(len, g.tokens - g.begin);
    if (g.index < 0 || g.index >= g.count) g.count = 0;
    return g;
}
inline int64_t piece_ids(const DeltaArgs &a, int64_t len) {
    if (a.offsets) return a.n_tokens / len + a.n_seq;
    return a.n_seq ? a.n_seq * ceil_div(a.n_tokens / a.n_seq, len) : 0;
}

// Token t of a sequence, head h.
template <class T> __device__ inline const T *at_token(const Heads &x, const DeltaArgs &a, const Piece &g, int64_t t, int64_t h) {
    const int64_t row = a.offsets ? (g.first + t) * x.tok : g.seq * x.seq + t * x.tok;
    return static_cast<const T *>(x.p) + row + int64_t(uint32_t(h) / uint32_t(x.group)) * x.head;
}

// The record of a chunk and head: 32 values each of b, exp G and exp(G_last - G), exp(G_last), and the first token whose k,
// g or beta is not finite (32: none); then 32 x 32 matrices as operands of the matrix instructions: row 16 t + l % 16 of tile
// t in lane l, its columns in the order of the accumulators' rows: 16 (e / 4) + 4 (l / 16) + e % 4, e = 0..7.  What a product
// leaves in a wave's accumulators is so the next one's operand as it stands.
constexpr int kRecordHead = 512, kTile = 1024;
struct RecordHead {
    float beta[32], rise[32], fall[32], whole;
    int bad;
};
static_assert(sizeof(RecordHead) <= kRecordHead, "");
constexpr int kRecordMatrix = 2 * kStateParts * kTile;
// forward: (I + A)^-1 and P; gradient: (I + A)^-1, (I + diag(b) A')^-T and P^T
template <class T> constexpr int kRecord = kRecordHead + kRecordMatrix + 2 * kResultParts<T> * kTile;
constexpr int kRecordGrad = kRecordHead + 3 * kRecordMatrix;

// A log decay as it is used: what lies below -128 is a factor of 0 in float in any case, and its sums stay exact.
template <class T> __device__ inline double log_decay(T g) {
    const float v = float(g);
    return v < -128.0f ? -128.0 : double(v);
}

// (16384 tokens x 16 heads of 128 bf16: 54 us, 134 MB read and 85 written; with the gradient's matrices 71, 151 written.)
// One wave: the record of chunk `id` and head h.  Its own LDS: 2 x 32 x 36 floats, 32 doubles and 32 floats.
constexpr int kPrepareLds = 2 * 32 * 36 * 4 + 384;
template <class T, bool GRAD> __global__ void __launch_bounds__(256) delta_prepare(DeltaArgs a, int64_t pairs) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int PARTS = kInputParts<T>, HELD = kResultParts<T>, LD = 36;
    __shared__ __align__(16) char shared[4][kPrepareLds];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int64_t pair = int64_t(blockIdx.x) * 4 + wave;
    if (pair >= pairs) return;
    float(*const m)[LD] = reinterpret_cast<float(*)[LD]>(shared[wave]), (*const p)[LD] = m + 32;
    double *const sum = reinterpret_cast<double *>(shared[wave] + 2 * 32 * LD * 4);
    float *const betas = reinterpret_cast<float *>(sum + 32);
    const int64_t h = pair % a.heads;
    const Piece g = find_piece(a, uint32_t(pair / a.heads), kDeltaChunk);
    if (g.count == 0) return;
    char *const record = a.chunks + pair * a.record;
    const int len = int(g.len);

    // k k^T and q k^T, the tiles (0, 0), (1, 0) and (1, 1)
    f32x4 kk[3], qk[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) kk[i] = qk[i] = 0;
    bool odd[2] = {false, false};
    const T *kp = at_token<T>(a.k, a, g, g.begin, h), *qp = at_token<T>(a.q, a, g, g.begin, h);
    const int most = int(a.dkp);
    uint32_t k_at[2], q_at[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t row = min(16 * t + lm, len - 1);
        k_at[t] = (row * uint32_t(a.k.tok) + 8 * lg) * sizeof(T);
        q_at[t] = (row * uint32_t(a.q.tok) + 8 * lg) * sizeof(T);
    }
    // (rows and widths that are not there are read at others' places, and are 0 when they are used)
    Eight<T> e[2], f[2];
    const auto fetch = [&](int c) __attribute__((always_inline)) {
        const uint32_t off = c + 8 * lg < most ? c * sizeof(T) : 0, back = 8 * lg < most ? 0 : 8 * lg * sizeof(T);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            get_eight(e[t], kp, k_at[t] + off - back);
            get_eight(f[t], qp, q_at[t] + off - back);
        }
    };
    fetch(0);
    for (int c = 0; c < most; c += 32) {
        bf16x8 k[2][PARTS], q[2][PARTS];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const bool in = 16 * t + lm < len && c + 8 * lg < most;
#pragma unroll
            for (int i = 0; i < 8; ++i) odd[t] |= in && !finite(value(e[t], i));
            parts_of(e[t], k[t]);
            parts_of(f[t], q[t]);
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                if (!in) k[t][i] = q[t][i] = bf16x8(bf16(0.0f));
            }
        }
        if (c + 32 < most) fetch(c + 32);
        kk[0] = multiply<2>(k[0], k[0], kk[0]);
        kk[1] = multiply<2>(k[1], k[0], kk[1]);
        kk[2] = multiply<2>(k[1], k[1], kk[2]);
        qk[0] = multiply<2>(q[0], k[0], qk[0]);
        qk[1] = multiply<2>(q[1], k[0], qk[1]);
        qk[2] = multiply<2>(q[1], k[1], qk[2]);
    }
    // gates: lane i % 32 has token i
    const int token = l % 32;
    float beta = 0.0f;
    double log_a = 0.0;
    if (token < len) {
        beta = float(*at_token<T>(a.beta, a, g, g.begin + token, h));
        log_a = log_decay(*at_token<T>(a.g, a, g, g.begin + token, h));
    }
    const auto rows = [](uint64_t b) { return uint32_t((b | b >> 16 | b >> 32 | b >> 48) & 0xffff); };
    const uint32_t unfit = rows(__ballot(odd[0])) | rows(__ballot(odd[1])) << 16 | uint32_t(__ballot(!finite(beta) || !(log_a <= 3.5e38)));
    const int bad = unfit ? __builtin_ctz(unfit) : 32, fit = min(bad, len);
    if (token >= fit) beta = 0.0f, log_a = 0.0;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const double before = __shfl_up(log_a, s, 32);
        if (token >= s) log_a += before;
    }
    const double last = __shfl(log_a, 31, 32);
    RecordHead *const head = reinterpret_cast<RecordHead *>(record);
    if (l < 32) {
        sum[l] = log_a;
        betas[l] = beta;
        head->beta[l] = beta;
        head->rise[l] = expf(float(log_a));
        head->fall[l] = expf(float(last - log_a));
        if (l == 0) {
            head->whole = expf(float(last));
            head->bad = bad;
        }
    }
    // A' and P
#pragma unroll
    for (int t = 0; t < 4; ++t) {       // tiles (0, 0), (0, 1), (1, 0), (1, 1)
        const int ti = t / 2, tj = t % 2, j = 16 * tj + lm;
        const double gj = sum[j];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * ti + 4 * lg + r;
            float ma = 0.0f, pa = 0.0f;
            if (t != 1) {
                const int at = t == 0 ? 0 : t - 1;
                const float decay = expf(float(sum[i] - gj));
                if (j < i && i < fit) ma = decay * kk[at][r];
                if (j <= i && i < fit) pa = decay * qk[at][r];
            }
            m[i][j] = ma;
            p[i][j] = pa;
        }
    }
    // B: its diagonal blocks by substitution, a column a lane; then the block below them, (I - B22 b2) A'21 (I - b1 B11).
    // Rows of the blocks are read before any is written over.
    {
        const int b = token / 16 * 16, c = token % 16;
        float x[16], bx[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = i > c ? m[b + i][b + c] : 0.0f;
#pragma unroll
            for (int j = 0; j < i; ++j) s -= m[b + i][b + j] * bx[j];
            x[i] = s;
            bx[i] = betas[b + i] * s;
        }
        float below[4];         // A' below the blocks, as an operand
#pragma unroll
        for (int r = 0; r < 4; ++r) below[r] = m[16 + lm][4 * r + lg];
#pragma unroll
        for (int i = 0; i < 16; ++i) m[b + i][b + c] = x[i];
        f32x4 y = 0, z = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int k = 4 * r + lg;
            y = mfma(below[r], (k == lm ? 1.0f : 0.0f) - betas[k] * m[k][lm], y);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {       // rows 4 (l / 16) + r of y are in lane l
            const int k = 4 * lg + r;
            z = mfma((k == lm ? 1.0f : 0.0f) - m[16 + lm][16 + k] * betas[16 + k], y[r], z);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) m[16 + 4 * lg + r][lm] = z[r];
    }
    char *to = record + kRecordHead + l * 16;
    const auto store = [&](auto parts, auto f) __attribute__((always_inline)) {
        constexpr int N = decltype(parts)::value;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 v[N];
#pragma unroll
            for (int e = 0; e < 8; ++e) split(f(16 * t + lm, 16 * (e / 4) + 4 * lg + e % 4), v, e);
#pragma unroll
            for (int q = 0; q < N; ++q) *reinterpret_cast<bf16x8 *>(to + (t * N + q) * kTile) = v[q];
        }
        to += 2 * N * kTile;
    };
    const std::integral_constant<int, kStateParts> of_state;
    const std::integral_constant<int, HELD> of_result;
    store(of_state, [&](int i, int j) { return (i == j ? 1.0f : 0.0f) - m[i][j] * betas[j]; });
    if constexpr (GRAD) {
        store(of_state, [&](int i, int j) { return (i == j ? 1.0f : 0.0f) - betas[j] * m[j][i]; });
        store(of_state, [&](int i, int j) { return p[j][i]; });
    } else {
        store(of_result, [&](int i, int j) { return p[i][j]; });
    }
#endif
}

// ---- rows of q and k in LDS, in granules of 16 bytes: granule i of row r of G lies at i ^ turned<G>(r), so that the rows
// one instruction reads, along them or (transposed) four of them across, are in different banks
template <int G> __device__ inline int turned(int r) {
    return G >= 16 ? r % 4 * 4 + r / 4 % 4 : G == 8 ? r / 2 % 2 * 4 + r / 4 % 4 : r / 4 % 4;
}

// Rows of heads with zeros behind them, up to `pad` values: what follows reads eight values of a row at a time, and q, k and
// do of widths that are no multiple of eight go through here first.
template <class T> __global__ void __launch_bounds__(256) delta_pad(DeltaArgs a, Heads from, T *to, int64_t heads, int64_t width, int64_t pad) {
    const int64_t per = a.n_tokens / a.n_seq, n = a.n_tokens * heads * pad;
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < n; at += int64_t(gridDim.x) * 256) {
        const int64_t c = at % pad, h = at / pad % heads, t = at / pad / heads;
        const int64_t row = a.offsets ? t * from.tok : t / per * from.seq + t % per * from.tok;
        to[at] = c < width ? static_cast<const T *>(from.p)[row + h * from.head + c] : T(0.0f);
    }
}
inline int64_t padded(int64_t width) { return (width + 7) / 8 * 8; }
// `from` or, where its width is no multiple of eight, its copy.
template <class T> void pad_rows(const DeltaArgs &a, Heads &from, void *copy, int64_t width, hipStream_t stream) {
    if (width % 8 == 0 || a.n_tokens == 0) return;
    const int64_t heads = a.heads / from.group, pad = padded(width);
    delta_pad<T><<<dim3(uint32_t(std::min(ceil_div(a.n_tokens * heads * pad, 256), int64_t(16384)))), 256, 0, stream>>>(a, from, static_cast<T *>(copy), heads, width, pad);
    from.p = copy;
    from.head = pad;
    from.tok = heads * pad;
    from.seq = a.n_tokens / a.n_seq * from.tok;
}

template <class F> void with_width(int64_t dk, F f) {
    using std::integral_constant;
    if (dk <= 32) f(integral_constant<int, 32>());
    else if (dk <= 64) f(integral_constant<int, 64>());
    else if (dk <= 128) f(integral_constant<int, 128>());
    else f(integral_constant<int, 256>());
}

}  // namespace
}  // namespace ops
}  // namespace ndvm
