// Walks of the gated delta rule over the chunks of a piece of a sequence, forwards and backwards.  (Formulas: delta_parts.h.)
// A wave has 16 columns of v and all widths of k of the state in its accumulators, and needs nothing of another wave: what a
// product leaves is the next one's operand as it stands (K S -> X -> M -> U -> S).  The four waves of a workgroup share the
// rows of k and q, which lie in LDS, one chunk ahead: one barrier a chunk.
#pragma once
#include "delta_parts.h"

namespace ndvm {
namespace ops {
namespace {

// What a walk leaves: outputs and the final state; what the gradient needs (the state before each block of 64 tokens, and m);
// or what a segment adds to a state of 0, and what it makes of other states.
enum Walk { kOutputs, kKept, kSums };

// Bytes of a chunk's rows of k (or q) in LDS, and how many chunks are there at once.
template <class T, int DK> constexpr int kRows = kInputParts<T> * 32 * DK * 2;
template <class T, int DK> constexpr int kBuffers = 4 * kRows<T, DK> <= 131072 ? 2 : 1;
template <class T, int DK, bool BOTH> constexpr int kWalkLds = kBuffers<T, DK> * kRows<T, DK> * (BOTH ? 2 : 1);

// The workgroup's way of the rows of a chunk into LDS.
template <class T, int DK> struct Stage {
    static constexpr int G = DK / 8, PARTS = kInputParts<T>, PART = 32 * G * 16, LOADS = 32 * G > 256 ? 32 * G / 256 : 1;
    Eight<T> held[LOADS];
    __device__ inline void fetch(const T *rows, int64_t step, int left, int64_t dk) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / G, gr = at % G;
            held[i] = load_eight(rows + row * step + gr * 8, row < left ? dk - gr * 8 : 0);
        }
    }
    __device__ inline void put(char *to) const {
        if (32 * G < 256 && int(threadIdx.x) >= 32 * G) return;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / G, gr = at % G;
            bf16x8 p[PARTS];
            parts_of(held[i], p);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8 *>(to + q * PART + (row * G + (gr ^ turned<G>(row))) * 16) = p[q];
        }
    }
};

#ifdef __HIP_DEVICE_COMPILE__
// Operands of a chunk's rows: 16 rows, widths 32 ks on;
template <class T, int DK> __device__ inline void rows_operand(const char *rows, int tile, int ks, bf16x8 (&x)[kInputParts<T>]) {
    constexpr int G = DK / 8;
    const int l = threadIdx.x % 64, row = 16 * tile + l % 16, at = (row * G + ((ks * 4 + l / 16) ^ turned<G>(row))) * 16;
#pragma unroll
    for (int q = 0; q < kInputParts<T>; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(rows + q * 32 * G * 16 + at);
}
// and transposed: widths 32 ks + 8 (m / 4) + 4 t + m % 4, the 32 tokens in the order of the accumulators' rows.
template <class T, int DK> __device__ inline void widths_operand(const char *rows, int ks, int t, bf16x8 (&x)[kInputParts<T>]) {
    constexpr int G = DK / 8;
    const int l = threadIdx.x % 64, row = 4 * (l / 16) + l % 16 / 4, gr = ks * 4 + l % 4;
#pragma unroll
    for (int q = 0; q < kInputParts<T>; ++q) {
        const char *from = rows + q * 32 * G * 16 + 8 * t;
        const bf16x4 lo = read_transposed(from + (row * G + (gr ^ turned<G>(row))) * 16);
        const bf16x4 hi = read_transposed(from + ((row + 16) * G + (gr ^ turned<G>(row + 16))) * 16);
        x[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}
#endif

// A wave's columns of a state: widths 32 ks + 8 (l / 16) + 4 t + r of column col, [dk][cols] in memory.
template <int DK> struct State {
    static constexpr int KS = DK / 32;
    f32x4 s[KS][2];
    template <class F> __device__ inline void each(F f) {
        const int lg = threadIdx.x % 64 / 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) f(s[ks][t], r, ks * 32 + 8 * lg + 4 * t + r);
    }
    __device__ inline void fill(float v) {
        each([&](f32x4 &x, int r, int) { x[r] = v; });
    }
    __device__ inline void load(const float *from, int64_t dk, int64_t cols, int64_t col) {
        each([&](f32x4 &x, int r, int d) { x[r] = d < dk && col < cols ? from[d * cols + col] : 0.0f; });
    }
    __device__ inline void store(float *to, int64_t dk, int64_t cols, int64_t col) {
        each([&](f32x4 &x, int r, int d) {
            if (d < dk && col < cols) to[d * cols + col] = x[r];
        });
    }
#ifdef __HIP_DEVICE_COMPILE__
    __device__ inline void operand(int ks, bf16x8 (&x)[kStateParts]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) split(s[ks][e / 4][e % 4], x, e);
    }
#endif
};

// Forwards.  tile: the wave's columns; from ceil(dv / 16) on (kSums) those of what the piece makes of a state.
// (Inlined by force: called, its arrays would live in memory.)
template <class T, int DK, Walk WALK> __device__ __forceinline__ void walk(const DeltaArgs &a, char *lds, const Piece &g, int64_t slot, int64_t h, int64_t tile) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int PARTS = kInputParts<T>, HELD = kResultParts<T>, SP = kStateParts, KS = DK / 32, BUFFERS = kBuffers<T, DK>;
    constexpr bool OUT = WALK == kOutputs;
    constexpr int MATRIX = kRows<T, DK>;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int64_t tiles = ceil_div(a.dv, 16);
    const bool moves = WALK == kSums && tile >= tiles;
    const int64_t cols = moves ? a.dk : a.dv, col = (moves ? tile - tiles : tile) * 16 + lm;
    const bool works = col - lm < cols;
    const auto token_of = [&](int e) { return 16 * (e / 4) + 4 * lg + e % 4; };
    const int64_t chunk0 = first_piece(a, g.seq, kDeltaChunk) + g.begin / kDeltaChunk;
    const int chunks = int((g.len + 31) / 32);
    const int64_t states = a.dk * a.dv;
    const auto left_of = [&](int c) { return int(min(g.len - int64_t(c) * 32, int64_t(32))); };

    State<DK> S;
    if (WALK == kSums) S.each([&](f32x4 &x, int r, int d) { x[r] = moves && d == col ? 1.0f : 0.0f; });
    else if (a.segments) S.load(a.segments + slot * states, a.dk, a.dv, col);
    else if (a.state_in) S.load(a.state_in + (g.seq * a.heads + h) * states, a.dk, a.dv, col);
    else S.fill(0.0f);

    const T *kp = at_token<T>(a.k, a, g, g.begin, h), *qp = OUT ? at_token<T>(a.q, a, g, g.begin, h) : nullptr;
    const T *vp = at_token<T>(a.v, a, g, g.begin, h) + col;
    T *op = OUT ? const_cast<T *>(at_token<T>(a.o, a, g, g.begin, h)) + col : nullptr;
    float *mp = WALK == kKept ? a.m + (h * a.n_tokens + g.first + g.begin) * a.dv + col : nullptr;
    Stage<T, DK> rk, rq;
    struct Small {
        bf16x8 t[2][SP], p[OUT ? 2 : 1][OUT ? HELD : 1];
        f32x4 beta[2], rise[2], fall[2];
        float whole;
        int bad;
        T v[8];
    };
    const auto fetch_small = [&](int c, Small &s) __attribute__((always_inline)) {
        const char *record = a.chunks + ((chunk0 + c) * a.heads + h) * a.record;
        const RecordHead *head = reinterpret_cast<const RecordHead *>(record);
        const char *t = record + kRecordHead + l * 16, *p = t + kRecordMatrix;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int q = 0; q < SP; ++q) s.t[i][q] = *reinterpret_cast<const bf16x8 *>(t + (i * SP + q) * kTile);
            if constexpr (OUT)
#pragma unroll
                for (int q = 0; q < HELD; ++q) s.p[i][q] = *reinterpret_cast<const bf16x8 *>(p + (i * HELD + q) * kTile);
            const int row = 16 * i + 4 * lg;
            s.beta[i] = *reinterpret_cast<const f32x4 *>(head->beta + row);
            s.rise[i] = *reinterpret_cast<const f32x4 *>(head->rise + row);
            s.fall[i] = *reinterpret_cast<const f32x4 *>(head->fall + row);
        }
        s.whole = head->whole;
        s.bad = head->bad;
        const int left = left_of(c);
        const bool there = !moves && col < cols;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s.v[e] = T(0.0f);
            if (there && token_of(e) < left) s.v[e] = vp[(int64_t(c) * 32 + token_of(e)) * a.v.tok];
        }
    };
    const auto fetch_rows = [&](int c) __attribute__((always_inline)) {
        rk.fetch(kp + int64_t(c) * 32 * a.k.tok, a.k.tok, left_of(c), a.dk);
        if constexpr (OUT) rq.fetch(qp + int64_t(c) * 32 * a.q.tok, a.q.tok, left_of(c), a.dk);
    };
    const auto put_rows = [&](int c) __attribute__((always_inline)) {
        char *to = lds + c % BUFFERS * MATRIX * (OUT ? 2 : 1);
        rk.put(to);
        if constexpr (OUT) rq.put(to + MATRIX);
    };

    Small cur;
    if (chunks) {
        fetch_rows(0);
        fetch_small(0, cur);
        put_rows(0);
    }
    __syncthreads();
    for (int c = 0; c < chunks; ++c) {
        const char *k = lds + c % BUFFERS * MATRIX * (OUT ? 2 : 1), *q = k + MATRIX;
        const int left = left_of(c);
        Small next;
        if (c + 1 < chunks) {
            fetch_rows(c + 1);
            fetch_small(c + 1, next);
        }
        if (works) {
            if (WALK == kKept && c % 2 == 0) {
                const int64_t block = first_piece(a, g.seq, kDeltaBlock) + (g.begin + int64_t(c) * 32) / kDeltaBlock;
                S.store(a.states + (block * a.heads + h) * states, a.dk, a.dv, col);
            }
            // Y = K S, Z = Q S
            f32x4 y[2], z[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) y[i] = z[i] = 0;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                bf16x8 s[SP], x[PARTS];
                S.operand(ks, s);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    rows_operand<T, DK>(k, i, ks, x);
                    y[i] = multiply<SP - 1>(x, s, y[i]);
                    if constexpr (OUT) {
                        rows_operand<T, DK>(q, i, ks, x);
                        z[i] = multiply<HELD - 1>(x, s, z[i]);
                    }
                }
            }
            // a value of v that is not finite counts as 0; what follows it in its column is set below
            int first = cur.bad;
            float v[8];
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = float(cur.v[e]);
                odd |= !finite(v[e]);
            }
            if (__ballot(odd)) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!finite(v[e])) {
                        v[e] = 0.0f;
                        first = min(first, token_of(e));
                    }
                first = min(first, __shfl_xor(first, 16));
                first = min(first, __shfl_xor(first, 32));
            }
            // X, M and U
            bf16x8 x[SP], w[SP], u[HELD];
#pragma unroll
            for (int e = 0; e < 8; ++e) split(token_of(e) < cur.bad ? v[e] - cur.rise[e / 4][e % 4] * y[e / 4][e % 4] : 0.0f, x, e);
            f32x4 m[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) m[i] = multiply<SP - 1>(cur.t[i], x, f32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float ue = cur.beta[e / 4][e % 4] * m[e / 4][e % 4];
                split(ue * cur.fall[e / 4][e % 4], w, e);
                if constexpr (OUT) split(ue, u, e);
                if (WALK == kKept && token_of(e) < left && col < cols)
                    mp[(int64_t(c) * 32 + token_of(e)) * a.dv] = token_of(e) < first ? m[e / 4][e % 4] : __builtin_nanf("");
            }
            // S' = exp(G_last) S + K^T (fall U)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    bf16x8 kt[PARTS];
                    widths_operand<T, DK>(k, ks, t, kt);
                    S.s[ks][t] = multiply<SP - 1>(kt, w, S.s[ks][t] * cur.whole);
                }
            if constexpr (OUT) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const f32x4 o = multiply<HELD - 1>(cur.p[i], u, cur.rise[i] * z[i]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int token = token_of(4 * i + r);
                        if (token < left && col < cols)
                            op[(int64_t(c) * 32 + token) * a.o.tok] = T(token < first ? o[r] * a.scale : __builtin_nanf(""));
                    }
                }
            }
            // a column with a value that is not finite, or a head with a key or gate that is not, has none from there on
            if (first < left) S.fill(__builtin_nanf(""));
        }
        if (BUFFERS == 1) __syncthreads();
        if (c + 1 < chunks) put_rows(c + 1);
        __syncthreads();
        cur = next;
    }
    if (!works) return;
    if (OUT && a.state_out && g.index == g.count - 1) S.store(a.state_out + (g.seq * a.heads + h) * states, a.dk, a.dv, col);
    if (WALK == kSums && !moves) S.store(a.segments + slot * states, a.dk, a.dv, col);
    if (WALK == kSums && moves) {
        S.store(a.moves + slot * a.dk * a.dk, a.dk, a.dk, col);
        if (a.moves_t)
            S.each([&](f32x4 &x, int r, int d) {
                if (d < a.dk && col < cols) a.moves_t[(slot * a.dk + col) * a.dk + d] = x[r];
            });
    }
#endif
}

// Backwards: the gradient of the state, from the piece's end to its beginning; e and the gradient of v.
template <class T, int DK, Walk WALK> __device__ __forceinline__ void walk_back(const DeltaArgs &a, char *lds, const Piece &g, int64_t slot, int64_t h, int64_t tile) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int PARTS = kInputParts<T>, SP = kStateParts, KS = DK / 32, BUFFERS = kBuffers<T, DK>, MATRIX = kRows<T, DK>;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int64_t col = tile * 16 + lm;
    const bool works = col - lm < a.dv;
    const auto token_of = [&](int e) { return 16 * (e / 4) + 4 * lg + e % 4; };
    const int64_t chunk0 = first_piece(a, g.seq, kDeltaChunk) + g.begin / kDeltaChunk;
    const int chunks = int((g.len + 31) / 32);
    const int64_t states = a.dk * a.dv;
    const auto left_of = [&](int c) { return int(min(g.len - int64_t(c) * 32, int64_t(32))); };

    State<DK> D;
    if (WALK == kSums) D.fill(0.0f);
    else if (a.d_segments) D.load(a.d_segments + slot * states, a.dk, a.dv, col);
    else if (a.d_state_out) D.load(a.d_state_out + (g.seq * a.heads + h) * states, a.dk, a.dv, col);
    else D.fill(0.0f);

    const T *kp = at_token<T>(a.k, a, g, g.begin, h), *qp = at_token<T>(a.q, a, g, g.begin, h);
    const T *dp = at_token<T>(a.d_o, a, g, g.begin, h) + col;
    T *vp = WALK == kKept && a.dv_out.p ? const_cast<T *>(at_token<T>(a.dv_out, a, g, g.begin, h)) + col : nullptr;
    float *ep = WALK == kKept && a.e ? a.e + (h * a.n_tokens + g.first + g.begin) * a.dv + col : nullptr;
    Stage<T, DK> rk, rq;
    struct Small {
        bf16x8 t[2][SP], p[2][SP];
        f32x4 beta[2], rise[2], fall[2];
        float whole;
        int bad;
        T d[8];
    };
    const auto fetch_small = [&](int c, Small &s) __attribute__((always_inline)) {
        const char *record = a.chunks + ((chunk0 + c) * a.heads + h) * a.record;
        const RecordHead *head = reinterpret_cast<const RecordHead *>(record);
        const char *t = record + kRecordHead + kRecordMatrix + l * 16, *p = t + kRecordMatrix;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int q = 0; q < SP; ++q) {
                s.t[i][q] = *reinterpret_cast<const bf16x8 *>(t + (i * SP + q) * kTile);
                s.p[i][q] = *reinterpret_cast<const bf16x8 *>(p + (i * SP + q) * kTile);
            }
            const int row = 16 * i + 4 * lg;
            s.beta[i] = *reinterpret_cast<const f32x4 *>(head->beta + row);
            s.rise[i] = *reinterpret_cast<const f32x4 *>(head->rise + row);
            s.fall[i] = *reinterpret_cast<const f32x4 *>(head->fall + row);
        }
        s.whole = head->whole;
        s.bad = head->bad;
        const int left = left_of(c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s.d[e] = T(0.0f);
            if (col < a.dv && token_of(e) < left) s.d[e] = dp[(int64_t(c) * 32 + token_of(e)) * a.d_o.tok];
        }
    };
    const auto fetch_rows = [&](int c) __attribute__((always_inline)) {
        rk.fetch(kp + int64_t(c) * 32 * a.k.tok, a.k.tok, left_of(c), a.dk);
        rq.fetch(qp + int64_t(c) * 32 * a.q.tok, a.q.tok, left_of(c), a.dk);
    };
    const auto put_rows = [&](int c) __attribute__((always_inline)) {
        char *to = lds + c % BUFFERS * MATRIX * 2;
        rk.put(to);
        rq.put(to + MATRIX);
    };

    Small cur;
    if (chunks) {
        fetch_rows(chunks - 1);
        fetch_small(chunks - 1, cur);
        put_rows(chunks - 1);
    }
    __syncthreads();
    for (int c = chunks - 1; c >= 0; --c) {
        const char *k = lds + c % BUFFERS * MATRIX * 2, *q = k + MATRIX;
        const int left = left_of(c);
        Small next;
        if (c > 0) {
            fetch_rows(c - 1);
            fetch_small(c - 1, next);
        }
        if (works) {
            if (WALK == kKept && a.d_states && (c % 2 == 1 || c == chunks - 1)) {
                const int64_t block = first_piece(a, g.seq, kDeltaBlock) + (g.begin + int64_t(c) * 32) / kDeltaBlock;
                D.store(a.d_states + (block * a.heads + h) * states, a.dk, a.dv, col);
            }
            f32x4 w[2], o[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = o[i] = 0;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                bf16x8 s[SP], x[PARTS];
                D.operand(ks, s);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    rows_operand<T, DK>(k, i, ks, x);
                    w[i] = multiply<SP - 1>(x, s, w[i]);
                }
            }
            bf16x8 od[PARTS], du[SP], x[SP];
#pragma unroll
            for (int e = 0; e < 8; ++e) split(float(cur.d[e]), od, e);
#pragma unroll
            for (int i = 0; i < 2; ++i) o[i] = multiply<SP - 1>(cur.p[i], od, o[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) split(a.scale * o[e / 4][e % 4] + cur.fall[e / 4][e % 4] * w[e / 4][e % 4], du, e);
#pragma unroll
            for (int i = 0; i < 2; ++i) o[i] = multiply<SP - 1>(cur.t[i], du, f32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float ee = o[e / 4][e % 4], xe = cur.beta[e / 4][e % 4] * ee, rise = cur.rise[e / 4][e % 4];
                split(rise * a.scale * float(cur.d[e]), du, e);
                split(-rise * xe, x, e);
                if (WALK == kKept && token_of(e) < left && col < a.dv) {
                    const int64_t token = int64_t(c) * 32 + token_of(e);
                    if (ep) ep[token * a.dv] = ee;
                    if (vp) vp[token * a.dv_out.tok] = T(xe);
                }
            }
            const float whole = cur.bad < left ? __builtin_nanf("") : cur.whole;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    bf16x8 kt[PARTS];
                    f32x4 d = D.s[ks][t] * whole;
                    widths_operand<T, DK>(q, ks, t, kt);
                    d = multiply<SP - 1>(kt, du, d);
                    widths_operand<T, DK>(k, ks, t, kt);
                    D.s[ks][t] = multiply<SP - 1>(kt, x, d);
                }
        }
        if (BUFFERS == 1) __syncthreads();
        if (c > 0) put_rows(c - 1);
        __syncthreads();
        cur = next;
    }
    if (!works) return;
    if (WALK == kKept && a.d_state_in && g.index == 0) D.store(a.d_state_in + (g.seq * a.heads + h) * states, a.dk, a.dv, col);
    if (WALK == kSums) D.store(a.d_segments + slot * states, a.dk, a.dv, col);
#endif
}

// From segment to segment of a sequence: what enters each takes the place of what it adds.  BACK: of the gradient, from the
// back.  Four waves, 16 columns of v each.  A sequence without tokens has its final state (its initial state's gradient) here.
template <int DK, bool BACK> __device__ __forceinline__ void carry(const DeltaArgs &a, int64_t seq, int64_t h, int64_t tile) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int KS = DK / 32, SP = kStateParts;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int64_t col = tile * 16 + lm, states = a.dk * a.dv, own = (seq * a.heads + h) * states;
    if (col - lm >= a.dv) return;
    const int64_t id0 = first_piece(a, seq, a.seg_len);
    const int64_t tokens = a.offsets ? max(token_at(a, seq + 1) - token_at(a, seq), int64_t(0)) : a.n_tokens / a.n_seq;
    const int64_t count = (tokens + a.seg_len - 1) / a.seg_len;
    const float *in = BACK ? a.d_state_out : a.state_in;
    float *const out = BACK ? a.d_state_in : a.state_out, *const adds = BACK ? a.d_segments : a.segments;
    const float *const moves = BACK ? a.moves_t : a.moves;
    State<DK> S;
    if (in) S.load(in + own, a.dk, a.dv, col);
    else S.fill(0.0f);
    if (count == 0 && out) S.store(out + own, a.dk, a.dv, col);
    for (int64_t i = 0; i < count; ++i) {
        const int64_t slot = (id0 + (BACK ? count - 1 - i : i)) * a.heads + h;
        State<DK> next;
        next.load(adds + slot * states, a.dk, a.dv, col);
        S.store(adds + slot * states, a.dk, a.dv, col);
        if (i == count - 1) return;
        const float *m = moves + slot * a.dk * a.dk;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            bf16x8 s[SP];
            S.operand(ks, s);
#pragma unroll
            for (int to = 0; to < 2 * KS; ++to) {
                const int64_t d = to / 2 * 32 + 8 * (lm / 4) + 4 * (to % 2) + lm % 4, from = ks * 32 + 8 * lg;
                bf16x8 x[SP];
                parts_of(load_eight(m + d * a.dk + from, d < a.dk ? a.dk - from : 0), x);
                next.s[to / 2][to % 2] = multiply<SP - 1>(x, s, next.s[to / 2][to % 2]);
            }
        }
        S = next;
    }
#endif
}

// Whether sequences are cut into segments, and how.  A walk takes as long for one wave as for two on each of the 1,024 matrix
// units, and segments cost two to three times the work.
inline bool cut(DeltaArgs &a) {
    constexpr int64_t kWaves = 2048, kShortest = 128;
    const int64_t per_token = a.heads * ceil_div(a.dv, 16);
    a.seg_len = kShortest;
    while (a.seg_len * kWaves < a.n_tokens * per_token) a.seg_len *= 2;
    if (a.n_seq && a.n_seq * per_token * 3 < kWaves && a.n_tokens / a.n_seq >= 3 * a.seg_len) {
        a.n_segments = piece_ids(a, a.seg_len);
        return true;
    }
    a.seg_len = std::max<int64_t>(kDeltaBlock, a.n_tokens);
    a.n_segments = a.n_seq;
    return false;
}

// Where a launch keeps what.
struct Space {
    char *base;
    size_t used = 0;
    explicit Space(void *p) : base(p ? reinterpret_cast<char *>(round256(reinterpret_cast<size_t>(p))) : nullptr) {}
    template <class P> void take(P *&p, int64_t bytes) {
        p = base ? reinterpret_cast<P *>(base + used) : nullptr;
        used += round256(size_t(bytes));
    }
};

}  // namespace
}  // namespace ops
}  // namespace ndvm
