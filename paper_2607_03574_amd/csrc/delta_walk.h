// Walks of the gated delta rule over the chunks of a piece of a sequence, forwards and backwards.  (Formulas: delta_parts.h.)
// A wave has 16 columns of v and all widths of k of the state in its accumulators, and needs nothing of another wave: what a
// product leaves is the next one's operand as it stands (K S -> X -> M -> U -> S).  The four waves of a workgroup share the
// rows of k and q and the chunk's record, which lie in LDS, one chunk ahead: one barrier a chunk.
// Bound by the issue of vector and matrix instructions, two waves on a matrix unit: 630 and 82 of a chunk, half of the former for
// the state's parts (16384 tokens x 16 heads of 128 bf16, 16 segments: outputs 115 us, sums and transitions 157; with the
// widths divided among the waves, whose sums met in LDS, the whole call was 1,976, now 417).
#pragma once
#include "delta_parts.h"

namespace ndvm {
namespace ops {
namespace {

// What a walk leaves: outputs and the final state; what the gradient needs (the state before each block of 64 tokens, and m);
// or what a segment adds to a state of 0, and what it makes of other states.
enum Walk { kOutputs, kKept, kSums };

// Bytes of a chunk's rows of k (or q) in LDS; how many chunks are there at once; and bytes of a record, as far as a walk reads it.
template <class T, int DK> constexpr int kRows = kInputParts<T> * 32 * DK * 2;
template <class T, int DK> constexpr int kBuffers = 4 * kRows<T, DK> <= 131072 ? 2 : 1;
template <class T, Walk WALK> constexpr int kRead = WALK == kOutputs ? kRecord<T> : kRecordHead + kRecordMatrix;
constexpr int kReadBack = kRecordHead + 2 * kRecordMatrix;
template <class T, int DK, bool BOTH, int READ> constexpr int kWalkLds = kBuffers<T, DK> * (kRows<T, DK> * (BOTH ? 2 : 1) + READ);
// workgroups on a compute unit: as many as their LDS leaves room for
template <class T, int DK> constexpr int kResident = kInputParts<T> * DK < 256 ? 2 : 1;

// The workgroup's way of the rows of a chunk into LDS.
template <class T, int DK> struct Stage {
    static constexpr int G = DK / 8, PARTS = kInputParts<T>, PART = 32 * G * 16, LOADS = 32 * G > 256 ? 32 * G / 256 : 1;
    Eight<T> held[LOADS];
    // what is not there is read at the first row's place, and is 0 when it is put
    __device__ inline void fetch(const T *rows, uint32_t step, int left, int dkp) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / G, gr = at % G;
            get_eight(held[i], rows, row < left && gr * 8 < dkp ? (uint32_t(row) * step + gr * 8) * sizeof(T) : 0);
        }
    }
    // (a chunk later: what touched the values before would wait for them)
    __device__ inline void put(char *to, int left, int dkp) const {
        if (32 * G < 256 && int(threadIdx.x) >= 32 * G) return;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / G, gr = at % G;
            bf16x8 p[PARTS];
            parts_of(held[i], p);
            const bool in = row < left && gr * 8 < dkp;
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8 *>(to + q * PART + (row * G + (gr ^ turned<G>(row))) * 16) = in ? p[q] : bf16x8(bf16(0.0f));
        }
    }
};
// And of a record: its first FIRST bytes, and those behind a gap.
template <int READ, int FIRST, int GAP> struct StageRecord {
    static constexpr int LOADS = (READ / 16 + 255) / 256;
    f32x4 held[LOADS];
    __device__ inline void fetch(const char *record) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t at = min(uint32_t(i * 256 + threadIdx.x) * 16, uint32_t(READ - 16));
            held[i] = get<f32x4>(record, at < uint32_t(FIRST) ? at : at + GAP);
        }
    }
    __device__ inline void put(char *to) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (i * 256 + threadIdx.x) * 16;
            if (at < READ) *reinterpret_cast<f32x4 *>(to + at) = held[i];
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

#ifdef __HIP_DEVICE_COMPILE__
// Reads of memory stay on their side; arithmetic need not.
__device__ inline void reads_stay() { __builtin_amdgcn_sched_barrier(0x000f); }
#endif

// A wave's columns of a state: widths 32 ks + 8 (l / 16) + 4 t + r of column col, [dk][cols] in memory.
template <int DK> struct State {
    static constexpr int KS = DK / 32;
    f32x4 s[KS][2];
    // f(values, place, width): the lane's own width is 8 (l / 16) more
    template <class F> __device__ inline void each(F f) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) f(s[ks][t], r, ks * 32 + 4 * t + r);
    }
    __device__ inline void fill(float v) {
        each([&](f32x4 &x, int r, int) { x[r] = v; });
    }
    // col0: the first of the wave's 16 columns; rows are `step` values apart.  (A lane has one offset for all its values: an
    // address for each, which the compiler would keep all the while, is twice as many registers as the state.)
    __device__ inline void load(const float *from, int dk, int cols, int step, int col0) {
        const int lm = threadIdx.x % 16, up = threadIdx.x % 64 / 16 * 8;
        from += col0;
        if (dk == DK && col0 + 16 <= cols) {
            const uint32_t at = here(uint32_t(up * step + lm) * 4);
            each([&](f32x4 &x, int r, int d) {
                x[r] = get<float>(from, at);
                from += d % 8 == 7 ? 25 * step : step;
            });
        } else {
            each([&](f32x4 &x, int r, int d) {
                const bool in = col0 + lm < cols && d + up < dk;
                const float v = get<float>(from, in ? uint32_t((d + up) * step + lm) * 4 : 0);
                x[r] = in ? v : 0.0f;
            });
        }
    }
    // (columns from `cols` to `step` are 0)
    __device__ inline void store(float *to, int dk, int cols, int step, int col0) {
        const int lm = threadIdx.x % 16, up = threadIdx.x % 64 / 16 * 8;
        to += col0;
        if (dk == DK && col0 + 16 <= cols) {
            const uint32_t at = here(uint32_t(up * step + lm) * 4);
            each([&](f32x4 &x, int r, int d) {
                set<float>(to, at, x[r]);
                to += d % 8 == 7 ? 25 * step : step;
            });
        } else if (col0 + lm < step) {
            each([&](f32x4 &x, int r, int d) {
                if (d + up < dk) set<float>(to + d * step, uint32_t(up * step + lm) * 4, col0 + lm < cols ? x[r] : 0.0f);
            });
        }
    }
#ifdef __HIP_DEVICE_COMPILE__
    __device__ inline void operand(int ks, bf16x8 (&x)[kStateParts]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) split(s[ks][e / 4][e % 4], x, e);
    }
#endif
};

// An address that is the same for the wave, in scalar registers.
template <class P> __device__ inline P *same(P *p) {
#ifdef __HIP_DEVICE_COMPILE__
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<P *>(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(v)))) |
                                 uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(v >> 32)))) << 32);
#else
    return p;
#endif
}

// A lane's eight tokens of a column: 16 (e / 4) + e % 4, and 4 (l / 16) more.  Accesses know the piece of memory that the chunk's
// `left` tokens and `cols` columns lie in: what is beyond it is not stored, and loaded as 0 (or, of columns that are not there, as
// any value).
// (Bits in registers of their own: 16-bit values side by side would wait for one another.)
template <class T> struct Bits {
    uint32_t b[8];
    __device__ inline void zero() {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = 0;
    }
#ifdef __HIP_DEVICE_COMPILE__
    __device__ inline void load(const T *p, uint32_t tok, int left, int cols) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(p), 0, ((left - 1) * tok + cols) * sizeof(T), 0x00020000);
        const uint32_t at = (threadIdx.x % 64 / 16 * 4 * tok + threadIdx.x % 16) * sizeof(T);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t off = at + (16 * (e / 4) + e % 4) * tok * uint32_t(sizeof(T));
            if constexpr (sizeof(T) == 4) b[e] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, off, 0, 0);
            else b[e] = __builtin_amdgcn_raw_buffer_load_b16(rsrc, off, 0, 0);
        }
    }
#endif
    __device__ inline float value(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(b[e]);
        else if constexpr (std::is_same<T, bf16>::value) return __uint_as_float(b[e] << 16);
        else return float(__builtin_bit_cast(f16, uint16_t(b[e])));
    }
};
#ifdef __HIP_DEVICE_COMPILE__
template <class T> __device__ inline void store_column(T *p, uint32_t tok, int left, int cols, const f32x4 (&v)[2]) {
    if (left == 1) tok = 256;       // (rows need not be apart where there is one)
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(p, 0, ((left - 1) * tok + cols) * sizeof(T), 0x00020000);
    const uint32_t at = (threadIdx.x % 64 / 16 * 4 * tok + threadIdx.x % 16) * sizeof(T);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t off = at + (16 * (e / 4) + e % 4) * tok * uint32_t(sizeof(T));
        const T x = T(v[e / 4][e % 4]);
        if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), rsrc, off, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, x), rsrc, off, 0, 0);
    }
}
#endif

// Forwards.  tile: the wave's columns; from ceil(dv / 16) on (kSums) those of what the piece makes of a state.
// (Inlined by force: called, its arrays would live in memory.)
template <class T, int DK, Walk WALK> __device__ __forceinline__ void walk(const DeltaArgs &a, char *lds, const Piece &g, int64_t slot, int64_t h, int tile) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int PARTS = kInputParts<T>, HELD = kResultParts<T>, SP = kStateParts, KS = DK / 32, BUFFERS = kBuffers<T, DK>;
    constexpr bool OUT = WALK == kOutputs;
    constexpr int MATRIX = kRows<T, DK>, READ = kRead<T, WALK>, SLOT = MATRIX * (OUT ? 2 : 1) + READ;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int dk = int(a.dk), dv = int(a.dv), dkp = int(a.dkp), dvp = int(a.dvp), tiles = (dv + 15) / 16;
    const float scale = a.scale;
    const bool moves = WALK == kSums && tile >= tiles;
    const int cols = moves ? dk : dv, col0 = (moves ? tile - tiles : tile) * 16, col = col0 + lm;
    const bool works = col0 < cols;
    const auto token_of = [&](int e) { return 16 * (e / 4) + 4 * lg + e % 4; };
    const int64_t chunk0 = first_piece(a, g.seq, kDeltaChunk) + g.begin / kDeltaChunk;
    const int chunks = int((g.len + 31) / 32);
    const int64_t states = a.dk * a.dv;
    const auto left_of = [&](int c) { return int(min(g.len - int64_t(c) * 32, int64_t(32))); };

    State<DK> S;
    if (WALK == kSums) S.each([&](f32x4 &x, int r, int d) { x[r] = moves && d + 8 * lg == col ? 1.0f : 0.0f; });
    else if (!works) S.fill(0.0f);
    else if (a.segments) S.load(a.segments + slot * states, dk, dv, dv, col0);
    else if (a.state_in) S.load(a.state_in + (g.seq * a.heads + h) * states, dk, dv, dv, col0);
    else S.fill(0.0f);

    const T *const kp = same(at_token<T>(a.k, a, g, g.begin, h)), *const qp = same(at_token<T>(a.q, a, g, g.begin, h));
    const T *const vp = same(at_token<T>(a.v, a, g, g.begin, h) + (moves ? 0 : col0));
    T *const op = OUT ? same(const_cast<T *>(at_token<T>(a.o, a, g, g.begin, h)) + col0) : nullptr;
    float *const mp = WALK == kKept ? same(a.m + (h * a.n_tokens + g.first + g.begin) * a.dvp + col0) : nullptr;
    Stage<T, DK> rk, rq;
    StageRecord<READ, READ, 0> record;
    Bits<T> v_next, v_now;
    const auto fetch = [&](int c) __attribute__((always_inline)) {
        const int left = left_of(c);
        record.fetch(a.chunks + ((chunk0 + c) * a.heads + h) * a.record);
        rk.fetch(kp + int64_t(c) * 32 * a.k.tok, uint32_t(a.k.tok), left, dkp);
        if constexpr (OUT) rq.fetch(qp + int64_t(c) * 32 * a.q.tok, uint32_t(a.q.tok), left, dkp);
        const T *v = vp + int64_t(c) * 32 * a.v.tok;
        if (moves || !works) v_next.zero();
        else v_next.load(v, uint32_t(a.v.tok), left, min(16, cols - col0));
    };
    const auto put = [&](int c) __attribute__((always_inline)) {
        char *to = lds + c % BUFFERS * SLOT;
        rk.put(to, left_of(c), dkp);
        if constexpr (OUT) rq.put(to + MATRIX, left_of(c), dkp);
        record.put(to + SLOT - READ);
    };

    // the state before a block
    float *const kept = WALK == kKept ? same(a.states + ((first_piece(a, g.seq, kDeltaBlock) + g.begin / kDeltaBlock) * a.heads + h) * dk * dvp) : nullptr;
    const auto keep = [&](int c) __attribute__((always_inline)) { S.store(kept + int64_t(c / 2) * a.heads * dk * dvp, dk, dv, dvp, col0); };
    if (chunks) {
        fetch(0);
        put(0);
        v_now = v_next;
    }
    if (WALK == kKept && works && chunks) keep(0);
    __syncthreads();
    for (int c = 0; c < chunks; ++c) {
        const char *k = lds + c % BUFFERS * SLOT, *q = k + MATRIX, *matrices = k + SLOT - READ + kRecordHead + l * 16;
        const RecordHead *head = reinterpret_cast<const RecordHead *>(k + SLOT - READ);
        const int left = left_of(c);
        if (c + 1 < chunks) fetch(c + 1);
        f32x4 o[2];
        int first = 32;
        if (works) {
            // Y = K S, Z = Q S; LDS is read one step ahead of what needs it
            f32x4 y[2], z[2], beta[2], rise[2], fall[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) y[i] = z[i] = 0;
            bf16x8 kx[2][2][PARTS], qx[2][2][PARTS], tx[2][SP];
            const auto read_rows = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    rows_operand<T, DK>(k, i, ks, kx[ks % 2][i]);
                    if constexpr (OUT) rows_operand<T, DK>(q, i, ks, qx[ks % 2][i]);
                }
            };
            read_rows(0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 1 < KS) {
                    read_rows(ks + 1);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int p = 0; p < SP; ++p) tx[i][p] = *reinterpret_cast<const bf16x8 *>(matrices + (i * SP + p) * kTile);
                }
                reads_stay();
                bf16x8 s[SP];
                S.operand(ks, s);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    y[i] = multiply<SP - 1>(kx[ks % 2][i], s, y[i]);
                    if constexpr (OUT) z[i] = multiply<HELD - 1>(qx[ks % 2][i], s, z[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                beta[i] = *reinterpret_cast<const f32x4 *>(head->beta + 16 * i + 4 * lg);
                rise[i] = *reinterpret_cast<const f32x4 *>(head->rise + 16 * i + 4 * lg);
                fall[i] = *reinterpret_cast<const f32x4 *>(head->fall + 16 * i + 4 * lg);
            }
            const float whole = head->whole;
            const int bad = head->bad, fit = min(bad, left);
            // a value of v that is not finite counts as 0; what follows it in its column is set below
            first = bad;
            float v[8];
            bool odd = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = v_now.value(e);
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
            for (int e = 0; e < 8; ++e) split(token_of(e) < fit ? v[e] - rise[e / 4][e % 4] * y[e / 4][e % 4] : 0.0f, x, e);
            bf16x8 kt[2][2][PARTS], px[OUT ? 2 : 1][OUT ? HELD : 1];
            const auto read_widths = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < 2; ++t) widths_operand<T, DK>(k, ks, t, kt[ks % 2][t]);
            };
            read_widths(0);
            reads_stay();
            f32x4 m[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) m[i] = multiply<SP - 1>(tx[i], x, f32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float ue = beta[e / 4][e % 4] * m[e / 4][e % 4];
                split(ue * fall[e / 4][e % 4], w, e);
                if constexpr (OUT) split(ue, u, e);
            }
            // S' = exp(G_last) S + K^T (fall U)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 1 < KS) {
                    read_widths(ks + 1);
                } else if constexpr (OUT) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int p = 0; p < HELD; ++p) px[i][p] = *reinterpret_cast<const bf16x8 *>(matrices + kRecordMatrix + (i * HELD + p) * kTile);
                }
                reads_stay();
#pragma unroll
                for (int t = 0; t < 2; ++t) S.s[ks][t] = multiply<SP - 1>(kt[ks % 2][t], w, S.s[ks][t] * whole);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if constexpr (OUT) {
                    o[i] = multiply<HELD - 1>(px[i], u, rise[i] * z[i]) * scale;
                } else {
                    o[i] = m[i];
                }
            }
            // a column with a value that is not finite, or a head with a key or gate that is not, has none from there on
            if (__ballot(first < left))
                S.each([&](f32x4 &x, int r, int) {
                    if (first < left) x[r] = __builtin_nanf("");
                });
        }
        if (BUFFERS == 1) __syncthreads();
        if (c + 1 < chunks) {
            put(c + 1);
            v_now = v_next;
        }
        // (what is stored comes behind the wait for what the next chunk brings)
        if (WALK == kKept && works && c % 2 && c + 1 < chunks) keep(c + 1);
        if (WALK != kSums && works && col < (OUT ? dv : dvp)) {
            if (__ballot(first < left))
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e / 4][e % 4] = token_of(e) < first ? o[e / 4][e % 4] : __builtin_nanf("");
            if (!OUT && col >= dv) o[0] = o[1] = 0;
            if constexpr (OUT) store_column(op + int64_t(c) * 32 * a.o.tok, uint32_t(a.o.tok), left, min(16, dv - col0), o);
            else store_column(mp + int64_t(c) * 32 * dvp, uint32_t(dvp), left, min(16, dvp - col0), o);
        }
        __syncthreads();
    }
    if (!works) return;
    if (OUT && a.state_out && g.index == g.count - 1) S.store(a.state_out + (g.seq * a.heads + h) * states, dk, dv, dv, col0);
    if (WALK == kSums && !moves) S.store(a.segments + slot * states, dk, dv, dv, col0);
    if (WALK == kSums && moves) {
        S.store(a.moves + slot * a.dk * a.dkp, dk, dk, dkp, col0);
        if (a.moves_t)      // (rows from dk on are 0)
            S.each([&](f32x4 &x, int r, int d) {
                if (d + 8 * lg < dkp && col < cols) set<float>(a.moves_t + (slot * dk + col0) * dkp, uint32_t(lm * dkp + d + 8 * lg) * 4, d + 8 * lg < dk ? x[r] : 0.0f);
            });
    }
#endif
}

// Backwards: the gradient of the state, from the piece's end to its beginning; e and the gradient of v.
template <class T, int DK, Walk WALK> __device__ __forceinline__ void walk_back(const DeltaArgs &a, char *lds, const Piece &g, int64_t slot, int64_t h, int tile) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int PARTS = kInputParts<T>, SP = kStateParts, KS = DK / 32, BUFFERS = kBuffers<T, DK>;
    constexpr int MATRIX = kRows<T, DK>, READ = kReadBack, SLOT = MATRIX * 2 + READ;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int dk = int(a.dk), dv = int(a.dv), dkp = int(a.dkp), dvp = int(a.dvp), col0 = tile * 16, col = col0 + lm;
    const bool works = col0 < dv;
    const auto token_of = [&](int e) { return 16 * (e / 4) + 4 * lg + e % 4; };
    const int64_t chunk0 = first_piece(a, g.seq, kDeltaChunk) + g.begin / kDeltaChunk;
    const int chunks = int((g.len + 31) / 32);
    const int64_t states = a.dk * a.dv;
    const auto left_of = [&](int c) { return int(min(g.len - int64_t(c) * 32, int64_t(32))); };

    State<DK> D;
    if (WALK == kSums || !works) D.fill(0.0f);
    else if (a.d_segments) D.load(a.d_segments + slot * states, dk, dv, dv, col0);
    else if (a.d_state_out) D.load(a.d_state_out + (g.seq * a.heads + h) * states, dk, dv, dv, col0);
    else D.fill(0.0f);

    const T *const kp = same(at_token<T>(a.k, a, g, g.begin, h)), *const qp = same(at_token<T>(a.q, a, g, g.begin, h));
    const T *const dp = same(at_token<T>(a.d_o, a, g, g.begin, h) + col0);
    T *const vp = WALK == kKept && a.dv_out.p ? same(const_cast<T *>(at_token<T>(a.dv_out, a, g, g.begin, h)) + col0) : nullptr;
    float *const ep = WALK == kKept && a.e ? same(a.e + (h * a.n_tokens + g.first + g.begin) * a.dvp + col0) : nullptr;
    Stage<T, DK> rk, rq;
    StageRecord<READ, kRecordHead, kRecordMatrix> record;
    Bits<T> d_next, d_now;
    const auto fetch = [&](int c) __attribute__((always_inline)) {
        const int left = left_of(c);
        record.fetch(a.chunks + ((chunk0 + c) * a.heads + h) * a.record);
        rk.fetch(kp + int64_t(c) * 32 * a.k.tok, uint32_t(a.k.tok), left, dkp);
        rq.fetch(qp + int64_t(c) * 32 * a.q.tok, uint32_t(a.q.tok), left, dkp);
        const T *d = dp + int64_t(c) * 32 * a.d_o.tok;
        if (works) d_next.load(d, uint32_t(a.d_o.tok), left, min(16, dv - col0));
    };
    const auto put = [&](int c) __attribute__((always_inline)) {
        char *to = lds + c % BUFFERS * SLOT;
        rk.put(to, left_of(c), dkp);
        rq.put(to + MATRIX, left_of(c), dkp);
        record.put(to + 2 * MATRIX);
    };

    // the gradient of the state after a block
    float *const kept = WALK == kKept && a.d_states ? same(a.d_states + ((first_piece(a, g.seq, kDeltaBlock) + g.begin / kDeltaBlock) * a.heads + h) * dk * dvp) : nullptr;
    const auto keep = [&](int c) __attribute__((always_inline)) { D.store(kept + int64_t(c / 2) * a.heads * dk * dvp, dk, dv, dvp, col0); };
    if (chunks) {
        fetch(chunks - 1);
        put(chunks - 1);
        d_now = d_next;
    }
    if (kept && works && chunks) keep(chunks - 1);
    __syncthreads();
    for (int c = chunks - 1; c >= 0; --c) {
        const char *k = lds + c % BUFFERS * SLOT, *q = k + MATRIX, *matrices = k + 2 * MATRIX + kRecordHead + l * 16;
        const RecordHead *head = reinterpret_cast<const RecordHead *>(k + 2 * MATRIX);
        const int left = left_of(c);
        if (c > 0) fetch(c - 1);
        f32x4 e_now[2], x_now[2];
        if (works) {
            f32x4 w[2], o[2], beta[2], rise[2], fall[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = 0;
            bf16x8 kx[2][2][PARTS], tx[2][SP];
            const auto read_rows = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) rows_operand<T, DK>(k, i, ks, kx[ks % 2][i]);
            };
            const auto read_matrix = [&](const char *from) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int p = 0; p < SP; ++p) tx[i][p] = *reinterpret_cast<const bf16x8 *>(from + (i * SP + p) * kTile);
            };
            read_rows(0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 1 < KS) read_rows(ks + 1);
                else read_matrix(matrices + kRecordMatrix);
                reads_stay();
                bf16x8 s[SP];
                D.operand(ks, s);
#pragma unroll
                for (int i = 0; i < 2; ++i) w[i] = multiply<SP - 1>(kx[ks % 2][i], s, w[i]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                beta[i] = *reinterpret_cast<const f32x4 *>(head->beta + 16 * i + 4 * lg);
                rise[i] = *reinterpret_cast<const f32x4 *>(head->rise + 16 * i + 4 * lg);
                fall[i] = *reinterpret_cast<const f32x4 *>(head->fall + 16 * i + 4 * lg);
            }
            bf16x8 od[PARTS], du[SP], x[SP];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (token_of(e) >= left) d_now.b[e] = 0;
                split(d_now.value(e), od, e);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) o[i] = multiply<SP - 1>(tx[i], od, f32x4{0, 0, 0, 0}) * a.scale + fall[i] * w[i];
            read_matrix(matrices);
            reads_stay();
#pragma unroll
            for (int e = 0; e < 8; ++e) split(o[e / 4][e % 4], du, e);
            bf16x8 kt[2][2][PARTS], qt[2][2][PARTS];
            const auto read_widths = [&](int ks) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    widths_operand<T, DK>(q, ks, t, qt[ks % 2][t]);
                    widths_operand<T, DK>(k, ks, t, kt[ks % 2][t]);
                }
            };
            read_widths(0);
            reads_stay();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e_now[i] = multiply<SP - 1>(tx[i], du, f32x4{0, 0, 0, 0});
                x_now[i] = beta[i] * e_now[i];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float up = rise[e / 4][e % 4];
                split(up * a.scale * d_now.value(e), du, e);
                split(-up * x_now[e / 4][e % 4], x, e);
            }
            const float whole = head->bad < left ? __builtin_nanf("") : head->whole;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 1 < KS) read_widths(ks + 1);
                reads_stay();
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const f32x4 d = multiply<SP - 1>(qt[ks % 2][t], du, D.s[ks][t] * whole);
                    D.s[ks][t] = multiply<SP - 1>(kt[ks % 2][t], x, d);
                }
            }
        }
        if (BUFFERS == 1) __syncthreads();
        if (c > 0) {
            put(c - 1);
            d_now = d_next;
        }
        // (what is stored comes behind the wait for what the next chunk brings)
        if (kept && works && c && c % 2 == 0) keep(c - 1);
        if (WALK == kKept && works && col < dvp) {
            if (col >= dv) e_now[0] = e_now[1] = 0;
            if (ep) store_column(ep + int64_t(c) * 32 * dvp, uint32_t(dvp), left, min(16, dvp - col0), e_now);
            if (vp && col < dv) store_column(vp + int64_t(c) * 32 * a.dv_out.tok, uint32_t(a.dv_out.tok), left, min(16, dv - col0), x_now);
        }
        __syncthreads();
    }
    if (!works) return;
    if (WALK == kKept && a.d_state_in && g.index == 0) D.store(a.d_state_in + (g.seq * a.heads + h) * states, dk, dv, dv, col0);
    if (WALK == kSums) D.store(a.d_segments + slot * states, dk, dv, dv, col0);
#endif
}

// From segment to segment of a sequence: what enters each takes the place of what it adds.  BACK: of the gradient, from the
// back.  A chain: 5.6 us a step of 128 x 128.  Four waves, 16 columns of v each; 64 widths at a time of what a segment makes of a state lie in LDS as parts, the next
// ones on their way.  A sequence without tokens has its final state (its initial state's gradient) here.
template <int DK> constexpr int kCarryWide = DK < 64 ? DK : 64;
template <int DK> constexpr int kCarryLds = kStateParts * kCarryWide<DK> * DK * 2;
template <int DK, bool BACK> __device__ __forceinline__ void carry(const DeltaArgs &a, char *lds, int64_t seq, int64_t h, int tile) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int KS = DK / 32, SP = kStateParts, WIDE = kCarryWide<DK>, G = WIDE / 8, PART = DK * G * 16, LOADS = DK * G / 256 > 0 ? DK * G / 256 : 1;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16;
    const int dk = int(a.dk), dv = int(a.dv), dkp = int(a.dkp), col0 = tile * 16;
    const int64_t states = a.dk * a.dv, own = (seq * a.heads + h) * states;
    const bool works = col0 < dv;
    const int64_t id0 = first_piece(a, seq, a.seg_len);
    const int64_t tokens = a.offsets ? max(token_at(a, seq + 1) - token_at(a, seq), int64_t(0)) : a.n_tokens / a.n_seq;
    const int count = __builtin_amdgcn_readfirstlane(int((tokens + a.seg_len - 1) / a.seg_len));
    const float *in = BACK ? a.d_state_out : a.state_in;
    float *const out = BACK ? a.d_state_in : a.state_out, *const adds = BACK ? a.d_segments : a.segments;
    const float *const moves = BACK ? a.moves_t : a.moves;
    State<DK> S, next, later;
    if (in && works) S.load(in + own, dk, dv, dv, col0);
    else S.fill(0.0f);
    if (count == 0 && out && works) S.store(out + own, dk, dv, dv, col0);
    const auto slot_of = [&](int i) { return (id0 + (BACK ? count - 1 - i : i)) * a.heads + h; };
    // widths `wide` on of the rows of what segment i makes of a state
    Eight<float> held[LOADS];
    const auto fetch = [&](int i, int wide) __attribute__((always_inline)) {
        const float *m = moves + slot_of(i) * dk * dkp;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int at = j * 256 + threadIdx.x, d = at / G, w = wide + at % G * 8;
            get_eight(held[j], m, d < dk && w < dkp ? uint32_t(d * dkp + w) * 4 : 0);
        }
    };
    if (count > 1) {
        fetch(0, 0);
        if (works) next.load(adds + slot_of(0) * states, dk, dv, dv, col0);
    }
    for (int i = 0; i < count; ++i) {
        if (works) S.store(adds + slot_of(i) * states, dk, dv, dv, col0);
        if (i + 1 == count) return;
#pragma unroll
        for (int wide = 0; wide < DK; wide += WIDE) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int at = j * 256 + threadIdx.x, row = at / G, gr = at % G;
                const bool in = row < dk && wide + gr * 8 < dkp;
                bf16x8 p[SP];
                parts_of(held[j], p);
                if (at < DK * G)
#pragma unroll
                    for (int q = 0; q < SP; ++q) *reinterpret_cast<bf16x8 *>(lds + q * PART + (row * G + (gr ^ turned<G>(row))) * 16) = in ? p[q] : bf16x8(bf16(0.0f));
            }
            __syncthreads();
            if (wide + WIDE < DK) {
                fetch(i, wide + WIDE);
            } else if (i + 2 < count) {
                fetch(i + 1, 0);
                if (works) later.load(adds + slot_of(i + 1) * states, dk, dv, dv, col0);
            }
            if (!works) continue;
#pragma unroll
            for (int ks = 0; ks < WIDE / 32; ++ks) {
                bf16x8 s[SP];
                S.operand(wide / 32 + ks, s);
#pragma unroll
                for (int to = 0; to < 2 * KS; ++to) {
                    const int row = to / 2 * 32 + 8 * (lm / 4) + 4 * (to % 2) + lm % 4, at = (row * G + ((4 * ks + lg) ^ turned<G>(row))) * 16;
                    bf16x8 x[SP];
#pragma unroll
                    for (int q = 0; q < SP; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(lds + q * PART + at);
                    next.s[to / 2][to % 2] = multiply<SP - 1>(x, s, next.s[to / 2][to % 2]);
                }
            }
        }
        S = next;
        next = later;
    }
#endif
}

// Whether sequences are cut into segments, and how.  Segments cost two to three times the work, so they pay where whole
// sequences leave the matrix units idle; their number is weighed against their length, since one hands its state on to the next
// (5 us where heads are 128 wide, 2 where 64), and two waves on each of 1,024 matrix units are enough.  us of the forward pass and of
// the gradient in bfloat16, whole | 128 | 256 | 512 | 1024 tokens a segment; what the rule takes is in brackets.  16 heads of 128, one
// series of 512 tokens 51, 93 | [58, 104] | 61, 111; 1024 87, 145 | 87, 147 | [75, 131]; 4096 311, 537 | 270, 511 | 178, 396 | [145, 353]
// | 175, 375; 16384 1251, 2235 | 1075, 2015 | 688, 1569 | 512, 1338 | [420, 1184]; two of 1024 88, 171 | 105, 217 | [84, 183]; two of
// 4096 332, 716 | 369, 851 | 264, 714 | [220, 628] | 216, 624; four of 4096 [365, 1030] | 583, 1517 | 457, 1325 | 394, 1217 | 351, 1121.
// 4 heads of 64, 4096 220, 343 | 91, 127 | [71, 112] | 80, 129; eight of 2048 119, 221 | 82, 173 | [68, 153]; sixteen of 1024 69, 145 |
// [67, 159] | 60, 146.  4 heads of 192, 1024 129, 257 | 310, 437 | [202, 306] | 184, 301; 4096 468, 795 | 1311, 1487 | 706, 882 |
// [426, 595] | 373, 545; 16384 1819, 3170 | - | 2709, 3799 | 1499, 2134 | [922, 1586], at 2048 729, 1419.
// It is off the best of these by up to 18% where sequences are barely long enough, and by up to 54% for heads of more than 128
// widths, whose transitions cost most (in half and float, by up to 26%).  Only the mean length counts: among many short or
// empty packed sequences a long one stays whole, 2.4 us for 32 of its tokens.
inline bool cut(DeltaArgs &a) {
    constexpr int64_t kWaves = 2048, kShortest = 128;
    const int64_t per_token = a.heads * ceil_div(a.dv, 16), mean = a.n_seq ? a.n_tokens / a.n_seq : 0;
    a.seg_len = kShortest;
    while (4 * a.seg_len * a.seg_len < mean * a.dk || a.seg_len * kWaves < a.n_tokens * per_token) a.seg_len *= 2;
    if (a.n_seq && a.n_seq * per_token * 8 <= kWaves && mean >= 4 * a.seg_len) {
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
