// Attention by the gated delta rule: the forward pass, and the step of a single token.  (Formulas: delta_parts.h.)
// Three launches: a record for each chunk of 32 tokens and head (the inverse of I + A, and P); then workgroups walk
// the chunks of a sequence for one head and 32 or more columns of v, with their columns of the state in the accumulators.
#include "delta_parts.h"

namespace ndvm {
namespace ops {
namespace {

// What a walk leaves: outputs and the final state; or, for the gradient, the state before each block of 64 tokens and u.
enum Walk { kOutputs, kKept };

// Four waves, Split<DK>.  A chunk: Y = K S and Z = Q S, each wave over its widths, added up through LDS; a wave then has
// one, two or four 16 x 16 tiles (token half a, column half n) of R = b (V - exp G Y), of U = (I + A)^-1 R and of the
// outputs; R and U go through LDS as parts, where every wave that needs them reads them as operands.
// Rows of S are numbered so that the eight values a lane holds in a pair of tiles are eight consecutive widths.
template <class T, int DK, Walk WALK> __global__ void __launch_bounds__(256) delta_walk(DeltaArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef Split<DK> S_;
    constexpr int PARTS = kInputParts<T>, HELD = kResultParts<T>, SP = kStateParts;
    constexpr int WK = S_::WK, WN = S_::WN, KPW = S_::KPW, G = S_::G, OWN = S_::OWN, NA = WK == 1 ? 2 : 1;
    constexpr bool OUT = WALK == kOutputs;
    constexpr int PART = 32 * G * 16;                       // bytes of a part of the chunk's rows
    constexpr int LOADS = 32 * G / 256 > 0 ? 32 * G / 256 : 1;      // granules a thread brings
    constexpr bool TWICE = PARTS * PART <= 32768 || DK < 256;       // two buffers of k
    constexpr int SLOT = 80;                                // bytes of a column of 32 tokens in LDS
    __shared__ __align__(16) char lk[TWICE ? 2 : 1][PARTS * PART], lq[OUT ? PARTS * PART : 16];
    __shared__ f32x4 py[4][4][64], pz[OUT ? 4 : 1][4][64];
    __shared__ __align__(16) char lr[WN][SP][32 * SLOT], lu[WN][SP][32 * SLOT], lp[OUT ? WN : 1][OUT ? HELD : 1][32 * SLOT];
    __shared__ int unfit[32 * WN];                          // of a column of v: its first token that is not finite

    const uint32_t id = blockIdx.x / uint32_t(a.heads);
    const int64_t h = blockIdx.x - id * uint32_t(a.heads);
    const Piece g = find_piece(a, id, a.seg_len, a.n_segments == a.n_seq);
    if (g.count == 0) return;
    const int l = threadIdx.x % 64, lm = l % 16, lg = l / 16, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int kp = wave % WK, np = wave / WK;
    const int64_t col0 = int64_t(blockIdx.y) * S_::NC + np * 32;
    const auto column = [&](int n) { return col0 + n * 16 + lm; };
    // tile o of the wave: token half, column half
    const auto half_a = [&](int o) { return WK == 4 ? kp / 2 : WK == 2 ? kp : o / 2; };
    const auto half_n = [&](int o) { return WK == 4 ? kp % 2 : o % 2; };
    const int64_t chunk0 = first_piece(a, g.seq, kDeltaChunk) + g.begin / kDeltaChunk;
    const int chunks = int((g.len + 31) / 32);
    constexpr int RECORD = OUT ? kRecord<T> : kRecordGrad<T>;
    const auto record_of = [&](int c) { return a.chunks + ((chunk0 + c) * a.heads + h) * RECORD; };

    // the state: widths (kp KPW + ks) 32 + 8 lg + 4 t + r, columns column(n)
    f32x4 S[KPW][2][2];
    const auto width = [&](int ks, int t, int r) { return (kp * KPW + ks) * 32 + 8 * lg + 4 * t + r; };
    {
        const float *in = a.state_in ? a.state_in + (g.seq * a.heads + h) * a.dk * a.dv : nullptr;
#pragma unroll
        for (int ks = 0; ks < KPW; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int64_t d = width(ks, t, r), c = column(n);
                        S[ks][t][n][r] = in && d < a.dk && c < a.dv ? in[d * a.dv + c] : 0.0f;
                    }
    }
    const auto store_state = [&](float *to) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < KPW; ++ks)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int64_t d = width(ks, t, r), c = column(n);
                        if (d < a.dk && c < a.dv) to[d * a.dv + c] = S[ks][t][n][r];
                    }
    };

    // what a chunk brings, a chunk ahead
    Eight<T> rk[LOADS], rq[OUT ? LOADS : 1];
    const int brings = 32 * G / 256 > 0 ? 256 : 32 * G;     // threads that bring rows
    const auto fetch_rows = [&](int c) __attribute__((always_inline)) {
        const int left = int(min(g.len - int64_t(c) * 32, int64_t(32)));
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / G, gr = at % G;
            const int64_t have = row < left && int(threadIdx.x) < brings ? a.dk - gr * 8 : 0;
            rk[i] = load_eight(at_token<T>(a.k, a, g, g.begin + c * 32 + row, h) + gr * 8, have);
            if (OUT) rq[i] = load_eight(at_token<T>(a.q, a, g, g.begin + c * 32 + row, h) + gr * 8, have);
        }
    };
    const auto put_rows = [&](const Eight<T>(&from)[LOADS], char *to) __attribute__((always_inline)) {
        if (int(threadIdx.x) >= brings) return;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = i * 256 + threadIdx.x, row = at / G, gr = at % G;
            bf16x8 p[PARTS];
            parts_of(from[i], p);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8 *>(to + q * PART + (row * G + (gr ^ turned<G>(row))) * 16) = p[q];
        }
    };
    struct Small {
        bf16x8 t[NA][SP], p[OUT ? NA : 1][OUT ? HELD : 1];
        f32x4 beta[NA], rise[NA], fall[NA];
        float whole;
        int bad;
        T v[OWN][4];
    };
    const auto fetch_small = [&](int c, Small &s) __attribute__((always_inline)) {
        const char *record = record_of(c);
        const RecordHead *head = reinterpret_cast<const RecordHead *>(record);
        const char *t = record + kRecordHead + l * 16, *p = t + kRecordMatrix;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int ha = WK == 1 ? i : half_a(0);
#pragma unroll
            for (int q = 0; q < SP; ++q) s.t[i][q] = *reinterpret_cast<const bf16x8 *>(t + (ha * SP + q) * kTile);
            if constexpr (OUT)
#pragma unroll
                for (int q = 0; q < HELD; ++q) s.p[i][q] = *reinterpret_cast<const bf16x8 *>(p + (ha * HELD + q) * kTile);
            const int row = 16 * ha + 4 * lg;
            s.beta[i] = *reinterpret_cast<const f32x4 *>(head->beta + row);
            s.rise[i] = *reinterpret_cast<const f32x4 *>(head->rise + row);
            s.fall[i] = *reinterpret_cast<const f32x4 *>(head->fall + row);
        }
        s.whole = head->whole;
        s.bad = head->bad;
        const int left = int(min(g.len - int64_t(c) * 32, int64_t(32)));
#pragma unroll
        for (int o = 0; o < OWN; ++o)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * half_a(o) + 4 * lg + r;
                const int64_t col = column(half_n(o));
                s.v[o][r] = T(0.0f);
                if (row < left && col < a.dv) s.v[o][r] = at_token<T>(a.v, a, g, g.begin + c * 32 + row, h)[col];
            }
    };

    Small cur;
    if (chunks) {
        fetch_rows(0);
        fetch_small(0, cur);
        put_rows(rk, lk[0]);
        if constexpr (OUT) put_rows(rq, lq);
    }
    if (threadIdx.x < 32 * WN) unfit[threadIdx.x] = 32;
    __syncthreads();
    for (int c = 0; c < chunks; ++c) {
        const char *k = lk[TWICE ? c % 2 : 0];
        const int left = int(min(g.len - int64_t(c) * 32, int64_t(32)));
        const int64_t token = g.begin + c * 32;
        if constexpr (!OUT)
            if (c % 2 == 0) {
                const int64_t block = first_piece(a, g.seq, kDeltaBlock) + token / kDeltaBlock;
                store_state(a.states + (block * a.heads + h) * a.dk * a.dv);
            }
        Small next;
        if (c + 1 < chunks) {
            fetch_rows(c + 1);
            fetch_small(c + 1, next);
        }
        // Y and Z over the wave's widths
        f32x4 y[2][2], z[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n) y[i][n] = z[i][n] = 0;
#pragma unroll
        for (int ks = 0; ks < KPW; ++ks) {
            bf16x8 s[2][SP];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) split(S[ks][e / 4][n][e % 4], s[n], e);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = 16 * i + lm, at = (row * G + (((kp * KPW + ks) * 4 + lg) ^ turned<G>(row))) * 16;
                bf16x8 x[PARTS];
#pragma unroll
                for (int q = 0; q < PARTS; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(k + q * PART + at);
#pragma unroll
                for (int n = 0; n < 2; ++n) y[i][n] = multiply<SP - 1>(x, s[n], y[i][n]);
                if constexpr (OUT) {
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(lq + q * PART + at);
#pragma unroll
                    for (int n = 0; n < 2; ++n) z[i][n] = multiply<HELD - 1>(x, s[n], z[i][n]);
                }
            }
        }
        f32x4 own_y[OWN], own_z[OWN];
        if constexpr (WK > 1) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    py[wave][i * 2 + n][l] = y[i][n];
                    if (OUT) pz[OUT ? wave : 0][i * 2 + n][l] = z[i][n];
                }
            __syncthreads();
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const int t = half_a(o) * 2 + half_n(o);
                own_y[o] = py[np * WK][t][l];
                if (OUT) own_z[o] = pz[OUT ? np * WK : 0][t][l];
#pragma unroll
                for (int w = 1; w < WK; ++w) {
                    own_y[o] += py[np * WK + w][t][l];
                    if (OUT) own_z[o] += pz[OUT ? np * WK + w : 0][t][l];
                }
            }
        } else {
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                own_y[o] = y[o / 2][o % 2];
                own_z[o] = z[o / 2][o % 2];
            }
            __syncthreads();      // the rows of q have been read, and those of k that the next ones replace
        }
        // R of the wave's tiles; a value of v that is not finite counts as 0, and what follows it in its column is set below
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int i = WK == 1 ? o / 2 : 0, row0 = 16 * half_a(o) + 4 * lg, slot = half_n(o) * 16 + lm;
            bf16x4 p[SP];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = float(cur.v[o][r]);
                if (!finite(v)) {
                    atomicMin(&unfit[np * 32 + slot], row0 + r);
                    v = 0.0f;
                }
                const float x = row0 + r < cur.bad ? cur.beta[i][r] * (v - cur.rise[i][r] * own_y[o][r]) : 0.0f;
                split(x, p, r);
            }
#pragma unroll
            for (int q = 0; q < SP; ++q) *reinterpret_cast<bf16x4 *>(lr[np][q] + slot * SLOT + row0 * 2) = p[q];
        }
        if constexpr (OUT)
            if (c + 1 < chunks) put_rows(rq, lq);
        if constexpr (TWICE)
            if (c + 1 < chunks) put_rows(rk, lk[(c + 1) % 2]);
        __syncthreads();
        // U of the wave's tiles
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            const int i = WK == 1 ? o / 2 : 0, row0 = 16 * half_a(o) + 4 * lg, slot = half_n(o) * 16 + lm;
            bf16x8 x[SP];
#pragma unroll
            for (int q = 0; q < SP; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(lr[np][q] + slot * SLOT + lg * 16);
            f32x4 u = 0;
            u = multiply<SP - 1>(cur.t[i], x, u);
            bf16x4 p[SP], w[HELD];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                split(u[r] * cur.fall[i][r], p, r);
                split(u[r], w, r);
            }
#pragma unroll
            for (int q = 0; q < SP; ++q) *reinterpret_cast<bf16x4 *>(lu[np][q] + slot * SLOT + row0 * 2) = p[q];
            if constexpr (OUT) {
#pragma unroll
                for (int q = 0; q < HELD; ++q) *reinterpret_cast<bf16x4 *>(lp[np][q] + slot * SLOT + row0 * 2) = w[q];
            } else {
                const int first = min(unfit[np * 32 + slot], cur.bad);
                const int64_t col = column(half_n(o));
                float *to = a.u + (h * a.n_tokens + g.first + token + row0) * a.dv + col;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (row0 + r < left && col < a.dv) to[r * a.dv] = row0 + r < first ? u[r] : __builtin_nanf("");
            }
        }
        __syncthreads();
        // S' = exp(G_last) S + K^T (fall U)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            bf16x8 x[SP];
#pragma unroll
            for (int q = 0; q < SP; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(lu[np][q] + (n * 16 + lm) * SLOT + lg * 16);
#pragma unroll
            for (int ks = 0; ks < KPW; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    bf16x8 kt[PARTS];
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) {
                        // lane 4 r + x: token 8 lg + r (and 4 on), widths 8 x + 4 t on
                        const int row = 8 * lg + lm / 4, gr = (kp * KPW + ks) * 4 + lm % 4;
                        const char *from = k + q * PART + 8 * t;
                        const bf16x4 lo = read_transposed(from + (row * G + (gr ^ turned<G>(row))) * 16);
                        const bf16x4 hi = read_transposed(from + ((row + 4) * G + (gr ^ turned<G>(row + 4))) * 16);
                        kt[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    }
                    S[ks][t][n] *= cur.whole;
                    S[ks][t][n] = multiply<SP - 1>(kt, x, S[ks][t][n]);
                }
        }
        if constexpr (OUT) {
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const int i = WK == 1 ? o / 2 : 0, row0 = 16 * half_a(o) + 4 * lg, slot = half_n(o) * 16 + lm;
                bf16x8 x[HELD];
#pragma unroll
                for (int q = 0; q < HELD; ++q) x[q] = *reinterpret_cast<const bf16x8 *>(lp[np][q] + slot * SLOT + lg * 16);
                f32x4 v = cur.rise[i] * own_z[o];
                v = multiply<HELD - 1>(cur.p[i], x, v);
                const int first = min(unfit[np * 32 + slot], cur.bad);
                const int64_t col = column(half_n(o));
                if (col < a.dv)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (row0 + r < left)
                            const_cast<T *>(at_token<T>(a.o, a, g, token + row0 + r, h))[col] = T(row0 + r < first ? v[r] * a.scale : __builtin_nanf(""));
            }
        }
        // a column with a value that is not finite, or a head with a key or gate that is not, has none from there on
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (min(unfit[np * 32 + n * 16 + lm], cur.bad) >= left) continue;
#pragma unroll
            for (int ks = 0; ks < KPW; ++ks)
#pragma unroll
                for (int t = 0; t < 2; ++t) S[ks][t][n] = __builtin_nanf("");
        }
        if constexpr (!TWICE)
            if (c + 1 < chunks) {
                __syncthreads();
                put_rows(rk, lk[0]);
                __syncthreads();
            }
        cur = next;
    }
    if (OUT && g.index == g.count - 1 && a.state_out) store_state(a.state_out + (g.seq * a.heads + h) * a.dk * a.dv);
#endif
}

// One token of every stream: S <- a S + k^T u, u = b (v - a k S), o = scale q S = scale (q (a S) + (q k) u).  Bound by the
// state's way through memory: 8 dk dv bytes.  X threads of four columns each side by side, 256 / X rows at a time; a thread's
// values of the state stay in its registers (at most RG of its rows) between the sums k S and q S, which are added up over
// the rows in one go, and the update.
template <class T, int X, int RG, bool PASSING> __global__ void __launch_bounds__(256) delta_step(DeltaStepArgs a) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int R = 256 / X;
    __shared__ float lq[256], lk[256], dots[4];
    __shared__ f32x4 part[2][R][X];
    const int64_t b = blockIdx.x, h = blockIdx.y;
    const int x = threadIdx.x % X, g = threadIdx.x / X;
    const int64_t c = (int64_t(blockIdx.z) * X + x) * 4;
    const int64_t slot = a.slots ? a.slots[b] : b;
    T *o = static_cast<T *>(const_cast<void *>(a.o.p)) + b * a.o.seq + h * a.o.head;
    const int have = int(min(max(a.dv - c, int64_t(0)), int64_t(4)));
    if (slot < 0 || slot >= a.n_slots) {        // a stream without a state: its output is 0
        if (g == 0)
            for (int j = 0; j < have; ++j) o[c + j] = T(0.0f);
        return;
    }
    const auto row = [&](const Heads &y) { return static_cast<const T *>(y.p) + b * y.seq + h / y.group * y.head; };
    const T *v = row(a.v);
    float dot = 0;
    {
        const int t = threadIdx.x;
        const float qt = t < a.dk ? float(row(a.q)[t]) : 0.0f, kt = t < a.dk ? float(row(a.k)[t]) : 0.0f;
        lq[t] = qt;
        lk[t] = kt;
        dot = qt * kt;
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) dot += __shfl_xor(dot, s);
        if (t % 64 == 0) dots[t / 64] = dot;
    }
    const float beta = float(*row(a.beta)), decay = expf(float(*row(a.g)));
    f32x4 vv = {0, 0, 0, 0}, ks = {0, 0, 0, 0}, qs = {0, 0, 0, 0}, S[RG];
    for (int j = 0; j < have; ++j) vv[j] = float(v[c + j]);
    float *base = a.state + (slot * a.heads + h) * a.dk * a.dv + c;
#pragma unroll
    for (int i = 0; i < RG; ++i) {
        const int64_t d = i * R + g;
        S[i] = f32x4{0, 0, 0, 0};
        if (d >= a.dk) continue;
        if (have == 4) {
            const f4 *at = reinterpret_cast<const f4 *>(base + d * a.dv);
            S[i] = PASSING ? __builtin_nontemporal_load(at) : *at;
        } else {
            for (int j = 0; j < have; ++j) S[i][j] = base[d * a.dv + j];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RG; ++i) {
        const int d = i * R + g;        // up to 255: k and q are 0 from dk on
        S[i] *= decay;
        ks += S[i] * lk[d];
        qs += S[i] * lq[d];
    }
    part[0][g][x] = ks;
    part[1][g][x] = qs;
    __syncthreads();
    ks = part[0][0][x];
    for (int i = 1; i < R; ++i) ks += part[0][i][x];
    const f32x4 u = beta * (vv - ks);
#pragma unroll
    for (int i = 0; i < RG; ++i) {
        const int64_t d = i * R + g;
        if (d >= a.dk) continue;
        const f32x4 s = S[i] + u * lk[d];
        if (have == 4) {
            f4 *at = reinterpret_cast<f4 *>(base + d * a.dv);
            if (PASSING) __builtin_nontemporal_store(f4(s), at);
            else *at = s;
        } else {
            for (int j = 0; j < have; ++j) base[d * a.dv + j] = s[j];
        }
    }
    if (g) return;
    qs = part[1][0][x];
    for (int i = 1; i < R; ++i) qs += part[1][i][x];
    qs += u * (dots[0] + dots[1] + dots[2] + dots[3]);
    for (int j = 0; j < have; ++j) o[c + j] = T(qs[j] * a.scale);
}

// Where a launch keeps what: the records of the chunks.
struct Space {
    char *base;
    size_t used = 0;
    explicit Space(void *p) : base(p ? reinterpret_cast<char *>(round256(reinterpret_cast<size_t>(p))) : nullptr) {}
    template <class P> void take(P *&p, int64_t bytes) {
        p = base ? reinterpret_cast<P *>(base + used) : nullptr;
        used += round256(size_t(bytes));
    }
};
template <class T> size_t lay_out(DeltaArgs &a, Space s) {
    s.take(a.chunks, piece_ids(a, kDeltaChunk) * a.heads * kRecord<T>);
    return s.used + 256;
}

void cut(DeltaArgs &a) {
    a.seg_len = std::max<int64_t>(kDeltaBlock, a.n_tokens);
    a.n_segments = a.n_seq;
}

template <class T> void delta(DeltaArgs a, hipStream_t stream) {
    cut(a);
    lay_out<T>(a, Space(a.ws));
    const int64_t pairs = piece_ids(a, kDeltaChunk) * a.heads;
    if (a.n_tokens) delta_prepare<T, false><<<dim3(uint32_t(ceil_div(pairs, 4))), 256, 0, stream>>>(a, pairs);
    with_width<T>(a.dk, [&](auto d) {
        constexpr int DK = decltype(d)::value;
        delta_walk<T, DK, kOutputs><<<dim3(uint32_t(a.n_segments * a.heads), uint32_t(ceil_div(a.dv, Split<DK>::NC))), 256, 0, stream>>>(a);
    });
}

}  // namespace

size_t delta_bytes(int dtype, const DeltaArgs &a, bool grad) {
    DeltaArgs b = a;
    return dtype == NDVM_F32 ? lay_out<float>(b, Space(nullptr)) : lay_out<bf16>(b, Space(nullptr));
}

hipError_t launch_delta(int dtype, DeltaArgs a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        delta<decltype(zero)>(a, stream);
        return hipGetLastError();
    });
}

hipError_t launch_delta_step(int dtype, const DeltaStepArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const auto grid = [&](int64_t x) { return dim3(uint32_t(a.n_seq), uint32_t(a.heads), uint32_t(ceil_div(a.dv, 4 * x))); };
        const bool passing = a.n_seq * a.heads * a.dk * a.dv * 4 >= kPassingStates, wide = a.n_seq * a.heads * ceil_div(a.dv, 128) >= 2 * kCus;
        if (a.dk <= 128) {
            if (passing) delta_step<T, 32, 16, true><<<grid(32), 256, 0, stream>>>(a);
            else if (wide) delta_step<T, 32, 16, false><<<grid(32), 256, 0, stream>>>(a);
            else delta_step<T, 8, 4, false><<<grid(8), 256, 0, stream>>>(a);
        } else {
            if (passing) delta_step<T, 32, 32, true><<<grid(32), 256, 0, stream>>>(a);
            else delta_step<T, 8, 8, false><<<grid(8), 256, 0, stream>>>(a);
        }
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
