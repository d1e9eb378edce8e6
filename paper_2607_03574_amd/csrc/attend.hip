// Linear attention with a decay for each head, in the chunked form.
//   out_i = sum_{j<=i} lambda^(i-j) (a_i . b_j) c_j + (what the sequence started with)
// The forward pass takes (a, b, c) = (q, k, v); its gradient is three more of the
// same sums: dq = (do, v, k), and from the last token to the first
// dv = (k, q, do), dk = (v, do, q).
// The sum over earlier tokens is a state S [da, dc] in float: with S what
// entered a chunk of n tokens (e = 1; reversed, the state has decayed once already: e = 0)
//   out_i = lambda^(i+e) a_i S + sum_{j<=i in chunk} lambda^(i-j) (a_i . b_j) c_j
//   S'    = lambda^n S + sum_j lambda^(n-e-j) b_j^T c_j
// A workgroup walks the chunks of one segment of a sequence for one head, with S
// in the accumulator registers of the matrix instructions.  Sequences are cut
// into segments where sequences and heads alone would not fill the GPU: then a
// first launch sums what each segment adds, a second one carries states over
// the segments in order, and the last one computes the outputs.
#include <algorithm>

#include "ops.h"
#include "ops_types.h"

namespace ndvm {
namespace ops {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// exp(g n) with lambda^0 = 1 for every g.
__device__ inline float decay(float g, int64_t n) { return n == 0 ? 1.0f : expf(g * float(n)); }

// Where a segment of the launch lies.
struct Segment {
    int64_t seq, first, tokens;     // sequence, its first token, its length
    int64_t begin, len;             // the segment's place in the sequence (in walking order)
    int64_t index, count;           // of the sequence's segments
};

// Segment `id`: sequences of equal length have equally many segments.  Packed
// sequences have ids from offsets[s] / seg_len + s on, which leaves room for all of
// theirs; the spare ids are segments without tokens (count 0).
__device__ inline Segment find_segment(const AttendArgs &a, int64_t id) {
    Segment g;
    const bool cut = a.n_segments > a.n_seq;
    if (!a.offsets) {
        g.tokens = a.n_tokens / a.n_seq;
        const int64_t per = a.n_segments / a.n_seq;
        g.seq = id / per;
        g.index = id % per;
        g.first = g.seq * g.tokens;
    } else {
        const auto at = [&](int64_t s) { return min(max(a.offsets[s], int64_t(0)), a.n_tokens); };
        const auto base = [&](int64_t s) { return at(s) / a.seg_len + s; };
        int64_t lo = 0;
        if (!cut) {
            lo = id;
        } else {
            int64_t hi = a.n_seq;       // the last sequence whose ids begin at or before id
            while (hi - lo > 1) {
                const int64_t mid = (lo + hi) / 2;
                if (base(mid) <= id) lo = mid;
                else hi = mid;
            }
        }
        g.seq = lo;
        g.index = cut ? id - base(lo) : 0;
        g.first = at(lo);
        g.tokens = max(at(lo + 1) - g.first, int64_t(0));
    }
    g.count = cut ? max((g.tokens + a.seg_len - 1) / a.seg_len, int64_t(1)) : 1;
    g.begin = g.index * a.seg_len;
    g.len = cut ? min(a.seg_len, g.tokens - g.begin) : g.tokens;
    if (g.index < 0 || g.index >= g.count) g.count = 0;
    return g;
}

template <class T> __device__ inline const T *token_ptr(const Heads &h, const AttendArgs &a, const Segment &g, int64_t pos,
                                                         int64_t head) {
    const int64_t t = a.reversed ? g.tokens - 1 - pos : pos;
    const int64_t row = a.offsets ? (g.first + t) * h.tok : g.seq * h.seq + t * h.tok;
    return static_cast<const T *>(h.p) + row + head / h.group * h.head;
}

// The general kernel: any type, widths up to 16 DT, float matrix instructions
// (16 x 16 x 4).  Four waves, 16 columns of c each; chunks of 16 tokens, STAGE
// tokens in LDS at a time.
// A 16 x 16 accumulator has column l % 16, rows 4 (l / 16) + r in lane l, register r.
// S (rows: widths of b) and the transposed products P^T (rows: j, columns: i) are
// accumulated in that layout and used from it as operands: step r of a product
// over 16 rows takes rows 4 (l / 16) + r from lane l, and the other operand is read
// from LDS in that order, so neither goes through LDS.
template <class T, int DT, int STAGE, bool OUT>
__global__ void __launch_bounds__(256) attend_general(AttendArgs A) {
    constexpr int D = 16 * DT, LD = D + 4, LC = 64 + 4, V = kVec<T>;
    __shared__ float la[STAGE][LD], lb[STAGE][LD], lc[STAGE][LC];
    __shared__ float power[17];     // lambda^n
    const Segment g = find_segment(A, blockIdx.x);
    if (g.count == 0 || (!OUT && g.index == g.count - 1)) return;
    const int64_t h = blockIdx.y, col0 = int64_t(blockIdx.z) * 64;
    const int l = threadIdx.x % 64, wave = threadIdx.x / 64, lm = l % 16, lg = l / 16;
    const int64_t col = col0 + wave * 16 + lm;
    const float gl = A.log_decay[h];
    if (threadIdx.x < 17) power[threadIdx.x] = decay(gl, threadIdx.x);
    const int e = A.reversed ? 0 : 1;
    const bool cut = A.n_segments > A.n_seq;

    f32x4 S[DT];
    const float *in = !OUT ? nullptr : cut ? A.segments + (int64_t(blockIdx.x) * A.heads + h) * A.da * A.dc : A.state_in ? A.state_in + (g.seq * A.heads + h) * A.da * A.dc : nullptr;
    const bool in_transposed = !cut && A.state_transposed;
    const auto place = [&](int t, int r, bool transposed) {
        const int64_t d = 16 * t + 4 * lg + r;
        return d < A.da && col < A.dc ? (transposed ? col * A.da + d : d * A.dc + col) : int64_t(-1);
    };
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t at = place(t, r, in_transposed);
            S[t][r] = in && at >= 0 ? in[at] : 0.0f;
        }

    for (int64_t base = 0; base < g.len; base += STAGE) {
        bool odd = false;       // a value of c that is not finite
        __syncthreads();
        const auto load = [&](const Heads &H, float *to, int ld, int width, int64_t c0, int64_t n, bool watch) {
            const int vecs = width / V;
            for (int i = threadIdx.x; i < STAGE * vecs; i += 256) {
                const int row = i / vecs, c = i % vecs * V;
                vec<T> x = 0;
                if (base + row < g.len && c0 + c < n)
                    x = load_vec(token_ptr<T>(H, A, g, g.begin + base + row, h) + c0 + c, n - c0 - c);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float f = float(x[j]);
                    to[row * ld + c + j] = f;
                    if (watch) odd |= !(fabsf(f) <= 3.402823466e38f);
                }
            }
        };
        if (OUT) load(A.a, &la[0][0], LD, D, 0, A.da, false);
        load(A.b, &lb[0][0], LD, D, 0, A.da, false);
        load(A.c, &lc[0][0], LC, 64, col0, A.dc, true);
        odd = __syncthreads_or(odd);
        for (int s0 = 0; s0 < STAGE && base + s0 < g.len; s0 += 16) {
            const int n = int(min(g.len - base - s0, int64_t(16)));
            if (OUT) {
                f32x4 P = {0, 0, 0, 0}, O = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < D; k += 4)
                    P = __builtin_amdgcn_mfma_f32_16x16x4f32(lb[s0 + lm][k + lg], la[s0 + lm][k + lg], P, 0, 0, 0);
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        O = __builtin_amdgcn_mfma_f32_16x16x4f32(la[s0 + lm][16 * t + 4 * lg + r], S[t][r], O, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    O[r] *= A.scale_read * power[4 * lg + r + e];
                    const int j = 4 * lg + r;       // P: row j, column i = lm; what is masked is replaced, not multiplied
                    P[r] = j <= lm ? P[r] * (A.scale_pair * power[lm - j]) : 0.0f;
                }
                if (!odd) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        O = __builtin_amdgcn_mfma_f32_16x16x4f32(P[r], lc[s0 + 4 * lg + r][wave * 16 + lm], O, 0, 0, 0);
                } else {
                    // 0 times an infinity of a later token would be NaN: add the terms up to i alone
                    for (int j = 0; j < 16; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float pj = j % 4 == 0 ? P[0] : j % 4 == 1 ? P[1] : j % 4 == 2 ? P[2] : P[3];
                            const float p = __shfl(pj, 4 * lg + r + 16 * (j / 4));
                            if (j <= 4 * lg + r) O[r] += p * lc[s0 + j][wave * 16 + lm];
                        }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 4 * lg + r;
                    if (i >= n || col >= A.dc) continue;
                    const int64_t pos = g.begin + base + s0 + i;
                    if (A.out_f32) const_cast<float *>(token_ptr<float>(A.out, A, g, pos, h))[col] = O[r];
                    else const_cast<T *>(token_ptr<T>(A.out, A, g, pos, h))[col] = T(O[r]);
                }
            }
            const float whole = power[n];
#pragma unroll
            for (int t = 0; t < DT; ++t) S[t] *= whole;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 4 * r + lg;
                const float c = j < n ? lc[s0 + j][wave * 16 + lm] * (A.scale_add * power[n - e - j]) : 0.0f;
#pragma unroll
                for (int t = 0; t < DT; ++t)
                    S[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(lb[s0 + j][16 * t + lm], c, S[t], 0, 0, 0);
            }
        }
    }
    float *out = !OUT ? A.segments + (int64_t(blockIdx.x) * A.heads + h) * A.da * A.dc : g.index == g.count - 1 && A.state_out ? A.state_out + (g.seq * A.heads + h) * A.da * A.dc : nullptr;
    if (!out) return;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t at = place(t, r, OUT && A.state_transposed);
            if (at >= 0) out[at] = S[t][r];
        }
}

// States over the segments of a sequence, in order: what each adds is replaced
// by what enters it.  A thread an element of the state.
__global__ void __launch_bounds__(256) attend_carry(AttendArgs A) {
    const int64_t size = A.da * A.dc, at = int64_t(blockIdx.z) * 256 + threadIdx.x;
    const int64_t seq = blockIdx.x, h = blockIdx.y;
    if (at >= size) return;
    int64_t id, count;
    if (!A.offsets) {
        count = A.n_segments / A.n_seq;
        id = seq * count;
    } else {
        const int64_t lo = min(max(A.offsets[seq], int64_t(0)), A.n_tokens);
        const int64_t hi = min(max(A.offsets[seq + 1], int64_t(0)), A.n_tokens);
        id = lo / A.seg_len + seq;
        count = max((max(hi - lo, int64_t(0)) + A.seg_len - 1) / A.seg_len, int64_t(1));
        count = min(count, A.n_segments - id);
    }
    const int64_t from = A.state_transposed ? at % A.dc * A.da + at / A.dc : at;
    float cur = A.state_in ? A.state_in[(seq * A.heads + h) * size + from] : 0.0f;
    const float whole = decay(A.log_decay[h], A.seg_len);
    float *p = A.segments + (id * A.heads + h) * size + at;
    float next = count > 1 ? *p : 0.0f;
    for (int64_t i = 0; i < count; ++i, p += A.heads * size) {
        const float add = next;
        if (i + 2 < count) next = p[A.heads * size];
        *p = cur;
        cur = whole * cur + add;
    }
}

template <class T> __global__ void __launch_bounds__(256) fold_heads(FoldHeadsArgs a) {
    const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int group = a.out.group;
    if (at >= a.n_tokens * a.d) return;
    const int64_t tok = at / a.d, c = at % a.d, kv = blockIdx.y;
    float s = 0;
    for (int i = 0; i < group; ++i) s += a.part[((kv * group + i) * a.n_tokens + tok) * a.d + c];
    const int64_t per = a.n_tokens / max(a.n_seq, int64_t(1));
    const int64_t row = a.packed ? tok * a.out.tok : tok / per * a.out.seq + tok % per * a.out.tok;
    static_cast<T *>(const_cast<void *>(a.out.p))[row + kv * a.out.head + c] = T(s);
}

// One token of every stream: S <- lambda S + k^T v, o = scale q S.  Bound by the
// state's way through memory: 8 dk dv bytes.  X threads of four columns each side by
// side, 256 / X rows at a time.
template <class T, int X> __global__ void __launch_bounds__(256) attend_step(StepArgs a) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
    constexpr int G = 256 / X;
    __shared__ float lq[256], lk[256];
    __shared__ f32x4 part[G][X];
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
    const T *q = static_cast<const T *>(a.q.p) + b * a.q.seq + h / a.q.group * a.q.head;
    const T *k = static_cast<const T *>(a.k.p) + b * a.k.seq + h / a.k.group * a.k.head;
    const T *v = static_cast<const T *>(a.v.p) + b * a.v.seq + h / a.v.group * a.v.head;
    if (threadIdx.x < a.dk) {
        lq[threadIdx.x] = float(q[threadIdx.x]);
        lk[threadIdx.x] = float(k[threadIdx.x]);
    }
    const float lambda = decay(a.log_decay[h], 1);
    f32x4 vv = {0, 0, 0, 0}, sum = {0, 0, 0, 0};
    for (int j = 0; j < have; ++j) vv[j] = float(v[c + j]);
    __syncthreads();
    float *S = a.state + (slot * a.heads + h) * a.dk * a.dv + c;
    if (have == 4) {
#pragma unroll 4
        for (int64_t d = g; d < a.dk; d += G) {
            f32x4 s = *reinterpret_cast<f4 *>(S + d * a.dv);
            s = s * lambda + vv * lk[d];
            *reinterpret_cast<f4 *>(S + d * a.dv) = s;
            sum += s * lq[d];
        }
    } else {
        for (int64_t d = g; d < a.dk; d += G)
            for (int j = 0; j < have; ++j) {
                const float s = S[d * a.dv + j] * lambda + vv[j] * lk[d];
                S[d * a.dv + j] = s;
                sum[j] += s * lq[d];
            }
    }
    part[g][x] = sum;
    __syncthreads();
    if (g) return;
    for (int i = 1; i < G; ++i) sum += part[i][x];
    for (int j = 0; j < have; ++j) o[c + j] = T(sum[j] * a.scale);
}

template <class T, int DT, int STAGE> void launch_general(const AttendArgs &a, hipStream_t stream) {
    const dim3 grid(uint32_t(a.n_segments), uint32_t(a.heads), uint32_t(ceil_div(a.dc, 64)));
    if (a.n_segments > a.n_seq) {
        attend_general<T, DT, STAGE, false><<<grid, 256, 0, stream>>>(a);
        attend_carry<<<dim3(uint32_t(a.n_seq), uint32_t(a.heads), uint32_t(ceil_div(a.da * a.dc, 256))), 256, 0, stream>>>(a);
    }
    attend_general<T, DT, STAGE, true><<<grid, 256, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_attend(int dtype, const AttendArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        if (a.da <= 64) launch_general<T, 4, 64>(a, stream);
        else if (a.da <= 128) launch_general<T, 8, 32>(a, stream);
        else launch_general<T, 16, 16>(a, stream);
        return hipGetLastError();
    });
}

hipError_t launch_fold_heads(int dtype, const FoldHeadsArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        fold_heads<T><<<dim3(uint32_t(ceil_div(a.n_tokens * a.d, 256)), uint32_t(a.heads / a.out.group)), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_step(int dtype, const StepArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        if (a.n_seq * a.heads * ceil_div(a.dv, 128) >= 2 * kCus)
            attend_step<T, 32><<<dim3(uint32_t(a.n_seq), uint32_t(a.heads), uint32_t(ceil_div(a.dv, 128))), 256, 0, stream>>>(a);
        else
            attend_step<T, 8><<<dim3(uint32_t(a.n_seq), uint32_t(a.heads), uint32_t(ceil_div(a.dv, 32))), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
