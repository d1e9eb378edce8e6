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
// first launch sums what each segment adds (the first one of a sequence: to what
// the sequence started with), a second one carries states over the segments in
// order, and the last one computes the outputs.  The gradient's three sums are formed
// together where their widths allow it: dq's and dk's segments in one launch (dv starts from dk's,
// transposed), all outputs in another.
// Bound, at heads of 128 in bfloat16, by memory and the vector instructions that split the state and pairs' products
// in two parts: 16 heads x 16384 tokens 115 to 118 us (the segments' sums 33 to 39, carrying 12, outputs 70 to 85: 270 MB
// of inputs and outputs, and as much again of segments' states and second reads, at 4.6 TB/s; with one part, an error of
// sqrt(2) of the result's rounding, 104); gradient of 8 x 2048 tokens, uncut, 205 to 217 us (470 MB needed, 730 moved
// at 3.4 TB/s: a tensor is read by up to three sums; one part: 177).  Half, through registers, 159 us and float 260 at
// the first size.
#include <algorithm>
#include <type_traits>

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
// theirs; the spare ids are segments without tokens (count 0).  seg_len is a power of two
// then, and the 64 lanes of a wave look for the sequence together.
__device__ inline Segment find_segment(const AttendArgs &a, uint32_t id) {
    Segment g;
    const bool cut = a.n_segments > a.n_seq;
    if (!a.offsets) {
        const uint32_t per = uint32_t(a.n_segments) / uint32_t(a.n_seq);
        g.tokens = uint32_t(a.n_tokens) / uint32_t(a.n_seq);
        g.seq = id / per;
        g.index = id % per;
        g.first = g.seq * g.tokens;
        g.count = per;
    } else {
        const auto at = [&](int64_t s) { return min(max(a.offsets[s], int64_t(0)), a.n_tokens); };
        const int shift = 63 - __builtin_clzll(a.seg_len);
        uint32_t lo = id, base = id;
        if (cut) {
            // the last sequence whose ids begin at or before id
            uint32_t hi = uint32_t(a.n_seq);
            lo = base = 0;
            while (hi - lo > 1) {
                const uint32_t step = (hi - lo + 63) / 64, s = lo + (threadIdx.x % 64) * step;
                const uint32_t mine = s < hi ? uint32_t(at(s) >> shift) + s : 0xffffffffu;
                const int n = max(__popcll(__ballot(mine <= id)), 1);
                base = __shfl(mine, n - 1);
                lo += (n - 1) * step;
                hi = min(lo + step, hi);
            }
            if (a.n_seq == 1) base = uint32_t(at(0) >> shift);
            lo = __builtin_amdgcn_readfirstlane(lo);
            base = __builtin_amdgcn_readfirstlane(base);
        }
        g.seq = lo;
        g.index = int64_t(id) - base;
        g.first = at(lo);
        g.tokens = max(at(int64_t(lo) + 1) - g.first, int64_t(0));
        g.count = cut ? max((g.tokens + a.seg_len - 1) >> shift, int64_t(1)) : 1;
    }
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

// The kernel for widths of a and b past 128: float matrix instructions (16 x 16 x 4).  Four waves, 16 columns of c each; chunks of 16 tokens, STAGE
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
    // heads first: workgroups that run together read whole rows of memory between them
    const uint32_t id = blockIdx.x / uint32_t(A.heads);
    const Segment g = find_segment(A, id);
    if (g.count == 0 || (!OUT && g.index == g.count - 1)) return;
    const int64_t h = blockIdx.x - id * uint32_t(A.heads), col0 = int64_t(blockIdx.y) * 64;
    const int l = threadIdx.x % 64, wave = threadIdx.x / 64, lm = l % 16, lg = l / 16;
    const int64_t col = col0 + wave * 16 + lm;
    const float gl = A.log_decay[h];
    if (threadIdx.x < 17) power[threadIdx.x] = decay(gl, threadIdx.x);
    const int e = A.reversed ? 0 : 1;

    f32x4 S[DT];
    const bool carried = OUT && g.index > 0;    // from an earlier segment
    float *mine = A.segments + int64_t(blockIdx.x) * ((A.da * A.dc + 3) / 4 * 4);
    const float *in = carried ? mine : g.index == 0 && A.state_in ? A.state_in + (g.seq * A.heads + h) * A.da * A.dc : nullptr;
    const bool in_transposed = !carried && A.state_transposed;
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
    float *out = !OUT ? mine : g.index == g.count - 1 && A.state_out ? A.state_out + (g.seq * A.heads + h) * A.da * A.dc : nullptr;
    if (!out) return;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t at = place(t, r, OUT && A.state_transposed);
            if (at >= 0) out[at] = S[t][r];
        }
}

// The kernel for widths of a and b up to 128: bf16 matrix instructions (16 x 16 x 32), chunks
// of 32 tokens.  Four waves, 16 NT columns of c each; all share the chunk's rows of a,
// b and c in LDS.
//  - P^T and S are used from the accumulators as above.  Rows of S are numbered so
//    that the eight a lane holds in a pair of tiles are eight consecutive widths,
//    which one 16-byte read of a matches; columns of c so that a lane's results
//    for a token are consecutive.
//  - b^T and c^T come from LDS through the transposing reads (four tokens of a
//    column each), tokens in the order that P^T has them.
//  - A float is multiplied as bf16 parts, each the next 8 bits of it: half inputs are
//    exactly two, float inputs three.  Parts are cut (the last one is rounded): a second part can be 2^-7 of
//    the value, a third 2^-15, so what is left out of a product is below 2^-21 of it for float (2^-24 on average)
//    and 2^-14 for half, whose results are rounded to 2^-11, and has the product's sign.  The state stays float for every type and takes c times
//    its decay as three parts; what is read from it, and the products of a pair, are two parts
//    (three for float): a 16-bit result then differs from the exact one by its own rounding alone.
// LDS rows lie in granules of 16 bytes, granule i of row r at i ^ swizzle(r): the 16 rows
// that one instruction reads are then in different banks.
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#ifdef __HIP_DEVICE_COMPILE__
__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// Lane 4 r + x of 16 names four values of row r; lane i gets column i of the four rows.
__device__ inline bf16x4 read_transposed(const char *p) {
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(p)));
}
// The upper 8 bits of v's significand.
__device__ inline float upper(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
template <int N> __device__ inline void split(float v, bf16x8 (&to)[N], int at) {
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        const float up = upper(v);
        to[i][at] = bf16(up);
        v -= up;
    }
    to[N - 1][at] = bf16(v);
}
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
template <class T> constexpr int input_parts() { return sizeof(T) == 4 ? 3 : std::is_same<T, f16>::value ? 2 : 1; }

// The segment and head of its set that a workgroup has, and the set: the sets of a segment and head lie eight
// workgroups apart, on the same XCD, since they read the same tensors.  Heads first: workgroups that run
// together read whole rows of memory between them.
__device__ inline uint32_t place_of(const AttendArgs &) { return blockIdx.x; }
__device__ inline uint32_t place_of(const AttendSets &s) { return __builtin_amdgcn_readfirstlane(blockIdx.x / 8 / s.count) * 8 + blockIdx.x % 8; }
__device__ inline const AttendArgs &set_of(const AttendArgs &a) { return a; }
__device__ inline const AttendArgs &set_of(const AttendSets &s) { return s.set[__builtin_amdgcn_readfirstlane(blockIdx.x / 8 % s.count)]; }

// DS: widths of a and b in 32s.  DIRECT (bfloat16): rows are 16-byte granules at 16-byte
// addresses, loaded to LDS directly, two chunks ahead; else through registers, one ahead.
// Args: AttendSets, or AttendArgs of a single set, whose values stay in scalar registers (16384 tokens x 16
// heads of 128 114 us, found by a set's number 116; 12 x 4096 tokens x 16 heads of 64 123 and 139).
// PASSING: the outputs, and a where no other set reads it, which this launch alone touches, are more than the
// last cache should hold next to b and c, which the launch before has read too.
template <class T, int DS, int NT, bool DIRECT, bool OUT, class Args, bool PASSING = false>
__global__ void __launch_bounds__(256, DIRECT && DS == 2 ? 3 : 2) attend_parts(Args args) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr bool MANY = std::is_same<Args, AttendSets>::value;
    constexpr int PARTS = input_parts<T>(), ORDER = PARTS - 1;
    constexpr int HELD = PARTS > 2 ? PARTS : 2;      // parts of the state where it is read, and of a pair's product
    constexpr int N = 32, GA = 4 * DS, GC = 8 * NT;      // tokens of a chunk; granules of a row
    constexpr int BYTES_A = OUT ? N * GA * 16 : 0, BYTES_B = N * GA * 16, BYTES_C = N * GC * 16;      // of a part
    constexpr int BYTES = BYTES_A + BYTES_B + BYTES_C;
    __shared__ __align__(1024) char buffer0[PARTS * BYTES], buffer1[DIRECT ? BYTES : 16], buffer2[DIRECT ? BYTES : 16];
    __shared__ float power[N + 2];      // lambda^n
    const AttendArgs &A = set_of(args);
    const uint32_t place = place_of(args), id = __builtin_amdgcn_readfirstlane(place / uint32_t(A.heads));
    if (MANY && id >= uint32_t(A.n_segments)) return;
    const Segment g = find_segment(A, id);
    if (g.count == 0 || (!OUT && g.index == g.count - 1)) return;
    const int64_t h = place - id * uint32_t(A.heads), col0 = int64_t(blockIdx.y) * 64 * NT;
    const int l = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lm = l % 16, lg = l / 16;
    const float gl = A.log_decay[h];
    const int e = A.reversed ? 0 : 1;

    const auto swizzle = [](int row, int granules) { return granules >= 16 ? row % 4 * 4 + row / 4 % 4 : row % 2 * 4 + row / 2 % 4; };

    // ---- loads: a wave takes 64 granules at a time
    constexpr int LA = N * GA / 256, LC = N * GC / 256, LOADS = (OUT ? 2 : 1) * LA + LC;
    constexpr unsigned kNowhere = 0x80000000u;
    const int len = int(g.len);
    struct Rows {
        int64_t at;         // of the first chunk's row that comes first in memory
        int64_t step;       // from a chunk's to the next chunk's, over the chunk's tokens
    };
    const auto rows_of = [&](const Heads &H) {
        const int64_t t = A.reversed ? g.tokens - g.begin - N : g.begin;
        const int64_t row = A.offsets ? (g.first + t) * H.tok : g.seq * H.seq + t * H.tok;
        return Rows{row + h / H.group * H.head, A.reversed ? -H.tok : H.tok};
    };
    const Rows ra = rows_of(A.a), rb = rows_of(A.b), rc = rows_of(A.c), ro = rows_of(A.out);
    using std::integral_constant;
    // a wave's loads of `count` granules a lane: where they lie in the chunk's rows
    const auto each = [&](const Heads &H, const Rows &R, auto granules_c, auto count_c, int64_t c0, int64_t width, int base, auto f) __attribute__((always_inline)) {
        constexpr int granules = decltype(granules_c)::value, count = decltype(count_c)::value;
        const T *from = static_cast<const T *>(H.p) + R.at + base * R.step + c0;
#pragma unroll
        for (int i = 0; i < count; ++i) {
            const int at = (wave + 4 * i) * 64 + l, row = at / granules, c = (at % granules ^ swizzle(row, granules)) * 8;
            f(i, from, A.reversed ? N - 1 - row : row, c, base + row < len && c0 + c < width);
        }
    };
    const integral_constant<int, GA> granules_a;
    const integral_constant<int, GC> granules_c;
    const integral_constant<int, LA> count_a;
    const integral_constant<int, LC> count_c;
    // To LDS directly: where the next chunk's rows begin, and a lane's first granule in them; the
    // others are 256 / granules rows apart (a multiple of 16: the same swizzle), counted from the end if reversed.
    struct Stream {
        const T *next;
        int64_t step;
        unsigned at, apart;
    };
    const bool reversed = A.reversed;
    const auto stream = [&](const Heads &H, const Rows &R, auto granules, auto count, int64_t c0, int64_t width) {
        constexpr int rows = 256 / granules.value;
        static_assert(rows % 16 == 0 && rows * count.value == N, "");
        const int first = (wave * 64 + l) / granules.value, c = ((wave * 64 + l) % granules.value ^ swizzle(first, granules.value)) * 8;
        const int row = reversed ? N - 1 - first - (count.value - 1) * rows : first;
        return Stream{static_cast<const T *>(H.p) + R.at + c0, N * R.step, c0 + c < width ? unsigned(row) * unsigned(H.tok * 2) + c * 2 : kNowhere,
                      unsigned(rows * H.tok * 2)};
    };
    Stream sa, sb = stream(A.b, rb, granules_a, count_a, 0, A.da), sc = stream(A.c, rc, granules_c, count_c, col0, A.dc);
    if (OUT) sa = stream(A.a, ra, granules_a, count_a, 0, A.da);
    int left = len;         // tokens from the next chunk's first on
    // always LOADS loads a wave (those past the segment's end fetch nothing)
    const auto load = [&](Stream &s, char *to, auto granules, auto count, auto passing) __attribute__((always_inline)) {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(s.next), 0, 0x7fffffff, 0x00020000);
        const int first = (wave * 64 + l) / granules.value;
#pragma unroll
        for (int i = 0; i < count.value; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(to + (wave + 4 * i) * 1024), 16,
                                                     first < left - i * (256 / granules.value) ? s.at : kNowhere,
                                                     __builtin_amdgcn_readfirstlane((reversed ? count.value - 1 - i : i) * s.apart), 0, passing.value ? 2 : 0);
        s.next += s.step;
    };
    const auto load_chunk = [&](char *to) __attribute__((always_inline)) {
        const std::false_type stays;
        if (OUT) load(sa, to, granules_a, count_a, integral_constant<bool, PASSING && !MANY>());
        load(sb, to + BYTES_A, granules_a, count_a, stays);
        load(sc, to + BYTES_A + BYTES_B, granules_c, count_c, stays);
        left -= N;
    };
    // Through registers: eight values a granule, split on their way to LDS.
    constexpr int V = kVec<T>;
    vec<T> held[LOADS][8 / V];
    const auto fetch = [&](int base) __attribute__((always_inline)) {
        int k = 0;
        const auto one = [&](const Heads &H, int64_t c0, int64_t width) {
            return [&, c0, width](int i, const T *from, int row, int c, bool there) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 8 / V; ++j) {
                    held[k + i][j] = T(0.0f);
                    if (there && c0 + c + j * V < width) held[k + i][j] = load_vec(from + row * H.tok + c + j * V, width - c0 - c - j * V);
                }
            };
        };
        if (OUT) {
            each(A.a, ra, granules_a, count_a, 0, A.da, base, one(A.a, 0, A.da));
            k += LA;
        }
        each(A.b, rb, granules_a, count_a, 0, A.da, base, one(A.b, 0, A.da));
        k += LA;
        each(A.c, rc, granules_c, count_c, col0, A.dc, base, one(A.c, col0, A.dc));
    };
    const auto put = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int of_a = OUT ? LA : 0, i = k < of_a ? k : k < of_a + LA ? k - of_a : k - of_a - LA;
            const int tile = k < of_a ? 0 : k < of_a + LA ? PARTS * BYTES_A : PARTS * (BYTES_A + BYTES_B);
            const int part = k < of_a ? BYTES_A : k < of_a + LA ? BYTES_B : BYTES_C;
            bf16x8 parts[PARTS];
#pragma unroll
            for (int j = 0; j < 8; ++j) split(float(held[k][j / V][j % V]), parts, j);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8 *>(buffer0 + tile + q * part + (wave + 4 * i) * 1024 + l * 16) = parts[q];
        }
    };

    if constexpr (DIRECT) {
        load_chunk(buffer0);
        load_chunk(buffer1);
    } else {
        fetch(0);
    }
    if (threadIdx.x < N + 2) power[threadIdx.x] = decay(gl, threadIdx.x);

    // ---- the state: tile 2 s + u, register r of lane l: width 32 s + 8 (l / 16) + 4 u + r, and
    // column (NT = 2) 8 (l % 16 / 4) + 4 nt + l % 4 of the wave's
    const auto column = [&](int nt) { return col0 + wave * 16 * NT + (NT == 2 ? lm / 4 * 8 + nt * 4 + lm % 4 : lm); };
    // A segment's state lies in memory as in the registers.
    f32x4 S[2 * DS][NT];
    f32x4 *mine = reinterpret_cast<f32x4 *>(A.segments) + ((int64_t(place) * gridDim.y + blockIdx.y) * 4 + wave) * (2 * DS * NT * 64) + l;
    if (OUT && g.index > 0 && A.shared_segments) {
        // the states as the transposed sum left them: its tiles, waves and lanes by (column, width)
        const int nt_of = A.da <= 64 ? 1 : 2, tiles = (A.dc <= 64 ? 4 : 8) * nt_of;
        const float *theirs = A.segments + int64_t(place) * (4 * 2 * DS * NT * 256);
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = t / 2 * 32 + lg * 8 + t % 2 * 4 + r, c = int(column(nt));
                    const int in = d % (16 * nt_of), lane = c % 32 / 8 * 16 + (nt_of == 2 ? in / 8 * 4 + in % 4 : in);
                    const int tile = (c / 32 * 2 + c % 8 / 4) * nt_of + (nt_of == 2 ? in / 4 % 2 : 0);
                    S[t][nt][r] = theirs[((d / (16 * nt_of) * tiles + tile) * 64 + lane) * 4 + c % 4];
                }
    } else if (OUT && g.index > 0) {
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[t][nt] = mine[(t * NT + nt) * 64];
    } else {
        const float *in = g.index == 0 && A.state_in ? A.state_in + (g.seq * A.heads + h) * A.da * A.dc : nullptr;
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[t][nt] = 0;
        if (in) {
            const int64_t step_d = A.state_transposed ? 1 : A.dc, step_c = A.state_transposed ? A.da : 1;
#pragma unroll
            for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int64_t d = t / 2 * 32 + lg * 8 + t % 2 * 4 + r, c = column(nt);
                        const bool there = d < A.da && c < A.dc;
                        const float v = in[there ? d * step_d + c * step_c : 0];
                        S[t][nt][r] = there ? v : 0.0f;
                    }
        }
    }

    __syncthreads();

    // ---- decays of a chunk: of a pair (row j of P^T, column i; the same tile, the next one), of what is
    // read from the state, of what it takes from a full chunk
    float w0[4], w1[4], rise[2], fall[8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int far = lm - 4 * lg - r;
        w0[r] = far >= 0 ? A.scale_pair * power[far] : 0.0f;
        w1[r] = A.scale_pair * power[far + 16];
        fall[r] = A.scale_add * power[N - e - 4 * lg - r];
        fall[4 + r] = A.scale_add * power[N - e - 16 - 4 * lg - r];
    }
#pragma unroll
    for (int it = 0; it < 2; ++it) rise[it] = A.scale_read * power[16 * it + lm + e];
    float whole = power[N];

    // byte of a lane's reads: 16 bytes of row lm, granule 4 s + lg; and transposed, four values of row
    // 4 lg + (l / 4 % 4): granule 4 s + l % 4 of b, half u; of c the wave's columns 4 (l % 4) on
    const int tr_row = 4 * lg + l / 4 % 4;
    const auto row_at = [&](int row16, int s) { return ((row16 * 16 + lm) * GA + (((4 * s + lg)) ^ swizzle(lm, GA))) * 16; };
    const auto b_at = [&](int row16, int s, int u) { return ((row16 * 16 + tr_row) * GA + ((4 * s + l % 4) ^ swizzle(tr_row, GA))) * 16 + u * 8; };
    const auto c_at = [&](int row16, int nt) {
        const int gr = NT == 2 ? wave * 4 + l % 4 : wave * 2 + l % 4 / 2, half = NT == 2 ? nt : l % 2;
        return ((row16 * 16 + tr_row) * GC + (gr ^ swizzle(tr_row, GC))) * 16 + half * 8;
    };

    // A chunk's results are stored during the next one, ahead of its loads: the last LOADS
    // of a wave's memory operations are then the loads of the chunk after.
    f32x4 O[2][NT];
    const auto store = [&](int base) __attribute__((always_inline)) {
        // lane l: token lm of the tile, columns 4 NT lg on
        const int c = wave * 16 * NT + lg * 4 * NT;
        constexpr int W = 4 * NT;
        const int have = int(min(A.dc - col0 - c, int64_t(W)));
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const int i = 16 * it + lm;
            if (base + i >= len || have <= 0) continue;
            const int64_t at = ro.at + base * ro.step + (A.reversed ? N - 1 - i : i) * A.out.tok + col0 + c;
            if (A.out_f32) {
                typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
                float *to = static_cast<float *>(const_cast<void *>(A.out.p)) + at;
                if (have == W) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f4 *>(to + 4 * nt) = O[it][nt];
                } else {
#pragma unroll
                    for (int r = 0; r < W; ++r)
                        if (r < have) to[r] = O[it][r / 4][r % 4];
                }
            } else {
                typedef T out_t __attribute__((ext_vector_type(W), aligned(sizeof(T))));
                T *to = static_cast<T *>(const_cast<void *>(A.out.p)) + at;
                out_t v;
#pragma unroll
                for (int r = 0; r < W; ++r) v[r] = T(O[it][r / 4][r % 4]);
                if (have == W) {
                    if (PASSING) __builtin_nontemporal_store(v, reinterpret_cast<out_t *>(to));
                    else *reinterpret_cast<out_t *>(to) = v;
                } else {
#pragma unroll
                    for (int r = 0; r < W; ++r)
                        if (r < have) to[r] = v[r];
                }
            }
        }
    };

    const auto compute = [&](const char *now, int base) __attribute__((always_inline)) {
        const int n = min(len - base, N);
        const char *la = now, *lb = now + PARTS * BYTES_A, *lc = now + PARTS * (BYTES_A + BYTES_B);
        const auto pair = [](const char *p, const char *q) { return __builtin_shufflevector(read_transposed(p), read_transposed(q), 0, 1, 2, 3, 4, 5, 6, 7); };
        bf16x8 fc[NT][PARTS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int q = 0; q < PARTS; ++q) fc[nt][q] = pair(lc + q * BYTES_C + c_at(0, nt), lc + q * BYTES_C + c_at(1, nt));
        if (OUT) {
            f32x4 P00 = 0, P01 = 0, P11 = 0;
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[it][nt] = 0;
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                bf16x8 a0[PARTS], a1[PARTS], b0[PARTS], b1[PARTS];
#pragma unroll
                for (int q = 0; q < PARTS; ++q) {
                    a0[q] = *reinterpret_cast<const bf16x8 *>(la + q * BYTES_A + row_at(0, s));
                    a1[q] = *reinterpret_cast<const bf16x8 *>(la + q * BYTES_A + row_at(1, s));
                    b0[q] = *reinterpret_cast<const bf16x8 *>(lb + q * BYTES_B + row_at(0, s));
                    b1[q] = *reinterpret_cast<const bf16x8 *>(lb + q * BYTES_B + row_at(1, s));
                }
                P00 = multiply<ORDER>(b0, a0, P00);
                P01 = multiply<ORDER>(b0, a1, P01);
                P11 = multiply<ORDER>(b1, a1, P11);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    bf16x8 state[HELD];
#pragma unroll
                    for (int r = 0; r < 8; ++r) split(S[2 * s + r / 4][nt][r % 4], state, r);
                    O[0][nt] = multiply<HELD - 1>(state, a0, O[0][nt]);
                    O[1][nt] = multiply<HELD - 1>(state, a1, O[1][nt]);
                }
            }
            bf16x8 p[2][HELD];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                // what is masked is replaced, not multiplied
                const bool seen = lm >= 4 * lg + r;
                split(seen ? P00[r] * w0[r] : 0.0f, p[0], r);
                split(0.0f, p[0], 4 + r);
                split(P01[r] * w1[r], p[1], r);
                split(seen ? P11[r] * w0[r] : 0.0f, p[1], 4 + r);
            }
            f32x4 near[2][NT];
            float odd = 0;      // NaN if a sum is not finite
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    near[it][nt] = multiply<HELD - 1>(fc[nt], p[it], f32x4(0.0f));
#pragma unroll
                    for (int r = 0; r < 4; ++r) odd = __builtin_fmaf(near[it][nt][r], 0.0f, odd);
                }
            if (__builtin_expect(__any(odd != 0.0f), 0)) {
                // a value of c may not be finite, and 0 times it is NaN: add the terms up to i alone
                for (int it = 0; it < 2; ++it) {
                    f32x4 sum[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) sum[nt] = 0;
#pragma unroll 1
                    for (int j = 0; j < N; ++j) {
                        const int at = j / 16 * 2 + j % 4 / 2;
                        float pij = 0;
#pragma unroll
                        for (int q = 0; q < HELD; ++q) {
                            typedef int i32x4 __attribute__((ext_vector_type(4)));
                            const i32x4 packed = __builtin_bit_cast(i32x4, it ? p[1][q] : p[0][q]);
                            const int two = __shfl(at == 0 ? packed[0] : at == 1 ? packed[1] : at == 2 ? packed[2] : packed[3], lm + 16 * (j % 16 / 4));
                            pij += __int_as_float(j % 2 ? two & 0xffff0000 : two << 16);
                        }
                        if (j > 16 * it + lm) continue;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const int c = wave * 16 * NT + (NT == 2 ? lg * 8 + nt * 4 + r : lg * 4 + r);
                                float cj = 0;
#pragma unroll
                                for (int q = 0; q < PARTS; ++q)
                                    cj += float(*reinterpret_cast<const bf16 *>(lc + q * BYTES_C + (j * GC + (c / 8 ^ swizzle(j, GC))) * 16 + c % 8 * 2));
                                sum[nt][r] += pij * cj;
                            }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) (it ? near[1][nt] : near[0][nt]) = sum[nt];
                }
            }
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) O[it][nt] = O[it][nt] * rise[it] + near[it][nt];
        }
        if (n < N) {        // the last chunk: decays to its own end; beyond it c is 0
            whole = power[n];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int to_end = n - e - (r / 4 * 16 + 4 * lg + r % 4);
                fall[r] = to_end >= 0 ? A.scale_add * power[to_end] : 0.0f;
            }
        }
        bf16x8 add[NT][3];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                float c = float(fc[nt][0][r]);
#pragma unroll
                for (int q = 1; q < PARTS; ++q) c += float(fc[nt][q][r]);
                split(c * fall[r], add[nt], r);
            }
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t) {
            bf16x8 fb[PARTS];
#pragma unroll
            for (int q = 0; q < PARTS; ++q) fb[q] = pair(lb + q * BYTES_B + b_at(0, t / 2, t % 2), lb + q * BYTES_B + b_at(1, t / 2, t % 2));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[t][nt] = multiply<2>(fb, add[nt], S[t][nt] * whole);
        }
    };
    if constexpr (DIRECT) {
        const auto chunk = [&](char *now, char *next, int base) __attribute__((always_inline)) {
            // this wave's loads of the chunk have landed (the next chunk's may not have) and its reads of the
            // last one are done; after the barrier everybody's
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(LOADS | 0x0070);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (OUT && base > 0) store(base - N);
            load_chunk(next);
            compute(now, base);
        };
        if (len > 0) {
            int base = 0;
            for (;;) {
                chunk(buffer0, buffer2, base);
                if ((base += N) >= len) break;
                chunk(buffer1, buffer0, base);
                if ((base += N) >= len) break;
                chunk(buffer2, buffer1, base);
                if ((base += N) >= len) break;
            }
            if (OUT) store(base - N);
        }
        // the loads past the end fetch nothing, but write zeros to LDS, which has to be this workgroup's still
        __builtin_amdgcn_s_waitcnt(0x0f70);
    } else {
        // The widest float tiles have no registers to hold the next chunk in meanwhile: the other workgroup on
        // the compute unit covers its loads (16384 tokens x 16 heads of 128: 260 us; held and spilled, 330).
        constexpr bool AHEAD = !(PARTS == 3 && DS == 4 && NT == 2);
        for (int base = 0; base < len; base += N) {
            __syncthreads();
            put();
            __syncthreads();
            if (AHEAD) fetch(base + N);
            compute(buffer0, base);
            if (!AHEAD) fetch(base + N);
            if (OUT) store(base);
        }
    }
    if (!OUT) {
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mine[(t * NT + nt) * 64] = S[t][nt];
    } else if (g.index == g.count - 1 && A.state_out) {
        float *out = A.state_out + (g.seq * A.heads + h) * A.da * A.dc;
        const int64_t step_d = A.state_transposed ? 1 : A.dc, step_c = A.state_transposed ? A.da : 1;
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t d = t / 2 * 32 + lg * 8 + t % 2 * 4 + r, c = column(nt);
                    if (d < A.da && c < A.dc) out[d * step_d + c * step_c] = S[t][nt][r];
                }
    }
#endif
}

// States over the segments of a sequence, in order: what each adds is replaced
// by what enters it (the first one's stays).  A thread four values of the state,
// wherever they lie; U segments' are read at once.  size: a multiple of 4.
__device__ inline const AttendArgs &carried_set(const AttendArgs &a, uint32_t) { return a; }
__device__ inline const AttendArgs &carried_set(const AttendSets &s, uint32_t tiles) { return s.set[__builtin_amdgcn_readfirstlane(blockIdx.z / tiles)]; }
template <class Args> __global__ void __launch_bounds__(256) attend_carry(Args args, uint32_t size) {
    constexpr int U = 8;
    const uint32_t tiles = (size + 1023) / 1024, at = blockIdx.z % tiles * 256 + threadIdx.x;
    const AttendArgs &A = carried_set(args, tiles);
    const uint32_t seq = blockIdx.x, h = blockIdx.y;
    uint32_t id, count;
    if (!A.offsets) {
        count = uint32_t(A.n_segments) / uint32_t(A.n_seq);
        id = seq * count;
    } else {
        const int shift = 63 - __builtin_clzll(A.seg_len);
        const int64_t lo = min(max(A.offsets[seq], int64_t(0)), A.n_tokens);
        const int64_t hi = min(max(A.offsets[seq + 1], int64_t(0)), A.n_tokens);
        id = uint32_t(lo >> shift) + seq;
        count = uint32_t((max(hi - lo, int64_t(0)) + A.seg_len - 1) >> shift);
        count = min(count, uint32_t(A.n_segments) - id);
    }
    if (count < 2 || at >= size / 4) return;
    const float whole = decay(A.log_decay[h], A.seg_len);
    const int64_t step = A.heads * int64_t(size / 4);
    f32x4 *p = reinterpret_cast<f32x4 *>(A.segments) + (int64_t(id) * A.heads + h) * (size / 4) + at;
    f32x4 cur = *p;
    for (uint32_t i = 1; i < count; i += U) {
        f32x4 add[U];
#pragma unroll
        for (int u = 0; u < U; ++u) add[u] = i + u + 1 < count ? p[(i + u) * step] : f32x4(0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u < count) {
                p[(i + u) * step] = cur;
                cur = whole * cur + add[u];
            }
    }
}

template <class T> __global__ void __launch_bounds__(256) fold_heads(FoldHeadsSets sets) {
    const FoldHeadsArgs &a = sets.set[blockIdx.z];
    const int group = a.out.group;
    const int64_t per = a.n_tokens / max(a.n_seq, int64_t(1));
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < a.n_tokens * a.d; at += int64_t(gridDim.x) * 256) {
        const int64_t tok = at / a.d, c = at % a.d, kv = blockIdx.y;
        float s = 0;
        for (int i = 0; i < group; ++i) s += a.part[((kv * group + i) * a.n_tokens + tok) * a.d + c];
        const int64_t row = a.packed ? tok * a.out.tok : tok / per * a.out.seq + tok % per * a.out.tok;
        static_cast<T *>(const_cast<void *>(a.out.p))[row + kv * a.out.head + c] = T(s);
    }
}

// One token of every stream: S <- lambda S + k^T v, o = scale q S.  Bound by the
// state's way through memory: 8 dk dv bytes (192 streams x 16 heads of 128 x 128: 79 us, 5.1 TB/s).  X
// threads of four columns each side by side, 256 / X rows at a time.
template <class T, int X, bool PASSING> __global__ void __launch_bounds__(256) attend_step(StepArgs a) {
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
            f4 *at = reinterpret_cast<f4 *>(S + d * a.dv);
            f32x4 s = PASSING ? __builtin_nontemporal_load(at) : *at;
            s = s * lambda + vv * lk[d];
            if (PASSING) __builtin_nontemporal_store(f4(s), at);
            else *at = s;
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

void launch_carry(const AttendSets &s, int64_t size, hipStream_t stream) {
    const AttendArgs &a = s.set[0];
    const dim3 grid(uint32_t(a.n_seq), uint32_t(a.heads), uint32_t(ceil_div(size, 1024) * s.count));
    if (s.count == 1) attend_carry<<<grid, 256, 0, stream>>>(a, uint32_t(size));
    else attend_carry<<<grid, 256, 0, stream>>>(s, uint32_t(size));
}

template <class T, bool OUT> void launch_general(const AttendArgs &a, hipStream_t stream) {
    attend_general<T, 16, 16, OUT><<<dim3(uint32_t(a.n_segments * a.heads), uint32_t(ceil_div(a.dc, 64))), 256, 0, stream>>>(a);
}

template <int NT> dim3 parts_grid(const AttendSets &s) {
    const int64_t n = s.set[0].n_segments * s.set[0].heads;
    return dim3(uint32_t(s.count == 1 ? n : ceil_div(n, 8) * 8 * s.count), uint32_t(ceil_div(s.set[0].dc, 64 * NT)));
}
template <class T, int DS, int NT, bool DIRECT, bool OUT, bool PASSING> void launch_parts(const AttendSets &s, hipStream_t stream) {
    if (s.count == 1) attend_parts<T, DS, NT, DIRECT, OUT, AttendArgs, PASSING><<<parts_grid<NT>(s), 256, 0, stream>>>(s.set[0]);
    else attend_parts<T, DS, NT, DIRECT, OUT, AttendSets, PASSING><<<parts_grid<NT>(s), 256, 0, stream>>>(s);
}

// Whether rows can be loaded to LDS directly: whole granules at 16-byte addresses, and
// offsets inside a chunk that 31 bits hold.
bool direct(const AttendArgs &a, const Heads &h, int64_t width) {
    return reinterpret_cast<uintptr_t>(h.p) % 16 == 0 && h.tok % 8 == 0 && h.head % 8 == 0 && (a.offsets || h.seq % 8 == 0) && width % 8 == 0 && h.tok < (1 << 24);
}

// Calls f with the sizes that the kernel is built for.
template <class T, class F> void with_parts(const AttendArgs &a, F f) {
    using std::integral_constant;
    const auto sized = [&](auto d) {
        const integral_constant<int, 1> one;
        const integral_constant<int, 2> two;
        const integral_constant<int, 4> four;
        if (a.da <= 64 && a.dc <= 64) f(two, one, d);
        else if (a.da <= 64) f(two, two, d);
        else if (a.dc <= 64) f(four, one, d);
        else f(four, two, d);
    };
    if constexpr (std::is_same<T, bf16>::value)
        if (direct(a, a.a, a.da) && direct(a, a.b, a.da) && direct(a, a.c, a.dc)) return sized(std::true_type());
    sized(std::false_type());
}

// Whether a launch can form the sets that it has, and another one.
template <class T> bool together(const AttendSets &s, const AttendArgs &b) {
    const AttendArgs &a = s.set[0];
    if (ceil_div(b.n_segments * b.heads, 8) * 8 * (s.count + 1) > kMostGroups) return false;
    const auto kind = [](const AttendArgs &x) {
        int64_t k = 0;
        with_parts<T>(x, [&](auto ds, auto nt, auto d) { k = (ds.value * 4 + nt.value) * 2 + d.value; });
        return k * 8 + ceil_div(x.dc, 64);
    };
    return kind(a) == kind(b);
}

}  // namespace

// How sequences are cut: into segments for two workgroups a compute unit (16 heads x
// 16384 tokens of 128: 108 us; for one, 113; for four, whose states are twice the traffic, 126),
// but of at least 128 tokens, a few chunks' work (16 heads x 2048 tokens: 31 us; of 64, 40; of
// 256, 36), or 64 in float, whose chunks take three times as long (2 x 1000 tokens, 4 heads of
// 100: 36 us; of 128, 48).  A packed batch is cut wherever a sequence may be longer than that: its
// longest sequence is not known here, and would be walked by one workgroup while the others
// are done.
// Sequences of equal length are left whole where they fill three quarters of the compute units: one walk of
// longer chains takes less than three launches and the states' way through memory.  Measured at 128 to 576
// workgroups of 16 heads and 256 to 16384 tokens, us cut / whole:
//   heads of 128   12 x 1024 tokens   12 x 16384       gradient of 4 x 4096   of 8 x 2048   of 3 x 4096, too few
//   bfloat16          96 /  65       1170 /  968         288 / 258             239 / 210      224 / 258
//   half             143 / 119       1949 / 1837         484 / 461             385 / 340      364 / 458
//   float            227 / 210       3441 / 3156         769 / 785             622 / 573      585 / 773
// Heads of up to 64 in 16 bits have shorter chunks, and up to three workgroups on a compute unit hide each other's
// latency: past 1536 tokens the gradient, and half's forward pass, gain from pieces (gradient of 4 x 4096: bfloat16
// cut 119 us, whole 139, half 208 and 246; forward of 12 x 4096: half 200 and 229, but bfloat16 142 and 125; gradient of
// 4 x 1024: 44 and 40).
Cut attend_cut(int dtype, int64_t n_seq, int64_t n_tokens, int64_t heads, int64_t da, int64_t dc, bool packed, int sets) {
    const int64_t least = dtype == NDVM_F32 ? 64 : 128;
    const bool matrix = da <= kMostPartsDim;
    const int64_t cols = matrix && dc > 64 ? 128 : 64;
    Cut c;
    c.state = matrix ? (da <= 64 ? 64 : 128) * ceil_div(dc, cols) * cols : ceil_div(da * dc, 4) * 4;
    const int64_t longest = packed || n_seq == 0 ? n_tokens : n_tokens / n_seq;
    const int64_t want = std::max<int64_t>(1, 2 * kCus / (heads * ceil_div(dc, cols) * sets));
    int64_t len = std::max<int64_t>(least, n_tokens / want);
    len = ceil_div(len, kSegStep) * kSegStep;
    const int64_t groups = n_seq * heads * ceil_div(dc, cols) * sets;
    const bool short_chunks = std::max(da, dc) <= 64 && (dtype == NDVM_F16 || (dtype == NDVM_BF16 && sets > 1));
    const bool whole = !packed && (n_seq >= want || (matrix && groups >= kCus * 3 / 4 && (!short_chunks || longest <= 1536)));
    if (len >= longest || whole) {
        c.seg_len = std::max<int64_t>(longest, 1);
        c.n_segments = n_seq;
    } else if (packed) {
        c.seg_len = least;
        while (c.seg_len * 2 <= len) c.seg_len *= 2;
        c.n_segments = n_tokens / c.seg_len + n_seq;
    } else {
        c.seg_len = ceil_div(ceil_div(longest, ceil_div(longest, len)), kSegStep) * kSegStep;
        c.n_segments = n_seq * ceil_div(longest, c.seg_len);
    }
    return c;
}

hipError_t launch_attend_segments(int dtype, const AttendSets &s, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const AttendArgs &a = s.set[0];
        if (a.n_segments <= a.n_seq) return hipSuccess;
        if (a.da > kMostPartsDim) {
            for (int i = 0; i < s.count; ++i) launch_general<T, false>(s.set[i], stream);
            launch_carry(s, ceil_div(a.da * a.dc, 4) * 4, stream);
            return hipGetLastError();
        }
        AttendSets run{};
        const auto launch = [&]() {
            with_parts<T>(run.set[0], [&](auto ds, auto nt, auto d) {
                launch_parts<T, ds.value, nt.value, d.value, false, false>(run, stream);
            });
            run.count = 0;
        };
        for (int i = 0; i < s.count; ++i) {
            if (run.count && !together<T>(run, s.set[i])) launch();
            run.set[run.count++] = s.set[i];
        }
        launch();
        const int64_t cols = a.dc <= 64 ? 64 : ceil_div(a.dc, 128) * 128;
        launch_carry(s, (a.da <= 64 ? 64 : 128) * cols, stream);
        return hipGetLastError();
    });
}

hipError_t launch_attend(int dtype, const AttendSets &s, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        bool done[kMostSets] = {};
        for (int i = 0; i < s.count; ++i) {
            if (done[i]) continue;
            if (s.set[i].da > kMostPartsDim) {
                launch_general<T, true>(s.set[i], stream);
                continue;
            }
            AttendSets run{};
            for (int j = i; j < s.count; ++j) {
                if (done[j] || s.set[j].da > kMostPartsDim || (run.count && !together<T>(run, s.set[j]))) continue;
                done[j] = true;
                run.set[run.count++] = s.set[j];
            }
            with_parts<T>(run.set[0], [&](auto ds, auto nt, auto d) {
                const AttendArgs &a = run.set[0];
                // 16 heads of 128: 16 x 2048 tokens 134 us, as if all data stayed 143; gradient of 16384 tokens 257 and 266
                const bool passing = d.value && a.n_tokens * a.heads * (a.da + a.dc) * 4 >= kPassingTraffic;
                if (passing) launch_parts<T, ds.value, nt.value, d.value, true, d.value>(run, stream);
                else launch_parts<T, ds.value, nt.value, d.value, true, false>(run, stream);
            });
        }
        return hipGetLastError();
    });
}

hipError_t launch_fold_heads(int dtype, const FoldHeadsSets &s, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const FoldHeadsArgs &a = s.set[0];
        const int64_t most = a.n_tokens * std::max(a.d, s.set[s.count - 1].d);
        fold_heads<T><<<dim3(uint32_t(std::min(ceil_div(most, 256), kMostGroups)), uint32_t(a.heads / a.out.group), uint32_t(s.count)), 256, 0, stream>>>(s);
        return hipGetLastError();
    });
}

hipError_t launch_step(int dtype, const StepArgs &a, hipStream_t stream) {
    return with_type(dtype, [&](auto zero) {
        typedef decltype(zero) T;
        const int64_t narrow = ceil_div(a.dv, 32), wide = ceil_div(a.dv, 128);
        const auto grid = [&](int64_t tiles) { return dim3(uint32_t(a.n_seq), uint32_t(a.heads), uint32_t(tiles)); };
        // states that do not stay in the last cache until the next token (16 heads of 128 x 128: 192 streams 79 us,
        // as if they stayed 87; 96 streams, which do stay, 33, as if they passed 44)
        if (a.n_seq * a.heads * a.dk * a.dv * 4 >= kPassingStates) attend_step<T, 32, true><<<grid(wide), 256, 0, stream>>>(a);
        else if (a.n_seq * a.heads * wide >= 2 * kCus) attend_step<T, 32, false><<<grid(wide), 256, 0, stream>>>(a);
        else attend_step<T, 8, false><<<grid(narrow), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

}  // namespace ops
}  // namespace ndvm
