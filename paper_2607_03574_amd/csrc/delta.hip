// Attention by the gated delta rule: the forward pass, and the step of a single token.  (Formulas: delta_parts.h.)
// Launches: a record for each chunk of 32 tokens and head (the inverse of I + A, and P); where few sequences are long, what
// each segment adds to a state and makes of it, and what enters each; then the walk that leaves the outputs.
#include "delta_walk.h"

namespace ndvm {
namespace ops {
namespace {

template <class T, int DK, Walk WALK> __global__ void __launch_bounds__(256, (kResident<T, DK>)) delta_walk(DeltaArgs a) {
    __shared__ __align__(16) char lds[kWalkLds<T, DK, WALK == kOutputs, kRead<T, WALK>>];
    const uint32_t id = blockIdx.x / uint32_t(a.heads);
    const int64_t h = blockIdx.x - id * uint32_t(a.heads);
    const Piece g = find_piece(a, id, a.seg_len, !a.segments);
    // (what the last segment makes of a state enters none)
    if (g.count == 0 || (WALK == kSums && g.index == g.count - 1)) return;
    walk<T, DK, WALK>(a, lds, g, blockIdx.x, h, int(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64));
}

template <int DK> __global__ void __launch_bounds__(256) delta_carry(DeltaArgs a) {
    __shared__ __align__(16) char lds[kCarryLds<DK>];
    const uint32_t seq = blockIdx.x / uint32_t(a.heads);
    carry<DK, false>(a, lds, seq, blockIdx.x - seq * uint32_t(a.heads), int(blockIdx.y) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64));
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

template <class T> size_t lay_out(DeltaArgs &a, Space s) {
    a.dkp = padded(a.dk);
    a.dvp = padded(a.dv);
    a.record = kRecord<T>;
    if (a.dk % 8) {
        s.take(a.k_rows, a.n_tokens * (a.heads / a.k.group) * a.dkp * int64_t(sizeof(T)));
        s.take(a.q_rows, a.n_tokens * (a.heads / a.k.group) * a.dkp * int64_t(sizeof(T)));
    }
    s.take(a.chunks, piece_ids(a, kDeltaChunk) * a.heads * a.record);
    if (cut(a)) {
        s.take(a.segments, a.n_segments * a.heads * a.dk * a.dv * 4);
        s.take(a.moves, a.n_segments * a.heads * a.dk * a.dkp * 4);
    }
    return s.used + 256;
}

template <class T> void delta(DeltaArgs a, hipStream_t stream) {
    lay_out<T>(a, Space(a.ws));
    pad_rows<T>(a, a.k, a.k_rows, a.dk, stream);
    pad_rows<T>(a, a.q, a.q_rows, a.dk, stream);
    const int64_t pairs = piece_ids(a, kDeltaChunk) * a.heads;
    if (a.n_tokens) delta_prepare<T, false><<<dim3(uint32_t(ceil_div(pairs, 4))), 256, 0, stream>>>(a, pairs);
    with_width(a.dk, [&](auto d) {
        constexpr int DK = decltype(d)::value;
        const auto grid = [&](int64_t ids, int64_t tiles) { return dim3(uint32_t(ids * a.heads), uint32_t(ceil_div(tiles, 4))); };
        const int64_t of_v = ceil_div(a.dv, 16), of_k = ceil_div(a.dk, 16);
        if (a.segments) {
            delta_walk<T, DK, kSums><<<grid(a.n_segments, of_v + of_k), 256, 0, stream>>>(a);
            delta_carry<DK><<<grid(a.n_seq, of_v), 256, 0, stream>>>(a);
        }
        delta_walk<T, DK, kOutputs><<<grid(a.n_segments, of_v), 256, 0, stream>>>(a);
    });
}

}  // namespace

size_t delta_bytes(int dtype, const DeltaArgs &a, bool grad) {
    if (grad) return delta_grad_bytes(dtype, a);
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
