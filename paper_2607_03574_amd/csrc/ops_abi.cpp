// C entry points of the encoder operators: every argument is checked before
// anything is enqueued; exceptions become status codes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <new>

#include "common.h"
#include "ops.h"

using namespace ndvm;
using namespace ndvm::ops;

namespace {

template <class F> ndvm_status guarded(F f) {
    try {
        return f();
    } catch (const std::bad_alloc &) {
        set_error("out of host memory");
        return NDVM_E_NOMEM;
    } catch (const std::exception &e) {
        set_error(std::string("internal error: ") + e.what());
        return NDVM_E_INTERNAL;
    }
}

ndvm_status fail(ndvm_status st, const char *who, const char *what) {
    set_error(std::string(who) + ": " + what);
    return st;
}
ndvm_status bad(const char *who, const char *what) { return fail(NDVM_E_ARG, who, what); }

ndvm_status launched(const char *who, hipError_t e) {
    if (e == hipSuccess) return NDVM_OK;
    set_error(std::string(who) + ": launch failed: " + hipGetErrorString(e));
    return NDVM_E_DEVICE;
}

bool known_type(int dtype) { return dtype == NDVM_F32 || dtype == NDVM_BF16 || dtype == NDVM_F16; }

// Products of sizes that a 64-bit address can hold.
constexpr int64_t kMostElements = int64_t(1) << 46;
bool fits(int64_t a, int64_t b) { return a == 0 || b == 0 || a <= kMostElements / b; }
bool fits(int64_t a, int64_t b, int64_t c) { return fits(a, b) && fits(a * b, c); }

// ---- linear attention
Cut cut_of(const ndvm_attention_shape *s, bool packed, int64_t da, int64_t dc, int sets = 1) {
    return attend_cut(s->dtype, s->n_seq, s->n_tokens, s->heads, da, dc, packed, sets);
}

// The gradient's three sums: of widths up to 128 they are cut alike and formed together, those of dq and dk in one
// launch, with dv where its widths have the same kernel; dk and dv start from the same segments' sums.
bool grad_together(const ndvm_attention_shape *s) { return std::max(s->dk, s->dv) <= kMostPartsDim; }
Cut grad_cut(const ndvm_attention_shape *s, bool packed) {
    return cut_of(s, packed, s->dk, s->dv, (s->dk <= 64) == (s->dv <= 64) ? 3 : 2);
}

ndvm_status check_shape(const char *who, const ndvm_attention_shape *s, bool tokens, bool packed) {
    if (!s) return bad(who, "null shape");
    if (!known_type(s->dtype)) return bad(who, "unknown type");
    if (s->n_seq < 0 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads || s->dk < 1 || s->dv < 1)
        return bad(who, "bad size, or heads that are no multiple of kv_heads");
    if (s->heads > kMostHeads || s->dk > kMostHeadDim || s->dv > kMostHeadDim)
        return fail(NDVM_E_UNSUPPORTED, who, "more than 65,535 heads, or a head wider than 256");
    if (!std::isfinite(s->scale)) return bad(who, "scale is not finite");
    if (s->n_seq > kMostGroups || !fits(s->n_seq, s->heads, s->dk * s->dv)) return fail(NDVM_E_UNSUPPORTED, who, "too many sequences");
    if (!tokens) return NDVM_OK;
    if (s->n_tokens < 0 || (s->n_seq == 0 && s->n_tokens)) return bad(who, "bad token count");
    if (s->n_tokens > kMostTokens || !fits(s->n_tokens, s->heads, std::max(s->dk, s->dv)))
        return fail(NDVM_E_UNSUPPORTED, who, "too many tokens");
    if (std::max(cut_of(s, packed, s->dk, s->dv).n_segments, cut_of(s, packed, s->dv, s->dk).n_segments) * s->heads > kMostGroups)
        return fail(NDVM_E_UNSUPPORTED, who, "too many sequences, tokens and heads for one launch");
    return NDVM_OK;
}

// Strides: magnitudes that keep the last element's offset in 64 bits.
bool bad_heads(const ndvm_heads *h, int64_t elements) {
    const auto far = [](int64_t v) { return v < 0 || v > kMostElements; };
    return (elements && !h->data) || far(h->seq_stride) || far(h->tok_stride) || far(h->head_stride);
}

Heads heads_of(const ndvm_heads *h, int64_t group) {
    return Heads{h->data, h->seq_stride, h->tok_stride, h->head_stride, int(group)};
}

size_t segment_bytes(const ndvm_attention_shape *s, const Cut &c) {
    return c.n_segments > s->n_seq ? round256(size_t(c.n_segments * s->heads) * size_t(c.state) * 4) : 0;
}

// of the gradient's calls: one for dq, one for dk and dv
size_t grad_segment_bytes(const ndvm_attention_shape *s, bool packed) {
    if (grad_together(s)) return 2 * segment_bytes(s, grad_cut(s, packed));
    return std::max(segment_bytes(s, cut_of(s, packed, s->dk, s->dv)), segment_bytes(s, cut_of(s, packed, s->dv, s->dk)));
}

// a gradient for each query head, before those that share a key are added up
size_t grad_part_bytes(const ndvm_attention_shape *s, int64_t d) { return round256(size_t(s->heads * s->n_tokens) * size_t(d) * 4); }

size_t attention_bytes(const ndvm_attention_shape *s, bool packed, bool grad) {
    if (!grad) {
        const size_t n = segment_bytes(s, cut_of(s, packed, s->dk, s->dv));
        return n ? n + 256 : 0;
    }
    size_t n = grad_segment_bytes(s, packed) + 256;
    if (s->heads > s->kv_heads) n += grad_part_bytes(s, s->dk) + grad_part_bytes(s, s->dv);
    return n;
}

void *aligned(void *p) { return reinterpret_cast<void *>(round256(reinterpret_cast<size_t>(p))); }

}  // namespace

extern "C" {

ndvm_status ndvm_layer_norm(int dtype, const void *x, int64_t rows, int64_t n, int64_t ld_x, const void *weight,
                            const void *bias, double eps, void *y, int64_t ld_y, float *mean, float *rstd,
                            void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_layer_norm";
        if (!known_type(dtype)) return bad(who, "unknown type");
        if (rows < 0 || n < 1 || ld_x < n || ld_y < n || !(eps >= 0.0) || !std::isfinite(eps))
            return bad(who, "bad size, stride or eps");
        if (!fits(rows, std::max(ld_x, ld_y))) return bad(who, "sizes overflow");
        if (rows == 0) return NDVM_OK;
        if (!x || !y) return bad(who, "null buffer");
        const NormArgs a{x, weight, bias, y, mean, rstd, rows, n, ld_x, ld_y, float(eps)};
        return launched(who, launch_norm(dtype, a, static_cast<hipStream_t>(stream)));
    });
}

ndvm_status ndvm_layer_norm_workspace_bytes(int64_t rows, int64_t n, size_t *bytes) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_layer_norm_workspace_bytes";
        if (!bytes) return bad(who, "null pointer");
        if (rows < 0 || n < 1 || !fits(rows, n)) return bad(who, "bad size");
        if (n > kMostNormGrad) return fail(NDVM_E_UNSUPPORTED, who, "more than 2^27 values in a row");
        *bytes = norm_grad_bytes(rows, n);
        return NDVM_OK;
    });
}

ndvm_status ndvm_layer_norm_grad(int dtype, const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, int64_t rows,
                                 int64_t n, const void *weight, const float *mean, const float *rstd, void *dx,
                                 int64_t ld_dx, void *dweight, void *dbias, void *workspace, size_t workspace_bytes,
                                 void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_layer_norm_grad";
        if (!known_type(dtype)) return bad(who, "unknown type");
        if (rows < 0 || n < 1 || ld_dy < n || ld_x < n || (dx && ld_dx < n)) return bad(who, "bad size or stride");
        if (!fits(rows, std::max(std::max(ld_x, ld_dy), dx ? ld_dx : 0))) return bad(who, "sizes overflow");
        if (n > kMostNormGrad) return fail(NDVM_E_UNSUPPORTED, who, "more than 2^27 values in a row");
        if (rows && (!dy || !x || !mean || !rstd)) return bad(who, "null buffer");
        if (!dx && !dweight && !dbias) return NDVM_OK;
        if (dweight || dbias) {
            if (workspace_bytes < norm_grad_bytes(rows, n)) return fail(NDVM_E_NOMEM, who, "workspace too small");
            if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 4) return bad(who, "null or misaligned workspace");
        }
        const NormGradArgs a{dy, x, weight, mean, rstd, dx, dweight, dbias, static_cast<float *>(workspace), rows, n, ld_dy, ld_x, ld_dx};
        return launched(who, launch_norm_grad(dtype, a, static_cast<hipStream_t>(stream)));
    });
}

ndvm_status ndvm_linear_attention_workspace_bytes(const ndvm_attention_shape *shape, int packed, int with_grad,
                                                  size_t *bytes) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_linear_attention_workspace_bytes";
        if (!bytes) return bad(who, "null pointer");
        if (const ndvm_status st = check_shape(who, shape, true, packed != 0)) return st;
        *bytes = attention_bytes(shape, packed != 0, with_grad != 0);
        return NDVM_OK;
    });
}

static ndvm_status check_call(const char *who, const ndvm_attention_shape *s, const ndvm_heads *q, const ndvm_heads *k,
                              const ndvm_heads *v, const float *log_decay, const int64_t *offsets) {
    if (const ndvm_status st = check_shape(who, s, true, offsets != nullptr)) return st;
    if (!offsets && s->n_seq && s->n_tokens % s->n_seq) return bad(who, "n_tokens is no multiple of n_seq, and there are no offsets");
    if (!q || !k || !v || (s->n_seq && !log_decay)) return bad(who, "null argument");
    if (bad_heads(q, s->n_tokens) || bad_heads(k, s->n_tokens) || bad_heads(v, s->n_tokens))
        return bad(who, "null buffer or bad stride");
    return NDVM_OK;
}

ndvm_status ndvm_linear_attention(const ndvm_attention_shape *shape, const ndvm_heads *q, const ndvm_heads *k,
                                  const ndvm_heads *v, const float *log_decay, const int64_t *offsets,
                                  const float *initial_state, const ndvm_heads *o, float *final_state,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_linear_attention";
        const ndvm_attention_shape *s = shape;
        if (const ndvm_status st = check_call(who, s, q, k, v, log_decay, offsets)) return st;
        if (!o || bad_heads(o, s->n_tokens)) return bad(who, "null buffer or bad stride");
        if (s->n_seq == 0) return NDVM_OK;
        const size_t need = attention_bytes(s, offsets != nullptr, false);
        if (workspace_bytes < need) return fail(NDVM_E_NOMEM, who, "workspace too small");
        if (need && !workspace) return bad(who, "null workspace");
        const Cut cut = cut_of(s, offsets != nullptr, s->dk, s->dv);
        const int64_t group = s->heads / s->kv_heads;
        AttendSets sets{};
        sets.count = 1;
        AttendArgs &a = sets.set[0];
        a.a = heads_of(q, 1);
        a.b = heads_of(k, group);
        a.c = heads_of(v, group);
        a.out = heads_of(o, 1);
        a.log_decay = log_decay;
        a.offsets = offsets;
        a.state_in = initial_state;
        a.state_out = final_state;
        a.segments = static_cast<float *>(aligned(workspace));
        a.n_seq = s->n_seq;
        a.n_tokens = s->n_tokens;
        a.heads = s->heads;
        a.da = s->dk;
        a.dc = s->dv;
        a.seg_len = cut.seg_len;
        a.n_segments = cut.n_segments;
        a.scale_pair = a.scale_read = float(s->scale);
        a.scale_add = 1.0f;
        if (const ndvm_status r = launched(who, launch_attend_segments(s->dtype, sets, static_cast<hipStream_t>(stream)))) return r;
        return launched(who, launch_attend(s->dtype, sets, static_cast<hipStream_t>(stream)));
    });
}

ndvm_status ndvm_linear_attention_grad(const ndvm_attention_shape *shape, const ndvm_heads *q, const ndvm_heads *k,
                                       const ndvm_heads *v, const float *log_decay, const int64_t *offsets,
                                       const float *initial_state, const ndvm_heads *d_o, const float *d_final,
                                       const ndvm_heads *dq, const ndvm_heads *dk, const ndvm_heads *dv,
                                       float *d_initial, void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_linear_attention_grad";
        const ndvm_attention_shape *s = shape;
        if (const ndvm_status st = check_call(who, s, q, k, v, log_decay, offsets)) return st;
        if (!d_o || !dq || !dk || !dv || bad_heads(d_o, s->n_tokens) || bad_heads(dq, 0) || bad_heads(dk, 0) || bad_heads(dv, 0))
            return bad(who, "null buffer or bad stride");
        if (d_initial && s->n_tokens && !dv->data) return bad(who, "d_initial without dv");
        if (s->n_seq == 0) return NDVM_OK;
        const size_t need = attention_bytes(s, offsets != nullptr, true);
        if (workspace_bytes < need) return fail(NDVM_E_NOMEM, who, "workspace too small");
        if (!workspace) return bad(who, "null workspace");
        const hipStream_t st = static_cast<hipStream_t>(stream);
        const int64_t group = s->heads / s->kv_heads;
        const Heads hq = heads_of(q, 1), hk = heads_of(k, group), hv = heads_of(v, group), ho = heads_of(d_o, 1);
        const bool packed = offsets != nullptr, together = grad_together(s);
        char *ws = static_cast<char *>(aligned(workspace));
        const size_t segments = grad_segment_bytes(s, packed);
        float *const of_q = reinterpret_cast<float *>(ws), *const of_kv = reinterpret_cast<float *>(ws + (together ? segments / 2 : 0));
        float *part = reinterpret_cast<float *>(ws + segments);
        AttendArgs all{};
        all.log_decay = log_decay;
        all.offsets = offsets;
        all.n_seq = s->n_seq;
        all.n_tokens = s->n_tokens;
        all.heads = s->heads;
        const auto widths = [&](AttendArgs &a, int64_t da, int64_t dc) {
            const Cut cut = together ? grad_cut(s, packed) : cut_of(s, packed, da, dc);
            a.da = da;
            a.dc = dc;
            a.seg_len = cut.seg_len;
            a.n_segments = cut.n_segments;
        };
        AttendArgs of_dq = all;
        of_dq.a = ho;
        of_dq.b = hv;
        of_dq.c = hk;
        of_dq.out = heads_of(dq, 1);
        widths(of_dq, s->dv, s->dk);
        of_dq.state_in = initial_state;
        of_dq.state_transposed = 1;
        of_dq.scale_pair = of_dq.scale_read = float(s->scale);
        of_dq.scale_add = 1.0f;
        of_dq.segments = of_q;
        all.reversed = 1;
        all.state_in = d_final;
        all.scale_pair = all.scale_add = float(s->scale);
        all.scale_read = 1.0f;
        all.segments = of_kv;
        // over the query heads of a group: each head's gradient in float, then their sum
        FoldHeadsSets folds{};
        const auto shared = [&](AttendArgs &a, const ndvm_heads *to, int64_t d) {
            if (group == 1) {
                a.out = heads_of(to, 1);
                return;
            }
            a.out = Heads{part, s->n_tokens / s->n_seq * d, d, s->n_tokens * d, 1};
            a.out_f32 = 1;
            folds.set[folds.count++] = FoldHeadsArgs{part, heads_of(to, group), s->n_seq, s->n_tokens, s->heads, d, packed};
            part += grad_part_bytes(s, d) / 4;
        };
        AttendArgs of_dk = all, of_dv = all;
        of_dk.a = hv;
        of_dk.b = ho;
        of_dk.c = hq;
        of_dk.state_transposed = 1;
        widths(of_dk, s->dv, s->dk);
        of_dv.a = hk;
        of_dv.b = hq;
        of_dv.c = ho;
        of_dv.state_out = d_initial;
        widths(of_dv, s->dk, s->dv);
        of_dv.shared_segments = together;
        const bool want_q = dq->data, want_k = dk->data, want_v = dv->data || d_initial;
        if (want_k) shared(of_dk, dk, s->dk);
        if (want_v) shared(of_dv, dv, s->dv);
        if (together) {
            AttendSets sums{}, sets{};
            if (want_q) sums.set[sums.count++] = of_dq;
            if (want_k || want_v) sums.set[sums.count++] = of_dk;
            if (want_q) sets.set[sets.count++] = of_dq;
            if (want_k) sets.set[sets.count++] = of_dk;
            if (want_v) sets.set[sets.count++] = of_dv;
            if (sets.count == 0) return NDVM_OK;
            if (const ndvm_status r = launched(who, launch_attend_segments(s->dtype, sums, st))) return r;
            if (const ndvm_status r = launched(who, launch_attend(s->dtype, sets, st))) return r;
        } else {
            for (const AttendArgs *a : {want_q ? &of_dq : nullptr, want_v ? &of_dv : nullptr, want_k ? &of_dk : nullptr}) {
                if (!a) continue;
                AttendSets one{};
                one.set[one.count++] = *a;
                if (const ndvm_status r = launched(who, launch_attend_segments(s->dtype, one, st))) return r;
                if (const ndvm_status r = launched(who, launch_attend(s->dtype, one, st))) return r;
            }
        }
        if (folds.count == 0 || s->n_tokens == 0) return NDVM_OK;
        return launched(who, launch_fold_heads(s->dtype, folds, st));
    });
}

ndvm_status ndvm_linear_attention_step(const ndvm_attention_shape *shape, const ndvm_heads *q, const ndvm_heads *k,
                                       const ndvm_heads *v, const float *log_decay, float *state, int64_t n_slots,
                                       const int64_t *slots, const ndvm_heads *o, void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_linear_attention_step";
        const ndvm_attention_shape *s = shape;
        if (const ndvm_status st = check_shape(who, s, false, false)) return st;
        if (n_slots < 0 || !fits(n_slots, s->heads, s->dk * s->dv) || (!slots && n_slots < s->n_seq))
            return bad(who, "bad slot count");
        if (!q || !k || !v || !o || bad_heads(q, s->n_seq) || bad_heads(k, s->n_seq) || bad_heads(v, s->n_seq) || bad_heads(o, s->n_seq))
            return bad(who, "null buffer or bad stride");
        if (s->n_seq == 0) return NDVM_OK;
        if (!log_decay || (n_slots && !state)) return bad(who, "null buffer");
        const int64_t group = s->heads / s->kv_heads;
        const StepArgs a{heads_of(q, 1), heads_of(k, group), heads_of(v, group), heads_of(o, 1), log_decay, state, slots,
                         s->n_seq, n_slots, s->heads, s->dk, s->dv, float(s->scale)};
        return launched(who, launch_step(s->dtype, a, static_cast<hipStream_t>(stream)));
    });
}

static ndvm_status check_ffn(const char *who, int dtype, int64_t rows, int64_t n_in, int64_t n_out) {
    if (!known_type(dtype)) return bad(who, "unknown type");
    if (rows < 0 || n_in < 1 || n_out < 1) return bad(who, "bad size");
    if (rows > kMostFfnRows || n_in > kMostFfnWidth || n_out > kMostFfnWidth)
        return fail(NDVM_E_UNSUPPORTED, who, "more than 2^22 rows, or a width past 2^21");
    return NDVM_OK;
}

ndvm_status ndvm_gated_ffn_workspace_bytes(int dtype, int64_t rows, int64_t n_in, int64_t n_out, int with_grad,
                                           size_t *bytes) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_gated_ffn_workspace_bytes";
        if (!bytes) return bad(who, "null pointer");
        if (const ndvm_status st = check_ffn(who, dtype, rows, n_in, n_out)) return st;
        *bytes = ffn_bytes(dtype, rows, n_in, n_out, with_grad != 0);
        return NDVM_OK;
    });
}

ndvm_status ndvm_gated_ffn(int dtype, int act, const void *x, int64_t rows, int64_t n_in, int64_t ld_x,
                           const void *w_gate, int64_t ld_gate, const void *w_up, int64_t ld_up, int64_t n_out,
                           void *h, int64_t ld_h, void *workspace, size_t workspace_bytes, void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_gated_ffn";
        if (const ndvm_status st = check_ffn(who, dtype, rows, n_in, n_out)) return st;
        if (act < NDVM_ACT_SILU || act > NDVM_ACT_RELU) return bad(who, "unknown activation");
        if (ld_x < n_in || ld_gate < n_in || ld_up < n_in || ld_h < n_out) return bad(who, "bad stride");
        if (!fits(rows, ld_x) || !fits(rows, ld_h) || !fits(n_out, ld_gate) || !fits(n_out, ld_up)) return bad(who, "sizes overflow");
        if (rows == 0) return NDVM_OK;
        if (!x || !w_gate || !w_up || !h) return bad(who, "null buffer");
        const size_t need = ffn_bytes(dtype, rows, n_in, n_out, false);
        if (workspace_bytes < need) return fail(NDVM_E_NOMEM, who, "workspace too small");
        if (need && !workspace) return bad(who, "null workspace");
        FfnArgs a{};
        a.dtype = dtype;
        a.act = act;
        a.x = x;
        a.wg = w_gate;
        a.wu = w_up;
        a.rows = rows;
        a.n_in = n_in;
        a.n_out = n_out;
        a.ld_x = ld_x;
        a.ld_wg = ld_gate;
        a.ld_wu = ld_up;
        a.h = h;
        a.ld_h = ld_h;
        a.ws = workspace;
        return launched(who, launch_ffn(a, static_cast<hipStream_t>(stream)));
    });
}

ndvm_status ndvm_gated_ffn_grad(int dtype, int act, const void *dh, int64_t ld_dh, const void *x, int64_t rows,
                                int64_t n_in, int64_t ld_x, const void *w_gate, int64_t ld_gate, const void *w_up,
                                int64_t ld_up, int64_t n_out, void *dx, int64_t ld_dx, void *dw_gate,
                                int64_t ld_dgate, void *dw_up, int64_t ld_dup, void *workspace,
                                size_t workspace_bytes, void *stream) {
    return guarded([&]() -> ndvm_status {
        const char *who = "ndvm_gated_ffn_grad";
        if (const ndvm_status st = check_ffn(who, dtype, rows, n_in, n_out)) return st;
        if (act < NDVM_ACT_SILU || act > NDVM_ACT_RELU) return bad(who, "unknown activation");
        if (ld_dh < n_out || ld_x < n_in || ld_gate < n_in || ld_up < n_in || (dx && ld_dx < n_in) ||
            (dw_gate && ld_dgate < n_in) || (dw_up && ld_dup < n_in))
            return bad(who, "bad stride");
        if (!fits(rows, ld_x) || !fits(rows, ld_dh) || !fits(n_out, ld_gate) || !fits(n_out, ld_up) ||
            (dx && !fits(rows, ld_dx)) || (dw_gate && !fits(n_out, ld_dgate)) || (dw_up && !fits(n_out, ld_dup)))
            return bad(who, "sizes overflow");
        if (!dw_gate != !dw_up) return bad(who, "dw_gate and dw_up come together");
        if (!dx && !dw_gate) return NDVM_OK;
        if (!w_gate || !w_up || (rows && (!x || !dh))) return bad(who, "null buffer");
        const size_t need = ffn_bytes(dtype, rows, n_in, n_out, true);
        if (workspace_bytes < need) return fail(NDVM_E_NOMEM, who, "workspace too small");
        if (!workspace) return bad(who, "null workspace");
        FfnArgs a{};
        a.dtype = dtype;
        a.act = act;
        a.x = x;
        a.wg = w_gate;
        a.wu = w_up;
        a.dh = dh;
        a.rows = rows;
        a.n_in = n_in;
        a.n_out = n_out;
        a.ld_x = ld_x;
        a.ld_wg = ld_gate;
        a.ld_wu = ld_up;
        a.ld_dh = ld_dh;
        a.dx = rows ? dx : nullptr;
        a.ld_dx = ld_dx;
        a.dwg = dw_gate;
        a.ld_dwg = ld_dgate;
        a.dwu = dw_up;
        a.ld_dwu = ld_dup;
        a.ws = workspace;
        return launched(who, launch_ffn_grad(a, static_cast<hipStream_t>(stream)));
    });
}

}  // extern "C"
