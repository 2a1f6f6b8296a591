// C ABI of the varlen attention with a sliding window and sinks: validation, and the layout of the backward's workspace.
#include "attention_plan.h"
#include "ob_internal.h"

using namespace ob;

namespace {

constexpr int MAX_STRIDE = 1 << 24;     // elements: the offsets inside a tile of 64 rows have 32 bits

// `window` is cut to the longest segment there may be
int validate(const ob_segments *seg, int nq, int nkv, int d, int ldq, int ldkv, int ldo, float scale, int *window, int sinks, int dtype,
             const char *who) {
    if (int rc = validate_attn(seg, nq, nkv, d, ldq, ldkv, ldo, OB_MASK_SEG_CAUSAL, dtype, who)) return rc;
    if (ldq > MAX_STRIDE || ldkv > MAX_STRIDE || ldo > MAX_STRIDE) return fail(OB_EUNSUPPORTED, "%s: a row stride beyond %d elements", who, MAX_STRIDE);
    // (times the scale, the -1e30 of a masked score is to be far below every other, and finite)
    if (!(scale >= 1e-20f && scale <= 1e6f)) return fail(OB_EINVAL, "%s: scale must lie in [1e-20, 1e6]", who);
    if (*window < 1) return fail(OB_EINVAL, "%s: window %d must be at least 1 (a row sees itself)", who, *window);
    if (sinks < 0) return fail(OB_EINVAL, "%s: sinks %d must not be negative", who, sinks);
    if (sinks > MAX_SINKS) return fail(OB_EUNSUPPORTED, "%s: sinks %d, at most %d", who, sinks, MAX_SINKS);
    if (*window > MAX_TOKENS) *window = MAX_TOKENS;
    return OB_OK;
}

struct WindowWork { size_t delta, lse2, part, total; };
WindowWork work_layout(const ob_segments *seg, int nq, int nkv, int d, int window, int sinks, int dtype) {
    const size_t rows = align_up((size_t)seg->total_tokens * nq * 4, 256);
    WindowWork w{0, rows, 2 * rows, rows};
    if (dtype == OB_BF16) w.total = w.part + align_up((size_t)sink_chunks(seg, sink_whole_rows(window, nq / nkv), sinks) * nkv * 2 * sinks * d * 4, 256);
    return w;
}

bool aligned16(const void *p) { return (uintptr_t)p % 16 == 0; }

}  // namespace

extern "C" int ob_varlen_attn_window_fwd(const void *q, const void *k, const void *v, void *o, float *lse, int ldq, int ldkv,
                                         int ldo, const ob_segments *seg, int nq, int nkv, int d, float scale, int window,
                                         int sinks, int dtype, void *hip_stream) {
    const char *who = "ob_varlen_attn_window_fwd";
    if (!q || !k || !v || !o || !lse) return fail(OB_EINVAL, "%s: null tensor pointer", who);
    if (int rc = validate(seg, nq, nkv, d, ldq, ldkv, ldo, scale, &window, sinks, dtype, who)) return rc;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return fail(OB_EINVAL, "%s: tensors must be aligned to 16 bytes", who);
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == OB_FP32) f32::attn_window_fwd(q, k, v, o, lse, ldq, ldkv, ldo, seg, nq, nkv, d, scale, window, sinks, s);
    else launch_attn_window_fwd(q, k, v, o, lse, ldq, ldkv, ldo, seg, nq, nkv, d, scale, window, sinks, s);
    return check_launch(who);
}

extern "C" size_t ob_varlen_attn_window_bwd_workspace_bytes(const ob_segments *seg, int nq, int nkv, int d, int window, int sinks,
                                                            int dtype) {
    if (validate(seg, nq, nkv, d, nq * d, nkv * d, nq * d, 1.f, &window, sinks, dtype, "ob_varlen_attn_window_bwd_workspace_bytes")) return 0;
    return work_layout(seg, nq, nkv, d, window, sinks, dtype).total;
}

extern "C" int ob_varlen_attn_window_bwd(const void *d_o, const void *q, const void *k, const void *v, const void *o,
                                         const float *lse, void *dq, void *dk, void *dv, int ldq, int ldkv, int ldo,
                                         const ob_segments *seg, int nq, int nkv, int d, float scale, int window, int sinks,
                                         int dtype, void *ws, size_t ws_bytes, void *hip_stream) {
    const char *who = "ob_varlen_attn_window_bwd";
    if (!d_o || !q || !k || !v || !o || !lse || !dq || !dk || !dv) return fail(OB_EINVAL, "%s: null tensor pointer", who);
    if (int rc = validate(seg, nq, nkv, d, ldq, ldkv, ldo, scale, &window, sinks, dtype, who)) return rc;
    if (!aligned16(d_o) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv))
        return fail(OB_EINVAL, "%s: tensors must be aligned to 16 bytes", who);
    const WindowWork w = work_layout(seg, nq, nkv, d, window, sinks, dtype);
    if (!ws || ws_bytes < w.total || !aligned16(ws)) return fail(OB_EWORKSPACE, "%s: workspace too small (%zu bytes given) or not aligned", who, ws_bytes);
    hipStream_t s = (hipStream_t)hip_stream;
    unsigned char *at = (unsigned char *)ws;
    if (dtype == OB_FP32)
        f32::attn_window_bwd(d_o, q, k, v, o, lse, dq, dk, dv, (float *)ws, ldq, ldkv, ldo, seg, nq, nkv, d, scale, window, sinks, s);
    else
        launch_attn_window_bwd(d_o, q, k, v, o, lse, (float *)(at + w.lse2), (float *)(at + w.delta), (float *)(at + w.part), dq, dk, dv, ldq,
                               ldkv, ldo, seg, nq, nkv, d, scale, window, sinks, s);
    return check_launch(who);
}

extern "C" int ob_varlen_attn_window_bwd_plan(const ob_segments *seg, int nq, int nkv, int d, int window, int sinks,
                                              ob_attn_bwd_launch *launch, int *threads, int *chunks) {
    const char *who = "ob_varlen_attn_window_bwd_plan";
    if (!launch || !threads || !chunks) return fail(OB_EINVAL, "%s: null output", who);
    if (int rc = validate(seg, nq, nkv, d, nq * d, nkv * d, nq * d, 1.f, &window, sinks, OB_BF16, who)) return rc;
    const int whole = sinks ? sink_whole_rows(window, nq / nkv) : 0, shape = dkv_shape(seg, nkv, nq / nkv, d, true, window, whole);
    const int key_rows = 32 * dkv_np(d, shape);
    TileOrder ord;
    const int places = make_order(seg, key_rows, true, true, ord, window, whole);
    *launch = ob_attn_bwd_launch{key_rows, dkv_sr(d, shape), places, ord.n ? key_rows << ord.unit_log2 : 0};
    *threads = dkv_threads(d, shape);
    *chunks = sink_chunks(seg, whole, sinks);
    return OB_OK;
}
