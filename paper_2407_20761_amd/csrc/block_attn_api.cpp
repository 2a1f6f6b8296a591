// C ABI of a block with a window, sinks or rotary positions of several axes in its attention: the block of api.cpp with these steps in place of its own.
#include <cmath>

#include "attention_plan.h"
#include "ob_internal.h"

using namespace ob;

namespace {

inline unsigned char *column(void *rows, size_t elements) { return (unsigned char *)rows + elements * 2; }
inline const unsigned char *column(const void *rows, size_t elements) { return (const unsigned char *)rows + elements * 2; }

void rotate(const BlockSteps &st, void *qkv, int T, int inverse, hipStream_t s) {
    const ob_block_desc &d = *st.desc;
    const int ld = (d.n_q_heads + 2 * d.n_kv_heads) * d.head_dim;
    launch_rotary_axes(qkv, ld, qkv, ld, T, d.n_q_heads + d.n_kv_heads, d.head_dim, st.table, st.pos, inverse, d.dtype, s);
}
void attn_fwd(const BlockSteps &st, const void *qkv, void *o, float *lse, const ob_segments *seg, hipStream_t s) {
    const ob_block_desc &d = *st.desc;
    const int nq = d.n_q_heads, nkv = d.n_kv_heads, hd = d.head_dim, ld = (nq + 2 * nkv) * hd;
    launch_attn_window_fwd(qkv, column(qkv, nq * hd), column(qkv, (nq + nkv) * hd), o, lse, ld, ld, nq * hd, seg, nq, nkv, hd,
                           1.0f / sqrtf((float)hd), st.window, st.sinks, s);
}
void attn_bwd(const BlockSteps &st, const void *d_o, const void *qkv, const void *o, const float *lse, float *lse2, float *delta, void *dqkv,
              const ob_segments *seg, hipStream_t s) {
    const ob_block_desc &d = *st.desc;
    const int nq = d.n_q_heads, nkv = d.n_kv_heads, hd = d.head_dim, ld = (nq + 2 * nkv) * hd;
    launch_attn_window_bwd(d_o, qkv, column(qkv, nq * hd), column(qkv, (nq + nkv) * hd), o, lse, lse2, delta, st.part, dqkv,
                           column(dqkv, nq * hd), column(dqkv, (nq + nkv) * hd), ld, ld, nq * hd, seg, nq, nkv, hd, 1.0f / sqrtf((float)hd),
                           st.window, st.sinks, s);
}

// what the description leaves to `attn`, checked
int make_steps(const ob_block_desc *desc, const ob_block_attn *attn, BlockSteps &st, const char *who) {
    if (!desc || !attn) return fail(OB_EINVAL, "%s: desc / attn is null", who);
    st = BlockSteps{};
    st.desc = desc;
    if (attn->window < 0 || attn->sinks < 0) return fail(OB_EINVAL, "%s: window %d and sinks %d must not be negative", who, attn->window, attn->sinks);
    if (attn->sinks > MAX_SINKS) return fail(OB_EUNSUPPORTED, "%s: sinks %d, at most %d", who, attn->sinks, MAX_SINKS);
    if (attn->window) {
        if (desc->mask != OB_MASK_SEG_CAUSAL) return fail(OB_EINVAL, "%s: a window needs the causal mask", who);
        st.window = attn->window < MAX_TOKENS ? attn->window : MAX_TOKENS;
        st.sinks = attn->sinks;
        st.attn_fwd = attn_fwd;
        st.attn_bwd = attn_bwd;
    } else if (attn->sinks) return fail(OB_EINVAL, "%s: sinks without a window", who);
    if (attn->rotary) {
        if (int rc = rotary_table(attn->rotary, st.table, who)) return rc;
        if (desc->use_rotary) return fail(OB_EINVAL, "%s: rotary positions with axes in place of use_rotary, not beside it", who);
        if (attn->rotary->head_dim != desc->head_dim) return fail(OB_EINVAL, "%s: rotary description for heads of %d", who, attn->rotary->head_dim);
        if (!attn->pos) return fail(OB_EINVAL, "%s: pos is null", who);
        st.pos = attn->pos;
        st.rotate = rotate;
    }
    st.f32_fwd = f32::block_steps_fwd;
    st.f32_bwd = f32::block_steps_bwd;
    return OB_OK;
}

// the block's own workspace, then the sums of the sinks
struct AttnWork { size_t part, total; };
AttnWork work_layout(const ob_block_desc *desc, const BlockSteps &st, const ob_segments *seg) {
    const size_t own = align_up(ob_block_workspace_bytes(desc, seg->total_tokens), 256);
    size_t sums = 0;
    if (st.window && desc->dtype == OB_BF16)
        sums = (size_t)sink_chunks(seg, sink_whole_rows(st.window, desc->n_q_heads / desc->n_kv_heads), st.sinks) * desc->n_kv_heads * 2 *
               st.sinks * desc->head_dim * 4;
    return AttnWork{own, own + align_up(sums, 256)};
}

}  // namespace

extern "C" size_t ob_block_attn_workspace_bytes(const ob_block_desc *desc, const ob_block_attn *attn, const ob_segments *seg) {
    const char *who = "ob_block_attn_workspace_bytes";
    BlockSteps st;
    if (make_steps(desc, attn, st, who) || !seg || !ob_block_workspace_bytes(desc, seg->total_tokens)) return 0;
    if (validate_attn(seg, desc->n_q_heads, desc->n_kv_heads, desc->head_dim, desc->n_q_heads * desc->head_dim,
                      desc->n_kv_heads * desc->head_dim, desc->n_q_heads * desc->head_dim, desc->mask, desc->dtype, who))
        return 0;
    return work_layout(desc, st, seg).total;
}

extern "C" int ob_block_attn_fwd(const ob_block_desc *desc, const ob_block_attn *attn, const ob_block_weights *w, const void *x, void *y,
                                 void *saved, size_t saved_bytes, const ob_segments *seg, void *ws, size_t ws_bytes, void *hip_stream) {
    BlockSteps st;
    if (int rc = make_steps(desc, attn, st, "ob_block_attn_fwd")) return rc;
    return block_fwd("ob_block_attn_fwd", desc, w, x, y, saved, saved_bytes, seg, ws, ws_bytes, (hipStream_t)hip_stream, &st);
}

extern "C" int ob_block_attn_bwd(const ob_block_desc *desc, const ob_block_attn *attn, const ob_block_weights *w, const ob_block_grads *g,
                                 int flags, const void *x, const void *dy, void *dx, void *saved, size_t saved_bytes,
                                 const ob_segments *seg, void *ws, size_t ws_bytes, void *hip_stream) {
    const char *who = "ob_block_attn_bwd";
    BlockSteps st;
    if (int rc = make_steps(desc, attn, st, who)) return rc;
    const size_t need = ob_block_attn_workspace_bytes(desc, attn, seg);
    // (0: arguments that block_bwd refuses)
    if (need && (!ws || ws_bytes < need)) return fail(OB_EWORKSPACE, "%s: workspace too small (%zu bytes given)", who, ws_bytes);
    if (need) st.part = (float *)((unsigned char *)ws + work_layout(desc, st, seg).part);
    return block_bwd(who, desc, w, g, flags, x, dy, dx, saved, saved_bytes, seg, ws, ws_bytes, (hipStream_t)hip_stream, &st);
}
