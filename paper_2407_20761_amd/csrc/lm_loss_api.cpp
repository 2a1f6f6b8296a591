// C ABI of the cross entropy over a vocabulary: validation, the pieces of the vocabulary, and its forward and backward out of the matrix
// products (gemm.hip) and row kernels (lm_loss.hip).
#include "gemm_plan.h"
#include "ob_internal.h"

using namespace ob;

namespace {

constexpr int MAX_HIDDEN = 8192, MAX_VOCAB = 1 << 21;
// a launch has fewer than 2^32 threads, 256 to a tile of 256 x 256 logits
constexpr long MAX_LOGITS = 1l << 39;
// Bytes that the gradient of the logits, in bf16, may take at a time (256 columns, if they are more)
constexpr size_t PIECE_BYTES = (size_t)1 << 30;

struct Bump {
    size_t off = 0;
    size_t take(size_t bytes) { const size_t o = off; off += align_up(bytes, 256); return o; }
};

struct Pieces {
    int cols, count, ld;      // columns of a piece (the last one's rest), pieces, row stride of the gradient
    Pieces(int n, int V) {
        const size_t most = PIECE_BYTES / ((size_t)n * 2) / 256 * 256;
        const int fit = most < 256 ? 256 : most > (size_t)V ? V : (int)most;
        count = (V + fit - 1) / fit;
        const int even = (V + count - 1) / count;
        cols = count == 1 ? V : (even + 255) / 256 * 256;
        count = (V + cols - 1) / cols;
        ld = (cols + 63) / 64 * 64;
    }
};

int slots_of(const Plan &p, int V) { return 2 * ((V + tile_cols(p.kind) - 1) / tile_cols(p.kind)); }

struct Work { size_t xs, stats, target, g, dxs, own, sums, sums_bytes, total; };
Work work_layout(int n, int V, int H) {
    const Plan logits = whole_plan(0, n, V, H);
    const Pieces pc(n, V);
    Work w{};
    Bump fwd;
    w.xs = fwd.take((size_t)n * H * 2);
    Bump bwd = fwd;
    w.stats = fwd.take((size_t)slots_of(logits, V) * n * 8);
    w.target = fwd.take((size_t)n * 4);
    w.dxs = bwd.take((size_t)n * H * 2);
    w.own = bwd.take((size_t)n * H * 2);
    w.g = bwd.take(loss_grad_bytes(n, pc.ld));
    if (pc.count > 1) {
        const Plan p = whole_plan(1, n, H, pc.cols);
        w.sums_bytes = (size_t)p.n_full * tile_rows(p.kind) * tile_cols(p.kind) * 4;
    } else {
        w.sums_bytes = gemm_workspace_bytes(1, n, H, V);
    }
    w.sums = bwd.take(w.sums_bytes);
    w.total = fwd.off > bwd.off ? fwd.off : bwd.off;
    return w;
}

int validate_desc(const ob_lm_loss_desc *desc, const char *who) {
    if (!desc) return fail(OB_EINVAL, "%s: desc is null", who);
    if (desc->dtype != OB_BF16 && desc->dtype != OB_FP32) return fail(OB_EINVAL, "%s: unknown dtype %d", who, desc->dtype);
    if (desc->hidden < 64 || desc->vocab < 1) return fail(OB_EINVAL, "%s: non-positive dimension", who);
    if (desc->hidden % 64) return fail(OB_EUNSUPPORTED, "%s: hidden must be a multiple of 64", who);
    if (desc->hidden > MAX_HIDDEN) return fail(OB_EUNSUPPORTED, "%s: hidden > %d", who, MAX_HIDDEN);
    if (desc->vocab > MAX_VOCAB) return fail(OB_EUNSUPPORTED, "%s: vocab > %d", who, MAX_VOCAB);
    return OB_OK;
}
size_t bytes_of(const ob_lm_loss_desc *desc, int n) {
    return desc->dtype == OB_FP32 ? f32::lm_loss_work_bytes(n, desc->hidden, desc->vocab) : work_layout(n, desc->vocab, desc->hidden).total;
}

bool aligned16(const void *p) { return (uintptr_t)p % 16 == 0; }

int validate(const ob_lm_loss_desc *desc, const void *w, const void *x, int total_tokens, const int32_t *rows_host, const int32_t *rows_dev,
             int n_rows, const int32_t *labels, const void *ws, size_t ws_bytes, const char *who) {
    if (int rc = validate_desc(desc, who)) return rc;
    if (!w || !x || (n_rows && !labels)) return fail(OB_EINVAL, "%s: w / x / labels is null", who);
    if (total_tokens < 1 || total_tokens > MAX_TOKENS) return fail(OB_EINVAL, "%s: total_tokens %d outside [1, %d]", who, total_tokens, MAX_TOKENS);
    if (n_rows < 0 || n_rows > total_tokens) return fail(OB_EINVAL, "%s: n_rows %d outside [0, total_tokens]", who, n_rows);
    if (!aligned16(w) || !aligned16(x)) return fail(OB_EINVAL, "%s: tensors must be aligned to 16 bytes", who);
    if (n_rows == 0) return OB_OK;
    if ((long)n_rows * desc->vocab > MAX_LOGITS) return fail(OB_EUNSUPPORTED, "%s: n_rows x vocab beyond 2^39", who);
    if (!rows_host != !rows_dev) return fail(OB_EINVAL, "%s: rows need a host and a device copy", who);
    if (!rows_host && n_rows != total_tokens) return fail(OB_EINVAL, "%s: without a row list n_rows is total_tokens", who);
    if (rows_host)
        for (int i = 0, last = -1; i < n_rows; last = rows_host[i++])
            if (rows_host[i] <= last || rows_host[i] >= total_tokens)
                return fail(OB_EINVAL, "%s: rows[%d] = %d, must ascend inside [0, %d)", who, i, rows_host[i], total_tokens);
    if (!ws || !aligned16(ws) || ws_bytes < bytes_of(desc, n_rows))
        return fail(OB_EWORKSPACE, "%s: workspace too small (%zu bytes given) or not aligned", who, ws_bytes);
    return OB_OK;
}

}  // namespace

extern "C" size_t ob_lm_loss_workspace_bytes(const ob_lm_loss_desc *desc, int n_rows) {
    if (validate_desc(desc, "ob_lm_loss_workspace_bytes") || n_rows < 1 || n_rows > MAX_TOKENS || (long)n_rows * desc->vocab > MAX_LOGITS)
        return 0;
    return bytes_of(desc, n_rows);
}

extern "C" int ob_lm_loss_plan(const ob_lm_loss_desc *desc, int n_rows, ob_lm_loss_launch *launch) {
    const char *who = "ob_lm_loss_plan";
    if (int rc = validate_desc(desc, who)) return rc;
    if (desc->dtype != OB_BF16) return fail(OB_EINVAL, "%s: the plan is that of bf16", who);
    if (!launch) return fail(OB_EINVAL, "%s: launch is null", who);
    if (!ob_lm_loss_workspace_bytes(desc, n_rows)) return fail(OB_EINVAL, "%s: n_rows %d out of range", who, n_rows);
    const int n = n_rows, V = desc->vocab, H = desc->hidden;
    const Pieces pc(n, V);
    const Plan fwd = whole_plan(0, n, V, H), piece = whole_plan(0, n, pc.cols, H), last = whole_plan(0, n, V - (pc.count - 1) * pc.cols, H);
    *launch = ob_lm_loss_launch{tile_rows(fwd.kind), fwd.n_full, pc.count, tile_rows(piece.kind), tile_rows(last.kind),
                                pc.count > 1 ? tile_rows(whole_plan(1, n, H, pc.cols).kind) : 0,
                                tile_rows(loss_dw_kind(pc.cols, H, n))};
    return OB_OK;
}

extern "C" int ob_lm_loss_fwd(const ob_lm_loss_desc *desc, const void *w, const void *x, int total_tokens, const int32_t *rows_host,
                              const int32_t *rows_dev, int n_rows, const int32_t *labels, float *nll, float *lse, void *ws,
                              size_t ws_bytes, void *hip_stream) {
    const char *who = "ob_lm_loss_fwd";
    if (int rc = validate(desc, w, x, total_tokens, rows_host, rows_dev, n_rows, labels, ws, ws_bytes, who)) return rc;
    if (n_rows == 0) return OB_OK;
    if (!nll || !lse) return fail(OB_EINVAL, "%s: nll / lse is null", who);
    hipStream_t s = (hipStream_t)hip_stream;
    const int n = n_rows, V = desc->vocab, H = desc->hidden;
    if (desc->dtype == OB_FP32) {
        f32::lm_loss_fwd(w, x, rows_dev, n, H, V, labels, nll, lse, ws, s);
        return check_launch(who);
    }
    const Work wk = work_layout(n, V, H);
    unsigned char *at = (unsigned char *)ws;
    const void *xs = x;
    if (rows_dev) {
        launch_rows_gather(at + wk.xs, x, rows_dev, n, H, s);
        xs = at + wk.xs;
    }
    const Plan p = whole_plan(0, n, V, H);
    launch_loss_stats(p, n, V, H, xs, w, labels, at + wk.stats, (float *)(at + wk.target), s);
    launch_loss_combine(at + wk.stats, (const float *)(at + wk.target), labels, n, V, slots_of(p, V), nll, lse, s);
    return check_launch(who);
}

extern "C" int ob_lm_loss_bwd(const ob_lm_loss_desc *desc, int flags, const void *w, const void *x, int total_tokens,
                              const int32_t *rows_host, const int32_t *rows_dev, int n_rows, const int32_t *labels, const float *lse,
                              const float *dnll, void *dx, void *dw, void *ws, size_t ws_bytes, void *hip_stream) {
    const char *who = "ob_lm_loss_bwd";
    if (int rc = validate(desc, w, x, total_tokens, rows_host, rows_dev, n_rows, labels, ws, ws_bytes, who)) return rc;
    if (flags & ~OB_BWD_ACCUMULATE) return fail(OB_EINVAL, "%s: unknown flag bits %d", who, flags);
    if ((n_rows && (!lse || !dnll)) || !dx || !dw) return fail(OB_EINVAL, "%s: lse / dnll / dx / dw is null", who);
    if (!aligned16(dx) || !aligned16(dw)) return fail(OB_EINVAL, "%s: tensors must be aligned to 16 bytes", who);
    hipStream_t s = (hipStream_t)hip_stream;
    const int n = n_rows, V = desc->vocab, H = desc->hidden, acc = flags & OB_BWD_ACCUMULATE;
    if (n == 0) {
        const int width = desc->dtype == OB_FP32 ? 2 * H : H;      // (rows of zeros, in elements of two bytes)
        launch_rows_spread(nullptr, dx, nullptr, 0, total_tokens, width, s);
        if (!acc) launch_rows_spread(nullptr, dw, nullptr, 0, V, width, s);
        return check_launch(who);
    }
    if (desc->dtype == OB_FP32) {
        f32::lm_loss_bwd(w, x, total_tokens, rows_dev, n, H, V, labels, lse, dnll, dx, dw, acc ? 1 : 0, ws, s);
        return check_launch(who);
    }
    const Work wk = work_layout(n, V, H);
    const Pieces pc(n, V);
    unsigned char *at = (unsigned char *)ws;
    const void *xs = x;
    void *dxs = dx;
    if (rows_dev) {
        launch_rows_gather(at + wk.xs, x, rows_dev, n, H, s);
        xs = at + wk.xs;
        dxs = at + wk.dxs;
    }
    // Per piece of the vocabulary: G = (softmax - one-hot) weight, its logits computed again; what its rounding took of the entries at the labels, which are
    // most of a row of dx and of the labels' rows of dw; dW rows of the piece = G^T x, whole; dx += G W
    const Plan p_dx = whole_plan(1, n, H, pc.cols);
    float *sums = (float *)(at + wk.sums);
    unsigned char *g = at + wk.g;
    for (int i = 0; i < pc.count; ++i) {
        const int v0 = i * pc.cols, cols = V - v0 < pc.cols ? V - v0 : pc.cols, ld = (cols + 63) / 64 * 64;
        const unsigned char *wp = (const unsigned char *)w + (size_t)v0 * H * 2;
        unsigned char *dwp = (unsigned char *)dw + (size_t)v0 * H * 2;
        launch_loss_grad(whole_plan(0, n, cols, H), n, cols, H, xs, wp, labels, V, lse, dnll, v0, g, ld, s);
        launch_loss_labels(n, H, V, v0, cols, loss_lack(g, n, ld), loss_lead(g, n, ld), labels, xs, wp, dxs, at + wk.own, s);
        launch_loss_dw(cols, H, n, g, ld, xs, dwp, acc ? dwp : nullptr, at + wk.own, s);
        if (pc.count > 1) launch_gemm_nn_piece(p_dx, n, H, cols, g, ld, wp, sums, i == 0, s);
        else launch_gemm_nn(n, H, cols, g, ld, wp, dxs, dxs, wk.sums_bytes ? sums : nullptr, wk.sums_bytes, s);
    }
    if (pc.count > 1) launch_gemm_nn_round(p_dx, n, H, sums, dxs, dxs, s);
    if (rows_dev) launch_rows_spread(dxs, dx, rows_dev, n, total_tokens, H, s);
    return check_launch(who);
}
