// Stand-ins for the device half of the language side, for its host-only sanitizer build.  Each writes all that its kernels write to the caller's buffers and
// reads all that they read of the workspace, so that a region that a size rule makes too small, or puts on another one still in use, is seen on the
// host.  (gemm_any and the other launchers of a block: stubs.cpp; they write nothing.)
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "../../paper_2407_20761_amd/csrc/attention_plan.h"
#include "../../paper_2407_20761_amd/csrc/gemm_plan.h"
#include "../../paper_2407_20761_amd/csrc/ob_internal.h"

extern bool launches_pass;
const void *part_begin = nullptr;      // the sinks' sums of the last windowed backward
size_t part_bytes = 0;
int launches = 0;

namespace {

void reach(const char *name) {
    ++launches;
    if (launches_pass) return;
    std::fprintf(stderr, "device launcher reached: %s\n", name);
    std::abort();
}
// every byte written as `mark`, and read as it
void put(void *p, size_t bytes, int mark) { std::memset(p, mark, bytes); }
void see(const void *p, size_t bytes, int mark, const char *what) {
    const unsigned char *b = (const unsigned char *)p;
    if (bytes && (b[0] != mark || std::memcmp(b, b + 1, bytes - 1))) {
        std::fprintf(stderr, "%s has been written over\n", what);
        std::abort();
    }
}
enum { XS = 1, STATS, TARGET, G, LACK, LEAD, OWN, SUMS, DXS, DELTA, LSE2, PART };
int xs_mark = 0;       // rows gathered: they have to be there for every product; 0: the caller's x itself
size_t slots(const ob::Plan &p, int V) { return 2 * (size_t)((V + ob::tile_cols(p.kind) - 1) / ob::tile_cols(p.kind)); }
size_t sums_of(const ob::Plan &p) { return (size_t)p.n_full * ob::tile_rows(p.kind) * ob::tile_cols(p.kind) * 4; }

}  // namespace

namespace ob {

void launch_loss_stats(const Plan &p, int n, int V, int H, const void *x, const void *, const int32_t *, void *stats, float *target, hipStream_t) {
    reach("launch_loss_stats");
    see(x, (size_t)n * H * 2, xs_mark, "xs");
    put(stats, slots(p, V) * n * 8, STATS);
    put(target, (size_t)n * 4, TARGET);
}
void launch_loss_combine(const void *stats, const float *target, const int32_t *, int n, int, int n_slots, float *nll, float *lse, hipStream_t) {
    reach("launch_loss_combine");
    see(stats, (size_t)n_slots * n * 8, STATS, "stats");
    see(target, (size_t)n * 4, TARGET, "target");
    put(nll, (size_t)n * 4, 0);
    put(lse, (size_t)n * 4, 0);
}
void launch_loss_grad(const Plan &, int n, int cols, int H, const void *x, const void *, const int32_t *, int, const float *, const float *, int, void *g, int ldg,
                      hipStream_t) {
    reach("launch_loss_grad");
    if (ldg < cols || ldg % 64 || ldg - cols >= 64) std::abort();
    see(x, (size_t)n * H * 2, xs_mark, "xs");
    put(g, (size_t)n * ldg * 2, G);
    put(loss_lack(g, n, ldg), (size_t)n * 4, LACK);
    put(loss_lead(g, n, ldg), (size_t)ldg * 4, LEAD);
}
void launch_loss_labels(int n, int H, int, int, int cols, const float *lack, int32_t *lead, const int32_t *, const void *x, const void *, void *dx, void *own, hipStream_t) {
    reach("launch_loss_labels");
    see(lack, (size_t)n * 4, LACK, "lack");
    see(lead, (size_t)cols * 4, LEAD, "lead");
    see(x, (size_t)n * H * 2, xs_mark, "xs");
    put(dx, (size_t)n * H * 2, DXS);
    put(own, (size_t)n * H * 2, OWN);
}
void launch_gemm_nn(int M, int N, int K, const void *A, int lda, const void *, void *C, const void *R, void *ws, size_t ws_bytes, hipStream_t) {
    reach("launch_gemm_nn");
    if (ws) put(ws, ws_bytes, SUMS);
    see(R, (size_t)M * N * 2, DXS, "dx's residual");
    if (ws && ws_bytes < gemm_workspace_bytes(1, M, N, K)) std::abort();
    see(A, (size_t)M * lda * 2, G, "g");
    put(C, (size_t)M * N * 2, DXS);
}
void launch_loss_dw(int M, int N, int K, const void *A, int lda, const void *B, void *C, const void *, const void *own, hipStream_t) {
    reach("launch_loss_dw");
    see(own, (size_t)K * N * 2, OWN, "own");
    see(loss_lead(A, K, lda), (size_t)M * 4, LEAD, "lead");
    see(A, (size_t)K * lda * 2, G, "g");
    see(B, (size_t)K * N * 2, xs_mark, "xs");
    put(C, (size_t)M * N * 2, 0);
}
void launch_gemm_nn_piece(const Plan &p, int M, int, int, const void *A, int lda, const void *, float *part, bool first, hipStream_t) {
    reach("launch_gemm_nn_piece");
    see(A, (size_t)M * lda * 2, G, "g");
    if (!first) see(part, sums_of(p), SUMS, "dx's sums");
    put(part, sums_of(p), SUMS);
}
void launch_gemm_nn_round(const Plan &p, int M, int N, float *part, void *C, const void *R, hipStream_t) {
    reach("launch_gemm_nn_round");
    see(R, (size_t)M * N * 2, DXS, "dx's residual");
    see(part, sums_of(p), SUMS, "dx's sums");
    put(C, (size_t)M * N * 2, DXS);
}
void launch_rows_spread(const void *small, void *big, const int32_t *, int n_rows, int T, int H, hipStream_t) {
    reach("launch_rows_spread");
    if (n_rows) see(small, (size_t)n_rows * H * 2, DXS, "dx's rows");
    put(big, (size_t)T * H * 2, 0);
}
void launch_rows_gather(void *small, const void *, const int32_t *, int n_rows, int H, hipStream_t) {
    reach("launch_rows_gather");
    put(small, (size_t)n_rows * H * 2, xs_mark = XS);
}

void launch_rotary_axes(const void *, int, void *, int, int, int, int, const RotaryTable &, const int32_t *, int, int, hipStream_t) { reach("launch_rotary_axes"); }
void launch_attn_window_fwd(const void *, const void *, const void *, void *, float *, int, int, int, const ob_segments *, int, int, int, float, int, int,
                            hipStream_t) { reach("launch_attn_window_fwd"); }
void launch_attn_window_bwd(const void *, const void *, const void *, const void *, const void *, const float *, float *lse2, float *delta, float *part, void *,
                            void *, void *, int, int, int, const ob_segments *seg, int nq, int nkv, int d, float, int window, int sinks, hipStream_t) {
    reach("launch_attn_window_bwd");
    const size_t rows = (size_t)seg->total_tokens * nq * 4;
    part_begin = part;
    part_bytes = (size_t)sink_chunks(seg, sink_whole_rows(window, nq / nkv), sinks) * nkv * 2 * sinks * d * 4;
    put(lse2, rows, LSE2);
    put(delta, rows, DELTA);
    put(part, part_bytes, PART);
    see(lse2, rows, LSE2, "lse2");
    see(delta, rows, DELTA, "delta");
}

namespace f32 {
size_t lm_loss_work_bytes(int n, int H, int V) { return (size_t)n * ((size_t)H + V) * 4; }
void lm_loss_fwd(const void *, const void *, const int32_t *, int, int, int, const int32_t *, float *, float *, void *, hipStream_t) { reach("f32::lm_loss_fwd"); }
void lm_loss_bwd(const void *, const void *, int, const int32_t *, int, int, int, const int32_t *, const float *, const float *, void *, void *, int, void *,
                 hipStream_t) { reach("f32::lm_loss_bwd"); }
void attn_window_fwd(const void *, const void *, const void *, void *, float *, int, int, int, const ob_segments *, int, int, int, float, int, int,
                     hipStream_t) { reach("f32::attn_window_fwd"); }
void attn_window_bwd(const void *, const void *, const void *, const void *, const void *, const float *, void *, void *, void *, float *delta, int, int, int,
                     const ob_segments *seg, int nq, int, int, float, int, int, hipStream_t) {
    reach("f32::attn_window_bwd");
    put(delta, (size_t)seg->total_tokens * nq * 4, DELTA);
}
void block_steps_fwd(const BlockSteps &, const ob_block_weights *, const void *, void *, void *, const ob_segments *, hipStream_t) { reach("f32::block_steps_fwd"); }
void block_steps_bwd(const BlockSteps &, const ob_block_weights *, const ob_block_grads *, int, const void *, const void *, void *, const void *,
                     const ob_segments *, void *, hipStream_t) { reach("f32::block_steps_bwd"); }
}  // namespace f32
}  // namespace ob

// (nothing is launched: a host without a GPU is no failed launch)
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

// the caller's x, all zeros
void x_is_the_callers() { xs_mark = 0; }
