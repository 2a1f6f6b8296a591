// Host-only driver of the language side (rotary axes, windowed attention, the cross entropy over a vocabulary, blocks with these in their attention) for the
// AddressSanitizer / UBSan build: every entry point on buffers of exactly the bytes that the size queries report, with stand-in launchers that touch all that the
// kernels touch, and its refusals, which come before any launch.  Exits 0 when every check holds.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <vector>

#include "../../include/omnibal.h"
#include "../../paper_2407_20761_amd/csrc/attention_plan.h"
#include "../../paper_2407_20761_amd/csrc/ob_internal.h"

extern bool launches_pass;
extern const void *part_begin;
extern size_t part_bytes;
extern int launches;
void x_is_the_callers();

static int failures = 0;
#define CHECK(cond)                                                            \
    do {                                                                       \
        if (!(cond)) { std::fprintf(stderr, "%s:%d: CHECK(%s) failed: %s\n", __FILE__, __LINE__, #cond, ob_last_error()); ++failures; } \
    } while (0)

// exactly `bytes` of memory, aligned to 16
struct Buffer {
    unsigned char *p;
    explicit Buffer(size_t bytes, int fill = 255) : p((unsigned char *)std::malloc(bytes ? bytes : 1)) { for (size_t i = 0; i < bytes; ++i) p[i] = (unsigned char)fill; }
    ~Buffer() { std::free(p); }
    Buffer(const Buffer &) = delete;
    operator void *() const { return p; }
    template <class T> T *as() const { return (T *)p; }
};

static ob_segments segments(std::vector<int32_t> &cu, const std::vector<int> &lens) {
    cu.assign(1, 0);
    int longest = 0;
    for (int n : lens) { cu.push_back(cu.back() + n); longest = n > longest ? n : longest; }
    return ob_segments{cu.data(), cu.data(), (int)lens.size(), cu.back(), longest};
}

static void loss_cases() {
    launches_pass = true;
    // (tokens, supervised rows, hidden, vocabulary): one token, ragged sizes, a whole number of tiles, split products, two pieces
    struct Case { int T, n, H, V; };
    for (const Case &c : std::initializer_list<Case>{{1, 1, 64, 1}, {3, 2, 64, 2}, {70, 70, 128, 65}, {129, 64, 320, 257}, {300, 299, 192, 1009}, {256, 256, 64, 256},
                                                     {40, 33, 4096, 8200}, {600, 513, 64, 30011}, {4100, 4100, 64, 131080}, {4400, 4099, 128, 131080}}) {
        const ob_lm_loss_desc d{c.H, c.V, OB_BF16};
        const size_t bytes = ob_lm_loss_workspace_bytes(&d, c.n);
        std::printf("loss %d %d %d %zu\n", c.H, c.V, c.n, bytes);
        std::vector<int32_t> rows(c.n), labels(c.n, 0);
        for (int i = 0; i < c.n; ++i) rows[i] = c.T - c.n + i;
        const bool list = c.n < c.T;
        Buffer ws(bytes), x((size_t)c.T * c.H * 2, 0), dx((size_t)c.T * c.H * 2), w((size_t)c.V * c.H * 2), dw((size_t)c.V * c.H * 2), nll(c.n * 4), lse(c.n * 4), dnll(c.n * 4);
        const int32_t *host = list ? rows.data() : nullptr;
        x_is_the_callers();
        CHECK(ob_lm_loss_fwd(&d, w, x, c.T, host, host, c.n, labels.data(), nll.as<float>(), lse.as<float>(), ws, bytes, nullptr) == OB_OK);
        for (int flags : {0, (int)OB_BWD_ACCUMULATE})
            CHECK(ob_lm_loss_bwd(&d, flags, w, x, c.T, host, host, c.n, labels.data(), lse.as<float>(), dnll.as<float>(), dx, dw, ws, bytes, nullptr) == OB_OK);
        CHECK(ob_lm_loss_fwd(&d, w, x, c.T, host, host, c.n, labels.data(), nll.as<float>(), lse.as<float>(), ws, bytes - 1, nullptr) == OB_EWORKSPACE);
        ob_lm_loss_launch plan;
        CHECK(ob_lm_loss_plan(&d, c.n, &plan) == OB_OK && (plan.pieces > 1) == (plan.dx_tile > 0) && plan.pieces == ((size_t)c.n * c.V * 2 > 1u << 30 ? 2 : 1));
        // no row is supervised: dx and dw are zeros
        const int before = launches;
        CHECK(ob_lm_loss_bwd(&d, 0, w, x, c.T, host, host, 0, nullptr, nullptr, nullptr, dx, dw, nullptr, 0, nullptr) == OB_OK && launches == before + 2);
    }
    // the largest sizes: a layout is there, and none of its sums overflows
    for (int V : {1, 255, 256, 257, 1 << 17, 1 << 21})
        for (int n : {1, 255, 65537, 1 << 18, 1 << 22})
            for (int H : {64, 8192}) {
                const ob_lm_loss_desc d{H, V, OB_BF16};
                const size_t bytes = ob_lm_loss_workspace_bytes(&d, n);
                CHECK(((long)n * V <= 1l << 39) == (bytes > 0) && (!bytes || bytes >= (size_t)n * H * 2));
            }
    launches_pass = false;
    const ob_lm_loss_desc d{64, 100, OB_BF16};
    void *p = (void *)0x1000;
    int32_t up[3] = {0, 2, 4}, twice[3] = {0, 2, 2};
    auto fwd = [&](const int32_t *rows, int n, size_t bytes) {
        return ob_lm_loss_fwd(&d, p, p, 5, rows, (const int32_t *)p, n, (const int32_t *)p, (float *)p, (float *)p, p, bytes, nullptr);
    };
    CHECK(fwd(twice, 3, 1 << 20) == OB_EINVAL && fwd(up, 6, 1 << 20) == OB_EINVAL && fwd(up, -1, 1 << 20) == OB_EINVAL && fwd(up, 3, 0) == OB_EWORKSPACE);
    CHECK(ob_lm_loss_workspace_bytes(nullptr, 3) == 0 && ob_lm_loss_plan(&d, 3, nullptr) == OB_EINVAL);
}

static void window_cases() {
    std::vector<int32_t> cu;
    std::vector<int> many(300, 20);
    for (int i = 0; i < 70; ++i) many.push_back(200);
    const std::vector<std::vector<int>> batches = {{1}, {5, 1, 64}, {1100}, {5000, 30, 2500, 4097, 4096}, many};
    for (const auto &lens : batches) {
        const ob_segments seg = segments(cu, lens);
        for (int d : {64, 128})
            for (int group : {1, 4, 16})
                for (int window : {1, 8, 700, INT_MAX})
                    for (int sinks : {0, 1, 33, 64}) {
                        const int nq = 2 * group, nkv = 2;
                        const size_t bytes = ob_varlen_attn_window_bwd_workspace_bytes(&seg, nq, nkv, d, window, sinks, OB_BF16);
                        ob_attn_bwd_launch launch;
                        int threads, chunks;
                        CHECK(ob_varlen_attn_window_bwd_plan(&seg, nq, nkv, d, window, sinks, &launch, &threads, &chunks) == OB_OK);
                        Buffer ws(bytes);
                        launches_pass = true;
                        void *p = ws;
                        auto bwd = [&](size_t n, int dtype) {
                            return ob_varlen_attn_window_bwd(p, p, p, p, p, (const float *)p, p, p, p, nq * d, nkv * d, nq * d, &seg, nq, nkv, d, 0.1f, window, sinks, dtype,
                                                             ws, n, nullptr);
                        };
                        CHECK(bwd(bytes, OB_BF16) == OB_OK && part_bytes == (size_t)chunks * nkv * 2 * sinks * d * 4);
                        CHECK(bwd(bytes - 1, OB_BF16) == OB_EWORKSPACE);
                        CHECK(bwd(ob_varlen_attn_window_bwd_workspace_bytes(&seg, nq, nkv, d, window, sinks, OB_FP32), OB_FP32) == OB_OK);
                        launches_pass = false;
                        if (d == 64 && sinks == 33) std::printf("window %d %d %d %d %zu\n", (int)(&lens - &batches[0]), nq, window, chunks, bytes);
                    }
    }
    const ob_segments seg = segments(cu, {5, 4});
    void *p = (void *)0x1000;
    auto fwd = [&](int window, int sinks, float scale) {
        return ob_varlen_attn_window_fwd(p, p, p, p, (float *)p, 128, 64, 128, &seg, 2, 1, 64, scale, window, sinks, OB_BF16, nullptr);
    };
    CHECK(fwd(0, 0, 1.f) == OB_EINVAL && fwd(INT_MIN, 0, 1.f) == OB_EINVAL && fwd(1, INT_MIN, 1.f) == OB_EINVAL && fwd(1, INT_MAX, 1.f) == OB_EUNSUPPORTED);
    CHECK(fwd(1, 0, NAN) == OB_EINVAL && fwd(1, 0, 0.f) == OB_EINVAL && fwd(1, 0, INFINITY) == OB_EINVAL);
}

// Every place of a launch in the order of its work is a tile, and every tile has one
static void order_cases() {
    std::vector<int32_t> cu;
    uint64_t st = 7;
    for (int t = 0; t < 60; ++t) {
        std::vector<int> lens;
        for (int i = 0, n = 1 + (int)((st = st * 6364136223846793005ull + 1442695040888963407ull) >> 33) % 40; i < n; ++i)
            lens.push_back(1 + (int)((st = st * 6364136223846793005ull + 1442695040888963407ull) >> 33) % (t % 3 ? 500 : 9000));
        const ob_segments seg = segments(cu, lens);
        for (int window : {1, 100, 4096})
            for (int rows : {64, 128})
                for (bool kv : {false, true}) {
                    ob::TileOrder ord;
                    const int places = ob::make_order(&seg, rows, true, kv, ord, window, kv ? ob::sink_whole_rows(window, 4) : 0);
                    long tiles = 0;
                    for (int n : lens) tiles += (n + rows - 1) / rows;
                    if (ord.n == 0) { CHECK(places == tiles); continue; }
                    std::vector<char> seen(tiles, 0);
                    long found = 0;
                    for (int rank = 0; rank < places; ++rank) {
                        const uint32_t e = ord.e[rank >> ord.unit_log2];
                        const int j = (int)(e >> 16), tile = ob::tile_of_rank(ord, e, rank);
                        if (tile * rows >= lens[j]) continue;
                        long first = 0;
                        for (int i = 0; i < j; ++i) first += (lens[i] + rows - 1) / rows;
                        CHECK(!seen[first + tile]);
                        seen[first + tile] = 1;
                        ++found;
                    }
                    CHECK(found == tiles);
                }
    }
}

static void rotary_cases() {
    ob_rotary_axes_desc d{128, 3, 10000.f, 0, {}};
    for (int i = 0; i < 64; ++i) d.axis_of_pair[i] = (int8_t)(i % 4 - 1);
    // the table: theta / 2 pi in units of 2^-64
    for (int per_axis : {0, 1})
        for (float base : {1.0001f, 10.f, 10000.f, 1e6f, 3e38f})
            for (int hd : {64, 128}) {
                ob::RotaryTable table;
                d.head_dim = hd; d.base = base; d.per_axis = per_axis;
                CHECK(ob::rotary_table(&d, table, "table") == OB_OK);
                int place[3] = {}, count[3] = {};
                for (int i = 0; i < hd / 2; ++i)
                    if (d.axis_of_pair[i] >= 0) ++count[d.axis_of_pair[i]];
                for (int i = 0; i < hd / 2; ++i) {
                    const int a = d.axis_of_pair[i];
                    CHECK(table.axis[i] == a);
                    if (a < 0) { CHECK(table.turn[i] == 0); continue; }
                    const long double power = per_axis ? (long double)place[a]++ / count[a] : 2.0L * i / hd;
                    const long double want = powl((long double)base, -power) * 0.159154943091895335768883763372514362L * 18446744073709551616.0L;
                    // (a unit is 7.3e-10 rad at the largest position)
                    CHECK(fabsl((long double)table.turn[i] - want) <= 3.0L + 3e-18L * want);
                }
            }
    void *p = (void *)0x1000;
    d.head_dim = 128; d.base = 10000.f;
    auto call = [&](const void *x, int ldx, int T, int heads) { return ob_rotary_axes(&d, x, ldx, p, 256, T, heads, (const int32_t *)p, 0, OB_BF16, nullptr); };
    CHECK(call(nullptr, 256, 4, 2) == OB_EINVAL && call(p, 248, 4, 2) == OB_EINVAL && call(p, 256, 0, 2) == OB_EINVAL && call(p, 256, 4, INT_MAX) == OB_EINVAL);
    launches_pass = true;
    CHECK(call(p, 256, 1 << 22, 2) == OB_OK);
    launches_pass = false;
    d.axis_of_pair[63] = 3;
    CHECK(call(p, 256, 4, 2) == OB_EINVAL);
    d.axis_of_pair[63] = -128;
    CHECK(call(p, 256, 4, 2) == OB_EINVAL);
}

static void block_cases() {
    std::vector<int32_t> cu;
    ob_rotary_axes_desc rotary{64, 2, 10000.f, 0, {}};
    for (const auto &lens : std::vector<std::vector<int>>{{9}, {1700}, {40, 1, 2300}}) {
        const ob_segments seg = segments(cu, lens);
        for (int dtype : {OB_BF16, OB_FP32})
            for (int window : {0, 1, 100})
                for (int sinks : {0, 16}) {
                    if (!window && sinks) continue;
                    const ob_block_desc d{128, 8, 1, 64, 128, OB_RMSNORM, OB_SWIGLU, OB_MASK_SEG_CAUSAL, dtype, 0, 10000.f, 1e-5f, 0};
                    const ob_block_attn attn{window, sinks, window ? &rotary : nullptr, window ? (const int32_t *)cu.data() : nullptr};
                    const size_t bytes = ob_block_attn_workspace_bytes(&d, &attn, &seg), own = ob_block_workspace_bytes(&d, seg.total_tokens);
                    const size_t sb = ob_block_saved_bytes(&d, seg.total_tokens);
                    CHECK(bytes >= own && own > 0);
                    Buffer ws(bytes), saved(sb);
                    void *p = saved;
                    ob_block_weights w{p, p, p, p, p, p, p, p, p, p, p, p};
                    ob_block_grads g{p, p, p, p, p, p, p, p, p, p, p, p};
                    launches_pass = true;
                    part_begin = nullptr;
                    CHECK(ob_block_attn_fwd(&d, &attn, &w, p, p, saved, sb, &seg, ws, own, nullptr) == OB_OK);
                    CHECK(ob_block_attn_bwd(&d, &attn, &w, &g, 0, p, p, p, saved, sb, &seg, ws, bytes, nullptr) == OB_OK);
                    // the sinks' sums lie behind the block's own workspace
                    if (window && dtype == OB_BF16) CHECK(part_begin == ws.p + (own + 255) / 256 * 256 && (size_t)((const unsigned char *)part_begin - ws.p) + part_bytes <= bytes);
                    launches_pass = false;
                    CHECK(ob_block_attn_bwd(&d, &attn, &w, &g, 0, p, p, p, saved, sb, &seg, ws, bytes - 1, nullptr) == OB_EWORKSPACE);
                    if (dtype == OB_BF16) std::printf("attn %d %d %d %zu\n", window, sinks, seg.total_tokens, bytes);
                }
    }
    const ob_segments seg = segments(cu, {9});
    const ob_block_desc d{128, 8, 1, 64, 128, OB_RMSNORM, OB_SWIGLU, OB_MASK_SEG_CAUSAL, OB_BF16, 0, 10000.f, 1e-5f, 0};
    for (const ob_block_attn &bad : {ob_block_attn{-1, 0, nullptr, nullptr}, ob_block_attn{INT_MIN, 0, nullptr, nullptr}, ob_block_attn{5, 65, nullptr, nullptr},
                                     ob_block_attn{0, 1, nullptr, nullptr}, ob_block_attn{5, 0, &rotary, nullptr}})
        CHECK(ob_block_attn_workspace_bytes(&d, &bad, &seg) == 0);
    CHECK(ob_block_attn_workspace_bytes(nullptr, nullptr, nullptr) == 0);
}

int main() {
    rotary_cases();
    order_cases();
    window_cases();
    block_cases();
    loss_cases();
    if (failures) { std::fprintf(stderr, "%d checks failed\n", failures); return 1; }
    std::puts("host sanitizer driver: all checks passed");
    return 0;
}
