// C ABI of the rotary positions with several axes: validation, and the table of frequencies.
#include <cmath>

#include "ob_internal.h"

namespace ob {

int rotary_table(const ob_rotary_axes_desc *desc, RotaryTable &table, const char *who) {
    if (!desc) return fail(OB_EINVAL, "%s: desc is null", who);
    if (desc->head_dim != 64 && desc->head_dim != 128) return fail(OB_EUNSUPPORTED, "%s: head_dim %d not in {64, 128}", who, desc->head_dim);
    if (desc->n_axes < 1 || desc->n_axes > OB_ROTARY_MAX_AXES)
        return fail(OB_EINVAL, "%s: n_axes %d outside [1, %d]", who, desc->n_axes, OB_ROTARY_MAX_AXES);
    if (!(desc->base > 1.f) || !std::isfinite(desc->base)) return fail(OB_EINVAL, "%s: base must be a number > 1", who);
    const int half = desc->head_dim / 2;
    int pairs[OB_ROTARY_MAX_AXES] = {};
    for (int i = 0; i < half; ++i) {
        const int a = desc->axis_of_pair[i];
        if (a < -1 || a >= desc->n_axes) return fail(OB_EINVAL, "%s: pair %d has axis %d, must be -1 or below n_axes %d", who, i, a, desc->n_axes);
        if (a >= 0) ++pairs[a];
    }
    // theta / 2 pi in units of 2^-64 of a turn (theta <= 1: at most 0.16 of the range), in the 64 bits of a long double's mantissa.  A spectrum is
    // a geometric sequence: one power, then products (64 of them, 2^-58 of the value: 2e-9 rad at the largest position; a power for each took
    // 13 us of a call, whose launch takes 4).
    const long double turn = ldexpl(0.159154943091895335768883763372514362L, 64), log_base = logl((long double)desc->base);
    const auto ratio_of = [&](int n) { return expl(-log_base / n); };
    long double theta[OB_ROTARY_MAX_AXES], ratio[OB_ROTARY_MAX_AXES], all = turn;
    const long double ratio_all = ratio_of(half);
    for (int a = 0; a < desc->n_axes; ++a) {
        theta[a] = turn;
        ratio[a] = desc->per_axis && pairs[a] > 1 ? ratio_of(pairs[a]) : 1;
    }
    for (int i = 0; i < half; ++i, all *= ratio_all) {
        const int a = desc->axis_of_pair[i];
        table.axis[i] = (int8_t)a;
        table.turn[i] = 0;
        if (a < 0) continue;
        table.turn[i] = (uint64_t)((desc->per_axis ? theta[a] : all) + 0.5L);
        theta[a] *= ratio[a];
    }
    return OB_OK;
}

}  // namespace ob

using namespace ob;

extern "C" int ob_rotary_axes(const ob_rotary_axes_desc *desc, const void *x, int ldx, void *y, int ldy, int total_tokens,
                              int n_heads, const int32_t *pos, int inverse, int dtype, void *hip_stream) {
    const char *who = "ob_rotary_axes";
    RotaryTable table;
    if (int rc = rotary_table(desc, table, who)) return rc;
    if (!x || !y || !pos) return fail(OB_EINVAL, "%s: x / y / pos is null", who);
    if (dtype != OB_BF16 && dtype != OB_FP32) return fail(OB_EINVAL, "%s: unknown dtype %d", who, dtype);
    if (total_tokens < 1 || total_tokens > MAX_TOKENS) return fail(OB_EINVAL, "%s: total_tokens %d outside [1, %d]", who, total_tokens, MAX_TOKENS);
    if (n_heads < 1 || n_heads > OB_ROTARY_MAX_HEADS) return fail(OB_EINVAL, "%s: n_heads %d outside [1, %d]", who, n_heads, OB_ROTARY_MAX_HEADS);
    const int row = n_heads * desc->head_dim;
    if (ldx < row || ldy < row || ldx % 8 || ldy % 8)
        return fail(OB_EINVAL, "%s: row strides must cover the heads and be multiples of 8 elements", who);
    if ((uintptr_t)x % 16 || (uintptr_t)y % 16 || (uintptr_t)pos % 4) return fail(OB_EINVAL, "%s: x and y must be aligned to 16 bytes", who);
    if (x == y && ldx != ldy) return fail(OB_EINVAL, "%s: in place, both row strides must be the same", who);
    launch_rotary_axes(x, ldx, y, ldy, total_tokens, n_heads, desc->head_dim, table, pos, inverse ? 1 : 0, dtype, (hipStream_t)hip_stream);
    return check_launch(who);
}
