// Rotary positions with several axes (time, height, width ...): every pair (i, i + d/2) of a head turns by the position
// of its token along the pair's own axis,
//   y_i = x_i cos a - x_{i+d/2} sin a,   y_{i+d/2} = x_{i+d/2} cos a + x_i sin a,   a = pos[axis(i), t] theta_i
// (the gradient turns back by the same angles).  A pair of axis -1 passes as it is.
//
// The angle: theta_i / 2 pi comes from the host as a 64-bit fraction of a turn, and position x fraction modulo 2^64 drops
// the whole turns exactly, for every 32-bit position; its nearest multiple of 2^-32 of a turn is off by 7.3e-10 rad.  A float has 24 bits of that: the
// sine and cosine of the nearest multiple of 2^-25 of a turn, which a float holds exactly, are turned on by the rest, at most 9.4e-8 rad (whose square is lost in
// any float).  In floating point a position of a million keeps two digits of its angle in 32 bits.
//
// Bound by memory: each value is read and written once.  The sines and cosines of a token are the same for all its heads: a workgroup
// works them out once per token and pair into LDS and walks the token's heads with them.
#include "ob_internal.h"

namespace ob {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

namespace {

constexpr int THREADS = 256, MAX_HALF = 64;
constexpr int TOKENS = 4;      // tokens per workgroup

// (a pair of axis -1 has a cosine that no angle has)
constexpr float PASSES = 2.f;

template <class V, class E, int N>
__device__ __forceinline__ void turn(const V a, const V b, const float2 *cs, V &ya, V &yb) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float c = cs[e].x, s = cs[e].y, fa = (float)a[e], fb = (float)b[e];
        const bool pass = c == PASSES;
        ya[e] = pass ? a[e] : (E)(fa * c - fb * s);
        yb[e] = pass ? b[e] : (E)(fb * c + fa * s);
    }
}

// V: 16 bytes of N elements E.  x and y may be the same tensor: a thread reads what it writes, and nothing else.  STREAM: results that do not fit the L2s beside x are
// stored past them, smaller ones stay for their reader.  Tensors that no call has touched before, 40 heads of 128, through the L2s and past them: 16327 tokens (334 MB)
// 66.6 and 63.3 us (5.3 TB/s; the same tensors again and again 63.3 and 51.0), 4096 18.5 and 18.0, 2048 11.5 and 10.9, 1024 (below the limit) 9.0 and 8.6.  With the
// windowed attention behind it in a block, the two together: 16327 tokens 380.3 and 379.5 us, 4096 100.4 and 99.5, 2048 52.6 and 53.8.  An elementwise pass that reads the
// results at once loses up to 8 % (16327 tokens, both launches: 121 and 131).
template <class V, class E, int N, bool STREAM>
__global__ __launch_bounds__(THREADS) void rotary_axes_kernel(const E *x, int ldx, E *y, int ldy, int T, int n_heads, int half,
                                                              RotaryTable table, const int32_t *__restrict__ pos, int inverse) {
    __shared__ float2 cs[TOKENS * MAX_HALF];
    const int t0 = blockIdx.x * TOKENS, n_tok = min(TOKENS, T - t0);
    for (int i = threadIdx.x; i < n_tok * half; i += THREADS) {
        const int t = i / half, p = i - t * half, axis = table.axis[p];
        float2 v{PASSES, 0.f};
        if (axis >= 0) {
            const uint64_t turns = (uint64_t)(int64_t)pos[(size_t)axis * T + t0 + t] * table.turn[p];
            const uint32_t angle = (uint32_t)((turns + 0x80000000u) >> 32), coarse = (angle + 64u) & ~127u;      // (modulo a turn)
            float sine, cosine;
            sincospif((float)(int32_t)coarse * 0x1p-31f, &sine, &cosine);
            const float rest = (float)(int32_t)(angle - coarse) * 0x1.921fb6p-30f;      // x pi / 2^31
            v = float2{cosine - rest * sine, sine + rest * cosine};
            if (inverse) v.y = -v.y;
        }
        cs[t * half + p] = v;
    }
    __syncthreads();
    const int groups = half / N, per_token = n_heads * groups;
    for (int i = threadIdx.x; i < n_tok * per_token; i += THREADS) {
        const int t = i / per_token, r = i - t * per_token, head = r / groups, p = (r - head * groups) * N;
        const E *src = x + (size_t)(t0 + t) * ldx + head * 2 * half + p;
        E *dst = y + (size_t)(t0 + t) * ldy + head * 2 * half + p;
        const V a = *(const V *)src, b = *(const V *)(src + half);
        V ya, yb;
        turn<V, E, N>(a, b, cs + t * half + p, ya, yb);
        if constexpr (STREAM) {
            __builtin_nontemporal_store(ya, (V *)dst);
            __builtin_nontemporal_store(yb, (V *)(dst + half));
        } else {
            *(V *)dst = ya;
            *(V *)(dst + half) = yb;
        }
    }
}

}  // namespace

void launch_rotary_axes(const void *x, int ldx, void *y, int ldy, int T, int n_heads, int d, const RotaryTable &table,
                        const int32_t *pos, int inverse, int dtype, hipStream_t s) {
    const int half = d / 2, size = dtype == OB_FP32 ? 4 : 2;
    ProfScope prof(K_ROTARY, s, 2.0 * size * T * n_heads * d);
    const dim3 grid((T + TOKENS - 1) / TOKENS);
    const bool stream = 2 * (size_t)T * n_heads * d * size >= (size_t)32 << 20;      // x and y against the eight L2s of 4 MB
#define OB_LAUNCH(V, E, N, STREAM)                                                                                                              \
    hipLaunchKernelGGL((rotary_axes_kernel<V, E, N, STREAM>), grid, dim3(THREADS), 0, s, (const E *)x, ldx, (E *)y, ldy, T, n_heads, half, table, \
                       pos, inverse)
    if (dtype == OB_FP32 && stream) OB_LAUNCH(f32x4, float, 4, true);
    else if (dtype == OB_FP32) OB_LAUNCH(f32x4, float, 4, false);
    else if (stream) OB_LAUNCH(bf16x8, __bf16, 8, true);
    else OB_LAUNCH(bf16x8, __bf16, 8, false);
#undef OB_LAUNCH
}

}  // namespace ob
