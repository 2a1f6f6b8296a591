// Windowed attention with every tensor in fp32: the checking variant of ob_varlen_attn_window_fwd / _bwd, plain fp32 sums, no matrix instructions.
// A wave takes a row (forward, dQ), a workgroup a key (dK / dV); sixteen lanes share a score, four of them to a wave at a time, each lane holding d / 16
// elements, so a score costs four exchanges between lanes instead of a wave's six, and four are on their way together (411 tokens, 4 / 2 heads of 64, window 33:
// a score at a time 20 us forward, 20 dQ, 57 dK / dV).  What the lanes hold is added up once, at the end.
#include <cmath>

#include "ob_internal.h"

namespace ob {
namespace f32 {
namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

// sum over the sixteen lanes of a score, over the wave's four scores
__device__ __forceinline__ float score_sum(float v) {
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float across(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <int E>
struct Part {          // a lane's E elements of a head's row
    float v[E];
    __device__ __forceinline__ Part() {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.f;
    }
    __device__ __forceinline__ explicit Part(const float *p) {
#pragma unroll
        for (int e = 0; e < E; e += 4) *(f32x4 *)(v + e) = *(const f32x4 *)(p + e);
    }
    __device__ __forceinline__ float dot(const Part &o) const {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += v[e] * o.v[e];
        return score_sum(s);
    }
    __device__ __forceinline__ void add(float f, const Part &o) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += f * o.v[e];
    }
    __device__ __forceinline__ void store(float *p, float f) const {
#pragma unroll
        for (int e = 0; e < E; e += 4) *(f32x4 *)(p + e) = f32x4{v[e] * f, v[e + 1] * f, v[e + 2] * f, v[e + 3] * f};
    }
};

__device__ __forceinline__ int segment_of(const int32_t *cu, int n_seg, int t) {
    int lo = 0, hi = n_seg;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

// the keys that row t of a segment from `start` on sees: `front` sinks, then the band
struct Keys {
    int start, front, from, n;
    __device__ __forceinline__ Keys(int t, int start_, int window, int sinks) : start(start_) {
        from = max(start, t - window + 1);
        front = min(sinks, from - start);
        n = front + t - from + 1;
    }
    __device__ __forceinline__ int at(int i) const { return i < front ? start + i : from + i - front; }
};

template <int D>
__global__ __launch_bounds__(256) void window_fwd_kernel(const float *__restrict__ q, const float *__restrict__ k, const float *__restrict__ v,
                                                         float *__restrict__ o, float *__restrict__ lse, int ldq, int ldkv, int ldo,
                                                         const int32_t *__restrict__ cu, int n_seg, int T, int nq, int group, float scale,
                                                         int window, int sinks) {
    constexpr int E = D / 16;
    for (long w = (long)blockIdx.x * 4 + (threadIdx.x >> 6); w < (long)T * nq; w += (long)gridDim.x * 4) {
        const int t = (int)(w / nq), head = (int)(w % nq), lane = threadIdx.x & 63, mine = lane >> 4, col = (lane & 15) * E;
        const Keys keys(t, cu[segment_of(cu, n_seg, t)], window, sinks);
        const float *const kp = k + head / group * D + col, *const vp = v + head / group * D + col;
        const Part<E> qv(q + (size_t)t * ldq + head * D + col);
        Part<E> ov;
        float m = -INFINITY, l = 0.f;
        for (int i = mine; i < (keys.n + 3) / 4 * 4; i += 4) {          // (all four groups as often: they exchange)
            const size_t row = (size_t)keys.at(min(i, keys.n - 1)) * ldkv;
            const Part<E> ke(kp + row), ve(vp + row);
            const float dot = qv.dot(ke);
            if (i >= keys.n) continue;
            const float s = dot * scale, mn = fmaxf(m, s), alpha = expf(m - mn), p = expf(s - mn);
            l = l * alpha + p;
#pragma unroll
            for (int e = 0; e < E; ++e) ov.v[e] = ov.v[e] * alpha + p * ve.v[e];
            m = mn;
        }
        const float top = fmaxf(fmaxf(m, __shfl_xor(m, 16)), fmaxf(__shfl_xor(m, 32), __shfl_xor(m, 48)));
        const float f = m == -INFINITY ? 0.f : expf(m - top);           // (a group without a key)
        const float total = across(l * f);
#pragma unroll
        for (int e = 0; e < E; ++e) ov.v[e] = across(ov.v[e] * f);
        if (mine == 0) ov.store(o + (size_t)t * ldo + head * D + col, 1.f / total);
        if (lane == 0) lse[(size_t)head * T + t] = top + logf(total);
    }
}

// dq[t] = scale sum_j P_tj (dP_tj - delta_t) k_j; leaves delta_t = sum_d dO O for dK / dV
template <int D>
__global__ __launch_bounds__(256) void window_bwd_dq_kernel(const float *__restrict__ d_o, const float *__restrict__ q, const float *__restrict__ k,
                                                            const float *__restrict__ v, const float *__restrict__ o,
                                                            const float *__restrict__ lse, float *__restrict__ delta, float *__restrict__ dq,
                                                            int ldq, int ldkv, int ldo, const int32_t *__restrict__ cu, int n_seg, int T, int nq,
                                                            int group, float scale, int window, int sinks) {
    constexpr int E = D / 16;
    for (long w = (long)blockIdx.x * 4 + (threadIdx.x >> 6); w < (long)T * nq; w += (long)gridDim.x * 4) {
        const int t = (int)(w / nq), head = (int)(w % nq), lane = threadIdx.x & 63, mine = lane >> 4, col = (lane & 15) * E;
        const Keys keys(t, cu[segment_of(cu, n_seg, t)], window, sinks);
        const float *const kp = k + head / group * D + col, *const vp = v + head / group * D + col;
        const Part<E> qv(q + (size_t)t * ldq + head * D + col), go(d_o + (size_t)t * ldo + head * D + col), ov(o + (size_t)t * ldo + head * D + col);
        const float ls = lse[(size_t)head * T + t], dl = go.dot(ov);
        if (lane == 0) delta[(size_t)head * T + t] = dl;
        Part<E> acc;
        for (int i = mine; i < (keys.n + 3) / 4 * 4; i += 4) {
            const size_t row = (size_t)keys.at(min(i, keys.n - 1)) * ldkv;
            const Part<E> ke(kp + row), ve(vp + row);
            const float s = qv.dot(ke), dp = go.dot(ve);
            if (i < keys.n) acc.add(expf(s * scale - ls) * (dp - dl), ke);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) acc.v[e] = across(acc.v[e]);
        if (mine == 0) acc.store(dq + (size_t)t * ldq + head * D + col, scale);
    }
}

// dk[j] = scale sum over the group's heads and the rows that see j of dS q; dv[j] = sum P dO: a workgroup to a key, sixteen rows at a time
template <int D>
__global__ __launch_bounds__(256) void window_bwd_dkv_kernel(const float *__restrict__ d_o, const float *__restrict__ q, const float *__restrict__ k,
                                                             const float *__restrict__ v, const float *__restrict__ lse,
                                                             const float *__restrict__ delta, float *__restrict__ dk, float *__restrict__ dv,
                                                             int ldq, int ldkv, int ldo, const int32_t *__restrict__ cu, int n_seg, int T, int nkv,
                                                             int group, float scale, int window, int sinks) {
    constexpr int E = D / 16;
    __shared__ float sums[4][2][D];
    for (long w = blockIdx.x; w < (long)T * nkv; w += gridDim.x) {
        const int j = (int)(w / nkv), kvh = (int)(w % nkv), lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = (lane & 15) * E;
        const int mine = threadIdx.x >> 4, seg = segment_of(cu, n_seg, j), start = cu[seg];
        const int end = j - start < sinks ? cu[seg + 1] : min(cu[seg + 1], j + window), rows = end - j;
        const Part<E> ke(k + (size_t)j * ldkv + kvh * D + col), ve(v + (size_t)j * ldkv + kvh * D + col);
        Part<E> ak, av;
        for (int head = kvh * group; head < (kvh + 1) * group; ++head)
            for (int i = mine; i < (rows + 15) / 16 * 16; i += 16) {
                const int t = j + min(i, rows - 1);
                const Part<E> qe(q + (size_t)t * ldq + head * D + col), ge(d_o + (size_t)t * ldo + head * D + col);
                const float ls = lse[(size_t)head * T + t], dl = delta[(size_t)head * T + t];
                const float s = qe.dot(ke), dp = ge.dot(ve);
                if (i >= rows) continue;
                const float p = expf(s * scale - ls);
                av.add(p, ge);
                ak.add(p * (dp - dl), qe);
            }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float a = across(ak.v[e]), b = across(av.v[e]);
            if (lane < 16) { sums[wave][0][col + e] = a; sums[wave][1][col + e] = b; }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * D; i += 256) {
            const int which = i / D, c = i % D;
            const float s = sums[0][which][c] + sums[1][which][c] + sums[2][which][c] + sums[3][which][c];
            float *const dst = (which ? dv : dk) + (size_t)j * ldkv + kvh * D + c;
            *dst = which ? s : s * scale;
        }
        __syncthreads();
    }
}

// (a launch has fewer than 2^32 threads: beyond, workgroups take several)
inline unsigned blocks_of(long n) { return (unsigned)(n < (1 << 22) ? n : 1 << 22); }

}  // namespace

#define OB_BY_SIZE(KERNEL, GRID, ...)                                                            \
    do {                                                                                         \
        if (d == 64) hipLaunchKernelGGL((KERNEL<64>), dim3(GRID), dim3(256), 0, s, __VA_ARGS__); \
        else hipLaunchKernelGGL((KERNEL<128>), dim3(GRID), dim3(256), 0, s, __VA_ARGS__);        \
    } while (0)

void attn_window_fwd(const void *q, const void *k, const void *v, void *o, float *lse, int ldq, int ldkv, int ldo,
                     const ob_segments *seg, int nq, int nkv, int d, float scale, int window, int sinks, hipStream_t s) {
    const int T = seg->total_tokens;
    OB_BY_SIZE(window_fwd_kernel, blocks_of(((long)T * nq + 3) / 4), (const float *)q, (const float *)k, (const float *)v, (float *)o, lse, ldq, ldkv, ldo,
               seg->cu_dev, seg->n_seg, T, nq, nq / nkv, scale, window, sinks);
}

void attn_window_bwd(const void *d_o, const void *q, const void *k, const void *v, const void *o, const float *lse,
                     void *dq, void *dk, void *dv, float *delta, int ldq, int ldkv, int ldo, const ob_segments *seg, int nq,
                     int nkv, int d, float scale, int window, int sinks, hipStream_t s) {
    const int T = seg->total_tokens;
    OB_BY_SIZE(window_bwd_dq_kernel, blocks_of(((long)T * nq + 3) / 4), (const float *)d_o, (const float *)q, (const float *)k, (const float *)v,
               (const float *)o, lse, delta, (float *)dq, ldq, ldkv, ldo, seg->cu_dev, seg->n_seg, T, nq, nq / nkv, scale, window, sinks);
    OB_BY_SIZE(window_bwd_dkv_kernel, blocks_of((long)T * nkv), (const float *)d_o, (const float *)q, (const float *)k, (const float *)v, lse,
               delta, (float *)dk, (float *)dv, ldq, ldkv, ldo, seg->cu_dev, seg->n_seg, T, nkv, nq / nkv, scale, window, sinks);
}

}  // namespace f32
}  // namespace ob
