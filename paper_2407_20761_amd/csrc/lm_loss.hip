// Row kernels of the cross entropy over a vocabulary: what stands between its matrix products (gemm.hip).
//   lse_r = log sum_v exp z_rv from the maxima and sums of the vocabulary's parts;  nll_r = lse_r - z_r,label
// All are bound by memory and small beside the products.
#include <cmath>

#include "ob_internal.h"

namespace ob {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// sums of exp(z - m) of two parts, as one
__device__ __forceinline__ void join(float &m, float &sum, float m2, float sum2) {
    if (sum2 == 0.f) return;                       // (a part without columns: its maximum is -infinity)
    const float top = fmaxf(m, m2);
    sum = (sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f((m - top) * LOG2E)) + sum2 * __builtin_amdgcn_exp2f((m2 - top) * LOG2E);
    m = top;
}

// ROWS rows to a workgroup, 256 / ROWS threads to a row, each every (256 / ROWS)-th part, eight of them in flight; stats [slots][n], so the rows of a
// part are read together
template <int ROWS>
__global__ __launch_bounds__(256) void loss_combine_kernel(const float2 *__restrict__ stats, const float *__restrict__ target,
                                                           const int32_t *__restrict__ labels, int n, int V, int slots,
                                                           float *__restrict__ nll, float *__restrict__ lse) {
    constexpr int PER = 256 / ROWS, AHEAD = 8;
    __shared__ float2 sh[PER][ROWS + 1];
    const int r = threadIdx.x % ROWS, row = blockIdx.x * ROWS + r, lane = threadIdx.x / ROWS;
    float m = -INFINITY, sum = 0.f;
    if (row < n) {
        for (int i = lane; i < slots; i += PER * AHEAD) {
            float2 p[AHEAD];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int at = i + a * PER;
                p[a] = stats[(size_t)min(at, slots - 1) * n + row];
                if (at >= slots) p[a].y = 0.f;
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) join(m, sum, p[a].x, p[a].y);
        }
    }
    sh[lane][r] = float2{m, sum};
    // pairs of threads, of pairs, ...: always the same order
#pragma unroll
    for (int half = PER / 2; half >= 1; half /= 2) {
        __syncthreads();
        if (lane < half) {
            join(m, sum, sh[lane + half][r].x, sh[lane + half][r].y);
            sh[lane][r] = float2{m, sum};
        }
    }
    if (lane != 0 || row >= n) return;
    const float l = m + logf(sum);
    const int label = labels[row];
    lse[row] = l;
    nll[row] = label >= 0 && label < V ? l - target[row] : 0.f;
}

// one wave to a row of `big`: its place in the list by bisection.  Stored past the caches (402 MB of rows of 6144, a quarter of them read: 103 us through them, 68)
__global__ __launch_bounds__(256) void rows_spread_kernel(const __bf16 *__restrict__ small, __bf16 *__restrict__ big,
                                                          const int32_t *__restrict__ rows, int n_rows, int T, int H) {
    const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= T) return;
    int lo = 0, hi = n_rows;                       // the first row of the list that is not below t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (rows[mid] < t) lo = mid + 1; else hi = mid;
    }
    const bool listed = lo < n_rows && rows[lo] == t;
    for (int c = (threadIdx.x & 63) * 8; c < H; c += 512) {
        bf16x8 v = {};
        if (listed) v = *(const bf16x8 *)(small + (size_t)lo * H + c);
        __builtin_nontemporal_store(v, (bf16x8 *)(big + (size_t)t * H + c));
    }
}

// The label's entry of a row of G is most of that row of dx and, with the others of its label, of a row of dw: rounded to bf16 it scales them by up to 2^-8, all
// of them alike where the weights are (dnll of 1 / 1020 for every row: dx and dw 0.0042 off, 0.0017 with this).  So what its rounding took, `lack` in fp32, goes into
// the products' epilogues: dx[r] = lack_r W[label], the residual of G W, and for the first row r of every label own[r] = sum of lack x over its rows (r, then the others
// in order), which the epilogue of G^T x finds by lead[column] = r.  bf16 will do for both, 2^-8 of what is lost.
// A workgroup to a row; it looks for an earlier row of its label first.  Bound by the labels that it reads out of the L2, n times the fewer of n and V (8185 rows, 131072 x
// 6144: 126 us of the step's 35.7 ms; 3271 rows, 65536 x 4096: 31 of 5.2; 40000 rows, 50000 x 1024: 0.79 of 16), and by the first row of a label that many share,
// whose workgroup adds them all up (4 % of those 8185 rows one label: 0.2 ms more, 30 %: 1.3).
constexpr int LABEL_SCAN = 2048, LABEL_VECS = 4;      // (LABEL_VECS vectors of 8 columns to a thread: rows of up to 8192)
__global__ __launch_bounds__(256) void loss_labels_kernel(int n, int H, int V, int first, int cols, const float *__restrict__ lack, int32_t *__restrict__ lead,
                                                          const int32_t *__restrict__ labels, const __bf16 *__restrict__ x, const __bf16 *__restrict__ w,
                                                          __bf16 *__restrict__ dx, __bf16 *__restrict__ own) {
    constexpr int PER = LABEL_SCAN / 256, AHEAD = 8;
    __shared__ uint64_t mask[PER][4];
    __shared__ int list[LABEL_SCAN];
    __shared__ float sums[256][8];
    const int r = blockIdx.x, label = labels[r], tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // narrow rows: `groups` of threads take rows in turns
    const int span = min(256, H / 8), groups = 256 / span, group = tid / span, c0 = (tid - group * span) * 8;
    if (label < 0 || label >= V) {
        if (first == 0 && group == 0)
            for (int c = c0; c < H; c += 2048) *(bf16x8 *)(dx + (size_t)r * H + c) = bf16x8{};
        return;
    }
    if (label < first || label - first >= cols) return;
    const float mine = lack[r];
    if (group == 0)
        for (int c = c0; c < H; c += 2048) {
            const bf16x8 v = *(const bf16x8 *)(w + (size_t)(label - first) * H + c);
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (__bf16)(mine * (float)v[e]);
            *(bf16x8 *)(dx + (size_t)r * H + c) = o;
        }
    for (int i0 = 0; i0 < r; i0 += 2 * LABEL_SCAN) {
        int same = 0;
#pragma unroll
        for (int k = 0; k < 2 * PER; ++k) {
            const int i = i0 + k * 256 + tid;
            same |= labels[min(i, r)] == label && i < r;
        }
        if (__syncthreads_or(same)) return;
    }
    float acc[LABEL_VECS][8] = {};
    for (int i0 = r; i0 < n; i0 += LABEL_SCAN) {
        bool hit[PER];
        int any = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = i0 + k * 256 + tid;
            hit[k] = labels[min(i, n - 1)] == label && i < n;
            any |= hit[k];
        }
        if (!__syncthreads_or(any)) continue;  // (also: the list of the rows before is done with)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint64_t m = __ballot(hit[k]);
            if (lane == 0) mask[k][wave] = m;
        }
        __syncthreads();
        int count = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const uint64_t m = mask[k][v];
                if (v == wave && hit[k]) list[count + __popcll(m & ((1ull << lane) - 1))] = i0 + k * 256 + tid;
                count += __popcll(m);
            }
        __syncthreads();
        // the rows in turns of the groups, AHEAD of them on their way
#pragma unroll
        for (int vec = 0; vec < LABEL_VECS; ++vec) {
            const int c = c0 + vec * 2048;
            if (c >= H || group >= groups) break;
            for (int at = group; at < count; at += groups * AHEAD) {
                bf16x8 v[AHEAD];
                float f[AHEAD];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    const int row = list[min(at + a * groups, count - 1)];
                    f[a] = lack[row];
                    v[a] = *(const bf16x8 *)(x + (size_t)row * H + c);
                }
#pragma unroll
                for (int a = 0; a < AHEAD; ++a)
                    if (at + a * groups < count) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[vec][e] += f[a] * (float)v[a][e];
                    }
            }
        }
    }
    if (groups > 1) {                          // (one vector to a thread)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[tid][e] = acc[0][e];
        __syncthreads();
        for (int g = 1; g < groups && group == 0; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[0][e] += sums[g * span + tid][e];
    }
    if (group != 0) return;                    // (threads of no group among them)
#pragma unroll
    for (int vec = 0; vec < LABEL_VECS; ++vec) {
        const int c = c0 + vec * 2048;
        if (c >= H) break;
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (__bf16)acc[vec][e];
        *(bf16x8 *)(own + (size_t)r * H + c) = o;
    }
    if (tid == 0) lead[label - first] = r;
}

}  // namespace

void launch_loss_labels(int n, int H, int V, int first, int cols, const float *lack, int32_t *lead, const int32_t *labels, const void *x, const void *w,
                        void *dx, void *own, hipStream_t s) {
    ProfScope prof(K_ROWS, s, 8.0 * n * H);
    hipLaunchKernelGGL(loss_labels_kernel, dim3(n), dim3(256), 0, s, n, H, V, first, cols, lack, lead, labels, (const __bf16 *)x, (const __bf16 *)w, (__bf16 *)dx,
                       (__bf16 *)own);
}
void launch_loss_combine(const void *stats, const float *target, const int32_t *labels, int n, int V, int slots, float *nll, float *lse,
                         hipStream_t s) {
    ProfScope prof(K_REDUCE, s, 8.0 * n * slots);
    // few rows: more threads to each
    if (n <= 2048)
        hipLaunchKernelGGL((loss_combine_kernel<4>), dim3((n + 3) / 4), dim3(256), 0, s, (const float2 *)stats, target, labels, n, V, slots, nll, lse);
    else
        hipLaunchKernelGGL((loss_combine_kernel<16>), dim3((n + 15) / 16), dim3(256), 0, s, (const float2 *)stats, target, labels, n, V, slots, nll, lse);
}
void launch_rows_spread(const void *small, void *big, const int32_t *rows_dev, int n_rows, int T, int H, hipStream_t s) {
    ProfScope prof(K_ROWS, s, 2.0 * H * ((double)T + n_rows));
    hipLaunchKernelGGL(rows_spread_kernel, dim3((T + 3) / 4), dim3(256), 0, s, (const __bf16 *)small, (__bf16 *)big, rows_dev, n_rows, T, H);
}

}  // namespace ob
