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

}  // namespace

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
