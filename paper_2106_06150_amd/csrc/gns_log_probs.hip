// Log probabilities of given classes, entropy and best classes of rows of logits, and the gradient of the first two.
#include "gns_learn.hpp"

namespace gns {

// A value's place in the order of all values: larger floats have larger keys, and of equal ones (0 and -0 too) the lower index.
__device__ __forceinline__ uint64_t order_key(float z, int32_t index)
{
    const uint32_t b = __float_as_uint(z + 0.f);
    return (uint64_t) (b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t) ~index;
}

template <typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, V* smem, Op op)
{
    for (int off = 32; off; off >>= 1) v = op(v, __shfl_xor(v, off));
    __syncthreads();
    if (lane_id() == 0) smem[threadIdx.x >> 6] = v;
    __syncthreads();
    v = smem[0];
    for (int w = 1; w < kBlock / kWave; ++w) v = op(v, smem[w]);
    return v;
}

// A block per row; a pass for the maximum, one for the sums and one per best class.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_log_probs(LogProbsArgs a)
{
    __shared__ float s_f[kBlock / kWave];
    __shared__ unsigned long long s_key[kBlock / kWave];
    const int32_t rows = a.count.get(), C = a.logits.width;
    auto add = [](float x, float y) { return x + y; };
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        float m = -__builtin_inff(), bad = 0.f;
        for (int32_t j = (int32_t) threadIdx.x; j < C; j += kBlock) {
            const float z = load_at<T>(a.logits, r, j);
            if (!(z < __builtin_inff())) bad = 1.f;
            m = fmaxf(m, z);
        }
        m = block_reduce(m, s_f, [](float x, float y) { return fmaxf(x, y); });
        bad = block_reduce(bad, s_f, add);
        const bool none = m == -__builtin_inff();
        float sum = 0.f, weighted = 0.f;
        for (int32_t j = (int32_t) threadIdx.x; !none && bad == 0.f && j < C; j += kBlock) {
            const float d = load_at<T>(a.logits, r, j) - m, p = expf(d);
            sum += p;
            if (p > 0.f) weighted = fmaf(p, d, weighted);
        }
        sum = block_reduce(sum, s_f, add);
        weighted = block_reduce(weighted, s_f, add);
        const float nan = quiet_nan();
        const float log_sum = bad != 0.f ? nan : none ? 0.f : logf(sum);
        if (threadIdx.x == 0) {
            if (a.logp) {
                const int32_t y = a.labels[r];
                float v = y < 0 ? 0.f : y >= C ? nan : none ? -__builtin_inff() : load_at<T>(a.logits, r, y) - m - log_sum;
                a.logp[r] = bad != 0.f ? nan : v;
            }
            if (a.entropy) a.entropy[r] = bad != 0.f ? nan : none ? 0.f : log_sum - weighted / sum;
            if (a.stats) { a.stats[2 * r] = bad != 0.f ? nan : m; a.stats[2 * r + 1] = log_sum; }
        }
        unsigned long long last = ~0ull;
        for (int32_t i = 0; i < a.top; ++i) {
            unsigned long long best = 0;
            for (int32_t j = (int32_t) threadIdx.x; bad == 0.f && j < C; j += kBlock) {
                const float z = load_at<T>(a.logits, r, j);
                const unsigned long long key = order_key(z, j);
                if (z > -__builtin_inff() && key < last && key > best) best = key;
            }
            best = block_reduce(best, s_key, [](unsigned long long x, unsigned long long y) { return x > y ? x : y; });
            if (threadIdx.x == 0) {
                const int32_t j = best ? (int32_t) ~(uint32_t) best : -1;
                a.top_index[r * a.top + i] = j;
                a.top_logp[r * a.top + i] = bad != 0.f ? nan : j < 0 ? -__builtin_inff() : load_at<T>(a.logits, r, j) - m - log_sum;
            }
            last = best;
        }
    }
}

template <typename T, typename O>
__global__ void __launch_bounds__(kBlock) k_log_probs_backward(LogProbsBackwardArgs a)
{
    const int32_t rows = a.count.get(), C = a.logits.width;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float m = a.stats[2 * r], log_sum = a.stats[2 * r + 1];
        const int32_t y = a.labels ? a.labels[r] : -1;
        const float g = y < 0 ? 0.f : y >= C ? quiet_nan() : a.g_logp[r];
        const float h = a.g_entropy ? a.g_entropy[r] : 0.f, entropy = a.entropy ? a.entropy[r] : 0.f;
        const bool none = m == -__builtin_inff();
        for (int32_t j = (int32_t) threadIdx.x; j < C; j += kBlock) {
            const float log_p = (load_at<T>(a.logits, r, j) - m) - log_sum, p = none ? 0.f : expf(log_p);
            float v = -g * p;
            if (p > 0.f) v -= h * p * (log_p + entropy);
            if (j == y && !none) v += g;
            store_at<O>(a.d_logits, r, j, none ? 0.f : p == p ? v : quiet_nan());
        }
    }
}

static unsigned row_grid(const gns_ctx* c, int32_t rows)
{
    const int64_t most = (int64_t) c->num_cus * 64;
    return (unsigned) (rows < most ? rows : most);
}

size_t log_probs_workspace(const gns_ctx*, int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_log_probs(const gns_ctx* c, const LogProbsArgs& a, int32_t type, hipStream_t s)
{
    const dim3 grid(row_grid(c, a.count.rows));
    if (type == GNS_FP32) hipLaunchKernelGGL(k_log_probs<float>, grid, dim3(kBlock), 0, s, a);
    else                  hipLaunchKernelGGL(k_log_probs<Bf16>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_log_probs_backward(const gns_ctx* c, const LogProbsBackwardArgs& a, int32_t type, int32_t out_type, hipStream_t s)
{
    const dim3 grid(row_grid(c, a.count.rows));
    if (type == GNS_FP32 && out_type == GNS_FP32) hipLaunchKernelGGL((k_log_probs_backward<float, float>), grid, dim3(kBlock), 0, s, a);
    else if (type == GNS_FP32)                    hipLaunchKernelGGL((k_log_probs_backward<float, Bf16>), grid, dim3(kBlock), 0, s, a);
    else if (out_type == GNS_FP32)                hipLaunchKernelGGL((k_log_probs_backward<Bf16, float>), grid, dim3(kBlock), 0, s, a);
    else                                          hipLaunchKernelGGL((k_log_probs_backward<Bf16, Bf16>), grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace gns
