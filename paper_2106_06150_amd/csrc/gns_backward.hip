// The backward pass of the update step, with the layer's inputs from their 8-bit checkpoints.
#include "gns_learn.hpp"

namespace gns {

// dz of row r, column n
template <typename T>
__device__ __forceinline__ float dz_at(const BackwardArgs& a, int64_t r, int32_t n)
{
    if (a.positive && !((a.positive[r * ((a.hdim + 31) / 32) + (n >> 5)] >> (n & 31)) & 1u)) return 0.f;
    return load_at<T>(a.d_out, r, n);
}

__device__ __forceinline__ float x_at(const BackwardArgs& a, int64_t r, int32_t k)
{
    const PackedRows& x = k < a.x1.width ? a.x1 : a.x2;
    const int32_t c = k < a.x1.width ? k : k - a.x1.width;
    const int64_t g = r * x.groups + (c >> 5);
    return (float) x.q[g * 32 + (c & 31)] * __uint_as_float((uint32_t) x.exponents[g] << 23);
}

constexpr int kSide = 32;                         // outputs of a block: kSide x kSide, 4 a thread

// dw and db: blocks (tile of k, tile of n), all rows.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_backward_weights(BackwardArgs a)
{
    __shared__ float s_x[kSide][kSide + 1], s_z[kSide][kSide + 1];
    const int32_t rows = a.count.get(), K = a.x1.width + a.x2.width;
    const int32_t k0 = (int32_t) blockIdx.x * kSide, n0 = (int32_t) blockIdx.y * kSide;
    const int tx = (int) threadIdx.x % 32, ty = (int) threadIdx.x / 32;
    float acc[4] = {}, sum = 0.f;
    for (int64_t r0 = 0; r0 < rows; r0 += kSide) {
        for (int i = ty; i < kSide; i += 8) {
            const int64_t r = r0 + i;
            s_x[i][tx] = a.dw && r < rows && k0 + tx < K ? x_at(a, r, k0 + tx) : 0.f;
            s_z[i][tx] = r < rows && n0 + tx < a.hdim ? dz_at<T>(a, r, n0 + tx) : 0.f;
        }
        __syncthreads();
        for (int i = 0; i < kSide; ++i) {
            for (int j = 0; j < 4; ++j) acc[j] = fmaf(s_x[i][ty + 8 * j], s_z[i][tx], acc[j]);
            sum += s_z[i][tx];
        }
        __syncthreads();
    }
    if (n0 + tx >= a.hdim) return;
    for (int j = 0; j < 4; ++j)
        if (a.dw && k0 + ty + 8 * j < K) a.dw[(int64_t) (k0 + ty + 8 * j) * a.hdim + n0 + tx] = acc[j];
    if (a.db && k0 == 0 && ty == 0) a.db[n0 + tx] = sum;
}

// dx: blocks (tile of rows, tile of k).
template <typename T>
__global__ void __launch_bounds__(kBlock) k_backward_input(BackwardArgs a)
{
    __shared__ float s_z[kSide][kSide + 1], s_w[kSide][kSide + 1];
    const int32_t rows = a.count.get(), K = a.x1.width + a.x2.width;
    const int64_t r0 = (int64_t) blockIdx.x * kSide;
    const int32_t k0 = (int32_t) blockIdx.y * kSide;
    if (r0 >= rows) return;
    const int tx = (int) threadIdx.x % 32, ty = (int) threadIdx.x / 32;
    float acc[4] = {};
    for (int32_t n0 = 0; n0 < a.hdim; n0 += kSide) {
        for (int i = ty; i < kSide; i += 8) {
            s_z[i][tx] = r0 + i < rows && n0 + tx < a.hdim ? dz_at<T>(a, r0 + i, n0 + tx) : 0.f;
            s_w[i][tx] = k0 + i < K && n0 + tx < a.hdim ? a.w[(int64_t) (k0 + i) * a.hdim + n0 + tx] : 0.f;
        }
        __syncthreads();
        for (int i = 0; i < kSide; ++i)
            for (int j = 0; j < 4; ++j) acc[j] = fmaf(s_z[ty + 8 * j][i], s_w[tx][i], acc[j]);
        __syncthreads();
    }
    for (int j = 0; j < 4; ++j)
        if (r0 + ty + 8 * j < rows && k0 + tx < K) store_at<T>(a.dx, r0 + ty + 8 * j, k0 + tx, acc[j]);
}

size_t backward_workspace(const gns_ctx*, int32_t, int32_t, int32_t) { return 256; }

template <typename T>
static hipError_t launch_typed(const BackwardArgs& a, hipStream_t s)
{
    const int32_t K = a.x1.width + a.x2.width;
    const unsigned tiles_k = (unsigned) ((K + kSide - 1) / kSide), tiles_n = (unsigned) ((a.hdim + kSide - 1) / kSide);
    if (a.dw || a.db)
        hipLaunchKernelGGL(k_backward_weights<T>, dim3(a.dw ? tiles_k : 1, tiles_n), dim3(kBlock), 0, s, a);
    if (a.dx.data && a.count.rows)
        hipLaunchKernelGGL(k_backward_input<T>, dim3((unsigned) ((a.count.rows + kSide - 1) / kSide), tiles_k), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_backward(const gns_ctx*, const BackwardArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_typed<float>(a, s) : launch_typed<Bf16>(a, s);
}

}  // namespace gns
