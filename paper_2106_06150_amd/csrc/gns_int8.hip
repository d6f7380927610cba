// The update step in 8-bit integers: rows quantised with a scale each, exact integer products, scales and bias behind them.
#include "gns_learn.hpp"

namespace gns {

// One wave per row, two passes over it: the largest magnitude, then the values.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_quantize_rows(QuantizeArgs a)
{
    const int32_t rows = a.count.get(), lane = lane_id();
    const int32_t f1 = a.x1.width, k = f1 + a.x2.width;
    for (int64_t r = (int64_t) blockIdx.x * (kBlock / kWave) + (threadIdx.x >> 6); r < rows; r += (int64_t) gridDim.x * (kBlock / kWave)) {
        uint32_t most = 0;
        auto at = [&](int32_t c) { return c < f1 ? load_at<T>(a.x1, r, c) : load_at<T>(a.x2, r, c - f1); };
        for (int32_t c = lane; c < k; c += kWave) most = max(most, magnitude_bits(at(c)));
        for (int off = 32; off; off >>= 1) most = max(most, (uint32_t) __shfl_xor((int) most, off));
        const float amax = __uint_as_float(most);
        const bool none = most >= kInfBits || amax < 0x1p-120f;
        const float inv = none ? 0.f : 127.f / amax;
        for (int32_t c = lane; c < (int32_t) a.stride; c += kWave)
            a.q[r * a.stride + c] = c < k && !none ? (int8_t) (int) rintf(at(c) * inv) : (int8_t) 0;
        if (lane == 0) a.scale[r] = most >= kInfBits ? quiet_nan() : none ? 0.f : amax / 127.f;
    }
}

// 64 x 64 outputs a block, 4 x 4 a thread, four products of bytes at a time.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_dense_int8(DenseInt8Args a)
{
    __shared__ int s_q[16][65], s_w[16][65];
    const int32_t rows = a.count.get(), n = a.out.width;
    const int64_t r0 = (int64_t) blockIdx.x * 64;
    const int32_t n0 = (int32_t) blockIdx.y * 64;
    if (r0 >= rows) return;
    const int tx = (int) threadIdx.x % 16, ty = (int) threadIdx.x / 16;
    int acc[4][4] = {};
    for (int32_t k0 = 0; k0 < (int32_t) a.stride; k0 += 64) {
        for (int i = (int) threadIdx.x; i < 16 * 64; i += kBlock) {
            const int row = i / 16, word = i % 16;
            s_q[word][row] = r0 + row < rows ? *reinterpret_cast<const int*>(a.q + (r0 + row) * a.stride + k0 + word * 4) : 0;
            s_w[word][row] = n0 + row < n ? *reinterpret_cast<const int*>(a.wq + (int64_t) (n0 + row) * a.stride + k0 + word * 4) : 0;
        }
        __syncthreads();
        for (int w = 0; w < 16; ++w)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_sdot4(s_q[w][ty + 16 * i], s_w[w][tx + 16 * j], acc[i][j], false);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + ty + 16 * i;
            const int32_t c = n0 + tx + 16 * j;
            if (r >= rows || c >= n) continue;
            float y = (float) acc[i][j] * a.w_scale[c] * a.scale[r];       // in this order only results that are too large overflow
            if (a.bias) y += a.bias[c];
            store_at<T>(a.out, r, c, a.relu ? relu_of(y) : y);
        }
}

static unsigned wave_rows_grid(const gns_ctx* c, int64_t rows)
{
    const int64_t blocks = (rows + kBlock / kWave - 1) / (kBlock / kWave), most = (int64_t) c->num_cus * 64;
    return (unsigned) (blocks < most ? blocks : most);
}

hipError_t launch_quantize(const gns_ctx* c, const QuantizeArgs& a, int32_t type, hipStream_t s)
{
    const dim3 grid(wave_rows_grid(c, a.count.rows));
    if (type == GNS_FP32) hipLaunchKernelGGL(k_quantize_rows<float>, grid, dim3(kBlock), 0, s, a);
    else                  hipLaunchKernelGGL(k_quantize_rows<Bf16>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_dense_int8(const gns_ctx*, const DenseInt8Args& a, int32_t out_type, hipStream_t s)
{
    const dim3 grid((unsigned) ((a.count.rows + 63) / 64), (unsigned) ((a.out.width + 63) / 64));
    if (out_type == GNS_FP32) hipLaunchKernelGGL(k_dense_int8<float>, grid, dim3(kBlock), 0, s, a);
    else                      hipLaunchKernelGGL(k_dense_int8<Bf16>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_sage_dense_int8(const gns_ctx* c, const QuantizeArgs& x, const DenseInt8Args& a, int32_t type, int32_t out_type,
                                  hipStream_t s)
{
    const hipError_t e = launch_quantize(c, x, type, s);
    return e != hipSuccess ? e : launch_dense_int8(c, a, out_type, s);
}

}  // namespace gns
