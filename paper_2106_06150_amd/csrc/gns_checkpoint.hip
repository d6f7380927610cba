// Activation checkpoints in 8 bits: 32 columns share a power of two.
#include "gns_learn.hpp"

namespace gns {

// Exponent byte of a group whose largest magnitude has these bits: e + 127 for the smallest e with a < 127.5 * 2^e.
__device__ __forceinline__ uint32_t group_exponent(uint32_t most)
{
    const uint32_t biased = most >> 23;                       // E + 127
    if (biased == 255) return 255;
    if (biased < 27) return 0;                                // below 2^-100
    const uint32_t e = biased - 6 + ((most & 0x7FFFFFu) >= 0x7F0000u ? 1u : 0u);
    return e < 248 ? e : 248;                                 // 127 * 2^121 at most
}

// 2^e; 0 for byte 0, infinity for byte 255
__device__ __forceinline__ float group_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ int32_t group_step(float x, uint32_t byte)
{
    if (byte == 0 || byte == 255) return 0;
    const float t = rintf(x * __uint_as_float((254u - byte) << 23));
    return (int32_t) fminf(fmaxf(t, -127.f), 127.f);
}

// 32 lanes per group, a value each.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_checkpoint_save(CheckpointArgs a)
{
    const int64_t total = (int64_t) a.count.get() * a.groups;
    const int lane = lane_id(), l32 = lane & 31;
    const int64_t step = (int64_t) gridDim.x * (kBlock / 32);
    // both halves of a wave make as many turns, as the exchange between lanes asks for
    for (int64_t g0 = (int64_t) blockIdx.x * (kBlock / 32) + (threadIdx.x >> 6) * 2; g0 < total; g0 += step) {
        const int64_t g = g0 + (lane >> 5), gc = g < total ? g : total - 1;
        const int64_t r = gc / a.groups;
        const int32_t col = (int32_t) (gc - r * a.groups) * 32 + l32;
        const float x = col < a.width ? load_at<T>(a.x, r, col) : 0.f;
        uint32_t most = magnitude_bits(x);
        for (int off = 16; off; off >>= 1) most = max(most, (uint32_t) __shfl_xor((int) most, off));
        const uint64_t up = __ballot(x > 0.f);
        if (g >= total) continue;
        const uint32_t byte = group_exponent(most);
        a.q[g * 32 + l32] = (int8_t) group_step(x, byte);
        if (l32 == 0) {
            a.exponents[g] = (uint8_t) byte;
            if (a.positive) a.positive[g] = (uint32_t) (up >> (lane & 32));
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kBlock) k_checkpoint_load(CheckpointArgs a)
{
    const int64_t total = (int64_t) a.count.get() * a.groups * 32;
    for (int64_t i = (int64_t) blockIdx.x * kBlock + threadIdx.x; i < total; i += (int64_t) gridDim.x * kBlock) {
        const int64_t g = i >> 5, r = g / a.groups;
        const int32_t col = (int32_t) (g - r * a.groups) * 32 + (int32_t) (i & 31);
        if (col < a.width) store_at<T>(a.out, r, col, (float) a.q[i] * group_scale(a.exponents[g]));
    }
}

static unsigned grid_of(const gns_ctx* c, int64_t blocks)
{
    const int64_t most = (int64_t) c->num_cus * 64;
    return (unsigned) (blocks < most ? blocks : most);
}

hipError_t launch_checkpoint_save(const gns_ctx* c, const CheckpointArgs& a, int32_t type, hipStream_t s)
{
    const dim3 grid(grid_of(c, ((int64_t) a.count.rows * a.groups + kBlock / 32 - 1) / (kBlock / 32)));
    if (type == GNS_FP32) hipLaunchKernelGGL(k_checkpoint_save<float>, grid, dim3(kBlock), 0, s, a);
    else                  hipLaunchKernelGGL(k_checkpoint_save<Bf16>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_checkpoint_load(const gns_ctx* c, const CheckpointArgs& a, int32_t type, hipStream_t s)
{
    const dim3 grid(grid_of(c, ((int64_t) a.count.rows * a.groups * 32 + kBlock - 1) / kBlock));
    if (type == GNS_FP32) hipLaunchKernelGGL(k_checkpoint_load<float>, grid, dim3(kBlock), 0, s, a);
    else                  hipLaunchKernelGGL(k_checkpoint_load<Bf16>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace gns
