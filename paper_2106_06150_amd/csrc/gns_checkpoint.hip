// Activation checkpoints in 8 bits: 32 columns share a power of two 2^e, the smallest with which the largest magnitude a of
// the group rounds to 127 steps or fewer, a < 127.5 * 2^e.  With a power of two the quantisation is exact arithmetic, and a
// value q * 2^e is a bf16 value, which the matrix cores take as it is.  Bound by the bytes.
#include "gns_learn.hpp"

namespace gns {

// Exponent byte (e + 127) of a group whose largest magnitude has these bits.
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

// 2^-e; 0 where a group has no values
__device__ __forceinline__ float group_inverse(uint32_t byte) { return byte == 0 || byte == 255 ? 0.f : __uint_as_float((254u - byte) << 23); }

__device__ __forceinline__ uint32_t step_of(float x, float inverse)
{
    const float t = fminf(fmaxf(rintf(x * inverse), -127.f), 127.f);
    return (uint32_t) (int32_t) t & 255u;
}

// Four lanes a group, eight consecutive values each (two pieces of 16 bytes of fp32, one of bf16), sixteen groups a wave.
// A lane's values are pieces whatever the row's alignment; where a row ends inside, they are read singly.  Bound by the bytes:
// 168,003 rows of 100 fp32 20 us, 16,384 of 4096 bf16 41 us (5.1 TB/s).  A row of such lanes is 64 bytes of the result, so sixteen
// rows' turns are one store; a lane per group would store its 32 bytes apart.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_checkpoint_save(CheckpointArgs a)
{
    const int64_t total = (int64_t) a.count.get() * a.groups;
    const int64_t step = (int64_t) gridDim.x * (kBlock / 4);
    // the lanes of a wave make as many turns, as the exchange between them asks for
    for (int64_t g0 = ((int64_t) blockIdx.x * kBlock + (threadIdx.x & ~(kWave - 1))) / 4; g0 < total; g0 += step) {
        const int lane = opaque_lane_id();
        const int64_t g = g0 + lane / 4, gc = g < total ? g : total - 1;
        const int64_t r = total <= 0xFFFFFFFFll ? (int64_t) ((uint32_t) gc / (uint32_t) a.groups) : gc / a.groups;
        const int32_t col = (int32_t) (gc - r * a.groups) * 32 + (lane & 3) * 8;
        const T* row = reinterpret_cast<const T*>(a.x.data) + r * a.x.stride;
        float x[8];
        if (col + 8 <= a.width) {
            uint32_t words[2 * sizeof(T)];
            load_words(row + col, words);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = value_of_words<T>(words, i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = col + i < a.width ? to_float(row[col + i]) : 0.f;
        }
        uint32_t most = 0, up = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            most = max(most, magnitude_bits(x[i]));
            up |= x[i] > 0.f ? 1u << i : 0u;
        }
        up <<= (lane & 3) * 8;
        most = max(most, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) most, 0xB1, 0xf, 0xf, true));       // lanes 1 0 3 2
        up |= (uint32_t) __builtin_amdgcn_update_dpp(0, (int) up, 0xB1, 0xf, 0xf, true);
        most = max(most, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) most, 0x4E, 0xf, 0xf, true));       // lanes 2 3 0 1
        up |= (uint32_t) __builtin_amdgcn_update_dpp(0, (int) up, 0x4E, 0xf, 0xf, true);
        if (g >= total) continue;
        const uint32_t byte = group_exponent(most);
        const float inverse = group_inverse(byte);
        uint2 q = make_uint2(0, 0);
        if (inverse != 0.f) {                                 // (a spoilt group's values times zero are no numbers)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                q.x |= step_of(x[i], inverse) << (8 * i);
                q.y |= step_of(x[4 + i], inverse) << (8 * i);
            }
        }
        *reinterpret_cast<uint2*>(a.q + g * 32 + (lane & 3) * 8) = q;
        if ((lane & 3) == 0) {
            a.exponents[g] = (uint8_t) byte;
            if (a.positive) a.positive[g] = up;
        }
    }
}

// Four lanes a group, eight values each.  168,003 rows of 100 fp32 21 us, 16,384 of 4096 bf16 31 us (6.7 TB/s).
template <typename T>
__global__ void __launch_bounds__(kBlock) k_checkpoint_load(CheckpointArgs a)
{
    const int64_t total = (int64_t) a.count.get() * a.groups * 4;
    for (int64_t i = (int64_t) blockIdx.x * kBlock + threadIdx.x; i < total; i += (int64_t) gridDim.x * kBlock) {
        const int64_t g = i >> 2;
        const int64_t r = total <= 0xFFFFFFFFll ? (int64_t) ((uint32_t) g / (uint32_t) a.groups) : g / a.groups;
        const int32_t col = (int32_t) (g - r * a.groups) * 32 + (int32_t) (i & 3) * 8;
        if (col >= a.width) continue;
        const uint2 q = *reinterpret_cast<const uint2*>(a.q + i * 8);
        const float scale = group_scale(a.exponents[g]);
        T* row = reinterpret_cast<T*>(a.out.data) + r * a.out.stride;
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = from_float<T>((float) (int8_t) ((j < 4 ? q.x : q.y) >> (8 * (j & 3))) * scale);
        if (col + 8 <= a.width) {
            uint32_t words[2 * sizeof(T)];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (sizeof(T) == 4) words[j] = __float_as_uint(v[j]);
                else if (j % 2 == 1)          words[j / 2] = v[j - 1].bits | (uint32_t) v[j].bits << 16;
            }
            store_words(row + col, words);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < a.width) row[col + j] = v[j];
        }
    }
}

static unsigned grid_of(const gns_ctx* c, int64_t blocks)
{
    const int64_t most = (int64_t) c->num_cus * 64;
    return (unsigned) (blocks < most ? blocks : most);
}

template <typename T>
static hipError_t launch_save(const gns_ctx* c, const CheckpointArgs& a, hipStream_t s)
{
    const dim3 grid(grid_of(c, ((int64_t) a.count.rows * a.groups + kBlock / 4 - 1) / (kBlock / 4)));
    hipLaunchKernelGGL(k_checkpoint_save<T>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_load(const gns_ctx* c, const CheckpointArgs& a, hipStream_t s)
{
    const dim3 grid(grid_of(c, ((int64_t) a.count.rows * a.groups + kBlock / 4 - 1) / (kBlock / 4)));
    hipLaunchKernelGGL(k_checkpoint_load<T>, grid, dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_checkpoint_save(const gns_ctx* c, const CheckpointArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_save<float>(c, a, s) : launch_save<Bf16>(c, a, s);
}

hipError_t launch_checkpoint_load(const gns_ctx* c, const CheckpointArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_load<float>(c, a, s) : launch_load<Bf16>(c, a, s);
}

}  // namespace gns
