// What the kernels of training and answering share: rows of either type, the row count, launches (gfx950, wave64).
#pragma once
#include "../../include/gns_learn.h"
#include "gns_internal.h"
#include "gns_device.hpp"

namespace gns {

struct Bf16 { uint16_t bits; };

// A row count that the host knows or the device holds (rows is then the worst case).
struct RowCount {
    int32_t rows;
    const int32_t* rows_dev;
    __device__ __forceinline__ int32_t get() const { return rows_dev ? (*rows_dev < rows ? *rows_dev : rows) : rows; }
};

struct ConstRows {
    const void* data;
    int64_t stride;
    int32_t width;
};

struct MutRows {
    void* data;
    int64_t stride;
    int32_t width;
};

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<Bf16>(Bf16 v) { return __uint_as_float((uint32_t) v.bits << 16); }

// Rounded to nearest, ties to even; a NaN stays one.
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ Bf16 from_float<Bf16>(float v)
{
    return Bf16{__builtin_bit_cast(uint16_t, (__bf16) v)};
}

template <typename T>
__device__ __forceinline__ float load_at(const ConstRows& x, int64_t r, int64_t c)
{
    return to_float<T>(reinterpret_cast<const T*>(x.data)[r * x.stride + c]);
}

template <typename T>
__device__ __forceinline__ void store_at(const MutRows& x, int64_t r, int64_t c, float v)
{
    reinterpret_cast<T*>(x.data)[r * x.stride + c] = from_float<T>(v);
}

constexpr uint32_t kInfBits = 0x7F800000u;
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// max(0, v) that keeps a NaN
__device__ __forceinline__ float relu_of(float v) { return v < 0.f ? 0.f : v; }

// Waits for this wave's LDS accesses and for the block's other waves; reads from memory stay on their way.
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// 16 bytes (a struct of four words would not always stay in registers, nor leave them as one)
typedef uint32_t Chunk __attribute__((ext_vector_type(4)));

// N words from or to wherever they begin, 16 bytes a read or write: global memory asks for no marks.
template <int N>
__device__ __forceinline__ void load_words(const void* from, uint32_t (&to)[N])
{
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        Chunk v;
        __builtin_memcpy(&v, static_cast<const char*>(from) + 16 * j, 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) to[4 * j + k] = v[k];
    }
}
template <int N>
__device__ __forceinline__ void store_words(void* to, const uint32_t (&from)[N])
{
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
        const Chunk v = {from[4 * j], from[4 * j + 1], from[4 * j + 2], from[4 * j + 3]};
        __builtin_memcpy(static_cast<char*>(to) + 16 * j, &v, 16);
    }
}

// Value i of packed ones, and values packed.
template <typename T, int N>
__device__ __forceinline__ float value_of_words(const uint32_t (&w)[N], int i)
{
    return sizeof(T) == 4 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}

// Rows of a tile lie in LDS 64 bytes each, four chunks of 16: chunk c of row r at c ^ row_turn(r), so that reads of the same chunk
// of eight or sixteen rows spread over all banks.
__device__ __forceinline__ int row_turn(int row) { return ((row >> 1) & 3) ^ ((row >> 3) & 1); }

// Tile (m, n) of a block.  Blocks go to the eight XCDs in turn; each XCD's L2 gets a run of consecutive tiles, and those go
// down eight rows of tiles before they go on to the next column, so that what runs together shares rows and weights.
__device__ __forceinline__ int32_t xcd_run(int32_t block, int32_t all)
{
    const int32_t each = all / kXcds, more = all % kXcds, xcd = block % kXcds;
    return xcd * each + (xcd < more ? xcd : more) + block / kXcds;
}
__device__ __forceinline__ void tile_of(int32_t t, int32_t m_tiles, int32_t n_tiles, int32_t* tm, int32_t* tn)
{
    constexpr int32_t kBand = 8;
    const int32_t band = t / (kBand * n_tiles), in = t - band * kBand * n_tiles;
    const int32_t height = m_tiles - band * kBand < kBand ? m_tiles - band * kBand : kBand;
    *tm = band * kBand + in % height;
    *tn = in / height;
}

struct QuantizeArgs {
    ConstRows x1, x2;             // x2.width 0: one input
    int8_t* q;
    float* scale;
    int64_t stride;               // of q
    RowCount count;
};

struct DenseInt8Args {
    const int8_t* q;
    const float* scale;
    const int8_t* wq;
    const float* w_scale;
    const float* bias;
    MutRows out;
    int64_t stride;               // of q and wq
    int32_t k, relu;
    RowCount count;
};

struct CheckpointArgs {
    ConstRows x;                  // save
    MutRows out;                  // load
    int8_t* q;
    uint8_t* exponents;
    uint32_t* positive;
    int32_t width, groups;
    RowCount count;
};

struct PackedRows {
    const int8_t* q;
    const uint8_t* exponents;
    int32_t width, groups;
};

struct BackwardArgs {
    ConstRows d_out;
    const uint32_t* positive;
    PackedRows x1, x2;
    const float* w;
    float* dw;
    float* db;
    MutRows dx;
    int32_t hdim;
    RowCount count;
    void* workspace;
};

struct LogProbsArgs {
    ConstRows logits;
    const int32_t* labels;
    float* logp;
    float* entropy;
    float* stats;
    int32_t* top_index;
    float* top_logp;
    int32_t top;
    RowCount count;
    void* workspace;
};

struct LogProbsBackwardArgs {
    ConstRows logits;
    const int32_t* labels;
    const float* stats;
    const float* entropy;
    const float* g_logp;
    const float* g_entropy;
    MutRows d_logits;
    RowCount count;
};

// gns_int8.hip
hipError_t launch_quantize(const gns_ctx* c, const QuantizeArgs& a, int32_t type, hipStream_t s);
hipError_t launch_dense_int8(const gns_ctx* c, const DenseInt8Args& a, int32_t out_type, hipStream_t s);
hipError_t launch_sage_dense_int8(const gns_ctx* c, const QuantizeArgs& x, const DenseInt8Args& a, int32_t type, int32_t out_type,
                                  hipStream_t s);
// gns_checkpoint.hip
hipError_t launch_checkpoint_save(const gns_ctx* c, const CheckpointArgs& a, int32_t type, hipStream_t s);
hipError_t launch_checkpoint_load(const gns_ctx* c, const CheckpointArgs& a, int32_t type, hipStream_t s);
// gns_backward.hip
// bytes that a call of so many rows takes, and the most that one of so many or fewer does
size_t backward_need(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int32_t rows);
size_t backward_workspace(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int32_t rows);
hipError_t launch_backward(const gns_ctx* c, const BackwardArgs& a, int32_t type, hipStream_t s);
// gns_log_probs.hip
size_t log_probs_need(const gns_ctx* c, int32_t classes, int32_t top, int32_t rows);
size_t log_probs_workspace(const gns_ctx* c, int32_t classes, int32_t top, int32_t rows);
hipError_t launch_log_probs(const gns_ctx* c, const LogProbsArgs& a, int32_t type, hipStream_t s);
hipError_t launch_log_probs_backward(const gns_ctx* c, const LogProbsBackwardArgs& a, int32_t type, int32_t out_type, hipStream_t s);

}  // namespace gns
