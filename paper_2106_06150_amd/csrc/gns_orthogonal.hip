// Orthogonalised updates: momentum, Newton-Schulz products on the matrix cores, the weights' step.
//
// Values v of X and of the matrices between are kept as two fp16 terms of 2^12 v: the value rounded, and what is left rounded.  A product
// of two values is three products of terms (what is left out is 2^-22 of it), summed in fp32.  All products are of rows with rows: X is
// kept as it is and turned, the others are symmetric.
#include "gns_layers.hpp"
#include <algorithm>

namespace gns {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;
constexpr int kPad = 128;                     // rows and columns of the matrices in terms are multiples of it, zeros behind the values
constexpr int kTermBlock = 32;                // values of a row whose first terms, then second terms lie together: 128 bytes

// Where the terms of 8 values of a row begin: c a multiple of 8; the second terms lie 64 bytes behind the first.
__device__ __forceinline__ int64_t terms_at(int64_t row, int32_t c, int32_t columns)
{
    return row * columns * 4 + (int64_t) (c / kTermBlock) * 128 + c % kTermBlock * 2;
}
__device__ __forceinline__ void store_terms(char* to, const float (&v)[8])
{
    half8 one, two;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        one[i] = (_Float16) v[i];
        two[i] = (_Float16) (v[i] - (float) one[i]);
    }
    *reinterpret_cast<half8*>(to) = one;
    *reinterpret_cast<half8*>(to + 64) = two;
}
__device__ __forceinline__ void load_terms(const char* from, float (&v)[8])
{
    const half8 one = *reinterpret_cast<const half8*>(from), two = *reinterpret_cast<const half8*>(from + 64);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float) one[i] + (float) two[i];
}

// Eight columns of a row of either type, of any alignment; columns past the last are zero.
__device__ __forceinline__ void load_eight(const ConstRows& x, int32_t type, int64_t r, int32_t c, float (&v)[8])
{
    if (c + 8 <= x.width) {
        if (type == GNS_FP32) {
            uint32_t w[8];
            load_words(reinterpret_cast<const float*>(x.data) + r * x.stride + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            uint32_t w[4];
            load_words(reinterpret_cast<const Bf16*>(x.data) + r * x.stride + c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = value_of_words<Bf16>(w, i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = c + i >= x.width ? 0.f : type == GNS_FP32 ? load_at<float>(x, r, c + i) : load_at<Bf16>(x, r, c + i);
    }
}
__device__ __forceinline__ void store_eight(const MutRows& x, int32_t type, int64_t r, int32_t c, const float (&v)[8])
{
    if (c + 8 <= x.width) {
        if (type == GNS_FP32) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
            store_words(reinterpret_cast<float*>(x.data) + r * x.stride + c, w);
        } else {
            struct Values { Bf16 v[8]; } out;
#pragma unroll
            for (int i = 0; i < 8; ++i) out.v[i] = from_float<Bf16>(v[i]);
            __builtin_memcpy(reinterpret_cast<Bf16*>(x.data) + r * x.stride + c, &out, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < x.width) {
                if (type == GNS_FP32) store_at<float>(x, r, c + i, v[i]);
                else                  store_at<Bf16>(x, r, c + i, v[i]);
            }
    }
}

struct MomentumArgs {
    ConstRows grad, momentum;
    MutRows momentum_out;
    int32_t grad_type, momentum_type, momentum_out_type, rows, nesterov;
    float mu;
    float* u;                     // rows of `pieces` times eight columns
    int32_t pieces;
    double* sums;                 // of squares, by block
};

constexpr int kSumBlocks = 1024;

// The momentum and u, and u's squares by block, in 64 bits: neither large nor small gradients leave their range.
__global__ void __launch_bounds__(kBlock) k_momentum(MomentumArgs a)
{
    __shared__ double s_sum[kBlock / kWave];
    const uint32_t all = (uint32_t) a.rows * (uint32_t) a.pieces;
    double sum = 0.0;
    for (uint32_t i = blockIdx.x * kBlock + threadIdx.x; i < all; i += gridDim.x * kBlock) {
        const uint32_t r = i / (uint32_t) a.pieces;
        const int32_t c = (int32_t) (i - r * (uint32_t) a.pieces) * 8;
        float g[8], u[8];
        load_eight(a.grad, a.grad_type, r, c, g);
        if (a.momentum.data) {
            load_eight(a.momentum, a.momentum_type, r, c, u);
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = a.mu * u[k] + g[k];
            store_eight(a.momentum_out, a.momentum_out_type, r, c, u);
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = a.nesterov ? g[k] + a.mu * u[k] : u[k];
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = a.nesterov ? g[k] + a.mu * g[k] : g[k];
        }
        float4* to = reinterpret_cast<float4*>(a.u + (int64_t) i * 8);
        to[0] = make_float4(u[0], u[1], u[2], u[3]);
        to[1] = make_float4(u[4], u[5], u[6], u[7]);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += (double) u[k] * (double) u[k];
    }
    for (int m = 1; m < kWave; m *= 2) sum += __shfl_xor(sum, m);
    if (opaque_lane_id() == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

struct SpreadArgs {
    const float* u;
    const double* sums;
    int32_t sum_count, rows, width, pitch;    // of u
    int32_t short_side, long_side, tall;      // padded; tall: X is u turned
    double eps;
    char* x;                      // [short][long]
    char* turned;                 // [long][short]
};

constexpr int kSpread = 64;

// X in terms, as it is and turned, a tile of 64 x 64 a block.
__global__ void __launch_bounds__(kBlock) k_spread(SpreadArgs a)
{
    __shared__ float s_tile[kSpread][kSpread + 1];
    __shared__ double s_sum[kBlock / kWave];
    double sum = 0.0;
    for (int32_t i = (int32_t) threadIdx.x; i < a.sum_count; i += kBlock) sum += a.sums[i];
    for (int m = 1; m < kWave; m *= 2) sum += __shfl_xor(sum, m);
    if (opaque_lane_id() == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double norm = sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
    const double inverse = !(norm < (double) __builtin_inff()) ? (double) quiet_nan() : norm > 0.0 ? (double) kUp / (norm + a.eps) : 0.0;
    // the tile as u has it
    const int32_t x0 = (int32_t) blockIdx.y * kSpread, y0 = (int32_t) blockIdx.x * kSpread;      // in X: rows, columns
    const int32_t u_row = a.tall ? y0 : x0, u_column = a.tall ? x0 : y0;
    for (int i = (int) threadIdx.x; i < kSpread * kSpread; i += kBlock) {
        const int32_t r = i / kSpread, c = i % kSpread;
        float v = 0.f;
        if (u_row + r < a.rows && u_column + c < a.width) v = (float) ((double) a.u[(int64_t) (u_row + r) * a.pitch + u_column + c] * inverse);
        if (a.tall) s_tile[c][r] = v;
        else        s_tile[r][c] = v;
    }
    __syncthreads();
    for (int i = (int) threadIdx.x; i < kSpread * kSpread / 8; i += kBlock) {
        const int32_t r = i / (kSpread / 8), c = i % (kSpread / 8) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s_tile[r][c + k];
        store_terms(a.x + terms_at(x0 + r, y0 + c, a.long_side), v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s_tile[c + k][r];
        store_terms(a.turned + terms_at(y0 + r, x0 + c, a.short_side), v);
    }
}

// What becomes of a product P of rows with rows.
enum { kGram = 0, kPoly = 1, kStep = 2, kLast = 3 };
struct ProductArgs {
    const char* left;             // [m][k] in terms
    const char* right;            // [n][k]
    int32_t m, n, k;              // multiples of kPad
    const char* same;             // kPoly: A; kStep, kLast: X, of the shape of P
    char* to;                     // kGram: P; kPoly: b A + c P; kStep: a X + P
    char* turned;                 // kStep: the same turned
    float a, b, c;
    // kLast: out = keep * w + rate * (a X + P), turned back if tall
    ConstRows w;
    MutRows out;
    int32_t w_type, out_type, rows, tall;
    float keep, rate;
};

// k_product: 128 x 128 of P a block, 64 x 64 a wave, products of 32 x 32 x 16.  A stage is 32 of k: 128 bytes of a row, both terms, from
// memory straight to LDS, where chunk c of 16 bytes of row r lies at c ^ (r & 7).  Symmetric products are made for the tiles
// on and below the diagonal and written to both places.
constexpr int kSide = 128, kStageBytes = 2 * kSide * 128, kOutPitch = kSide + 4;

template <int kWhat>
__global__ void __launch_bounds__(kBlock, 2) k_product(ProductArgs a)
{
    constexpr bool kSymmetric = kWhat == kGram || kWhat == kPoly;
    __shared__ __attribute__((aligned(128))) char s_stage[kSide * kOutPitch * 4 > 2 * kStageBytes ? kSide * kOutPitch * 4 : 2 * kStageBytes];
    int32_t tm, tn;
    if (kSymmetric) {
        // block b is the pair (tm, tn), tn <= tm, in the order of rows
        const int32_t b = (int32_t) blockIdx.x;
        tm = (int32_t) ((sqrtf(8.f * (float) b + 1.f) - 1.f) * 0.5f);
        while (tm * (tm + 1) / 2 > b) --tm;
        while ((tm + 1) * (tm + 2) / 2 <= b) ++tm;
        tn = b - tm * (tm + 1) / 2;
    } else {
        tile_of(xcd_run((int32_t) blockIdx.x, (int32_t) gridDim.x), a.m / kSide, a.n / kSide, &tm, &tn);
    }
    const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63;
    const int64_t row_bytes = (int64_t) a.k * 4;
    // this wave's pieces of a stage: 8 rows each, 8 of either side; a lane's 16 bytes come from where its place in LDS has them
    const int32_t piece_row = lane >> 3, chunk = (lane & 7) ^ piece_row;
    const char* from = (wave < 2 ? a.left + ((int64_t) tm * kSide + wave * 64) * row_bytes : a.right + ((int64_t) tn * kSide + (wave - 2) * 64) * row_bytes) +
                       piece_row * row_bytes + chunk * 16;
    auto fetch = [&](int buffer, int32_t step) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*) (from + (int64_t) step * 128 + (int64_t) i * 8 * row_bytes),
                (__attribute__((address_space(3))) void*) (s_stage + buffer * kStageBytes + (wave * 64 + i * 8) * 128), 16, 0, 0);
    };
    const int wm = wave / 2 * 64, wn = wave % 2 * 64, l32 = lane & 31, kh = lane >> 5;
    float16v acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    const int32_t steps = a.k / kTermBlock;
    fetch(0, 0);
    for (int32_t step = 0; step < steps; ++step) {
        __syncthreads();          // this stage has come, and the one before has been read
        if (step + 1 < steps) fetch((step + 1) & 1, step + 1);
        const char* at = s_stage + (step & 1) * kStageBytes;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            half8 x[2][2], y[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int32_t place = ((t * 4 + s * 2 + kh) ^ (l32 & 7)) * 16;
                    x[i][t] = *reinterpret_cast<const half8*>(at + (wm + i * 32 + l32) * 128 + place);
                    y[i][t] = *reinterpret_cast<const half8*>(at + (kSide + wn + i * 32 + l32) * 128 + place);
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][1], y[j][0], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[j][1], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[j][0], acc[i][j], 0, 0, 0);
                }
        }
    }
    __syncthreads();
    float (*s_out)[kOutPitch] = reinterpret_cast<float (*)[kOutPitch]>(s_stage);
    // element v of lane l is row 8 * (v / 4) + 4 * (l / 32) + v % 4, column l % 32
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) s_out[wm + i * 32 + 8 * (v / 4) + 4 * kh + v % 4][wn + j * 32 + l32] = acc[i][j][v] * kDown;
    __syncthreads();
    // s_out holds 2^12 P; by rows
    const int32_t m0 = tm * kSide, n0 = tn * kSide;
    for (int i = (int) threadIdx.x; i < kSide * kSide / 8; i += kBlock) {
        const int32_t r = i / (kSide / 8), c = i % (kSide / 8) * 8;
        float v[8], x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s_out[r][c + k];
        const int64_t place = terms_at(m0 + r, n0 + c, a.n);
        if (kWhat != kGram) {
            load_terms(a.same + place, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = kWhat == kPoly ? a.b * x[k] + a.c * v[k] : a.a * x[k] + v[k];
#pragma unroll
            for (int k = 0; k < 8; ++k) s_out[r][c + k] = v[k];
        }
        if (kWhat != kLast) {
            store_terms(a.to + place, v);
        } else if (!a.tall && m0 + r < a.rows && n0 + c < a.out.width) {
            float w[8];
            if (a.w.data) load_eight(a.w, a.w_type, m0 + r, n0 + c, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = (a.w.data ? a.keep * w[k] : 0.f) + a.rate * (v[k] * kDown);
            store_eight(a.out, a.out_type, m0 + r, n0 + c, v);
        }
    }
    if (kWhat == kLast ? !a.tall : kSymmetric && tm == tn) return;
    __syncthreads();
    // and by columns
    for (int i = (int) threadIdx.x; i < kSide * kSide / 8; i += kBlock) {
        const int32_t r = i % kSide, c = i / kSide * 8;        // row of the turned tile
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = s_out[c + k][r];
        if (kWhat == kLast) {
            if (n0 + r < a.rows && m0 + c < a.out.width) {
                float w[8];
                if (a.w.data) load_eight(a.w, a.w_type, n0 + r, m0 + c, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = (a.w.data ? a.keep * w[k] : 0.f) + a.rate * (v[k] * kDown);
                store_eight(a.out, a.out_type, n0 + r, m0 + c, v);
            }
        } else {
            store_terms((kSymmetric ? a.to : a.turned) + terms_at(n0 + r, m0 + c, a.m), v);
        }
    }
}

// No steps: out = keep * w + rate * X from X in terms.
__global__ void __launch_bounds__(kBlock) k_no_step(ProductArgs a, int32_t pieces)
{
    const uint32_t all = (uint32_t) a.rows * (uint32_t) pieces;
    for (uint32_t i = blockIdx.x * kBlock + threadIdx.x; i < all; i += gridDim.x * kBlock) {
        const uint32_t r = i / (uint32_t) pieces;
        const int32_t c = (int32_t) (i - r * (uint32_t) pieces) * 8;
        float v[8], w[8];
        load_terms(a.same + terms_at(r, c, a.k), v);
        if (a.w.data) load_eight(a.w, a.w_type, r, c, w);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (a.w.data ? a.keep * w[k] : 0.f) + a.rate * (v[k] * kDown);
        store_eight(a.out, a.out_type, r, c, v);
    }
}

namespace {

struct Space {
    int32_t short_side, long_side;
    size_t sums, x, turned[2], gram, poly, all;       // where each begins; u lies where the second turned X will
};
Space space_of(int32_t width, int32_t rows)
{
    auto padded = [](int32_t n) { return (n + kPad - 1) / kPad * kPad; };
    Space s;
    s.short_side = padded(std::min(width, rows));
    s.long_side = padded(std::max(width, rows));
    const size_t large = (size_t) s.short_side * s.long_side * 4, small = (size_t) s.short_side * s.short_side * 4;
    s.sums = 0;
    s.x = kSumBlocks * sizeof(double);
    s.turned[0] = s.x + large;
    s.turned[1] = s.turned[0] + large;
    s.gram = s.turned[1] + large;
    s.poly = s.gram + small;
    s.all = s.poly + small;
    return s;
}

}  // namespace

// A workspace for a matrix of so many rows serves those of fewer: a shorter side's padding is no longer.
size_t orthogonal_workspace(int32_t width, int32_t rows) { return space_of(width, rows).all; }

hipError_t launch_orthogonal(const gns_ctx* c, const OrthogonalArgs& a, hipStream_t s)
{
    const int32_t width = a.grad.width, rows = a.rows, pieces = (width + 7) / 8;
    const Space space = space_of(width, rows);
    char* const at = static_cast<char*>(a.workspace);
    const bool tall = rows > width;
    double* const sums = reinterpret_cast<double*>(at + space.sums);
    float* const u = reinterpret_cast<float*>(at + space.turned[1]);
    const int32_t blocks = (int32_t) std::min<int64_t>(((int64_t) rows * pieces + kBlock - 1) / kBlock, kSumBlocks);
    MomentumArgs m = {a.grad, a.momentum, a.momentum_out, a.grad_type, a.momentum_type, a.momentum_out_type, rows, a.how->nesterov, a.how->mu, u, pieces, sums};
    hipLaunchKernelGGL(k_momentum, dim3((unsigned) blocks), dim3(kBlock), 0, s, m);
    SpreadArgs p = {u, sums, blocks, rows, width, pieces * 8, space.short_side, space.long_side, tall, (double) a.how->eps, at + space.x, at + space.turned[0]};
    hipLaunchKernelGGL(k_spread, dim3((unsigned) (space.long_side / kSpread), (unsigned) (space.short_side / kSpread)), dim3(kBlock), 0, s, p);
    ProductArgs q = {};
    q.w = a.w; q.out = a.out; q.w_type = a.w_type; q.out_type = a.out_type; q.rows = rows; q.tall = tall;
    q.keep = a.how->keep; q.rate = a.how->rate;
    const unsigned side = (unsigned) (space.short_side / kSide), whole = side * (unsigned) (space.long_side / kSide);
    int32_t turn = 0;
    for (int32_t i = 0; i < a.how->steps; ++i) {
        const float* f = a.how->coefficients[i];
        ProductArgs g = q;
        g.a = f[0]; g.b = f[1]; g.c = f[2];
        g.left = g.right = at + space.x;
        g.m = g.n = space.short_side; g.k = space.long_side;
        g.to = at + space.gram;
        hipLaunchKernelGGL((k_product<kGram>), dim3(side * (side + 1) / 2), dim3(kBlock), 0, s, g);
        g.left = g.right = g.same = at + space.gram;
        g.k = space.short_side;
        g.to = at + space.poly;
        hipLaunchKernelGGL((k_product<kPoly>), dim3(side * (side + 1) / 2), dim3(kBlock), 0, s, g);
        g.left = at + space.poly; g.right = at + space.turned[turn]; g.same = at + space.x;
        g.n = space.long_side;
        g.to = at + space.x; g.turned = at + space.turned[1 - turn];
        if (i + 1 < a.how->steps) hipLaunchKernelGGL((k_product<kStep>), dim3(whole), dim3(kBlock), 0, s, g);
        else                      hipLaunchKernelGGL((k_product<kLast>), dim3(whole), dim3(kBlock), 0, s, g);
        turn = 1 - turn;
    }
    if (!a.how->steps) {
        q.same = tall ? at + space.turned[0] : at + space.x;
        q.k = tall ? space.short_side : space.long_side;
        hipLaunchKernelGGL(k_no_step, dim3((unsigned) blocks), dim3(kBlock), 0, s, q, pieces);
    }
    return hipGetLastError();
}

}  // namespace gns
