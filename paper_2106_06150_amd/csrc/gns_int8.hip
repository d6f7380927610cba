// The update step in 8-bit integers: rows quantised with a scale each, exact integer products, scales and bias behind them.
#include "gns_learn.hpp"
#include <type_traits>

namespace gns {

// With channel scales of up to 2^96 a sum times one does not overflow, and only results that are too large do.  kFar: with any,
// where the smaller scale comes first (a NaN counts as that), which the kernels that are bound by such instructions do for
// tiles alone that have a larger one.
constexpr float kFarScale = 0x1p96f;
template <bool kFar>
__device__ __forceinline__ float output_of(int sum, float w_scale, float scale, float bias, int32_t relu)
{
    const bool turn = kFar && !(w_scale < scale);
    const float y = (float) sum * (turn ? scale : w_scale) * (turn ? w_scale : scale) + bias;
    return relu ? relu_of(y) : y;
}

// Pieces of V consecutive columns of a row [x1 | x2]: 16 bytes of either type.
template <typename T> constexpr int kPiece = 16 / (int) sizeof(T);
template <typename T> struct alignas(16) Piece { T v[kPiece<T>]; };

// A piece that lies in one input's row is one read, whatever the row's alignment; where an input ends inside, its values are read
// singly.  Columns past the last are zero.
template <typename T>
__device__ __forceinline__ void load_piece(const QuantizeArgs& a, int64_t r, int32_t c, float (&x)[kPiece<T>])
{
    constexpr int V = kPiece<T>;
    const int32_t f1 = a.x1.width, k = f1 + a.x2.width;
    if (c + V <= f1 || (c >= f1 && c + V <= k)) {
        uint32_t words[4];
        load_words(c < f1 ? reinterpret_cast<const T*>(a.x1.data) + r * a.x1.stride + c
                          : reinterpret_cast<const T*>(a.x2.data) + r * a.x2.stride + (c - f1), words);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = value_of_words<T>(words, i);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            x[i] = c + i < f1 ? load_at<T>(a.x1, r, c + i) : c + i < k ? load_at<T>(a.x2, r, c + i - f1) : 0.f;
    }
}

struct RowScale {
    float scale, inverse;         // inverse 0: the row has no values
};
__device__ __forceinline__ RowScale row_scale(uint32_t most)
{
    const float amax = __uint_as_float(most);
    if (most >= kInfBits) return RowScale{quiet_nan(), 0.f};
    if (amax < 0x1p-120f) return RowScale{0.f, 0.f};
    return RowScale{amax / 127.f, 127.f * (1.f / amax)};
}

template <int V>
__device__ __forceinline__ uint32_t largest_of(const float (&x)[V], uint32_t most)
{
#pragma unroll
    for (int i = 0; i < V; ++i) most = max(most, magnitude_bits(x[i]));
    return most;
}

// Four values as bytes of a word; |x * inverse| is at most 127 and a bit, which rounds to 127.
__device__ __forceinline__ uint32_t pack4(const float* x, float inverse)
{
    if (inverse == 0.f) return 0;                             // (an infinity times zero is no number)
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t) (int32_t) rintf(x[i] * inverse) & 255u) << (8 * i);
    return w;
}

template <typename T>
__device__ __forceinline__ void store_piece(int8_t* to, const float (&x)[kPiece<T>], float inverse)
{
    if (kPiece<T> == 4) *reinterpret_cast<uint32_t*>(to) = pack4(x, inverse);
    else                *reinterpret_cast<uint2*>(to) = make_uint2(pack4(x, inverse), pack4(x + 4, inverse));
}

template <int L>
__device__ __forceinline__ uint32_t largest_of_lanes(uint32_t v)
{
    if (L > 1) v = max(v, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) v, 0xB1, 0xf, 0xf, true));       // lanes 1 0 3 2
    if (L > 2) v = max(v, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) v, 0x4E, 0xf, 0xf, true));       // lanes 2 3 0 1
    if (L > 4) v = max(v, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) v, 0x141, 0xf, 0xf, true));      // mirrored in 8
    if (L > 8) v = max(v, (uint32_t) __builtin_amdgcn_update_dpp(0, (int) v, 0x140, 0xf, 0xf, true));      // mirrored in 16
    if (L > 16) v = max(v, (uint32_t) __shfl_xor((int) v, 16));
    if (L > 32) v = max(v, (uint32_t) __shfl_xor((int) v, 32));
    return v;
}

// Rows of up to L * P pieces: L lanes a row, P pieces a lane in registers; the row is read once, and nothing but its bytes counts
// where it is long enough: 85,000 rows of 256 fp32 17 us (6.4 TB/s).  Narrow ones are bound by instructions, so lanes should not
// idle: 79,214 rows of 32 bf16, four lanes each, 7 us, sixteen 14; but 100,000 rows of 100 bf16 with eight lanes 19.5, with
// sixteen, whose exchange costs the same, 18.
template <typename T, int L, int P>
__global__ void __launch_bounds__(kBlock) k_quantize_rows(QuantizeArgs a)
{
    constexpr int V = kPiece<T>;
    const int32_t rows = a.count.get();
    const int64_t step = (int64_t) gridDim.x * (kBlock / L);
    // the lanes of a wave make as many turns, as the exchange between them asks for
    for (int64_t r0 = ((int64_t) blockIdx.x * kBlock + (threadIdx.x & ~(kWave - 1))) / L; r0 < rows; r0 += step) {
        const int lane = opaque_lane_id(), l = lane & (L - 1);
        const int64_t row = r0 + lane / L, r = row < rows ? row : rows - 1;
        float x[P][V];
        uint32_t most = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) load_piece<T>(a, r, (p * L + l) * V, x[p]);
#pragma unroll
        for (int p = 0; p < P; ++p) most = largest_of(x[p], most);
        const RowScale s = row_scale(largest_of_lanes<L>(most));
        if (row >= rows) continue;
#pragma unroll
        for (int p = 0; p < P; ++p)
            if ((p * L + l) * V < (int32_t) a.stride) store_piece<T>(a.q + r * a.stride + (p * L + l) * V, x[p], s.inverse);
        if (l == 0) a.scale[r] = s.scale;
    }
}

// Longer rows: a block per row, P pieces a thread.  8192 rows of 8192 bf16: 62 to 71 us (2.8 to 3.2 TB/s; a copy of as many bytes 39):
// each row's values are held as fp32, twice their bytes, across a barrier.  Read twice by 1024 threads instead 100.
template <typename T, int P>
__global__ void __launch_bounds__(kBlock) k_quantize_block(QuantizeArgs a)
{
    constexpr int V = kPiece<T>, kWaves = kBlock / kWave;
    __shared__ uint32_t s_most[2][kWaves];                    // of this row and the one before
    const int32_t rows = a.count.get();
    int turn = 0;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x, turn ^= 1) {
        const int32_t c0 = (int32_t) threadIdx.x * V;
        float x[P][V];
        uint32_t most = 0;
#pragma unroll
        for (int p = 0; p < P; ++p) load_piece<T>(a, r, p * kBlock * V + c0, x[p]);
#pragma unroll
        for (int p = 0; p < P; ++p) most = largest_of(x[p], most);
        most = largest_of_lanes<kWave>(most);
        if (opaque_lane_id() == 0) s_most[turn][threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = max(most, s_most[turn][w]);
        const RowScale s = row_scale(most);
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (p * kBlock * V + c0 < (int32_t) a.stride) store_piece<T>(a.q + r * a.stride + p * kBlock * V + c0, x[p], s.inverse);
        if (threadIdx.x == 0) a.scale[r] = s.scale;
    }
}

// Rows of any length: a block per row, which reads it twice (the second time near by).
constexpr int kLongBlock = 1024;
template <typename T>
__global__ void __launch_bounds__(kLongBlock) k_quantize_long(QuantizeArgs a)
{
    constexpr int V = kPiece<T>;
    __shared__ uint32_t s_most[kLongBlock / kWave];
    const int32_t rows = a.count.get(), k = a.x1.width + a.x2.width;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        uint32_t most = 0;
        for (int32_t c = (int32_t) threadIdx.x * V; c < k; c += kLongBlock * V) {
            float x[V];
            load_piece<T>(a, r, c, x);
            most = largest_of(x, most);
        }
        most = largest_of_lanes<kWave>(most);
        __syncthreads();
        if (opaque_lane_id() == 0) s_most[threadIdx.x >> 6] = most;
        __syncthreads();
        for (int w = 0; w < kLongBlock / kWave; ++w) most = max(most, s_most[w]);
        const RowScale s = row_scale(most);
        for (int32_t c = (int32_t) threadIdx.x * V; c < (int32_t) a.stride; c += kLongBlock * V) {
            float x[V];
            load_piece<T>(a, r, c, x);
            store_piece<T>(a.q + r * a.stride + c, x, s.inverse);
        }
        if (threadIdx.x == 0) a.scale[r] = s.scale;
    }
}

typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int16v __attribute__((ext_vector_type(16)));

constexpr int kStepBytes = 64;                // k of a stage

// k_int8_tiles: BM x BN outputs a block, WM x WN a wave, products of 32 x 32 x 32 bytes.  A stage of 64 k of the rows and weights
// is read two stages before it is written to LDS, and written two before it is multiplied; one barrier a stage.  So
// nothing that the products wait for is less than a stage old: the last fragments of a stage are read while its first are
// multiplied, the first of the next one while its last are.  Chunk c of 16 bytes of row r lies at c ^ row_turn(r) of the
// row, so that reads of the same chunk of eight or sixteen rows spread over all banks.  The weights are the products' left factor,
// so that a lane holds four consecutive outputs of a row.
// 8192 x 8192 x 8192, bf16 out: 490 to 610 us, 1.8 to 2.2 POP/s (a large library product of integers: 2.15), bound by the matrix
// cores' cycles at the clock that the power leaves; with outputs stored value by value 40 us more.
// Blocks of 128 x 128 are three a CU, for which the compiler has to be told (two: 79,214 rows of 32 x 4096 bf16 164 -> 203 us).
template <typename T, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * kWave, BM == 128 ? 3 : 2) k_int8_tiles(DenseInt8Args a, int32_t m_tiles, int32_t n_tiles)
{
    constexpr int kWaves = (BM / WM) * (BN / WN), kLoads = (BM + BN) / 16 / kWaves;     // of 16 rows, by a wave and stage
    constexpr int MI = WM / 32, NI = WN / 32, kStage = (BM + BN) * 4;
    static_assert((BM + BN) / 16 % kWaves == 0 && BM / 16 % kLoads == 0, "a wave loads whole pieces of one side");
    __shared__ int4v s_stage[3 * kStage];
    __shared__ float s_scale[BM], s_w_scale[BN], s_bias[BN];
    const int32_t rows = a.count.get(), n = a.out.width;
    const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63;
    const int32_t block = (int32_t) (blockIdx.y * gridDim.x + blockIdx.x);
    if (block >= m_tiles * n_tiles) return;
    int32_t tm, tn;
    tile_of(xcd_run(block, m_tiles * n_tiles), m_tiles, n_tiles, &tm, &tn);
    const int64_t m0 = (int64_t) tm * BM;
    const int32_t n0 = tn * BN;
    if (m0 >= rows) return;
    const int32_t steps = (int32_t) (a.stride / kStepBytes);
    for (int i = (int) threadIdx.x; i < BM; i += kWaves * kWave) s_scale[i] = a.scale[m0 + i < rows ? m0 + i : rows - 1];
    for (int i = (int) threadIdx.x; i < BN; i += kWaves * kWave) {
        const int32_t c = n0 + i < n ? n0 + i : n - 1;
        s_w_scale[i] = a.w_scale[c];
        s_bias[i] = a.bias ? a.bias[c] : 0.f;
    }
    // this wave's pieces: 16 rows each, of the rows' side or the weights'; those past the end repeat the last
    const bool weights = wave * kLoads * 16 >= BM;
    const int32_t first = wave * kLoads * 16 - (weights ? BM : 0);
    const int64_t last = weights ? n - 1 - n0 : rows - 1 - m0;
    const int8_t* base = weights ? a.wq + (int64_t) n0 * a.stride : a.q + m0 * a.stride;
    const int32_t turned = (lane & 3) ^ row_turn(lane >> 2);
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int32_t row = first + i * 16 + (lane >> 2), at = (int32_t) (row < last ? row : last);
        from[i] = (uint32_t) at * (uint32_t) a.stride + (uint32_t) (lane & 3) * 16;
    }
    int4v* put_at = s_stage + (wave * kLoads * 16 + (lane >> 2)) * 4 + turned;
    int4v read[2][kLoads];
    const int8_t* next;                                       // of the step that is read
    auto seek = [&](int32_t step) { next = base + (int64_t) (step < steps ? step : steps - 1) * kStepBytes; };   // past the last: the last again
    auto fetch = [&](int set, int i) { read[set][i] = *reinterpret_cast<const int4v*>(next + from[i]); };
    auto put = [&](int set, int stage, int i) { put_at[stage * kStage + i * 64] = read[set][i]; };
    auto fetch_all = [&](int set, int32_t step) {
        seek(step);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) fetch(set, i);
        __builtin_amdgcn_sched_barrier(0);                    // in this order, or the first waits of the loop are for all reads
    };
    auto put_all = [&](int set, int stage) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) put(set, stage, i);
    };
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
    const int l32 = lane & 31, kh = lane >> 5, bank = row_turn(l32);
    int16v acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
    int4v f[2][MI + NI];                                      // fragments of the rows, then of the weights
    const int4v* x_at = s_stage + (wm + l32) * 4;
    const int4v* w_at = s_stage + (BM + wn + l32) * 4;
    auto get = [&](int h, int stage, int i) {
        const int chunk = (2 * h + kh) ^ bank;
        f[h][i] = i < MI ? x_at[stage * kStage + i * 128 + chunk] : w_at[stage * kStage + (i - MI) * 128 + chunk];
    };
    // the products of one half of a stage, and between them, one after the other, what else there is to do
    auto multiply = [&](int h, auto&& other, int others) {
        constexpr int kProducts = MI * NI;
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
            acc[m / NI][m % NI] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f[h][MI + m % NI], f[h][m / NI], acc[m / NI][m % NI], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int o = others * m / kProducts; o < others * (m + 1) / kProducts; ++o) other(o);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int s0 = 0, s1 = 1, s2 = 2;                               // stages of this step, the next and the one after
    fetch_all(0, 0);
    fetch_all(1, 1);
    put_all(0, 0);
    fetch_all(0, 2);
    put_all(1, 1);
    fetch_all(1, 3);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < MI + NI; ++i) get(0, 0, i);
    // stage `step` is multiplied; what was read for step + 2 goes to LDS, what is read now is for step + 4
    auto turn = [&](int set, int32_t step) {
        seek(step + 4);
        multiply(0, [&](int o) { if (o < MI + NI) get(1, s0, o); else put(set, s2, o - (MI + NI)); }, MI + NI + kLoads);
        multiply(1, [&](int o) { if (o < MI + NI) get(0, s1, o); else fetch(set, o - (MI + NI)); }, MI + NI + kLoads);
        const int t = s0;
        s0 = s1; s1 = s2; s2 = t;
        lds_barrier();
    };
    int32_t step = 0;
    for (; step + 2 <= steps; step += 2) {
        turn(0, step);
        turn(1, step + 1);
    }
    if (step < steps) turn(0, step);
    // Each strip of 32 rows goes through a piece of LDS of the wave's own, so that rows leave in pieces of 16 bytes.
    // (from a lane id the compiler cannot see through: what it would work out of this in front of the loop costs registers)
    constexpr int V = 16 / (int) sizeof(T), kLanes = WN / V, kPitch = WN * (int) sizeof(T) + 16;
    static_assert(kWaves * 32 * kPitch <= 3 * kStage * 16, "the strips lie in the stages' place");
    const int e_lane = opaque_lane_id(), e32 = e_lane & 31, four = 4 * (e_lane >> 5);
    char* const strip = reinterpret_cast<char*>(s_stage) + wave * (32 * kPitch);
    const int32_t c = n0 + wn + e_lane % kLanes * V;
    const bool far = __ballot(fabsf(s_w_scale[wn + e_lane % WN]) > kFarScale) != 0;
    auto finish = [&](auto is_far) {
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const float scale = s_scale[wm + i * 32 + e32];
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {                 // elements 4 q .. 4 q + 3: four columns of row e32
                    const int at = j * 32 + 8 * q + four;
                    const float4 ws = *reinterpret_cast<const float4*>(s_w_scale + wn + at), b = *reinterpret_cast<const float4*>(s_bias + wn + at);
                    struct alignas(4 * sizeof(T)) Four { T v[4]; } y;
                    constexpr bool kFar = decltype(is_far)::value;
                    y.v[0] = from_float<T>(output_of<kFar>(acc[i][j][4 * q], ws.x, scale, b.x, a.relu));
                    y.v[1] = from_float<T>(output_of<kFar>(acc[i][j][4 * q + 1], ws.y, scale, b.y, a.relu));
                    y.v[2] = from_float<T>(output_of<kFar>(acc[i][j][4 * q + 2], ws.z, scale, b.z, a.relu));
                    y.v[3] = from_float<T>(output_of<kFar>(acc[i][j][4 * q + 3], ws.w, scale, b.w, a.relu));
                    *reinterpret_cast<Four*>(strip + e32 * kPitch + at * (int) sizeof(T)) = y;
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < 32 * kLanes / kWave; ++t) {
                const int row = t * (kWave / kLanes) + e_lane / kLanes;
                const Chunk y = *reinterpret_cast<const Chunk*>(strip + row * kPitch + e_lane % kLanes * 16);
                const int64_t r = m0 + wm + i * 32 + row;
                if (r >= rows) continue;
                T* out = reinterpret_cast<T*>(a.out.data) + r * a.out.stride + c;
                if (c + V <= n) {
                    __builtin_memcpy(out, &y, 16);            // whatever the row's alignment
                } else {
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        if (c + k < n) out[k] = __builtin_bit_cast(Piece<T>, y).v[k];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (far) finish(std::true_type{});
    else     finish(std::false_type{});
}

// k_int8_few: for rows by the ten, where the weights' bytes are all there is to do (one row of 4096 bf16, 4096 channels: 6 us, 2.8
// TB/s of weights, half of it launch and the chain of three dependent reads).  A block has 16 output channels and
// all rows (16 a tile, up to MT tiles), its eight waves an eighth of k each, products of 16 x 16 x 64 bytes; their sums meet in
// LDS.  kFused: the block quantises the rows itself into LDS (every block does, which costs less than a launch in front), while
// its first weights are on their way.
constexpr int kFewBlock = 512, kFewWaves = kFewBlock / kWave, kFewColumns = 16;
constexpr int kFewDepth = 8;                  // reads of weights in flight
constexpr size_t kFewLds = 64 * 1024;         // of quantised rows

__host__ __device__ constexpr int64_t few_stride(int64_t stride) { return stride + 16; }        // of rows in LDS, off the banks' period

template <typename T, typename X, bool kFused, int MT>
__global__ void __launch_bounds__(kFewBlock) k_int8_few(DenseInt8Args a, QuantizeArgs x)
{
    constexpr int V = kPiece<X>;
    extern __shared__ int4v s_rows[];                         // kFused: the rows in 8 bits
    __shared__ int s_sum[kFewWaves][MT][4][kWave];
    __shared__ uint32_t s_most[16];
    const int32_t rows = a.count.get(), n = a.out.width, steps = (int32_t) (a.stride / 64);
    const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63;
    const int l16 = lane & 15, kg = lane >> 4;
    const int32_t n0 = (int32_t) blockIdx.x * kFewColumns, column = n0 + l16 < n ? n0 + l16 : n - 1;
    const int32_t s0 = (int32_t) ((int64_t) steps * wave / kFewWaves), s1 = (int32_t) ((int64_t) steps * (wave + 1) / kFewWaves);
    const int8_t* w = a.wq + (int64_t) column * a.stride + kg * 16;
    int4v read[kFewDepth];
    auto fetch = [&](int32_t from) {                          // steps past the last repeat it
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) read[d] = *reinterpret_cast<const int4v*>(w + (int64_t) (from + d < s1 ? from + d : s1 - 1) * 64);
    };
    if (s0 < s1) fetch(s0);
    if (rows <= 0) return;
    const int64_t pitch = few_stride(a.stride);
    int8_t* const s_q = reinterpret_cast<int8_t*>(s_rows);
    if (kFused) {
        // all rows at once, a team of 32 to 512 threads each; the second reading finds them near by
        const int32_t team = kFewBlock >> (rows > 1 ? 32 - __builtin_clz((uint32_t) rows - 1) : 0);
        const int32_t r = (int32_t) threadIdx.x / team, c0 = (int32_t) threadIdx.x % team * V;
        if (threadIdx.x < 16) s_most[threadIdx.x] = 0;
        __syncthreads();
        uint32_t most = 0;
        if (r < rows) {
#pragma unroll 4
            for (int32_t c = c0; c < a.k; c += team * V) {
                float v[V];
                load_piece<X>(x, r, c, v);
                most = largest_of(v, most);
            }
        }
        most = largest_of_lanes<32>(most);
        if ((lane & 31) == 0 && r < rows) atomicMax(&s_most[r], most);
        __syncthreads();
        if (r < rows) {
            const float inverse = row_scale(s_most[r]).inverse;
#pragma unroll 4
            for (int32_t c = c0; c < (int32_t) a.stride; c += team * V) {
                float v[V];
                load_piece<X>(x, r, c, v);
                store_piece<X>(s_q + r * pitch + c, v, inverse);
            }
        }
        __syncthreads();
    }
    const int8_t* q[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int32_t r = t * 16 + l16 < rows ? t * 16 + l16 : rows - 1;
        q[t] = (kFused ? s_q + r * pitch : a.q + (int64_t) r * a.stride) + kg * 16;
    }
    int4v acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = int4v{0, 0, 0, 0};
    for (int32_t s = s0; s < s1; s += kFewDepth) {
        int4v now[kFewDepth];
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) now[d] = read[d];
        if (s + kFewDepth < s1) fetch(s + kFewDepth);
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            if (s + d >= s1) break;                           // wave-uniform
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const int4v v = *reinterpret_cast<const int4v*>(q[t] + (int64_t) (s + d) * 64);
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v, now[d], acc[t], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) s_sum[wave][t][v][lane] = acc[t][v];
    __syncthreads();
    // element v of lane l is row 4 * (l / 16) + v, column l % 16
    for (int i = (int) threadIdx.x; i < MT * 4 * kWave; i += kFewBlock) {
        const int t = i / (4 * kWave), v = i / kWave % 4, l = i % kWave;
        const int32_t r = t * 16 + 4 * (l >> 4) + v, c = n0 + (l & 15);
        if (r >= rows || c >= n) continue;
        int sum = 0;
#pragma unroll
        for (int u = 0; u < kFewWaves; ++u) sum += s_sum[u][t][v][l];
        const float scale = kFused ? row_scale(s_most[r & 15]).scale : a.scale[r];
        store_at<T>(a.out, r, c, output_of<true>(sum, a.w_scale[c], scale, a.bias ? a.bias[c] : 0.f, a.relu));
    }
}

// k_int8_rows: many rows against weights that fit LDS: rows come in, are quantised and multiplied, and leave, without a
// trip through memory in 8 bits (85,000 rows, 256 x 256, fp32: 34 us, 5.1 TB/s in and out, with rows from the infinity cache, a call
// of 49 without, where a copy takes 34; in two kernels 17 and 44).
// A block per CU holds all weights; its waves walk tiles of 16 rows: a row is read by L lanes, P pieces each, quantised, turned
// through a piece of LDS of the wave's own and multiplied, 16 x 16 x 64 bytes, with the weights as the left factor, so that a
// lane gets four consecutive outputs of a row.  Bound by the rows' bytes, in and out; 85,000 rows are 1.3 tiles a wave, so
// reading, multiplying and writing overlap little.
constexpr int64_t rows_lds(int64_t stride, int32_t n, int waves)
{
    return (few_stride(stride) * ((n + 15) / 16 * 16 + waves * 16)) + (int64_t) (n + 15) / 16 * 16 * 8;
}

template <typename T, int L, int P, int kWaves>
__global__ void __launch_bounds__(kWaves * kWave) k_int8_rows(DenseInt8Args a, QuantizeArgs x)
{
    constexpr int V = kPiece<T>, kTurns = 16 * L / kWave;      // of a wave over a tile's rows
    constexpr int kGroups = 4;                                 // of 16 output columns, multiplied together
    extern __shared__ int4v s_rows[];
    const int32_t rows = a.count.get(), n = a.out.width, n16 = (n + 15) / 16 * 16, steps = (int32_t) (a.stride / 64);
    const int32_t pitch = (int32_t) few_stride(a.stride), f1 = x.x1.width, k = a.k;
    int8_t* const s_w = reinterpret_cast<int8_t*>(s_rows);
    const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6));
    int8_t* const s_q = s_w + n16 * pitch + wave * 16 * pitch;
    float* const s_scale = reinterpret_cast<float*>(s_w + (n16 + kWaves * 16) * pitch);
    float* const s_bias = s_scale + n16;
    const int32_t chunks = (int32_t) (a.stride / 16);
    for (int32_t i = (int32_t) threadIdx.x; i < n16 * chunks; i += kWaves * kWave) {
        const int32_t row = i / chunks, chunk = i - row * chunks;
        *reinterpret_cast<int4v*>(s_w + row * pitch + chunk * 16) =
            *reinterpret_cast<const int4v*>(a.wq + (int64_t) (row < n ? row : n - 1) * a.stride + chunk * 16);
    }
    for (int32_t i = (int32_t) threadIdx.x; i < n16; i += kWaves * kWave) {
        s_scale[i] = a.w_scale[i < n ? i : n - 1];
        s_bias[i] = a.bias ? a.bias[i < n ? i : n - 1] : 0.f;
    }
    __syncthreads();
    bool far = false;
    for (int32_t i = lane_id(); i < n16; i += kWave) far |= fabsf(s_scale[i]) > kFarScale;
    far = __ballot(far) != 0;
    const int32_t tiles = (rows + 15) / 16;
    const bool stores = n % 4 == 0 && reinterpret_cast<uintptr_t>(a.out.data) % 16 == 0 && (uint64_t) a.out.stride * sizeof(T) % 16 == 0;
    // A tile's rows are read when the one before has been quantised, and come while that one is multiplied and stored.  Rows past
    // the last are read as the last, lanes past the last column read the first.
    Piece<T> v[kTurns][P];
    auto fetch = [&](int32_t tile) {
        const int lane = opaque_lane_id(), l = lane & (L - 1);
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int64_t row = (int64_t) tile * 16 + t * (kWave / L) + lane / L, r = row < rows ? row : rows - 1;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int32_t c = (p * L + l) * V, cc = c < k ? c : 0;
                __builtin_memcpy(&v[t][p], cc < f1 ? reinterpret_cast<const T*>(x.x1.data) + r * x.x1.stride + cc
                                                   : reinterpret_cast<const T*>(x.x2.data) + r * x.x2.stride + (cc - f1), 16);
            }
        }
    };
    // the blocks' first waves take the first tiles: a remainder spreads over all CUs
    int32_t tile = wave * (int32_t) gridDim.x + (int32_t) blockIdx.x;
    if (tile < tiles) fetch(tile);
    for (; tile < tiles; tile += (int32_t) gridDim.x * kWaves) {
        const int lane = opaque_lane_id(), l = lane & (L - 1), l16 = lane & 15, kg = lane >> 4;
        const int64_t r0 = (int64_t) tile * 16;
        float scale = 0.f;                                    // of row l16
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            uint32_t most = 0;
            float f[P][V];
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int i = 0; i < V; ++i) f[p][i] = (p * L + l) * V < k ? to_float(v[t][p].v[i]) : 0.f;
                most = largest_of(f[p], most);
            }
            const RowScale s = row_scale(largest_of_lanes<L>(most));
            const int32_t row = t * (kWave / L) + lane / L;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if ((p * L + l) * V < (int32_t) a.stride) store_piece<T>(s_q + row * pitch + (p * L + l) * V, f[p], s.inverse);
            const float other = __shfl(s.scale, l16 % (kWave / L) * L);
            if (l16 / (kWave / L) == t) scale = other;
        }
        __builtin_amdgcn_wave_barrier();
        if (tile + (int32_t) gridDim.x * kWaves < tiles) fetch(tile + (int32_t) gridDim.x * kWaves);
        const int8_t* q = s_q + l16 * pitch + kg * 16;
        T* out = reinterpret_cast<T*>(a.out.data) + (r0 + l16) * a.out.stride;
        for (int32_t c0 = 0; c0 < n16; c0 += 16 * kGroups) {
            const int8_t* w[kGroups];
            int4v acc[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {               // groups past the last repeat it
                w[g] = s_w + ((c0 + g * 16 < n16 ? c0 + g * 16 : n16 - 16) + l16) * pitch + kg * 16;
                acc[g] = int4v{0, 0, 0, 0};
            }
            for (int32_t s = 0; s < steps; ++s) {
                const int4v right = *reinterpret_cast<const int4v*>(q + s * 64);
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
                    acc[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const int4v*>(w[g] + s * 64), right, acc[g], 0, 0, 0);
            }
            // element i of lane l is output column 4 * (l / 16) + i of row l % 16
            auto store_group = [&](auto is_far, int g) {
                constexpr bool kFar = decltype(is_far)::value;
                const int32_t c = c0 + g * 16 + 4 * kg;
                if (c0 + g * 16 >= n16 || r0 + l16 >= rows) return;
                const float4 ws = *reinterpret_cast<const float4*>(s_scale + c), b = *reinterpret_cast<const float4*>(s_bias + c);
                struct alignas(4 * sizeof(T)) Four { T v[4]; } y;
                y.v[0] = from_float<T>(output_of<kFar>(acc[g][0], ws.x, scale, b.x, a.relu));
                y.v[1] = from_float<T>(output_of<kFar>(acc[g][1], ws.y, scale, b.y, a.relu));
                y.v[2] = from_float<T>(output_of<kFar>(acc[g][2], ws.z, scale, b.z, a.relu));
                y.v[3] = from_float<T>(output_of<kFar>(acc[g][3], ws.w, scale, b.w, a.relu));
                if (stores) {
                    if (c < n) *reinterpret_cast<Four*>(out + c) = y;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c + i < n) out[c + i] = y.v[i];
                }
            };
            if (far) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) store_group(std::true_type{}, g);
            } else {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) store_group(std::false_type{}, g);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

static unsigned grid_of(const gns_ctx* c, int64_t blocks, int per_cu)
{
    const int64_t most = (int64_t) c->num_cus * per_cu;
    return (unsigned) (blocks < most ? blocks : most);
}

template <typename T>
static hipError_t launch_quantize_typed(const gns_ctx* c, const QuantizeArgs& a, hipStream_t s)
{
    const int64_t rows = a.count.rows, pieces = a.stride / kPiece<T>;
    const dim3 short_grid(grid_of(c, (rows + 15) / 16, 32)), wave_grid(grid_of(c, (rows + 3) / 4, 32)), block_grid(grid_of(c, rows, 32));
    if constexpr (kPiece<T> == 8) {               // rows in 8 bits are 64 bytes at least, sixteen pieces of fp32
        if (pieces <= 8) {
            hipLaunchKernelGGL((k_quantize_rows<T, 4, 2>), dim3(grid_of(c, (rows + 63) / 64, 32)), dim3(kBlock), 0, s, a);
            return hipGetLastError();
        }
    }
    if (pieces <= 32)        hipLaunchKernelGGL((k_quantize_rows<T, 16, 2>), short_grid, dim3(kBlock), 0, s, a);
    else if (pieces <= 64)   hipLaunchKernelGGL((k_quantize_rows<T, 16, 4>), short_grid, dim3(kBlock), 0, s, a);
    else if (pieces <= 256)  hipLaunchKernelGGL((k_quantize_rows<T, 64, 4>), wave_grid, dim3(kBlock), 0, s, a);
    else if (pieces <= 512)  hipLaunchKernelGGL((k_quantize_rows<T, 64, 8>), wave_grid, dim3(kBlock), 0, s, a);
    else if (pieces <= 1024) hipLaunchKernelGGL((k_quantize_block<T, 4>), block_grid, dim3(kBlock), 0, s, a);
    else if (pieces <= 2048) hipLaunchKernelGGL((k_quantize_block<T, 8>), block_grid, dim3(kBlock), 0, s, a);
    else                     hipLaunchKernelGGL((k_quantize_long<T>), dim3(grid_of(c, rows, 8)), dim3(kLongBlock), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_quantize(const gns_ctx* c, const QuantizeArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_quantize_typed<float>(c, a, s) : launch_quantize_typed<Bf16>(c, a, s);
}

template <typename T, int BM, int BN, int WM, int WN>
static hipError_t launch_tiles(const DenseInt8Args& a, hipStream_t s)
{
    // a dimension of a grid has fewer than 2^32 threads; 2^31 tiles of outputs fit no memory
    const int64_t m_tiles = ((int64_t) a.count.rows + BM - 1) / BM, n_tiles = (a.out.width + BN - 1) / BN, tiles = m_tiles * n_tiles, most = 1 << 22;
    if (tiles > INT32_MAX - most) return hipErrorInvalidValue;
    const dim3 grid((unsigned) (tiles < most ? tiles : most), (unsigned) ((tiles + most - 1) / most));
    hipLaunchKernelGGL((k_int8_tiles<T, BM, BN, WM, WN>), grid, dim3((BM / WM) * (BN / WN) * kWave), 0, s, a, (int32_t) m_tiles, (int32_t) n_tiles);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_typed(const gns_ctx* c, const DenseInt8Args& a, hipStream_t s)
{
    auto tiles = [&](int64_t bm, int64_t bn) { return (a.count.rows + bm - 1) / bm * ((a.out.width + bn - 1) / bn); };
    // Up to 64 rows a block per 16 channels, which divides k among its waves, while tiles would fill less than half the chip (with the
    // quantisation, bf16, 33 x 4096 x 4096: 16 us, 19 in tiles; 20 x 4096 x 4096: 13.5 and 19; 64 x 8192 x 8192: 46 and 32; 128 x 4096
    // x 4096 and smaller ones of that many rows: 27 and 20)
    if (a.count.rows <= 32 || (a.count.rows <= 64 && tiles(64, 64) * 2 < c->num_cus)) {
        const dim3 grid((unsigned) ((a.out.width + kFewColumns - 1) / kFewColumns));
        if (a.count.rows <= 16)      hipLaunchKernelGGL((k_int8_few<T, float, false, 1>), grid, dim3(kFewBlock), 0, s, a, QuantizeArgs{});
        else if (a.count.rows <= 32) hipLaunchKernelGGL((k_int8_few<T, float, false, 2>), grid, dim3(kFewBlock), 0, s, a, QuantizeArgs{});
        else                         hipLaunchKernelGGL((k_int8_few<T, float, false, 4>), grid, dim3(kFewBlock), 0, s, a, QuantizeArgs{});
        return hipGetLastError();
    }
    // Large tiles where five in eight CUs have one and a tile is long enough for a block to be alone on its CU (with the quantisation,
    // bf16, 3000 x 4096 x 4096, 192 tiles: 67 us, 80 with the next; 4096 x 4096 x 2048, 128 tiles: 63 and 59; 10,000 x 1500 x 4096:
    // 102 and 111; 40,000 x 768 x 1024: 94 and 88)
    if (tiles(256, 256) * 8 >= (int64_t) c->num_cus * 5 && a.k >= 1024) return launch_tiles<T, 256, 256, 128, 64>(a, s);
    if (tiles(128, 128) >= c->num_cus) return launch_tiles<T, 128, 128, 64, 64>(a, s);
    return launch_tiles<T, 64, 64, 32, 32>(a, s);
}

hipError_t launch_dense_int8(const gns_ctx* c, const DenseInt8Args& a, int32_t out_type, hipStream_t s)
{
    return out_type == GNS_FP32 ? launch_typed<float>(c, a, s) : launch_typed<Bf16>(c, a, s);
}

// Rows and weights of k_int8_rows: rows of whole pieces, as many as a tile's registers hold, weights that leave room in LDS, and
// two tiles for each wave of a block per CU, or reading the weights into every LDS costs more than it saves
template <typename T>
static bool rows_fit(const gns_ctx* c, const QuantizeArgs& x, const DenseInt8Args& a)
{
    return a.count.rows >= c->num_cus * 32 && a.stride <= 512 && a.k % kPiece<T> == 0 && x.x1.width % kPiece<T> == 0 &&
           rows_lds(a.stride, a.out.width, 8) <= (int64_t) c->lds_bitmap_limit;
}

template <typename T, int L, int P>
static void launch_rows_of(const gns_ctx* c, const QuantizeArgs& x, const DenseInt8Args& a, hipStream_t s)
{
    const int64_t lds16 = rows_lds(a.stride, a.out.width, 16), lds8 = rows_lds(a.stride, a.out.width, 8);
    if (P == 1 && lds16 <= (int64_t) c->lds_bitmap_limit) {
        const dim3 grid((unsigned) (c->num_cus * (lds16 <= 80 * 1024 ? 2 : 1)));
        hipLaunchKernelGGL((k_int8_rows<T, L, P, P == 1 ? 16 : 8>), grid, dim3(16 * kWave), (size_t) lds16, s, a, x);
    } else {
        const dim3 grid((unsigned) (c->num_cus * (lds8 <= 80 * 1024 ? 2 : 1)));
        hipLaunchKernelGGL((k_int8_rows<T, L, P, 8>), grid, dim3(8 * kWave), (size_t) lds8, s, a, x);
    }
}

template <typename T>
static hipError_t launch_rows(const gns_ctx* c, const QuantizeArgs& x, const DenseInt8Args& a, hipStream_t s)
{
    constexpr int V = kPiece<T>;
    if (a.stride <= 16 * V)      launch_rows_of<T, 16, 1>(c, x, a, s);
    else if (a.stride <= 32 * V) launch_rows_of<T, 32, 1>(c, x, a, s);
    else if (a.stride <= 64 * V) launch_rows_of<T, 64, 1>(c, x, a, s);
    else if constexpr (V == 4)   launch_rows_of<T, 64, 2>(c, x, a, s);
    return hipGetLastError();
}

template <typename T, typename X>
static void launch_few_fused(const QuantizeArgs& x, const DenseInt8Args& a, size_t lds, hipStream_t s)
{
    const dim3 grid((unsigned) ((a.out.width + kFewColumns - 1) / kFewColumns));
    hipLaunchKernelGGL((k_int8_few<T, X, true, 1>), grid, dim3(kFewBlock), lds, s, a, x);
}

hipError_t launch_sage_dense_int8(const gns_ctx* c, const QuantizeArgs& x, const DenseInt8Args& a, int32_t type, int32_t out_type,
                                  hipStream_t s)
{
    const int64_t lds = a.count.rows * few_stride(a.stride);
    if (a.count.rows <= 16 && lds <= (int64_t) kFewLds) {
        if (type == GNS_FP32 && out_type == GNS_FP32) launch_few_fused<float, float>(x, a, (size_t) lds, s);
        else if (type == GNS_FP32)                    launch_few_fused<Bf16, float>(x, a, (size_t) lds, s);
        else if (out_type == GNS_FP32)                launch_few_fused<float, Bf16>(x, a, (size_t) lds, s);
        else                                          launch_few_fused<Bf16, Bf16>(x, a, (size_t) lds, s);
        return hipGetLastError();
    }
    if (type == GNS_FP32 && out_type == GNS_FP32 && rows_fit<float>(c, x, a)) return launch_rows<float>(c, x, a, s);
    if (type == GNS_BF16 && out_type == GNS_BF16 && rows_fit<Bf16>(c, x, a)) return launch_rows<Bf16>(c, x, a, s);
    const hipError_t e = launch_quantize(c, x, type, s);
    return e != hipSuccess ? e : launch_dense_int8(c, a, out_type, s);
}

}  // namespace gns
