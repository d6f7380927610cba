// The backward pass of the update step out = g([x1 | x2] . W + b), with the layer's inputs from their 8-bit checkpoints:
//   dz = d_out where the output was positive,  dw = X^T dz,  db = sum_r dz,  dx = dz W^T.
// Both products run on the bf16 matrix cores at fp32's precision.  A checkpoint's values q * 2^e are bf16 values as they are.
// An fp32 value is cut into three bf16 terms of eight bits each, which hold it exactly: so dw takes three products of fp32
// gradients and one of bf16 ones, and is exact up to the fp32 sums.  dx of fp32 gradients takes the six products of terms that
// are not below 2^-23 of the largest; dx of bf16 gradients, itself rounded to bf16, takes W in two terms (2^-16).
#include "gns_learn.hpp"

namespace gns {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// Upper halves of two words, a's in the lower half.
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t lower_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Two values' three terms as packed pairs: each term is what is left, cut to its upper half.
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&t)[3])
{
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
        t[q] = upper_halves(ua, ub);
        a -= __uint_as_float(ua & 0xFFFF0000u);
        b -= __uint_as_float(ub & 0xFFFF0000u);
    }
}

// The products of terms: which term of the left factor meets which of the right, the smallest first.
template <int NA, int NB> struct Pairs;
template <> struct Pairs<1, 1> { static constexpr int kCount = 1, kA[1] = {0}, kB[1] = {0}; };
template <> struct Pairs<1, 2> { static constexpr int kCount = 2, kA[2] = {0, 0}, kB[2] = {1, 0}; };
template <> struct Pairs<1, 3> { static constexpr int kCount = 3, kA[3] = {0, 0, 0}, kB[3] = {2, 1, 0}; };
template <> struct Pairs<3, 3> { static constexpr int kCount = 6, kA[6] = {2, 0, 1, 1, 0, 0}, kB[6] = {0, 2, 1, 0, 1, 0}; };

constexpr int kStageK = 32;                   // k of a stage: 64 bytes of a row and plane

// BM x BN outputs of a block, WM x WN of a wave, from factors that lie in LDS as rows of kStageK bf16, a plane for each
// term, in products of 32 x 32 x 16.  There are three stages: one is multiplied, one is complete, one is being written.  What a
// wave reads from memory is read two stages before it is written to LDS, and that is one before its first fragments are
// taken; one barrier a stage.  Between the products, one after the other, stands what else there is to do.
template <int BM, int BN, int WM, int WN, int NA, int NB>
struct Tile {
    static constexpr int kM = BM, kN = BN, kThreads = (BM / WM) * (BN / WN) * kWave, MI = WM / 32, NI = WN / 32;
    static constexpr int kStage = (BM * NA + BN * NB) * 4, kFragments = MI * NA + NI * NB;
    typedef Pairs<NA, NB> P;

    uint4* lds;                               // [3 * kStage]
    const uint4 *a_at, *b_at;
    int kh, bank;
    uint4 f[2][kFragments];
    floatx16 acc[MI][NI];

    __device__ __forceinline__ explicit Tile(uint4* s) : lds(s)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63, l32 = lane & 31;
        kh = lane >> 5;
        bank = row_turn(l32);
        a_at = lds + (wave / (BN / WN) * WM + l32) * 4;
        b_at = lds + (BM * NA + wave % (BN / WN) * WN + l32) * 4;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    }
    // where a chunk of eight k of a row of the left or right factor goes
    static __device__ __forceinline__ int place_a(int plane, int row, int chunk) { return (plane * BM + row) * 4 + (chunk ^ row_turn(row)); }
    static __device__ __forceinline__ int place_b(int plane, int row, int chunk) { return (BM * NA + plane * BN + row) * 4 + (chunk ^ row_turn(row)); }

    __device__ __forceinline__ void get(int h, int stage, int i)
    {
        const int chunk = stage * kStage + ((2 * h + kh) ^ bank);
        if (i < MI * NA) f[h][i] = a_at[chunk + (i / MI * BM + i % MI * 32) * 4];
        else             f[h][i] = b_at[chunk + ((i - MI * NA) / NI * BN + (i - MI * NA) % NI * 32) * 4];
    }
    template <typename Other>
    __device__ __forceinline__ void multiply(int h, int others, Other&& other)
    {
        constexpr int kProducts = MI * NI * P::kCount;
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
            const int p = m / (MI * NI), i = m / NI % MI, j = m % NI;
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[h][P::kA[p] * MI + i]),
                                                                __builtin_bit_cast(bf16x8, f[h][MI * NA + P::kB[p] * NI + j]), acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int o = others * m / kProducts; o < others * (m + 1) / kProducts; ++o) other(o);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // Source: seek(set, step), then fetch(set, i), i < kFetches; put(set, stage, i), i < kPuts.  Steps past the last are read
    // and never multiplied.
    template <typename Source>
    __device__ __forceinline__ void run(Source& source, int32_t steps)
    {
        if (steps <= 0) return;
        int s0 = 0, s1 = 1, s2 = 2;                           // stages of this step, the next and the one after
        auto fetch_all = [&](int set, int32_t step) {
            source.seek(set, step);
#pragma unroll
            for (int i = 0; i < Source::kFetches; ++i) source.fetch(set, i);
            __builtin_amdgcn_sched_barrier(0);                // in this order, or the first waits of the loop are for all reads
        };
        auto put_all = [&](int set, int stage) {
#pragma unroll
            for (int i = 0; i < Source::kPuts; ++i) source.put(set, stage, i);
        };
        fetch_all(0, 0);
        fetch_all(1, 1);
        put_all(0, 0);
        fetch_all(0, 2);
        put_all(1, 1);
        fetch_all(1, 3);
        lds_barrier();
#pragma unroll
        for (int i = 0; i < kFragments; ++i) get(0, 0, i);
        auto turn = [&](int set, int32_t step) {
            multiply(0, kFragments + Source::kPuts, [&](int o) { if (o < kFragments) get(1, s0, o); else source.put(set, s2, o - kFragments); });
            source.seek(set, step + 4);
            multiply(1, kFragments + Source::kFetches, [&](int o) { if (o < kFragments) get(0, s1, o); else source.fetch(set, o - kFragments); });
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
    }
    // visit(row of LDS of the left factor, of the right one, value) for the lane's outputs; adjacent lanes have adjacent rows
    // of the right factor
    template <typename Visit>
    __device__ __forceinline__ void each(Visit&& visit)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = opaque_lane_id();
        const int m0 = wave / (BN / WN) * WM + 4 * (lane >> 5), n0 = wave % (BN / WN) * WN + (lane & 31);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v)
#pragma unroll
                for (int j = 0; j < NI; ++j) visit(m0 + i * 32 + 8 * (v >> 2) + (v & 3), n0 + j * 32, acc[i][j][v]);
    }
};

// ---- dw and db ----------------------------------------------------------------------------------------------------
// k of these products are the rows of the batch, so both factors are turned on their way to LDS: a thread reads columns of a few
// rows and writes them as rows.  X: four columns (a word) of four rows; dz: of eight rows a column of fp32 or two of bf16.
// What a wave needs of exponents and masks is one read, lane by lane, and handed round.  Columns are placed such that
// adjacent threads write adjacent rows of LDS.
struct WeightsArgs {
    BackwardArgs a;
    int32_t m_tiles, n_tiles, splits;
    float* dw;                                // [splits x (f1 + f2) x hdim]: the caller's if there is one split
    float* db;                                // [splits x hdim], or null
};

// Packed columns of X are those of x1's groups, then those of x2's.  Row of dw, or -1 where a group is padded.
__device__ __forceinline__ int32_t weight_row(const BackwardArgs& a, int32_t c)
{
    const int32_t p1 = a.x1.groups * 32;
    if (c < p1) return c < a.x1.width ? c : -1;
    return c - p1 < a.x2.width ? a.x1.width + c - p1 : -1;
}

// Column c of four (of two) read together lies at this row of LDS, and back.
__device__ __forceinline__ int quad_row(int c) { return (c & ~127) + (c & 3) * 32 + ((c & 127) >> 2); }
__device__ __forceinline__ int quad_column(int row) { return (row & ~127) + (row & 31) * 4 + ((row & 127) >> 5); }
__device__ __forceinline__ int pair_row(int c) { return (c & ~63) + (c & 1) * 32 + ((c & 63) >> 1); }
__device__ __forceinline__ int pair_column(int row) { return (row & ~63) + (row & 31) * 2 + ((row & 63) >> 5); }

// Threads and outputs of a block: 512 threads for 256 columns of X and 128 (fp32) or 256 (bf16) of dz, 256 threads for half of
// either.
template <typename T, int kThreads> struct WeightsTile;
template <> struct WeightsTile<float, 512> { typedef Tile<256, 128, 64, 64, 1, 3> Type; };
template <> struct WeightsTile<float, 256> { typedef Tile<128, 64, 64, 32, 1, 3> Type; };
template <> struct WeightsTile<Bf16, 512> { typedef Tile<256, 256, 128, 64, 1, 1> Type; };
template <> struct WeightsTile<Bf16, 256> { typedef Tile<128, 128, 64, 64, 1, 1> Type; };

// kPairs: bf16 columns are read two at a time (rows of an even number of them at 4-byte marks); else singly.
template <typename T, int kThreads, bool kMask, bool kPairs>
struct WeightsSource {
    typedef typename WeightsTile<T, kThreads>::Type Tiles;
    static constexpr bool kFloat = sizeof(T) == 4;
    static constexpr int kQuads = Tiles::kM / 4, kQuadsWave = kQuads < kWave ? kQuads : kWave;       // of columns, of X
    static constexpr int kLanes = kFloat ? Tiles::kN : Tiles::kN / 2;                               // that read a row of dz
    static constexpr int kReads = kFloat || kPairs ? 8 : 16;
    static constexpr int kFetches = 4 + 1 + (kMask ? 1 : 0) + kReads, kPuts = 4 + 4;
    static_assert(kQuads * 8 == kThreads && kLanes * 4 == kThreads, "each thread has its share of a stage");

    const BackwardArgs& a;
    Tiles& tile;
    int64_t r0, r1;                           // rows of the split
    int quad, rows4;                          // this thread's columns of X, and its four rows of a stage
    int column, chunk;                        // its first column of dz, and its eight rows
    const int8_t* q;                          // its columns, row 0
    const uint8_t* e;                         // the exponent this lane reads, row 0
    const T* z;                               // its column, row 0
    const uint32_t* m;                        // the word of the mask this lane reads, row 0
    int64_t q_stride, e_stride, m_stride, r;
    int e_row, m_row, to_second;
    bool sums;                                // whether db is wanted of this block
    uint32_t x[2][4], ex[2], d[2][kReads], words[2];
    int32_t left[2];                          // rows of the split from the step's first on
    uint32_t t[3][4];
    float sum[2];

    __device__ __forceinline__ WeightsSource(const BackwardArgs& args, Tiles& tiles, int64_t first, int64_t end, int32_t c0, int32_t n0)
        : a(args), tile(tiles), r0(first), r1(end)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63;
        const int32_t p1 = a.x1.groups * 32, all = p1 + a.x2.groups * 32, hdim = a.hdim;
        // columns past the last read the last ones again; they are not stored
        auto part_of = [&](int32_t c, int32_t* in) -> const PackedRows& { *in = c < p1 ? c : c - p1; return c < p1 ? a.x1 : a.x2; };
        quad = (int) threadIdx.x % kQuads;
        rows4 = (kQuads == kWave ? wave : (int) threadIdx.x / kQuads) * 4;
        int32_t in;
        const PackedRows& part = part_of(min(c0 + quad * 4, all - 4), &in);
        q = part.q + in;
        q_stride = (int64_t) part.groups * 32;
        constexpr int kGroups = kQuadsWave / 8;                // of the wave's columns; the first 32 lanes read a byte each
        e_row = wave * (kWave / kQuads) * 4 + (lane & 31) / kGroups;
        const PackedRows& part_e = part_of(min(c0 + ((lane & 31) % kGroups) * 32, all - 32), &in);
        e = part_e.exponents + in / 32;
        e_stride = part_e.groups;
        const int lanes0 = wave * kWave % kLanes;              // the wave's first column of dz (of bf16: first pair)
        chunk = wave * kWave / kLanes;
        column = kFloat ? lanes0 + lane : 2 * (lanes0 + lane);
        const int32_t n = min(n0 + column, kFloat ? hdim - 1 : kPairs ? hdim - 2 : hdim - 1);
        z = reinterpret_cast<const T*>(a.d_out.data) + n;
        to_second = min(n + 1, hdim - 1) - n;
        m_stride = (hdim + 31) / 32;
        constexpr int kWords = kFloat ? 2 : 4;                 // of the wave's columns; the first 16 or 32 lanes read one each
        m_row = chunk * 8 + (lane & (8 * kWords - 1)) / kWords;
        m = kMask ? a.positive + min((n0 + (kFloat ? lanes0 : 2 * lanes0)) / 32 + lane % kWords, (int32_t) m_stride - 1) : nullptr;
        sums = false;
        sum[0] = sum[1] = 0.f;
    }
    __device__ __forceinline__ void seek(int set, int32_t step)
    {
        r = r0 + (int64_t) step * kStageK;
        const int64_t rest = r1 - r;
        left[set] = (int32_t) (rest < kStageK ? rest : kStageK);
    }
    // Rows past the split's last are read as the last; they count as nothing.
    __device__ __forceinline__ int64_t row_at(int i) const { return r + i < r1 ? r + i : r1 - 1; }
    __device__ __forceinline__ void fetch(int set, int i)
    {
        if (i < 4) {
            x[set][i] = *reinterpret_cast<const uint32_t*>(q + row_at(rows4 + i) * q_stride);
        } else if (i == 4) {
            ex[set] = e[row_at(e_row) * e_stride];
        } else if (i < 5 + kReads) {
            const int j = i - 5;
            const T* from = z + row_at(chunk * 8 + j % 8) * a.d_out.stride;
            if constexpr (kFloat)      d[set][j] = *reinterpret_cast<const uint32_t*>(from);
            else if constexpr (kPairs) d[set][j] = *reinterpret_cast<const uint32_t*>(from);
            else                       d[set][j] = from[j < 8 ? 0 : to_second].bits;
        } else {
            words[set] = m[row_at(m_row) * m_stride];
        }
    }
    __device__ __forceinline__ void put(int set, int stage, int i)
    {
        if (i < 4) put_x(set, stage, i);
        else       put_z(set, stage, i - 4);
    }
    __device__ __forceinline__ void put_x(int set, int stage, int j)          // column j of the four
    {
        const int lane = (int) threadIdx.x & 63;
        constexpr int kGroups = kQuadsWave / 8;
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t byte = (uint32_t) __shfl((int) ex[set], (lane / kQuadsWave * 4 + i) * kGroups + lane % kQuadsWave / 8);
            const float scale = __uint_as_float(rows4 + i < left[set] ? byte << 23 : 0u);
            v[i] = __float_as_uint((float) (int8_t) (x[set][i] >> (8 * j)) * scale);
        }
        uint2* to = reinterpret_cast<uint2*>(tile.lds + stage * Tiles::kStage + Tiles::place_a(0, quad_row(quad * 4 + j), rows4 >> 3));
        to[(rows4 >> 2) & 1] = make_uint2(upper_halves(v[0], v[1]), upper_halves(v[2], v[3]));
    }
    __device__ __forceinline__ void put_z(int set, int stage, int p)          // rows 2 p and 2 p + 1 of the eight
    {
        const int lane = (int) threadIdx.x & 63;
        uint32_t v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = 2 * p + h;
            if constexpr (kFloat) {
                bool keep = chunk * 8 + i < left[set];
                if (kMask) keep = keep && ((uint32_t) __shfl((int) words[set], i * 2 + (lane >> 5)) >> (lane & 31) & 1u);
                v[h] = keep ? d[set][i] : 0u;
            } else {
                v[h] = kPairs ? d[set][i] : d[set][i] | d[set][i + kReads - 8] << 16;
                uint32_t keep = chunk * 8 + i < left[set] ? 3u : 0u;
                if (kMask) keep &= (uint32_t) __shfl((int) words[set], i * 4 + (lane >> 4)) >> (2 * (lane & 15));
                v[h] &= (keep & 1u ? 0xFFFFu : 0u) | (keep & 2u ? 0xFFFF0000u : 0u);
            }
        }
        if constexpr (kFloat) {
            if (sums) sum[0] += __uint_as_float(v[0]) + __uint_as_float(v[1]);
            uint32_t pair[3];
            split_pair(__uint_as_float(v[0]), __uint_as_float(v[1]), pair);
#pragma unroll
            for (int k = 0; k < 3; ++k) t[k][p] = pair[k];
        } else {
            t[0][p] = lower_halves(v[0], v[1]);
            t[1][p] = upper_halves(v[0], v[1]);
            if (sums) {
                sum[0] += __uint_as_float(v[0] << 16) + __uint_as_float(v[1] << 16);
                sum[1] += __uint_as_float(v[0] & 0xFFFF0000u) + __uint_as_float(v[1] & 0xFFFF0000u);
            }
        }
        if (p < 3) return;
        uint4* to = tile.lds + stage * Tiles::kStage;
        if constexpr (kFloat) {
#pragma unroll
            for (int k = 0; k < 3; ++k) to[Tiles::place_b(k, column, chunk)] = make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]);
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) to[Tiles::place_b(0, pair_row(column + k), chunk)] = make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]);
        }
    }
};

template <typename T, int kThreads, bool kMask, bool kPairs>
__global__ void __launch_bounds__(kThreads) k_backward_weights(WeightsArgs g)
{
    typedef WeightsSource<T, kThreads, kMask, kPairs> Source;
    typedef typename Source::Tiles Tiles;
    __shared__ uint4 s_stage[3 * Tiles::kStage];
    const BackwardArgs& a = g.a;
    const int64_t rows = a.count.get();
    const int32_t all = g.m_tiles * g.n_tiles, t = xcd_run((int32_t) blockIdx.x, all * g.splits), split = t / all;
    int32_t tm, tn;
    tile_of(t - split * all, g.m_tiles, g.n_tiles, &tm, &tn);
    const int32_t c0 = tm * Tiles::kM, n0 = tn * Tiles::kN;
    const int64_t each = ((rows + g.splits - 1) / g.splits + kStageK - 1) / kStageK * kStageK;
    const int64_t first = split * each < rows ? split * each : rows, end = first + each < rows ? first + each : rows;
    Tiles tile(s_stage);
    Source source(a, tile, first, end, c0, n0);
    source.sums = g.db && tm == 0;
    tile.run(source, (int32_t) ((end - first + kStageK - 1) / kStageK));
    if (g.db && tm == 0) {                                    // eight rows a thread and stage, four chunks of them
        float* s_sum = reinterpret_cast<float*>(s_stage);     // [4][Tiles::kN]
        __syncthreads();
        s_sum[source.chunk * Tiles::kN + source.column] = source.sum[0];
        if (sizeof(T) == 2) s_sum[source.chunk * Tiles::kN + source.column + 1] = source.sum[1];
        __syncthreads();
        const int n = (int) threadIdx.x;
        if (n < Tiles::kN && n0 + n < a.hdim)
            g.db[(int64_t) split * a.hdim + n0 + n] = (s_sum[n] + s_sum[Tiles::kN + n]) + (s_sum[2 * Tiles::kN + n] + s_sum[3 * Tiles::kN + n]);
    }
    float* dw = g.dw + (int64_t) split * (a.x1.width + a.x2.width) * a.hdim;
    tile.each([&](int m, int n, float v) {
        const int32_t k = weight_row(a, c0 + quad_column(m)), c = n0 + (sizeof(T) == 4 ? n : pair_column(n));
        if (k >= 0 && c < a.hdim) dw[(int64_t) k * a.hdim + c] = v;
    });
}

// Sums of the splits, in their order.
__global__ void __launch_bounds__(kBlock) k_join_splits(const float* parts, int32_t splits, int64_t n, float* out)
{
    for (int64_t i = (int64_t) blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t) gridDim.x * kBlock) {
        float v = 0.f;
#pragma unroll 8
        for (int32_t s = 0; s < splits; ++s) v += parts[s * n + i];
        out[i] = v;
    }
}

// ---- dx -----------------------------------------------------------------------------------------------------------
// W in bf16 terms: [plane][f1 + f2][hdim rounded up to kStageK], zeros behind hdim.
__global__ void __launch_bounds__(kBlock) k_split_weights(const float* w, int64_t rows, int32_t hdim, int32_t pitch, int planes, uint16_t* out)
{
    const int64_t n = rows * pitch;
    for (int64_t i = (int64_t) blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t) gridDim.x * kBlock) {
        const int64_t r = i / pitch;
        const int32_t c = (int32_t) (i - r * pitch);
        float v = c < hdim ? w[r * hdim + c] : 0.f;
        for (int p = 0; p < planes; ++p) {
            const uint32_t u = __float_as_uint(v);
            out[p * n + i] = (uint16_t) (u >> 16);
            v -= __uint_as_float(u & 0xFFFF0000u);
        }
    }
}

struct InputArgs {
    BackwardArgs a;
    int32_t m_tiles, n_tiles, pitch;
    const uint16_t* w;                        // k_split_weights' planes
};

template <typename T, int kThreads> struct InputTile;
template <> struct InputTile<float, 512> { typedef Tile<128, 128, 64, 32, 3, 3> Type; };
template <> struct InputTile<float, 256> { typedef Tile<64, 64, 32, 32, 3, 3> Type; };
template <> struct InputTile<Bf16, 512> { typedef Tile<256, 128, 64, 64, 1, 2> Type; };
template <> struct InputTile<Bf16, 256> { typedef Tile<128, 128, 64, 64, 1, 2> Type; };

// A thread reads eight columns of a row of dz (of two rows of bf16), and as many of W's planes.  kWhole: rows of dz begin at
// 16-byte marks and hdim is a multiple of eight, so eight columns are one or two reads; else they are read singly.
template <typename T, int kThreads, bool kMask, bool kWhole>
struct InputSource {
    typedef typename InputTile<T, kThreads>::Type Tiles;
    static constexpr bool kFloat = sizeof(T) == 4;
    static constexpr int kPlanes = kFloat ? 3 : 2, kStep = kThreads / 4;                            // rows the threads cover at once
    static constexpr int kRowsA = Tiles::kM / kStep, kRowsB = Tiles::kN / kStep, kWords = kFloat ? 8 : 4;
    static constexpr int kFetches = kRowsA * (1 + (kMask ? 1 : 0)) + kRowsB * kPlanes;
    static constexpr int kPuts = kRowsA * 4 + kRowsB * kPlanes;

    const BackwardArgs& a;
    Tiles& tile;
    int row, chunk;
    int32_t n, pitch, words_each;
    const T* z[kRowsA];
    const uint32_t* m[kRowsA];
    const uint16_t* w[kRowsB];
    int64_t plane;
    uint32_t d[2][kRowsA][kWords], words[2][kRowsA];
    uint4 planes[2][kRowsB][kPlanes];
    int32_t at[2];                            // the step's first column for this thread
    uint32_t t[3][4];

    __device__ __forceinline__ InputSource(const InputArgs& g, Tiles& tiles, int64_t r0, int64_t rows, int32_t k0) : a(g.a), tile(tiles), pitch(g.pitch)
    {
        row = (int) threadIdx.x >> 2;
        chunk = (int) threadIdx.x & 3;
        words_each = (a.hdim + 31) / 32;
        const int64_t K = a.x1.width + a.x2.width;
        plane = K * pitch;
#pragma unroll
        for (int i = 0; i < kRowsA; ++i) {                    // rows past the last are read as the last; they are not stored
            const int64_t r = min(r0 + row + i * kStep, rows - 1);
            z[i] = reinterpret_cast<const T*>(a.d_out.data) + r * a.d_out.stride;
            if constexpr (kMask) m[i] = a.positive + r * words_each;
        }
#pragma unroll
        for (int i = 0; i < kRowsB; ++i) w[i] = g.w + min((int64_t) k0 + row + i * kStep, K - 1) * pitch;
    }
    __device__ __forceinline__ void seek(int set, int32_t step)
    {
        n = step * kStageK + chunk * 8;
        at[set] = n;
    }
    __device__ __forceinline__ void fetch(int set, int i)
    {
        if (i < kRowsA) {
            if constexpr (kWhole) {
                const T* from = z[i] + min(n, a.hdim - 8);
#pragma unroll
                for (int j = 0; j < kWords / 4; ++j) {
                    const uint4 v = reinterpret_cast<const uint4*>(from)[j];
                    d[set][i][4 * j] = v.x; d[set][i][4 * j + 1] = v.y; d[set][i][4 * j + 2] = v.z; d[set][i][4 * j + 3] = v.w;
                }
            } else if constexpr (kFloat) {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[set][i][j] = reinterpret_cast<const uint32_t*>(z[i])[min(n + j, a.hdim - 1)];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    d[set][i][j] = z[i][min(n + 2 * j, a.hdim - 1)].bits | (uint32_t) z[i][min(n + 2 * j + 1, a.hdim - 1)].bits << 16;
            }
        } else if (i < kRowsA + kRowsB * kPlanes) {
            const int b = (i - kRowsA) / kPlanes, p = (i - kRowsA) % kPlanes;
            planes[set][b][p] = *reinterpret_cast<const uint4*>(w[b] + p * plane + min(n, pitch - 8));
        } else {
            const int b = i - kRowsA - kRowsB * kPlanes;
            words[set][b] = m[b][min(n >> 5, words_each - 1)];
        }
    }
    __device__ __forceinline__ void put(int set, int stage, int i)
    {
        uint4* to = tile.lds + stage * Tiles::kStage;
        if (i >= kRowsA * 4) {
            const int b = (i - kRowsA * 4) / kPlanes, p = (i - kRowsA * 4) % kPlanes;
            to[Tiles::place_b(p, row + b * kStep, chunk)] = planes[set][b][p];
            return;
        }
        const int b = i / 4, p = i % 4;                       // columns 2 p and 2 p + 1 of the eight
        const int32_t c = at[set] + 2 * p;
        uint32_t keep = (c < a.hdim ? 1u : 0u) | (c + 1 < a.hdim ? 2u : 0u);
        if (kMask) keep &= words[set][b] >> (chunk * 8 + 2 * p);
        if constexpr (kFloat) {
            uint32_t pair[3];
            split_pair(__uint_as_float(keep & 1u ? d[set][b][2 * p] : 0u), __uint_as_float(keep & 2u ? d[set][b][2 * p + 1] : 0u), pair);
#pragma unroll
            for (int k = 0; k < 3; ++k) t[k][p] = pair[k];
        } else {
            t[0][p] = d[set][b][p] & ((keep & 1u ? 0xFFFFu : 0u) | (keep & 2u ? 0xFFFF0000u : 0u));
        }
        if (p < 3) return;
#pragma unroll
        for (int k = 0; k < (kFloat ? 3 : 1); ++k) to[Tiles::place_a(k, row + b * kStep, chunk)] = make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]);
    }
};

template <typename T, int kThreads, bool kMask, bool kWhole>
__global__ void __launch_bounds__(kThreads) k_backward_input(InputArgs g)
{
    typedef InputSource<T, kThreads, kMask, kWhole> Source;
    typedef typename Source::Tiles Tiles;
    __shared__ uint4 s_stage[3 * Tiles::kStage];
    const BackwardArgs& a = g.a;
    const int64_t rows = a.count.get();
    int32_t tm, tn;
    tile_of(xcd_run((int32_t) blockIdx.x, g.m_tiles * g.n_tiles), g.m_tiles, g.n_tiles, &tm, &tn);
    const int64_t r0 = (int64_t) tm * Tiles::kM;
    const int32_t k0 = tn * Tiles::kN, K = a.x1.width + a.x2.width;
    if (r0 >= rows) return;
    Tiles tile(s_stage);
    Source source(g, tile, r0, rows, k0);
    tile.run(source, g.pitch / kStageK);
    T* out = reinterpret_cast<T*>(a.dx.data);
    tile.each([&](int m, int n, float v) {
        if (r0 + m < rows && k0 + n < K) out[(r0 + m) * a.dx.stride + k0 + n] = from_float<T>(v);
    });
}

// ---- launches -----------------------------------------------------------------------------------------------------
static size_t align256(size_t n) { return (n + 255) / 256 * 256; }

static unsigned grid_of(const gns_ctx* c, int64_t n)
{
    const int64_t blocks = (n + kBlock - 1) / kBlock, most = (int64_t) c->num_cus * 16;
    return (unsigned) (blocks < most ? blocks : most);
}

// Whether bf16 columns are read two at a time
static bool reads_pairs(const ConstRows& d_out)
{
    return d_out.width % 2 == 0 && reinterpret_cast<uintptr_t>(d_out.data) % 4 == 0 && d_out.stride % 2 == 0;
}

// How a call's weights' gradient is shared out.
struct WeightsPlan {
    bool wide;                                // blocks of 512 threads
    int32_t m_tiles, n_tiles, splits;
};

static WeightsPlan plan_weights(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int64_t rows, bool fp32, bool wide)
{
    WeightsPlan p;
    const int32_t columns = ((f1 + 31) / 32 + (f2 + 31) / 32) * 32, n512 = fp32 ? 128 : 256;
    p.wide = wide && columns > 128 && hdim > n512 / 2;
    const int32_t bm = p.wide ? 256 : 128, bn = p.wide ? n512 : n512 / 2;
    p.m_tiles = (columns + bm - 1) / bm;
    p.n_tiles = (hdim + bn - 1) / bn;
    const int64_t blocks = (int64_t) c->num_cus * (p.wide ? 1 : 2), most = (rows + 127) / 128;
    int64_t s = blocks / ((int64_t) p.m_tiles * p.n_tiles);
    if (s > most) s = most;
    p.splits = s < 1 ? 1 : (int32_t) s;
    return p;
}

size_t backward_workspace(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int32_t rows)
{
    const size_t k = (size_t) f1 + (size_t) f2, pitch = ((size_t) hdim + kStageK - 1) / kStageK * kStageK;
    size_t parts = 0;
    for (int i = 0; i < 3; ++i) {                              // of either type, and of bf16 columns read singly
        const WeightsPlan p = plan_weights(c, f1, f2, hdim, rows, i == 0, i < 2);
        const size_t need = p.splits > 1 ? align256((size_t) p.splits * k * (size_t) hdim * 4) + align256((size_t) p.splits * (size_t) hdim * 4) : 0;
        if (need > parts) parts = need;
    }
    return parts + align256(3 * k * pitch * 2);
}

// A grid's blocks times their threads stay below 2^32.
static bool too_many(int64_t blocks, int threads) { return blocks * threads >= (int64_t) 1 << 32; }

template <typename T, int kThreads>
static hipError_t launch_weights(const WeightsArgs& g, hipStream_t s)
{
    if (too_many((int64_t) g.m_tiles * g.n_tiles * g.splits, kThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned) (g.m_tiles * g.n_tiles * g.splits)), block(kThreads);
    if constexpr (sizeof(T) == 2 && kThreads == 256) {
        if (!reads_pairs(g.a.d_out)) {
            if (g.a.positive) hipLaunchKernelGGL((k_backward_weights<T, kThreads, true, false>), grid, block, 0, s, g);
            else              hipLaunchKernelGGL((k_backward_weights<T, kThreads, false, false>), grid, block, 0, s, g);
            return hipGetLastError();
        }
    }
    if (g.a.positive) hipLaunchKernelGGL((k_backward_weights<T, kThreads, true, true>), grid, block, 0, s, g);
    else              hipLaunchKernelGGL((k_backward_weights<T, kThreads, false, true>), grid, block, 0, s, g);
    return hipGetLastError();
}

template <typename T, int kThreads>
static hipError_t launch_input(InputArgs g, hipStream_t s)
{
    typedef typename InputTile<T, kThreads>::Type Tiles;
    g.m_tiles = (int32_t) (((int64_t) g.a.count.rows + Tiles::kM - 1) / Tiles::kM);
    g.n_tiles = (g.a.x1.width + g.a.x2.width + Tiles::kN - 1) / Tiles::kN;
    if (too_many((int64_t) g.m_tiles * g.n_tiles, kThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned) (g.m_tiles * g.n_tiles)), block(kThreads);
    const bool whole = g.a.hdim % 8 == 0 && reinterpret_cast<uintptr_t>(g.a.d_out.data) % 16 == 0 && (uint64_t) g.a.d_out.stride * sizeof(T) % 16 == 0;
    if (g.a.positive && whole)  hipLaunchKernelGGL((k_backward_input<T, kThreads, true, true>), grid, block, 0, s, g);
    else if (g.a.positive)      hipLaunchKernelGGL((k_backward_input<T, kThreads, true, false>), grid, block, 0, s, g);
    else if (whole)             hipLaunchKernelGGL((k_backward_input<T, kThreads, false, true>), grid, block, 0, s, g);
    else                        hipLaunchKernelGGL((k_backward_input<T, kThreads, false, false>), grid, block, 0, s, g);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_typed(const gns_ctx* c, const BackwardArgs& a, hipStream_t s)
{
    constexpr bool kFloat = sizeof(T) == 4;
    const int32_t K = a.x1.width + a.x2.width;
    const int64_t pitch = ((int64_t) a.hdim + kStageK - 1) / kStageK * kStageK;
    char* at = static_cast<char*>(a.workspace);
    if (a.dw) {
        const WeightsPlan p = plan_weights(c, a.x1.width, a.x2.width, a.hdim, a.count.rows, kFloat, kFloat || reads_pairs(a.d_out));
        WeightsArgs g = {a, p.m_tiles, p.n_tiles, p.splits, a.dw, a.db};
        if (p.splits > 1) {
            g.dw = reinterpret_cast<float*>(at);
            at += align256((size_t) p.splits * (size_t) K * (size_t) a.hdim * 4);
            g.db = a.db ? reinterpret_cast<float*>(at) : nullptr;
            at += align256((size_t) p.splits * (size_t) a.hdim * 4);
        }
        const hipError_t e = p.wide ? launch_weights<T, 512>(g, s) : launch_weights<T, 256>(g, s);
        if (e != hipSuccess) return e;
        if (p.splits > 1) {
            const int64_t n = (int64_t) K * a.hdim;
            hipLaunchKernelGGL(k_join_splits, dim3(grid_of(c, n)), dim3(kBlock), 0, s, g.dw, p.splits, n, a.dw);
            if (a.db) hipLaunchKernelGGL(k_join_splits, dim3(grid_of(c, a.hdim)), dim3(kBlock), 0, s, g.db, p.splits, (int64_t) a.hdim, a.db);
        }
    }
    if (a.dx.data && a.count.rows) {
        InputArgs g = {a, 0, 0, (int32_t) pitch, reinterpret_cast<const uint16_t*>(at)};
        hipLaunchKernelGGL(k_split_weights, dim3(grid_of(c, K * pitch)), dim3(kBlock), 0, s, a.w, (int64_t) K, a.hdim, (int32_t) pitch, kFloat ? 3 : 2,
                           reinterpret_cast<uint16_t*>(at));
        typedef typename InputTile<T, 512>::Type Wide;
        const int64_t tiles = ((int64_t) a.count.rows + Wide::kM - 1) / Wide::kM * ((K + Wide::kN - 1) / Wide::kN);
        return tiles >= c->num_cus ? launch_input<T, 512>(g, s) : launch_input<T, 256>(g, s);
    }
    return hipGetLastError();
}

hipError_t launch_backward(const gns_ctx* c, const BackwardArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_typed<float>(c, a, s) : launch_typed<Bf16>(c, a, s);
}

}  // namespace gns
