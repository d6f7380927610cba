// The backward pass of the update step out = g([x1 | x2] . W + b), with the layer's inputs from their 8-bit checkpoints:
//   dz = d_out where the output was positive,  dw = X^T dz,  db = sum_r dz,  dx = dz W^T.
// Both products run on the bf16 matrix cores at fp32's precision.  A checkpoint's values q * 2^e are bf16 values as they are.
// An fp32 value is cut into three bf16 terms, each what is left rounded to nearest, which hold it exactly: so dw takes three
// products of fp32 gradients and one of bf16 ones, and is exact up to the fp32 sums.  dx of bf16 gradients takes three products
// with W's terms and is as exact (two terms that are cut moved single bf16 results, 2.1e-4 of dx's 2-norm from the fp32 products'
// at hdim 4096, and saved a fifth of a large call); dx of fp32 gradients takes six products of terms: the three left out are at
// most 2^-24 of the factors' magnitudes together, to either side (of terms that are cut, 2^-21 and always to one).
#include "gns_learn.hpp"

namespace gns {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// Upper halves of two words, a's in the lower half.
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t lower_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// fp32 values are multiplied by 2^24 before they are cut, so that every term of every value is a normal bf16 value or zero (the
// matrix cores take subnormal ones as zero), and sums of products by as many 2^-24 as there are such factors.  What overflows on the
// way (a factor of 2^104, a sum of 2^80 with both factors scaled) is a sum that is not finite.  It costs fp32 calls 1 to 3 %.
constexpr float kTermScale = 0x1p24f;
__device__ __forceinline__ void scale_up(uint32_t (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * kTermScale);
}

// The leading bf16 terms of two values (rounded to nearest), packed, which are taken off the values.
__device__ __forceinline__ uint32_t take_term(float& a, float& b)
{
    const uint32_t t = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
    a -= __uint_as_float(t << 16);
    b -= __uint_as_float(t & 0xFFFF0000u);
    return t;
}
__device__ __forceinline__ Chunk take_terms(uint32_t (&v)[8])
{
    Chunk t;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        float a = __uint_as_float(v[2 * p]), b = __uint_as_float(v[2 * p + 1]);
        t[p] = take_term(a, b);
        v[2 * p] = __float_as_uint(a);
        v[2 * p + 1] = __float_as_uint(b);
    }
    return t;
}

// All bits set if bit i of w is, else none.
__device__ __forceinline__ uint32_t spread_bit(uint32_t w, int i) { return (uint32_t) __builtin_amdgcn_sbfe((int) w, (uint32_t) i, 1); }

// Lane kLane of each row of sixteen lanes, for all of the row (kBanks: for those of its quarters that have a bit; others keep `old`)
template <int kLane, int kBanks = 0xf>
__device__ __forceinline__ uint32_t row_broadcast(uint32_t old, uint32_t v)
{
    return (uint32_t) __builtin_amdgcn_update_dpp((int) old, (int) v, 0x150 + kLane, 0xf, kBanks, false);
}

// ---- sums that are not finite --------------------------------------------------------------------------------------
// The terms of an infinity do not add up to it, and what only fills a tile (zeros times repeated rows) makes NaN of one.  A sum
// that is not finite is therefore computed once more by a thread alone, with plain fp32 products; a NaN ends it.
__device__ __forceinline__ bool is_finite(float v) { return fabsf(v) < __builtin_inff(); }

// dz[r, n]
template <typename T, bool kMask>
__device__ __forceinline__ float masked_at(const BackwardArgs& a, int64_t r, int32_t n)
{
    if (kMask && !(a.positive[r * ((a.hdim + 31) / 32) + n / 32] >> (n & 31) & 1u)) return 0.f;
    return load_at<T>(a.d_out, r, n);
}

// dx[r, k] of columns `begin` to `end` of dz
template <typename T, bool kMask>
__device__ __forceinline__ float input_again(const BackwardArgs& a, int64_t r, int32_t k, int32_t begin, int32_t end)
{
    const float* w = a.w + (int64_t) k * a.hdim;
    float sum = 0.f;
    for (int32_t n = begin; n < end && sum == sum; ++n) sum = fmaf(masked_at<T, kMask>(a, r, n), w[n], sum);
    return sum;
}

// dw[k, n] of rows `begin` to `end`
template <typename T, bool kMask>
__device__ __forceinline__ float weight_again(const BackwardArgs& a, int32_t k, int32_t n, int64_t begin, int64_t end)
{
    const PackedRows& x = k < a.x1.width ? a.x1 : a.x2;
    const int32_t c = k < a.x1.width ? k : k - a.x1.width;
    float sum = 0.f;
    for (int64_t r = begin; r < end && sum == sum; ++r) {
        const float scale = __uint_as_float((uint32_t) x.exponents[r * x.groups + c / 32] << 23);
        sum = fmaf((float) x.q[r * x.groups * 32 + c] * scale, masked_at<T, kMask>(a, r, n), sum);
    }
    return sum;
}

// The products of terms: which term of the left factor meets which of the right, the smallest first.  Where both factors are cut,
// the leading terms' product, the last, has an accumulator of its own: the large sum is rounded once with every k of a product and
// not six times (dx of 85,000 rows of 256 x 256 7.0e-8 off in the 2-norm, 2.3e-7 with one, fp32 products 2.0e-7).
template <int NA, int NB> struct Pairs;
template <> struct Pairs<1, 1> { static constexpr int kCount = 1, kA[1] = {0}, kB[1] = {0}; };
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
    static constexpr bool kTwo = NA > 1 && NB > 1;

    Chunk* lds;                               // [3 * kStage]
    const Chunk *a_at, *b_at;
    int kh, bank;
    Chunk f[2][kFragments];
    floatx16 acc[MI][NI], rest[kTwo ? MI : 1][kTwo ? NI : 1];

    __device__ __forceinline__ explicit Tile(Chunk* s) : lds(s)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63, l32 = lane & 31;
        kh = lane >> 5;
        bank = row_turn(l32);
        a_at = lds + (wave / (BN / WN) * WM + l32) * 4;
        b_at = lds + (BM * NA + wave % (BN / WN) * WN + l32) * 4;
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
            floatx16& to = kTwo && p + 1 < P::kCount ? rest[kTwo ? i : 0][kTwo ? j : 0] : acc[i][j];
            to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[h][P::kA[p] * MI + i]),
                                                         __builtin_bit_cast(bf16x8, f[h][MI * NA + P::kB[p] * NI + j]), to, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int o = others * m / kProducts; o < others * (m + 1) / kProducts; ++o) other(o);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // `tiles` tiles of `steps` steps each (a multiple of Source::kSets), one after the other without a pause; finish(tile) takes
    // each one's outputs.  Source: seek(set), which goes on to the next step, then fetch(set, i), i < kFetches; put(set, stage, i),
    // i < kPuts.  Steps past the last are read and never multiplied.
    template <typename Source, typename Finish>
    __device__ __forceinline__ void run(Source& source, int32_t steps, int32_t tiles, Finish&& finish)
    {
        constexpr int kSets = Source::kSets;
        int s0 = 0, s1 = 1, s2 = 2;                           // stages of this step, the next and the one after
        auto fetch_all = [&](int set) {
            source.seek(set);
#pragma unroll
            for (int i = 0; i < Source::kFetches; ++i) source.fetch(set, i);
            __builtin_amdgcn_sched_barrier(0);                // in this order, or the first waits of the loop are for all reads
        };
        auto put_all = [&](int set, int stage) {
#pragma unroll
            for (int i = 0; i < Source::kPuts; ++i) source.put(set, stage, i);
        };
        // a stage is multiplied; what was read for the step after the next goes to LDS, what is read now is for kSets further on
        auto turn = [&](int set) {
            multiply(0, kFragments + Source::kPuts, [&](int o) { if (o < kFragments) get(1, s0, o); else source.put(set, s2, o - kFragments); });
            source.seek(set);
            multiply(1, kFragments + Source::kFetches, [&](int o) { if (o < kFragments) get(0, s1, o); else source.fetch(set, o - kFragments); });
            const int t = s0;
            s0 = s1; s1 = s2; s2 = t;
            lds_barrier();
        };
        if (steps > 0) {
            fetch_all(0);
            fetch_all(1);
            put_all(0, 0);
            put_all(1, 1);
#pragma unroll
            for (int i = 0; i < kSets; ++i) fetch_all(i);
            lds_barrier();
#pragma unroll
            for (int i = 0; i < kFragments; ++i) get(0, 0, i);
        }
        for (int32_t tile = 0; tile < tiles; ++tile) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        acc[i][j][v] = 0.f;
                        if (kTwo) rest[i][j][v] = 0.f;
                    }
            for (int32_t step = 0; step < steps; step += kSets) {
#pragma unroll
                for (int i = 0; i < kSets; ++i) turn(i);
            }
            if constexpr (kTwo) {
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] += rest[i][j];
            }
            finish(tile);
        }
    }
    // Output acc[i][j][v] of a lane is that of row first_row + row_step(i, v) of the left factor in LDS and of row first_column
    // + 32 j of the right one.
    static __device__ __forceinline__ int first_row(int lane)
    {
        return __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)) / (BN / WN) * WM + 4 * (lane >> 5);
    }
    static __device__ __forceinline__ int first_column(int lane)
    {
        return __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)) % (BN / WN) * WN + (lane & 31);
    }
    static constexpr int row_step(int i, int v) { return i * 32 + 8 * (v >> 2) + (v & 3); }
    // the same for outputs numbered 0 .. kOutputs - 1 in a loop that is not unrolled
    static constexpr int kOutputs = MI * 16 * NI;
    static __device__ __forceinline__ int row_of(int e) { return row_step(e / (16 * NI), e / NI % 16); }
    static __device__ __forceinline__ int column_step(int e) { return e % NI; }
};

// ---- dw and db ----------------------------------------------------------------------------------------------------
// k of these products are the rows of the batch, so both factors are turned on their way to LDS: a thread reads columns of a few
// rows and writes them as rows.  X: four columns (a word) of four rows; dz: of eight rows a column of fp32 or two of bf16.
// What a wave needs of exponents and masks is one read, lane by lane, and handed round.  Columns are placed such that
// adjacent threads write adjacent rows of LDS.  Splits of the rows fill the chip where dw has few tiles.
// 85,000 rows, 256 x 256, fp32: 48 us (87 MB of gradients, 22 of checkpoints, 33 of the splits' sums: 3.0 TB/s); 16,384 rows,
// 4096 x 4096, bf16: 590 to 720 us (0.76 to 0.93 PFLOP/s, by the clock that dx leaves it), bound by the issue of matrix and vector instructions together: a value
// of X takes three of the latter on its way to LDS.
struct WeightsArgs {
    BackwardArgs a;
    int32_t m_tiles, n_tiles, splits;
    int32_t db_shares;                        // of the m_tiles blocks that read the same rows, how many add up db: all or one
    float* dw;                                // [splits x (f1 + f2) x hdim]: the caller's if there is one split
    float* db;                                // [splits x db_shares x hdim]: the caller's if that is one; or null
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
    static constexpr int kSets = 2, kFetches = 1 + (kMask ? 1 : 0) + 4 + kReads, kPuts = 1 + 4 + 2 + 1 + (kFloat ? 3 : 2);
    static_assert(kQuads * 8 == kThreads && kLanes * 4 == kThreads, "each thread has its share of a stage");

    Chunk* const lds;
    const uint32_t row_bytes;                 // of d_out
    const int32_t db_shares;                  // this block adds up db over every so many steps
    int64_t rest;                             // rows there are from the next step's first on
    int32_t until_sum;
    bool begun;
    int quad, rows4;                          // this thread's columns of X, and its four rows of a stage
    int column, chunk;                        // its first column of dz, and its eight rows
    // of the step that is read:
    const char* z[8];                         // the wave's eight rows of dz
    uint32_t z_at, second;                    // bytes from there to this lane's column, and to the next one
    const int8_t* q[4];                       // this thread's columns of X
    const uint8_t* e;                         // the exponent this lane reads
    const uint32_t* m;                        // the word of the mask this lane reads
    uint32_t q_stride, e_stride, m_stride;
    int e_row, m_row;
    int32_t left[kSets];                      // rows there are from the step's first on
    bool sums[kSets];
    uint32_t x[kSets][4], ex[kSets], d[kSets][kReads], words[kSets];
    float scale[4], sum[2];

    __device__ __forceinline__ WeightsSource(const BackwardArgs& a, Chunk* stages, int64_t first, int64_t end, int32_t c0, int32_t n0, int32_t shares, int32_t share)
        : lds(stages), row_bytes((uint32_t) a.d_out.stride * (uint32_t) sizeof(T)), db_shares(shares), rest(end - first),
          until_sum(share < shares ? share : INT32_MAX), begun(false)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63;
        const int row16 = lane >> 4, i8 = lane & 7;
        const int32_t p1 = a.x1.groups * 32, all = p1 + a.x2.groups * 32, hdim = a.hdim;
        // columns past the last read the last ones again; they are not stored
        auto part_of = [&](int32_t c, int32_t* in) -> const PackedRows& { *in = c < p1 ? c : c - p1; return c < p1 ? a.x1 : a.x2; };
        quad = (int) threadIdx.x % kQuads;
        rows4 = (kQuads == kWave ? wave : (int) threadIdx.x / kQuads) * 4;
        int32_t in;
        const PackedRows& part = part_of(min(c0 + quad * 4, all - 4), &in);
        q_stride = (uint32_t) part.groups * 32;
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = part.q + (first + rows4 + j) * (int64_t) q_stride + in;
        // Eight lanes share a group's exponents; a row of sixteen lanes has two groups, of which its first eight lanes read the
        // exponents: of the first group's four rows, of the second's.
        const int group = quad_group(row16) + (i8 >> 2);
        e_row = (kQuadsWave == kWave ? wave * 4 : wave * 8 + (row16 >> 1) * 4) + (i8 & 3);
        const PackedRows& part_e = part_of(min(c0 + group * 32, all - 32), &in);
        e_stride = (uint32_t) part_e.groups;
        e = part_e.exponents + (first + e_row) * (int64_t) e_stride + in / 32;
        const int lanes0 = wave * kWave % kLanes;              // the wave's first column of dz (of bf16: first pair)
        chunk = wave * kWave / kLanes;
        column = kFloat ? lanes0 + lane : 2 * (lanes0 + lane);
        const int32_t n = min(n0 + column, !kFloat && kPairs ? hdim - 2 : hdim - 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = static_cast<const char*>(a.d_out.data) + (first + chunk * 8 + j) * (int64_t) row_bytes;
        z_at = (uint32_t) n * (uint32_t) sizeof(T);
        second = n + 1 < hdim ? (uint32_t) sizeof(T) : 0u;
        // a row of sixteen lanes has columns of one word; its first eight lanes read that of eight rows
        m_stride = (uint32_t) (hdim + 31) / 32;
        m_row = chunk * 8 + i8;
        if constexpr (kMask) {
            const int32_t word = kFloat ? (n0 + lanes0) / 32 + (row16 >> 1) : (n0 + 2 * lanes0) / 32 + row16;
            m = a.positive + (first + m_row) * (int64_t) m_stride + min(word, (int32_t) m_stride - 1);
        }
        sum[0] = sum[1] = 0.f;
    }
    static __device__ __forceinline__ int quad_group(int row16) { return kQuadsWave == kWave ? 2 * row16 : 2 * (row16 & 1); }
    __device__ __forceinline__ void seek(int set)
    {
        // steps past the last read the last one again, which counts as nothing
        if (begun && rest > 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] += (uint64_t) q_stride * kStageK;
            e += e_stride * kStageK;
            if constexpr (kMask) m += m_stride * kStageK;
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += (uint64_t) row_bytes * kStageK;
        }
        begun = true;
        // rows past the last of the last step are read as that one
        if (rest > 0 && rest < kStageK) {
            const int last = (int) rest - 1;
            auto back = [&](int row) { return max(row - last, 0); };
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] -= (uint64_t) (uint32_t) back(rows4 + j) * q_stride;
            e -= (uint64_t) (uint32_t) back(e_row) * e_stride;
            if constexpr (kMask) m -= (uint64_t) (uint32_t) back(m_row) * m_stride;
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] -= (uint64_t) (uint32_t) back(chunk * 8 + j) * row_bytes;
        }
        left[set] = (int32_t) (rest < kStageK ? rest : kStageK);
        rest -= kStageK;
        sums[set] = until_sum == 0;
        until_sum = until_sum == 0 ? db_shares - 1 : until_sum - 1;
    }
    __device__ __forceinline__ void fetch(int set, int i)
    {
        if (i == 0) {
            ex[set] = *e;
        } else if (kMask && i == 1) {
            words[set] = *m;
        } else if (i < (kMask ? 6 : 5)) {
            const int j = i - (kMask ? 2 : 1);
            x[set][j] = *reinterpret_cast<const uint32_t*>(q[j]);
        } else {
            const int j = i - (kMask ? 6 : 5);
            if constexpr (kFloat || kPairs) d[set][j] = *reinterpret_cast<const uint32_t*>(z[j] + z_at);
            else                            d[set][j] = *reinterpret_cast<const uint16_t*>(z[j % 8] + (j < 8 ? z_at : z_at + second));
        }
    }
    __device__ __forceinline__ void put(int set, int stage, int i)
    {
        if (i == 0) {
            const uint32_t own = e_row < left[set] ? ex[set] << 23 : 0u;
            scale[0] = __uint_as_float(row_broadcast<4, 0xc>(row_broadcast<0>(0u, own), own));
            scale[1] = __uint_as_float(row_broadcast<5, 0xc>(row_broadcast<1>(0u, own), own));
            scale[2] = __uint_as_float(row_broadcast<6, 0xc>(row_broadcast<2>(0u, own), own));
            scale[3] = __uint_as_float(row_broadcast<7, 0xc>(row_broadcast<3>(0u, own), own));
        } else if (i < 5) {
            const int j = i - 1;                              // column j of the four
            uint32_t v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __float_as_uint((float) (int8_t) (x[set][k] >> (8 * j)) * scale[k]);
            uint2* to = reinterpret_cast<uint2*>(lds + stage * Tiles::kStage + Tiles::place_a(0, quad_row(quad * 4 + j), rows4 >> 3));
            to[(rows4 >> 2) & 1] = make_uint2(upper_halves(v[0], v[1]), upper_halves(v[2], v[3]));
        } else if (i == 5) {
            const uint32_t own = kMask && m_row < left[set] ? words[set] : 0u;
            keep_positive<0>(set, own); keep_positive<1>(set, own); keep_positive<2>(set, own); keep_positive<3>(set, own);
        } else if (i == 6) {
            const uint32_t own = kMask && m_row < left[set] ? words[set] : 0u;
            keep_positive<4>(set, own); keep_positive<5>(set, own); keep_positive<6>(set, own); keep_positive<7>(set, own);
        } else if (i == 7) {
            if (sums[set]) add_up(set);
        } else if constexpr (kFloat) {
            uint32_t (&v)[8] = d[set];
            if (i == 8) scale_up(v);
            lds[stage * Tiles::kStage + Tiles::place_b(i - 8, column, chunk)] = take_terms(v);
        } else {
            const int k = i - 8;
            uint32_t t[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) t[p] = k == 0 ? lower_halves(d[set][2 * p], d[set][2 * p + 1]) : upper_halves(d[set][2 * p], d[set][2 * p + 1]);
            lds[stage * Tiles::kStage + Tiles::place_b(0, pair_row(column + k), chunk)] = Chunk{t[0], t[1], t[2], t[3]};
        }
    }
    // What the mask leaves of row kRow of the eight.  (A row past the last has no exponents, so its products are zero.)
    template <int kRow>
    __device__ __forceinline__ void keep_positive(int set, uint32_t own)
    {
        const int lane = (int) threadIdx.x & 63;
        uint32_t v = d[set][kRow];
        if constexpr (!kFloat && !kPairs) v |= d[set][kRow + kReads - 8] << 16;
        if constexpr (kMask) {
            const uint32_t w = row_broadcast<kRow>(0u, own);
            if constexpr (kFloat) v &= spread_bit(w, lane & 31);
            else                  v &= (spread_bit(w, 2 * (lane & 15)) & 0xFFFFu) | (spread_bit(w, 2 * (lane & 15) + 1) & 0xFFFF0000u);
        }
        d[set][kRow] = v;
    }
    __device__ __forceinline__ void add_up(int set)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t v = chunk * 8 + i < left[set] ? d[set][i] : 0u;
            if constexpr (kFloat) {
                sum[0] += __uint_as_float(v);
            } else {
                sum[0] += __uint_as_float(v << 16);
                sum[1] += __uint_as_float(v & 0xFFFF0000u);
            }
        }
    }
};

template <typename T, int kThreads, bool kMask, bool kPairs>
__device__ __forceinline__ void weights_block(const WeightsArgs& g, int32_t block, Chunk* s_stage)
{
    typedef WeightsSource<T, kThreads, kMask, kPairs> Source;
    typedef typename Source::Tiles Tiles;
    const BackwardArgs& a = g.a;
    const int64_t rows = a.count.get();
    const int32_t all = g.m_tiles * g.n_tiles, t = xcd_run(block, all * g.splits), split = t / all;
    int32_t tm, tn;
    tile_of(t - split * all, g.m_tiles, g.n_tiles, &tm, &tn);
    const int32_t c0 = tm * Tiles::kM, n0 = tn * Tiles::kN;
    constexpr int kRound = kStageK * Source::kSets;
    const int64_t each = ((rows + g.splits - 1) / g.splits + kRound - 1) / kRound * kRound;
    const int64_t first = split * each < rows ? split * each : rows, end = first + each < rows ? first + each : rows;
    Tiles tile(s_stage);
    Source source(a, s_stage, first, end, c0, n0, g.db ? g.db_shares : 0, tm);
    float* dw = g.dw + (int64_t) split * (a.x1.width + a.x2.width) * a.hdim;
    tile.run(source, (int32_t) ((end - first + kRound - 1) / kRound) * Source::kSets, 1, [&](int32_t) {
        const int lane = opaque_lane_id(), m0 = Tiles::first_row(lane), n = Tiles::first_column(lane);
        auto column_of = [&](int j) { return sizeof(T) == 4 ? n + 32 * j : pair_column(n + 32 * j); };
        float any = 0.f;                                      // NaN if a sum is not finite
#pragma unroll
        for (int i = 0; i < Tiles::MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int32_t k = weight_row(a, c0 + quad_column(m0 + Tiles::row_step(i, v)));
                if (k < 0) continue;
                float* row = dw + (int64_t) k * a.hdim + n0;
#pragma unroll
                for (int j = 0; j < Tiles::NI; ++j) {
                    any = fmaf(tile.acc[i][j][v], 0.f, any);
                    if (n0 + column_of(j) < a.hdim) row[column_of(j)] = sizeof(T) == 4 ? tile.acc[i][j][v] * (1.f / kTermScale) : tile.acc[i][j][v];
                }
            }
        if (any == 0.f) return;
#pragma unroll 1
        for (int e = 0; e < Tiles::kOutputs; ++e) {           // those in place that are not
            const int32_t k = weight_row(a, c0 + quad_column(m0 + Tiles::row_of(e))), c = n0 + column_of(Tiles::column_step(e));
            if (k < 0 || c >= a.hdim) continue;
            float* at = dw + (int64_t) k * a.hdim + c;
            if (!is_finite(*at)) *at = weight_again<T, kMask>(a, k, c, first, end);
        }
    });
    if (!g.db || tm >= g.db_shares) return;
    float* s_sum = reinterpret_cast<float*>(s_stage);         // [4][Tiles::kN]: of the four threads that read a column
    __syncthreads();
    s_sum[source.chunk * Tiles::kN + source.column] = source.sum[0];
    if (sizeof(T) == 2) s_sum[source.chunk * Tiles::kN + source.column + 1] = source.sum[1];
    __syncthreads();
    const int n = (int) threadIdx.x;
    if (n < Tiles::kN && n0 + n < a.hdim)
        g.db[((int64_t) split * g.db_shares + tm) * a.hdim + n0 + n] = (s_sum[n] + s_sum[Tiles::kN + n]) + (s_sum[2 * Tiles::kN + n] + s_sum[3 * Tiles::kN + n]);
}

template <typename T, int kThreads, bool kMask, bool kPairs>
__global__ void __launch_bounds__(kThreads, 2) k_backward_weights(WeightsArgs g)
{
    __shared__ Chunk s_stage[3 * WeightsTile<T, kThreads>::Type::kStage];
    weights_block<T, kThreads, kMask, kPairs>(g, (int32_t) blockIdx.x, s_stage);
}

// ---- sums and terms -------------------------------------------------------------------------------------------------
// Sums over splits, four at a time; `threads` of a block share one, since there may be few sums of many splits.
struct JoinArgs {
    const float* parts;                       // [splits x count]
    float* out;
    int64_t count;
    int32_t splits, threads, blocks;          // blocks 0: nothing to join
};

// One launch for what is left to do beside the products: db and dw from their splits, dx from its splits, and W in bf16
// terms for dx: [plane][f1 + f2][hdim rounded up to kStageK], zeros behind hdim.  Each has so many of the grid's blocks.
struct BetweenArgs {
    JoinArgs db, dw;
    const float* dx_parts;                    // [dx_splits x rows x (f1 + f2)]
    MutRows dx;
    RowCount count;
    int32_t dx_type, dx_splits, dx_blocks;
    const float* w;
    uint16_t* terms;
    int64_t k;
    int32_t hdim, pitch, term_blocks;
};

// Values i .. i + 3 of n; marks: they are one read.
__device__ __forceinline__ float4 load_four(const float* p, int64_t i, int64_t n, bool marks)
{
    if (marks && i + 4 <= n) return *reinterpret_cast<const float4*>(p + i);
    return make_float4(i < n ? p[i] : 0.f, i + 1 < n ? p[i + 1] : 0.f, i + 2 < n ? p[i + 2] : 0.f, i + 3 < n ? p[i + 3] : 0.f);
}

__device__ __forceinline__ void join_sums(const JoinArgs& a, int32_t block, float4* s_part)
{
    const int items = kBlock / a.threads, item = (int) threadIdx.x % items, part = (int) threadIdx.x / items;
    const int64_t fours = (a.count + 3) / 4;
    const bool marks = a.count % 4 == 0;
    for (int64_t i0 = (int64_t) block * items; i0 < fours; i0 += (int64_t) a.blocks * items) {
        const int64_t i = 4 * (i0 + item);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < a.count) {
#pragma unroll 8
            for (int32_t s = part; s < a.splits; s += a.threads) {
                const float4 p = load_four(a.parts + s * a.count, i, a.count, marks);
                v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
            }
        }
        for (int w = a.threads / 2; w > 0; w /= 2) {
            __syncthreads();
            if (part >= w && part < 2 * w) s_part[(part - w) * items + item] = v;
            __syncthreads();
            if (part < w) {
                const float4 p = s_part[part * items + item];
                v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
            }
        }
        if (part == 0 && i < a.count) {
            a.out[i] = v.x;
            if (i + 1 < a.count) a.out[i + 1] = v.y;
            if (i + 2 < a.count) a.out[i + 2] = v.z;
            if (i + 3 < a.count) a.out[i + 3] = v.w;
        }
    }
}

__global__ void __launch_bounds__(kBlock) k_backward_between(BetweenArgs a)
{
    __shared__ float4 s_part[kBlock / 2];
    int32_t block = (int32_t) blockIdx.x;
    if (block < a.db.blocks) return join_sums(a.db, block, s_part);
    block -= a.db.blocks;
    if (block < a.dw.blocks) return join_sums(a.dw, block, s_part);
    block -= a.dw.blocks;
    if (block < a.dx_blocks) {
        const uint32_t K = (uint32_t) a.k, all = (uint32_t) max(a.count.get(), 0) * K, each = (uint32_t) a.count.rows * K;
        for (uint32_t i = (uint32_t) block * kBlock + threadIdx.x; i < all; i += (uint32_t) a.dx_blocks * kBlock) {
            float v = 0.f;
#pragma unroll 4
            for (int32_t s = 0; s < a.dx_splits; ++s) v += a.dx_parts[(uint64_t) s * each + i];
            const uint32_t r = i / K;
            if (a.dx_type == GNS_FP32) store_at<float>(a.dx, r, (int32_t) (i - r * K), v);
            else                       store_at<Bf16>(a.dx, r, (int32_t) (i - r * K), v);
        }
        return;
    }
    block -= a.dx_blocks;
    const int64_t fours = a.pitch / 4, terms = a.k * fours;
    const bool marks = a.hdim % 4 == 0 && reinterpret_cast<uintptr_t>(a.w) % 16 == 0;
    for (int64_t t = (int64_t) block * kBlock + threadIdx.x; t < terms; t += (int64_t) a.term_blocks * kBlock) {
        const int64_t row = t / fours, c = (t - row * fours) * 4;
        const float4 four = load_four(a.w + row * a.hdim, c, a.hdim, marks);
        float v[4] = {four.x * kTermScale, four.y * kTermScale, four.z * kTermScale, four.w * kTermScale};
        for (int p = 0; p < 3; ++p) {
            const uint32_t lower = take_term(v[0], v[1]), upper = take_term(v[2], v[3]);
            *reinterpret_cast<uint2*>(a.terms + (p * a.k + row) * a.pitch + c) = make_uint2(lower, upper);
        }
    }
}

// ---- dx -----------------------------------------------------------------------------------------------------------
struct InputArgs {
    BackwardArgs a;
    int32_t m_tiles, n_tiles, pitch;
    int32_t splits;                           // of hdim
    const uint16_t* w;                        // planes of k_backward_between
    float* parts;                             // [splits x rows x (f1 + f2)], if there are splits
};

// The columns of a step that count, for a thread that reads eight of them from column n on, but none past the last: where a row
// ends inside, it reads the row's last eight, and of those the last `inside` count.
__device__ __forceinline__ uint32_t columns_kept(int32_t inside)
{
    return inside >= 8 ? 0xFFu : inside > 0 ? 0xFFu << (8 - inside) & 0xFFu : 0u;
}
// and those that are left of them by a mask's bits from column n on
__device__ __forceinline__ uint32_t columns_left(uint32_t kept, uint32_t bits) { return kept & bits << ((__ffs((int) kept) - 1) & 31); }

// of sums of products of W's terms and dz's, which are terms in fp32 alone
template <typename T> constexpr float kInputScale = sizeof(T) == 4 ? 1.f / (kTermScale * kTermScale) : 1.f / kTermScale;

template <typename T, int kThreads> struct InputTile;
template <> struct InputTile<float, 512> { typedef Tile<128, 128, 64, 32, 3, 3> Type; };
template <> struct InputTile<float, 256> { typedef Tile<64, 64, 32, 32, 3, 3> Type; };
template <> struct InputTile<Bf16, 512> { typedef Tile<256, 128, 64, 64, 1, 3> Type; };
template <> struct InputTile<Bf16, 256> { typedef Tile<128, 64, 64, 32, 1, 3> Type; };

// 85,000 rows, 256 x 256, fp32: 83 us (six products of terms; 0.81 PFLOP/s of them); 16,384 rows, 4096 x 4096, bf16: 1415 to 1480 us
// (three products; 1.1 to 1.17 PFLOP/s, the matrix cores busy in 70 % of the cycles at the 1.5 GHz that the power leaves).
// A thread reads eight columns of a row of dz (of two rows of bf16), and as many of W's planes.  kWhole: hdim is a multiple of
// eight.  Chunks past the last are read as the last: W's planes are zero there.  Else a row's last chunk is its last eight
// columns, for dz as for W, and those that the chunk before has are left out of dz.  hdim is eight at least.
// A block goes through tiles, `stride` apart, or has a split of one tile's hdim.
// kPlain: W is read as it is and cut here, by every block that needs it, which where there is no more than a block or two per
// CU costs less than a launch and a trip through memory in front (the planes of 4096 x 4096 take 31 us).
template <typename T, int kThreads, bool kMask, bool kWhole, bool kPlain>
struct InputSource {
    typedef typename InputTile<T, kThreads>::Type Tiles;
    static constexpr bool kFloat = sizeof(T) == 4;
    static constexpr int kPlanes = 3, kStep = kThreads / 4;                                         // rows the threads cover at once
    static constexpr int kRowsA = Tiles::kM / kStep, kRowsB = Tiles::kN / kStep, kWords = kFloat ? 8 : 4;
    static constexpr int kSets = kFloat && kPlain ? 4 : 2, kReadsB = kPlain ? 1 : kPlanes;
    static constexpr bool kKeeps = kMask || !kWhole;          // dz has columns left out
    static constexpr int kFetches = kRowsA * (1 + (kMask ? 1 : 0)) + kRowsB * kReadsB;
    static constexpr int kPutsA = (kKeeps ? 1 : 0) + (kFloat ? 3 : 1), kPuts = kRowsA * kPutsA + kRowsB * kPlanes;

    const InputArgs& g;
    Chunk* const lds;
    const int64_t rows, K;
    const int32_t m_tiles, stride, begin, end;          // begin, end: of the columns, in whole turns of kSets steps
    int32_t t, n0;                            // tile and first column of the next step
    int row, chunk;
    const char* z[kRowsA];                    // this thread's rows of dz
    const uint32_t* m[kRowsA];                // and of the mask
    const char* w;                            // the tile's first row of W or its planes
    uint32_t w_at[kRowsB];                    // from there to this thread's rows and columns
    int32_t n, word;                          // of the step that is read: this thread's first column, its word of the mask
    int64_t w_step;                           // and bytes from a plane's row to its columns
    uint32_t d[kSets][kRowsA][kWords], words[kSets][kRowsA], keep[kSets];
    Chunk planes[kSets][kRowsB][kPlain ? 1 : kPlanes];
    uint32_t plain[kSets][kRowsB][kPlain ? 8 : 1];

    static constexpr int kTurn = kStageK * kSets;
    static __device__ __forceinline__ int32_t turns_before(int32_t hdim, int32_t split, int32_t splits)
    {
        return (int32_t) ((int64_t) ((hdim + kTurn - 1) / kTurn) * split / splits);
    }
    __device__ __forceinline__ InputSource(const InputArgs& args, Chunk* stages, int64_t rows_, int32_t tiles_, int32_t first, int32_t stride_, int32_t split)
        : g(args), lds(stages), rows(rows_), K(args.a.x1.width + args.a.x2.width), m_tiles(tiles_), stride(stride_),
          begin(turns_before(args.a.hdim, split, args.splits) * kTurn), end(turns_before(args.a.hdim, split + 1, args.splits) * kTurn), t(first), n0(begin)
    {
        row = (int) threadIdx.x >> 2;
        chunk = (int) threadIdx.x & 3;
        begin_tile();
    }
    __device__ __forceinline__ void begin_tile()
    {
        const BackwardArgs& a = g.a;
        const int32_t all = m_tiles * g.n_tiles;
        int32_t tm, tn;
        tile_of(t < all ? t : all - 1, m_tiles, g.n_tiles, &tm, &tn);
#pragma unroll
        for (int i = 0; i < kRowsA; ++i) {                    // rows past the last are read as the last; they are not stored
            const int64_t r = min((int64_t) tm * Tiles::kM + row + i * kStep, rows - 1);
            z[i] = static_cast<const char*>(a.d_out.data) + r * a.d_out.stride * (int64_t) sizeof(T);
            if constexpr (kMask) m[i] = a.positive + r * ((a.hdim + 31) / 32);
        }
        const int64_t k0 = (int64_t) tn * Tiles::kN;
        if constexpr (kPlain) w = reinterpret_cast<const char*>(a.w + k0 * a.hdim);
        else                  w = reinterpret_cast<const char*>(g.w + k0 * g.pitch);
#pragma unroll
        for (int i = 0; i < kRowsB; ++i) {
            const uint32_t k = (uint32_t) min((int64_t) row + i * kStep, K - 1 - k0);
            w_at[i] = kPlain ? k * (uint32_t) a.hdim * 4u : k * (uint32_t) g.pitch * 2u + (kWhole ? (uint32_t) chunk * 16u : 0u);
        }
    }
    __device__ __forceinline__ void seek(int set)
    {
        if (n0 >= end) {
            n0 = begin;
            t += stride;
            begin_tile();
        }
        const int32_t hdim = g.a.hdim, at = n0 < g.pitch ? n0 : g.pitch - kStageK;       // steps that only fill a turn read the last again
        n = n0 + chunk * 8;
        if constexpr (kKeeps || kPlain) keep[set] = columns_kept(hdim - n);
        else                            keep[set] = n0 < g.pitch ? 1u : 0u;               // wave-uniform
        n = min(n, hdim - 8);
        word = at >> 5;
        w_step = kWhole ? (int64_t) at * 2 : 0;
        n0 += kStageK;
    }
    __device__ __forceinline__ void fetch(int set, int i)
    {
        if (i < kRowsA) {
            load_words(z[i] + (uint64_t) ((uint32_t) n * (uint32_t) sizeof(T)), d[set][i]);
        } else if (kPlain && i < kRowsA + kRowsB) {
            if constexpr (kPlain) load_words(w + ((uint64_t) w_at[i - kRowsA] + (uint32_t) n * 4u), plain[set][i - kRowsA]);
        } else if (i < kRowsA + kRowsB * kReadsB) {
            const int b = (i - kRowsA) / kPlanes, p = (i - kRowsA) % kPlanes;
            __builtin_memcpy(&planes[set][b][p], __builtin_assume_aligned(w + (w_step + p * K * g.pitch * 2) + (w_at[b] + (kWhole ? 0u : (uint32_t) n * 2u)), kWhole ? 16 : 2), 16);
        } else {
            const int b = i - kRowsA - kRowsB * kReadsB;
            words[set][b] = m[b][word];
        }
    }
    __device__ __forceinline__ void put(int set, int stage, int i)
    {
        Chunk* to = lds + stage * Tiles::kStage;
        if (i >= kRowsA * kPutsA) {
            const int b = (i - kRowsA * kPutsA) / kPlanes, p = (i - kRowsA * kPutsA) % kPlanes;
            if constexpr (kPlain) {
                uint32_t (&v)[8] = plain[set][b];
                if (p == 0 && !kKeeps) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] &= keep[set] ? ~0u : 0u;
                }
                if (p == 0) scale_up(v);
                to[Tiles::place_b(p, row + b * kStep, chunk)] = take_terms(v);
            } else {
                Chunk v = planes[set][b][p];
                if (!kKeeps) v = keep[set] ? v : Chunk{0, 0, 0, 0};
                to[Tiles::place_b(p, row + b * kStep, chunk)] = v;
            }
            return;
        }
        const int b = i / kPutsA, u = i % kPutsA - (kKeeps ? 1 : 0);
        if (u < 0) {                                          // what is left of the columns
            const uint32_t k8 = kMask ? columns_left(keep[set], words[set][b] >> (chunk * 8)) : keep[set];
            if constexpr (kFloat) {
#pragma unroll
                for (int j = 0; j < 8; ++j) d[set][b][j] &= spread_bit(k8, j);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) d[set][b][j] &= (spread_bit(k8, 2 * j) & 0xFFFFu) | (spread_bit(k8, 2 * j + 1) & 0xFFFF0000u);
            }
        } else if constexpr (kFloat) {
            if (u == 0) scale_up(d[set][b]);
            to[Tiles::place_a(u, row + b * kStep, chunk)] = take_terms(d[set][b]);
        } else {
            to[Tiles::place_a(0, row + b * kStep, chunk)] = Chunk{d[set][b][0], d[set][b][1], d[set][b][2], d[set][b][3]};
        }
    }
};

template <typename T, int kThreads, bool kMask, bool kWhole, bool kPlain>
__device__ __forceinline__ void input_block(const InputArgs& g, int32_t block, int32_t blocks, Chunk* s_stage)
{
    typedef InputSource<T, kThreads, kMask, kWhole, kPlain> Source;
    typedef typename Source::Tiles Tiles;
    const BackwardArgs& a = g.a;
    const int64_t rows = a.count.get();
    if (rows <= 0) return;
    // a block's tiles: of those that have rows, every `stride`-th of its XCD's; where hdim is split, a split of one
    const int32_t stride = kPlain ? blocks / g.splits : blocks, at = xcd_run(block, blocks);
    const int32_t split = kPlain ? at / stride : 0, first = kPlain ? at - split * stride : at;
    const int32_t m_tiles = (int32_t) ((rows + Tiles::kM - 1) / Tiles::kM), all = m_tiles * g.n_tiles;
    const int32_t tiles = first < all ? (all - first + stride - 1) / stride : 0;
    if (tiles == 0) return;
    Tiles tile(s_stage);
    Source source(g, s_stage, rows, m_tiles, first, stride, split);
    const int32_t K = a.x1.width + a.x2.width;
    T* out = reinterpret_cast<T*>(a.dx.data);
    tile.run(source, (source.end - source.begin) / kStageK, tiles, [&](int32_t i) {
        int32_t tm, tn;
        tile_of(first + i * stride, m_tiles, g.n_tiles, &tm, &tn);
        const int64_t r0 = (int64_t) tm * Tiles::kM;
        const int32_t k0 = tn * Tiles::kN;
        const int lane = opaque_lane_id(), m0 = Tiles::first_row(lane), n = Tiles::first_column(lane);
        const bool whole = r0 + Tiles::kM <= rows && k0 + Tiles::kN <= K;
        float any = 0.f;                                      // NaN if a sum is not finite
#pragma unroll
        for (int i = 0; i < Tiles::MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v)
#pragma unroll
                for (int j = 0; j < Tiles::NI; ++j) any = fmaf(tile.acc[i][j][v], 0.f, any);
        // outputs in place that are not finite, of columns `begin` to `end`
        auto again = [&](auto* at, int64_t stride, int32_t begin, int32_t end, auto&& value, auto&& make) {
#pragma unroll 1
            for (int e = 0; e < Tiles::kOutputs; ++e) {
                const int32_t k = k0 + n + 32 * Tiles::column_step(e);
                const int64_t r = r0 + m0 + Tiles::row_of(e);
                if (r >= rows || k >= K) continue;
                auto* to = at + (int64_t) Tiles::row_of(e) * stride + 32 * Tiles::column_step(e);
                if (!is_finite(value(*to))) *to = make(input_again<T, kMask>(a, r, k, begin, end));
            }
        };
        if (kPlain && g.parts) {
            float* part = g.parts + ((int64_t) split * a.count.rows + r0 + m0) * K + k0 + n;
#pragma unroll
            for (int i = 0; i < Tiles::MI; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v)
#pragma unroll
                    for (int j = 0; j < Tiles::NI; ++j)
                        if (whole || (r0 + m0 + Tiles::row_step(i, v) < rows && k0 + n + 32 * j < K)) part[(int64_t) Tiles::row_step(i, v) * K + 32 * j] = tile.acc[i][j][v] * kInputScale<T>;
            if (any != 0.f) again(part, K, source.begin, min(source.end, a.hdim), [](float v) { return v; }, [](float v) { return v; });
            return;
        }
        T* first = out + (r0 + m0) * a.dx.stride + k0 + n;
#pragma unroll
        for (int i = 0; i < Tiles::MI; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                T* row = first + Tiles::row_step(i, v) * a.dx.stride;
#pragma unroll
                for (int j = 0; j < Tiles::NI; ++j)
                    if (whole || (r0 + m0 + Tiles::row_step(i, v) < rows && k0 + n + 32 * j < K)) row[32 * j] = from_float<T>(tile.acc[i][j][v] * kInputScale<T>);
            }
        if (any != 0.f) again(first, a.dx.stride, 0, a.hdim, [](T v) { return to_float(v); }, [](float v) { return from_float<T>(v); });
    });
}

template <typename T, int kThreads, bool kMask, bool kWhole, bool kPlain>
__global__ void __launch_bounds__(kThreads, 2) k_backward_input(InputArgs g)
{
    __shared__ Chunk s_stage[3 * InputTile<T, kThreads>::Type::kStage];
    input_block<T, kThreads, kMask, kWhole, kPlain>(g, (int32_t) blockIdx.x, (int32_t) gridDim.x, s_stage);
}

// Both products of a small call in one launch, since neither waits for the other: the grid's first blocks are dw's.  fp32, 64 rows
// of 256 x 256: 10 us, one after the other 17; 1772 rows of 400 x 18 bf16 16 and 24; 300 of 1000 x 1000 23 and 44.
template <typename T, bool kMask, bool kWhole, bool kPairs>
__global__ void __launch_bounds__(256, 2) k_backward_both(WeightsArgs g, InputArgs h, int32_t weights_blocks)
{
    constexpr int kWeights = WeightsTile<T, 256>::Type::kStage, kInput = InputTile<T, 256>::Type::kStage, kStage = kWeights > kInput ? kWeights : kInput;
    __shared__ Chunk s_stage[3 * kStage];
    const int32_t block = (int32_t) blockIdx.x;
    if (block < weights_blocks) weights_block<T, 256, kMask, kPairs>(g, block, s_stage);
    else                        input_block<T, 256, kMask, kWhole, true>(h, block - weights_blocks, (int32_t) gridDim.x - weights_blocks, s_stage);
}

// k_backward_few: dx of up to sixteen rows, where W's bytes are all there is to do.  A block has 16 columns of dx (rows of W) and
// all rows; its eight waves an eighth of hdim each, 16 x 16 x 32 products; their sums meet in LDS.  W is cut into terms on the
// way, as dz is.  One row, 4096 x 4096, fp32, dw too: 40 us, 56 in tiles with hdim split; 17 rows would take 66 and take 52 in tiles.
constexpr int kFewRows = 16, kFewBlock = 512, kFewWaves = kFewBlock / kWave, kFewColumns = 16;
typedef float floatx4 __attribute__((ext_vector_type(4)));

template <typename T, bool kMask>
__global__ void __launch_bounds__(kFewBlock) k_backward_few(BackwardArgs a)
{
    constexpr bool kFloat = sizeof(T) == 4;
    constexpr int kTermsA = kFloat ? 3 : 1, kTermsB = 3, kSets = 4;
    typedef Pairs<kTermsA, kTermsB> P;
    __shared__ float s_sum[kFewWaves][4][kWave];
    const int32_t rows = a.count.get(), K = a.x1.width + a.x2.width, hdim = a.hdim, steps = (hdim + 31) / 32;
    if (rows <= 0) return;
    const int wave = __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)), lane = (int) threadIdx.x & 63;
    const int l16 = lane & 15, kg = lane >> 4;
    const int32_t k0 = (int32_t) blockIdx.x * kFewColumns;
    const int32_t s0 = (int32_t) ((int64_t) steps * wave / kFewWaves), s1 = (int32_t) ((int64_t) steps * (wave + 1) / kFewWaves);
    const float* w = a.w + (int64_t) min(k0 + l16, K - 1) * hdim;
    const int64_t own = min(l16, rows - 1);                   // rows past the last are read as the last; they are not stored
    const T* z = reinterpret_cast<const T*>(a.d_out.data) + own * a.d_out.stride;
    const uint32_t* m = nullptr;
    if constexpr (kMask) m = a.positive + own * steps;
    uint32_t wv[kSets][8], zv[kSets][kFloat ? 8 : 4], words[kSets];
    auto fetch = [&](int set, int32_t step) {                 // steps past the wave's last read that one again
        step = min(step, s1 - 1);
        const int32_t n = min(step * 32 + kg * 8, hdim - 8);
        load_words(w + n, wv[set]);
        load_words(z + n, zv[set]);
        if constexpr (kMask) words[set] = m[step];
    };
    floatx4 acc = {0.f, 0.f, 0.f, 0.f}, rest = acc;           // as in Tile
    auto multiply = [&](int set, int32_t step) {
        const uint32_t keep = columns_kept(hdim - step * 32 - kg * 8), k8 = kMask ? columns_left(keep, words[set] >> (kg * 8)) : keep;
        Chunk wt[kTermsB], zt[kTermsA];
#pragma unroll
        for (int j = 0; j < 8; ++j) wv[set][j] &= spread_bit(keep, j);
        scale_up(wv[set]);
#pragma unroll
        for (int k = 0; k < kTermsB; ++k) wt[k] = take_terms(wv[set]);
        if constexpr (kFloat) {
#pragma unroll
            for (int j = 0; j < 8; ++j) zv[set][j] &= spread_bit(k8, j);
            scale_up(zv[set]);
#pragma unroll
            for (int k = 0; k < kTermsA; ++k) zt[k] = take_terms(zv[set]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) zt[0][j] = zv[set][j] & ((spread_bit(k8, 2 * j) & 0xFFFFu) | (spread_bit(k8, 2 * j + 1) & 0xFFFF0000u));
        }
#pragma unroll
        for (int p = 0; p < P::kCount; ++p) {
            floatx4& to = kFloat && p + 1 < P::kCount ? rest : acc;
            to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, zt[P::kA[p]]), __builtin_bit_cast(bf16x8, wt[P::kB[p]]), to, 0, 0, 0);
        }
    };
    if (s0 < s1) {
#pragma unroll
        for (int d = 0; d < kSets; ++d) fetch(d, s0 + d);
        for (int32_t s = s0; s < s1; s += kSets) {
#pragma unroll
            for (int d = 0; d < kSets; ++d) {
                if (s + d < s1) multiply(d, s + d);           // wave-uniform
                fetch(d, s + d + kSets);
            }
        }
    }
    if (kFloat) acc += rest;
#pragma unroll
    for (int v = 0; v < 4; ++v) s_sum[wave][v][lane] = acc[v];
    __syncthreads();
    // element v of lane l is row 4 * (l / 16) + v, column l % 16
    const int i = (int) threadIdx.x;
    if (i >= 4 * kWave) return;
    const int v = i / kWave, l = i % kWave;
    const int32_t r = 4 * (l >> 4) + v, k = k0 + (l & 15);
    if (r >= rows || k >= K) return;
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < kFewWaves; ++u) sum += s_sum[u][v][l];
    sum *= kInputScale<T>;
    if (!is_finite(sum)) sum = input_again<T, kMask>(a, r, k, 0, hdim);
    store_at<T>(a.dx, r, k, sum);
}

// k_backward_narrow: dx of fewer than eight columns of dz, by as many multiplications each, in fp32.  A lane has four columns of
// dx, whose rows of W stay in registers, and rows one after the other; 2^lanes_log2 lanes have a row.  Bound by the bytes of dx: 85,000 rows of 100 bf16 columns from two, dw
// too, 34 us; as tiles of products 50.
constexpr int kNarrow = 8, kNarrowRows = 16;  // rows of a lane
template <typename T, bool kMask>
__global__ void __launch_bounds__(kBlock) k_backward_narrow(BackwardArgs a, int32_t lanes_log2)
{
    const int32_t rows = a.count.get(), K = a.x1.width + a.x2.width, hdim = a.hdim;
    const int32_t per_wave = kWave >> lanes_log2, each = per_wave * kNarrowRows, lane = lane_id(), chunks = (K + (4 << lanes_log2) - 1) / (4 << lanes_log2);
    const int64_t work = ((int64_t) rows + each - 1) / each * chunks;
    for (int64_t i = (int64_t) blockIdx.x * (kBlock / kWave) + __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)); i < work;
         i += (int64_t) gridDim.x * (kBlock / kWave)) {
        const int64_t group = i / chunks, r0 = group * each + (lane >> lanes_log2);
        const int32_t k = ((int32_t) (i - group * chunks) << lanes_log2) * 4 + (lane & ((1 << lanes_log2) - 1)) * 4;
        float w[4][kNarrow - 1];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < kNarrow - 1; ++n) w[j][n] = n < hdim ? a.w[(int64_t) min(k + j, K - 1) * hdim + n] : 0.f;
#pragma unroll 4
        for (int t = 0; t < kNarrowRows; ++t) {
            const int64_t row = r0 + t * per_wave, r = row < rows ? row : rows - 1;
            const uint32_t keep = kMask ? a.positive[r] : ~0u;
            float z[kNarrow - 1];
#pragma unroll
            for (int n = 0; n < kNarrow - 1; ++n) {
                const float v = load_at<T>(a.d_out, r, n < hdim ? n : 0);
                z[n] = __uint_as_float(__float_as_uint(v) & spread_bit(keep, n));
            }
            struct alignas(4 * sizeof(T)) Four { T v[4]; } y;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < kNarrow - 1; ++n) sum = n < hdim ? fmaf(z[n], w[j][n], sum) : sum;
                y.v[j] = from_float<T>(sum);
            }
            if (row >= rows || k >= K) continue;
            T* out = reinterpret_cast<T*>(a.dx.data) + r * a.dx.stride + k;
            if (k + 4 <= K) {
                typedef uint32_t Word __attribute__((ext_vector_type(sizeof(T))));
                const Word v = __builtin_bit_cast(Word, y);
                __builtin_memcpy(out, &v, sizeof(v));         // whatever the row's alignment
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k + j < K) out[j] = y.v[j];
            }
        }
    }
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
    int32_t m_tiles, n_tiles, splits, db_shares;
};

static WeightsPlan plan_weights_of(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int64_t rows, bool fp32, bool wide)
{
    const int32_t columns = ((f1 + 31) / 32 + (f2 + 31) / 32) * 32, n512 = fp32 ? 128 : 256, bm = wide ? 256 : 128, bn = wide ? n512 : n512 / 2;
    const int64_t most = (rows + 127) / 128;                  // splits of four steps at least
    WeightsPlan p;
    p.wide = wide;
    p.m_tiles = (columns + bm - 1) / bm;
    p.n_tiles = (hdim + bn - 1) / bn;
    int64_t s = (int64_t) c->num_cus * (wide ? 1 : 2) / ((int64_t) p.m_tiles * p.n_tiles);
    if (s > most) s = most;
    p.splits = s < 1 ? 1 : (int32_t) s;
    // a few steps more of one block in m_tiles cost less than the launch that joins the shares
    p.db_shares = p.splits == 1 && rows <= 512 ? 1 : p.m_tiles;
    return p;
}

// Wide blocks where layers fill them and they fill half the chip at least (dx too, 16,384 rows of 2048 x 2048 bf16: 540 us, 604 with
// narrow ones; 85,000 of 256 x 256 fp32: 139 and 153; 12,600 of 512 x 256: no difference)
static bool may_be_wide(int32_t f1, int32_t f2, int32_t hdim, bool fp32) { return (f1 + 31) / 32 + (f2 + 31) / 32 > 4 && hdim > (fp32 ? 64 : 128); }

static WeightsPlan plan_weights(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int64_t rows, bool fp32, bool wide)
{
    const WeightsPlan p = plan_weights_of(c, f1, f2, hdim, rows, fp32, true);
    if (wide && may_be_wide(f1, f2, hdim, fp32) && (int64_t) p.m_tiles * p.n_tiles * p.splits >= c->num_cus / 2) return p;
    return plan_weights_of(c, f1, f2, hdim, rows, fp32, false);
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

// Tiles of dx in blocks of so many threads
template <typename T, int kThreads>
static int64_t input_tiles(const BackwardArgs& a, int32_t* m_tiles, int32_t* n_tiles)
{
    typedef typename InputTile<T, kThreads>::Type Tiles;
    *m_tiles = (int32_t) (((int64_t) a.count.rows + Tiles::kM - 1) / Tiles::kM);
    *n_tiles = (a.x1.width + a.x2.width + Tiles::kN - 1) / Tiles::kN;
    return (int64_t) *m_tiles * *n_tiles;
}

// Splits of hdim for dx where its tiles are few: those that fill the chip, of four turns at least, and one more launch joins them
// (or the one that joins dw's splits anyway).  fp32, 1104 rows of 128 x 2048: 15 us, 37 unsplit.
template <typename T>
static int32_t input_splits(const gns_ctx* c, int64_t tiles, int32_t hdim)
{
    constexpr int32_t kLeast = 4 * kStageK * (sizeof(T) == 4 ? 4 : 2);
    const int64_t s = min((int64_t) c->num_cus / max(tiles, (int64_t) 1), (int64_t) hdim / kLeast);
    return s < 2 ? 1 : (int32_t) s;
}

template <typename T, int kThreads, bool kPlain>
static hipError_t launch_input(const gns_ctx* c, InputArgs g, hipStream_t s)
{
    const int64_t tiles = input_tiles<T, kThreads>(g.a, &g.m_tiles, &g.n_tiles), most = (int64_t) c->num_cus * (kThreads == 512 ? 1 : 2);
    if (tiles >= (int64_t) 1 << 30) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned) (kPlain ? tiles * g.splits : tiles < most ? tiles : most)), block(kThreads);
    const bool whole = g.a.hdim % 8 == 0;
    if (g.a.positive && whole)  hipLaunchKernelGGL((k_backward_input<T, kThreads, true, true, kPlain>), grid, block, 0, s, g);
    else if (g.a.positive)      hipLaunchKernelGGL((k_backward_input<T, kThreads, true, false, kPlain>), grid, block, 0, s, g);
    else if (whole)             hipLaunchKernelGGL((k_backward_input<T, kThreads, false, true, kPlain>), grid, block, 0, s, g);
    else                        hipLaunchKernelGGL((k_backward_input<T, kThreads, false, false, kPlain>), grid, block, 0, s, g);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_both(const WeightsArgs& g, InputArgs h, hipStream_t s)
{
    const int64_t tiles = input_tiles<T, 256>(h.a, &h.m_tiles, &h.n_tiles), blocks = (int64_t) g.m_tiles * g.n_tiles * g.splits;
    if (too_many(blocks + tiles * h.splits, 256)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned) (blocks + tiles * h.splits)), block(256);
    const int32_t first = (int32_t) blocks;
    const bool whole = g.a.hdim % 8 == 0;
    if constexpr (sizeof(T) == 2) {
        if (!reads_pairs(g.a.d_out)) {
            if (g.a.positive) hipLaunchKernelGGL((k_backward_both<T, true, false, false>), grid, block, 0, s, g, h, first);
            else              hipLaunchKernelGGL((k_backward_both<T, false, false, false>), grid, block, 0, s, g, h, first);
            return hipGetLastError();
        }
    }
    if (g.a.positive && whole)  hipLaunchKernelGGL((k_backward_both<T, true, true, true>), grid, block, 0, s, g, h, first);
    else if (g.a.positive)      hipLaunchKernelGGL((k_backward_both<T, true, false, true>), grid, block, 0, s, g, h, first);
    else if (whole)             hipLaunchKernelGGL((k_backward_both<T, false, true, true>), grid, block, 0, s, g, h, first);
    else                        hipLaunchKernelGGL((k_backward_both<T, false, false, true>), grid, block, 0, s, g, h, first);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_few(const BackwardArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned) ((a.x1.width + a.x2.width + kFewColumns - 1) / kFewColumns)), block(kFewBlock);
    if (a.positive) hipLaunchKernelGGL((k_backward_few<T, true>), grid, block, 0, s, a);
    else            hipLaunchKernelGGL((k_backward_few<T, false>), grid, block, 0, s, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_narrow(const gns_ctx* c, const BackwardArgs& a, hipStream_t s)
{
    const int32_t K = a.x1.width + a.x2.width;
    int32_t lanes_log2 = 0;
    while (lanes_log2 < 6 && (4 << lanes_log2) < K) ++lanes_log2;
    const int64_t each = (int64_t) (kWave >> lanes_log2) * kNarrowRows, chunks = (K + (4 << lanes_log2) - 1) / (4 << lanes_log2);
    const dim3 grid(grid_of(c, ((int64_t) a.count.rows + each - 1) / each * chunks * kWave)), block(kBlock);
    if (a.positive) hipLaunchKernelGGL((k_backward_narrow<T, true>), grid, block, 0, s, a, lanes_log2);
    else            hipLaunchKernelGGL((k_backward_narrow<T, false>), grid, block, 0, s, a, lanes_log2);
    return hipGetLastError();
}

// How a call's dx is made.
enum class Way { kNarrow, kFew, kPlain, kCut, kWide };
struct InputPlan {
    Way way;
    int32_t splits;
};
// Blocks of 512 threads where they fill half the chip and layers are not too narrow for them (fp32, dw too, 2400 rows of 1000 x 1000:
// 80 us, 99 with 256 threads; 600 rows of 4096 x 4096: 245 and 338; with less than half 1400 rows of 1000 x 1000: 71 and 66, bf16
// 3000: 79 and 73).  Else of 256, and W is read as it is by no more of them than CUs, or than run at once where dw goes with them
// (fp32, 6000 rows of 256 x 256: 25 us, 36 with W cut in a launch between).
template <typename T>
static InputPlan plan_input(const gns_ctx* c, const BackwardArgs& a, bool both)
{
    typedef typename InputTile<T, 512>::Type Wide;
    int32_t m_tiles, n_tiles;
    if (a.hdim < kNarrow) return {Way::kNarrow, 1};
    if (a.count.rows <= kFewRows && !both) return {Way::kFew, 1};
    if (input_tiles<T, 512>(a, &m_tiles, &n_tiles) * 2 >= c->num_cus && a.x1.width + a.x2.width > Wide::kN / 2) return {Way::kWide, 1};
    const int64_t tiles = input_tiles<T, 256>(a, &m_tiles, &n_tiles);
    return tiles <= (int64_t) c->num_cus * (both ? 2 : 1) ? InputPlan{Way::kPlain, input_splits<T>(c, tiles, a.hdim)} : InputPlan{Way::kCut, 1};
}

// Splits where dw and dx go together: steps a block, four for dw and two turns for dx at least, such that all blocks run at once.
// fp32, 1104 rows of 128 x 2048: 24 us, with dw and dx each split for a chip of its own 28; 400 of 200 x 700: 17 and 22; bf16, 189 of
// 2141 x 1102: 21 and 30.
template <typename T>
static int32_t both_least() { return 2 * (sizeof(T) == 4 ? 4 : 2); }
template <typename T>
static void plan_both(const gns_ctx* c, const BackwardArgs& a, WeightsPlan* weights, InputPlan* input)
{
    int32_t m_tiles, n_tiles;
    const int64_t dw_tiles = (int64_t) weights->m_tiles * weights->n_tiles, dx_tiles = input_tiles<T, 256>(a, &m_tiles, &n_tiles);
    const int32_t dw_steps = (a.count.rows + kStageK - 1) / kStageK, dx_steps = (a.hdim + kStageK - 1) / kStageK;
    for (int32_t each = 4;; each += each / 4) {
        const int32_t dx_each = each > both_least<T>() ? each : both_least<T>();
        weights->splits = (dw_steps + each - 1) / each;
        input->splits = dx_steps >= 2 * dx_each ? dx_steps / dx_each : 1;
        if (weights->splits * dw_tiles + input->splits * dx_tiles <= (int64_t) c->num_cus * 2 || (weights->splits == 1 && input->splits == 1)) break;
    }
    weights->db_shares = weights->splits == 1 && a.count.rows <= 512 ? 1 : weights->m_tiles;
}

// The most splits of hdim that a call may take.
template <typename T>
static int32_t most_input_splits(const gns_ctx* c, const BackwardArgs& a)
{
    int32_t m_tiles, n_tiles;
    const int64_t tiles = input_tiles<T, 256>(a, &m_tiles, &n_tiles), s = min((int64_t) c->num_cus * 2 / max(tiles, (int64_t) 1), (int64_t) (a.hdim + kStageK - 1) / kStageK / both_least<T>());
    return s < 2 ? 1 : (int32_t) s;
}

// Bytes of the sums of dw's and db's parts
static size_t parts_bytes(const WeightsPlan& p, size_t k, size_t hdim)
{
    return (p.splits > 1 ? align256((size_t) p.splits * k * hdim * 4) : 0) + align256((size_t) p.splits * (size_t) p.db_shares * hdim * 4);
}
static size_t terms_bytes(size_t k, size_t hdim) { return align256(3 * k * ((hdim + kStageK - 1) / kStageK * kStageK) * 2); }

size_t backward_need(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int32_t rows)
{
    const size_t k = (size_t) f1 + (size_t) f2;
    size_t parts = 0;
    for (int i = 0; i < 3; ++i)                                // of either type, and of bf16 columns read singly
        parts = max(parts, parts_bytes(plan_weights(c, f1, f2, hdim, rows, i == 0, i < 2), k, (size_t) hdim));
    BackwardArgs a = {};
    a.x1.width = f1; a.x2.width = f2; a.hdim = hdim; a.count.rows = rows;
    const int32_t splits = max(most_input_splits<float>(c, a), most_input_splits<Bf16>(c, a));
    return parts + max(terms_bytes(k, (size_t) hdim), splits > 1 ? align256((size_t) splits * (size_t) rows * k * 4) : 0);
}

// The most bytes that dx's splits take in calls of so many rows or fewer: s splits of r rows where s times the tiles of r rows is no
// more than two for each CU.
template <typename T>
static size_t most_input_bytes(const gns_ctx* c, size_t k, int32_t hdim, int32_t rows)
{
    typedef typename InputTile<T, 256>::Type Tiles;
    const int64_t bands = (int64_t) c->num_cus * 2 / (((int64_t) k + Tiles::kN - 1) / Tiles::kN);      // of kM rows, times splits
    const int64_t splits = min(bands, (int64_t) (hdim + kStageK - 1) / kStageK / both_least<T>());
    return splits < 2 ? 0 : align256((size_t) min(splits * rows, bands * Tiles::kM) * k * 4);
}

size_t backward_workspace(const gns_ctx* c, int32_t f1, int32_t f2, int32_t hdim, int32_t rows)
{
    const size_t k = (size_t) f1 + (size_t) f2;
    size_t parts = 0;
    for (int i = 0; i < 3; ++i) {
        // The splits of a plan grow with the rows, but narrow blocks have more tiles, so the most of both is taken: narrow ones
        // are used up to the last rows whose wide blocks fill less than half the chip.
        const bool fp32 = i == 0;
        const WeightsPlan wide = plan_weights_of(c, f1, f2, hdim, rows, fp32, true);
        int64_t narrow_rows = rows;
        if (i < 2 && may_be_wide(f1, f2, hdim, fp32)) {
            const int64_t tiles = (int64_t) wide.m_tiles * wide.n_tiles, splits = (c->num_cus / 2 + tiles - 1) / tiles;
            if (tiles * wide.splits >= c->num_cus / 2) {
                narrow_rows = min(narrow_rows, (splits - 1) * 128);
                parts = max(parts, parts_bytes(wide, k, (size_t) hdim));
            }
        }
        parts = max(parts, parts_bytes(plan_weights_of(c, f1, f2, hdim, narrow_rows, fp32, false), k, (size_t) hdim));
    }
    return parts + max(terms_bytes(k, (size_t) hdim), max(most_input_bytes<float>(c, k, hdim, rows), most_input_bytes<Bf16>(c, k, hdim, rows)));
}

// Threads that share a sum: all sums' first reads should be on their way at once.
static JoinArgs join_of(const gns_ctx* c, const float* parts, float* out, int64_t count, int32_t splits)
{
    const int64_t fours = (count + 3) / 4;
    const int32_t threads = splits <= 8 ? 1 : fours * 16 > (int64_t) c->num_cus * kBlock ? 16 : 64;
    return {parts, out, count, splits, threads, (int32_t) grid_of(c, fours * threads)};
}

template <typename T>
static hipError_t launch_typed(const gns_ctx* c, const BackwardArgs& a, hipStream_t s)
{
    constexpr bool kFloat = sizeof(T) == 4;
    const int32_t K = a.x1.width + a.x2.width;
    const int64_t pitch = ((int64_t) a.hdim + kStageK - 1) / kStageK * kStageK;
    char* at = static_cast<char*>(a.workspace);
    BetweenArgs b = {};
    b.k = K;
    const bool dx = a.dx.data && a.count.rows;
    WeightsPlan pw = {};
    if (a.dw) pw = plan_weights(c, a.x1.width, a.x2.width, a.hdim, a.count.rows, kFloat, kFloat || reads_pairs(a.d_out));
    // dw and dx in one launch where both have blocks of 256 threads and dx takes W as it is
    const bool may_both = dx && a.dw && !pw.wide;
    InputPlan p = dx ? plan_input<T>(c, a, may_both) : InputPlan{Way::kFew, 1};
    const bool both = may_both && p.way == Way::kPlain;
    if (both) plan_both<T>(c, a, &pw, &p);
    WeightsArgs gw = {a, pw.m_tiles, pw.n_tiles, pw.splits, pw.db_shares, a.dw, a.db};
    if (a.dw && pw.splits > 1) {
        gw.dw = reinterpret_cast<float*>(at);
        at += align256((size_t) pw.splits * (size_t) K * (size_t) a.hdim * 4);
        b.dw = join_of(c, gw.dw, a.dw, (int64_t) K * a.hdim, pw.splits);
    }
    if (a.dw && a.db && pw.splits * pw.db_shares > 1) {
        gw.db = reinterpret_cast<float*>(at);
        at += align256((size_t) pw.splits * (size_t) pw.db_shares * (size_t) a.hdim * 4);
        b.db = join_of(c, gw.db, a.db, a.hdim, pw.splits * pw.db_shares);
    }
    if (dx && (p.way == Way::kCut || p.way == Way::kWide)) {
        b.w = a.w;
        b.terms = reinterpret_cast<uint16_t*>(at);
        b.hdim = a.hdim; b.pitch = (int32_t) pitch;
        b.term_blocks = (int32_t) grid_of(c, K * (pitch / 4));
    }
    InputArgs g = {a, 0, 0, (int32_t) pitch, p.splits, b.terms, nullptr};
    if (p.splits > 1) {
        b.dx_parts = g.parts = reinterpret_cast<float*>(at);
        b.dx = a.dx; b.count = a.count;
        b.dx_type = kFloat ? GNS_FP32 : GNS_BF16;
        b.dx_splits = p.splits;
        b.dx_blocks = (int32_t) grid_of(c, (int64_t) a.count.rows * K);
    }
    hipError_t e = hipSuccess;
    if (both)      e = launch_both<T>(gw, g, s);
    else if (a.dw) e = pw.wide ? launch_weights<T, 512>(gw, s) : launch_weights<T, 256>(gw, s);
    if (e == hipSuccess && p.splits > 1 && !both) e = launch_input<T, 256, true>(c, g, s);      // in front of the sums
    if (e != hipSuccess) return e;
    const int32_t blocks = b.db.blocks + b.dw.blocks + b.dx_blocks + b.term_blocks;
    if (blocks) hipLaunchKernelGGL(k_backward_between, dim3((unsigned) blocks), dim3(kBlock), 0, s, b);
    if (!dx || p.splits > 1 || both) return hipGetLastError();
    switch (p.way) {
    case Way::kNarrow: return launch_narrow<T>(c, a, s);
    case Way::kFew:    return launch_few<T>(a, s);
    case Way::kPlain:  return launch_input<T, 256, true>(c, g, s);
    case Way::kCut:    return launch_input<T, 256, false>(c, g, s);
    default:           return launch_input<T, 512, false>(c, g, s);
    }
}

hipError_t launch_backward(const gns_ctx* c, const BackwardArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_typed<float>(c, a, s) : launch_typed<Bf16>(c, a, s);
}

}  // namespace gns
