// Log probabilities of given classes, entropy and best classes of rows of logits, and the gradient of the first two.
//
// With m the largest logit, S = sum e^(z - m) and T = sum e^(z - m) (z - m):  log p_y = (z_y - m) - log S and the entropy is
// log S - T / S.  A row is read once: maximum, S and T are kept together, and what was summed so far is rescaled when the
// maximum grows (with d = m_old - m_new: S <- e^d S, T <- e^d (T + d S)).  All of it, and exp itself, is bound by the bytes of
// the logits; the arithmetic (ten instructions a value, four of them the exponential's cycles) is just short enough for bf16.
#include "gns_learn.hpp"

namespace gns {

constexpr float kLog2E = 1.44269504f, kLog2High = 0.693147182f, kLog2Low = 1.90465429e-9f;       // log 2 = high - low
constexpr float kFar = -1000.f;               // e^kFar is zero in fp32

// e^x but for an error of |x| roundings.  In the sums it adds up to no more than log S is rounded by, since the mean of |z - m| by
// the probabilities is at most log S, and T / S does not notice what S and T share: with exact_exp_of the entropy of 4096 rows of
// 100,003 classes was 2 % nearer in the 2-norm, and the call took 18 % longer.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// e^x to two roundings, where single values are results (the gradient, bound by its bytes): 2^t times 1 + (x - t log 2).  Below
// 2^-126 it is zero.
__device__ __forceinline__ float exact_exp_of(float x)
{
    const float t = x * kLog2E, p = __builtin_amdgcn_exp2f(t), rest = fmaf(t, kLog2Low, fmaf(t, -kLog2High, x));
    return fmaf(p, fmaxf(rest, -1.f), p);         // from -infinity: `rest` is no number, and p zero
}

// A value's place in the order of all values: larger floats have larger keys, and of equal ones (0 and -0 too) the lower index.
typedef unsigned long long Key;
constexpr Key kNoKey = 0x007FFFFFFFFFFFFFull;     // above every class of -infinity, below every other
__device__ __forceinline__ Key key_of(float z, int32_t index)
{
    const uint32_t b = __float_as_uint(z + 0.f), flip = (uint32_t) ((int32_t) b >> 31) | 0x80000000u;
    return (Key) (b ^ flip) << 32 | (uint32_t) ~index;
}
__device__ __forceinline__ float value_of(Key k)
{
    const uint32_t b = (uint32_t) (k >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int32_t index_of(Key k) { return (int32_t) ~(uint32_t) k; }

template <int kCtrl>
__device__ __forceinline__ float dpp_float(float v)
{
    return __uint_as_float((uint32_t) __builtin_amdgcn_update_dpp(0, (int) __float_as_uint(v), kCtrl, 0xf, 0xf, true));
}
template <int kCtrl>
__device__ __forceinline__ int32_t dpp_int(int32_t v) { return __builtin_amdgcn_update_dpp(0, v, kCtrl, 0xf, 0xf, true); }

// Reduction over groups of L consecutive lanes; every lane gets the result.  Up to 16 lanes it stays in the registers.
template <int L, typename Op>
__device__ __forceinline__ float reduce_float(float v, Op op)
{
    if (L > 1) v = op(v, dpp_float<0xB1>(v));      // lanes 1 0 3 2
    if (L > 2) v = op(v, dpp_float<0x4E>(v));      // lanes 2 3 0 1
    if (L > 4) v = op(v, dpp_float<0x141>(v));     // mirrored in halves of a row of 16
    if (L > 8) v = op(v, dpp_float<0x140>(v));     // mirrored in the row
    if (L > 16) v = op(v, __shfl_xor(v, 16));
    if (L > 32) v = op(v, __shfl_xor(v, 32));
    return v;
}
template <int L>
__device__ __forceinline__ float sum_of(float v) { return reduce_float<L>(v, [](float a, float b) { return a + b; }); }
template <int L>
__device__ __forceinline__ float max_of(float v) { return reduce_float<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ __forceinline__ int32_t min_of(int32_t v)
{
    if (L > 1) v = min(v, dpp_int<0xB1>(v));
    if (L > 2) v = min(v, dpp_int<0x4E>(v));
    if (L > 4) v = min(v, dpp_int<0x141>(v));
    if (L > 8) v = min(v, dpp_int<0x140>(v));
    if (L > 16) v = min(v, __shfl_xor(v, 16));
    if (L > 32) v = min(v, __shfl_xor(v, 32));
    return v;
}

// Running maximum and sums.  A NaN or +infinity among the values makes S NaN.
struct Softmax {
    float m, S, T;
};

// The values' maximum becomes (at least) `most`.
__device__ __forceinline__ void raise(Softmax& s, float most)
{
    const float d = fmaxf(s.m - most, kFar);        // from -infinity: nothing was summed yet
    if (most > s.m) {
        const float f = exp_of(d);
        s.T = f * fmaf(d, s.S, s.T);
        s.S *= f;
        s.m = most;
    }
}

// Adds N values none of which is above s.m, summed first, so that a long row's sums are rounded once for N of them (the entropy of
// 100,003 classes 5.2e-8 off in the 2-norm, 8.6e-8 one by one).  Masked ones (-infinity) make T NaN, and it is summed once more with
// their share left out: a test per value would cost all rows what only masked ones need.
template <int N>
__device__ __forceinline__ void add_values(Softmax& s, const float (&z)[N])
{
    const float m = s.m == -__builtin_inff() ? 0.f : s.m;
    float S = 0.f, T = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = z[i] - m, p = exp_of(d);
        S += p;
        T = fmaf(p, d, T);
    }
    if (__builtin_expect(T != T, 0)) {
        T = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = z[i] - m;
            T = fmaf(exp_of(d), fmaxf(d, kFar), T);
        }
    }
    s.S += S;
    s.T += T;
}

// The sums of a group of L lanes; every lane gets them.
template <int L>
__device__ __forceinline__ void join_lanes(Softmax& s)
{
    const float most = max_of<L>(s.m), d = fmaxf(s.m - most, kFar), f = exp_of(d);
    s.T = sum_of<L>(f * fmaf(d, s.S, s.T));
    s.S = sum_of<L>(f * s.S);
    s.m = most;
}

struct RowResult {
    float m, log_sum, entropy;
    bool bad, none;
};
__device__ __forceinline__ RowResult result_of(const Softmax& s)
{
    RowResult o;
    o.bad = s.S != s.S;
    o.none = !o.bad && s.m == -__builtin_inff();
    o.m = o.bad ? quiet_nan() : s.m;
    o.log_sum = o.none ? 0.f : logf(s.S);
    o.entropy = o.none ? 0.f : o.log_sum - s.T / s.S;
    return o;
}
// log p of a class with logit z
__device__ __forceinline__ float log_p_of(const RowResult& o, float z) { return o.none ? -__builtin_inff() : (z - o.m) - o.log_sum; }

template <typename T>
__device__ __forceinline__ void write_row(const LogProbsArgs& a, int64_t r, const RowResult& o, int32_t label, float z_label)
{
    if (a.logp) a.logp[r] = o.bad || label >= a.logits.width ? quiet_nan() : label < 0 ? 0.f : log_p_of(o, z_label);
    if (a.entropy) a.entropy[r] = o.entropy;
    if (a.stats) *reinterpret_cast<float2*>(a.stats + 2 * r) = make_float2(o.m, o.log_sum);
}

template <typename T>
__device__ __forceinline__ float label_logit(const LogProbsArgs& a, int64_t r, int32_t* label)
{
    *label = a.labels ? a.labels[r] : -1;
    return *label >= 0 && *label < a.logits.width ? load_at<T>(a.logits, r, *label) : 0.f;
}

// Rows of up to L * E classes: L lanes a row, E values a lane in registers, 64 / L rows a wave.  The best classes come one
// after the other: each lane has its own best at hand, the lane that wins looks for its next.
// 85,000 rows of 172 classes, fp32: 12.8 us (4.6 TB/s), with five best 25 to 27, with twenty 66: 70 instructions for a best class of
// four rows.  Three in order at hand for each lane, found in one pass, take as long (26.6; twenty 84).
template <typename T, int L, int E>
__global__ void __launch_bounds__(kBlock) k_log_probs_short(LogProbsArgs a)
{
    constexpr float kNone = -__builtin_inff();
    const int32_t rows = a.count.get(), C = a.logits.width;
    const int64_t step = (int64_t) gridDim.x * (kBlock / L);
    // the lanes of a wave make as many turns, as the exchange between them asks for
    for (int64_t r0 = ((int64_t) blockIdx.x * kBlock + (threadIdx.x & ~(kWave - 1))) / L; r0 < rows; r0 += step) {
        const int lane = opaque_lane_id(), l = lane & (L - 1);
        const int64_t row = r0 + lane / L, r = row < rows ? row : rows - 1;
        float z[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int32_t c = e * L + l;
            z[e] = c < C ? load_at<T>(a.logits, r, c) : kNone;
        }
        int32_t label;
        const float z_label = label_logit<T>(a, r, &label);
        Softmax s = {kNone, 0.f, 0.f};
        float mine = kNone;                       // (the larger of a NaN and a number is the number)
#pragma unroll
        for (int e = 0; e < E; ++e) mine = fmaxf(mine, z[e]);
        s.m = max_of<L>(mine);
        add_values(s, z);
        s.S = sum_of<L>(s.S);
        s.T = sum_of<L>(s.T);
        const RowResult o = result_of(s);
        if (l == 0 && row < rows) write_row<T>(a, r, o, label, z_label);
        for (int32_t i = 0; i < a.top; ++i) {
            int32_t slot = 0;
#pragma unroll
            for (int e = E - 1; e >= 0; --e) slot = z[e] == mine ? e : slot;
            const float best = max_of<L>(mine);
            const int32_t index = min_of<L>(mine == best ? slot * L + l : INT32_MAX);
            if (l == 0 && row < rows) {
                const bool gone = o.bad || best == kNone;
                a.top_index[r * a.top + i] = gone ? -1 : index;
                a.top_logp[r * a.top + i] = o.bad ? quiet_nan() : gone ? kNone : log_p_of(o, best);
            }
            const int32_t drop = index == slot * L + l ? slot : -1;
            mine = kNone;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                z[e] = e == drop ? kNone : z[e];
                mine = fmaxf(mine, z[e]);
            }
        }
    }
}

// The best classes a wave has seen, one a lane, in order (kNoKey: none).  What is not above `last` is not among the row's
// best; `last_z` is its value.
struct WaveList {
    Key mine, last;
    float last_z;
};
__device__ __forceinline__ WaveList empty_list() { return WaveList{kNoKey, kNoKey, -__builtin_inff()}; }

__device__ __forceinline__ Key read_lane(Key k, int lane)
{
    return (Key) (uint32_t) __builtin_amdgcn_readlane((int) (uint32_t) (k >> 32), lane) << 32 |
           (uint32_t) __builtin_amdgcn_readlane((int) (uint32_t) k, lane);
}

__device__ __forceinline__ void insert(WaveList& list, Key k)
{
    const int lane = opaque_lane_id(), at = __popcll(__ballot(list.mine > k));
    const uint32_t hi = (uint32_t) __builtin_amdgcn_update_dpp(0, (int) (uint32_t) (list.mine >> 32), 0x138, 0xf, 0xf, true);
    const uint32_t lo = (uint32_t) __builtin_amdgcn_update_dpp(0, (int) (uint32_t) list.mine, 0x138, 0xf, 0xf, true);
    const Key below = (Key) hi << 32 | lo;                     // of the lane below
    list.mine = lane < at ? list.mine : lane == at ? k : below;
}

// Takes up N values a lane; class_of(i) is the class of the lane's i-th.  Nearly all values are passed over by one comparison
// of the lane's largest; equal values are told apart by their classes, so a row of one value costs no insertions after
// the first.
template <int N, typename Class>
__device__ __forceinline__ void take_up(WaveList& list, const float (&z)[N], float largest, int32_t top, Class&& class_of)
{
    if (!__ballot(largest >= list.last_z)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Key k = key_of(z[i], class_of(i));
        uint64_t hits = __ballot(k > list.last);
        if (!hits) continue;
        for (; hits; hits &= hits - 1) insert(list, read_lane(k, __builtin_ctzll(hits)));
        const Key bound = read_lane(list.mine, top - 1);       // none while the list is short
        if (bound > list.last) list.last = bound;
    }
    list.last_z = value_of(list.last);
}

// A bound that at least `top` of the wave's values reach, by way of the lanes' largest: the top-th of those.
__device__ __forceinline__ void bound_by_lanes(WaveList& list, float largest, int32_t top)
{
    int32_t above = 0;
    for (int i = 0; i < kWave; ++i)
        above += __uint_as_float((uint32_t) __builtin_amdgcn_readlane((int) __float_as_uint(largest), i)) > largest ? 1 : 0;
    const float bound = -max_of<kWave>(above < top ? -largest : -__builtin_inff());
    const Key k = key_of(bound, INT32_MAX);                    // every class of that value is above it
    if (k > list.last) {
        list.last = k;
        list.last_z = bound;
    }
}

template <typename T> constexpr int kVec = 16 / (int) sizeof(T);

// Sixteen values of a lane: 16 / kVec<T> pieces of 16 bytes, pieces kWave * kVec<T> values apart.
constexpr int kLaneValues = 16;
constexpr int kWaveTile = kLaneValues * kWave;

template <typename T> struct alignas(16) Piece { T v[kVec<T>]; };

// What a part of a row leaves for the join.
struct PartSums {
    float m, S, T, unused;
};

struct LongArgs {
    LogProbsArgs a;
    int32_t parts;                // of a row
    int32_t tiles;                // of a part
    PartSums* sums;               // [rows x parts], if parts > 1
    Key* best;                    // [rows x parts x top]
};

// 4096 rows of 100,003 classes, bf16, twenty best: 177 us (4.6 TB/s); one row of 131,072, fp32: 12 us and 7 for the join.
// Rows of any length: a wave per row, or per part of a row where there are few.  Pieces of 16 bytes are read at 16-byte
// marks whatever the row's own alignment; the few values in front of the first mark and behind the last are read singly.
template <typename T>
__global__ void __launch_bounds__(kBlock) k_log_probs_long(LongArgs g)
{
    constexpr float kNone = -__builtin_inff();
    constexpr int V = kVec<T>, kPieces = kLaneValues / V;
    const LogProbsArgs& a = g.a;
    const int32_t rows = a.count.get(), C = a.logits.width, top = a.top;
    const int64_t work = (int64_t) rows * g.parts;
    for (int64_t w = (int64_t) blockIdx.x * (kBlock / kWave) + __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)); w < work;
         w += (int64_t) gridDim.x * (kBlock / kWave)) {
        const int lane = opaque_lane_id();
        const int64_t r = w / g.parts;
        const int32_t part = (int32_t) (w - r * g.parts);
        const T* row = reinterpret_cast<const T*>(a.logits.data) + r * a.logits.stride;
        const int32_t off = (int32_t) (reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
        const int32_t head = min((V - off) % V, C), body = (C - head) / V;         // pieces
        const Piece<T>* pieces = reinterpret_cast<const Piece<T>*>(row + head);
        const int32_t p0 = (int32_t) min((int64_t) part * g.tiles * (kPieces * kWave), (int64_t) body);
        const int32_t p1 = (int32_t) min((int64_t) (part + 1) * g.tiles * (kPieces * kWave), (int64_t) body);
        int32_t label = -1;
        float z_label = 0.f;
        if (g.parts == 1) z_label = label_logit<T>(a, r, &label);
        Softmax s = {kNone, 0.f, 0.f};
        WaveList list = empty_list();
        bool first = true;
        if (part == 0) {                          // the single values: lanes 0 .. head - 1 and from 32 on
            const int32_t behind = C - head - body * V;
            float z[1] = {kNone};
            const int32_t c = lane < 32 ? lane : head + body * V + lane - 32;
            if (lane < 32 ? lane < head : lane - 32 < behind) z[0] = to_float(row[c]);
            raise(s, z[0]);
            add_values(s, z);
            if (top) take_up(list, z, z[0], top, [&](int) { return c; });
        }
        // pieces of the next tile are on their way while this one's are worked on; those past the part repeat its last one and
        // count as nothing
        Piece<T> x[kPieces];
        auto fetch = [&](int32_t p) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int32_t at = p + j * kWave + lane;
                x[j] = pieces[at < p1 ? at : p1 - 1];
            }
        };
        if (p0 < p1) fetch(p0);
        for (int32_t p = p0; p < p1; p += kPieces * kWave) {
            float z[kLaneValues];
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) z[j * V + v] = p + j * kWave + lane < p1 ? to_float(x[j].v[v]) : kNone;
            if (p + kPieces * kWave < p1) fetch(p + kPieces * kWave);
            float largest = kNone;
#pragma unroll
            for (int i = 0; i < kLaneValues; ++i) largest = fmaxf(largest, z[i]);
            raise(s, largest);
            add_values(s, z);
            if (top) {
                if (first) bound_by_lanes(list, largest, top);
                first = false;
                take_up(list, z, largest, top, [&](int i) { return head + (p + i / V * kWave + lane) * V + i % V; });
            }
        }
        join_lanes<kWave>(s);
        if (g.parts > 1) {
            if (lane == 0) g.sums[w] = PartSums{s.m, s.S, s.T, 0.f};
            if (lane < top) g.best[w * top + lane] = list.mine;
            continue;
        }
        const RowResult o = result_of(s);
        if (lane == 0) write_row<T>(a, r, o, label, z_label);
        if (lane < top) {
            const bool gone = o.bad || list.mine == kNoKey;
            a.top_index[r * top + lane] = gone ? -1 : index_of(list.mine);
            a.top_logp[r * top + lane] = o.bad ? quiet_nan() : gone ? kNone : log_p_of(o, value_of(list.mine));
        }
    }
}

// A wave per row: its parts' sums and best classes, which are on their way first.  A row has no more best classes in its parts than
// a wave reads at once (split_rows).  Bound by latency, 6 to 7 us.
constexpr int kJoinKeys = 16;                 // of a lane
template <typename T>
__global__ void __launch_bounds__(kWave) k_log_probs_join(LongArgs g)
{
    constexpr float kNone = -__builtin_inff();
    const LogProbsArgs& a = g.a;
    const int32_t rows = a.count.get(), top = a.top, n = g.parts * top;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int lane = opaque_lane_id();
        const Key* from = g.best + r * n;
        float z[kJoinKeys];
        int32_t index[kJoinKeys];
        float largest = kNone;
        if (top) {
#pragma unroll
            for (int j = 0; j < kJoinKeys; ++j) {
                const int32_t i = j * kWave + lane;
                const Key k = i < n ? from[i] : kNoKey;
                z[j] = value_of(k);
                index[j] = index_of(k);
                largest = fmaxf(largest, z[j]);
            }
        }
        int32_t label;
        const float z_label = label_logit<T>(a, r, &label);
        Softmax s = {kNone, 0.f, 0.f};
        for (int32_t p = lane; p < g.parts; p += kWave) {
            const PartSums q = g.sums[r * g.parts + p];
            raise(s, q.m);
            const float d = fmaxf(q.m - s.m, kFar), f = exp_of(d);
            s.T += f * fmaf(d, q.S, q.T);
            s.S += f * q.S;
        }
        join_lanes<kWave>(s);
        const RowResult o = result_of(s);
        if (lane == 0) write_row<T>(a, r, o, label, z_label);
        if (!top) continue;
        WaveList list = empty_list();
        bound_by_lanes(list, largest, top);
        take_up(list, z, largest, top, [&](int j) { return index[j]; });
        if (lane < top) {
            const bool gone = o.bad || list.mine == kNoKey;
            a.top_index[r * top + lane] = gone ? -1 : index_of(list.mine);
            a.top_logp[r * top + lane] = o.bad ? quiet_nan() : gone ? kNone : log_p_of(o, value_of(list.mine));
        }
    }
}

// What a row's gradient is made of: p_j (slope (log p_j) + base), and `at` more for the label's class.
struct RowGradient {
    float m, log_sum, base, slope, at;
    int32_t label;
};
__device__ __forceinline__ RowGradient row_gradient(const LogProbsBackwardArgs& a, int64_t r)
{
    const float2 stats = *reinterpret_cast<const float2*>(a.stats + 2 * r);
    RowGradient o;
    o.label = a.labels ? a.labels[r] : -1;
    o.m = stats.x;
    o.log_sum = stats.y;
    o.at = o.label < 0 ? 0.f : o.label >= a.logits.width ? quiet_nan() : a.g_logp[r];
    o.slope = a.g_entropy ? -a.g_entropy[r] : 0.f;
    o.base = -o.at + (a.g_entropy ? o.slope * a.entropy[r] : 0.f);
    if (stats.x == -__builtin_inff()) o.m = o.base = o.slope = o.at = 0.f;      // no class left: every p is zero
    if (stats.x != stats.x) o.base = quiet_nan();                               // where a masked class has p = 0 too
    return o;
}
template <bool kEntropy>
__device__ __forceinline__ float gradient_of(const RowGradient& o, float z)
{
    const float log_p = (z - o.m) - o.log_sum, p = exact_exp_of(log_p);
    return p * (kEntropy ? fmaf(o.slope, fmaxf(log_p, kFar), o.base) : o.base);
}

// L lanes a row (of short rows several a wave), a value at a time; `chunk` columns of a long row.  1000 rows of 47 classes: 2.7 us, a
// launch.
template <typename T, typename O, bool kEntropy, int L>
__global__ void __launch_bounds__(kBlock) k_log_probs_backward(LogProbsBackwardArgs a, int32_t chunk)
{
    const int32_t rows = a.count.get(), C = a.logits.width, l = lane_id() & (L - 1);
    const int32_t chunks = (C + chunk - 1) / chunk;
    const int64_t work = (int64_t) rows * chunks;
    for (int64_t w = ((int64_t) blockIdx.x * kBlock + threadIdx.x) / L; w < work; w += (int64_t) gridDim.x * (kBlock / L)) {
        const int64_t r = chunks == 1 ? w : w / chunks;
        const int32_t c0 = (int32_t) (w - r * chunks) * chunk, c1 = min(c0 + chunk, C);
        const RowGradient o = row_gradient(a, r);
        const T* in = reinterpret_cast<const T*>(a.logits.data) + r * a.logits.stride;
        O* out = reinterpret_cast<O*>(a.d_logits.data) + r * a.d_logits.stride;
        constexpr int kTurn = 4;                  // values on their way together
        for (int32_t c = c0 + l; c < c1; c += kTurn * L) {
            float z[kTurn];
#pragma unroll
            for (int i = 0; i < kTurn; ++i) z[i] = to_float(in[min(c + i * L, c1 - 1)]);
#pragma unroll
            for (int i = 0; i < kTurn; ++i) {
                const float v = gradient_of<kEntropy>(o, z[i]) + (c + i * L == o.label ? o.at : 0.f);
                if (c + i * L < c1) out[c + i * L] = from_float<O>(v);
            }
        }
    }
}

// Long rows whose logits and gradients lie alike against the 16-byte marks: pieces of 16 bytes at the marks, single values
// in front of and behind them.  A wave has `tiles` tiles of a row.  4096 rows of 100,003 classes, bf16: 317 us, 5.2 TB/s, the rate of
// a copy.
template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kBlock) k_log_probs_backward_long(LogProbsBackwardArgs a, int32_t parts, int32_t tiles)
{
    constexpr int V = kVec<T>, kPieces = kLaneValues / V;
    const int32_t rows = a.count.get(), C = a.logits.width, lane = lane_id();
    const int64_t work = (int64_t) rows * parts;
    for (int64_t w = (int64_t) blockIdx.x * (kBlock / kWave) + __builtin_amdgcn_readfirstlane((int) (threadIdx.x >> 6)); w < work;
         w += (int64_t) gridDim.x * (kBlock / kWave)) {
        const int64_t r = w / parts;
        const int32_t part = (int32_t) (w - r * parts);
        const T* in = reinterpret_cast<const T*>(a.logits.data) + r * a.logits.stride;
        T* out = reinterpret_cast<T*>(a.d_logits.data) + r * a.d_logits.stride;
        const int32_t off = (int32_t) (reinterpret_cast<uintptr_t>(in) % 16 / sizeof(T));
        const int32_t head = min((V - off) % V, C), body = (C - head) / V;
        const int32_t p0 = (int32_t) min((int64_t) part * tiles * (kPieces * kWave), (int64_t) body);
        const int32_t p1 = (int32_t) min((int64_t) (part + 1) * tiles * (kPieces * kWave), (int64_t) body);
        const Piece<T>* from = reinterpret_cast<const Piece<T>*>(in + head);
        Piece<T>* to = reinterpret_cast<Piece<T>*>(out + head);
        const RowGradient o = row_gradient(a, r);
        auto value = [&](float z, int32_t c) { return from_float<T>(gradient_of<kEntropy>(o, z) + (c == o.label ? o.at : 0.f)); };
        if (part == 0) {
            const int32_t behind = C - head - body * V, c = lane < 32 ? lane : head + body * V + lane - 32;
            if (lane < 32 ? lane < head : lane - 32 < behind) out[c] = value(to_float(in[c]), c);
        }
        for (int32_t p = p0 + lane; p < p1; p += kPieces * kWave) {
            Piece<T> x[kPieces];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) x[j] = from[min(p + j * kWave, p1 - 1)];
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int32_t c = head + (p + j * kWave) * V;
                const bool here = o.label >= c && o.label < c + V;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float y = gradient_of<kEntropy>(o, to_float(x[j].v[v]));
                    if (here && c + v == o.label) y += o.at;
                    x[j].v[v] = from_float<T>(y);
                }
                if (p + j * kWave < p1) to[p + j * kWave] = x[j];
            }
        }
    }
}

static unsigned grid_of(const gns_ctx* c, int64_t blocks, int per_cu)
{
    const int64_t most = (int64_t) c->num_cus * per_cu;
    return (unsigned) (blocks < most ? blocks : most);
}

constexpr int32_t kShortClasses = 256;

// Parts of a row: two waves on every SIMD, or four of at least 24 tiles, each of two tiles at least, and no more best classes
// than the join reads at once.  A wave's first tile and the join are what best classes cost most: bf16, top 5, 3000 rows of
// 9776 classes whole 24 us, in two parts 31; 1000 rows of 100,003 in four parts 57, in two 60, in eight 63.
static void split_rows(const gns_ctx* c, int32_t classes, int32_t top, int32_t rows, int32_t* parts, int32_t* tiles)
{
    const int32_t all = (int32_t) (((int64_t) classes + kWaveTile - 1) / kWaveTile);
    const int64_t simds = (int64_t) c->num_cus * 4, least = simds * 2 / max(rows, 1), most = simds * 4 / max(rows, 1);
    int64_t p = all / 24 < least ? least : all / 24 < most ? all / 24 : most;
    if (p > all / 2) p = all / 2;
    if (top && p > kJoinKeys * kWave / top) p = kJoinKeys * kWave / top;
    if (p < 1) p = 1;
    *tiles = (int32_t) ((all + p - 1) / p);
    *parts = (all + *tiles - 1) / *tiles;
}

static size_t sums_bytes(int64_t rows, int32_t parts) { return ((size_t) rows * (size_t) parts * sizeof(PartSums) + 255) / 256 * 256; }

size_t log_probs_need(const gns_ctx* c, int32_t classes, int32_t top, int32_t rows)
{
    if (classes <= kShortClasses) return 0;
    int32_t parts, tiles;
    split_rows(c, classes, top, rows, &parts, &tiles);
    return parts == 1 ? 0 : sums_bytes(rows, parts) + (size_t) rows * (size_t) parts * (size_t) top * sizeof(Key);
}

// Few rows have many parts: those of all rows together are no more than four for each SIMD, and those of one no more than it has
// two tiles or the join has room for.
size_t log_probs_workspace(const gns_ctx* c, int32_t classes, int32_t top, int32_t rows)
{
    if (classes <= kShortClasses) return 0;
    const int64_t pairs = ((int64_t) classes + kWaveTile - 1) / kWaveTile / 2;
    const int64_t one = top && pairs > kJoinKeys * kWave / top ? kJoinKeys * kWave / top : pairs, simds = (int64_t) c->num_cus * 4;
    if (one < 2) return 0;
    const int64_t all = one * rows < simds * 4 ? one * rows : simds * 4;
    return sums_bytes(all, 1) + (size_t) all * (size_t) top * sizeof(Key);
}

template <typename T, int L, int E>
static hipError_t launch_short(const gns_ctx* c, const LogProbsArgs& a, hipStream_t s)
{
    const int64_t per_block = kBlock / L;
    hipLaunchKernelGGL((k_log_probs_short<T, L, E>), dim3(grid_of(c, (a.count.rows + per_block - 1) / per_block, 32)), dim3(kBlock), 0, s, a);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_typed(const gns_ctx* c, const LogProbsArgs& a, hipStream_t s)
{
    const int32_t C = a.logits.width;
    if (C <= 16) return launch_short<T, 4, 4>(c, a, s);
    if (C <= 64) return launch_short<T, 8, 8>(c, a, s);
    if (C <= 128) return launch_short<T, 16, 8>(c, a, s);
    if (C <= 192) return launch_short<T, 16, 12>(c, a, s);
    if (C <= kShortClasses) return launch_short<T, 16, 16>(c, a, s);
    LongArgs g = {};
    g.a = a;
    split_rows(c, C, a.top, a.count.rows, &g.parts, &g.tiles);
    if (g.parts > 1) {
        g.sums = static_cast<PartSums*>(a.workspace);
        g.best = reinterpret_cast<Key*>(static_cast<char*>(a.workspace) + sums_bytes(a.count.rows, g.parts));
    }
    const int64_t blocks = ((int64_t) a.count.rows * g.parts + kBlock / kWave - 1) / (kBlock / kWave);
    hipLaunchKernelGGL(k_log_probs_long<T>, dim3(grid_of(c, blocks, 32)), dim3(kBlock), 0, s, g);
    if (g.parts > 1) hipLaunchKernelGGL(k_log_probs_join<T>, dim3(grid_of(c, a.count.rows, 32)), dim3(kWave), 0, s, g);
    return hipGetLastError();
}

hipError_t launch_log_probs(const gns_ctx* c, const LogProbsArgs& a, int32_t type, hipStream_t s)
{
    return type == GNS_FP32 ? launch_typed<float>(c, a, s) : launch_typed<Bf16>(c, a, s);
}

template <typename T, typename O, bool kEntropy>
static hipError_t launch_backward_typed(const gns_ctx* c, const LogProbsBackwardArgs& a, hipStream_t s)
{
    const int32_t C = a.logits.width;
    const int64_t rows = a.count.rows;
    auto lies = [](const void* p, int64_t stride, size_t size) {      // of all rows against the 16-byte marks: their stride and first
        return (uint32_t) (reinterpret_cast<uintptr_t>(p) % 16 + (uint64_t) stride * size % 16 * 16);
    };
    if constexpr (sizeof(T) == sizeof(O)) {
        if (C > kShortClasses && lies(a.logits.data, a.logits.stride, sizeof(T)) == lies(a.d_logits.data, a.d_logits.stride, sizeof(T))) {
            constexpr int32_t kTiles = 4;
            const int32_t parts = (int32_t) (((int64_t) C + kTiles * kWaveTile - 1) / (kTiles * kWaveTile));
            hipLaunchKernelGGL((k_log_probs_backward_long<T, kEntropy>), dim3(grid_of(c, (rows * parts + 3) / 4, 64)), dim3(kBlock), 0, s, a, parts, kTiles);
            return hipGetLastError();
        }
    }
    if (C <= 16) {
        hipLaunchKernelGGL((k_log_probs_backward<T, O, kEntropy, 4>), dim3(grid_of(c, (rows + 63) / 64, 64)), dim3(kBlock), 0, s, a, C);
    } else if (C <= kShortClasses) {
        hipLaunchKernelGGL((k_log_probs_backward<T, O, kEntropy, 16>), dim3(grid_of(c, (rows + 15) / 16, 64)), dim3(kBlock), 0, s, a, C);
    } else {
        constexpr int32_t kChunk = 4096;
        const int64_t work = rows * ((C + kChunk - 1) / kChunk);
        hipLaunchKernelGGL((k_log_probs_backward<T, O, kEntropy, kWave>), dim3(grid_of(c, (work + 3) / 4, 64)), dim3(kBlock), 0, s, a, kChunk);
    }
    return hipGetLastError();
}

hipError_t launch_log_probs_backward(const gns_ctx* c, const LogProbsBackwardArgs& a, int32_t type, int32_t out_type, hipStream_t s)
{
    const bool entropy = a.g_entropy != nullptr;
    if (type == GNS_FP32 && out_type == GNS_FP32)
        return entropy ? launch_backward_typed<float, float, true>(c, a, s) : launch_backward_typed<float, float, false>(c, a, s);
    if (type == GNS_FP32)
        return entropy ? launch_backward_typed<float, Bf16, true>(c, a, s) : launch_backward_typed<float, Bf16, false>(c, a, s);
    if (out_type == GNS_FP32)
        return entropy ? launch_backward_typed<Bf16, float, true>(c, a, s) : launch_backward_typed<Bf16, float, false>(c, a, s);
    return entropy ? launch_backward_typed<Bf16, Bf16, true>(c, a, s) : launch_backward_typed<Bf16, Bf16, false>(c, a, s);
}

}  // namespace gns
