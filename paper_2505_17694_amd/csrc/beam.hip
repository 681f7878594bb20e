// Beam search: the best continuations over beams and vocabulary, and the states of the beams that go on.
//
// Continuing a beam of score c with token t scores c + (x_t - m) - log S, with m the largest logit of the beam and
// S = sum_u exp(x_u - m).  Inside a beam the order is that of the logits, so a beam brings at most its k best tokens; which
// of those the search keeps is decided between the beams, on scores in 64 bits.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "operators.hpp"

namespace codec {
namespace {

constexpr float kMinusInf = -__builtin_inff();

template <int DT>
__device__ __forceinline__ float logit_at(const char *row, int64_t i)
{
    float x;
    if constexpr (DT == CODEC_DTYPE_FP32) x = reinterpret_cast<const float *>(row)[i];
    else if constexpr (DT == CODEC_DTYPE_FP16) x = float(reinterpret_cast<const _Float16 *>(row)[i]);
    else x = __uint_as_float(uint32_t(reinterpret_cast<const uint16_t *>(row)[i]) << 16);
    // NaN is ruled out like -inf; +inf is the largest number, so that differences stay numbers
    return x != x ? kMinusInf : fminf(x, 3.402823466e38f);
}

// Order of (logit, token) as an integer: the higher logit, then the lower token, is the larger key.  -0 is 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) { return uint64_t(order_of(x)) << 32 | (0xffffffffu - token); }
__device__ __forceinline__ uint32_t token_of(uint64_t key) { return 0xffffffffu - uint32_t(key); }
__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t b = uint32_t(key >> 32);
    return __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b);
}

// A beam whose logits do not count: finished, or of score -inf (NaN and +inf are taken for that).
__device__ __forceinline__ bool score_counts(float s) { return s > kMinusInf && s < __builtin_inff(); }
__device__ __forceinline__ bool reads_logits(const BeamParams &P, int row)
{
    return score_counts(P.scores[row]) && !(P.finished && P.finished[row]);
}

// ---- the 64 best of many, one in a lane ------------------------------------------------------------------
//
// A wave keeps a list of keys in decreasing order, the i-th best in lane i, 0 where there is none; keys are distinct.

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane)
{
    const uint32_t lo = __builtin_amdgcn_readlane(uint32_t(v), lane), hi = __builtin_amdgcn_readlane(uint32_t(v >> 32), lane);
    return uint64_t(hi) << 32 | lo;
}

// The value of lane ^ N, without the LDS unit: row operations up to 15, swaps of rows and halves above.
template <int N>
__device__ __forceinline__ uint32_t from_lane_xor(uint32_t v)
{
    auto moved = [](uint32_t x, auto control) { return uint32_t(__builtin_amdgcn_update_dpp(0, x, decltype(control)::value, 0xf, 0xf, true)); };
    if constexpr (N == 1) return moved(v, std::integral_constant<int, 0xb1>{});             // quad_perm 1 0 3 2
    else if constexpr (N == 2) return moved(v, std::integral_constant<int, 0x4e>{});        // quad_perm 2 3 0 1
    else if constexpr (N == 4) return moved(moved(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1b>{});   // ^ 7 ^ 3
    else if constexpr (N == 8) return moved(v, std::integral_constant<int, 0x128>{});       // row_ror 8
    else if constexpr (N == 16) {
        const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);             // even rows twice, odd rows twice
        return threadIdx.x & 16 ? rows[0] : rows[1];
    } else if constexpr (N == 32) {
        const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? halves[0] : halves[1];
    } else {
        static_assert(N == 63);
        return from_lane_xor<32>(from_lane_xor<16>(moved(v, std::integral_constant<int, 0x140>{})));    // row_mirror
    }
}
template <int N>
__device__ __forceinline__ uint64_t from_lane_xor(uint64_t v)
{
    return uint64_t(from_lane_xor<N>(uint32_t(v >> 32))) << 32 | from_lane_xor<N>(uint32_t(v));
}

// A bitonic list (over runs of 2 * N lanes) into decreasing order, or increasing where `up`.
template <int N, class T>
__device__ __forceinline__ T bitonic_steps(T v, int lane, bool up)
{
    const T other = from_lane_xor<N>(v);
    const bool first = (lane & N) == 0;                 // the lower lane of the two takes the larger key
    v = (other > v) == (first != up) ? other : v;
    if constexpr (N > 1) return bitonic_steps<N / 2>(v, lane, up);
    else return v;
}

template <class T>
__device__ __forceinline__ T sort_lanes(T v, int lane)
{
    v = bitonic_steps<1>(v, lane, lane & 2);
    v = bitonic_steps<2>(v, lane, lane & 4);
    v = bitonic_steps<4>(v, lane, lane & 8);
    v = bitonic_steps<8>(v, lane, lane & 16);
    v = bitonic_steps<16>(v, lane, lane & 32);
    return bitonic_steps<32>(v, lane, false);
}

// The 64 best of two decreasing lists: the larger of entry i of one and entry 63 - i of the other, which is bitonic.
template <class T>
__device__ __forceinline__ T merge_lanes(T a, T b, int lane)
{
    const T other = from_lane_xor<63>(b);
    return bitonic_steps<32>(other > a ? other : a, lane, false);
}

struct BestList {
    uint64_t key = 0;       // this lane's entry
    uint64_t least = 0;     // the entry a newcomer has to beat: number `wanted`, 0 while there are fewer
    int lane, wanted;

    __device__ BestList(int lane_, int wanted_) : lane(lane_), wanted(wanted_) {}

    // One newcomer a lane (0: none).  A few are put in their places one by one; many are sorted and merged.
    __device__ void absorb(uint64_t newcomer)
    {
        uint64_t hits = __ballot(newcomer > least);
        if (__popcll(hits) > 10) {
            const uint64_t sorted = sort_lanes(newcomer > least ? newcomer : uint64_t(0), lane);
            key = __any(key != 0) ? merge_lanes(key, sorted, lane) : sorted;
            least = lane_value(key, wanted - 1);
            return;
        }
        for (; hits; hits &= hits - 1) {
            const uint64_t k = lane_value(newcomer, __builtin_ctzll(hits));
            if (k <= least) continue;
            const int at = __popcll(__ballot(key > k));
            const uint32_t lo = __builtin_amdgcn_update_dpp(0, uint32_t(key), 0x138 /* wave_shr:1 */, 0xf, 0xf, false);
            const uint32_t hi = __builtin_amdgcn_update_dpp(0, uint32_t(key >> 32), 0x138, 0xf, 0xf, false);
            key = lane < at ? key : lane == at ? k : uint64_t(hi) << 32 | lo;
            least = lane_value(key, wanted - 1);
        }
    }
};

// Over all lanes, in every lane.
template <class T, class Combine>
__device__ __forceinline__ T wave_reduce(T x, Combine combine)
{
    typedef std::conditional_t<sizeof(T) == 8, uint64_t, uint32_t> Bits;
    auto step = [&](auto n) { x = combine(x, __builtin_bit_cast(T, from_lane_xor<decltype(n)::value>(__builtin_bit_cast(Bits, x)))); };
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 8>{});
    step(std::integral_constant<int, 16>{});
    step(std::integral_constant<int, 32>{});
    return x;
}
__device__ __forceinline__ float wave_max(float x) { return wave_reduce(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ double wave_sum(double x) { return wave_reduce(x, [](double a, double b) { return a + b; }); }

// One instruction; fmaxf of values that may be signalling NaN takes another one for each.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}

// ---- the sum of exponentials -----------------------------------------------------------------------------
//
// Kept as sum * 2^ref, in 64 bits, with whole references.  log2(e) stands for its 32-bit value throughout: what that is off by,
// 1.3e-8 of itself, weighs on the distance from the largest logit only, because that is brought to the same scale at the end.

constexpr float kLog2e = 1.44269502f;
constexpr double kNoRef = -1e300;

// sum * 2^(from - to) for a whole from <= to.
__device__ __forceinline__ double rescaled(double sum, double from, double to)
{
    const double by = from - to;
    return __builtin_ldexp(sum, by > -4000.0 ? int(by) : -4000);
}

// The lanes' sums joined, in every lane.
__device__ __forceinline__ PartialSum joined(PartialSum x)
{
    const double ref = wave_reduce(x.ref, [](double a, double b) { return a > b ? a : b; });
    return {ref, wave_sum(rescaled(x.sum, x.ref, ref))};
}

constexpr int kPieces = 32;                 // tokens of a lane in a chunk
constexpr int kChunk = 64 * kPieces;

typedef uint32_t __attribute__((ext_vector_type(4), aligned(2))) AnyVec;        // rows start at any element

template <int DT>
struct Logits {
    static constexpr int kSize = DT == CODEC_DTYPE_FP32 ? 4 : 2;
    static constexpr int kPerLoad = 16 / kSize;
    static constexpr int kLoads = kPieces / kPerLoad;
    typedef AnyVec Vec;

    // Tokens of a lane: kPerLoad consecutive ones of each of kLoads consecutive pieces of 64 lanes.
    __device__ static __forceinline__ int token(int chunk, int lane, int e)
    {
        return chunk * kChunk + (e / kPerLoad * 64 + lane) * kPerLoad + e % kPerLoad;
    }
    __device__ static __forceinline__ float widen(Vec v, int e)
    {
        if constexpr (DT == CODEC_DTYPE_FP32) return __uint_as_float(v[e]);
        else if constexpr (DT == CODEC_DTYPE_FP16) return float(__builtin_bit_cast(_Float16, uint16_t(e & 1 ? v[e / 2] >> 16 : v[e / 2])));
        else return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    }
    template <bool ONCE>
    __device__ static __forceinline__ void load(const char *row, int chunk, int lane, Vec (&raw)[kLoads])
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const Vec *at = reinterpret_cast<const Vec *>(row + int64_t(token(chunk, lane, j * kPerLoad)) * kSize);
            if constexpr (ONCE) raw[j] = __builtin_nontemporal_load(at);
            else raw[j] = *at;
        }
    }
    // The row's last chunk: tokens behind the last one are -inf.
    __device__ static __forceinline__ void load_last(const char *row, int chunk, int lane, int vocab, Vec (&raw)[kLoads])
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int t = token(chunk, lane, j * kPerLoad);
            const char *at = row + int64_t(t) * kSize;
            if (t + kPerLoad <= vocab) {
                raw[j] = *reinterpret_cast<const Vec *>(at);
                continue;
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if constexpr (kSize == 4) {
                    raw[j][w] = t + w < vocab ? reinterpret_cast<const uint32_t *>(at)[w] : 0xff800000u;
                } else {
                    constexpr uint32_t kInf = DT == CODEC_DTYPE_FP16 ? 0xfc00u : 0xff80u;
                    const uint16_t *p = reinterpret_cast<const uint16_t *>(at);
                    const uint32_t lo = t + 2 * w < vocab ? p[2 * w] : kInf, hi = t + 2 * w + 1 < vocab ? p[2 * w + 1] : kInf;
                    raw[j][w] = hi << 16 | lo;
                }
            }
        }
    }
};

constexpr int kRowWaves = 8;                // most waves of a workgroup that share a beam's tokens
constexpr int kTops = 16;                   // of a lane's chunks it keeps the largest logit; from the 17th on two or more share one

// Newcomers of a wave, collected 64 at a time in LDS before they are sorted into its list.
struct Collector {
    uint64_t *room;                         // 64 entries of LDS, this wave's own
    BestList best;
    int count = 0;
    bool sorted = false;                    // some have gone into the list

    __device__ Collector(uint64_t *room_, int lane, int wanted) : room(room_), best(lane, wanted) {}

    // The wave's LDS operations are in order; the compiler is told.
    __device__ static void settle()
    {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __device__ void flush()
    {
        settle();
        best.absorb(best.lane < count ? room[best.lane] : 0);
        settle();
        count = 0;
        sorted = true;
    }
    __device__ void add(bool has, uint64_t key)
    {
        has = has && key > best.least;
        const uint64_t mask = __ballot(has);
        const int n = __popcll(mask);
        if (!n) return;
        if (count + n > 64) flush();
        if (has) room[count + __popcll(mask & ((uint64_t(1) << best.lane) - 1))] = key;
        count += n;
    }
    // What there is, at most 64 entries, in `room`; how many.
    __device__ int finish()
    {
        if (!sorted) return count;
        flush();
        room[best.lane] = best.key;
        return __popcll(__ballot(best.key != 0 && best.lane < best.wanted));
    }
};

// The best tokens and the sum of a beam's part of the vocabulary, read once: 32 tokens of a chunk in a lane, of which it keeps
// the largest and the sum of 2^(x log2 e - ref).  Tokens are found afterwards.  The workgroup's lanes form groups; the
// `kept`-th largest of the groups' largest is a bar that at least `kept` tokens reach, all of them in lanes whose largest does.
// Groups are as wide as leaves two for every token wanted: with 32 groups and 16 wanted half of the groups reach the bar, which
// 22 tokens then do.  Only the chunks of a lane whose largest reaches it are read again: 134 MB of logits make 139 MB fetched
// (all chunks of such a lane: 170 MB, and 2 us more).  A mask that leaves tokens in fewer groups than are wanted leaves no bar: every
// logit is looked at again, and a selection of 64 x 8 x 131072 takes 165 us in the place of 34.
// Bound by the loads: a token takes seven lane operations, four of them the exponential.  64 x 8 beams of 131072 bf16 logits
// (134 MB) take 27 us, of which the search for the tokens is 3 to 4; the read alone would be 20 at 6.9 TB/s.  The waves of a
// workgroup take turns along the vocabulary: without that search, and with the kernel that follows, 34.0 us where each has a
// stretch of its own, 31.6 in turn, 28.7 with the streaming hint too (ONCE); 4 x 32768 fp32 logits, which stay in the caches, 6.4
// in turn and 7.6 with the hint.
template <int DT, bool ONCE>
__global__ __launch_bounds__(kRowWaves * 64) void beam_rows_kernel(BeamParams P)
{
    typedef Logits<DT> L;
    __shared__ uint64_t lists[kRowWaves * 64];
    __shared__ uint32_t groups[kRowWaves * 64], wanted[1];
    __shared__ PartialSum sums[kRowWaves];
    __shared__ int counts[kRowWaves];
    __shared__ float chunk_tops[kRowWaves][kTops][64];
    const int row = blockIdx.x, part = blockIdx.y;
    if (!reads_logits(P, row)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const char *x = P.logits + (row / P.beams * P.batch_stride + row % P.beams * P.beam_stride) * L::kSize;
    const int chunks = (P.vocab + kChunk - 1) / kChunk, whole = P.vocab / kChunk;
    const int first = part * waves + wave, step = int(gridDim.y) * waves;

    double ref = kNoRef, sum = 0.0;
    float mine = kMinusInf;
    auto load = [&](int chunk, typename L::Vec (&raw)[L::kLoads]) {
        if (chunk < whole) L::template load<ONCE>(x, chunk, lane, raw);
        else L::load_last(x, chunk, lane, P.vocab, raw);
    };
    typename L::Vec raw[L::kLoads];
    if (first < chunks) load(first, raw);
    int turn = 0;
    for (int chunk = first; chunk < chunks; chunk += step, ++turn) {
        float v[kPieces];
#pragma unroll
        for (int e = 0; e < kPieces; ++e) v[e] = L::widen(raw[e / L::kPerLoad], e % L::kPerLoad);
        if (chunk + step < chunks) load(chunk + step, raw);

        auto largest = [&] {
            float m[2] = {max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5])};
#pragma unroll
            for (int e = 6; e < kPieces; e += 2) m[e / 2 % 2] = max3(m[e / 2 % 2], v[e], v[e + 1]);
            return fmaxf(m[0], m[1]);
        };
        auto total = [&](auto term) {
            float t[4] = {term(v[0]), term(v[1]), term(v[2]), term(v[3])};
#pragma unroll
            for (int e = 4; e < kPieces; ++e) t[e % 4] += term(v[e]);
            return (t[0] + t[1]) + (t[2] + t[3]);
        };
        float top = largest();
        if (ref == kNoRef) {
            const float all = wave_max(top);
            if (__builtin_fabsf(all) < 0x1p20f) ref = __builtin_ceilf(all * kLog2e);
        }
        // The chunk's terms go by the reference where 32 bits hold it (2^24; one that the other branch has set may be of any size)
        // and none lies far above it; false for NaN, too.
        const float r = float(ref);
        const float chunk_sum = total([r](float a) { return __builtin_amdgcn_exp2f(__builtin_fmaf(a, kLog2e, -r)); });
        if (__builtin_fabs(ref) <= 0x1p24 && __all(chunk_sum < 0x1p20f)) {
            sum += double(chunk_sum);
        } else {
            // no reference yet or one too large, terms far above it, +inf, NaN, no token at all: differences from the
            // chunk's largest, whose distance to the reference is taken in 64 bits
#pragma unroll
            for (int e = 0; e < kPieces; ++e) v[e] = v[e] != v[e] ? kMinusInf : fminf(v[e], 3.402823466e38f);
            top = largest();
            const float all = wave_max(top);
            if (all > kMinusInf) {
                const double at = double(all) * double(kLog2e);
                if (at > ref) {
                    sum = rescaled(sum, ref, __builtin_ceil(at));
                    ref = __builtin_ceil(at);
                }
                sum += double(total([all](float a) { return __builtin_amdgcn_exp2f((a - all) * kLog2e); })) * exp2(at - ref);
            }
        }
        if (chunks > step) {                            // else `mine` is all there is
            float *kept_top = &chunk_tops[wave][turn % kTops][lane];
            *kept_top = turn < kTops ? top : fmaxf(*kept_top, top);
        }
        mine = fmaxf(mine, top);
    }

    // the bar; 0 where there are fewer groups with tokens than tokens wanted
    const uint32_t reach = first < chunks && L::token(first, lane, 0) < P.vocab ? order_of(mine) : 0;
    const int width = waves * 64 >= 32 * P.kept ? 16 : waves * 64 >= 16 * P.kept ? 8 : waves * 64 >= 8 * P.kept ? 4 : waves * 64 >= 4 * P.kept ? 2 : 1;
    uint32_t group = reach;
    auto join = [&](auto n) {
        const uint32_t other = from_lane_xor<decltype(n)::value>(group);
        if (width > decltype(n)::value) group = other > group ? other : group;
    };
    join(std::integral_constant<int, 1>{});
    join(std::integral_constant<int, 2>{});
    join(std::integral_constant<int, 4>{});
    join(std::integral_constant<int, 8>{});
    const int entries = waves * 64 / width;
    if (lane % width == 0) groups[(wave * 64 + lane) / width] = group;
    __syncthreads();
    if (wave == 0) {
        uint32_t best = 0;
        for (int i = lane; i - lane < entries; i += 64) {
            const uint32_t sorted = sort_lanes(i < entries ? groups[i] : 0u, lane);
            best = i == lane ? sorted : merge_lanes(best, sorted, lane);
        }
        if (lane == P.kept - 1) *wanted = best;
    }
    __syncthreads();
    const uint32_t bar = *wanted;
    const float least = bar > order_of(kMinusInf) ? logit_of(uint64_t(bar) << 32) : kMinusInf;      // -inf: any token, NaN too

    // the tokens that reach it, of the lanes' chunks that do: up to 64 (lane, place of the chunk's largest) at a time, 16 bytes of
    // one of them in a lane
    uint32_t *places = groups + wave * 64;              // nobody reads the groups any more
    const int tops = turn < kTops ? turn : kTops;
    const int pieces = (turn + kTops - 1) / kTops * L::kLoads;
    Collector found(lists + wave * 64, lane, P.kept);
    int listed = 0;
#pragma unroll 1
    for (int top = 0; top <= tops; ++top) {
        const bool reaches = top < tops && reach >= bar && reach && (chunks <= step || least == kMinusInf || chunk_tops[wave][top][lane] >= least);
        const uint64_t reaching = __ballot(reaches);
        const int more = __popcll(reaching);
        if (top == tops || listed + more > 64) {
            Collector::settle();
            for (int i = lane; i - lane < listed * pieces; i += 64) {
                uint32_t hits = 0;
                int t = 0;
                if (i < listed * pieces) {
                    const uint32_t place = places[i / pieces];
                    const int piece = i % pieces;
                    t = L::token(first + (int(place / 64) + piece / L::kLoads * kTops) * step, place % 64, piece % L::kLoads * L::kPerLoad);
                    const int n = P.vocab - t;
                    if (n >= L::kPerLoad) {
                        const typename L::Vec some = *reinterpret_cast<const typename L::Vec *>(x + int64_t(t) * L::kSize);
#pragma unroll
                        for (int e = 0; e < L::kPerLoad; ++e) hits |= L::widen(some, e) >= least || least == kMinusInf ? 1u << e : 0u;
                    } else {
                        for (int e = 0; e < n; ++e) hits |= logit_at<DT>(x, t + e) >= least ? 1u << e : 0u;
                    }
                }
                while (__any(hits != 0)) {
                    const int token = t + __builtin_ctz(hits | 0x80000000u);
                    found.add(hits != 0, hits ? key_of(logit_at<DT>(x, token), token) : 0);
                    hits &= hits - 1;
                }
            }
            Collector::settle();
            listed = 0;
        }
        if (reaches) places[listed + __popcll(reaching & ((uint64_t(1) << lane) - 1))] = uint32_t(top * 64 + lane);
        listed += more;
    }

    const int count = found.finish();
    const double wave_total = wave_sum(sum);
    if (lane == 0) {
        sums[wave] = {ref, wave_total};
        counts[wave] = count;
    }
    __syncthreads();
    if (wave) return;
    // what the waves have found, 64 entries at a time
    BestList best(lane, P.kept);
    int all = 0;
    for (int w = 0; w < waves; ++w) all += counts[w];
    for (int i = lane; i - lane < all; i += 64) {
        uint64_t key = 0;
        int at = i;
        for (int w = 0; w < waves; ++w) {
            if (at >= 0 && at < counts[w]) key = lists[w * 64 + at];
            at -= counts[w];
        }
        best.absorb(key);
    }
    const PartialSum total = joined(lane < waves ? sums[lane] : PartialSum{kNoRef, 0.0});
    if (lane == 0) P.sums[int64_t(row) * P.parts + part] = total;
    if (lane < P.kept) P.best[(int64_t(row) * P.parts + part) * P.kept + lane] = best.key;
}

// Order of (score, beam, place in the beam's list) as an integer: the higher score, then the lower beam and place, is the
// larger key.  The score keeps 52 of its 64 bits, 2^-40 of itself: what is nearer counts as equal.
__device__ __forceinline__ uint64_t score_key(double score, int place)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, score + 0.0);
    return ((b ^ (b >> 63 ? ~uint64_t(0) : uint64_t(1) << 63)) & ~uint64_t(0xfff)) | uint64_t(0xfff - place);
}

constexpr int kMergeBeams = 8;              // most waves of a workgroup, a beam at a time each

// A workgroup per search: every beam's parts are joined by a wave, which scores the beam's best tokens; then one wave
// finds the best of all.
__global__ __launch_bounds__(kMergeBeams * 64) void beam_merge_kernel(BeamParams P)
{
    extern __shared__ uint64_t keys[];      // per beam and place: the score's key, the score, the token; 64 KB at most
    float *scores = reinterpret_cast<float *>(keys + P.beams * P.kept);
    int32_t *tokens = reinterpret_cast<int32_t *>(scores + P.beams * P.kept);
    const int search = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    for (int beam = wave; beam < P.beams; beam += waves) {
        const int row = search * P.beams + beam;
        // everything is fetched at once; of a beam whose logits do not count nothing was stored, and nothing is used
        const uint64_t *from = P.best + int64_t(row) * P.parts * P.kept;
        const int entries = P.parts * P.kept;
        const uint64_t some = lane < entries ? from[lane] : 0;
        const PartialSum part = lane < P.parts ? P.sums[int64_t(row) * P.parts + lane] : PartialSum{kNoRef, 0.0};
        const float before = P.scores[row];
        const bool done = P.finished && P.finished[row];
        double score = -__builtin_inf();
        int token = lane;
        if (!score_counts(before)) {
            // every token of it scores -inf
        } else if (done) {
            if (lane == 0) score = before;
            token = lane == 0 ? P.eos : lane - 1 < P.eos ? lane - 1 : lane;
        } else {
            BestList best(lane, P.kept);
            if (P.parts == 1) best.key = some;
            else best.absorb(some);
            for (int i = lane + 64; i - lane < entries; i += 64) best.absorb(i < entries ? from[i] : 0);
            PartialSum all = joined(part);
            for (int i = lane + 64; i - lane < P.parts; i += 64) {
                const PartialSum next = joined(i < P.parts ? P.sums[int64_t(row) * P.parts + i] : PartialSum{kNoRef, 0.0});
                all = joined(lane == 0 ? all : lane == 1 ? next : PartialSum{kNoRef, 0.0});
            }
            const float top = logit_of(lane_value(best.key, 0)), x = logit_of(best.key);
            // log of the sum of exp(x - top)
            const double log_sum = log(all.sum) + (all.ref - double(top) * double(kLog2e)) * 0.6931471805599453;
            if (x > kMinusInf) score = double(before) + ((double(x) - double(top)) - log_sum);
            token = int(token_of(best.key));
        }
        if (lane < P.kept) {
            const int at = beam * P.kept + lane;
            scores[at] = float(score);
            keys[at] = score_key(score, beam * 64 + lane);
            tokens[at] = token;
        }
    }
    __syncthreads();
    if (wave) return;
    // the beams' best first: what follows seldom beats them
    BestList best(lane, P.k);
    const int entries = P.beams * P.kept;
    for (int i = lane; i - lane < entries; i += 64) best.absorb(i < entries ? keys[i % P.beams * P.kept + i / P.beams] : 0);
    if (lane < P.k) {
        const int place = 0xfff - int(best.key & 0xfff), beam = place / 64, at = beam * P.kept + place % 64;
        const int64_t to = int64_t(search) * P.k + lane;
        P.out_scores[to] = scores[at];
        P.out_beams[to] = beam;
        P.out_tokens[to] = tokens[at];
    }
}

// A workgroup copies PIECES * 256 units of one row of one state, PIECES of a lane in flight.  Bound by HBM: 33 states of 16 KB a
// beam of 512 beams (277 MB written, 181 MB of rows that a beam follows) take 79 us, whether the same buffers are moved again or
// others.  PIECES 2, 4 and 8: 79, 81 and 81 us there; 8 states of 16386 bytes, in units of two, 57, 37 and 29 us out of HBM, 46, 31
// and 25 out of the last-level cache.  LARGE: with the streaming hint; 86 us without.  One state of single bytes beside 32 of 16 KB
// makes bytes the unit of all: 108 us in the place of 77.  (All with random contents: zeros move up to a fifth faster.)
template <class Unit, int PIECES, bool LARGE>
__global__ __launch_bounds__(256) void reorder_kernel(ReorderParams P)
{
    const ReorderState &state = P.states[blockIdx.z];
    const int64_t begin = int64_t(blockIdx.y) * (PIECES * 256) + threadIdx.x;
    if (begin - threadIdx.x >= state.row_units) return;
    const int row = blockIdx.x;
    const int beam = P.beams[row];
    if (beam < 0 || beam >= P.beams_in) return;
    const int64_t search = row / P.beams_out, to = row % P.beams_out;
    const Unit *src = reinterpret_cast<const Unit *>(state.src + search * state.src_batch + beam * state.src_beam);
    Unit *dst = reinterpret_cast<Unit *>(state.dst + search * state.dst_batch + to * state.dst_beam);
    for (int64_t i = begin; i - threadIdx.x < state.row_units; i += int64_t(gridDim.y) * (PIECES * 256)) {
        Unit x[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int64_t at = i + j * 256;
            x[j] = src[at < state.row_units ? at : 0];          // no branch around a load: it would be waited for at once
        }
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            if (i + j * 256 >= state.row_units) break;
            if constexpr (LARGE) __builtin_nontemporal_store(x[j], dst + i + j * 256);
            else dst[i + j * 256] = x[j];
        }
    }
}

}  // namespace

// Waves that share a beam: enough for 16 on every CU, each with a chunk at least.  From 1366 rows on a workgroup has fewer than four
// waves, and a CU's LDS holds four workgroups: 1024 rows of 131072 bf16 logits (16 waves a CU) are read at 5.0 TB/s, 4096 rows
// (four) at 3.8, 285 us.
BeamSplit beam_split(int64_t rows, int vocab)
{
    const int64_t chunks = (int64_t(vocab) + kChunk - 1) / kChunk;
    int64_t waves = (4096 + rows - 1) / rows;
    if (waves > chunks) waves = chunks;
    const int64_t parts = (waves + kRowWaves - 1) / kRowWaves;
    return {int((waves + parts - 1) / parts), int(parts)};
}

int launch_beam_select(const BeamParams &p, int dtype, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t rows = int64_t(p.batch) * p.beams;
    const BeamSplit split = beam_split(rows, p.vocab);
    if (split.parts != p.parts) return int(hipErrorInvalidValue);
    const dim3 grid(unsigned(rows), unsigned(split.parts)), block(unsigned(split.waves) * 64);
    const bool once = double(rows) * p.vocab * (dtype == CODEC_DTYPE_FP32 ? 4 : 2) > kLargeBytes;
    auto launch = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (once) hipLaunchKernelGGL((beam_rows_kernel<DT, true>), grid, block, 0, s, p);
        else      hipLaunchKernelGGL((beam_rows_kernel<DT, false>), grid, block, 0, s, p);
    };
    switch (dtype) {
    case CODEC_DTYPE_FP16: launch(std::integral_constant<int, CODEC_DTYPE_FP16>{}); break;
    case CODEC_DTYPE_BF16: launch(std::integral_constant<int, CODEC_DTYPE_BF16>{}); break;
    default: launch(std::integral_constant<int, CODEC_DTYPE_FP32>{}); break;
    }
    if (hipError_t e = hipGetLastError()) return int(e);
    const unsigned waves = unsigned(p.beams < kMergeBeams ? p.beams : kMergeBeams);
    hipLaunchKernelGGL(beam_merge_kernel, dim3(unsigned(p.batch)), dim3(waves * 64), size_t(16) * p.beams * p.kept, s, p);
    return int(hipGetLastError());
}

int launch_reorder(const ReorderParams &p, int unit, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    typedef uint32_t __attribute__((ext_vector_type(2))) Unit8;
    typedef uint32_t __attribute__((ext_vector_type(4))) Unit16;
    auto launch = [&](auto unit_value, auto pieces) {
        typedef decltype(unit_value) Unit;
        constexpr int N = decltype(pieces)::value;
        const int64_t groups = (p.most_units + N * 256 - 1) / (N * 256);
        const dim3 grid(unsigned(p.batch) * unsigned(p.beams_out), unsigned(groups < 1024 ? groups : 1024), unsigned(p.num_states));
        if (p.large) hipLaunchKernelGGL((reorder_kernel<Unit, N, true>), grid, dim3(256), 0, s, p);
        else         hipLaunchKernelGGL((reorder_kernel<Unit, N, false>), grid, dim3(256), 0, s, p);
    };
    auto launch_size = [&](auto unit_value) {
        constexpr int kMany = sizeof(unit_value) == 16 ? 2 : 8;
        if (p.most_units <= 256) launch(unit_value, std::integral_constant<int, 1>{});
        else                     launch(unit_value, std::integral_constant<int, kMany>{});
    };
    switch (unit) {
    case 16: launch_size(Unit16{}); break;
    case 8: launch_size(Unit8{}); break;
    case 4: launch_size(uint32_t{}); break;
    case 2: launch_size(uint16_t{}); break;
    case 1: launch_size(uint8_t{}); break;
    default: return int(hipErrorInvalidValue);
    }
    return int(hipGetLastError());
}

}  // namespace codec
