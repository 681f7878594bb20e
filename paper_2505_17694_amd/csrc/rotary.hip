// Rotary positions of new tokens' queries and keys, and their keys and values into the pages of the cache.
//
// A head's channels form pairs: (i, i + r/2) or (2i, 2i + 1) for i < r/2, r the number of channels that turn.  At
// position n pair i turns by n * t_i whole turns: (a, b) -> m (a cos - b sin, b cos + a sin).  Only the fraction of
// n * t_i counts; at position 10^6 it is what 20 bits of the product leave, so the product is taken in 64 bits and
// reduced to an eighth of a turn around the next quarter before the series of sine and cosine run in 32.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "operators.hpp"

namespace codec {
namespace {

template <int DT>
__device__ __forceinline__ float widen(uint16_t x)
{
    if constexpr (DT == CODEC_DTYPE_FP16) return float(__builtin_bit_cast(_Float16, x));
    else return __uint_as_float(uint32_t(x) << 16);
}

// To nearest even
template <int DT>
__device__ __forceinline__ uint16_t narrow(float x)
{
    if constexpr (DT == CODEC_DTYPE_FP16) return __builtin_bit_cast(uint16_t, _Float16(x));
    else return __builtin_bit_cast(uint16_t, __bf16(x));
}

struct Turn { float cos, sin; };

// Cosine and sine of `turns` whole turns.  The Taylor series around the nearest quarter turn: |x| <= pi/4, so the first
// terms left out are below x^11/11! = 2e-9 and x^12/12! = 1e-10, under the half step 3e-8 of 32-bit results near one.
__device__ __forceinline__ Turn turn_of(double turns)
{
    const double quarters = 4.0 * turns;
    const double nearest = __builtin_rint(quarters);
    const float x = float((quarters - nearest) * 1.5707963267948966);
    const float x2 = x * x;
    const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
    const float c = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
    // quarter 0: (c, s); 1: (-s, c); 2: (-c, -s); 3: (s, -c); the remainder of a negative count is negative
    const int q = int(nearest - 4.0 * __builtin_floor(nearest * 0.25));
    const float a = q & 1 ? s : c, b = q & 1 ? c : s;
    return {(q == 1 || q == 2) ? -a : a, q >= 2 ? -b : b};
}

typedef uint32_t __attribute__((ext_vector_type(4))) Vec;      // eight channels

template <int DT>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi)
{
    if constexpr (DT == CODEC_DTYPE_FP16) {
        typedef _Float16 Two __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, Two{_Float16(lo), _Float16(hi)});
    } else {
        typedef __bf16 Two __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, Two{__bf16(lo), __bf16(hi)});
    }
}

// One of three values.  (They are arguments: written out where they are used, the choice is made between the places they are
// kept in, and each lane loads its own.)
template <class T>
__device__ __forceinline__ T one_of(bool first, bool second, T a, T b, T c) { return first ? a : second ? b : c; }

// Where a token's rows come from and go to: its queries, its keys, its values.
struct TokenRows {
    const char *q, *k, *v;
    char *q_out, *k_slot, *v_slot;
    int stored;                     // rows that go anywhere: without a slot the queries only

    __device__ __forceinline__ TokenRows(const RotaryParams &P, int64_t token)
    {
        q = P.q.data + token * P.q.token_stride;
        k = P.k.data + token * P.k.token_stride;
        v = P.v.data + token * P.v.token_stride;
        q_out = P.q_out.data + token * P.q_out.token_stride;
        k_slot = v_slot = nullptr;
        stored = P.q_heads;
        if (!P.kv_heads) return;
        const int64_t slot = P.slots[token];
        if (slot < 0 || slot >= P.num_slots) return;
        const int64_t at = (slot >> P.page_shift) * P.page_stride + (slot & ((int64_t(1) << P.page_shift) - 1)) * P.slot_stride;
        k_slot = P.k_pages + at;
        v_slot = P.v_pages + at;
        stored += 2 * P.kv_heads;
    }
    // Loads have no branches around them, so that the wait for one round's leaves the next round's under way: a row that goes
    // nowhere reads the last one that does.
    __device__ __forceinline__ const char *source(const RotaryParams &P, int row) const
    {
        row = row < stored ? row : stored - 1;
        const bool query = row < P.q_heads, key = row < P.q_heads + P.kv_heads;
        const int64_t stride = one_of(query, key, P.q.head_stride, P.k.head_stride, P.v.head_stride);
        return one_of(query, key, q, k, v) + (row - one_of(query, key, 0, P.q_heads, P.q_heads + P.kv_heads)) * stride;
    }
    __device__ __forceinline__ char *target(const RotaryParams &P, int row) const
    {
        const bool query = row < P.q_heads, key = row < P.q_heads + P.kv_heads;
        const int64_t stride = one_of(query, true, P.q_out.head_stride, P.head_stride, P.head_stride);
        return one_of(query, key, q_out, k_slot, v_slot) + (row - one_of(query, key, 0, P.q_heads, P.q_heads + P.kv_heads)) * stride;
    }
};

// A copy with some arithmetic on the way, bound by HBM.  A lane takes 16 bytes of a row and 16 others that the same cosines and
// sines serve: the other halves of its eight pairs, or, with neighbouring pairs, the same four pairs of another row, so that
// the lanes of a wave write consecutive memory.  It keeps the cosines and sines for all rows it takes: a wave takes
// 64 / U rows of one token at a time, U = head_dim / 16, `rounds` times in all; `splits` waves share a token.  The next
// round's loads are under way while a round is turned (two rounds at a time: 66 registers, seven waves a SIMD in the place of
// eight, a sixth slower for the 671 MB below).
// LARGE: with the streaming hint.  Out of HBM 16384 tokens of 64 + 8 + 8 heads of 128 channels take 122 us with it (5.5 TB/s) and
// 131 without, 2048 tokens of 32 + 8 + 8 heads 11.4 and 13.4, but 64 tokens 3.8 and 3.3, where the attention that follows finds
// its rows in the caches besides.
template <int DT, bool INTERLEAVED, int U, bool LARGE>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams P, uint32_t splits, uint32_t rounds)
{
    constexpr int kRows = 64 / U;
    constexpr int kLanes = INTERLEAVED ? 2 * U : U;     // of a row
    constexpr int kPairs = INTERLEAVED ? 4 : 8;         // of a lane
    constexpr int kOther = INTERLEAVED ? kRows / 2 : 0; // rows from a lane's first 16 bytes to its second
    const int lane = threadIdx.x & 63, unit = lane % kLanes, sub = lane / kLanes;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const uint32_t token = wave / splits, part = wave % splits;
    if (token >= P.num_tokens) return;

    const int turning = P.rotary_dim / 2;               // pairs
    const int pair = unit * kPairs;                     // the lane's first
    const bool turns = pair < turning;
    const int first = INTERLEAVED || turns ? unit * 8 : unit * 16;                                  // channels
    const int second = INTERLEAVED ? first : turns ? first + turning : first + 8;

    const TokenRows places(P, token);
    if (places.stored == 0) return;
    auto row_of = [&](uint32_t round, int other) { return int(round * kRows) + sub + other * kOther; };
    auto load_row = [&](int row, int channel) -> Vec {
        const Vec *at = reinterpret_cast<const Vec *>(places.source(P, row) + 2 * channel);
        if constexpr (LARGE) return __builtin_nontemporal_load(at);
        else return *at;
    };
    auto store_row = [&](int row, int channel, Vec x) {
        if (row >= places.stored) return;
        Vec *at = reinterpret_cast<Vec *>(places.target(P, row) + 2 * channel);
        if constexpr (LARGE) __builtin_nontemporal_store(x, at);
        else *at = x;
    };
    Vec a = load_row(row_of(part, 0), first), b = load_row(row_of(part, 1), second);

    float c[kPairs], s[kPairs];
    if (turning) {
        const double position = double(P.positions[token]);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const Turn t = turn_of(position * P.turns[INTERLEAVED ? (pair + i < turning ? pair + i : 0) : (turns ? pair : 0) + i]);
            c[i] = t.cos * P.magnitude;
            s[i] = t.sin * (P.magnitude * P.sign);
        }
    }
    auto turn_neighbours = [&](Vec &x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = widen<DT>(uint16_t(x[i])), hi = widen<DT>(uint16_t(x[i] >> 16));
            const uint32_t turned = narrow2<DT>(lo * c[i] - hi * s[i], hi * c[i] + lo * s[i]);
            x[i] = pair + i < turning ? turned : x[i];
        }
    };

    auto finish = [&](uint32_t round, Vec &x, Vec &y) {
        const int row = row_of(round, 0), other = row_of(round, 1), values = P.q_heads + P.kv_heads;
        if constexpr (INTERLEAVED) {
            if (turns && row < values) turn_neighbours(x);
            if (turns && other < values) turn_neighbours(y);
        } else if (turns && row < values) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int i = 2 * w;
                const float x0 = widen<DT>(uint16_t(x[w])), x1 = widen<DT>(uint16_t(x[w] >> 16));
                const float y0 = widen<DT>(uint16_t(y[w])), y1 = widen<DT>(uint16_t(y[w] >> 16));
                x[w] = narrow2<DT>(x0 * c[i] - y0 * s[i], x1 * c[i + 1] - y1 * s[i + 1]);
                y[w] = narrow2<DT>(y0 * c[i] + x0 * s[i], y1 * c[i + 1] + x1 * s[i + 1]);
            }
        }
        store_row(row, first, x);
        store_row(other, second, y);
    };
    // two sets of registers in turn: a copy from one to the other would wait for the loads, and for the stores behind them
    for (uint32_t round = part; round < rounds; round += 2 * splits) {
        Vec a_next = load_row(row_of(round + splits, 0), first), b_next = load_row(row_of(round + splits, 1), second);
        finish(round, a, b);
        if (round + splits >= rounds) break;
        a = load_row(row_of(round + 2 * splits, 0), first);
        b = load_row(row_of(round + 2 * splits, 1), second);
        finish(round + splits, a_next, b_next);
    }
}

// Halves whose pairs do not come in eights (rotary_dim no multiple of 16): a lane takes the eight channels of one piece of 16 bytes,
// as if neighbours were paired, and loads their other halves too, from before and behind, at any alignment.  All of a row's
// loads come before its stores, in one wave, which a call in place needs.  16384 tokens of 64 + 8 + 8 heads, 126 of 128 channels turning,
// take 155 us (4.3 TB/s) where the other kernel takes 122 for 128: three loads for a store, two of them at any alignment.
template <int DT, int U>
__global__ __launch_bounds__(256) void rotary_uneven_kernel(RotaryParams P, uint32_t splits, uint32_t rounds)
{
    constexpr int kLanes = 2 * U, kRows = 64 / U, kOther = kRows / 2;
    const int lane = threadIdx.x & 63, channel = lane % kLanes * 8, sub = lane / kLanes;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const uint32_t token = wave / splits, part = wave % splits;
    if (token >= P.num_tokens) return;
    const TokenRows places(P, token);
    if (places.stored == 0) return;

    typedef uint32_t __attribute__((ext_vector_type(4), aligned(2))) AnyPiece;
    const int half = P.rotary_dim / 2, d = P.head_dim;
    // other halves of channels below `half`, from channel + half on; of those above, from channel - half on.  A piece that would
    // reach over the row's end or begin starts at the nearest place that does not, and is shifted.
    const bool low = channel < half, high = channel + 7 >= half && channel < P.rotary_dim;
    const int behind = low ? (channel + half < d - 8 ? channel + half : d - 8) : 0, behind_by = low ? channel + half - behind : 0;
    const int before = high && channel > half ? channel - half : 0, before_by = high && channel < half ? half - channel : 0;
    float c[8], s[8];
    const double position = double(P.positions[token]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int x = channel + e;
        const Turn t = turn_of(position * P.turns[x < half ? x : x < P.rotary_dim ? x - half : 0]);
        c[e] = t.cos * P.magnitude;
        s[e] = t.sin * (x < half ? -P.magnitude * P.sign : P.magnitude * P.sign);
    }
    for (uint32_t round = part; round < rounds; round += splits) {
        Vec own[2], a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const char *from = places.source(P, int(round * kRows) + sub + i * kOther);
            own[i] = *reinterpret_cast<const Vec *>(from + 2 * channel);
            a[i] = *reinterpret_cast<const AnyPiece *>(from + 2 * behind);
            b[i] = *reinterpret_cast<const AnyPiece *>(from + 2 * before);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = int(round * kRows) + sub + i * kOther;
            if (row >= places.stored) continue;
            Vec out = own[i];
            if (row < P.q_heads + P.kv_heads) {
                typedef unsigned __int128 Bits;
                const Vec lows = __builtin_bit_cast(Vec, __builtin_bit_cast(Bits, a[i]) >> (16 * behind_by));
                const Vec highs = __builtin_bit_cast(Vec, __builtin_bit_cast(Bits, b[i]) << (16 * before_by));
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t turned[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int e = 2 * w + j, x = channel + e;
                        const uint16_t mine = uint16_t(own[i][w] >> (16 * j)), other = uint16_t((x < half ? lows[w] : highs[w]) >> (16 * j));
                        const uint16_t y = narrow<DT>(widen<DT>(mine) * c[e] + widen<DT>(other) * s[e]);
                        turned[j] = x < P.rotary_dim ? y : mine;
                    }
                    out[w] = turned[0] | turned[1] << 16;
                }
            }
            *reinterpret_cast<Vec *>(places.target(P, row) + 2 * channel) = out;
        }
    }
}

}  // namespace

namespace {

int launch_slice(const RotaryParams &p, int dtype, bool interleaved, hipStream_t s)
{
    const int64_t rows = p.q_heads + 2 * p.kv_heads;
    // a wave for every token, or as many as it takes to have 32 on every CU
    const int64_t at_once = 64 / (p.head_dim / 16), rounds = (rows + at_once - 1) / at_once;
    int64_t splits = (8192 + p.num_tokens - 1) / p.num_tokens;
    if (splits > rounds) splits = rounds;
    const dim3 grid(unsigned((p.num_tokens * splits + 3) / 4));
    const bool large = 4.0 * double(p.num_tokens) * double(rows) * p.head_dim > kLargeBytes;
    const bool uneven = !interleaved && p.rotary_dim % 16;
    const uint32_t n = uint32_t(splits), r = uint32_t(rounds);
    auto launch_dim = [&](auto dt, auto u) {
        constexpr int DT = decltype(dt)::value, U = decltype(u)::value;
        if (uneven)                    hipLaunchKernelGGL((rotary_uneven_kernel<DT, U>), grid, dim3(256), 0, s, p, n, r);
        else if (interleaved && large) hipLaunchKernelGGL((rotary_kernel<DT, true, U, true>), grid, dim3(256), 0, s, p, n, r);
        else if (interleaved)          hipLaunchKernelGGL((rotary_kernel<DT, true, U, false>), grid, dim3(256), 0, s, p, n, r);
        else if (large)                hipLaunchKernelGGL((rotary_kernel<DT, false, U, true>), grid, dim3(256), 0, s, p, n, r);
        else                           hipLaunchKernelGGL((rotary_kernel<DT, false, U, false>), grid, dim3(256), 0, s, p, n, r);
    };
    auto launch = [&](auto dt) {
        if (p.head_dim == 64)       launch_dim(dt, std::integral_constant<int, 4>{});
        else if (p.head_dim == 128) launch_dim(dt, std::integral_constant<int, 8>{});
        else                        launch_dim(dt, std::integral_constant<int, 16>{});
    };
    if (dtype == CODEC_DTYPE_FP16) launch(std::integral_constant<int, CODEC_DTYPE_FP16>{});
    else                           launch(std::integral_constant<int, CODEC_DTYPE_BF16>{});
    return int(hipGetLastError());
}

}  // namespace

// A launch takes 2^24 tokens: its threads are counted in 32 bits.
int launch_rotary(const RotaryParams &p, int dtype, bool interleaved, void *stream)
{
    constexpr int64_t kSlice = int64_t(1) << 24;
    for (int64_t at = 0; at < p.num_tokens; at += kSlice) {
        RotaryParams part = p;
        part.num_tokens = p.num_tokens - at < kSlice ? p.num_tokens - at : kSlice;
        for (RowsView *r : {&part.q, &part.q_out, &part.k, &part.v})
            if (r->data) r->data += at * r->token_stride;
        if (p.positions) part.positions = p.positions + at;
        if (p.slots) part.slots = p.slots + at;
        if (int e = launch_slice(part, dtype, interleaved, static_cast<hipStream_t>(stream))) return e;
    }
    return 0;
}

}  // namespace codec
