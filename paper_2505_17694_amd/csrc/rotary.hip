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

// A copy with some arithmetic on the way, bound by HBM.  A lane takes 16 bytes of a row and 16 others that the same cosines and
// sines serve: the other halves of its eight pairs, or, with neighbouring pairs, the same four pairs of another row, so that
// the lanes of a wave write consecutive memory.  It keeps the cosines and sines for all rows it takes: a wave takes
// 64 / U rows of one token at a time, U = head_dim / 16, `rounds` times in all; `splits` waves share a token.  The next
// round's loads are under way while a round is turned (two rounds at a time: 66 registers, seven waves a SIMD in the place of
// eight, 150 us in the place of 129 for the 671 MB below).
// LARGE: with the streaming hint.  16384 tokens of 64 + 8 + 8 heads of 128 channels take 129 us with it (5.2 TB/s) and 143
// without, 64 tokens of 32 + 8 + 8 heads 4.2 and 3.7, where the attention that follows finds its rows in the caches besides.
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

    const char *q = P.q.data + int64_t(token) * P.q.token_stride, *k = P.k.data + int64_t(token) * P.k.token_stride,
               *v = P.v.data + int64_t(token) * P.v.token_stride;
    char *q_out = P.q_out.data + int64_t(token) * P.q_out.token_stride;
    const int rows = P.q_heads + 2 * P.kv_heads;
    char *k_slot = nullptr, *v_slot = nullptr;
    if (P.kv_heads) {
        const int64_t slot = P.slots[token];
        if (slot >= 0 && slot < P.num_slots) {
            const int64_t at = (slot >> P.page_shift) * P.page_stride + (slot & ((int64_t(1) << P.page_shift) - 1)) * P.slot_stride;
            k_slot = P.k_pages + at;
            v_slot = P.v_pages + at;
        }
    }
    const int stored = k_slot ? rows : P.q_heads;       // rows that go anywhere
    if (stored == 0) return;
    auto row_of = [&](uint32_t round, int other) { return int(round * kRows) + sub + other * kOther; };
    // Loads have no branches around them, so that the wait for one round's leaves the next round's under way: a row that goes
    // nowhere reads the last one that does.
    auto load_row = [&](int row, int channel) -> Vec {
        row = row < stored ? row : stored - 1;
        const bool query = row < P.q_heads, key = row < P.q_heads + P.kv_heads;
        const char *base = one_of(query, key, q, k, v);
        const int64_t stride = one_of(query, key, P.q.head_stride, P.k.head_stride, P.v.head_stride);
        const int head = row - one_of(query, key, 0, P.q_heads, P.q_heads + P.kv_heads);
        const Vec *at = reinterpret_cast<const Vec *>(base + head * stride + 2 * channel);
        if constexpr (LARGE) return __builtin_nontemporal_load(at);
        else return *at;
    };
    auto store_row = [&](int row, int channel, Vec x) {
        const bool query = row < P.q_heads, key = row < P.q_heads + P.kv_heads;
        char *base = one_of(query, key, q_out, k_slot, v_slot);
        const int64_t stride = one_of(query, true, P.q_out.head_stride, P.head_stride, P.head_stride);
        const int head = row - one_of(query, key, 0, P.q_heads, P.q_heads + P.kv_heads);
        Vec *at = reinterpret_cast<Vec *>(base + head * stride + 2 * channel);
        if (row >= stored) return;
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

// Halves whose pairs do not come in eights: one thread per pair of channels of a row, the pairs that turn first, then the
// others two by two.  Rows of a token: its queries, its keys, its values.
template <int DT>
__global__ __launch_bounds__(256) void rotary_pair_kernel(RotaryParams P)
{
    const int pairs = P.head_dim / 2, turning = P.rotary_dim / 2;
    const int rows = P.q_heads + 2 * P.kv_heads;
    const int64_t total = P.num_tokens * rows * pairs;
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < total; at += int64_t(gridDim.x) * 256) {
        const int pair = int(at % pairs);
        const int64_t token_row = at / pairs;
        const int row = int(token_row % rows);
        const int64_t token = token_row / rows;
        const bool query = row < P.q_heads, value = row >= P.q_heads + P.kv_heads;
        const int head = query ? row : value ? row - P.q_heads - P.kv_heads : row - P.q_heads;
        const RowsView &in = query ? P.q : value ? P.v : P.k;
        const uint16_t *from = reinterpret_cast<const uint16_t *>(in.data + token * in.token_stride + head * in.head_stride);
        uint16_t *to;
        if (query) {
            to = reinterpret_cast<uint16_t *>(P.q_out.data + token * P.q_out.token_stride + head * P.q_out.head_stride);
        } else {
            const int64_t slot = P.slots[token];
            if (slot < 0 || slot >= P.num_slots) continue;
            const int64_t page = slot >> P.page_shift, in_page = slot & ((int64_t(1) << P.page_shift) - 1);
            to = reinterpret_cast<uint16_t *>((value ? P.v_pages : P.k_pages) + page * P.page_stride + in_page * P.slot_stride + head * P.head_stride);
        }
        const bool turns = !value && pair < turning;
        const int first = turns ? pair : value ? 2 * pair : P.rotary_dim + 2 * (pair - turning);
        const int second = turns ? first + turning : first + 1;
        uint16_t a = from[first], b = from[second];
        if (turns) {
            const Turn t = turn_of(double(P.positions[token]) * P.turns[pair]);
            const float c = t.cos * P.magnitude, s = t.sin * (P.magnitude * P.sign);
            const float x = widen<DT>(a), y = widen<DT>(b);
            a = narrow<DT>(x * c - y * s);
            b = narrow<DT>(y * c + x * s);
        }
        to[first] = a;
        to[second] = b;
    }
}

}  // namespace

int launch_rotary(const RotaryParams &p, int dtype, bool interleaved, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t rows = p.q_heads + 2 * p.kv_heads;
    // pairs of halves are taken eight at a time: 16 channels that turn, or a multiple of them
    if (!interleaved && p.rotary_dim % 16) {
        const int64_t blocks = (p.num_tokens * rows * (p.head_dim / 2) + 255) / 256;
        const dim3 grid(unsigned(blocks < (int64_t(1) << 22) ? blocks : int64_t(1) << 22));
        if (dtype == CODEC_DTYPE_FP16) hipLaunchKernelGGL(rotary_pair_kernel<CODEC_DTYPE_FP16>, grid, dim3(256), 0, s, p);
        else                           hipLaunchKernelGGL(rotary_pair_kernel<CODEC_DTYPE_BF16>, grid, dim3(256), 0, s, p);
        return int(hipGetLastError());
    }
    // a wave for every token, or as many as it takes to have 32 on every CU
    const int64_t at_once = 64 / (p.head_dim / 16), rounds = (rows + at_once - 1) / at_once;
    int64_t splits = (8192 + p.num_tokens - 1) / p.num_tokens;
    if (splits > rounds) splits = rounds;
    const dim3 grid(unsigned((p.num_tokens * splits + 3) / 4));
    const bool large = 4.0 * double(p.num_tokens) * double(rows) * p.head_dim > kLargeBytes;
    const uint32_t n = uint32_t(splits), r = uint32_t(rounds);
    auto launch_dim = [&](auto dt, auto layout, auto u) {
        constexpr int DT = decltype(dt)::value, U = decltype(u)::value;
        constexpr bool I = decltype(layout)::value;
        if (large) hipLaunchKernelGGL((rotary_kernel<DT, I, U, true>), grid, dim3(256), 0, s, p, n, r);
        else       hipLaunchKernelGGL((rotary_kernel<DT, I, U, false>), grid, dim3(256), 0, s, p, n, r);
    };
    auto launch = [&](auto dt, auto layout) {
        if (p.head_dim == 64)       launch_dim(dt, layout, std::integral_constant<int, 4>{});
        else if (p.head_dim == 128) launch_dim(dt, layout, std::integral_constant<int, 8>{});
        else                        launch_dim(dt, layout, std::integral_constant<int, 16>{});
    };
    using f16 = std::integral_constant<int, CODEC_DTYPE_FP16>;
    using b16 = std::integral_constant<int, CODEC_DTYPE_BF16>;
    if (dtype == CODEC_DTYPE_FP16) interleaved ? launch(f16{}, std::true_type{}) : launch(f16{}, std::false_type{});
    else                           interleaved ? launch(b16{}, std::true_type{}) : launch(b16{}, std::false_type{});
    return int(hipGetLastError());
}

}  // namespace codec
