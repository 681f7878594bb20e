// Rotary positions of new tokens' queries and keys, and their keys and values into the pages of the cache.
//
// A head's channels form pairs: (i, i + r/2) or (2i, 2i + 1) for i < r/2, r the number of channels that turn.  At
// position n pair i turns by n * t_i whole turns: (a, b) -> m (a cos - b sin, b cos + a sin).  Only the fraction of
// n * t_i counts; at position 10^6 it is what 20 bits of the product leave, so the product is taken in 64 bits and
// reduced to an eighth of a turn around the next quarter before the series of sine and cosine run in 32.
#include <hip/hip_runtime.h>

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

// One thread per pair of channels of a row: the pairs that turn first, then the others two by two.  Rows of a token:
// its queries, its keys, its values.
template <int DT, bool INTERLEAVED>
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
        const int first = turns ? (INTERLEAVED ? 2 * pair : pair) : value ? 2 * pair : P.rotary_dim + 2 * (pair - turning);
        const int second = turns && !INTERLEAVED ? first + turning : first + 1;
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
    const int64_t pairs = p.num_tokens * (p.q_heads + 2 * p.kv_heads) * (p.head_dim / 2);
    const int64_t blocks = (pairs + 255) / 256;
    const dim3 grid(unsigned(blocks < (int64_t(1) << 22) ? blocks : int64_t(1) << 22));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p); };
    if (dtype == CODEC_DTYPE_FP16) interleaved ? launch(rotary_pair_kernel<CODEC_DTYPE_FP16, true>) : launch(rotary_pair_kernel<CODEC_DTYPE_FP16, false>);
    else                           interleaved ? launch(rotary_pair_kernel<CODEC_DTYPE_BF16, true>) : launch(rotary_pair_kernel<CODEC_DTYPE_BF16, false>);
    return int(hipGetLastError());
}

}  // namespace codec
