// Differential attention: out = norm(o_1 - lambda o_2), o_m = softmax(scale q_m K_m^T) V.
//
// A KV head of the pools is [K_1 | K_2], two maps' keys of d channels each, beside V of 2d.  With the query of map m in its half of
// a row of 2d channels and zeros in the other, scale q_m K_m^T is an ordinary score of that head, exactly: what the zeros
// multiply adds nothing.  So the attention kernels run as they are, on a plan with two query heads for every head of the result,
// and K_1, K_2 and V are read once for both maps.  The products with zeros cost nothing where a tile holds at most sixteen rows
// (its rows are of both maps, and the tile is as wide as it is); dense tasks do a third more matrix work than they have to.
#include "kernels.hpp"

namespace codec {
namespace {

// Query rows [request][head][map][d] to rows of 2d channels, 16 bytes a thread.
__global__ __launch_bounds__(256) void spread_queries_kernel(const u32x4 *q, u32x4 *rows, int64_t units, int half)
{
    const int64_t unit = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (unit >= units) return;
    const int64_t row = unit / (2 * half);
    const int at = int(unit - row * (2 * half)), map = int(row & 1), channel = at - map * half;
    rows[unit] = channel >= 0 && channel < half ? q[row * half + channel] : u32x4{0u, 0u, 0u, 0u};
}

// The two rows of a head in a wave: row `row` (the map) in 32 lanes, whose channels are 128 * (c / 4) + 4 * lane + c % 4 (64
// channels: 2 * lane + c).
template <int D>
struct PairRows {
    static constexpr int CPL = D / 32, PIECE = CPL < 4 ? CPL : 4;
    int lane, row;
    int64_t first;                              // row of the head's partials behind an entry of the list

    __device__ __forceinline__ PairRows(const MergeParams &P, int head, int hj)
    {
        lane = threadIdx.x & 31;
        row = (threadIdx.x >> 5) & 1;
        first = int64_t(head) * P.part_rows + hj + row;
    }
    __device__ __forceinline__ void load(const MergeParams &P, int entry, float2 &ml, float (&o)[CPL]) const
    {
        const int64_t prow = first + entry;
        ml = *reinterpret_cast<const float2 *>(P.part_ml + prow * 2);
        const float *src = P.part_o + prow * D + lane * PIECE;
#pragma unroll
        for (int u = 0; u < CPL / PIECE; ++u) {
            if constexpr (PIECE == 2) {
                const float2 x = *reinterpret_cast<const float2 *>(src);
                o[0] = x.x;
                o[1] = x.y;
            } else {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(src + u * 128);
#pragma unroll
                for (int c = 0; c < 4; ++c) o[u * 4 + c] = x[c];
            }
        }
    }
};

// Weight of channel `channel` of the norm
__device__ __forceinline__ float norm_weight(const DifferentialParams &P, int channel)
{
    if (P.weight_dtype == CODEC_DTYPE_FP32) return static_cast<const float *>(P.weight)[channel];
    const uint16_t bits = static_cast<const uint16_t *>(P.weight)[channel];
    return P.weight_dtype == CODEC_DTYPE_FP16 ? float(__builtin_bit_cast(_Float16, bits)) : __uint_as_float(uint32_t(bits) << 16);
}

// Both rows of a head, unnormalised, to its result.
template <int DT, int D>
__device__ __forceinline__ void finish_pair(const DifferentialParams &P, const PairRows<D> &at, int r, int h, float l, float (&o)[PairRows<D>::CPL])
{
    constexpr int CPL = PairRows<D>::CPL, PIECE = PairRows<D>::PIECE;
    const float inv = 1.f / l, lambda = P.lambda[r * P.lambda_request_stride + h * P.lambda_head_stride];
    float x[CPL], squares = 0.f;
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
        const float mine = o[c] * inv, other = __shfl_xor(mine, 32);
        x[c] = __builtin_fmaf(-lambda, at.row ? mine : other, at.row ? other : mine);
        squares = __builtin_fmaf(x[c], x[c], squares);
    }
    float factor = P.gain;
    if (P.norm) {
#pragma unroll
        for (int d = 1; d < 32; d *= 2) squares += __shfl_xor(squares, d);
        factor = P.gain / __builtin_sqrtf(squares * (1.f / D) + P.eps);
    }
    if (at.row) return;
    char *out = static_cast<char *>(P.merge.out) + ((int64_t(r) * (P.merge.h_q / 2) + h) * D + at.lane * PIECE) * 2;
#pragma unroll
    for (int u = 0; u < CPL / PIECE; ++u) {
        float y[PIECE];
#pragma unroll
        for (int c = 0; c < PIECE; ++c) {
            y[c] = x[u * PIECE + c] * factor;
            if (P.weight) y[c] *= norm_weight(P, u * 128 + at.lane * PIECE + c);
        }
#pragma unroll
        for (int c = 0; c < PIECE; c += 2) *reinterpret_cast<unsigned int *>(out + u * 256 + c * 2) = pack2<DT>(y[c], y[c + 1]);
    }
}

// The reduction (Alg. 3) of both rows of a head and what becomes of them.  W = 1: a wave a head, two in a workgroup; W > 1: a list
// shared by W waves, whose sums meet in LDS.  Grid as in merge_kernel: blockIdx.x is the KV head.
template <int DT, int D, int W>
__global__ void __launch_bounds__((W == 1 ? kMergeWaves : W) * 64) differential_reduction_kernel(const DifferentialParams P)
{
    constexpr int CPL = PairRows<D>::CPL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave_lane = threadIdx.x & 63;
    const int heads = P.merge.group / 2;
    int unit = blockIdx.z * gridDim.y + blockIdx.y;
    if constexpr (W == 1) unit = unit * kMergeWaves + wave;
    if (unit >= P.merge.num_requests * heads) return;
    const int r = unit / heads, member = unit - r * heads;
    const PairRows<D> at(P.merge, blockIdx.x, 2 * member);
    const int32_t *line = W == 1 ? P.merge.req_inline + int64_t(r) * (kInlineParts + 1) : P.merge.req_line + int64_t(r) * split_line_words(W);
    constexpr int kInLine = W == 1 ? kInlineParts : split_rows(W);
    const int total = line[0];
    const int32_t *list = total <= kInLine ? line + 1 : P.merge.req_part + P.merge.req_part_off[r];

    float M = -INFINITY, L = 0.f, acc[CPL];
#pragma unroll
    for (int c = 0; c < CPL; ++c) acc[c] = 0.f;
#pragma unroll 1
    for (int base = (W == 1 ? 0 : wave) * kFoldChunk; base < total; base += W * kFoldChunk) {
        const int cnt = total - base < kFoldChunk ? total - base : kFoldChunk;
        int rows[kFoldChunk];
#pragma unroll
        for (int j = 0; j < kFoldChunk; ++j) rows[j] = list[base + (j < cnt ? j : 0)];
        Chunk<kFoldChunk, CPL> x;
        x.load(P.merge, at, rows, cnt);
        const float mm = x.top(M, cnt);
        float l, sum[CPL];
        x.sum_up(cnt, mm, l, sum);
        add_chunk(M, L, acc, mm, l, sum);
        M = mm;
    }
    if constexpr (W > 1) {
        __shared__ float sums[W - 1][CPL + 2][64];
        if (wave > 0) {
            float (*put)[64] = sums[wave - 1];
            put[CPL][wave_lane] = L;
            put[CPL + 1][wave_lane] = M;
#pragma unroll
            for (int c = 0; c < CPL; ++c) put[c][wave_lane] = acc[c];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < W - 1; ++w) {
            const float m = sums[w][CPL + 1][wave_lane], mm = fmaxf(M, m), theirs = weight(m, mm);
            float sum[CPL];
#pragma unroll
            for (int c = 0; c < CPL; ++c) sum[c] = sums[w][c][wave_lane] * theirs;
            add_chunk(M, L, acc, mm, sums[w][CPL][wave_lane] * theirs, sum);
            M = mm;
        }
    }
    finish_pair<DT, D>(P, at, r, blockIdx.x * heads + member, L, acc);
}

template <int DT, int D>
int launch_differential_of(const DifferentialParams &p, hipStream_t s)
{
    const int64_t units = int64_t(p.merge.num_requests) * (p.merge.group / 2);
    constexpr int64_t kMaxY = 32768;
    auto launch = [&](auto kernel, int units_of, int waves) {
        const int64_t groups = (units + units_of - 1) / units_of, y = groups < kMaxY ? groups : kMaxY;
        const dim3 grid(unsigned(p.merge.h_q / p.merge.group), unsigned(y), unsigned((groups + y - 1) / y)), block(waves * 64);
        hipLaunchKernelGGL(kernel, grid, block, 0, s, p);
    };
    if (p.merge.split_waves == 8)      launch(differential_reduction_kernel<DT, D, 8>, 1, 8);
    else if (p.merge.split_waves == 4) launch(differential_reduction_kernel<DT, D, 4>, 1, 4);
    else                               launch(differential_reduction_kernel<DT, D, 1>, kMergeWaves, kMergeWaves);
    return int(hipGetLastError());
}

}  // namespace

int launch_spread_queries(const void *q, void *rows, int64_t num_rows, int head_dim, void *stream)
{
    const int half = head_dim / 16;                     // 16-byte pieces of a map's row
    const int64_t units = num_rows * 2 * half;
    hipLaunchKernelGGL(spread_queries_kernel, dim3(unsigned((units + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<const u32x4 *>(q), static_cast<u32x4 *>(rows), units, half);
    return int(hipGetLastError());
}

int launch_differential(const DifferentialParams &p, int dtype, int head_dim, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool half = dtype == CODEC_DTYPE_FP16;
    if (head_dim == 64)  return half ? launch_differential_of<CODEC_DTYPE_FP16, 64>(p, s) : launch_differential_of<CODEC_DTYPE_BF16, 64>(p, s);
    if (head_dim == 128) return half ? launch_differential_of<CODEC_DTYPE_FP16, 128>(p, s) : launch_differential_of<CODEC_DTYPE_BF16, 128>(p, s);
    if (head_dim == 256) return half ? launch_differential_of<CODEC_DTYPE_FP16, 256>(p, s) : launch_differential_of<CODEC_DTYPE_BF16, 256>(p, s);
    return int(hipErrorInvalidValue);
}

}  // namespace codec
