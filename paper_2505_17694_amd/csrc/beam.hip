// Beam search: the best continuations over beams and vocabulary, and the states of the beams that go on.
//
// Continuing a beam of score c with token t scores c + (x_t - m) - log S, with m the largest logit of the beam and
// S = sum_u exp(x_u - m).  Inside a beam the order is that of the logits, so a beam brings at most its k best tokens; which
// of those the search keeps is decided between the beams, on scores in 64 bits.
#include <hip/hip_runtime.h>

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
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return uint64_t(b ^ (b >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - token);
}
__device__ __forceinline__ uint32_t token_of(uint64_t key) { return 0xffffffffu - uint32_t(key); }
__device__ __forceinline__ float logit_of(uint64_t key)
{
    const uint32_t b = uint32_t(key >> 32);
    return __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b);
}

// exp(d) for d <= 0 (or d = -inf).  2^y alone would be off by half a step of y = d log2 e, 3e-7 at d = -10, and equally so for
// every logit of that value: y's whole part is split off first, its fraction taken with 1 / ln 2 in two pieces.
__device__ __forceinline__ float exp_below(float d)
{
    const float whole = __builtin_rintf(d * 1.44269504f);
    const float part = __builtin_fmaf(d, 1.92596303e-8f, __builtin_fmaf(d, 1.44269502f, -whole));
    return d < -200.f ? 0.f : __builtin_ldexpf(__builtin_amdgcn_exp2f(part), int(whole));
}

// A beam whose logits do not count: finished, or of score -inf (NaN and +inf are taken for that).
__device__ __forceinline__ bool score_counts(float s) { return s > kMinusInf && s < __builtin_inff(); }
__device__ __forceinline__ bool reads_logits(const BeamParams &P, int row)
{
    return score_counts(P.scores[row]) && !(P.finished && P.finished[row]);
}

template <class T, class Combine>
__device__ __forceinline__ T block_reduce(T v, T *lds, Combine combine)
{
    __syncthreads();
    lds[threadIdx.x] = v;
    for (int n = blockDim.x / 2; n; n /= 2) {
        __syncthreads();
        if (int(threadIdx.x) < n) lds[threadIdx.x] = combine(lds[threadIdx.x], lds[threadIdx.x + n]);
    }
    __syncthreads();
    return lds[0];
}

// A workgroup per beam: largest logit, sum, then one best token after the other.
template <int DT>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamParams P)
{
    __shared__ uint64_t keys[256];
    __shared__ double sums[256];
    const int row = blockIdx.x;
    if (!reads_logits(P, row)) return;
    constexpr int kSize = DT == CODEC_DTYPE_FP32 ? 4 : 2;
    const char *x = P.logits + (row / P.beams * P.batch_stride + row % P.beams * P.beam_stride) * kSize;
    uint64_t last = ~uint64_t(0);
    for (int i = 0; i < P.kept; ++i) {
        uint64_t best = 0;
        for (int t = threadIdx.x; t < P.vocab; t += 256) {
            const uint64_t key = key_of(logit_at<DT>(x, t), t);
            if (key < last && key > best) best = key;
        }
        last = block_reduce(best, keys, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        if (threadIdx.x == 0) P.best[int64_t(row) * P.kept + i] = last;
        if (i == 0) {
            const float top = logit_of(last);
            double sum = 0.0;
            for (int t = threadIdx.x; t < P.vocab && top > kMinusInf; t += 256) sum += double(exp_below(logit_at<DT>(x, t) - top));
            sum = block_reduce(sum, sums, [](double a, double b) { return a + b; });
            if (threadIdx.x == 0) {
                P.sums[row] = sum;
                P.tops[row] = top;
            }
        }
    }
}

struct Candidate { double score; int32_t beam, token; };

__device__ __forceinline__ bool before(const Candidate &a, const Candidate &b)
{
    return a.score != b.score ? a.score > b.score : a.beam != b.beam ? a.beam < b.beam : a.token < b.token;
}

// The i-th best continuation of a beam, i < kept.
__device__ __forceinline__ Candidate candidate(const BeamParams &P, int search, int beam, int i)
{
    const int row = search * P.beams + beam;
    const double ruled_out = -__builtin_inf();
    const float score = P.scores[row];
    if (!score_counts(score)) return {ruled_out, beam, i};
    if (P.finished && P.finished[row]) {
        if (i == 0) return {double(score), beam, P.eos};
        return {ruled_out, beam, i - 1 < P.eos ? i - 1 : i};
    }
    const uint64_t key = P.best[int64_t(row) * P.kept + i];
    const float x = logit_of(key);
    const int32_t token = int32_t(token_of(key));
    if (x == kMinusInf) return {ruled_out, beam, token};
    return {double(score) + ((double(x) - double(P.tops[row])) - log(P.sums[row])), beam, token};
}

// A wave per search: k times the best of what is left.
__global__ __launch_bounds__(64) void beam_merge_kernel(BeamParams P)
{
    const int search = blockIdx.x;
    Candidate last{__builtin_inf(), -1, -1};
    for (int i = 0; i < P.k; ++i) {
        Candidate best{-__builtin_inf(), 1 << 30, 0};
        for (int at = threadIdx.x; at < P.beams * P.kept; at += 64) {
            const Candidate c = candidate(P, search, at / P.kept, at % P.kept);
            if (before(last, c) && before(c, best)) best = c;
        }
        for (int n = 32; n; n /= 2) {
            const Candidate c{__shfl_xor(best.score, n), __shfl_xor(best.beam, n), __shfl_xor(best.token, n)};
            if (before(c, best)) best = c;
        }
        last = best;
        if (threadIdx.x == 0) {
            P.out_scores[int64_t(search) * P.k + i] = float(best.score);
            P.out_beams[int64_t(search) * P.k + i] = best.beam;
            P.out_tokens[int64_t(search) * P.k + i] = best.token;
        }
    }
}

// A thread per unit of a state's row.
template <class Unit>
__global__ __launch_bounds__(256) void reorder_kernel(ReorderParams P)
{
    const ReorderState &state = P.states[blockIdx.z];
    const int row = blockIdx.x;
    const int beam = P.beams[row];
    if (beam < 0 || beam >= P.beams_in) return;
    const int64_t search = row / P.beams_out, to = row % P.beams_out;
    const Unit *src = reinterpret_cast<const Unit *>(state.src + search * state.src_batch + beam * state.src_beam);
    Unit *dst = reinterpret_cast<Unit *>(state.dst + search * state.dst_batch + to * state.dst_beam);
    for (int64_t i = int64_t(blockIdx.y) * 256 + threadIdx.x; i < state.row_units; i += int64_t(gridDim.y) * 256) dst[i] = src[i];
}

}  // namespace

int launch_beam_select(const BeamParams &p, int dtype, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 rows(unsigned(p.batch) * unsigned(p.beams));
    switch (dtype) {
    case CODEC_DTYPE_FP16: hipLaunchKernelGGL(beam_rows_kernel<CODEC_DTYPE_FP16>, rows, dim3(256), 0, s, p); break;
    case CODEC_DTYPE_BF16: hipLaunchKernelGGL(beam_rows_kernel<CODEC_DTYPE_BF16>, rows, dim3(256), 0, s, p); break;
    default: hipLaunchKernelGGL(beam_rows_kernel<CODEC_DTYPE_FP32>, rows, dim3(256), 0, s, p); break;
    }
    if (hipError_t e = hipGetLastError()) return int(e);
    hipLaunchKernelGGL(beam_merge_kernel, dim3(unsigned(p.batch)), dim3(64), 0, s, p);
    return int(hipGetLastError());
}

int launch_reorder(const ReorderParams &p, int unit, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t pieces = (p.most_units + 255) / 256;
    const dim3 grid(unsigned(p.batch) * unsigned(p.beams_out), unsigned(pieces < 1024 ? pieces : 1024), unsigned(p.num_states));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p); };
    switch (unit) {
    case 16: launch(reorder_kernel<uint4>); break;
    case 8: launch(reorder_kernel<uint2>); break;
    case 4: launch(reorder_kernel<uint32_t>); break;
    case 2: launch(reorder_kernel<uint16_t>); break;
    case 1: launch(reorder_kernel<uint8_t>); break;
    default: return int(hipErrorInvalidValue);
    }
    return int(hipGetLastError());
}

}  // namespace codec
