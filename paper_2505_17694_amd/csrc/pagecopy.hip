// Copies of token runs between the pages of a cache, in the K and V pools of all layers.
//
// Nothing is computed: the copy reads and writes every byte once and is bound by HBM.  The list of runs and the pools'
// addresses travel in the kernel's arguments (scalar loads).
#include <hip/hip_runtime.h>

#include "operators.hpp"

namespace codec {
namespace {

// A workgroup copies 256 pieces of 16 bytes of one run in one pool.
__global__ __launch_bounds__(256) void page_copy_kernel(CopyParams P)
{
    const CopyRun run = P.runs[blockIdx.y];
    char *pool = P.pools[blockIdx.z];
    const int pieces = P.head_bytes / 16, tokens = run.tokens;          // of a head's channels
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= int64_t(pieces) * tokens * P.heads) return;
    const int piece = int(i % pieces), row = int(i / pieces);
    const int token = row % tokens, head = row / tokens;
    const int64_t in_page = head * P.head_stride + piece * 16;
    const char *from = pool + run.src_page * P.page_stride + (run.src_token + token) * P.slot_stride + in_page;
    char *to = pool + run.dst_page * P.page_stride + (run.dst_token + token) * P.slot_stride + in_page;
    *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
}

}  // namespace

int launch_copy(const CopyParams &p, void *stream)
{
    const int64_t pieces = int64_t(p.head_bytes / 16) * p.most_tokens * p.heads;
    const dim3 grid(unsigned((pieces + 255) / 256), unsigned(p.num_runs), unsigned(p.num_pools));
    hipLaunchKernelGGL(page_copy_kernel, grid, dim3(256), 0, static_cast<hipStream_t>(stream), p);
    return int(hipGetLastError());
}

}  // namespace codec
