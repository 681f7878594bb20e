// Copies of token runs between the pages of a cache, in the K and V pools of all layers.
//
// Nothing is computed: the copy reads and writes every byte once and is bound by HBM.  The list of runs and the pools'
// addresses travel in the kernel's arguments (scalar loads).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "operators.hpp"

namespace codec {
namespace {

typedef uint32_t __attribute__((ext_vector_type(4))) Piece;

// A workgroup copies PIECES * 256 pieces of 16 bytes of one run in one pool, PIECES of a lane in flight.  The run is rows of
// consecutive memory, `row_pieces` long: with tokens side by side a head's, with heads side by side a token's, else a token's in
// one head (a plane each).  A lane finds its first piece by a division and the others by steps of 256.
// Bound by HBM: 1000 pages of 8 x 128 channels in 8 layers (1.05 GB read and written) take 198 us, 5.3 TB/s; a plain copy of 1 GiB
// reaches 5.15.  STORES_ONCE, LOADS_ONCE: with the streaming hint; without either 222 us, with that on the stores 207.  What
// may lie in the last-level cache is loaded without: the last pages of 192 sequences in 16 layers (207 MB) take 32 us where the cache
// has them and 45 with the hint, out of HBM 51 (4.1 TB/s) and 49.  PIECES 8 and 2: those pages 32 and 38 us, out of HBM 51 and 49;
// 96 pages out of runs of one to five tokens of 8 x 64 channels in 8 layers (two launches) 18.6 and 13.7 out of HBM, 14.4 and 9.6
// out of the cache; four pages of one layer 3.05 and 2.85.  (All with random contents: zeros move up to a fifth faster.)
template <bool TOKENS_INSIDE, int PIECES, bool STORES_ONCE, bool LOADS_ONCE>
__global__ __launch_bounds__(256) void page_copy_kernel(CopyParams P)
{
    const CopyRun run = P.runs[blockIdx.y];
    const uint32_t row_pieces = TOKENS_INSIDE ? P.row_pieces * run.tokens : P.row_pieces;
    const uint32_t all = row_pieces * (TOKENS_INSIDE ? P.heads : run.tokens);
    const int64_t row_stride = TOKENS_INSIDE ? P.head_stride : P.slot_stride;
    const uint32_t tile = P.planes == 1 ? blockIdx.x : blockIdx.x / P.planes, plane = blockIdx.x - tile * P.planes;
    const uint32_t begin = tile * (PIECES * 256);
    if (begin >= all) return;
    char *pool = P.pools[blockIdx.z] + plane * P.head_stride;
    auto token_at = [&](uint32_t slot) { return (slot >> P.page_shift) * P.page_stride + (slot & ((1u << P.page_shift) - 1)) * P.slot_stride; };
    const char *src = pool + token_at(run.src);
    char *dst = pool + token_at(run.dst);
    const uint32_t step_rows = 256 / row_pieces, step_pieces = 256 - step_rows * row_pieces;
    uint32_t row = (begin + threadIdx.x) / row_pieces, piece = begin + threadIdx.x - row * row_pieces;
    Piece x[PIECES];
    int64_t at[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        // a lane behind the run's end reads its first piece: a load with a branch around it is waited for at once
        at[j] = begin + j * 256 + threadIdx.x < all ? row * row_stride + piece * 16 : 0;
        const Piece *from = reinterpret_cast<const Piece *>(src + at[j]);
        if constexpr (LOADS_ONCE) x[j] = __builtin_nontemporal_load(from);
        else x[j] = *from;
        row += step_rows;
        piece += step_pieces;
        if (piece >= row_pieces) {
            piece -= row_pieces;
            ++row;
        }
    }
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        if (begin + j * 256 + threadIdx.x >= all) break;
        Piece *to = reinterpret_cast<Piece *>(dst + at[j]);
        if constexpr (STORES_ONCE) __builtin_nontemporal_store(x[j], to);
        else *to = x[j];
    }
}

}  // namespace

int launch_copy(CopyParams &p, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t head_pieces = uint32_t(p.head_bytes) / 16;
    const bool tokens_inside = p.slot_stride == p.head_bytes, heads_inside = !tokens_inside && p.head_stride == p.head_bytes;
    p.row_pieces = heads_inside ? head_pieces * p.heads : head_pieces;
    p.planes = tokens_inside || heads_inside ? 1 : p.heads;
    const int64_t most = int64_t(head_pieces) * p.most_tokens * (p.heads / p.planes);       // pieces of a run in a plane
    using no = std::false_type;
    using yes = std::true_type;
    auto launch = [&](auto inside, auto pieces, auto stores_once, auto loads_once) {
        constexpr int N = decltype(pieces)::value;
        const dim3 grid(unsigned((most + N * 256 - 1) / (N * 256) * p.planes), unsigned(p.num_runs), unsigned(p.num_pools));
        hipLaunchKernelGGL((page_copy_kernel<decltype(inside)::value, N, decltype(stores_once)::value, decltype(loads_once)::value>), grid,
                           dim3(256), 0, s, p);
    };
    auto launch_size = [&](auto inside) {
        using two = std::integral_constant<int, 2>;
        using eight = std::integral_constant<int, 8>;
        if (!p.large)         launch(inside, two{}, no{}, no{});
        else if (most < 1024) launch(inside, two{}, yes{}, no{});
        else if (!p.huge)     launch(inside, eight{}, yes{}, no{});
        else                  launch(inside, eight{}, yes{}, yes{});
    };
    tokens_inside ? launch_size(yes{}) : launch_size(no{});
    return int(hipGetLastError());
}

}  // namespace codec
