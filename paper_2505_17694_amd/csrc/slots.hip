// Block tables, and positions and slots of a step's new tokens, from the lengths of the sequences on the GPU.
//
// Sequence s holds len_s tokens in pages of 2^k and gets new_s more.  With T_s and N_s the sums over the sequences before s of new
// tokens and of new pages, ceil((len + new) / page) - ceil(len / page) each, token t belongs to the last s with T_s <= t and lies at
// place len_s + t - T_s of it; page p of the sequence that the table does not hold yet is spare page N_s + p - ceil(len_s / page).
#include <hip/hip_runtime.h>

#include "operators.hpp"

namespace codec {
namespace {

__device__ __forceinline__ int64_t at_least_0(int32_t n) { return n > 0 ? n : 0; }

// A table's row in units of four entries.  Bound by HBM, mostly by the writes: entries behind a sequence's pages are -1 without a
// read (4096 sequences of up to 64k tokens: 67 MB written, 33 MB read, 17.4 us, 5.8 TB/s; 33 sequences 2.3).
template <bool ALIGNED>
__global__ __launch_bounds__(256) void block_table_kernel(TableParams P)
{
    typedef int32_t __attribute__((ext_vector_type(4))) Four;
    typedef int32_t __attribute__((ext_vector_type(4), aligned(4))) AnyFour;
    for (uint64_t unit = uint64_t(blockIdx.x) * 256 + threadIdx.x; unit < P.units; unit += uint64_t(gridDim.x) * 256) {
        const uint32_t row = uint32_t(unit / P.row_units);
        const int first = int(unit - uint64_t(row) * P.row_units) * 4;
        const int64_t begin = P.page_off[row], end = P.page_off[row + 1];
        int64_t pages = (at_least_0(P.tokens[row]) + (int64_t(1) << P.page_shift) - 1) >> P.page_shift;
        if (pages > end - begin) pages = end - begin;
        if (pages > P.num_ids - begin) pages = P.num_ids - begin;
        if (pages > P.width) pages = P.width;
        if (pages < 0 || begin < 0) pages = 0;          // (end - begin may be beyond 32 bits)
        const int held = int(pages) - first, room = P.width - first;        // of these four
        int32_t *at = P.table + int64_t(row) * P.table_stride + first;
        Four x = {-1, -1, -1, -1};
        const int32_t *from = P.page_ids + begin + first;
        if (held >= 4) {
            x = *reinterpret_cast<const AnyFour *>(from);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < held) x[i] = from[i];
        }
        if (ALIGNED && room >= 4) {
            *reinterpret_cast<Four *>(at) = x;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < room) at[i] = x[i];
        }
    }
}

struct Growth { uint64_t tokens, pages; };

// What a sequence brings: new tokens, and pages that the table has room for and does not hold.
__device__ __forceinline__ Growth growth(const SlotParams &P, int64_t len, int64_t more)
{
    const int64_t last = (int64_t(1) << P.page_shift) - 1;
    int64_t held = (len + last) >> P.page_shift, need = (len + more + last) >> P.page_shift;
    if (held > P.width) held = P.width;
    if (need > P.width) need = P.width;
    return {uint64_t(more), P.spare ? uint64_t(need - held) : 0};
}

// Exclusive sums over the threads of a workgroup of WAVES waves.
template <int WAVES>
__device__ __forceinline__ Growth before_thread(Growth own)
{
    __shared__ Growth sums[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Growth to = own;                                    // the wave's lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint64_t t = __shfl_up(to.tokens, d), p = __shfl_up(to.pages, d);
        if (lane >= d) {
            to.tokens += t;
            to.pages += p;
        }
    }
    if (lane == 63) sums[wave] = to;
    __syncthreads();
    to.tokens -= own.tokens;
    to.pages -= own.pages;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w)
        if (w < wave) {
            to.tokens += sums[w].tokens;
            to.pages += sums[w].pages;
        }
    return to;
}

// Sums of all sequences: token_off [n + 1] (no more than num_tokens), page_first [n].  A thread sums up neighbouring sequences,
// which it reads twice.  OUT: the call's outputs of a sequence as well.
template <int WAVES, bool OUT>
__device__ __forceinline__ void sum_sequences(const SlotParams &P, uint32_t *token_off, uint32_t *page_first)
{
    const int n = P.num_seq, share = (n + WAVES * 64 - 1) / (WAVES * 64);
    const int begin = min(n, int(threadIdx.x) * share), end = min(n, begin + share);
    Growth own = {0, 0};
#pragma unroll 4
    for (int s = begin; s < end; ++s) {
        const Growth g = growth(P, at_least_0(P.tokens[s]), at_least_0(P.new_tokens[s]));
        own.tokens += g.tokens;
        own.pages += g.pages;
    }
    Growth at = before_thread<WAVES>(own);
    const uint64_t most = uint64_t(P.num_tokens);
    auto page_count = [](uint64_t pages) { return uint32_t(pages < 0x7fffffff ? pages : 0x7fffffff); };
#pragma unroll 4
    for (int s = begin; s < end; ++s) {
        const int64_t len = at_least_0(P.tokens[s]);
        const Growth g = growth(P, len, at_least_0(P.new_tokens[s]));
        const uint64_t first = at.tokens < most ? at.tokens : most, behind = at.tokens + g.tokens < most ? at.tokens + g.tokens : most;
        token_off[s] = uint32_t(first);
        page_first[s] = page_count(at.pages);
        if constexpr (OUT) {
            const int64_t now = len + int64_t(behind - first);
            P.offsets[s] = int32_t(first);
            P.tokens_out[s] = int32_t(now < 0x7fffffff ? now : 0x7fffffff);
            // more new tokens than there is room for: the pages of those that fit
            if (at.tokens <= most && at.tokens + g.tokens > most) *P.taken = int32_t(page_count(at.pages + growth(P, len, int64_t(behind - first)).pages));
        }
        at.tokens += g.tokens;
        at.pages += g.pages;
    }
    if (end == n && (begin < n || threadIdx.x == 0)) {  // the thread of the last sequence
        token_off[n] = uint32_t(at.tokens < most ? at.tokens : most);
        if constexpr (OUT) {
            P.offsets[n] = int32_t(token_off[n]);
            if (at.tokens <= most) *P.taken = int32_t(page_count(at.pages));
        }
    }
}

// Tokens of the map, a thread each.
__device__ __forceinline__ void map_tokens(const SlotParams &P, const uint32_t *token_off, const uint32_t *page_first)
{
    const uint32_t total = token_off[P.num_seq];
    const int64_t in_page = (int64_t(1) << P.page_shift) - 1;
    for (int64_t t = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; t < P.num_tokens; t += int64_t(gridDim.x) * blockDim.x) {
        int64_t position = 0, slot = -1;
        int32_t sequence = -1;
        if (t < total) {
            int s = 0;                                  // the last sequence that begins at t or before
            for (int left = P.num_seq; left > 1;) {
                const int half = left / 2;
                s = token_off[s + half] <= t ? s + half : s;
                left -= half;
            }
            const int64_t len = at_least_0(P.tokens[s]), place = len + (t - token_off[s]), page = place >> P.page_shift;
            sequence = s;
            position = place + (P.before ? P.before[s] : 0);
            if (page < P.width) {
                const int64_t held = (len + in_page) >> P.page_shift;
                int32_t *entry = P.table + s * P.table_stride + page;
                int32_t id = -1;
                if (P.spare && page >= held) {
                    const int64_t i = page_first[s] + (page - held);
                    if (i < P.num_spare) id = P.spare[i];
                    if (id >= P.num_pages || id < 0) id = -1;
                    if ((place & in_page) == 0) *entry = id;        // a page's first token is a new one if the page is
                } else {
                    id = *entry;
                }
                if (id >= 0 && id < P.num_pages) slot = (int64_t(id) << P.page_shift) + (place & in_page);
            }
        }
        P.positions[t] = position;
        P.slots[t] = slot;
        if (P.sequences) P.sequences[t] = sequence;
    }
}

// Up to kSlotsAtOnce sequences: every workgroup sums them up for itself, in LDS.  Bound by dependent reads: 48 sequences with a token
// each 3.3 us, 65k tokens of 300 sequences 5.1; a launch for the sums would be 2 more (see kSlotsAtOnce), and 3 on the host.
__global__ __launch_bounds__(256) void slot_map_kernel(SlotParams P)
{
    extern __shared__ uint32_t sums[];                  // [n + 1], [n]
    uint32_t *page_first = sums + P.num_seq + 1;
    if (blockIdx.x == 0) sum_sequences<4, true>(P, sums, page_first);
    else                 sum_sequences<4, false>(P, sums, page_first);
    __syncthreads();
    map_tokens(P, sums, page_first);
}

// More: one workgroup sums them up, all others' search goes through L2.  A thread reads neighbouring sequences, its wave's lanes so many
// entries apart: 20000 sequences take 69 us, 100000 take 387.
__global__ __launch_bounds__(1024) void slot_sums_kernel(SlotParams P)
{
    sum_sequences<16, true>(P, P.sums, P.sums + P.num_seq + 1);
}

__global__ __launch_bounds__(256) void slot_find_kernel(SlotParams P)
{
    map_tokens(P, P.sums, P.sums + P.num_seq + 1);
}

}  // namespace

int launch_block_table(TableParams p, void *stream)
{
    p.row_units = uint32_t((int64_t(p.width) + 3) / 4);
    p.units = uint64_t(p.row_units) * uint64_t(p.num_seq);
    constexpr uint64_t kMost = 1 << 16;                 // workgroups
    const uint64_t blocks = (p.units + 255) / 256;
    const dim3 grid(unsigned(blocks < kMost ? blocks : kMost));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool aligned = reinterpret_cast<uintptr_t>(p.table) % 16 == 0 && p.table_stride % 4 == 0;
    if (aligned) hipLaunchKernelGGL(block_table_kernel<true>, grid, dim3(256), 0, s, p);
    else         hipLaunchKernelGGL(block_table_kernel<false>, grid, dim3(256), 0, s, p);
    return int(hipGetLastError());
}

int launch_slot_map(const SlotParams &p, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int64_t blocks = (int64_t(p.num_tokens) + 255) / 256;
    const dim3 grid(unsigned(blocks < 1 ? 1 : blocks < 1024 ? blocks : 1024));
    if (p.num_seq <= kSlotsAtOnce) {
        hipLaunchKernelGGL(slot_map_kernel, grid, dim3(256), (2 * unsigned(p.num_seq) + 1) * 4, s, p);
        return int(hipGetLastError());
    }
    hipLaunchKernelGGL(slot_sums_kernel, dim3(1), dim3(1024), 0, s, p);
    if (int e = int(hipGetLastError())) return e;
    if (p.num_tokens) hipLaunchKernelGGL(slot_find_kernel, grid, dim3(256), 0, s, p);
    return int(hipGetLastError());
}

}  // namespace codec
