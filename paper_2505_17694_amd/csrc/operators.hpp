// Launch interface of the kernels around a decode step, and checks their entry points share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "codec.h"

namespace codec {

// What the L2s of the eight dies hold together.  Calls that read and write more use the streaming hint: what they leave would
// not be found there.
constexpr double kLargeBytes = 32 << 20;
// What the last-level cache holds.
constexpr double kHugeBytes = 256 << 20;

// Rows of one kind (queries, keys, values) of the tokens: strides in bytes.
struct RowsView {
    char *data;
    int64_t token_stride, head_stride;
};

struct RotaryParams {
    RowsView q, q_out, k, v;        // q.data == nullptr: no queries; k.data == nullptr: no keys and values
    char *k_pages, *v_pages;
    int64_t page_stride, slot_stride, head_stride;      // bytes
    const int64_t *positions;
    const int64_t *slots;
    const double *turns;            // [rotary_dim / 2]; not read where rotary_dim == 0
    int64_t num_tokens, num_slots;  // slots of the pools: slot s is token s % page size of page s / page size
    int32_t q_heads, kv_heads, head_dim, rotary_dim, page_shift;
    float magnitude, sign;          // factors on the turned channels and on the sine
};

constexpr int kMaxAxes = 4;

struct AxesParams : RotaryParams {
    const uint8_t *axes;            // [rotary_dim / 2]: the axis whose positions turn a pair
    int64_t axis_stride;            // positions of an axis, from one axis to the next
    int32_t num_axes, block_pairs;  // pairs of a block of halves
};

// A launch's worth of codec_cache_copy: pools and runs travel in the kernel's arguments, which hold 4 KB.
constexpr int kCopyPools = 64;
constexpr int kCopyRuns = 288;

struct CopyRun {
    uint32_t src, dst;              // first token's slot: page * page size + token
    uint32_t tokens;
};

struct CopyParams {
    int64_t page_stride, slot_stride, head_stride;      // bytes
    int32_t heads, head_bytes, page_shift, num_pools, num_runs, most_tokens;
    uint32_t row_pieces, planes;                        // set by launch_copy
    bool large, huge;                                   // the call moves more than kLargeBytes, reads more than kHugeBytes
    char *pools[kCopyPools];
    CopyRun runs[kCopyRuns];
};
static_assert(sizeof(CopyParams) <= 4096, "kernel arguments");

struct TableParams {
    const int32_t *page_off, *page_ids, *tokens;        // [num_seq + 1], [num_ids], [num_seq]
    int32_t *table;
    int64_t table_stride, num_ids;
    int32_t num_seq, width, page_shift;
    uint32_t row_units;                                 // set by launch_block_table
    uint64_t units;
};

// Most sequences whose sums every workgroup makes for itself, in LDS, in the place of a launch that makes them once.  us by one launch
// and by two, a token each: 48 sequences 3.5 and 5.6, 1000 4.9 and 8.1, 2000 6.9 and 10.1, 4096 12.2 and 13.4, 6000 20.0 and 15.6; 500000
// tokens of 1000 sequences 8.9 and 13.2, of 4096 17.7 and 18.9.
constexpr int kSlotsAtOnce = 4096;

struct SlotParams {
    int32_t *table;
    int64_t table_stride, num_pages;
    const int32_t *tokens, *new_tokens;     // [num_seq]
    const int64_t *before;                  // [num_seq] or nullptr
    const int32_t *spare;                   // [num_spare] or nullptr: the table holds the new tokens' pages
    int64_t *positions, *slots;             // [num_tokens]
    int32_t *sequences;                     // [num_tokens] or nullptr
    int32_t *offsets, *tokens_out, *taken;  // [num_seq + 1], [num_seq], [1]
    uint32_t *sums;                         // [2 * num_seq + 1], more than kSlotsAtOnce sequences: new tokens, new pages before each
    int32_t num_seq, width, num_tokens, num_spare, page_shift;
};

// A sum of exponentials: sum * 2^ref
struct PartialSum { double ref, sum; };

struct BeamParams {
    const char *logits;
    int64_t batch_stride, beam_stride;      // elements
    const float *scores;
    const uint8_t *finished;                // or nullptr
    float *out_scores;
    int32_t *out_beams, *out_tokens;
    // Of every part of a beam's vocabulary ([batch * beams][parts]): its best tokens, its sum of exponentials
    uint64_t *best;
    PartialSum *sums;
    int32_t batch, beams, vocab, k, kept, eos, parts;   // kept = min(k, vocab): tokens a beam can bring
};

// How many workgroups share a beam's vocabulary, and how many waves each has.
struct BeamSplit { int waves, parts; };
BeamSplit beam_split(int64_t rows, int vocab);

constexpr int kReorderStates = 64;      // of a launch

struct ReorderState {
    const char *src;
    char *dst;
    int64_t src_batch, src_beam, dst_batch, dst_beam;   // bytes
    int64_t row_units;
};

struct ReorderParams {
    const int32_t *beams;
    int32_t batch, beams_in, beams_out, num_states;
    int64_t most_units;
    bool large;                                         // the call moves more than kLargeBytes
    ReorderState states[kReorderStates];
};
static_assert(sizeof(ReorderParams) <= 4096, "kernel arguments");

// All return a hipError_t value (0 = success) without synchronising.
int launch_rotary(const RotaryParams &p, int dtype, bool interleaved, void *stream);
int launch_rotary_axes(const AxesParams &p, int dtype, bool interleaved, void *stream);
int launch_copy(CopyParams &p, void *stream);
int launch_block_table(TableParams p, void *stream);
int launch_slot_map(const SlotParams &p, void *stream);
int launch_beam_select(const BeamParams &p, int dtype, void *stream);
// `unit`: bytes moved at a time, 1, 2, 4, 8 or 16
int launch_reorder(const ReorderParams &p, int unit, void *stream);

}  // namespace codec
