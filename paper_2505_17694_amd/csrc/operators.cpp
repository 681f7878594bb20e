// C ABI of the operators around a decode step: argument checks and launches.
#include "operators.hpp"

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <new>
#include <vector>

#include "status.hpp"

namespace {

using codec::hip_failure;

constexpr double kTwoPi = 6.283185307179586476925;
constexpr int64_t kMaxSpan = int64_t(1) << 58;          // elements: byte offsets, and sums of a few, stay in 64 bits
constexpr int32_t kMaxSequences = 1 << 22;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// What the pools of this library hold; the codes codec_plan_create returns.
int check_rows_of(int32_t head_dim, int32_t dtype)
{
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return CODEC_ERR_UNSUPPORTED;
    if (dtype != CODEC_DTYPE_FP16 && dtype != CODEC_DTYPE_BF16) return CODEC_ERR_UNSUPPORTED;
    return CODEC_OK;
}

bool page_size_ok(int32_t n) { return n >= 16 && n <= 4096 && (n & (n - 1)) == 0; }

int check_head(const codec_head_config &h)
{
    if (h.num_kv_heads < 1 || h.num_q_heads < 1 || h.num_kv_heads > (1 << 12) || h.num_q_heads > (1 << 16)) return CODEC_ERR_INVALID_ARGUMENT;
    if (int st = check_rows_of(h.head_dim, h.dtype)) return st;
    return page_size_ok(h.page_size) ? CODEC_OK : CODEC_ERR_UNSUPPORTED;
}

struct Extent { int64_t count, stride; };

// Elements from the first to behind the last of `inner` contiguous ones repeated along `dims`; -1 where two coincide.
template <size_t N>
int64_t separate_span(int64_t inner, Extent (&dims)[N])
{
    std::sort(dims, dims + N, [](const Extent &a, const Extent &b) { return a.stride < b.stride; });
    int64_t span = inner;
    for (const Extent &d : dims) {
        if (d.count <= 1) continue;
        if (d.stride < span || d.stride > kMaxSpan / d.count) return -1;
        span += (d.count - 1) * d.stride;
        if (span > kMaxSpan) return -1;
    }
    return span;
}

// Elements of a pool behind its first one that `layout` reaches; -1 for a layout a cache cannot be written by.
int64_t pool_span(const codec_head_config &h, const codec_kv_layout &l)
{
    if (l.num_pages < 1 || l.num_pages > (int64_t(1) << 31) || l.page_stride < 1 || l.token_stride < h.head_dim || l.head_stride < h.head_dim) return -1;
    if (l.page_stride % 8 || l.token_stride % 8 || l.head_stride % 8) return -1;
    Extent dims[] = {{l.num_pages, l.page_stride}, {h.page_size, l.token_stride}, {h.num_kv_heads, l.head_stride}};
    return separate_span(h.head_dim, dims);
}

// Whether two pools of this layout have no element in common: apart in memory, or one between the parts of the other (K and V
// side by side).
bool pools_apart(const codec_head_config &h, const codec_kv_layout &l, const void *a, const void *b)
{
    const int64_t distance = std::abs(static_cast<const char *>(a) - static_cast<const char *>(b)) / 2;
    Extent dims[] = {{l.num_pages, l.page_stride}, {h.page_size, l.token_stride}, {h.num_kv_heads, l.head_stride}, {2, distance}};
    return separate_span(h.head_dim, dims) >= 0;
}

struct Range { const char *begin, *end; };
bool overlap(const Range &a, const Range &b) { return a.begin < b.end && b.begin < a.end; }
Range bytes_at(const void *p, int64_t n) { return {static_cast<const char *>(p), static_cast<const char *>(p) + n}; }

bool rows_ok(const codec_rows *r, int64_t tokens, int64_t heads)
{
    return r && r->data && aligned16(r->data) && r->token_stride >= 0 && r->head_stride >= 0 && r->token_stride % 8 == 0 &&
           r->head_stride % 8 == 0 && r->token_stride <= kMaxSpan / tokens && r->head_stride <= kMaxSpan / heads;
}

int64_t rows_span(const codec_rows &r, int64_t tokens, int64_t heads, int64_t d)
{
    return (tokens - 1) * r.token_stride + (heads - 1) * r.head_stride + d;
}

Range range_of(const codec_rows &r, int64_t tokens, int64_t heads, int64_t d)
{
    const char *p = static_cast<const char *>(r.data);
    return {p, p + 2 * rows_span(r, tokens, heads, d)};
}

// Rows that may be written: none overlaps another.
bool separate(const codec_rows &r, int64_t tokens, int64_t heads, int64_t d)
{
    Extent dims[] = {{tokens, r.token_stride}, {heads, r.head_stride}};
    return separate_span(d, dims) >= 0;
}

bool same_rows(const codec_rows &a, const codec_rows &b, int64_t tokens, int64_t heads)
{
    return a.data == b.data && (tokens == 1 || a.token_stride == b.token_stride) && (heads == 1 || a.head_stride == b.head_stride);
}

// No element of a is one of b: apart in memory, or other heads of the same tokens' tensor.
bool apart(const codec_rows &a, int64_t heads_a, const codec_rows &b, int64_t heads_b, int64_t tokens, int64_t d)
{
    if (!overlap(range_of(a, tokens, heads_a, d), range_of(b, tokens, heads_b, d))) return true;
    if (a.token_stride != b.token_stride) return false;
    const bool a_first = a.data < b.data;
    const codec_rows &lo = a_first ? a : b, &hi = a_first ? b : a;
    const int64_t offset = (static_cast<const char *>(hi.data) - static_cast<const char *>(lo.data)) / 2;
    return offset >= rows_span(lo, 1, a_first ? heads_a : heads_b, d) &&
           offset + rows_span(hi, 1, a_first ? heads_b : heads_a, d) <= a.token_stride;
}

int check_rotary(const codec_rotary_config &r, int32_t head_dim, const int64_t *positions)
{
    if (r.rotary_dim < 2 || r.rotary_dim > head_dim || r.rotary_dim % 2 || !r.turns || !positions) return CODEC_ERR_INVALID_ARGUMENT;
    if (r.layout != CODEC_ROTARY_HALF && r.layout != CODEC_ROTARY_INTERLEAVED) return CODEC_ERR_INVALID_ARGUMENT;
    if (!std::isfinite(r.magnitude)) return CODEC_ERR_INVALID_ARGUMENT;
    return CODEC_OK;
}

int check_axes(const codec_rotary_axes &a, int32_t head_dim, const int64_t *positions)
{
    if (int st = check_rotary(a.rotary, head_dim, positions)) return st;
    if (a.num_axes < 1 || a.num_axes > codec::kMaxAxes || !a.axes || a.axis_stride < 0 || a.axis_stride > kMaxSpan) return CODEC_ERR_INVALID_ARGUMENT;
    if (a.block_dim < 0 || (a.block_dim && a.rotary.rotary_dim % a.block_dim)) return CODEC_ERR_INVALID_ARGUMENT;
    const bool blocks = a.block_dim && a.block_dim != a.rotary.rotary_dim;
    if (blocks && (a.block_dim % 2 || (a.rotary.layout == CODEC_ROTARY_HALF && a.block_dim % 16))) return CODEC_ERR_UNSUPPORTED;
    return CODEC_OK;
}

// Tokens of the pages that a list of copies writes, as bits: an open-addressing table of pages.
class WrittenTokens {
public:
    WrittenTokens(int32_t runs, int32_t page_size)
    {
        while ((page_size >> shift_) > 64) ++shift_;
        size_t n = 16;
        while (n < 2 * size_t(runs)) n *= 2;
        slots_.resize(n);
    }
    // Marks tokens [at, at + n) of the page; whether one of them may be marked already.
    bool mark(int32_t page, int32_t at, int32_t n)
    {
        Slot &s = slot(page);
        s.page = page;
        const uint64_t b = bits(at, n);
        const bool met = s.bits & b;
        s.bits |= b;
        return met;
    }
    // Whether one of these tokens may be marked.
    bool holds(int32_t page, int32_t at, int32_t n) { return slot(page).bits & bits(at, n); }
    bool exact() const { return shift_ == 0; }          // a bit is a token

private:
    struct Slot { int32_t page = -1; uint64_t bits = 0; };
    Slot &slot(int32_t page)
    {
        size_t i = (uint32_t(page) * 2654435769u >> 8) & (slots_.size() - 1);
        while (slots_[i].page >= 0 && slots_[i].page != page) i = (i + 1) & (slots_.size() - 1);
        return slots_[i];
    }
    uint64_t bits(int32_t at, int32_t n) const
    {
        const int first = at >> shift_, last = (at + n - 1) >> shift_;
        return (~uint64_t(0) >> (63 - last)) & (~uint64_t(0) << first);
    }
    int shift_ = 0;
    std::vector<Slot> slots_;
};

// Whether a token is written twice or both read and written.
bool runs_collide(const codec_run *runs, int32_t n, int32_t page_size)
{
    WrittenTokens written(n, page_size);
    bool met = false;
    for (int32_t i = 0; i < n; ++i) met |= written.mark(runs[i].dst_page, runs[i].dst_token, runs[i].tokens);
    for (int32_t i = 0; i < n && !met; ++i) met = written.holds(runs[i].src_page, runs[i].src_token, runs[i].tokens);
    if (!met || written.exact()) return met;
    // pages of more than 64 tokens share bits: compare the token ranges themselves
    struct Span { int64_t begin, end; };
    std::vector<Span> spans(n);
    for (int32_t i = 0; i < n; ++i) {
        const int64_t at = int64_t(runs[i].dst_page) * page_size + runs[i].dst_token;
        spans[i] = {at, at + runs[i].tokens};
    }
    std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.begin < b.begin; });
    for (int32_t i = 1; i < n; ++i)
        if (spans[i].begin < spans[i - 1].end) return true;
    for (int32_t i = 0; i < n; ++i) {
        const int64_t at = int64_t(runs[i].src_page) * page_size + runs[i].src_token, end = at + runs[i].tokens;
        const auto next = std::lower_bound(spans.begin(), spans.end(), end, [](const Span &a, int64_t e) { return a.begin < e; });
        if (next != spans.begin() && std::prev(next)->end > at) return true;
    }
    return false;
}

int check_beams(const codec_beam_config &c)
{
    if (c.batch < 0 || c.beams < 1 || c.beams > 64 || c.vocab < 1 || c.vocab > (1 << 24) || c.k < 1 || c.k > 64 ||
        c.k > int64_t(c.beams) * c.vocab || int64_t(c.batch) * c.beams > (1 << 22))
        return CODEC_ERR_INVALID_ARGUMENT;
    if (c.dtype != CODEC_DTYPE_FP16 && c.dtype != CODEC_DTYPE_BF16 && c.dtype != CODEC_DTYPE_FP32) return CODEC_ERR_UNSUPPORTED;
    return CODEC_OK;
}

size_t align_up(size_t n) { return (n + 255) / 256 * 256; }

// Scratch of a selection: best tokens, then sums.
struct BeamScratch { int parts; size_t sums, total; };
BeamScratch beam_scratch(const codec_beam_config &c)
{
    BeamScratch s{};
    if (c.batch == 0) return s;
    s.parts = codec::beam_split(int64_t(c.batch) * c.beams, c.vocab).parts;
    const size_t lists = size_t(c.batch) * c.beams * s.parts;
    s.sums = align_up(lists * std::min(c.k, c.vocab) * sizeof(uint64_t));
    s.total = s.sums + align_up(lists * sizeof(codec::PartialSum));
    return s;
}

// Bytes from the first to behind the last of a state's rows; -1 for strides that are out of range.
int64_t state_span(int64_t row_bytes, int64_t batch, int64_t batch_stride, int64_t beams, int64_t beam_stride)
{
    if (row_bytes > kMaxSpan || batch_stride < 0 || beam_stride < 0 || batch_stride > kMaxSpan / batch || beam_stride > kMaxSpan / beams) return -1;
    return (batch - 1) * batch_stride + (beams - 1) * beam_stride + row_bytes;
}

codec::RowsView view_of(const codec_rows &r) { return {static_cast<char *>(r.data), 2 * r.token_stride, 2 * r.head_stride}; }

void set_rotary(codec::RotaryParams &p, const codec_rotary_config &r, const int64_t *positions)
{
    p.positions = positions;
    p.turns = r.turns;
    p.rotary_dim = r.rotary_dim;
    p.magnitude = r.magnitude;
    p.sign = r.inverse ? -1.f : 1.f;
}

// The launch of either form: by one position a token, or by several axes.
int launch(const codec::RotaryParams &p, int dtype, const codec_rotary_config *rotary, const codec_rotary_axes *axes, const char *what, void *stream)
{
    const bool interleaved = rotary && rotary->layout == CODEC_ROTARY_INTERLEAVED;
    int e;
    if (axes) {
        codec::AxesParams by{};
        static_cast<codec::RotaryParams &>(by) = p;
        by.axes = axes->axes;
        by.axis_stride = axes->axis_stride;
        by.num_axes = axes->num_axes;
        by.block_pairs = (axes->block_dim ? axes->block_dim : rotary->rotary_dim) / 2;
        e = codec::launch_rotary_axes(by, dtype, interleaved, stream);
    } else {
        e = codec::launch_rotary(p, dtype, interleaved, stream);
    }
    return e ? hip_failure(what, e) : CODEC_OK;
}

// codec_rotary, and codec_rotary_by_axes where `axes` is not NULL (`rotary` is then its first member).
int rotate_rows(const codec_rotary_config *rotary, const codec_rotary_axes *axes, int32_t num_heads, int32_t head_dim, int32_t dtype,
                const codec_rows *x, const codec_rows *out, const int64_t *positions, int32_t num_tokens, void *stream)
{
    if (!rotary || num_heads < 1 || num_heads > (1 << 16) || num_tokens < 0) return CODEC_ERR_INVALID_ARGUMENT;
    if (int st = check_rows_of(head_dim, dtype)) return st;
    if (num_tokens == 0) return CODEC_OK;
    if (int st = axes ? check_axes(*axes, head_dim, positions) : check_rotary(*rotary, head_dim, positions)) return st;
    if (!rows_ok(x, num_tokens, num_heads) || !rows_ok(out, num_tokens, num_heads) || !separate(*out, num_tokens, num_heads, head_dim)) return CODEC_ERR_INVALID_ARGUMENT;
    if (!same_rows(*x, *out, num_tokens, num_heads) && !apart(*x, num_heads, *out, num_heads, num_tokens, head_dim)) return CODEC_ERR_INVALID_ARGUMENT;

    codec::RotaryParams p{};
    p.q = view_of(*x);
    p.q_out = view_of(*out);
    p.q_heads = num_heads;
    p.head_dim = head_dim;
    p.num_tokens = num_tokens;
    set_rotary(p, *rotary, positions);
    return launch(p, dtype, rotary, axes, "rotary launch", stream);
}

// codec_append and codec_append_by_axes, alike.
int append_rows(const codec_head_config *head, const codec_rotary_config *rotary, const codec_rotary_axes *axes, const codec_rows *q,
                const codec_rows *q_out, const codec_rows *k, const codec_rows *v, const int64_t *positions, const int64_t *slots,
                int32_t num_tokens, void *k_pages, void *v_pages, const codec_kv_layout *layout, void *stream)
{
    if (!head || !layout || num_tokens < 0 || !q != !q_out) return CODEC_ERR_INVALID_ARGUMENT;
    if (int st = check_head(*head)) return st;
    const int64_t pool = pool_span(*head, *layout);
    if (pool < 0) return CODEC_ERR_INVALID_ARGUMENT;
    if (num_tokens == 0) return CODEC_OK;
    if (rotary)
        if (int st = axes ? check_axes(*axes, head->head_dim, positions) : check_rotary(*rotary, head->head_dim, positions)) return st;
    if (!slots || !k_pages || !v_pages || !aligned16(k_pages) || !aligned16(v_pages) || !pools_apart(*head, *layout, k_pages, v_pages)) return CODEC_ERR_INVALID_ARGUMENT;
    const int64_t t = num_tokens, d = head->head_dim, hq = head->num_q_heads, h = head->num_kv_heads;
    if (!rows_ok(k, t, h) || !rows_ok(v, t, h) || (q && (!rows_ok(q, t, hq) || !rows_ok(q_out, t, hq)))) return CODEC_ERR_INVALID_ARGUMENT;
    for (const void *pages : {k_pages, v_pages}) {
        const Range r{static_cast<const char *>(pages), static_cast<const char *>(pages) + 2 * pool};
        if (overlap(r, range_of(*k, t, h, d)) || overlap(r, range_of(*v, t, h, d))) return CODEC_ERR_INVALID_ARGUMENT;
        if (q && (overlap(r, range_of(*q, t, hq, d)) || overlap(r, range_of(*q_out, t, hq, d)))) return CODEC_ERR_INVALID_ARGUMENT;
    }
    if (q) {
        if (!separate(*q_out, t, hq, d)) return CODEC_ERR_INVALID_ARGUMENT;
        if (!same_rows(*q, *q_out, t, hq) && !apart(*q, hq, *q_out, hq, t, d)) return CODEC_ERR_INVALID_ARGUMENT;
        if (!apart(*q_out, hq, *k, h, t, d) || !apart(*q_out, hq, *v, h, t, d)) return CODEC_ERR_INVALID_ARGUMENT;
    }

    codec::RotaryParams p{};
    if (q) {
        p.q = view_of(*q);
        p.q_out = view_of(*q_out);
        p.q_heads = head->num_q_heads;
    }
    p.k = view_of(*k);
    p.v = view_of(*v);
    p.kv_heads = head->num_kv_heads;
    p.k_pages = static_cast<char *>(k_pages);
    p.v_pages = static_cast<char *>(v_pages);
    p.page_stride = 2 * layout->page_stride;
    p.slot_stride = 2 * layout->token_stride;
    p.head_stride = 2 * layout->head_stride;
    p.slots = slots;
    p.num_slots = layout->num_pages * head->page_size;
    while ((1 << p.page_shift) < head->page_size) ++p.page_shift;
    p.head_dim = head->head_dim;
    p.num_tokens = num_tokens;
    if (rotary) set_rotary(p, *rotary, positions);
    return launch(p, head->dtype, rotary, axes, "append launch", stream);
}

}  // namespace

extern "C" {

int codec_rotary_turns(int32_t rotary_dim, double theta, const codec_rotary_scaling *scaling, double *turns, float *magnitude)
{
    if (!turns || !magnitude || rotary_dim < 2 || rotary_dim > 256 || rotary_dim % 2) return CODEC_ERR_INVALID_ARGUMENT;
    if (!(theta > 1.0) || !std::isfinite(theta)) return CODEC_ERR_INVALID_ARGUMENT;
    codec_rotary_scaling s{};
    if (scaling) s = *scaling;
    if (s.kind < CODEC_ROTARY_UNSCALED || s.kind > CODEC_ROTARY_YARN) return CODEC_ERR_INVALID_ARGUMENT;
    if (s.kind != CODEC_ROTARY_UNSCALED && (!(s.factor > 0.0) || !std::isfinite(s.factor))) return CODEC_ERR_INVALID_ARGUMENT;
    const bool long_context = s.kind == CODEC_ROTARY_WAVELENGTH || s.kind == CODEC_ROTARY_YARN;
    if (long_context && s.original_length < 1) return CODEC_ERR_INVALID_ARGUMENT;
    if (s.kind == CODEC_ROTARY_WAVELENGTH && (!(s.low < s.high) || !std::isfinite(s.low) || !std::isfinite(s.high))) return CODEC_ERR_INVALID_ARGUMENT;
    if (s.kind == CODEC_ROTARY_YARN && (!(s.slow > 0.0) || !(s.fast > s.slow) || !std::isfinite(s.fast))) return CODEC_ERR_INVALID_ARGUMENT;

    const int32_t pairs = rotary_dim / 2;
    if (s.kind == CODEC_ROTARY_NTK && rotary_dim > 2) theta *= std::pow(s.factor, double(rotary_dim) / (rotary_dim - 2));
    if (!(theta > 0.0) || !std::isfinite(theta)) return CODEC_ERR_INVALID_ARGUMENT;
    double from = 0.0, to = 0.0;                // YARN: the pairs between which the two frequencies are blended
    if (s.kind == CODEC_ROTARY_YARN) {
        auto pair_of = [&](double n) { return rotary_dim * std::log(s.original_length / (n * kTwoPi)) / (2.0 * std::log(theta)); };
        from = std::max(std::floor(pair_of(s.fast)), 0.0);
        to = std::min(std::ceil(pair_of(s.slow)), double(rotary_dim - 1));
    }
    for (int32_t i = 0; i < pairs; ++i) {
        double f = std::pow(theta, -2.0 * i / rotary_dim);
        if (s.kind == CODEC_ROTARY_LINEAR) {
            f /= s.factor;
        } else if (long_context) {
            const double scaled = s.kind == CODEC_ROTARY_WAVELENGTH ? 1.0 - (s.original_length * f / kTwoPi - s.low) / (s.high - s.low)
                                                                    : (i - from) / std::max(to - from, 0.001);
            const double w = std::min(std::max(scaled, 0.0), 1.0);
            f = (1.0 - w) * f + w * (f / s.factor);
        }
        turns[i] = f / kTwoPi;
    }
    *magnitude = s.kind == CODEC_ROTARY_YARN && s.factor > 1.0 ? float(0.1 * std::log(s.factor) + 1.0) : 1.f;
    return CODEC_OK;
}

int codec_rotary(const codec_rotary_config *rotary, int32_t num_heads, int32_t head_dim, int32_t dtype, const codec_rows *x,
                 const codec_rows *out, const int64_t *positions, int32_t num_tokens, void *stream)
{
    return rotate_rows(rotary, nullptr, num_heads, head_dim, dtype, x, out, positions, num_tokens, stream);
}

int codec_rotary_by_axes(const codec_rotary_axes *rotary, int32_t num_heads, int32_t head_dim, int32_t dtype, const codec_rows *x,
                         const codec_rows *out, const int64_t *positions, int32_t num_tokens, void *stream)
{
    return rotate_rows(rotary ? &rotary->rotary : nullptr, rotary, num_heads, head_dim, dtype, x, out, positions, num_tokens, stream);
}

int codec_append(const codec_head_config *head, const codec_rotary_config *rotary, const codec_rows *q, const codec_rows *q_out,
                 const codec_rows *k, const codec_rows *v, const int64_t *positions, const int64_t *slots, int32_t num_tokens,
                 void *k_pages, void *v_pages, const codec_kv_layout *layout, void *stream)
{
    return append_rows(head, rotary, nullptr, q, q_out, k, v, positions, slots, num_tokens, k_pages, v_pages, layout, stream);
}

int codec_append_by_axes(const codec_head_config *head, const codec_rotary_axes *rotary, const codec_rows *q, const codec_rows *q_out,
                         const codec_rows *k, const codec_rows *v, const int64_t *positions, const int64_t *slots, int32_t num_tokens,
                         void *k_pages, void *v_pages, const codec_kv_layout *layout, void *stream)
{
    if (!rotary) return CODEC_ERR_INVALID_ARGUMENT;
    return append_rows(head, &rotary->rotary, rotary, q, q_out, k, v, positions, slots, num_tokens, k_pages, v_pages, layout, stream);
}

int codec_cache_copy(const codec_head_config *head, const codec_kv_layout *layout, int32_t num_layers, void *const *k_pages,
                     void *const *v_pages, const codec_run *runs, int32_t num_runs, void *stream)
{
    if (!head || !layout || num_layers < 1 || num_runs < 0) return CODEC_ERR_INVALID_ARGUMENT;
    if (int st = check_head(*head)) return st;
    if (pool_span(*head, *layout) < 0) return CODEC_ERR_INVALID_ARGUMENT;
    if (layout->num_pages * head->page_size > int64_t(1) << 32) return CODEC_ERR_UNSUPPORTED;      // slots are 32-bit: 512 GB a pool
    if (!k_pages || !v_pages || (num_runs && !runs)) return CODEC_ERR_INVALID_ARGUMENT;
    for (int32_t l = 0; l < num_layers; ++l)
        if (!k_pages[l] || !v_pages[l] || !aligned16(k_pages[l]) || !aligned16(v_pages[l]) || !pools_apart(*head, *layout, k_pages[l], v_pages[l])) return CODEC_ERR_INVALID_ARGUMENT;
    if (num_runs == 0) return CODEC_OK;
    const int32_t ps = head->page_size;
    for (int32_t i = 0; i < num_runs; ++i) {
        const codec_run &r = runs[i];
        if (r.src_page < 0 || r.src_page >= layout->num_pages || r.dst_page < 0 || r.dst_page >= layout->num_pages) return CODEC_ERR_INVALID_ARGUMENT;
        if (r.tokens < 1 || r.tokens > ps || r.src_token < 0 || r.src_token > ps - r.tokens || r.dst_token < 0 || r.dst_token > ps - r.tokens) return CODEC_ERR_INVALID_ARGUMENT;
    }
    try {
        if (runs_collide(runs, num_runs, ps)) return CODEC_ERR_INVALID_ARGUMENT;
    } catch (const std::bad_alloc &) {
        return CODEC_ERR_OUT_OF_MEMORY;
    }

    codec::CopyParams p{};
    p.page_stride = 2 * layout->page_stride;
    p.slot_stride = 2 * layout->token_stride;
    p.head_stride = 2 * layout->head_stride;
    p.heads = head->num_kv_heads;
    p.head_bytes = 2 * head->head_dim;
    while ((1 << p.page_shift) < ps) ++p.page_shift;
    double tokens = 0.0;
    for (int32_t i = 0; i < num_runs; ++i) tokens += runs[i].tokens;
    const double read = 2.0 * tokens * num_layers * p.heads * p.head_bytes;
    p.large = 2.0 * read > codec::kLargeBytes;
    p.huge = read > codec::kHugeBytes;
    for (int64_t first = 0; first < 2 * int64_t(num_layers); first += codec::kCopyPools) {
        p.num_pools = int32_t(std::min<int64_t>(codec::kCopyPools, 2 * int64_t(num_layers) - first));
        for (int32_t i = 0; i < p.num_pools; ++i) p.pools[i] = static_cast<char *>(((first + i) & 1 ? v_pages : k_pages)[(first + i) / 2]);
        for (int32_t at = 0; at < num_runs; at += codec::kCopyRuns) {
            p.num_runs = std::min(codec::kCopyRuns, num_runs - at);
            p.most_tokens = 0;
            for (int32_t i = 0; i < p.num_runs; ++i) {
                const codec_run &r = runs[at + i];
                p.runs[i] = {uint32_t(r.src_page) * uint32_t(ps) + uint32_t(r.src_token), uint32_t(r.dst_page) * uint32_t(ps) + uint32_t(r.dst_token), uint32_t(r.tokens)};
                p.most_tokens = std::max(p.most_tokens, r.tokens);
            }
            if (int e = codec::launch_copy(p, stream)) return hip_failure("page copy launch", e);
        }
    }
    return CODEC_OK;
}

int codec_block_table(int32_t page_size, int32_t num_seq, const int32_t *page_off, const int32_t *page_ids, int32_t num_ids,
                      const int32_t *tokens, int32_t *table, int64_t table_stride, int32_t width, void *stream)
{
    if (num_seq < 0 || num_seq > kMaxSequences || num_ids < 0 || width < 0 || table_stride < width || table_stride > kMaxSpan / kMaxSequences) return CODEC_ERR_INVALID_ARGUMENT;
    if (!page_size_ok(page_size)) return CODEC_ERR_UNSUPPORTED;
    if (num_seq == 0 || width == 0) return CODEC_OK;
    if (!page_off || (num_ids && !page_ids) || !tokens || !table) return CODEC_ERR_INVALID_ARGUMENT;
    for (const void *p : {static_cast<const void *>(page_off), static_cast<const void *>(page_ids), static_cast<const void *>(tokens), static_cast<const void *>(table)})
        if (reinterpret_cast<uintptr_t>(p) % 4) return CODEC_ERR_INVALID_ARGUMENT;
    const Range written = bytes_at(table, 4 * ((num_seq - 1) * table_stride + width));
    if (overlap(written, bytes_at(page_off, 4 * (int64_t(num_seq) + 1))) || overlap(written, bytes_at(page_ids, 4 * int64_t(num_ids))) ||
        overlap(written, bytes_at(tokens, 4 * int64_t(num_seq))))
        return CODEC_ERR_INVALID_ARGUMENT;
    codec::TableParams p{};
    p.page_off = page_off;
    p.page_ids = page_ids;
    p.tokens = tokens;
    p.table = table;
    p.table_stride = table_stride;
    p.num_ids = num_ids;
    p.num_seq = num_seq;
    p.width = width;
    while ((1 << p.page_shift) < page_size) ++p.page_shift;
    if (int e = codec::launch_block_table(p, stream)) return hip_failure("block table launch", e);
    return CODEC_OK;
}

size_t codec_slot_workspace_bytes(const codec_slot_config *config)
{
    return config && config->num_seq > codec::kSlotsAtOnce && config->num_seq <= kMaxSequences ? align_up(8 * size_t(config->num_seq) + 4) : 0;
}

int codec_slot_map(const codec_slot_config *config, int32_t *table, const int32_t *tokens, const int32_t *new_tokens, const int64_t *before,
                   const int32_t *spare, int64_t *positions, int64_t *slots, int32_t *sequences, int32_t *offsets, int32_t *tokens_out,
                   int32_t *taken, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!config) return CODEC_ERR_INVALID_ARGUMENT;
    const codec_slot_config &c = *config;
    if (c.num_seq < 0 || c.num_seq > kMaxSequences || c.width < 0 || c.num_tokens < 0 || c.num_spare < 0 || c.num_pages < 0 ||
        c.num_pages > (int64_t(1) << 31) || c.table_stride < c.width || c.table_stride > kMaxSpan / kMaxSequences)
        return CODEC_ERR_INVALID_ARGUMENT;
    if (!page_size_ok(c.page_size)) return CODEC_ERR_UNSUPPORTED;
    const size_t need = codec_slot_workspace_bytes(config);
    if (workspace_bytes < need) return CODEC_ERR_WORKSPACE_TOO_SMALL;
    if (need && !workspace) return CODEC_ERR_INVALID_ARGUMENT;
    if (!offsets || !taken || (c.num_seq && (!tokens || !new_tokens || !tokens_out)) || (c.num_seq && c.width && !table) ||
        (c.num_tokens && (!positions || !slots)))
        return CODEC_ERR_INVALID_ARGUMENT;
    if (reinterpret_cast<uintptr_t>(need ? workspace : nullptr) % 256) return CODEC_ERR_INVALID_ARGUMENT;
    for (const void *p : {static_cast<const void *>(table), static_cast<const void *>(tokens), static_cast<const void *>(new_tokens),
                          static_cast<const void *>(spare), static_cast<const void *>(sequences), static_cast<const void *>(offsets),
                          static_cast<const void *>(tokens_out), static_cast<const void *>(taken)})
        if (reinterpret_cast<uintptr_t>(p) % 4) return CODEC_ERR_INVALID_ARGUMENT;
    for (const void *p : {static_cast<const void *>(before), static_cast<const void *>(positions), static_cast<const void *>(slots)})
        if (reinterpret_cast<uintptr_t>(p) % 8) return CODEC_ERR_INVALID_ARGUMENT;
    {
        // what is written is neither read elsewhere nor written twice; the table is written only where pages are taken for it
        const int64_t n = c.num_seq, t = c.num_tokens, rows = n && c.width ? (n - 1) * c.table_stride + c.width : 0;
        const Range out[] = {bytes_at(positions, 8 * t), bytes_at(slots, 8 * t), bytes_at(sequences, sequences ? 4 * t : 0), bytes_at(offsets, 4 * (n + 1)),
                             bytes_at(tokens_out, 4 * n), bytes_at(taken, 4), bytes_at(workspace, int64_t(need)), bytes_at(table, 4 * rows)};
        const Range in[] = {bytes_at(tokens, 4 * n), bytes_at(new_tokens, 4 * n), bytes_at(before, before ? 8 * n : 0), bytes_at(spare, spare ? 4 * int64_t(c.num_spare) : 0)};
        auto meet = [](const Range &a, const Range &b) { return a.begin < a.end && b.begin < b.end && overlap(a, b); };
        for (int i = 0; i < 8; ++i) {
            for (int j = i + 1; j < 8; ++j)
                if (meet(out[i], out[j])) return CODEC_ERR_INVALID_ARGUMENT;
            for (const Range &r : in)
                if (meet(out[i], r) && (i < 7 || spare)) return CODEC_ERR_INVALID_ARGUMENT;
        }
    }
    codec::SlotParams p{};
    p.table = table;
    p.table_stride = c.table_stride;
    p.num_pages = c.num_pages;
    p.tokens = tokens;
    p.new_tokens = new_tokens;
    p.before = before;
    p.spare = spare;
    p.positions = positions;
    p.slots = slots;
    p.sequences = sequences;
    p.offsets = offsets;
    p.tokens_out = tokens_out;
    p.taken = taken;
    p.sums = static_cast<uint32_t *>(workspace);
    p.num_seq = c.num_seq;
    p.width = c.width;
    p.num_tokens = c.num_tokens;
    p.num_spare = c.num_spare;
    while ((1 << p.page_shift) < c.page_size) ++p.page_shift;
    if (int e = codec::launch_slot_map(p, stream)) return hip_failure("slot map launch", e);
    return CODEC_OK;
}

size_t codec_beam_workspace_bytes(const codec_beam_config *config)
{
    if (!config || check_beams(*config)) return 0;
    return std::max<size_t>(beam_scratch(*config).total, 256);
}

int codec_beam_select(const codec_beam_config *config, const void *logits, int64_t batch_stride, int64_t beam_stride, const float *scores,
                      const uint8_t *finished, float *out_scores, int32_t *out_beams, int32_t *out_tokens, void *workspace,
                      size_t workspace_bytes, void *stream)
{
    if (!config) return CODEC_ERR_INVALID_ARGUMENT;
    const codec_beam_config &c = *config;
    if (int st = check_beams(c)) return st;
    if (c.batch == 0) return CODEC_OK;
    if (!logits || !scores || !out_scores || !out_beams || !out_tokens || !workspace) return CODEC_ERR_INVALID_ARGUMENT;
    const int size = c.dtype == CODEC_DTYPE_FP32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(workspace) % 256) return CODEC_ERR_INVALID_ARGUMENT;
    if (batch_stride < 0 || beam_stride < 0 || batch_stride > kMaxSpan / c.batch || beam_stride > kMaxSpan / c.beams) return CODEC_ERR_INVALID_ARGUMENT;
    if (finished && (c.eos < 0 || c.eos >= c.vocab)) return CODEC_ERR_INVALID_ARGUMENT;
    const BeamScratch s = beam_scratch(c);
    if (workspace_bytes < s.total) return CODEC_ERR_WORKSPACE_TOO_SMALL;
    {
        // what is written is neither read nor written twice; scores may go back to where they came from, search by search
        const int64_t rows = int64_t(c.batch) * c.beams, span = (c.batch - 1) * batch_stride + (c.beams - 1) * beam_stride + c.vocab;
        const Range out[] = {bytes_at(out_scores, 4 * int64_t(c.batch) * c.k), bytes_at(out_beams, 4 * int64_t(c.batch) * c.k),
                             bytes_at(out_tokens, 4 * int64_t(c.batch) * c.k), bytes_at(workspace, int64_t(s.total))};
        const Range in[] = {bytes_at(logits, size * span), bytes_at(scores, 4 * rows), bytes_at(finished, finished ? rows : 0)};
        for (int i = 0; i < 4; ++i) {
            for (int j = i + 1; j < 4; ++j)
                if (overlap(out[i], out[j])) return CODEC_ERR_INVALID_ARGUMENT;
            for (int j = 0; j < 3; ++j)
                if (overlap(out[i], in[j]) && !(i == 0 && j == 1 && out_scores == scores && c.k == c.beams)) return CODEC_ERR_INVALID_ARGUMENT;
        }
    }

    char *ws = static_cast<char *>(workspace);
    codec::BeamParams p{};
    p.logits = static_cast<const char *>(logits);
    p.batch_stride = batch_stride;
    p.beam_stride = beam_stride;
    p.scores = scores;
    p.finished = finished;
    p.out_scores = out_scores;
    p.out_beams = out_beams;
    p.out_tokens = out_tokens;
    p.best = reinterpret_cast<uint64_t *>(ws);
    p.sums = reinterpret_cast<codec::PartialSum *>(ws + s.sums);
    p.parts = s.parts;
    p.batch = c.batch;
    p.beams = c.beams;
    p.vocab = c.vocab;
    p.k = c.k;
    p.kept = std::min(c.k, c.vocab);
    p.eos = c.eos;
    if (int e = codec::launch_beam_select(p, c.dtype, stream)) return hip_failure("beam selection launch", e);
    return CODEC_OK;
}

int codec_beam_reorder(const codec_state *states, int32_t num_states, const int32_t *beams, int32_t batch, int32_t beams_in,
                       int32_t beams_out, void *stream)
{
    if (num_states < 0 || batch < 0 || beams_in < 1 || beams_out < 1 || int64_t(batch) * beams_out > (1 << 22)) return CODEC_ERR_INVALID_ARGUMENT;
    if (num_states == 0 || batch == 0) return CODEC_OK;
    if (!states || !beams) return CODEC_ERR_INVALID_ARGUMENT;
    struct Touched { Range range; bool written; };
    std::vector<Touched> touched;
    try {
        touched.reserve(2 * size_t(num_states) + 1);
    } catch (const std::bad_alloc &) {
        return CODEC_ERR_OUT_OF_MEMORY;
    }
    touched.push_back({{reinterpret_cast<const char *>(beams), reinterpret_cast<const char *>(beams + int64_t(batch) * beams_out)}, false});
    uint64_t bits = 0;                      // of every address, stride and size: their common factor of two
    for (int32_t i = 0; i < num_states; ++i) {
        const codec_state &s = states[i];
        if (s.row_bytes < 0) return CODEC_ERR_INVALID_ARGUMENT;
        if (s.row_bytes == 0) continue;
        if (!s.src || !s.dst) return CODEC_ERR_INVALID_ARGUMENT;
        const int64_t src_span = state_span(s.row_bytes, batch, s.src_batch_stride, beams_in, s.src_beam_stride);
        Extent dims[] = {{batch, s.dst_batch_stride}, {beams_out, s.dst_beam_stride}};
        const int64_t dst_span = state_span(s.row_bytes, batch, s.dst_batch_stride, beams_out, s.dst_beam_stride);
        if (src_span < 0 || dst_span < 0 || separate_span(s.row_bytes, dims) < 0) return CODEC_ERR_INVALID_ARGUMENT;
        const char *src = static_cast<const char *>(s.src), *dst = static_cast<const char *>(s.dst);
        touched.push_back({{src, src + src_span}, false});
        touched.push_back({{dst, dst + dst_span}, true});
        bits |= reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | uint64_t(s.row_bytes);
        if (batch > 1) bits |= uint64_t(s.src_batch_stride) | uint64_t(s.dst_batch_stride);
        if (beams_in > 1) bits |= uint64_t(s.src_beam_stride);
        if (beams_out > 1) bits |= uint64_t(s.dst_beam_stride);
    }
    // a sweep over the ranges by their begin: what is read must end before what is written begins, and the other way round
    std::sort(touched.begin(), touched.end(), [](const Touched &a, const Touched &b) { return a.range.begin < b.range.begin; });
    const char *read_end = nullptr, *written_end = nullptr;
    for (const Touched &t : touched) {
        if (t.range.begin < (t.written ? read_end : written_end)) return CODEC_ERR_INVALID_ARGUMENT;
        const char *&end = t.written ? written_end : read_end;
        end = std::max(end, t.range.end);
    }
    const int unit = bits & 1 ? 1 : bits & 2 ? 2 : bits & 4 ? 4 : bits & 8 ? 8 : 16;

    codec::ReorderParams p{};
    p.beams = beams;
    p.batch = batch;
    p.beams_in = beams_in;
    p.beams_out = beams_out;
    double row_bytes = 0.0;
    for (int32_t i = 0; i < num_states; ++i) row_bytes += double(states[i].row_bytes);
    p.large = 2.0 * row_bytes * batch * beams_out > codec::kLargeBytes;
    for (int32_t i = 0; i < num_states; ++i) {
        const codec_state &s = states[i];
        if (s.row_bytes) {
            p.states[p.num_states++] = {static_cast<const char *>(s.src), static_cast<char *>(s.dst), s.src_batch_stride, s.src_beam_stride,
                                        s.dst_batch_stride, s.dst_beam_stride, s.row_bytes / unit};
            p.most_units = std::max(p.most_units, s.row_bytes / unit);
        }
        if (p.num_states == codec::kReorderStates || (i == num_states - 1 && p.num_states)) {
            if (int e = codec::launch_reorder(p, unit, stream)) return hip_failure("beam reorder launch", e);
            p.num_states = 0;
            p.most_units = 0;
        }
    }
    return CODEC_OK;
}

}  // extern "C"
