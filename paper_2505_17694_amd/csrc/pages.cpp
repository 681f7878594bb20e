// Who holds the pages of a cache: page lists that share pages, branches, moves to the low ids.
#include <climits>
#include <cstdint>
#include <new>
#include <vector>

#include "codec.h"

struct codec_pages {
    std::vector<int32_t> holders;
    std::vector<uint64_t> free_bits;    // bit p % 64 of word p / 64: page p has no holder
    size_t first_word = 0;              // no free page below this word
    int32_t num_free = 0;

    int32_t size() const { return int32_t(holders.size()); }

    int32_t take_lowest()               // there has to be one
    {
        while (!free_bits[first_word]) ++first_word;
        const int bit = __builtin_ctzll(free_bits[first_word]);
        free_bits[first_word] &= free_bits[first_word] - 1;
        --num_free;
        return int32_t(first_word * 64 + bit);
    }
    void set_free(int32_t page)
    {
        const size_t word = size_t(page) / 64;
        free_bits[word] |= uint64_t(1) << (page % 64);
        if (word < first_word) first_word = word;
        ++num_free;
    }
    void set_held(int32_t page)
    {
        free_bits[size_t(page) / 64] &= ~(uint64_t(1) << (page % 64));
        --num_free;
    }
    bool in_range(const int32_t *ids, int64_t n) const
    {
        for (int64_t i = 0; i < n; ++i)
            if (ids[i] < 0 || ids[i] >= size()) return false;
        return true;
    }
    // One holder less for every entry; false, and nothing changed, if one has none left.  Free pages are not marked yet.
    bool let_go(const int32_t *ids, int64_t n)
    {
        for (int64_t i = 0; i < n; ++i)
            if (holders[ids[i]]-- == 0) {
                for (; i >= 0; --i) ++holders[ids[i]];
                return false;
            }
        return true;
    }
    void mark_free(const int32_t *ids, int64_t n)
    {
        for (int64_t i = 0; i < n; ++i) {
            const bool marked = free_bits[size_t(ids[i]) / 64] >> (ids[i] % 64) & 1;
            if (holders[ids[i]] == 0 && !marked) set_free(ids[i]);
        }
    }
};

extern "C" {

int codec_pages_create(int32_t num_pages, codec_pages_t **out)
{
    if (!out || num_pages < 1) return CODEC_ERR_INVALID_ARGUMENT;
    codec_pages *p = new (std::nothrow) codec_pages;
    if (!p) return CODEC_ERR_OUT_OF_MEMORY;
    try {
        p->holders.assign(size_t(num_pages), 0);
        p->free_bits.assign((size_t(num_pages) + 63) / 64, ~uint64_t(0));
    } catch (const std::bad_alloc &) {
        delete p;
        return CODEC_ERR_OUT_OF_MEMORY;
    }
    if (num_pages % 64) p->free_bits.back() = (uint64_t(1) << (num_pages % 64)) - 1;
    p->num_free = num_pages;
    *out = p;
    return CODEC_OK;
}

int codec_pages_destroy(codec_pages_t *pages)
{
    delete pages;
    return CODEC_OK;
}

int32_t codec_pages_free(const codec_pages_t *pages) { return pages ? pages->num_free : CODEC_ERR_INVALID_ARGUMENT; }

int codec_pages_take(codec_pages_t *pages, int32_t n, int32_t *ids)
{
    if (!pages || n < 0 || (n && !ids)) return CODEC_ERR_INVALID_ARGUMENT;
    if (n > pages->num_free) return CODEC_ERR_NO_PAGES;
    for (int32_t i = 0; i < n; ++i) {
        ids[i] = pages->take_lowest();
        pages->holders[ids[i]] = 1;
    }
    return CODEC_OK;
}

int codec_pages_hold(codec_pages_t *pages, const int32_t *ids, int32_t n)
{
    if (!pages || n < 0 || (n && !ids) || !pages->in_range(ids, n)) return CODEC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < n; ++i)
        if (pages->holders[ids[i]] > INT_MAX - n) return CODEC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < n; ++i)
        if (pages->holders[ids[i]]++ == 0) pages->set_held(ids[i]);
    return CODEC_OK;
}

int codec_pages_release(codec_pages_t *pages, const int32_t *ids, int32_t n)
{
    if (!pages || n < 0 || (n && !ids) || !pages->in_range(ids, n)) return CODEC_ERR_INVALID_ARGUMENT;
    if (!pages->let_go(ids, n)) return CODEC_ERR_INVALID_ARGUMENT;
    pages->mark_free(ids, n);
    return CODEC_OK;
}

int codec_pages_fork(codec_pages_t *pages, int32_t page_size, int32_t num_seq, const int32_t *page_off, const int32_t *page_ids,
                     const int32_t *tokens, int32_t num_out, const int32_t *parents, int32_t *out_off, int32_t *out_ids,
                     int32_t out_capacity, codec_run *runs, int32_t *num_runs)
{
    if (!pages || page_size < 1 || num_seq < 0 || num_out < 0 || out_capacity < 0 || !page_off || !out_off || !num_runs) return CODEC_ERR_INVALID_ARGUMENT;
    if ((num_seq && !tokens) || (num_out && (!parents || !runs)) || page_off[0] != 0) return CODEC_ERR_INVALID_ARGUMENT;
    for (int32_t s = 0; s < num_seq; ++s) {
        const int64_t have = int64_t(page_off[s + 1]) - page_off[s];
        if (have < 0 || tokens[s] < 0 || tokens[s] > have * page_size) return CODEC_ERR_INVALID_ARGUMENT;
    }
    const int64_t listed = page_off[num_seq];
    if ((listed && !page_ids) || !pages->in_range(page_ids, listed)) return CODEC_ERR_INVALID_ARGUMENT;
    int64_t total = 0;
    for (int32_t j = 0; j < num_out; ++j) {
        if (parents[j] < 0 || parents[j] >= num_seq) return CODEC_ERR_INVALID_ARGUMENT;
        total += page_off[parents[j] + 1] - page_off[parents[j]];
    }
    if (total > out_capacity) return CODEC_ERR_WORKSPACE_TOO_SMALL;
    if (total && !out_ids) return CODEC_ERR_INVALID_ARGUMENT;

    // Per sequence: its pages that are not full, whether it alone holds them (kept by the first that goes on)
    std::vector<char> keeps;
    try {
        keeps.assign(size_t(num_seq), 0);
    } catch (const std::bad_alloc &) {
        return CODEC_ERR_OUT_OF_MEMORY;
    }
    auto open_of = [&](int32_t s) { return page_off[s] + tokens[s] / page_size; };
    for (int32_t s = 0; s < num_seq; ++s) {
        keeps[s] = 1;
        for (int32_t i = open_of(s); i < page_off[s + 1]; ++i)
            if (pages->holders[page_ids[i]] != 1) keeps[s] = 0;
    }
    if (!pages->let_go(page_ids, listed)) return CODEC_ERR_INVALID_ARGUMENT;
    int64_t need = 0;
    {
        // `keeps` is 2 once the first has gone on with the open pages
        for (int32_t j = 0; j < num_out; ++j) {
            const int32_t s = parents[j];
            if (keeps[s] == 1) keeps[s] = 2;
            else need += page_off[s + 1] - open_of(s);
        }
        for (int32_t s = 0; s < num_seq; ++s) keeps[s] = keeps[s] != 0;
    }
    if (need > pages->num_free) {
        for (int64_t i = 0; i < listed; ++i) ++pages->holders[page_ids[i]];
        return CODEC_ERR_NO_PAGES;
    }

    int32_t at = 0, n = 0;
    out_off[0] = 0;
    for (int32_t j = 0; j < num_out; ++j) {
        const int32_t s = parents[j], open = open_of(s);
        for (int32_t i = page_off[s]; i < page_off[s + 1]; ++i) {
            int32_t page = page_ids[i];
            if (i >= open && keeps[s] != 1) {
                page = pages->take_lowest();
                if (i == open && tokens[s] % page_size) runs[n++] = {page_ids[i], 0, page, 0, tokens[s] % page_size};
            }
            ++pages->holders[page];
            out_ids[at++] = page;
        }
        keeps[s] = keeps[s] == 1 ? 2 : keeps[s];
        out_off[j + 1] = at;
    }
    pages->mark_free(page_ids, listed);
    *num_runs = n;
    return CODEC_OK;
}

int codec_pages_compact(codec_pages_t *pages, int32_t page_size, codec_run *runs, int32_t capacity, int32_t *num_runs)
{
    if (!pages || page_size < 1 || capacity < 0 || (capacity && !runs) || !num_runs) return CODEC_ERR_INVALID_ARGUMENT;
    const int32_t held = pages->size() - pages->num_free;
    int32_t moves = 0;
    for (int32_t p = held; p < pages->size(); ++p) moves += pages->holders[p] != 0;
    if (moves > capacity) return CODEC_ERR_WORKSPACE_TOO_SMALL;
    int32_t to = 0;
    moves = 0;
    for (int32_t p = held; p < pages->size(); ++p) {
        if (pages->holders[p] == 0) continue;
        while (pages->holders[to] != 0) ++to;
        pages->holders[to] = pages->holders[p];
        pages->set_held(to);
        pages->holders[p] = 0;
        pages->set_free(p);
        runs[moves++] = {p, 0, to, 0, page_size};
    }
    *num_runs = moves;
    return CODEC_OK;
}

}  // extern "C"
