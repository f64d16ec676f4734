// The cache's shape and book as its kernels take them (rr_cache.cu, rr_attend.cu).  Not
// part of the public ABI; include/rr.h has the layout.
#pragma once

#include "rr_kernels.cuh"

namespace {

// Words of the book's control block.
// kState: why a call was not done; kLate: what calls found that were done but for it.
enum { kState = 0, kLate = 1, kMoves = 2, kUsed = 3 };
constexpr int kControlWords = 64;

// Bits of its state.
enum { kBadRange = 1, kBadTwice = 2, kBadPool = 4, kBadChild = 8, kBadTable = 16, kBadWait = 32 };

struct Book {
    int32_t *control, *table, *lengths, *refs;
    // Within one call:
    int64_t* sums;           // in the control block: what each block counted
    int32_t *held, *last;    // per page, zero between calls: listed holders, the last of them
    int32_t *free;           // pages to be taken, or a moved page's new place
    int32_t *plan;           // per listed sequence: its place among `free`
    int4* moves;             // from, to, tokens
};

struct CacheShape {
    int32_t n_kv, dim, pitch, page, shift;       // page = 1 << shift tokens
    int32_t n_pages, max_seqs, max_pages;
    int32_t runs;                                // of a page: layers x keys and values x heads,
    int64_t run_bytes, layer_bytes, page_bytes;  //   one head's rows each

    __device__ __forceinline__ bool has_seq(int s) const { return unsigned(s) < unsigned(max_seqs); }
    __device__ __forceinline__ bool has_page(int p) const { return unsigned(p) < unsigned(n_pages); }
    __device__ __forceinline__ int64_t max_length() const { return int64_t(max_pages) << shift; }
    __device__ __forceinline__ bool has_length(int n) const { return n >= 0 && n <= max_length(); }
};

inline rr_status check_cache(const rr_cache* C) {
    if (!C) return rr_fail(RR_EINVAL, "cache is NULL");
    if (C->layers < 1 || C->layers > 1024 || C->n_kv < 1 || C->n_kv > 1024 || C->dim < 1 || C->dim > 256)
        return rr_fail(RR_ELAYOUT, "%d layers of %d heads of %d: 1..1024, 1..1024 and 1..256", C->layers, C->n_kv, C->dim);
    if (C->page_tokens < 8 || C->page_tokens > 128 || (C->page_tokens & (C->page_tokens - 1)))
        return rr_fail(RR_ELAYOUT, "pages of %d tokens: 8, 16, 32, 64 or 128", C->page_tokens);
    if (C->n_pages < 1 || C->n_pages > 1 << 26 || C->max_seqs < 1 || C->max_seqs > 1 << 16 || C->max_pages < 1)
        return rr_fail(RR_ELAYOUT, "%d pages, %d sequences of up to %d: 1..2^26, 1..65536 and 1 or more", C->n_pages, C->max_seqs,
                       C->max_pages);
    if (int64_t(C->max_pages) * C->page_tokens > 1 << 30)
        return rr_fail(RR_ELAYOUT, "sequences of up to %d pages of %d: 2^30 tokens at most", C->max_pages, C->page_tokens);
    if (C->dtype != RR_DST_BF16 && C->dtype != RR_DST_F16) return rr_fail(RR_EINVAL, "unknown element type %d", C->dtype);
    return RR_OK;
}

inline CacheShape shape_of(const rr_cache* C) {
    CacheShape c;
    c.n_kv = C->n_kv;
    c.dim = C->dim;
    c.pitch = (C->dim + 7) / 8 * 8;
    c.page = C->page_tokens;
    for (c.shift = 0; 1 << c.shift < c.page; ++c.shift) {}
    c.n_pages = C->n_pages;
    c.max_seqs = C->max_seqs;
    c.max_pages = C->max_pages;
    c.runs = C->layers * 2 * C->n_kv;
    c.run_bytes = int64_t(c.page) * c.pitch * 2;
    c.layer_bytes = c.run_bytes * 2 * C->n_kv;
    c.page_bytes = c.run_bytes * c.runs;
    return c;
}

// The book's parts, 16-byte aligned; returns its bytes.
inline int64_t book_of(const rr_cache* C, void* book, Book* b) {
    int32_t* const base = static_cast<int32_t*>(book);
    int64_t at = kControlWords;
    const auto part = [&](int64_t words) {
        const int64_t here = at;
        at += (words + 3) / 4 * 4;
        return here;
    };
    const int64_t table = part(int64_t(C->max_seqs) * C->max_pages), lengths = part(C->max_seqs), refs = part(C->n_pages),
                  held = part(C->n_pages), last = part(C->n_pages), free = part(C->n_pages), plan = part(C->max_seqs),
                  moves = part(4 * int64_t(C->n_pages));
    if (b) {
        b->control = base;
        b->sums = reinterpret_cast<int64_t*>(base + 16);
        b->table = base + table;
        b->lengths = base + lengths;
        b->refs = base + refs;
        b->held = base + held;
        b->last = base + last;
        b->free = base + free;
        b->plan = base + plan;
        b->moves = reinterpret_cast<int4*>(base + moves);
    }
    return at * 4;
}

}  // namespace
