// The K/V cache in pages: what its kernels share (paged_book.hip: tables, page copies, new rows; paged_attn.hip: attention).
#pragma once
#include "kernels.h"

#define PG_MAX_SEQS 4096
#define PG_MAX_PAGES (1 << 24)

// A cache as its kernels see it.  Pools are [layer][page][kv head][1 << pb][32 * Dh] elements: blocks of 32 positions in the
// order of k_index and v_index.
struct PagedView {
    int32_t L, N, pb, Hkv, Dh, S, MP;      // pb: log2 of the blocks of a page
    char* k; char* v;
    int32_t* table; int32_t* len; int32_t* ref;
};
// Rows of a pass: sequence i of it has rows first .. first + count - 1.
struct PagedRows {
    int32_t B, R, n_rows;                  // sequences, most rows of one, rows of the buffers
    const int32_t* seqs; const int32_t* start;
};
#if defined(__HIPCC__)
// (what the device arrays hold is checked here: whatever they hold, rows lie inside 0 .. n_rows - 1 and sequences inside the table)
__device__ inline int pg_seq(const PagedRows& r, const PagedView& c, int i) {
    const int s = r.seqs ? r.seqs[i] : i;
    return s >= 0 && s < c.S ? s : -1;
}
__device__ inline void pg_rows(const PagedRows& r, int i, int& first, int& count) {
    if (!r.start) { first = i * r.R; count = r.R; return; }
    int a = r.start[i], b = r.start[i + 1];
    a = a < 0 ? 0 : a < r.n_rows ? a : r.n_rows;
    b = b < a ? a : b < r.n_rows ? b : r.n_rows;
    first = a; count = b - a < r.R ? b - a : r.R;
}
// committed length of sequence s, with room for nothing that would pass the table
__device__ inline int pg_len(const PagedView& c, int s) {
    const int n = c.len[s], most = c.MP << (c.pb + 5);
    return n < 0 ? 0 : n < most ? n : most;
}
#endif

struct PagedJoin { int32_t row0, nrows, first, kvh, parts; };       // a unit whose parts a second launch joins; parts = 0: none
struct PagedAttnArgs {
    PagedView c;
    PagedRows r;
    const char* kl; const char* vl;        // the layer's part of the pools
    const void* q; int64_t q_row, q_head;
    void* out; int64_t out_row;
    float* lse;
    int32_t H, act;                        // act: 0 fp32, 1 bf16 rows
    int32_t g; uint32_t g_inv;             // query heads of a K/V head, and 2^32 / g rounded up
    int32_t esz;                           // bytes of a cached value
    int32_t window, sinks;                 // window 0: none, and no sinks
    uint32_t reach;                        // a row sees what lies less far back: the window, or 2^31
    int32_t whole;                         // most blocks of a unit that is not cut
    int32_t* cnt; PagedJoin* joins; float* part;       // hand-off of parts: counters (zero between launches), units to join, partial results
};
size_t fc_paged_attn_scratch_bytes(int Dh);
hipError_t fc_paged_attn(const PagedAttnArgs& a, hipStream_t st);
