// The K/V cache in pages: tables and use counts, copies of pages, K/V of new rows, and the C entry points.
//
// The bookkeeping of a call is one workgroup of sixteen waves: sixteen lanes look at an entry's part of the table, the entries' needs are
// summed in order, and the use counts are walked 4096 pages at a time until enough free ones are found, so that pages go out lowest
// first whatever the timing.  It is bound by its chain of dependent loads (entry, length, table, use counts), about a microsecond each.
// Page data move in blocks of 32 positions of one head (8 KB at 128 bf16 elements), a workgroup each: bound by HBM, bytes read and written once.
#include <limits.h>
#include <stdio.h>
#include "paged.h"
#include "gemmco.h"      // fc_num_cus

#define PG_WG 1024
#define PG_HEAD 16384        // bytes of the scratch in front of the lists: number of moves, at 256 the counters of 512 workgroups, at 4096 their units to join
#define NONE_FIRST INT_MAX

// exclusive prefix sum over the workgroup; *total: the sum.  lds: 17 ints
__device__ inline int pg_scan(int v, int* lds, int* total) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const int y = __shfl_up(x, d, 64); if (lane >= d) x += y; }
    __syncthreads();                              // (lds may still be read from the last call)
    if (lane == 63) lds[wv] = x;
    __syncthreads();
    if (wv == 0) {
        int t = lane < PG_WG / 64 ? lds[lane] : 0, y = t;
#pragma unroll
        for (int d = 1; d < PG_WG / 64; d <<= 1) { const int z = __shfl_up(y, d, 64); if (lane >= d) y += z; }
        if (lane < PG_WG / 64) lds[lane] = y - t;
        if (lane == PG_WG / 64 - 1) lds[16] = y;
    }
    __syncthreads();
    *total = lds[16];
    return lds[wv] + x - v;
}
// the lowest free pages, up to `want` of them, into list; how many there are (at most `want`).  For the whole workgroup
__device__ inline int pg_find_free(const PagedView& c, int want, int* list, int* lds) {
    int found = 0;
    for (int base = 0; base < c.N && found < want; base += 4 * PG_WG) {
        const int p0 = base + 4 * (int)threadIdx.x;
        int f[4], n = 0, total;
#pragma unroll
        for (int e = 0; e < 4; ++e) { f[e] = p0 + e < c.N && c.ref[p0 + e] == 0; n += f[e]; }
        int at = found + pg_scan(n, lds, &total);
#pragma unroll
        for (int e = 0; e < 4; ++e) if (f[e]) { if (at < want) list[at] = p0 + e; ++at; }
        found += total;
    }
    __syncthreads();
    return found < want ? found : want;
}
// index of the first entry of the call that names each sequence
__device__ inline void pg_first(const PagedView& c, int count, const int32_t* seqs, int* first) {
    for (int s = threadIdx.x; s < c.S; s += PG_WG) first[s] = NONE_FIRST;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += PG_WG) { const int s = seqs[i]; if (s >= 0 && s < c.S) atomicMin(&first[s], i); }
    __syncthreads();
}
__device__ inline bool pg_none(const PagedView& c, int page) { return page < 0 || page >= c.N; }
// number of set lanes among the sixteen of this one's group, and among those in front of it
__device__ inline int pg_group_count(bool x, int* before) {
    const int lane = threadIdx.x & 63;
    const uint32_t m = (uint32_t)(__ballot(x) >> (lane & 48)) & 0xFFFFu;
    *before = __popc(m & ((1u << (lane & 15)) - 1));
    return __popc(m);
}
// needs of the entries (below zero: a status) -> exclusive sums in pre; the sum of all.  For the whole workgroup
__device__ inline int pg_sum_needs(int count, const int* need, int* pre, int* lds) {
    int sum = 0;
    for (int base = 0; base < count; base += PG_WG) {
        const int i = base + threadIdx.x;
        int total;
        const int v = i < count && need[i] > 0 ? need[i] : 0, at = pg_scan(v, lds, &total);
        if (i < count) pre[i] = sum + at;
        sum += total;
    }
    __syncthreads();
    return sum;
}

// slots [n / P, end) of a sequence that the positions n .. n + rows - 1 fall into; end > MP: they pass the table
__device__ inline int64_t pg_end_slot(const PagedView& c, int n, int rows) {
    const int64_t P = (int64_t)32 << c.pb;
    return (n + (int64_t)rows + P - 1) >> (c.pb + 5);
}

__global__ __launch_bounds__(PG_WG) void k_paged_grow(PagedView c, int count, const int32_t* seqs, const int32_t* rows, int32_t* status, int* list) {
    __shared__ int first[PG_MAX_SEQS], need[PG_MAX_SEQS], pre[PG_MAX_SEQS], lds[17];
    const int grp = threadIdx.x >> 4, l = threadIdx.x & 15;
    pg_first(c, count, seqs, first);
    for (int i = grp; i < count; i += PG_WG / 16) {
        const int s = seqs[i], r = rows[i];
        int v = FASTCOT_EINVAL, before;
        if (s >= 0 && s < c.S && r >= 0 && first[s] == i) {
            const int n = pg_len(c, s);
            const int64_t end = pg_end_slot(c, n, r);
            v = FASTCOT_ECAPACITY;
            if (end <= c.MP) {
                v = 0;
                for (int k = n >> (c.pb + 5); k < end; k += 16) v += pg_group_count(k + l < end && pg_none(c, c.table[(size_t)s * c.MP + k + l]), &before);
            }
        }
        if (l == 0) need[i] = v;
    }
    __syncthreads();
    const int total = pg_sum_needs(count, need, pre, lds), found = pg_find_free(c, total, list, lds);
    for (int i = grp; i < count; i += PG_WG / 16) {
        const int v = need[i];
        const bool given = v >= 0 && (v == 0 || pre[i] + v <= found);
        if (l == 0 && status) status[i] = v < 0 ? v : given ? 0 : FASTCOT_ECAPACITY;
        if (v <= 0 || !given) continue;
        const int s = seqs[i], n = pg_len(c, s);
        const int end = (int)pg_end_slot(c, n, rows[i]);
        int at = pre[i], before;
        for (int k = n >> (c.pb + 5); k < end; k += 16) {
            const bool want = k + l < end && pg_none(c, c.table[(size_t)s * c.MP + k + l]);
            const int m = pg_group_count(want, &before);
            if (want) {
                const int page = list[at + before];
                c.table[(size_t)s * c.MP + k + l] = page;
                c.ref[page] = 1;
            }
            at += m;
        }
    }
}

__global__ __launch_bounds__(PG_WG) void k_paged_advance(PagedView c, int count, const int32_t* seqs, const int32_t* rows, int32_t* status) {
    __shared__ int first[PG_MAX_SEQS];
    const int grp = threadIdx.x >> 4, l = threadIdx.x & 15;
    pg_first(c, count, seqs, first);
    for (int i = grp; i < count; i += PG_WG / 16) {
        const int s = seqs[i], r = rows[i];
        int v = FASTCOT_EINVAL, before, n = 0;
        if (s >= 0 && s < c.S && r >= 0 && first[s] == i) {
            n = pg_len(c, s);
            const int64_t end = pg_end_slot(c, n, r);
            v = FASTCOT_ECAPACITY;
            if (end <= c.MP) {
                int missing = 0;
                for (int k = n >> (c.pb + 5); k < end; k += 16) missing += pg_group_count(k + l < end && pg_none(c, c.table[(size_t)s * c.MP + k + l]), &before);
                if (!missing) v = 0;
            }
        }
        if (l == 0) {
            if (v == 0) c.len[s] = n + r;
            if (status) status[i] = v;
        }
    }
}

// moves: list of page copies (from, to, blocks of 32 positions), their number in *n_moves
__global__ __launch_bounds__(PG_WG) void k_paged_fork(PagedView c, int count, const int32_t* src, const int32_t* dst, int32_t* status, int* n_moves, int* from,
                                                      int* to, int* blocks) {
    __shared__ int first[PG_MAX_SEQS], need[PG_MAX_SEQS], pre[PG_MAX_SEQS], lds[17];
    const int grp = threadIdx.x >> 4, l = threadIdx.x & 15, P = 32 << c.pb;
    pg_first(c, count, dst, first);
    for (int i = threadIdx.x; i < count; i += PG_WG) {
        const int s = src[i], d = dst[i];
        int v = FASTCOT_EINVAL;
        if (s >= 0 && s < c.S && d >= 0 && d < c.S && first[d] == i && first[s] == NONE_FIRST && c.len[d] == 0 && pg_none(c, c.table[(size_t)d * c.MP])) {
            const int n = pg_len(c, s);
            v = n & (P - 1) && !pg_none(c, c.table[(size_t)s * c.MP + (n >> (c.pb + 5))]);
        }
        need[i] = v;
    }
    __syncthreads();
    const int total = pg_sum_needs(count, need, pre, lds), found = pg_find_free(c, total, to, lds);
    for (int i = grp; i < count; i += PG_WG / 16) {
        const int v = need[i];
        const bool given = v >= 0 && (v == 0 || pre[i] < found);
        if (l == 0 && status) status[i] = v < 0 ? v : given ? 0 : FASTCOT_ECAPACITY;
        if (!given) continue;
        const int s = src[i], d = dst[i], n = pg_len(c, s), last = n >> (c.pb + 5);
        for (int k = l; k < last; k += 16) {
            const int page = c.table[(size_t)s * c.MP + k];
            c.table[(size_t)d * c.MP + k] = page;
            if (!pg_none(c, page)) atomicAdd(&c.ref[page], 1);
        }
        if (l == 0) {
            c.len[d] = n;
            if (v) {
                const int at = pre[i], page = to[at];
                c.table[(size_t)d * c.MP + last] = page;
                c.ref[page] = 1;
                from[at] = c.table[(size_t)s * c.MP + last];
                blocks[at] = ((n & (P - 1)) + 31) >> 5;
            }
        }
    }
    if (threadIdx.x == 0) *n_moves = found;
}

// a workgroup per entry; sinks < 0: every page leaves.  An entry exchanges what it takes out of the table, so one that is named twice leaves once
__global__ __launch_bounds__(256) void k_paged_leave(PagedView c, const int32_t* seqs, int window, int sinks, int32_t* status) {
    const int i = blockIdx.x, s = seqs[i];
    const bool ok = s >= 0 && s < c.S;
    if (threadIdx.x == 0 && status) status[i] = ok ? 0 : FASTCOT_EINVAL;
    if (!ok) return;
    const int P = 32 << c.pb, n = c.len[s];
    int k0 = 0, k1 = c.MP;
    if (sinks >= 0) {
        // pages k with k * P >= sinks and (k + 1) * P - 1 <= n - window
        k0 = (int)(((int64_t)sinks + P - 1) >> (c.pb + 5));
        const int64_t seen = (int64_t)n - window + 1;
        k1 = seen <= 0 ? 0 : (int)(seen >> (c.pb + 5));
        if (k1 > c.MP) k1 = c.MP;
    }
    for (int k = k0 + threadIdx.x; k < k1; k += 256) {
        const int page = atomicExch(&c.table[(size_t)s * c.MP + k], -1);
        if (!pg_none(c, page)) atomicSub(&c.ref[page], 1);
    }
    if (sinks < 0) {
        __syncthreads();
        if (threadIdx.x == 0) c.len[s] = 0;
    }
}

__global__ __launch_bounds__(PG_WG) void k_paged_compact(PagedView c, int32_t* d_used, int* n_moves, int* from, int* to, int* map) {
    __shared__ int lds[17];
    int used = 0, moves = 0, holes = 0, total;
    for (int base = 0; base < c.N; base += 4 * PG_WG) {
        const int p0 = base + 4 * (int)threadIdx.x;
        int n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) n += p0 + e < c.N && c.ref[p0 + e] > 0;
        pg_scan(n, lds, &total);
        used += total;
    }
    for (int base = 0; base < c.N; base += 4 * PG_WG) {
        const int p0 = base + 4 * (int)threadIdx.x;
        int in[4], n = 0;                                // pages that move in the upper half of a word, free places in the lower one
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int p = p0 + e;
            in[e] = p >= c.N ? 0 : c.ref[p] > 0 ? (p >= used ? 1 << 16 : 0) : p < used ? 1 : 0;
            if (p < c.N) map[p] = p;
            n += in[e];
        }
        const int at = pg_scan(n, lds, &total);
        int a = moves + (at >> 16), b = holes + (at & 0xFFFF);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (in[e] == 1) to[b++] = p0 + e;
            else if (in[e]) from[a++] = p0 + e;
        }
        moves += total >> 16;
        holes += total & 0xFFFF;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < moves; i += PG_WG) {   // (as many free places among the first `used` as pages in use behind them)
        c.ref[to[i]] = c.ref[from[i]];
        c.ref[from[i]] = 0;
        map[from[i]] = to[i];
    }
    if (threadIdx.x == 0) { *n_moves = moves; if (d_used) *d_used = used; }
}

// Copies page data by a list of moves, block by block: of a fork the first blocks[m] of each page, the copies of one block after each other (children of one
// sequence read it from the L2 then), of a compaction whole pages, and the table follows the map.  What is written goes past the caches, and what a
// compaction reads, once, too (15 children of a 7B sequence 274 us with everything cached, 308 with nothing, 189 so; 1.1 GB compacted 453, 426 so, of
// which 4.9 TB/s, the rate of a large copy, are 458).
template <bool FORK>
__global__ __launch_bounds__(256) void k_paged_move(PagedView c, int block16, const int* n_moves, const int* from, const int* to, const int* blocks, const int* map) {
    typedef __attribute__((__vector_size__(16))) uint32_t u32x4;
    const int moves = *n_moves, tid = threadIdx.x;
    if (!FORK)
        for (size_t i = (size_t)blockIdx.x * 256 + tid; i < (size_t)c.S * c.MP; i += (size_t)gridDim.x * 256) {
            const int page = c.table[i];
            if (!pg_none(c, page)) c.table[i] = map[page];
        }
    const int PB = 1 << c.pb;
    const int64_t per = (int64_t)c.L * 2 * c.Hkv << c.pb, all = per * moves;
    for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
        const int m = FORK ? (int)(x % moves) : (int)(x / per);
        const uint32_t y = FORK ? (uint32_t)(x / moves) : (uint32_t)(x - m * per), blk = y & (PB - 1), z = y >> c.pb, h = z % c.Hkv, w = z / c.Hkv;
        if (FORK && (int)blk >= blocks[m]) continue;
        char* pool = w & 1 ? c.v : c.k;
        const size_t layer = (size_t)(w >> 1) * c.N;
        const u32x4* a = (const u32x4*)pool + ((((layer + from[m]) * c.Hkv + h) << c.pb) + blk) * block16;
        u32x4* b = (u32x4*)pool + ((((layer + to[m]) * c.Hkv + h) << c.pb) + blk) * block16;
        for (int e = tid; e < block16; e += 256) __builtin_nontemporal_store(FORK ? a[e] : __builtin_nontemporal_load(a + e), b + e);
    }
}

__global__ __launch_bounds__(256) void k_paged_reset(PagedView c) {
    const size_t i0 = (size_t)blockIdx.x * 256 + threadIdx.x, step = (size_t)gridDim.x * 256;
    for (size_t i = i0; i < (size_t)c.S * c.MP; i += step) c.table[i] = -1;
    for (size_t i = i0; i < (size_t)c.S; i += step) c.len[i] = 0;
    for (size_t i = i0; i < (size_t)c.N; i += step) c.ref[i] = 0;
}

typedef __attribute__((__vector_size__(16))) uint32_t pg_u32x4;
// eight values next to each other, in the cache's type: one or two pieces of 16 bytes
template <typename T, typename A> __device__ inline void pg_load8(const A* p, pg_u32x4* to) {
    if constexpr (sizeof(A) == sizeof(T)) {
#pragma unroll
        for (unsigned w = 0; w < sizeof(T) / 2; ++w) to[w] = ((const pg_u32x4*)p)[w];
    } else {
        const float4 x = *(const float4*)p, y = *(const float4*)(p + 4);
        to[0] = (pg_u32x4){pk_bf16(x.x, x.y), pk_bf16(x.z, x.w), pk_bf16(y.x, y.y), pk_bf16(y.z, y.w)};
    }
}

// New rows into the pages, a workgroup per block of 32 positions and K/V head (grid: x over blocks and heads, y over sequences): rows come in whole lines,
// meet in LDS in the cache's type, and go out in the order of the block, in 16-byte pieces of whole lines (V: eight positions of a head element; pieces that
// the rows fill in part, value by value).  Bound by HBM, one token of each sequence by latency.  4096 fp32 rows of 32 heads, not in the caches: threads by
// eight elements of a row 143 us, by what they store without the LDS 56.
template <typename T, typename A>
__global__ __launch_bounds__(256) void k_paged_write(PagedView c, PagedRows r, T* kl, T* vl, const A* k, const A* v, int64_t row_stride) {
    constexpr int E = 16 / sizeof(T), W = sizeof(T) / 2;       // values of a piece, pieces of eight values
    extern __shared__ __align__(16) char lds[];
    const int i = blockIdx.y, s = pg_seq(r, c, i), G = c.Dh >> 5, D8 = c.Dh >> 3, tid = threadIdx.x;
    if (s < 0) return;
    int first, count;
    pg_rows(r, i, first, count);
    const int n = pg_len(c, s), h = blockIdx.x % c.Hkv, blk = (n >> 5) + blockIdx.x / c.Hkv, p0 = blk << 5;
    const int slot = blk >> c.pb;
    if (p0 >= n + count || slot >= c.MP) return;
    const int page = c.table[(size_t)s * c.MP + slot];
    if (pg_none(c, page)) return;
    const int lo = n - p0 > 0 ? n - p0 : 0, hi = n + count - p0 < 32 ? n + count - p0 : 32;          // positions of the block that are written
    const int LR = c.Dh + E;                                   // values of a row in LDS (one piece more: the rows begin on different banks)
    T* kt = (T*)lds; T* vt = kt + 32 * LR;
    for (int x = tid + lo * D8; x < hi * D8; x += 256) {
        const int p = x / D8, d = 8 * (x - p * D8);
        const int64_t at = (int64_t)(first + p0 + p - n) * row_stride + (int64_t)h * c.Dh + d;
        pg_u32x4 a[W], b[W];
        pg_load8<T>(k + at, a);
        pg_load8<T>(v + at, b);
#pragma unroll
        for (int w = 0; w < W; ++w) { *(pg_u32x4*)(kt + p * LR + d + w * E) = a[w]; *(pg_u32x4*)(vt + p * LR + d + w * E) = b[w]; }
    }
    __syncthreads();
    const size_t base = ((((size_t)page * c.Hkv + h) << c.pb) + (blk & ((1 << c.pb) - 1))) * 32 * c.Dh;
    for (int x = tid; x < 4 * c.Dh; x += 256) {                // eights of the block, in its order
        T* kd = kl + base + (size_t)x * 8; T* vd = vl + base + (size_t)x * 8;
        // K: t, s, then 16 positions of each of the head's 32s
        const int y = x % (16 * G), ts = x / (16 * G), q = y & 15, p = 8 * (q >> 2) + 4 * (ts >> 2) + (q & 3), d = 32 * (y >> 4) + 8 * (ts & 3);
        if (p >= lo && p < hi)
#pragma unroll
            for (int w = 0; w < W; ++w) __builtin_nontemporal_store(*(const pg_u32x4*)(kt + p * LR + d + w * E), (pg_u32x4*)kd + w);
        // V: sixteen head elements, then four times eight positions of them
        const int e0 = (x >> 6) * 16 + (x & 15), v0 = 8 * (x >> 4 & 3);
        if (v0 >= lo && v0 + 8 <= hi) {
            alignas(16) T z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = vt[(v0 + e) * LR + e0];
#pragma unroll
            for (int w = 0; w < W; ++w) __builtin_nontemporal_store(*(const pg_u32x4*)(z + w * E), (pg_u32x4*)vd + w);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (v0 + e >= lo && v0 + e < hi) vd[e] = vt[(v0 + e) * LR + e0];
        }
    }
}

// ------------------------------------------------------------------ C entry points
#define FAIL(rc, ...) do { char text_[256]; snprintf(text_, sizeof text_, __VA_ARGS__); fc_set_error(text_); return rc; } while (0)

static bool head_dim_ok(int Dh) { return Dh == 32 || Dh == 64 || Dh == 96 || Dh == 128 || Dh == 192 || Dh == 256; }
static bool shape_ok(const fastcot_paged* c) {
    return c && c->n_layers >= 1 && c->n_layers <= 4096 && c->n_pages >= 1 && c->n_pages <= PG_MAX_PAGES && c->page_size >= 32 && c->page_size <= 4096 &&
           !(c->page_size & (c->page_size - 1)) && c->n_kv_heads >= 1 && c->n_kv_heads <= 4096 && head_dim_ok(c->head_dim) &&
           (c->dtype == FASTCOT_F32 || c->dtype == FASTCOT_BF16) && c->max_seqs >= 1 && c->max_seqs <= PG_MAX_SEQS && c->max_pages >= 1 &&
           (int64_t)c->max_pages * c->page_size <= (int64_t)1 << 30 && (int64_t)c->n_layers * c->n_kv_heads * (c->page_size / 16) < (int64_t)1 << 31 &&
           // (what an entry may need is summed in 32 bits, bytes of a pool in 64)
           (int64_t)c->max_seqs * c->max_pages < (int64_t)1 << 31 &&
           (double)c->n_layers * c->n_pages * c->n_kv_heads * c->page_size * c->head_dim < (double)((int64_t)1 << 60);
}
static size_t esz_of(const fastcot_paged* c) { return c->dtype == FASTCOT_BF16 ? 2 : 4; }
static size_t page_bytes(const fastcot_paged* c) { return (size_t)c->n_kv_heads * c->page_size * c->head_dim * esz_of(c); }
static size_t list_bytes(const fastcot_paged* c) { return FC_ALIGN((size_t)c->n_pages * 4); }

static int view_of(const char* name, const fastcot_paged* c, PagedView* v) {
    if (!shape_ok(c)) FAIL(FASTCOT_EINVAL, "%s: bad cache description", name);
    if (!c->k_pool || !c->v_pool || !c->table || !c->len || !c->ref) FAIL(FASTCOT_EINVAL, "%s: NULL device pointer in the cache", name);
    if (((uintptr_t)c->k_pool | (uintptr_t)c->v_pool) & 15) FAIL(FASTCOT_EINVAL, "%s: pools have to be aligned to 16 bytes", name);
    if (((uintptr_t)c->table | (uintptr_t)c->len | (uintptr_t)c->ref) & 3) FAIL(FASTCOT_EINVAL, "%s: misaligned int32 array", name);
    v->L = c->n_layers; v->N = c->n_pages; v->Hkv = c->n_kv_heads; v->Dh = c->head_dim; v->S = c->max_seqs; v->MP = c->max_pages;
    v->pb = __builtin_ctz((unsigned)c->page_size) - 5;
    v->k = (char*)c->k_pool; v->v = (char*)c->v_pool; v->table = c->table; v->len = c->len; v->ref = c->ref;
    return 0;
}
static int entries_of(const char* name, const fastcot_paged* c, int32_t count, const void* a, const void* b) {
    if (count < 0 || count > c->max_seqs) FAIL(FASTCOT_EINVAL, "%s: count %d outside 0..max_seqs", name, (int)count);
    if (count && (!a || !b)) FAIL(FASTCOT_EINVAL, "%s: NULL device pointer", name);
    if (((uintptr_t)a | (uintptr_t)b) & 3) FAIL(FASTCOT_EINVAL, "%s: misaligned int32 array", name);
    return 0;
}
static int scratch_of(const char* name, void* d_scratch) {
    if (!d_scratch || ((uintptr_t)d_scratch & 255)) FAIL(FASTCOT_EINVAL, "%s: scratch has to be given, aligned to 256 bytes", name);
    return 0;
}
static int rows_of(const char* name, const fastcot_paged_rows* r, int32_t layer, int32_t act, const fastcot_paged* c, PagedRows* o) {
    if (!r || r->n_seqs < 0 || r->rows < 0 || r->n_rows < 0) FAIL(FASTCOT_EINVAL, "%s: bad rows", name);
    if (r->n_seqs > 65535) FAIL(FASTCOT_EINVAL, "%s: more than 65535 sequences", name);
    if (!r->d_seqs && r->n_seqs > c->max_seqs) FAIL(FASTCOT_EINVAL, "%s: more sequences than the cache has", name);
    if (!r->d_row_start && (int64_t)r->n_seqs * r->rows != r->n_rows) FAIL(FASTCOT_EINVAL, "%s: n_rows is not n_seqs * rows", name);
    if (((uintptr_t)r->d_seqs | (uintptr_t)r->d_row_start) & 3) FAIL(FASTCOT_EINVAL, "%s: misaligned int32 array", name);
    if (layer < 0 || layer >= c->n_layers) FAIL(FASTCOT_EINVAL, "%s: layer %d outside the cache", name, (int)layer);
    if (act != FASTCOT_F32 && act != FASTCOT_BF16) FAIL(FASTCOT_EINVAL, "%s: unknown type of rows", name);
    if (act == FASTCOT_BF16 && c->dtype == FASTCOT_F32) FAIL(FASTCOT_EINVAL, "%s: an fp32 cache takes fp32 rows", name);
    o->B = r->n_seqs; o->R = r->rows < r->n_rows ? r->rows : r->n_rows; o->n_rows = r->n_rows; o->seqs = r->d_seqs; o->start = r->d_row_start;
    return 0;
}
static int launched(const char* name, hipError_t e) {
    if (e != hipSuccess) FAIL(FASTCOT_EHIP, "%s: launch failed (%s)", name, hipGetErrorString(e));
    return 0;
}
#define TRY(x) do { const int rc_ = (x); if (rc_) return rc_; } while (0)

extern "C" size_t fastcot_paged_pool_bytes(const fastcot_paged* c) {
    return shape_ok(c) ? (size_t)c->n_layers * c->n_pages * page_bytes(c) : 0;
}
extern "C" size_t fastcot_paged_scratch_bytes(const fastcot_paged* c) {
    return shape_ok(c) ? PG_HEAD + 3 * list_bytes(c) + fc_paged_attn_scratch_bytes(c->head_dim) : 0;
}
extern "C" int fastcot_paged_reset(const fastcot_paged* c, void* hip_stream) {
    const char* name = "fastcot_paged_reset";
    PagedView v;
    TRY(view_of(name, c, &v));
    k_paged_reset<<<256, 256, 0, (hipStream_t)hip_stream>>>(v);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_grow(const fastcot_paged* c, int32_t count, const int32_t* d_seqs, const int32_t* d_rows, int32_t* d_status, void* d_scratch,
                                  void* hip_stream) {
    const char* name = "fastcot_paged_grow";
    PagedView v;
    TRY(view_of(name, c, &v));
    TRY(entries_of(name, c, count, d_seqs, d_rows));
    TRY(scratch_of(name, d_scratch));
    if (!count) return 0;
    k_paged_grow<<<1, PG_WG, 0, (hipStream_t)hip_stream>>>(v, count, d_seqs, d_rows, d_status, (int*)((char*)d_scratch + PG_HEAD));
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_advance(const fastcot_paged* c, int32_t count, const int32_t* d_seqs, const int32_t* d_rows, int32_t* d_status, void* hip_stream) {
    const char* name = "fastcot_paged_advance";
    PagedView v;
    TRY(view_of(name, c, &v));
    TRY(entries_of(name, c, count, d_seqs, d_rows));
    if (!count) return 0;
    k_paged_advance<<<1, PG_WG, 0, (hipStream_t)hip_stream>>>(v, count, d_seqs, d_rows, d_status);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_fork(const fastcot_paged* c, int32_t count, const int32_t* d_src, const int32_t* d_dst, int32_t* d_status, void* d_scratch,
                                  void* hip_stream) {
    const char* name = "fastcot_paged_fork";
    PagedView v;
    TRY(view_of(name, c, &v));
    TRY(entries_of(name, c, count, d_src, d_dst));
    TRY(scratch_of(name, d_scratch));
    if (!count) return 0;
    char* l = (char*)d_scratch + PG_HEAD;
    int *n = (int*)d_scratch, *from = (int*)l, *to = (int*)(l + list_bytes(c)), *blocks = (int*)(l + 2 * list_bytes(c));
    hipStream_t st = (hipStream_t)hip_stream;
    k_paged_fork<<<1, PG_WG, 0, st>>>(v, count, d_src, d_dst, d_status, n, from, to, blocks);
    TRY(launched(name, hipGetLastError()));
    const int64_t most = (int64_t)count * c->n_layers * c->n_kv_heads * (c->page_size / 16);         // (blocks that can be copied)
    const int grid = most < 32 * fc_num_cus() ? (int)most : 32 * fc_num_cus();
    k_paged_move<true><<<grid, 256, 0, st>>>(v, (int)(32 * c->head_dim * esz_of(c) / 16), n, from, to, blocks, nullptr);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_trim(const fastcot_paged* c, int32_t count, const int32_t* d_seqs, int32_t window, int32_t sinks, int32_t* d_status, void* hip_stream) {
    const char* name = "fastcot_paged_trim";
    PagedView v;
    TRY(view_of(name, c, &v));
    TRY(entries_of(name, c, count, d_seqs, d_seqs));
    if (window < 1 || sinks < 0) FAIL(FASTCOT_EINVAL, "%s: window below 1 or sinks below 0", name);
    if (!count) return 0;
    k_paged_leave<<<count, 256, 0, (hipStream_t)hip_stream>>>(v, d_seqs, window, sinks, d_status);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_free(const fastcot_paged* c, int32_t count, const int32_t* d_seqs, int32_t* d_status, void* hip_stream) {
    const char* name = "fastcot_paged_free";
    PagedView v;
    TRY(view_of(name, c, &v));
    TRY(entries_of(name, c, count, d_seqs, d_seqs));
    if (!count) return 0;
    k_paged_leave<<<count, 256, 0, (hipStream_t)hip_stream>>>(v, d_seqs, 0, -1, d_status);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_compact(const fastcot_paged* c, int32_t* d_used, void* d_scratch, void* hip_stream) {
    const char* name = "fastcot_paged_compact";
    PagedView v;
    TRY(view_of(name, c, &v));
    TRY(scratch_of(name, d_scratch));
    char* l = (char*)d_scratch + PG_HEAD;
    int *n = (int*)d_scratch, *from = (int*)l, *to = (int*)(l + list_bytes(c)), *map = (int*)(l + 2 * list_bytes(c));
    hipStream_t st = (hipStream_t)hip_stream;
    k_paged_compact<<<1, PG_WG, 0, st>>>(v, d_used, n, from, to, map);
    TRY(launched(name, hipGetLastError()));
    k_paged_move<false><<<32 * fc_num_cus(), 256, 0, st>>>(v, (int)(32 * c->head_dim * esz_of(c) / 16), n, from, to, nullptr, map);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_write(const fastcot_paged* c, int32_t layer, const fastcot_paged_rows* rows, const void* d_k, const void* d_v, int64_t row_stride,
                                   int32_t act_dtype, void* hip_stream) {
    const char* name = "fastcot_paged_write";
    PagedView v;
    PagedRows r;
    TRY(view_of(name, c, &v));
    TRY(rows_of(name, rows, layer, act_dtype, c, &r));
    if (!r.B || !r.R || !r.n_rows) return 0;
    if (!d_k || !d_v || (((uintptr_t)d_k | (uintptr_t)d_v) & 15)) FAIL(FASTCOT_EINVAL, "%s: K and V have to be given, aligned to 16 bytes", name);
    if (row_stride % 8 || row_stride < (int64_t)c->n_kv_heads * c->head_dim) FAIL(FASTCOT_EINVAL, "%s: row stride below a row or no multiple of 8", name);
    char* kl = v.k + (size_t)layer * c->n_pages * page_bytes(c);
    char* vl = v.v + (size_t)layer * c->n_pages * page_bytes(c);
    const int64_t gx = (((int64_t)r.R + 31) / 32 + 1) * c->n_kv_heads;             // (rows may begin inside a block)
    if (r.R > 1 << 30 || gx > 0x7FFFFFFF) FAIL(FASTCOT_ECAPACITY, "%s: too many rows of one sequence", name);
    const dim3 grid((unsigned)gx, (unsigned)r.B);
    const size_t lds = 2 * 32 * (c->head_dim * esz_of(c) + 16);
    hipStream_t st = (hipStream_t)hip_stream;
    if (lds > 65536)                                           // (fp32 heads of 256: more than 64 KB have to be asked for)
        TRY(launched(name, hipFuncSetAttribute((const void*)k_paged_write<float, float>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)));
    if (c->dtype == FASTCOT_F32) k_paged_write<float, float><<<grid, 256, lds, st>>>(v, r, (float*)kl, (float*)vl, (const float*)d_k, (const float*)d_v, row_stride);
    else if (act_dtype == FASTCOT_F32)
        k_paged_write<bf16_t, float><<<grid, 256, lds, st>>>(v, r, (bf16_t*)kl, (bf16_t*)vl, (const float*)d_k, (const float*)d_v, row_stride);
    else k_paged_write<bf16_t, bf16_t><<<grid, 256, lds, st>>>(v, r, (bf16_t*)kl, (bf16_t*)vl, (const bf16_t*)d_k, (const bf16_t*)d_v, row_stride);
    return launched(name, hipGetLastError());
}
extern "C" int fastcot_paged_attn(const fastcot_paged* c, int32_t layer, const fastcot_paged_rows* rows, const void* d_q, int64_t q_row_stride,
                                  int64_t q_head_stride, int32_t n_heads, int32_t act_dtype, int32_t window, int32_t sinks, void* d_out, int64_t out_row_stride,
                                  float* d_lse, void* d_scratch, void* hip_stream) {
    const char* name = "fastcot_paged_attn";
    PagedAttnArgs a;
    TRY(view_of(name, c, &a.c));
    TRY(rows_of(name, rows, layer, act_dtype, c, &a.r));
    TRY(scratch_of(name, d_scratch));
    if (n_heads < 1 || n_heads % c->n_kv_heads || n_heads / c->n_kv_heads > 64) FAIL(FASTCOT_EINVAL, "%s: heads are no multiple (up to 64) of the cache's", name);
    if (window < 0 || sinks < 0) FAIL(FASTCOT_EINVAL, "%s: window or sinks below 0", name);
    if (!a.r.B || !a.r.R || !a.r.n_rows) return 0;
    // (what the kernel deals to its workgroups: blocks of 32 positions, and some more, for every 16 rows of a K/V head)
    const double g = n_heads / c->n_kv_heads, tiles = (a.r.R * g + 15) / 16, blocks = (double)c->max_pages * (c->page_size / 32) + a.r.R / 32 + 10;
    if (a.r.R * g >= (1 << 26) || (double)a.r.B * c->n_kv_heads * tiles * blocks >= 2147483648.0)
        FAIL(FASTCOT_ECAPACITY, "%s: rows times positions of the table pass 2^31 blocks", name);
    if ((uintptr_t)d_lse & 3) FAIL(FASTCOT_EINVAL, "%s: misaligned d_lse", name);
    if (!d_q || !d_out || (((uintptr_t)d_q | (uintptr_t)d_out) & 15)) FAIL(FASTCOT_EINVAL, "%s: queries and output have to be given, aligned to 16 bytes", name);
    if (q_row_stride % 8 || q_head_stride % 8 || q_row_stride < 0 || q_head_stride < 0) FAIL(FASTCOT_EINVAL, "%s: strides of the queries are no multiples of 8", name);
    if (out_row_stride % 8 || out_row_stride < (int64_t)n_heads * c->head_dim) FAIL(FASTCOT_EINVAL, "%s: row stride of the output below a row or no multiple of 8", name);
    a.kl = a.c.k + (size_t)layer * c->n_pages * page_bytes(c);
    a.vl = a.c.v + (size_t)layer * c->n_pages * page_bytes(c);
    a.q = d_q; a.q_row = q_row_stride; a.q_head = q_head_stride;
    a.out = d_out; a.out_row = out_row_stride; a.lse = d_lse;
    a.H = n_heads; a.act = act_dtype; a.g = n_heads / c->n_kv_heads; a.g_inv = (uint32_t)(((1ull << 32) + a.g - 1) / a.g); a.esz = (int32_t)esz_of(c); a.window = window; a.sinks = window ? sinks : 0; a.reach = window ? (uint32_t)window : 0x80000000u;
    a.cnt = (int32_t*)d_scratch + 64;
    a.joins = (PagedJoin*)((char*)d_scratch + 4096);
    a.part = (float*)((char*)d_scratch + PG_HEAD + 3 * list_bytes(c));
    return launched(name, fc_paged_attn(a, (hipStream_t)hip_stream));
}
