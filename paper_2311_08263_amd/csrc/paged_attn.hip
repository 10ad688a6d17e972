// Attention of a pass's rows over a K/V cache in pages: row at position p sees k <= p that has a page and, under a sliding window,
// k > p - window or k < sinks.
//
//   s_k = q . k / sqrt(Dh),  m = max s_k,  l = sum e^(s_k - m),  out = sum e^(s_k - m) v_k / l,  lse = m + ln l
//
// A unit is 16 or 32 rows (token by token, the query heads of a K/V head next to each other) of one sequence and K/V head.  The visible blocks of
// 32 positions of all units, one after the other, are dealt to the launch's workgroups in equal parts (pg_deal): lengths come from device memory, so
// a captured launch stays balanced while they move on.  A workgroup's waves take the blocks of its part of a unit in turn, keep m, l and the sums
// in registers and meet in LDS; parts of one unit meet in memory, where the last workgroup to arrive joins them in order.  Scores S^T = K . Q^T and
// sums O^T += V^T . P^T are matrix instructions whose operands lie in the cache as they are needed (k_index, v_index); for any head size
// the 16-byte pieces u = 4 f + lane / 16 of a score tile's fragment f hold head elements 32 (u % G) + 8 (u / G) .. + 7, G = Dh / 32.
// bf16 caches run on bf16 instructions with fp32 queries and weights in three parts (24 bits, so results are those of fp32 arithmetic) or bf16
// queries in one and weights in two; fp32 caches on fp32 instructions.
// Blocks that some row does not see whole are edges: their scores are masked, and V of positions that no row of the unit sees is taken as zero (a
// weight of zero times an infinity is none).  Where V is not finite at a position that some rows see and others do not, the block's products
// are summed position by position.
#include "gemmco.h"      // fc_num_cus
#include "paged.h"
#include "xwg.h"

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;

#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f

// The parts of a fp32 value are cut off its bits from the top, so that none overflows and three hold all 24 bits
// (one or two: the last one is rounded)
template <int TERMS> __device__ inline void pg_split8(const float* v, u32x4_t* part) {
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e];
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t a = __float_as_uint(x[2 * e]), b = __float_as_uint(x[2 * e + 1]);
            if (t == TERMS - 1 && TERMS < 3) w[e] = pk_bf16(x[2 * e], x[2 * e + 1]);
            else w[e] = (a >> 16) | (b & 0xFFFF0000u);
            if (t < TERMS - 1) { x[2 * e] -= __uint_as_float(a & 0xFFFF0000u); x[2 * e + 1] -= __uint_as_float(b & 0xFFFF0000u); }
        }
        part[t] = (u32x4_t){w[0], w[1], w[2], w[3]};
    }
}
#define ROW_NONE (-3.0e38f)      // reference of a row that has seen nothing
// Products p become the exponents by * p - from, each operation rounded: where the reference is far from zero a product as large as the largest one has to
// give an exponent of zero, which a fused multiply-add with the rounded reference does not
__device__ inline void pg_far(float* p, float& by, float& from) {
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = p[e] * by - from;
    by = 1.f; from = 0.f;
}
__device__ inline bool pg_sees(const PagedAttnArgs& a, int key, int pos) {
    return (uint32_t)(pos - key) < a.reach || (key < a.sinks && key <= pos);
}
// scores p of positions key .. key + 7 for a row at position pos: what it does not see becomes -infinity.  sunk: some of them are among the sinks
__device__ inline void pg_mask8(const PagedAttnArgs& a, int key, int pos, bool sunk, float* p) {
    if (sunk) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = pg_sees(a, key + e, pos) ? p[e] : -INFINITY;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (uint32_t)(pos - key - e) < a.reach ? p[e] : -INFINITY;
    }
}
// whether any of eight bf16 values is not finite (their exponents are all ones: a carry out of each when the lowest bit is added)
__device__ inline bool pg_not_finite(const u32x4_t& v) {
    uint32_t x = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) x |= (v[w] & 0x7F807F80u) + 0x00800080u;
    return (x & 0x80008000u) != 0;
}
// zeros in their place: an infinity or NaN is added by itself to the rows that see it, whatever its weight; multiplied by a weight of zero it would reach the others
__device__ inline void pg_make_finite(u32x4_t& v) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
        v[w] &= ((v[w] & 0x7F80u) == 0x7F80u ? 0u : 0x0000FFFFu) | ((v[w] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
}
// What is not finite among eight values of V: ones where it is +infinity or NaN, and where it is -infinity or NaN
__device__ inline void pg_infinite(u32x4_t& up, u32x4_t& down) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t x = up[w], lo = x & 0xFFFFu, hi = x >> 16;
        auto one = [](uint32_t b, uint32_t sign) { return (b & 0x7FFFu) > 0x7F80u || b == (sign | 0x7F80u) ? 0x3F80u : 0u; };
        up[w] = one(lo, 0u) | one(hi, 0u) << 16;
        down[w] = one(lo, 0x8000u) | one(hi, 0x8000u) << 16;
    }
}
// ones where a row at position pos sees position key, key + 1, .. key + 7
__device__ inline u32x4_t pg_seen8(const PagedAttnArgs& a, int key, int pos) {
    u32x4_t r;
#pragma unroll
    for (int w = 0; w < 4; ++w) r[w] = (pg_sees(a, key + 2 * w, pos) ? 0x3F80u : 0u) | (pg_sees(a, key + 2 * w + 1, pos) ? 0x3F800000u : 0u);
    return r;
}
__device__ inline void pg_add_infinite(f32x4_t& acc, const u32x4_t& up, const u32x4_t& down, const u32x4_t& seen) {
    const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
    const f32x4_t x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, up), __builtin_bit_cast(bf16x8_t, seen), zero, 0, 0, 0);
    const f32x4_t y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, down), __builtin_bit_cast(bf16x8_t, seen), zero, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += (x[i] > 0.f ? INFINITY : 0.f) + (y[i] > 0.f ? -INFINITY : 0.f);
}
// the blocks of 32 positions that rows at positions p0 .. p1 see: the first `sunk`, then lo .. hi - 1
struct PagedRange { int sunk, lo, hi; };
__device__ inline PagedRange pg_range(const PagedAttnArgs& a, int p0, int p1) {
    PagedRange r;
    r.hi = (p1 >> 5) + 1;
    const int first = a.window && p0 - a.window + 1 > 0 ? p0 - a.window + 1 : 0;
    r.lo = first >> 5;
    r.sunk = a.window ? (a.sinks >> 5) + ((a.sinks & 31) != 0) : 0;
    if (r.sunk > r.lo) r.sunk = r.lo;
    return r;
}

// One workgroup's part of a unit: blocks off .. off + len - 1 of its `blocks` visible ones
struct PagedPart {
    int b, kvh, tile;
    int seq, n, first, rows;               // rows of the sequence times query heads of a K/V head
    int off, len, blocks;
    uint32_t base;                         // place of the unit's first block in what is dealt
};
struct PagedDeal { uint32_t share, at, end; int least; };         // what a workgroup gets, this one's places at .. end - 1, fewest blocks of a part
__device__ inline int pg_uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// a structure of 32-bit words that is the same in every lane
template <class T> __device__ inline T pg_uniform(const T& x) {
    T y = x;
    int* w = (int*)&y;
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 4; ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    return y;
}
// token of row x of a sequence: x / (query heads of a K/V head), x below 2^26
__device__ inline int pg_token(const PagedAttnArgs& a, int x) { return a.g == 1 ? x : (int)__umulhi((uint32_t)x, a.g_inv); }
// visible blocks of a tile of RT rows; rows of no sequence get one, that is not there
template <int RT> __device__ inline int pg_blocks(const PagedAttnArgs& a, int seq, int n, int rows, int tile) {
    if (tile * RT >= rows) return 0;
    if (seq < 0) return 1;
    const int last = tile * RT + RT < rows ? tile * RT + RT - 1 : rows - 1;
    const PagedRange r = pg_range(a, n + pg_token(a, tile * RT), n + pg_token(a, last));
    return r.sunk + r.hi - r.lo;
}
__device__ inline void pg_load(const PagedAttnArgs& a, int b, int& seq, int& n, int& first, int& rows) {
    int count;
    pg_rows(a.r, b, first, count);
    seq = pg_seq(a.r, a.c, b);
    n = seq < 0 ? 0 : pg_len(a.c, seq);
    rows = count * a.g;
}
// inclusive prefix sum over the wave's lanes
__device__ inline uint32_t pg_wave_scan(uint32_t x) {
    int v = (int)x;
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);        // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);        // row_bcast 15, 31
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
    return (uint32_t)v;
}
__device__ inline uint32_t pg_lane(uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); }
// What is dealt: PG_UNIT places for every unit and one for each of its blocks; units ordered by sequence, K/V head, tile.  Every workgroup gets an equal
// share of at least PG_UNIT places, every wave finds its workgroup's by itself: lanes take sequences (or, where a sequence has more than four tiles,
// tiles).  A unit of at most a.whole blocks is not cut, it belongs to the share that its first block falls into.  The host has checked that all
// places fit 31 bits.  false: nothing for this worker.  p: the first part of its share.
// A unit's queries, meeting and output take about as long as eight blocks: 48 sequences of 60 to 8100 positions over 40 heads take 302 us with 4 places a
// unit, 256 with 8, 255 with 16; three short ones 10.9, 8.7 and 8.7 us, 200 of 20 to 300 positions over 8 heads 32.8, 32.9 and 35.3.  (The kernel for many
// rows: 4.3 us a unit, 0.72 us a block.)
#define PG_UNIT (RT > 32 ? 6 : 8)
template <int RT> __device__ inline void pg_part(const PagedAttnArgs& a, PagedDeal& d, PagedPart& p) {     // the share's part of the unit p, from the place d.at on
    if (p.blocks <= a.whole) { p.off = 0; p.len = p.base >= d.at && p.base < d.end ? p.blocks : 0; return; }
    // (a cut close to an end of the unit is moved there)
    auto cut = [&](uint32_t place) {
        const int c = (int)(place - p.base);
        return c < d.least ? 0 : p.blocks - c < d.least ? p.blocks : c;
    };
    p.off = cut(d.at);
    p.len = cut(d.end) - p.off;
}
// workgroups that share a cut unit
__device__ inline int pg_first_worker(const PagedDeal& d, const PagedPart& p) { return (int)((p.base + d.least - 1) / d.share); }
__device__ inline int pg_last_worker(const PagedDeal& d, const PagedPart& p) { return (int)((p.base + p.blocks - d.least) / d.share); }
template <int RT> __device__ inline bool pg_deal(const PagedAttnArgs& a, int tiles, int worker, int workers, PagedDeal& d, PagedPart& p) {
    const int lane = threadIdx.x & 63, Hkv = a.c.Hkv;
    const bool by_seq = tiles <= 4;
    // places of one K/V head of sequence b in tiles t0 .. t1 - 1
    int seq = -1, n = 0, first = 0, rows = 0;                  // of the sequence that was looked at last
    auto places = [&](int b, int t0, int t1) -> uint32_t {
        if (b >= a.r.B) return 0;
        pg_load(a, b, seq, n, first, rows);
        uint32_t s = 0;
        for (int t = t0; t < t1; ++t) { const int x = pg_blocks<RT>(a, seq, n, rows, t); s += x ? x + PG_UNIT : 0; }
        return s;
    };
    uint32_t total = 0, mine = 0, incl = 0;
    if (by_seq) {
        for (int b = 0; b < a.r.B; b += 64) { mine = places(b + lane, 0, tiles) * Hkv; incl = pg_wave_scan(mine); total += pg_lane(incl, 63); }
    } else {
        for (int b = 0; b < a.r.B; ++b) for (int t = 0; t < tiles; t += 64) mine += places(b, t + lane, t + lane + 1);
        total = pg_lane(pg_wave_scan(mine), 63) * Hkv;
    }
    d.share = (total + workers - 1) / workers;
    if (d.share < PG_UNIT) d.share = PG_UNIT;
    d.least = d.share < 32 ? 1 : d.share < 64 ? 2 : 4;
    d.at = d.share * worker;
    if (d.at >= total) return false;
    d.end = d.at + d.share < total ? d.at + d.share : total;
    // the sequence that place d.at falls into, the places in front of it, and those of one of its heads
    uint32_t before = 0, head = 0;
    int b = 0, from = 0;                                       // from: a lane that has looked at it
    // (each walk also ends where the numbers end: lengths that change under a call give wrong results, not an endless one)
    if (by_seq) {
        for (;; b += 64) {
            if (b >= a.r.B) return false;
            if (a.r.B > 64) { mine = places(b + lane, 0, tiles) * Hkv; incl = pg_wave_scan(mine); }
            const uint64_t hit = __ballot(before + incl > d.at);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                const uint32_t w = pg_lane(mine, l);
                before += pg_lane(incl, l) - w;
                head = w / Hkv;
                b += l;
                from = l;
                break;
            }
            before += pg_lane(incl, 63);
        }
    } else {
        for (;; ++b) {
            if (b >= a.r.B) return false;
            mine = 0;
            for (int t = 0; t < tiles; t += 64) mine += places(b, t + lane, t + lane + 1);
            head = pg_lane(pg_wave_scan(mine), 63);
            if (before + head * Hkv > d.at) break;
            before += head * Hkv;
        }
    }
    p.b = b;
    p.seq = __builtin_amdgcn_readlane(seq, from); p.n = __builtin_amdgcn_readlane(n, from);
    p.first = __builtin_amdgcn_readlane(first, from); p.rows = __builtin_amdgcn_readlane(rows, from);
    p.kvh = pg_uniform((int)((d.at - before) / head));
    before += head * p.kvh;
    p.tile = 0;
    if (by_seq) {
        for (;; ++p.tile) {
            if (p.tile >= tiles) return false;
            p.blocks = pg_blocks<RT>(a, p.seq, p.n, p.rows, p.tile);
            if (before + p.blocks + PG_UNIT > d.at) break;
            before += p.blocks + PG_UNIT;
        }
    } else {
        for (int t = 0;; t += 64) {
            if (t >= tiles) return false;
            mine = pg_blocks<RT>(a, p.seq, p.n, p.rows, t + lane);
            if (mine) mine += PG_UNIT;
            incl = pg_wave_scan(mine);
            const uint64_t hit = __ballot(before + incl > d.at);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                const uint32_t w = pg_lane(mine, l);
                before += pg_lane(incl, l) - w;
                p.blocks = (int)w - PG_UNIT;
                p.tile = t + l;
                break;
            }
            before += pg_lane(incl, 63);
        }
    }
    p.blocks = pg_uniform(p.blocks); p.tile = pg_uniform(p.tile);
    p.base = (uint32_t)pg_uniform((int)before) + PG_UNIT;
    pg_part<RT>(a, d, p);
    return true;
}
// the next part of the share (of which there may be nothing but places without a block)
template <int RT> __device__ inline bool pg_next(const PagedAttnArgs& a, const PagedDeal& d, PagedPart& p) {
    const uint32_t next = p.base + p.blocks;
    if (next >= d.end) return false;
    if (++p.tile * RT >= p.rows) {
        p.tile = 0;
        if (++p.kvh == a.c.Hkv) {
            p.kvh = 0;
            do {
                if (++p.b >= a.r.B) return false;
                pg_load(a, p.b, p.seq, p.n, p.first, p.rows);
                p.seq = pg_uniform(p.seq); p.n = pg_uniform(p.n); p.first = pg_uniform(p.first); p.rows = pg_uniform(p.rows);
            } while (p.rows == 0);
        }
    }
    p.blocks = pg_blocks<RT>(a, p.seq, p.n, p.rows, p.tile);
    p.base = next + PG_UNIT;
    PagedDeal e = d;
    e.at = next;
    pg_part<RT>(a, e, p);
    return true;
}
// Where a part of a unit that several workgroups share keeps its results: a workgroup has at most two such parts, one that another one began (slot 0)
// and one that another one ends.  Slots hold RT rows of Dh sums, then m and l of each row.

// two joined sums of row x of a sequence to the output
__device__ inline void pg_out(const PagedAttnArgs& a, int x, int first, int kvh, int Dh, int d, float M, float L, float o0, float o1) {
    const int j = pg_token(a, x), row = first + j, h = kvh * a.g + x - j * a.g;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const size_t at = (size_t)row * a.out_row + (size_t)h * Dh + d;
    if (a.act == FASTCOT_BF16) *(uint32_t*)((bf16_t*)a.out + at) = pk_bf16(o0 * inv, o1 * inv);
    else *(float2*)((float*)a.out + at) = make_float2(o0 * inv, o1 * inv);
    if (a.lse && d == 0) a.lse[(size_t)row * a.H + h] = (M == -INFINITY ? 0.f : M) * LN2 + logf(L);
}
// Joins the parts of a unit: a thread takes two sums of a row, of every part or, where that leaves threads idle, of every groups-th one; eight
// parts are requested at a time.  (One after the other 32 parts took 15 us.)
template <int G, int RT, int NW> __device__ inline void pg_join(const PagedAttnArgs& a, float* lds, int row0, int nrows, int first, int kvh, int w0, int parts) {
    constexpr int Dh = 32 * G, SLOT = RT * (Dh + 2), T = NW * 64;
    const int rows = nrows - row0 < RT ? nrows - row0 : RT, pairs = rows * (Dh / 2);
    const float* p0 = a.part + (size_t)(2 * w0 + 1) * SLOT;    // the first part's slot; the others' are the even ones behind it
    const int groups = pairs < T ? T / pairs : 1, grp = pairs < T ? (int)threadIdx.x / pairs : 0, y0 = pairs < T ? (int)threadIdx.x - grp * pairs : (int)threadIdx.x;
    float M = -INFINITY, L = 0.f, o0 = 0.f, o1 = 0.f;
    auto add = [&](float m, float l, float v0, float v1) {
        const float Mn = fmaxf(M, m), Ms = Mn == -INFINITY ? 0.f : Mn;
        const float x = __builtin_amdgcn_exp2f(M - Ms), w = __builtin_amdgcn_exp2f(m - Ms);
        L = L * x + l * w; o0 = o0 * x + v0 * w; o1 = o1 * x + v1 * w;
        M = Mn;
    };
    for (int y = y0; y < pairs && grp < groups; y += T) {
        const int r = y / (Dh / 2), d = 2 * (y % (Dh / 2));
        M = -INFINITY; L = o0 = o1 = 0.f;
        for (int i0 = grp; i0 < parts; i0 += 8 * groups) {
            float m[8], l[8], v0[8], v1[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = i0 + e * groups < parts ? i0 + e * groups : i0;
                const float* s = p0 + (i ? (size_t)(2 * i - 1) * SLOT : 0);
                ld_agent_f32x2(s + RT * Dh + 2 * r, m[e], l[e]);
                ld_agent_f32x2(s + r * Dh + d, v0[e], v1[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) if (i0 + e * groups < parts) add(m[e], l[e], v0[e], v1[e]);
        }
        if (groups == 1) pg_out(a, row0 + r, first, kvh, Dh, d, M, L, o0, o1);
    }
    if (groups > 1) {
        if (grp < groups) *(float4*)(lds + 4 * threadIdx.x) = make_float4(M, L, o0, o1);
        __syncthreads();
        if ((int)threadIdx.x < pairs) {
            for (int k = 1; k < groups; ++k) { const float4 z = *(const float4*)(lds + 4 * (threadIdx.x + k * pairs)); add(z.x, z.y, z.z, z.w); }
            pg_out(a, row0 + y0 / (Dh / 2), first, kvh, Dh, 2 * (y0 % (Dh / 2)), M, L, o0, o1);
        }
    }
}

// G: 32s of a head; F32: fp32 cache; QT: tiles of 16 rows of a unit; NW: waves; QP, PP: bf16 parts of queries and weights
template <int G, bool F32, int QT, int NW, int QP, int PP>
__global__ __launch_bounds__(NW * 64, QT == 1 && G <= 4 ? 2 : 1) void k_paged_attn(PagedAttnArgs a, int tiles) {
    constexpr int Dh = 32 * G, NV = 2 * G, RT = 16 * QT;       // NV: fragments of V, four sums of a lane each
    constexpr int PART = Dh * 16 + 32;                         // floats of a wave's tile: sums, then m and l of the 16 rows
    extern __shared__ __align__(16) float lds[];
    __shared__ int arrived;
    const int lane = threadIdx.x & 63, lm = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PagedDeal deal;
    PagedPart part;
    // fp32 caches run many rows here too: consecutive shares go to one XCD, whose L2 holds the blocks that units of one K/V head find after each other (they are
    // loaded to stay there: 1695, 21 and 2001 rows of 7B heads 1205 / 886 us, 1000 rows of 8 heads on 4 of 256 164 / 110)
    const int worker = F32 && !(gridDim.x & 7) ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;
    if (!pg_deal<RT>(a, tiles, worker, gridDim.x, deal, part)) return;
  do {
    if (part.len <= 0) continue;                               // (a share that ends in front of the unit's first block)
    const int kvh = part.kvh, first = part.first, nrows = part.rows, seq = part.seq, n = part.n;
    const int row0 = part.tile * RT;                           // rows of the unit: row0 .. of nrows, row x = head x % g of token x / g
    const int g = a.g, last = row0 + RT < nrows ? row0 + RT - 1 : nrows - 1;
    const int j0 = pg_token(a, row0), j1 = pg_token(a, last);
    const int p0 = n + j0, p1 = n + j1;
    const PagedRange vis = pg_range(a, p0, p1);
    const int* table = a.c.table + (size_t)(seq < 0 ? 0 : seq) * a.c.MP;
    const float scale2 = LOG2E / sqrtf((float)Dh);             // the softmax runs in powers of two

    int pos[QT];                                               // this lane's rows: row row0 + 16 * qt + lm (-1: none)
    u32x4_t qf[F32 ? 1 : QT][G][QP];
    float qx[F32 ? QT : 1][G][8];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int x = row0 + 16 * qt + lm, row = x < nrows ? x : last, j = pg_token(a, row);
        pos[qt] = x < nrows ? n + j : -1;
        const size_t at = (size_t)(first + j) * a.q_row + (size_t)(kvh * g + row - j * g) * a.q_head;
#pragma unroll
        for (int f = 0; f < G; ++f) {
            const int u = 4 * f + lg, dh = 32 * (u % G) + 8 * (u / G);
            if constexpr (!F32 && QP == 1) qf[qt][f][0] = *(const u32x4_t*)((const bf16_t*)a.q + at + dh);
            else {
                float v[8];
                const float4 y = *(const float4*)((const float*)a.q + at + dh), z = *(const float4*)((const float*)a.q + at + dh + 4);
                v[0] = y.x * scale2; v[1] = y.y * scale2; v[2] = y.z * scale2; v[3] = y.w * scale2;
                v[4] = z.x * scale2; v[5] = z.y * scale2; v[6] = z.z * scale2; v[7] = z.w * scale2;
                if constexpr (F32) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) qx[qt][f][e] = v[e];
                } else pg_split8<QP>(v, qf[qt][f]);
            }
        }
    }
    f32x4_t acc[QT][NV];
    float m[QT], l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        m[qt] = -INFINITY; l[qt] = 0.f;
#pragma unroll
        for (int f = 0; f < NV; ++f) acc[qt][f] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }

    // pages of this wave's next 64 blocks, one a lane
    const int end = part.off + part.len;
    auto pages_from = [&](int x0) {
        const int x = x0 + lane * NW, blk = x < vis.sunk ? x : x - vis.sunk + vis.lo, slot = blk >> a.c.pb;
        const int page = seq >= 0 && x < end && slot < a.c.MP ? table[slot] : -1;
        return page >= 0 && page < a.c.N ? page : -1;
    };
    int pages = pages_from(part.off + wv), held = part.off + wv;
    for (int x = held; x < end; x += NW) {
        if (x - held == 64 * NW) { held = x; pages = pages_from(x); }
        const int blk = x < vis.sunk ? x : x - vis.sunk + vis.lo, kb = blk << 5;
        const int page = __builtin_amdgcn_readlane(pages, (x - held) / NW);
        if (page < 0) continue;
        const size_t at = ((((size_t)page * a.c.Hkv + kvh) << a.c.pb) + (blk & ((1 << a.c.pb) - 1))) * 32 * Dh;
        constexpr int FW = F32 ? 2 : 1;                        // 16-byte words of a lane's eight values
        const u32x4_t* kp = (const u32x4_t*)(a.kl + at * (F32 ? 4 : 2)) + lane * FW;
        const u32x4_t* vp = (const u32x4_t*)(a.vl + at * (F32 ? 4 : 2)) + lane * FW;
        // (bf16 blocks go past the caches: 48 sequences of 60 to 8100 positions 264 us, 297 if not.  Of fp32 ones a lane takes its 32 bytes in two loads, which
        // share their lines: one token of 20 sequences of 8000 positions 864, past the caches 904)
        u32x4_t kf[2 * G][FW], vf[NV][FW];
#pragma unroll
        for (int f = 0; f < 2 * G; ++f)
#pragma unroll
            for (int w = 0; w < FW; ++w) kf[f][w] = F32 ? kp[f * 64 * FW + w] : __builtin_nontemporal_load(kp + f * 64 * FW + w);
#pragma unroll
        for (int f = 0; f < NV; ++f)
#pragma unroll
            for (int w = 0; w < FW; ++w) vf[f][w] = F32 ? vp[f * 64 * FW + w] : __builtin_nontemporal_load(vp + f * 64 * FW + w);
        // every row sees all 32 positions
        const bool whole = kb + 31 <= p0 && (!a.window || kb > p1 - a.window || kb + 31 < a.sinks);
        bool odd = false;                                      // V is not finite where some rows see it and others do not
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = kb + 8 * lg + e;
                const bool any = key <= p1 && (!a.window || key > p0 - a.window || key < a.sinks);
#pragma unroll
                for (int f = 0; f < NV; ++f) {
                    // bits of this position's value in its word, and of its exponent
                    const uint32_t bits = F32 ? 0xFFFFFFFFu : e & 1 ? 0xFFFF0000u : 0x0000FFFFu, ex = bits & (F32 ? 0x7F800000u : 0x7F807F80u);
                    const int wd = F32 ? e >> 2 : 0, el = F32 ? e & 3 : e >> 1;
                    const uint32_t w = any ? vf[f][wd][el] : vf[f][wd][el] & ~bits;
                    vf[f][wd][el] = w;
                    odd |= (w & ex) == ex;
                }
            }
            odd = __any(odd);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
#pragma clang fp contract(off)           // (a score meets the maximum in its own rounding)
            f32x4_t sc[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                sc[t] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int f = 0; f < G; ++f) {
                    if constexpr (F32) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            sc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[t * G + f][e >> 2][e & 3]), qx[qt][f][e], sc[t], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int q = QP - 1; q >= 0; --q)      // (small parts first)
                            sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[t * G + f][0]), __builtin_bit_cast(bf16x8_t, qf[qt][f][q]), sc[t], 0, 0, 0);
                    }
                }
            }
            // lane: row lm, positions kb + 8 * lg + e (e = 4 * t + i)
            float p[8], bm = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = !F32 && QP == 1 ? sc[e >> 2][e & 3] * scale2 : sc[e >> 2][e & 3];
            if (!whole) pg_mask8(a, kb + 8 * lg, pos[qt], F32 || kb < a.sinks, p);          // (fp32: no registers for two forms)
#pragma unroll
            for (int e = 0; e < 8; ++e) bm = fmaxf(bm, p[e]);
            bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
            bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
            const float mnew = fmaxf(m[qt], bm), ms = mnew == -INFINITY ? 0.f : mnew;          // (a row that has seen nothing yet)
            const float alpha = __builtin_amdgcn_exp2f(m[qt] - ms);
            float ps = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) { p[e] = __builtin_amdgcn_exp2f(p[e] - ms); ps += p[e]; }
            m[qt] = mnew;
            l[qt] = l[qt] * alpha + ps;
#pragma unroll
            for (int f = 0; f < NV; ++f) acc[qt][f] *= alpha;
            if (odd) {
                for (int k = 0; k < 32; ++k) {
                        const int e = k & 7, kg = k >> 3;
                        const float w4 = e & 2 ? (e & 1 ? p[3] : p[2]) : (e & 1 ? p[1] : p[0]), w8 = e & 2 ? (e & 1 ? p[7] : p[6]) : (e & 1 ? p[5] : p[4]);
                        const float w = __shfl(e & 4 ? w8 : w4, lm + 16 * kg, 64);
                        const bool sees = pg_sees(a, kb + k, pos[qt]);
#pragma unroll
                        for (int f = 0; f < NV; ++f)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const size_t y = at + (size_t)(f * 64 + 4 * lg + i + 16 * kg) * 8 + e;
                                const float v = F32 ? ((const float*)a.vl)[y] : bf16_to_f32(((const bf16_t*)a.vl)[y]);
                                if (sees) acc[qt][f][i] += w * v;
                            }
                    }
            } else if constexpr (F32) {
#pragma unroll
                for (int f = 0; f < NV; ++f)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        acc[qt][f] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[f][e >> 2][e & 3]), p[e], acc[qt][f], 0, 0, 0);
            } else {
                u32x4_t pf[PP];
                pg_split8<PP>(p, pf);
#pragma unroll
                for (int f = 0; f < NV; ++f)
#pragma unroll
                    for (int q = PP - 1; q >= 0; --q)
                        acc[qt][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf[f][0]), __builtin_bit_cast(bf16x8_t, pf[q]), acc[qt][f], 0, 0, 0);
            }
        }
    }

    // the waves meet: wave w finishes fragments w, w + NW, ..
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        l[qt] += __shfl_xor(l[qt], 16, 64);
        l[qt] += __shfl_xor(l[qt], 32, 64);
        float* dst = lds + (wv * QT + qt) * PART;
#pragma unroll
        for (int f = 0; f < NV; ++f) *(f32x4_t*)(dst + (f * 64 + lane) * 4) = acc[qt][f];
        if (lg == 0) { dst[Dh * 16 + lm] = m[qt]; dst[Dh * 16 + 16 + lm] = l[qt]; }
    }
    __syncthreads();
    const bool shared = part.len < part.blocks;
    float* mine = a.part + (size_t)(2 * worker + (part.off == 0)) * RT * (Dh + 2);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int x = row0 + 16 * qt + lm;
        float M = -INFINITY, L = 0.f, w[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) { w[i] = lds[(i * QT + qt) * PART + Dh * 16 + lm]; M = fmaxf(M, w[i]); }
        const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int i = 0; i < NW; ++i) { w[i] = __builtin_amdgcn_exp2f(w[i] - Ms); L += lds[(i * QT + qt) * PART + Dh * 16 + 16 + lm] * w[i]; }
        const float inv = shared ? 1.f : L == 0.f ? 0.f : 1.f / L;
        const int j = pg_token(a, x), row = first + j, h = kvh * g + x - j * g;
        for (int f = wv; f < NV; f += NW) {
            f32x4_t o = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const f32x4_t y = *(const f32x4_t*)(lds + (i * QT + qt) * PART + (f * 64 + lane) * 4);
                o += y * w[i];
            }
            if (x >= nrows) continue;
            if (shared) {
                float* to = mine + (16 * qt + lm) * Dh + 16 * f + 4 * lg;
                st_agent_f32x2(to, o[0], o[1]);
                st_agent_f32x2(to + 2, o[2], o[3]);
                continue;
            }
            o *= inv;
            const size_t at = (size_t)row * a.out_row + (size_t)h * Dh + 16 * f + 4 * lg;
            if (a.act == FASTCOT_BF16) *(uint2*)((bf16_t*)a.out + at) = make_uint2(pk_bf16(o[0], o[1]), pk_bf16(o[2], o[3]));
            else *(f32x4_t*)((float*)a.out + at) = o;
        }
        if (wv == 0 && lg == 0 && x < nrows) {
            if (shared) st_agent_f32x2(mine + RT * Dh + 2 * (16 * qt + lm), M, L);
            else if (a.lse) a.lse[(size_t)row * a.H + h] = Ms * LN2 + logf(L);
        }
    }
    if (shared) {
        wait_vmem_done();
        __syncthreads();
        const int w0 = pg_first_worker(deal, part), parts = pg_last_worker(deal, part) - w0 + 1;
        if (threadIdx.x == 0) arrived = arrive_agent(a.cnt + w0);
        __syncthreads();
        if (arrived == parts - 1) {
            pg_join<G, RT, NW>(a, lds, row0, nrows, first, kvh, w0, parts);
            if (threadIdx.x == 0) st_agent_i32(a.cnt + w0, 0);
        }
    }
    __syncthreads();                                           // (the LDS is written again)
  } while (pg_next<RT>(a, deal, part));
}

// The kernel for many rows: tiles of a wave, groups of rows (KG waves each), waves on a SIMD, and whether the lower
// parts of fp32 queries lie in LDS: what finds its registers without spilling, and 160 KB.
static constexpr int many_tiles(int G) { return G > 4 ? 1 : 2; }
static constexpr int many_groups(int G, int QP) { return G == 8 && QP == 3 ? 2 : 4; }
static constexpr int many_waves(int G, int QP) { return G == 8 && QP == 3 ? 1 : 2; }
static constexpr bool many_low(int G, int QP) { return G < 8 && QP == 3; }
// Many rows of a sequence (prompt chunks, wide windows, windows over grouped heads; bf16 caches): 16 * RG * QT rows a unit, RG waves of QT tiles each, or KG = 2
// times as many, the one half for the even blocks and the other for the odd ones.  The next block (KG of them) goes global -> LDS while the present one is
// used, so that K and V are read once for all the unit's rows and a fragment from LDS once for a wave's QT tiles.  Two waves of the same rows exchange half of
// their sums at the end.  Units that several workgroups share are joined by a launch of its own (k_paged_join).
// Sums are taken relative to a reference that moves only when a score passes it by 8 powers of two: weights are at most 2^8, and in most blocks nothing is
// rescaled.  With bf16 rows the weights are rounded to bf16 once in front of the product with V: as large an error as the rounding of the output, half a
// step of each weight; their sum is taken before the rounding.
// V is multiplied as it is; only where a sum comes out not finite the part is walked once more, carefully (checked in every block, infinities and NaN in V
// cost 3 % of a long walk).
// Bound: per block and tile 16 matrix instructions (bf16 rows; 48 with fp32 rows) beside about 30 vector instructions and 8 exponentials, and a kilobyte out of
// LDS for every two (six) matrix instructions of a wave.  1024 bf16 rows of 32 heads over 20000 positions: 735 TFLOP/s, matrix pipes busy 32 % of the
// cycles, LDS 42, vector unit 38; fp32 rows 365, times three parts 1100, of 1333 that a large product reaches.  Two waves on a SIMD do not fill each other's
// waits, and what would help does not find its registers: three tiles a wave 686, two blocks at a time 703 (both spill), four tiles and one wave a SIMD 454.
template <int G, int QT, int RG, int KG, int QP, int PP>
__global__ __launch_bounds__(64 * RG * KG, many_waves(G, QP)) void k_paged_many(PagedAttnArgs a, int tiles) {
    constexpr int Dh = 32 * G, NV = 2 * G, RT = 16 * RG * QT, SEC = 128 * G, T = 64 * RG * KG;    // SEC: 16-byte words of one block of K or V
    extern __shared__ __align__(16) float lds[];
    __shared__ PagedPart kept_part;
    __shared__ PagedDeal kept_deal;
    __shared__ int bad[2][KG], redo;
    constexpr bool LOW = many_low(G, QP);
    u32x4_t* ql = (u32x4_t*)lds + 4 * KG * SEC;                     // LOW: the lower parts of fp32 queries [row group][tile][fragment][part][64]
    u32x4_t* kv = (u32x4_t*)lds;                               // [buffer][block of the stage][K, V][SEC]
    const int tid = threadIdx.x, lane = tid & 63, lm = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wv / RG, rg = wv % RG;
    // consecutive shares on one XCD: units of one K/V head follow each other and find its blocks in that L2
    const int per = gridDim.x >> 3, worker = gridDim.x & 7 ? blockIdx.x : (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    PagedDeal deal;
    PagedPart part;
    if (tid == 0) a.joins[worker].parts = 0;
    if (!pg_deal<RT>(a, tiles, worker, gridDim.x, deal, part)) return;
    const float scale2 = LOG2E / sqrtf((float)Dh);
    const float unscaled = QP == 1 ? scale2 : 1.f;             // what turns a product into an exponent of two
  do {
    if (part.len <= 0) continue;
    const int kvh = part.kvh, first = part.first, nrows = part.rows, seq = part.seq, n = part.n, g = a.g;
    const int row0 = part.tile * RT, r0 = row0 + 16 * QT * rg; // the unit's rows, this wave's
    const int last = row0 + RT < nrows ? row0 + RT - 1 : nrows - 1;
    const PagedRange vis = pg_range(a, n + pg_token(a, row0), n + pg_token(a, last));
    const int plast = n + pg_token(a, last);
    const bool any_rows = r0 < nrows;
    const int lastw = r0 + 16 * QT < nrows ? r0 + 16 * QT - 1 : nrows - 1;
    const int p0 = n + pg_token(a, any_rows ? r0 : lastw), p1 = n + pg_token(a, lastw);        // positions of the wave's rows
    const int* table = a.c.table + (size_t)(seq < 0 ? 0 : seq) * a.c.MP;
    const int end = part.off + part.len;

    int pos[QT];
    u32x4_t qf[QT][G][LOW ? 1 : QP];                           // queries, or their upper parts
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int x = r0 + 16 * qt + lm, row = x < nrows ? x : nrows - 1, j = pg_token(a, row);
        pos[qt] = x < nrows ? n + j : -1;
        const size_t at = (size_t)(first + j) * a.q_row + (size_t)(kvh * g + row - j * g) * a.q_head;
#pragma unroll
        for (int f = 0; f < G; ++f) {
            const int u = 4 * f + lg, dh = 32 * (u % G) + 8 * (u / G);
            if constexpr (QP == 1) qf[qt][f][0] = *(const u32x4_t*)((const bf16_t*)a.q + at + dh);
            else {
                const float4 y = *(const float4*)((const float*)a.q + at + dh), z = *(const float4*)((const float*)a.q + at + dh + 4);
                const float v[8] = {y.x * scale2, y.y * scale2, y.z * scale2, y.w * scale2, z.x * scale2, z.y * scale2, z.z * scale2, z.w * scale2};
                u32x4_t parts[QP];
                pg_split8<QP>(v, parts);
#pragma unroll
                for (int q = 0; q < (LOW ? 1 : QP); ++q) qf[qt][f][q] = parts[q];
                if constexpr (LOW) ql[(((rg * QT + qt) * G + f) * 2 + kg) * 64 + lane] = kg ? parts[2] : parts[1];
            }
        }
    }
    f32x4_t acc[QT][NV];
    float R[QT], l[QT];                                        // reference of the row's exponents, this lane's share of the sum of weights
    bool far = false;                                          // some reference is far from zero

    // pages of 64 blocks of the part at a time, one a lane: those at hand and the next ones (-1: no page, the block is not used)
    auto pages_from = [&](int x0) {
        const int x = x0 + lane, blk = x < vis.sunk ? x : x - vis.sunk + vis.lo, slot = blk >> a.c.pb;
        const int page = seq >= 0 && x < end && slot < a.c.MP ? table[slot] : -1;
        return page >= 0 && page < a.c.N ? page : -1;
    };
    int now, next, held;                                       // held: the first block of those at hand
    const int inpage = (1 << a.c.pb) - 1;
    u32x4_t stage[4 * G / RG];
    const uint32_t lane16 = lane * 16;
    // requests blocks x .. x + KG - 1, whose pages become page[]
    int page[KG];
    auto load = [&](int x) {
        if (x - held == 64) { held += 64; now = next; next = pages_from(held + 64); }
        size_t at[KG];
#pragma unroll
        for (int y = 0; y < KG; ++y) {
            page[y] = __builtin_amdgcn_readlane(now, x + y - held);
            const int blk = x + y < vis.sunk ? x + y : x + y - vis.sunk + vis.lo;
            at[y] = ((((size_t)(page[y] < 0 ? 0 : page[y]) * a.c.Hkv + kvh) << a.c.pb) + (blk & inpage)) * SEC;
        }
#pragma unroll
        for (int i = 0; i < 4 * G / RG; ++i) {
            const int w0 = i * T + wv * 64, sec = SEC % T ? w0 / SEC : i * T / SEC;         // sec: block of the stage, K or V
            const char* from = (sec & 1 ? a.vl : a.kl) + ((sec & 2 ? at[KG - 1] : at[0]) + (w0 - sec * SEC)) * 16;
            stage[i] = *(const u32x4_t*)(pg_uniform(from) + lane16);
        }
    };
    // puts blocks x .. x + KG - 1 into a buffer.  V gets zeros where the unit's last row does not see it (a weight of zero times an infinity would be none) and,
    // in a careful walk, for what is not finite: of that `bad` keeps the stage's first block, and it is added by itself to the rows that see it
    bool careful = false;
    auto store = [&](int buf, int x) {
#pragma unroll
        for (int i = 0; i < 4 * G / RG; ++i) {
            const int w0 = i * T + wv * 64, sec = SEC % T ? w0 / SEC : i * T / SEC;
            u32x4_t v = stage[i];
            if (sec & 1) {
                const int y = x + (sec >> 1), kb = (y < vis.sunk ? y : y - vis.sunk + vis.lo) << 5;
                if (kb + 31 > plast) {
                    const int past = kb + 8 * lg;              // the positions of this lane's eight values
#pragma unroll
                    for (int w = 0; w < 4; ++w) v[w] &= (past + 2 * w <= plast ? 0x0000FFFFu : 0u) | (past + 2 * w + 1 <= plast ? 0xFFFF0000u : 0u);
                }
                if (careful && pg_not_finite(v)) { pg_make_finite(v); bad[buf][sec >> 1] = x; }
            }
            kv[buf * 2 * KG * SEC + i * T + tid] = v;
        }
    };

    auto compute = [&](const u32x4_t* kb_lds, int kb, bool whole) {
        const u32x4_t* vb_lds = kb_lds + SEC;
        f32x4_t sc[QT][2];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) sc[qt][0] = sc[qt][1] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        // (fragments are read all at once, those of V in front of the softmax: one by one, in front of their instructions, each is a wait)
        u32x4_t kf[2 * G], vf[NV];
#pragma unroll
        for (int f = 0; f < 2 * G; ++f) kf[f] = kb_lds[f * 64 + lane];
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);                         // (the other wave of the SIMD has exponentials to do)
#pragma unroll
        for (int f = 0; f < G; ++f) {
            if constexpr (QP == 3) {                           // (small parts first)
                u32x4_t lower[2][QT];
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
#pragma unroll
                    for (int q = 1; q >= 0; --q) lower[q][qt] = LOW ? ql[(((rg * QT + qt) * G + f) * 2 + q) * 64 + lane] : qf[qt][f][LOW ? 0 : q + 1];
#pragma unroll
                for (int q = 1; q >= 0; --q)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int qt = 0; qt < QT; ++qt)
                            sc[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[t * G + f]), __builtin_bit_cast(bf16x8_t, lower[q][qt]), sc[qt][t], 0, 0, 0);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                    sc[qt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[t * G + f]), __builtin_bit_cast(bf16x8_t, qf[qt][f][0]), sc[qt][t], 0, 0, 0);
        }
#pragma unroll
        for (int f = 0; f < NV; ++f) vf[f] = vb_lds[f * 64 + lane];
        __builtin_amdgcn_s_setprio(0);
        float p[QT][8], by = unscaled, from[QT], top[QT];
        bool moves = false;                                    // weights are 2^(by * p - from)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int e = 0; e < 8; ++e) p[qt][e] = sc[qt][e >> 2][e & 3];
        if (!whole) {
            const bool sunk = kb < a.sinks;
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) pg_mask8(a, kb + 8 * lg, pos[qt], sunk, p[qt]);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            top[qt] = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) top[qt] = fmaxf(top[qt], p[qt][e]);
            top[qt] *= by;
            moves |= top[qt] > R[qt] + 8.f;
        }
        if (__any(moves)) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                float m = fmaxf(top[qt], __shfl_xor(top[qt], 16, 64));
                m = fmaxf(m, __shfl_xor(m, 32, 64));
                if (!(m > R[qt] + 8.f)) m = R[qt];
                const float alpha = __builtin_amdgcn_exp2f(R[qt] - m);
                R[qt] = m;
                far = far || __any(m > 1048576.f || (m < -1048576.f && m > ROW_NONE));
                l[qt] *= alpha;
#pragma unroll
                for (int f = 0; f < NV; ++f) acc[qt][f] *= alpha;
            }
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) from[qt] = R[qt];
        if (QP == 1 && far) {
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) { by = unscaled; pg_far(p[qt], by, from[qt]); }
        }
        // one tile's weights beside another one's products
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            u32x4_t pf[PP];
#pragma unroll
            for (int e = 0; e < 8; ++e) { p[qt][e] = __builtin_amdgcn_exp2f(fmaf(p[qt][e], by, -from[qt])); l[qt] += p[qt][e]; }
            pg_split8<PP>(p[qt], pf);
#pragma unroll
            for (int q = PP - 1; q >= 0; --q)
#pragma unroll
                for (int f = 0; f < NV; ++f) acc[qt][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf[f]), __builtin_bit_cast(bf16x8_t, pf[q]), acc[qt][f], 0, 0, 0);
        }
    };
    // what is not finite in V of block blk of a page, for the rows that see it
    auto add_infinite = [&](int blk, int page) {
        const u32x4_t* v = (const u32x4_t*)a.vl + ((((size_t)page * a.c.Hkv + kvh) << a.c.pb) + (blk & inpage)) * SEC + lane;
        u32x4_t sees[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) sees[qt] = pg_seen8(a, (blk << 5) + 8 * lg, pos[qt]);
#pragma unroll
        for (int f = 0; f < NV; ++f) {
            u32x4_t up = v[f * 64], down;
            pg_infinite(up, down);
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) pg_add_infinite(acc[qt][f], up, down, sees[qt]);
        }
    };

    if (tid == 0) { kept_part = part; kept_deal = deal; redo = 0; }        // (scalar registers are short in the walk)
    for (;;) {
        now = pages_from(part.off); next = pages_from(part.off + 64); held = part.off;
        far = false;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            R[qt] = ROW_NONE; l[qt] = 0.f;
#pragma unroll
            for (int f = 0; f < NV; ++f) acc[qt][f] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        if (tid < 2 * KG) bad[tid / KG][tid % KG] = -1;
        load(part.off);
        __syncthreads();
        store(0, part.off);
        __syncthreads();
        int buf = 0;
        for (int x = part.off; x < end; x += KG) {
            const int blk = x + kg < vis.sunk ? x + kg : x + kg - vis.sunk + vis.lo, kb = blk << 5, here = page[kg ? KG - 1 : 0];
            if (x + KG < end) load(x + KG);                        // travels while this stage is used
            __builtin_amdgcn_sched_barrier(0);
            // does any row of the wave see the block, and do all of them see all of it
            const bool seen = any_rows && x + kg < end && here >= 0 && kb <= p1 && (!a.window || kb + 31 > p0 - a.window || kb < a.sinks);
            const bool whole = kb + 31 <= p0 && (!a.window || kb > p1 - a.window || kb + 31 < a.sinks);
            if (seen) {
                const u32x4_t* at = kv + (buf * 2 * KG + 2 * kg) * SEC;
                compute(at, kb, whole);
                if (careful && bad[buf][kg] == x) add_infinite(blk, here);
            }
            if (x + KG < end) store(buf ^ 1, x + KG);
            __syncthreads();
            buf ^= 1;
        }
        if (careful) break;
        float z = 0.f;                                         // not a number where a sum is not finite
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
            for (int f = 0; f < NV; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = fmaf(acc[qt][f][i], 0.f, z);
        if (z != z) redo = 1;
        __syncthreads();
        if (!redo) break;
        careful = true;                                        // once more: V is not finite somewhere (or a query or a key is not)
    }

    part = pg_uniform(kept_part); deal = pg_uniform(kept_deal);
    // two waves of the same rows exchange half of their sums: group 0 finishes the lower half of the fragments, group 1 the upper one
    constexpr int FW = NV / KG, XW = QT * (FW * 256 + 128);
    const float* theirs = lds + (wv ^ RG) * XW;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        l[qt] += __shfl_xor(l[qt], 16, 64);
        l[qt] += __shfl_xor(l[qt], 32, 64);
        if constexpr (KG == 2) {
            float* to = lds + wv * XW + qt * (FW * 256 + 128);
#pragma unroll
            for (int f = 0; f < FW; ++f) *(f32x4_t*)(to + (f * 64 + lane) * 4) = kg == 0 ? acc[qt][NV - FW + f] : acc[qt][f];
            to[FW * 256 + lane] = R[qt];
            to[FW * 256 + 64 + lane] = l[qt];
        }
    }
    if constexpr (KG == 2) __syncthreads();
    const bool shared = part.len < part.blocks;
    float* slot = a.part + (size_t)(2 * worker + (part.off == 0)) * RT * (Dh + 2);
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const float* from = theirs + qt * (FW * 256 + 128);
        float M = R[qt], L = l[qt], wi = 1.f, wo = 0.f;
        if constexpr (KG == 2) {
            const float Ro = from[FW * 256 + lane];
            M = fmaxf(R[qt], Ro); wi = __builtin_amdgcn_exp2f(R[qt] - M); wo = __builtin_amdgcn_exp2f(Ro - M);
            L = l[qt] * wi + from[FW * 256 + 64 + lane] * wo;
        }
        const float inv = shared ? 1.f : L == 0.f ? 0.f : 1.f / L;
        const int x = r0 + 16 * qt + lm, j = pg_token(a, x), row = first + j, h = kvh * g + x - j * g, xs = x - row0;
        if (x >= nrows) continue;
        const size_t at = (size_t)row * a.out_row + (size_t)h * Dh + 4 * lg;
#pragma unroll
        for (int f = 0; f < FW; ++f) {
            f32x4_t o = kg == 0 ? acc[qt][f] : acc[qt][NV - FW + f];
            if constexpr (KG == 2) o = o * wi + *(const f32x4_t*)(from + (f * 64 + lane) * 4) * wo;
            o *= inv;
            const int ff = kg * FW + f;
            if (shared) {
                *(f32x4_t*)(slot + xs * Dh + 16 * ff + 4 * lg) = o;
            } else if (a.act == FASTCOT_BF16) *(uint2*)((bf16_t*)a.out + at + 16 * ff) = make_uint2(pk_bf16(o[0], o[1]), pk_bf16(o[2], o[3]));
            else *(f32x4_t*)((float*)a.out + at + 16 * ff) = o;
        }
        if (kg == 0 && lg == 0) {
            if (shared) *(float2*)(slot + RT * Dh + 2 * xs) = make_float2(M, L);
            else if (a.lse) a.lse[(size_t)row * a.H + h] = M * LN2 + logf(L);
        }
    }
    if (shared && part.off == 0 && tid == 0) {
        a.joins[worker] = PagedJoin{row0, nrows, first, kvh, pg_last_worker(deal, part) - worker + 1};
    }
    __syncthreads();
  } while (pg_next<RT>(a, deal, part));
}

// Joins the units that several workgroups of k_paged_many share, 16 rows a workgroup (a launch of its own: the last workgroup to arrive would read
// 66 KB a part alone, 60 us for 16 rows of 64 heads on 8 over 2000 positions)
template <int G, int RT>
__global__ __launch_bounds__(256, 1) void k_paged_join(PagedAttnArgs a) {
    constexpr int Dh = 32 * G, SLOT = RT * (Dh + 2);
    const int w0 = blockIdx.x / (RT / 16), chunk = blockIdx.x % (RT / 16);
    const PagedJoin j = a.joins[w0];
    const float* p0 = a.part + (size_t)(2 * w0 + 1) * SLOT;    // the first part's slot; the others' are the even ones behind it
    for (int y = threadIdx.x; y < 16 * Dh / 4; y += 256) {
        const int r = 16 * chunk + y / (Dh / 4), d = 4 * (y % (Dh / 4));
        if (j.parts == 0 || j.row0 + r >= j.nrows) return;
        float M = -INFINITY, L = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0; i0 < j.parts; i0 += 8) {
            float2 ml[8];
            f32x4_t v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = i0 + e < j.parts ? i0 + e : i0;
                const float* s = p0 + (i ? (size_t)(2 * i - 1) * SLOT : 0);
                ml[e] = *(const float2*)(s + RT * Dh + 2 * r);
                v[e] = *(const f32x4_t*)(s + r * Dh + d);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (i0 + e >= j.parts) continue;
                const float Mn = fmaxf(M, ml[e].x), x = __builtin_amdgcn_exp2f(M - Mn), w = __builtin_amdgcn_exp2f(ml[e].x - Mn);
                L = L * x + ml[e].y * w;
                o = o * x + v[e] * w;
                M = Mn;
            }
        }
        const int tk = pg_token(a, j.row0 + r), row = j.first + tk, h = j.kvh * a.g + j.row0 + r - tk * a.g;
        o *= L == 0.f ? 0.f : 1.f / L;
        const size_t at = (size_t)row * a.out_row + (size_t)h * Dh + d;
        if (a.act == FASTCOT_BF16) *(uint2*)((bf16_t*)a.out + at) = make_uint2(pk_bf16(o[0], o[1]), pk_bf16(o[2], o[3]));
        else *(f32x4_t*)((float*)a.out + at) = o;
        if (a.lse && d == 0) a.lse[(size_t)row * a.H + h] = M * LN2 + logf(L);
    }
}

#define PG_WORKERS 512           // most workgroups of a launch
// partial results: two slots a workgroup, of up to 32 rows, or of a unit of many rows
size_t fc_paged_attn_scratch_bytes(int Dh) {
    const size_t few = (size_t)PG_WORKERS * 2 * 32, many = (size_t)PG_WORKERS * 2 * 64 * many_tiles(Dh / 32);
    return (few > many ? few : many) * (Dh + 2) * 4;
}

template <int G, bool F32, int QT, int NW, int QP, int PP>
static hipError_t launch_as(PagedAttnArgs a, int grid, hipStream_t st) {
    const int rows = a.r.R * a.g;
    const size_t bytes = (size_t)NW * QT * (32 * G * 16 + 32) * 4;
    auto kernel = k_paged_attn<G, F32, QT, NW, QP, PP>;
    // (more than 64 KB of LDS have to be asked for)
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
    a.whole = 4 * NW;          // blocks of a unit that is not cut: four rounds of its waves take about as long as a meeting in memory
    kernel<<<grid < PG_WORKERS ? grid : PG_WORKERS, NW * 64, bytes, st>>>(a, (rows + 16 * QT - 1) / (16 * QT));
    return hipGetLastError();
}
// Many rows.  bf16 rows: with more units than CUs two workgroups of four waves on every CU, so that one's products go on while the other one is between
// units (4096 rows of 32 heads under a window of 1024: 146 us with eight waves, 129 so); fewer units find eight waves sooner done (1024 rows from the
// start of a sequence 38 / 44, 128 rows 16 / 20, 64 rows of 64 heads on 8 over 20000 positions 78 / 82).  fp32 rows, whose lower parts fill the LDS: eight waves.
template <int G, int QP, int KG>
static hipError_t launch_many(PagedAttnArgs a, int grid, hipStream_t st) {
    constexpr int QT = many_tiles(G), RG = many_groups(G, QP), RT = 16 * RG * QT;
    const size_t stage = KG * 4 * 128 * G * 16, low = many_low(G, QP) ? RG * QT * G * 2 * 1024 : 0, meet = KG == 2 ? 2 * RG * QT * (G * 256 + 128) * 4 : 0;
    const size_t bytes = stage + low > meet ? stage + low : meet;
    auto kernel = k_paged_many<G, QT, RG, KG, QP, QP>;
    const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
    a.whole = 16;
    if (grid > PG_WORKERS) grid = PG_WORKERS;
    kernel<<<grid, 64 * RG * KG, bytes, st>>>(a, (a.r.R * a.g + RT - 1) / RT);
    k_paged_join<G, RT><<<grid * (RT / 16), 256, 0, st>>>(a);
    return hipGetLastError();
}
// Up to 16 rows: where every unit finds a CU of its own, eight waves share its blocks; with more units two workgroups of four waves on every CU, so that
// one's loads go on while the other one's waves meet (32 sequences of 100 to 500 positions over 32 heads 36.7 / 31.3 us, 200 of 20 to 300 over 8 heads
// 41.7 / 32.9; the other way round 7B heads, 8000 positions 26.5 / 26.8, 70B heads, 120000 positions 88 / 100, 7B window of 16, 777 positions 13.3 / 15.8).
// 17 to 32 rows run as two tiles, by as many waves as find their registers (eight instead of four, bf16 rows: 64 heads on 8, 4 rows, 2000 positions 27.2 / 22.7 us,
// 40 sequences of 1000 54.9 / 48.2; the kernel for many rows 20.7 and 44.9 there, but 16 heads on 4 27.6 for 15.9), bf16 heads of more than 128 elements as many
// rows (8 heads on 4 of 256, fp32 rows: 66.6 / 34.9), fp32 heads of 256, which would spill, as single tiles (88.7 / 53.1).
static constexpr int pair_waves(int G, bool F32, int QP) { return G <= (F32 ? 2 : QP == 1 ? 4 : 3) ? 8 : 4; }
template <int G, bool F32, int QP, int PP>
static hipError_t launch(const PagedAttnArgs& a, hipStream_t st) {
    const int cus = fc_num_cus();
    if constexpr (!F32) {
        if (a.r.R * a.g > (G > 4 ? 16 : 32)) {
            constexpr int RT = 16 * many_groups(G, QP) * many_tiles(G);
            if constexpr (QP == 1)
                if ((int64_t)a.r.B * a.c.Hkv * ((a.r.R * a.g + RT - 1) / RT) > cus) return launch_many<G, QP, 1>(a, 2 * cus, st);
            return launch_many<G, QP, 2>(a, cus, st);
        }
    }
    if constexpr (G <= 4 || (F32 && G < 8))
        if (a.r.R * a.g > 16) return launch_as<G, F32, 2, pair_waves(G, F32, QP), QP, PP>(a, cus, st);
    if constexpr (G <= 4) {
        if ((int64_t)a.r.B * a.c.Hkv <= cus) return launch_as<G, F32, 1, 8, QP, PP>(a, cus, st);
        return launch_as<G, F32, 1, 4, QP, PP>(a, 2 * cus, st);
    }
    return launch_as<G, F32, 1, 4, QP, PP>(a, cus, st);
}
template <int G> static hipError_t by_type(const PagedAttnArgs& a, hipStream_t st) {
    if (a.esz == 4) return launch<G, true, 1, 1>(a, st);
    return a.act == FASTCOT_BF16 ? launch<G, false, 1, 2>(a, st) : launch<G, false, 3, 3>(a, st);
}
hipError_t fc_paged_attn(const PagedAttnArgs& a, hipStream_t st) {
    switch (a.c.Dh) {
    case 32: return by_type<1>(a, st);
    case 64: return by_type<2>(a, st);
    case 96: return by_type<3>(a, st);
    case 128: return by_type<4>(a, st);
    case 192: return by_type<6>(a, st);
    case 256: return by_type<8>(a, st);
    }
    return hipErrorInvalidValue;
}
