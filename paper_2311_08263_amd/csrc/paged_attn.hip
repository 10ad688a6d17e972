// Attention of a pass's rows over a K/V cache in pages: row at position p sees k <= p that has a page and, under a sliding window,
// k > p - window or k < sinks.
//
//   s_k = q . k / sqrt(Dh),  m = max s_k,  l = sum e^(s_k - m),  out = sum e^(s_k - m) v_k / l,  lse = m + ln l
//
// A unit is 16 or 32 rows (token by token, the query heads of a K/V head next to each other) of one sequence and K/V head, a workgroup's work:
// its waves take the visible blocks of 32 positions in turn, keep m, l and the sums in registers and meet in LDS.  Scores S^T = K . Q^T and
// sums O^T += V^T . P^T are matrix instructions whose operands lie in the cache as they are needed (k_index, v_index); for any head size
// the 16-byte pieces u = 4 f + lane / 16 of a score tile's fragment f hold head elements 32 (u % G) + 8 (u / G) .. + 7, G = Dh / 32.
// bf16 caches run on bf16 instructions with fp32 queries and weights in three parts (24 bits, so results are those of fp32 arithmetic) or bf16
// queries in one and weights in two; fp32 caches on fp32 instructions.
// Blocks that some row does not see whole are edges: their scores are masked, and V of positions that no row of the unit sees is taken as zero (a
// weight of zero times an infinity is none).  Where V is not finite at a position that some rows see and others do not, the block's products
// are summed position by position.
#include "paged.h"

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;

#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f

// The parts of a fp32 value are cut off its bits from the top, so that none overflows and three hold all 24 bits
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
            if (t == TERMS - 1 && TERMS < 3) w[e] = pk_bf16(x[2 * e], x[2 * e + 1]);          // the last of fewer parts is rounded
            else w[e] = (a >> 16) | (b & 0xFFFF0000u);
            if (t < TERMS - 1) { x[2 * e] -= __uint_as_float(a & 0xFFFF0000u); x[2 * e + 1] -= __uint_as_float(b & 0xFFFF0000u); }
        }
        part[t] = (u32x4_t){w[0], w[1], w[2], w[3]};
    }
}
__device__ inline bool pg_sees(const PagedAttnArgs& a, int key, int pos) {
    return key <= pos && (!a.window || key > pos - a.window || key < a.sinks);
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

// G: 32s of a head; F32: fp32 cache; QT: tiles of 16 rows of a unit; NW: waves; QP, PP: bf16 parts of queries and weights
template <int G, bool F32, int QT, int NW, int QP, int PP>
__global__ __launch_bounds__(NW * 64, 1) void k_paged_attn(PagedAttnArgs a, int tiles) {
    constexpr int Dh = 32 * G, NV = 2 * G, RT = 16 * QT;       // NV: fragments of V, four sums of a lane each
    constexpr int PART = Dh * 16 + 32;                         // floats of a wave's tile: sums, then m and l of the 16 rows
    extern __shared__ float lds[];
    const int lane = threadIdx.x & 63, lm = lane & 15, lg = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x % tiles, kvh = blockIdx.x / tiles % a.c.Hkv, b = blockIdx.x / tiles / a.c.Hkv;
    const int g = a.H / a.c.Hkv;
    int first, count;
    pg_rows(a.r, b, first, count);
    const int row0 = tile * RT, nrows = count * g;             // rows of the unit: row0 .. of nrows, row x = head x % g of token x / g
    if (row0 >= nrows) return;
    const int seq = pg_seq(a.r, a.c, b), n = seq < 0 ? 0 : pg_len(a.c, seq);
    const int j0 = row0 / g, last = row0 + RT < nrows ? row0 + RT - 1 : nrows - 1, j1 = last / g;
    const int p0 = n + j0, p1 = n + j1;
    const PagedRange vis = pg_range(a, p0, p1);
    const int* table = a.c.table + (size_t)(seq < 0 ? 0 : seq) * a.c.MP;
    const int blocks = seq < 0 ? 0 : vis.sunk + vis.hi - vis.lo;
    const float scale2 = LOG2E / sqrtf((float)Dh);             // the softmax runs in powers of two

    int pos[QT];                                               // this lane's rows: row row0 + 16 * qt + lm (-1: none)
    u32x4_t qf[F32 ? 1 : QT][G][QP];
    float qx[F32 ? QT : 1][G][8];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int x = row0 + 16 * qt + lm, row = x < nrows ? x : last, j = row / g;
        pos[qt] = x < nrows ? n + j : -1;
        const size_t at = (size_t)(first + j) * a.q_row + (size_t)(kvh * g + row % g) * a.q_head;
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

    for (int x = wv; x < blocks; x += NW) {
        const int blk = x < vis.sunk ? x : x - vis.sunk + vis.lo, kb = blk << 5;
        const int slot = blk >> a.c.pb;
        const int page = slot < a.c.MP ? table[slot] : -1;
        if (page < 0 || page >= a.c.N) continue;
        const size_t at = ((((size_t)page * a.c.Hkv + kvh) << a.c.pb) + (blk & ((1 << a.c.pb) - 1))) * 32 * Dh;
        constexpr int FW = F32 ? 2 : 1;                        // 16-byte words of a lane's eight values
        const u32x4_t* kp = (const u32x4_t*)(a.kl + at * (F32 ? 4 : 2)) + lane * FW;
        const u32x4_t* vp = (const u32x4_t*)(a.vl + at * (F32 ? 4 : 2)) + lane * FW;
        u32x4_t kf[2 * G][FW], vf[NV][FW];
#pragma unroll
        for (int f = 0; f < 2 * G; ++f)
#pragma unroll
            for (int w = 0; w < FW; ++w) kf[f][w] = __builtin_nontemporal_load(kp + f * 64 * FW + w);
#pragma unroll
        for (int f = 0; f < NV; ++f)
#pragma unroll
            for (int w = 0; w < FW; ++w) vf[f][w] = __builtin_nontemporal_load(vp + f * 64 * FW + w);
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
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = pg_sees(a, kb + 8 * lg + e, pos[qt]) ? p[e] : -INFINITY;
            }
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
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int x = row0 + 16 * qt + lm;
        float M = -INFINITY, L = 0.f, w[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) { w[i] = lds[(i * QT + qt) * PART + Dh * 16 + lm]; M = fmaxf(M, w[i]); }
        const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int i = 0; i < NW; ++i) { w[i] = __builtin_amdgcn_exp2f(w[i] - Ms); L += lds[(i * QT + qt) * PART + Dh * 16 + 16 + lm] * w[i]; }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int row = first + x / g, h = kvh * g + x % g;
        for (int f = wv; f < NV; f += NW) {
            f32x4_t o = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const f32x4_t y = *(const f32x4_t*)(lds + (i * QT + qt) * PART + (f * 64 + lane) * 4);
                o += y * w[i];
            }
            o *= inv;
            if (x >= nrows) continue;
            const size_t at = (size_t)row * a.out_row + (size_t)h * Dh + 16 * f + 4 * lg;
            if (a.act == FASTCOT_BF16) *(uint2*)((bf16_t*)a.out + at) = make_uint2(pk_bf16(o[0], o[1]), pk_bf16(o[2], o[3]));
            else *(f32x4_t*)((float*)a.out + at) = o;
        }
        if (a.lse && wv == 0 && lg == 0 && x < nrows) a.lse[(size_t)row * a.H + h] = Ms * LN2 + logf(L);
    }
}

size_t fc_paged_attn_scratch_bytes(int Dh) { return 0 * Dh; }

template <int G, bool F32, int QP, int PP>
static hipError_t launch(const PagedAttnArgs& a, hipStream_t st) {
    constexpr int NW = G <= 4 ? 8 : 4;
    const int rows = a.r.R * (a.H / a.c.Hkv);
    const bool two = rows > 16;
    const int tiles = (rows + (two ? 31 : 15)) / (two ? 32 : 16);
    const unsigned grid = (unsigned)(tiles * a.c.Hkv) * (unsigned)a.r.B;
    const size_t bytes = (size_t)NW * (two ? 2 : 1) * (32 * G * 16 + 32) * 4;
    auto one = k_paged_attn<G, F32, 1, NW, QP, PP>;
    auto pair = k_paged_attn<G, F32, 2, NW, QP, PP>;
    // (more than 64 KB of LDS have to be asked for)
    const hipError_t e = hipFuncSetAttribute((const void*)(two ? pair : one), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
    if (two) pair<<<grid, NW * 64, bytes, st>>>(a, tiles);
    else one<<<grid, NW * 64, bytes, st>>>(a, tiles);
    return hipGetLastError();
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
