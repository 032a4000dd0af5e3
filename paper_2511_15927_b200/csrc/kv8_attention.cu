// Attention of a block's queries over the 8-bit key/value cache, one length per sequence, and what each cached row receives.
//   s_rj = f_rj q'_r . k_j,  p_rj = 2^(s_rj - m_r),  out_r = sum_j p_rj vs_j v_j / sum_j p_rj          (k, v: codes;  f: every scale, in log2 units)
// Bound by reading the cache: 2 D bytes per row and head against 4 D products per query.  All keys of all heads are cut into shares, a CTA each;
// its four warps take tiles of 32 rows (= the rows that share a scale) in turn, each through a ring of untiled bulk copies of its own (a tile is contiguous), with a running
// maximum and sum of its own, and are joined in shared memory; the pieces of a head that several shares have are joined by a second launch.  At 32 and fewer queries the products are a
// fraction of a tcgen05 tile and run on mma.sync, with nothing but the copies between memory and its operands:
//   - a tile's codes are operands after one conversion (e4m3 -> f16, exact).  The order of a product's inner index is free as long as both operands agree, so
//     a thread's K operand is 16 consecutive channels of one row and its V operand 8 consecutive rows of one channel: 16- and 8-byte shared-memory loads, no transposition.
//   - Q is brought to f16 by a power of two per row (its largest channel in [1, 2)): exact for all channels above 2^-14 of it, the others lose less than the sum's rounding.
//   - P is rounded to f16 (11 significant bits where bf16 has 8) with the tile's V scale in it: p' = 2^(s + e + nref), e the scale's exponent, so the running output is the
//     product's own accumulator.  nref follows the maximum of s + e, what the output is made of; the sum of p alone has a reference of its own, kept at 2^(s + nref + lr), lr whole.
// Measured in a captured graph, joining launch included: 16 sequences of up to 16384 rows, 8 kv heads of 128, 4 queries each, 73 us = 5.6 TB/s (the floor 63; the rest is start and end); 4 x up to
// 65536 rows, 16 heads of 64, 32 queries, 115 us = 3.8 TB/s: there the products take 59 us of the tensor pipe (half of the time, 16 clocks between two products of one warp), and the
// copies alone take 79.  One sequence of 8192 rows, 24 heads of 80: 32 queries 19.4 us; 16 heads of 64, one query 11.4 us, launches and latencies (2 us of them the joining launch).
// Where many queries meet a head the products bound it, at 221 TFLOP/s (4 x 16384 rows, 8 heads of 128, 128 rows of queries each: 126 us) and 260 (a prompt of 8191, 24 heads of 80: 1982 us): each
// 16 or 32 rows of queries convert the codes anew.
#include "kv8.cuh"
#include "tc_ptx.cuh"

namespace dm {
namespace {

using namespace kv8;
using namespace tc;

constexpr int NW = 4, NT = NW * 32;
// p' is 2^8 at a row's maximum when its reference is set and may grow to 2^15 before the reference moves: f16 ends at 2^16, and below 2^-22 of the maximum P loses bits one by one until
// 2^-33.  So the reference needs no agreement between the four lanes of a row in every tile: a lane whose own scores stay below the limit has nothing to do, and
// after the first tiles one vote per tile is all that is left of the running maximum.
// lr is about what the row's largest s + e exceeds its largest s by, the exponent of the scales that matter to it.  A term of the sum is p' 2^(lr - e): where e lies no more than L_SPAN below lr it
// is at most 2^(P_LIMIT + L_SPAN).  A tile of smaller scale than that (2^-100 where V is nothing but zeros) may have rows that the sum is made of while p' underflows: its terms are formed on
// their own, and the sum's reference moves when one would exceed the same limit.
constexpr float P_START = 8.f, P_LIMIT = 15.f, NO_REF = 3.0e38f;
constexpr int L_SPAN = 25;
__device__ __forceinline__ int exponent_of(float pow2) { return (__float_as_int(pow2) >> 23) - 127; }
__device__ __forceinline__ float pow2_of(int e) { return __int_as_float((e + 127) << 23); }        // e in [-126, 127]

struct AttnArgs {
    Cache c;
    const __nv_bfloat16 *q;                        // [B * G] rows of pitch ld_q, heads side by side
    int64_t ld_q;
    const int32_t *lens, *counts;
    __nv_bfloat16 *out;                            // [B * G] rows of pitch ld_out
    int64_t ld_out;
    int B, G, H, Hkv, group, R;                    // R = group * G rows per (sequence, kv head): row = head of the group * G + token
    int max_rows;                                  // lens[b] + counts[b] is clamped to it
    int slots, by_pair;                            // shares of the work, and how they are cut (see Shares)
    int rt;                                        // row tiles of 16 MT rows
    int join_tiles;                                // row tiles of the joining launch
    float scale_log2;                              // log2(e) / sqrt(D)
    float *po;                                     // [slots][2][R][D] unnormalised outputs of the pieces of (sequence, head) pairs that several shares have
    float2 *pml;                                   // [slots][2][R]    their (reference, sum)
    float2 *stat;                                  // [B * Hkv][R] (reference, 1 / sum) of every row, or NULL
    int *status;
};

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_16816_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {      // D = A B
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void four_codes(uint32_t w, uint32_t &lo, uint32_t &hi) {      // e4m3 -> f16, codes 0, 1 and 2, 3
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The channels that K step `k` of thread column `qc` covers: four consecutive ones from chan(k, qc).  Whole 64-channel pieces are 16 channels (16 bytes of codes) per
// thread; 16 left over (D = 80) are four.
template <int D> __device__ __forceinline__ constexpr int chan(int k, int qc) { return k < D / 64 * 4 ? 64 * (k / 4) + 16 * qc + 4 * (k & 3) : 16 * k + 4 * qc; }

// One row's four K-step channels of Q as f16 pairs; `up`: the row's power of two.
struct QRow {
    const __nv_bfloat16 *p;                        // NULL: a row of zeros
    __device__ __forceinline__ uint2 raw(int c) const { return p ? __ldg(reinterpret_cast<const uint2 *>(p + c)) : make_uint2(0, 0); }
};
__device__ __forceinline__ uint32_t absmax2(uint32_t w) { return max((w << 16) & 0x7fff0000u, w & 0x7fff0000u); }
__device__ __forceinline__ uint32_t f16_pair(uint32_t bf2, float up) { return pack_f16(__uint_as_float(bf2 << 16) * up, __uint_as_float(bf2 & 0xffff0000u) * up); }

// Q operand fragments of 16 rows: rows gr and gr + 8 of this thread; f: what a score of each row is to be multiplied with
template <int D>
__device__ __forceinline__ void load_q(const QRow (&row)[2], int qc, uint32_t (&qf)[D / 16][4], float (&f)[2]) {
    float up[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            const uint2 w = row[r].raw(chan<D>(k, qc));
            qf[k][r] = w.x; qf[k][2 + r] = w.y;
            top = max(top, max(absmax2(w.x), absmax2(w.y)));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^-e of the largest magnitude's exponent e, kept to normal numbers; an infinite or NaN channel stays what it is
        const int e = min(max((int)(top >> 23), 2), 252);
        up[r] = __int_as_float((254 - e) << 23);
        f[r] = __int_as_float(e << 23);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) { qf[k][r] = f16_pair(qf[k][r], up[r]); qf[k][2 + r] = f16_pair(qf[k][2 + r], up[r]); }
    }
}

// K operands of the eight rows that tile column group j of a 32-row tile stands for: row 8 (gr / 2) + 2 j + (gr & 1), so that the scores' columns 2 qc, 2 qc + 1 of
// group j are rows 8 qc + 2 j, + 1: the rows whose V codes a thread loads as eight consecutive bytes.
template <int D>
__device__ __forceinline__ void load_k(const uint8_t *tile, int gr, int qc, int j, uint32_t (&w)[D / 16]) {
    const uint8_t *p = tile + (8 * (gr >> 1) + 2 * j + (gr & 1)) * D;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p + 64 * i + 16 * qc);
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
#pragma unroll
    for (int k = D / 64 * 4; k < D / 16; ++k) w[k] = *reinterpret_cast<const uint32_t *>(p + 16 * k + 4 * qc);
}

template <int D, int MT> struct Smem {
    static constexpr uint32_t TILE = BLK * D;                                        // bytes of a K or V tile
    // CTAs per SM and stages of the rings: two tiles' scores at a time take 160 registers with 16 query rows, 250 with 32; the rings share what shared memory there is.  Tiles of 128 channels
    // want three stages more than a third CTA (16 x up to 16384 rows, 8 heads: 72.6 us, with three CTAs of two stages 76.0).
    static constexpr int CTAS = MT == 1 && D < 128 ? 3 : 2;
    static constexpr int STAGES = D == 64 ? (MT == 1 ? 4 : 6) : D == 80 ? (MT == 1 ? 3 : 4) : 3;
    static constexpr uint32_t ring = 0, q = ring + NW * STAGES * 2 * TILE, bar = q + MT * (D / 16) * 512, abort_flag = bar + NW * STAGES * 8, total = abort_flag + 16;
    // after the loop the ring's bytes hold the warps' outputs, references and sums
    static constexpr uint32_t ow = 0, mw = ow + NW * 16 * MT * D * 4, lw = mw + NW * 16 * MT * 4, join_end = lw + NW * 16 * MT * 4;
    static_assert(join_end <= q && (total + 1024) * CTAS <= 227 * 1024, "the join fits the ring, the CTAs fit an SM");
};

struct Place { int b, h, len, n, live; };          // sequence, kv head, committed rows, rows to attend to, tokens of the block
__device__ __forceinline__ Place place(const AttnArgs &a, int bh) {
    Place p;
    p.b = bh / a.Hkv; p.h = bh - p.b * a.Hkv;
    p.live = a.counts ? min(max(a.counts[p.b], 0), a.G) : a.G;
    const int top = min(a.c.cap, a.max_rows);
    p.len = min(max(a.lens[p.b], 0), top);
    p.n = min(p.len + p.live, top);
    return p;
}
__device__ __forceinline__ QRow q_row(const AttnArgs &a, const Place &p, int row, int D) {
    const int hl = row / a.G, t = row - hl * a.G;
    return QRow{row < a.R && t < p.live ? a.q + ((int64_t)p.b * a.G + t) * a.ld_q + (int64_t)(p.h * a.group + hl) * D : nullptr};
}

// The work is the sequence of all groups of NW tiles, by sequence, then kv head, then row.  A share of it is a CTA's (one CTA's for each row tile).
//   - Few (sequence, head) pairs: each is cut into pieces, as many as its part of the slots, and a share is a piece.
//   - Many: the whole is cut into equal shares, whatever the sequences' lengths are.  A share begins and ends inside a pair as a rule, and starts anew (queries, references, the ring) at each
//     pair, 4 us or so, which is why few pairs are not cut this way.
// Pieces of a pair go to the workspace and are joined by the second launch, which finds them by the same arithmetic; pairs that lie inside a share are written
// at once.  A sequence without rows but with queries counts as one group (its output is zeros).
__device__ __forceinline__ int groups_of(const AttnArgs &a, int b) {
    if (b >= a.B) return 0;
    const int live = a.counts ? min(max(a.counts[b], 0), a.G) : a.G, top = min(a.c.cap, a.max_rows);
    const int n = min(min(max(a.lens[b], 0), top) + live, top);
    return live == 0 ? 0 : max(1, (n + NW * BLK - 1) / (NW * BLK));
}
struct Shares { long long total; int n; };         // groups in all, shares in use
__device__ __forceinline__ long long div_of(long long x, long long y) {   // non-negative; a 64-bit division takes half a microsecond here
    return (unsigned long long)(x | y) >> 32 ? x / y : (long long)((uint32_t)x / (uint32_t)y);
}
__device__ __forceinline__ int pieces_of(const AttnArgs &a, const Shares &s, int g) { return g ? max(1, min(g, (int)div_of((long long)a.slots * g, s.total))) : 0; }
__device__ __forceinline__ long long share_begin(const Shares &s, int i) { return div_of(s.total * i, s.n); }
__device__ __forceinline__ int share_of(const Shares &s, long long g) { return (int)div_of((g + 1) * s.n - 1, s.total); }     // the one that holds group g
// A sum over sequences, each kv head once: of what comes before sequence b, and of all; whole warp.  (Below 2^31: a group is 128 rows of memory.)  `mine`: lane i's groups of sequence i, read
// once and enough when there are no more than 32.
template <typename F> __device__ __forceinline__ int sum_of(const AttnArgs &a, int mine, int b, int *before, F weight) {
    const int lane = threadIdx.x & 31;
    int all = weight(mine), bef = lane < b ? all : 0;
    for (int i = 32 + lane; i < a.B; i += 32) {
        const int g = weight(groups_of(a, i));
        all += g;
        bef += i < b ? g : 0;
    }
    *before = __reduce_add_sync(0xffffffffu, bef);
    return __reduce_add_sync(0xffffffffu, all);
}
__device__ __forceinline__ Shares shares_of(const AttnArgs &a, int mine) {
    int none;
    const long long t = (long long)sum_of(a, mine, 0, &none, [](int g) { return g; }) * a.Hkv;
    return Shares{t, (int)(t < a.slots ? t : a.slots)};
}
// the sequence that unit u of all heads' weights belongs to (a.B: none), its groups, and u's number within it; whole warp
template <typename F> __device__ __forceinline__ int find_unit(const AttnArgs &a, int mine, long long u, int *groups, long long *rest, F weight) {
    const int lane = threadIdx.x & 31;
    long long base = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int g = b0 ? groups_of(a, b0 + lane) : mine, v = weight(g);
        int x = v;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, off);
            if (lane >= off) x += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, base + (long long)x * a.Hkv > u);
        if (past) {
            const int l = __ffs(past) - 1;
            *rest = u - base - (long long)__shfl_sync(0xffffffffu, x - v, l) * a.Hkv;
            *groups = __shfl_sync(0xffffffffu, g, l);
            return b0 + l;
        }
        base += (long long)__shfl_sync(0xffffffffu, x, 31) * a.Hkv;
    }
    return a.B;
}

// grid: slots * rt, row tiles of one share next to each other (they read the same codes)
template <int D, int MT>
__global__ void __launch_bounds__(NT, Smem<D, MT>::CTAS)
kv8_attention_kernel(const AttnArgs a) {
    using S = Smem<D, MT>;
    constexpr int KS = D / 16, NO = D / 8, ST = S::STAGES;
    extern __shared__ __align__(128) uint8_t sm[];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gr = lane >> 2, qc = lane & 3;
    const int slot = blockIdx.x / a.rt, row0 = (blockIdx.x - slot * a.rt) * 16 * MT;
    const int mine = groups_of(a, lane);
    const Shares shares = shares_of(a, mine);
    long long rest, todo;
    int b, gb, h, group, tail = 1;                 // tail: which piece of the workspace a pair's beginning goes to
    if (a.by_pair) {
        b = find_unit(a, mine, slot, &gb, &rest, [&](int g) { return pieces_of(a, shares, g); });
        if (b >= a.B) return;
        const int k = pieces_of(a, shares, gb), i = (int)rest % k;
        h = (int)rest / k;
        group = (int)div_of((long long)gb * i, k);
        todo = div_of((long long)gb * (i + 1), k) - group;
        tail = 0;
    } else {
        if (slot >= shares.n) return;
        const long long begin = share_begin(shares, slot);
        todo = share_begin(shares, slot + 1) - begin;
        b = find_unit(a, mine, begin, &gb, &rest, [](int g) { return g; });
        h = (int)div_of(rest, gb); group = (int)(rest - (long long)h * gb);
    }
    const bool starts_inside = group > 0;          // the first piece's pair began in an earlier share

    uint64_t *bars = reinterpret_cast<uint64_t *>(sm + S::bar) + warp * ST;
    volatile int *abort_flag = reinterpret_cast<int *>(sm + S::abort_flag);
    if (tid == 0) *abort_flag = 0;
    if (lane < ST) mbar_init(bars + lane, 1);
    mbar_fence_init();
    __syncthreads();
    uint8_t *ring = sm + S::ring + warp * (ST * 2 * S::TILE);
    uint4 *qs = reinterpret_cast<uint4 *>(sm + S::q);
    int st = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (bool is_first = true; todo > 0 && ok; is_first = false) {
    const int bh = b * a.Hkv + h, take = (int)(todo < gb - group ? todo : gb - group);
    const Place p = place(a, bh);
    const int t_end = min((group + take) * NW, (p.n + BLK - 1) / BLK), last = min(p.n, (group + take) * NW * BLK);
    const bool whole = take == gb;
    const int64_t part = ((int64_t)slot * 2 + (is_first && starts_inside ? 0 : tail)) * a.R;
    const uint8_t *kg = a.c.k + (int64_t)bh * a.c.cap * D, *vg = a.c.v + (int64_t)bh * a.c.cap * D;
    const float *ksg = a.c.ks + (int64_t)bh * (a.c.cap / BLK), *vsg = a.c.vs + (int64_t)bh * (a.c.cap / BLK);
    int t = group * NW + warp;
    auto fetch = [&](int tile, int st) {           // lane 0
        mbar_expect_tx(bars + st, 2 * S::TILE);
        bulk_load(ring + st * 2 * S::TILE, kg + (int64_t)tile * S::TILE, S::TILE, bars + st);
        bulk_load(ring + st * 2 * S::TILE + S::TILE, vg + (int64_t)tile * S::TILE, S::TILE, bars + st);
    };
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < ST; ++i) if (t + i * NW < t_end) fetch(t + i * NW, (st + i) % ST);
    }
    float ks_next = t < t_end ? ksg[t] : 0.f, vs_next = t < t_end ? vsg[t] : 0.f;
    // Q fragments: warp w brings the K steps of all rows of row tile w to shared memory; the score factors stay in registers
    float fr[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const QRow rows[2] = {q_row(a, p, row0 + 16 * mt + gr, D), q_row(a, p, row0 + 16 * mt + 8 + gr, D)};
        uint32_t qf[KS][4];
        load_q<D>(rows, qc, qf, fr[mt]);
        fr[mt][0] *= a.scale_log2; fr[mt][1] *= a.scale_log2;
        if (warp == mt) {
#pragma unroll
            for (int k = 0; k < KS; ++k) qs[(mt * KS + k) * 32 + lane] = make_uint4(qf[k][0], qf[k][1], qf[k][2], qf[k][3]);
        }
    }
    __syncthreads();
    float o[MT][NO][4];
    float nref[MT][2], l[MT][2];
    int lr[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        nref[mt][0] = nref[mt][1] = NO_REF; l[mt][0] = l[mt][1] = 0.f; lr[mt][0] = lr[mt][1] = 0;
#pragma unroll
        for (int n = 0; n < NO; ++n) o[mt][n][0] = o[mt][n][1] = o[mt][n][2] = o[mt][n][3] = 0.f;
    }
    auto k_step = [&](int k, const uint32_t (&w)[4][KS], float (&s)[MT][4][4]) {      // scores: 16 channels of a tile's products
        uint32_t qf[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const uint4 v = qs[(mt * KS + k) * 32 + lane];
            qf[mt][0] = v.x; qf[mt][1] = v.y; qf[mt][2] = v.z; qf[mt][3] = v.w;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t b0, b1;
            four_codes(w[j][k], b0, b1);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if (k == 0) mma_f16_16816_first(s[mt][j], qf[mt], b0, b1);
                else mma_f16_16816(s[mt][j], qf[mt], b0, b1);
            }
        }
    };
    // A tile's scores are formed while the terms of the one before it are: one warp issues a product every 16 clocks at most, and the exponentials fill what is between. (16 heads of
    // 64 channels, 32 queries, 4 x 65536 rows: 112.6 us with 8 warps per SM; in a row 113.3 with 12 warps, which then have the registers, and 135 with 8.)
    float s[MT][4][4], sn[MT][4][4];
    float ks = ks_next, vs = vs_next;
    if (t < t_end) {
        if (!mbar_wait_warp(bars + st, phase, abort_flag, a.status)) ok = false;
        else {
            const uint8_t *kt = ring + st * 2 * S::TILE;
            uint32_t w[4][KS];
#pragma unroll
            for (int j = 0; j < 4; ++j) load_k<D>(kt, gr, qc, j, w[j]);
#pragma unroll
            for (int k = 0; k < KS; ++k) k_step(k, w, s);
        }
    }
    for (; ok && t < t_end; t += NW) {
        const int sx = st + 1 == ST ? 0 : st + 1;
        const uint32_t px = st + 1 == ST ? phase ^ 1 : phase;
        const uint8_t *vt = ring + st * 2 * S::TILE + S::TILE, *kt = ring + sx * 2 * S::TILE;
        const int left = last - t * BLK;           // rows of this tile that are there
        if (left < BLK) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (8 * qc + 2 * j + e >= left) {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) s[mt][j][e] = s[mt][j][2 + e] = -INFINITY;
                    }
        }
        // the reference moves only when a term would leave f16
        const int ei = exponent_of(vs);
        const float ev = (float)ei;
        float mx[MT][2], f[MT][2];
        auto far_from = [&]() {                    // some row's sum is made of scales far above this tile's
            int top = max(lr[0][0], lr[0][1]);
            if (MT > 1) top = max(top, max(lr[MT - 1][0], lr[MT - 1][1]));
            return top - ei > L_SPAN;
        };
        bool grown = far_from(), apart = false;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                f[mt][r] = fmaxf(fr[mt][r] * ks, 1.18e-38f);                      // (not 0: a masked score times it has to stay -infinity)
                const float x0 = fmaxf(fmaxf(s[mt][0][2 * r], s[mt][0][2 * r + 1]), s[mt][1][2 * r]);
                const float x1 = fmaxf(fmaxf(s[mt][1][2 * r + 1], s[mt][2][2 * r]), s[mt][2][2 * r + 1]);
                mx[mt][r] = fmaxf(fmaxf(fmaxf(x0, x1), s[mt][3][2 * r]), s[mt][3][2 * r + 1]);
                grown |= fmaf(mx[mt][r], f[mt][r], nref[mt][r]) > P_LIMIT - ev;
            }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float m = mx[mt][r];
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2)) * f[mt][r];
                    // (m = -infinity, scores beyond fp32: nothing moves.  The first time the old references are NO_REF, and both are new.)
                    const float was = nref[mt][r], sum_was = was + (float)lr[mt][r], to = fminf(was, P_START - ev - m), sum_to = m + sum_was > P_LIMIT + L_SPAN ? P_START - m : sum_was;
                    const int lto = __float2int_rn(sum_to - to);
                    const float move = to - was, alpha = ex2f(move);
                    nref[mt][r] = to;
                    l[mt][r] *= ex2f(move + (float)(lto - lr[mt][r]));
                    lr[mt][r] = lto;
#pragma unroll
                    for (int n = 0; n < NO; ++n) { o[mt][n][2 * r] *= alpha; o[mt][n][2 * r + 1] *= alpha; }
                }
            apart = __any_sync(0xffffffffu, far_from());
            if (apart) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) l[mt][r] += ex2f(fmaf(s[mt][j][2 * r + e], f[mt][r], nref[mt][r] + (float)lr[mt][r]));
            }
        }
        if (left < BLK) {                          // codes behind the last row may be anything, NaN included: zeros in their place
            for (int c = lane; c < D; c += 32)
                for (int r = left; r < BLK; ++r) const_cast<uint8_t *>(vt)[c * BLK + r] = 0;
            __syncwarp();
        }
        if (t + NW < t_end) {
            ks_next = ksg[t + NW]; vs_next = vsg[t + NW];
            if (!mbar_wait_warp(bars + sx, px, abort_flag, a.status)) { ok = false; break; }
        }
        uint32_t pf[MT][2][4], w[4][KS];
#pragma unroll
        for (int j = 0; j < 4; ++j) load_k<D>(kt, gr, qc, j, w[j]);
        auto term = [&](int mt, int r) {           // p' of this thread's eight columns of a row
            const f32x2 f2 = pk2(f[mt][r], f[mt][r]), n2 = pk2(nref[mt][r] + ev, nref[mt][r] + ev);
            f32x2 sum;
            float x[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                upk2(fma2(pk2(s[mt][j][2 * r], s[mt][j][2 * r + 1]), f2, n2), x[2 * j], x[2 * j + 1]);
                x[2 * j] = ex2f(x[2 * j]); x[2 * j + 1] = ex2f(x[2 * j + 1]);
                sum = j ? add2(sum, pk2(x[2 * j], x[2 * j + 1])) : pk2(x[0], x[1]);
            }
            float s0, s1;
            upk2(sum, s0, s1);
            const float lf = apart ? 0.f : __int_as_float(max(lr[mt][r] - ei + 127, 0) << 23);
            l[mt][r] = fmaf(s0 + s1, lf, l[mt][r]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {          // rows 8 qc + 4 i + (0, 1) and + (2, 3)
                pf[mt][i][r] = pack_f16(x[4 * i], x[4 * i + 1]);
                pf[mt][i][2 + r] = pack_f16(x[4 * i + 2], x[4 * i + 3]);
            }
        };
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            k_step(k, w, sn);
            if (k < 2 * MT) term(k >> 1, k & 1);
        }
        // two column tiles at a time: an accumulator's second product comes after those of the others, not into its own latency
#pragma unroll
        for (int n0 = 0; n0 < NO; n0 += 2) {
            uint32_t bv[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const uint2 w = *reinterpret_cast<const uint2 *>(vt + (8 * (n0 + n) + gr) * BLK + 8 * qc);
                four_codes(w.x, bv[n][0], bv[n][1]);
                four_codes(w.y, bv[n][2], bv[n][3]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) mma_f16_16816(o[mt][n0 + n], pf[mt][i], bv[n][2 * i], bv[n][2 * i + 1]);
        }
        __syncwarp();                              // every lane is done with the stage
        if (lane == 0 && t + ST * NW < t_end) fetch(t + ST * NW, st);
        st = sx; phase = px;
        ks = ks_next; vs = vs_next;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[mt][j][e] = sn[mt][j][e];
    }
    if (!ok) {                                     // a copy did not arrive: wait for those in flight, quietly, and leave
        if (lane == 0)
            for (int i = 0; i < ST; ++i) mbar_wait_quiet(bars + i, i >= st ? phase : phase ^ 1, 1000000ull);
        __syncwarp();
    }
    ok = !__syncthreads_or(!ok);                   // the ring is free: its bytes take the warps' results
    float *ow = reinterpret_cast<float *>(sm + S::ow), *mw = reinterpret_cast<float *>(sm + S::mw), *lw = reinterpret_cast<float *>(sm + S::lw);
    constexpr int M = 16 * MT;
    // From here on output and sum share one reference: nref + lr is the sum's, and each goes half of the way, so that neither leaves fp32 however large or small V is (|lr| < 160)
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = 16 * mt + 8 * r + gr;
            float ls = l[mt][r];
            ls += __shfl_xor_sync(0xffffffffu, ls, 1);
            ls += __shfl_xor_sync(0xffffffffu, ls, 2);
            const int h = lr[mt][r] >> 1;
            const float of = pow2_of(lr[mt][r] - h);
            if (qc == 0) { mw[warp * M + row] = nref[mt][r] + (float)(lr[mt][r] - h); lw[warp * M + row] = ls * pow2_of(-h); }
#pragma unroll
            for (int n = 0; n < NO; ++n)
                *reinterpret_cast<float2 *>(ow + (warp * M + row) * D + 8 * n + 2 * qc) = make_float2(o[mt][n][2 * r] * of, o[mt][n][2 * r + 1] * of);
        }
    __syncthreads();
    for (int e = tid; e < M * D / 4; e += NT) {
        const int row = e / (D / 4), c = (e - row * (D / 4)) * 4, grow = row0 + row, hl = grow / a.G, tok = grow - hl * a.G;
        if (grow >= a.R || tok >= p.live) continue;
        float ref = mw[row];                       // the smallest nref belongs to the largest maximum
#pragma unroll
        for (int w = 1; w < NW; ++w) ref = fminf(ref, mw[w * M + row]);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        float ls = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = ex2f(ref - mw[w * M + row]);
            const float4 v = *reinterpret_cast<const float4 *>(ow + (w * M + row) * D + c);
            x.x = fmaf(f, v.x, x.x); x.y = fmaf(f, v.y, x.y); x.z = fmaf(f, v.z, x.z); x.w = fmaf(f, v.w, x.w);
            ls = fmaf(f, lw[w * M + row], ls);
        }
        if (whole) {
            const float inv = ls == 0.f ? 0.f : 1.f / ls;          // no row to attend to: zeros
            *reinterpret_cast<uint2 *>(a.out + ((int64_t)p.b * a.G + tok) * a.ld_out + (int64_t)(p.h * a.group + hl) * D + c) =
                make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
            if (c == 0 && a.stat) a.stat[(int64_t)bh * a.R + grow] = make_float2(ref, inv);
        } else {
            *reinterpret_cast<float4 *>(a.po + (part + grow) * D + c) = x;
            if (c == 0) a.pml[part + grow] = make_float2(ref, ls);
        }
    }
    todo -= take;
    group = 0;
    if (todo > 0) {
        if (++h == a.Hkv) {
            h = 0;
            do { gb = groups_of(a, ++b); } while (gb == 0 && b + 1 < a.B);
        }
        fence_proxy_async();                       // what was written to the ring comes before the next copies into it
        __syncthreads();
    }
    }
}

// Joins the pieces of a row: D / 4 threads hold its channels, `groups` of them share the pieces, each with a running reference
constexpr int JT = 128;                            // (256: 24 heads, 32 queries, 8192 rows 19.7 -> 21.8 us; each CTA finds its pieces first, and more of them hide that)
template <int D>
__global__ void __launch_bounds__(JT)
kv8_join_kernel(const AttnArgs a, int groups) {
    constexpr int Q = D / 4, U = 4;
    __shared__ float4 xs[JT];
    __shared__ float2 ms[JT];
    const int bh = blockIdx.x / a.join_tiles, tile = blockIdx.x - bh * a.join_tiles;
    const Place p = place(a, bh);
    const int mine = groups_of(a, threadIdx.x & 31);
    const Shares shares = shares_of(a, mine);
    if (p.live == 0) { pdl_wait(); return; }
    const int gb = groups_of(a, p.b);
    int before, s0, np;
    if (a.by_pair) {
        sum_of(a, mine, p.b, &before, [&](int g) { return pieces_of(a, shares, g); });
        np = pieces_of(a, shares, gb);
        s0 = before * a.Hkv + p.h * np;
    } else {
        sum_of(a, mine, p.b, &before, [](int g) { return g; });
        const long long g0 = (long long)before * a.Hkv + (long long)p.h * gb;
        s0 = share_of(shares, g0); np = share_of(shares, g0 + gb - 1) - s0 + 1;
    }
    pdl_wait();                                    // (what comes before reads only what the caller had ready before the first launch)
    pdl_trigger();
    if (np <= 1) return;
    // cut across pairs, a pair's first piece lies behind others in its share, or begins it: place 1; the other shares begin inside the pair: place 0
    const int rows = JT / (Q * groups), q = threadIdx.x % Q, rr = threadIdx.x / Q % rows, g = threadIdx.x / (Q * rows);
    for (int row0 = tile * rows; row0 < a.R; row0 += a.join_tiles * rows) {
    const int row = row0 + rr, hl = row / a.G, t = row - hl * a.G;
    const bool valid = g < groups && row < a.R && t < p.live;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    float ref = NO_REF, l = 0.f;
    if (valid) {
        const int64_t base = (int64_t)s0 * 2 * a.R + row;
        for (int i = g; i < np; i += U * groups) {
            float2 m[U];
            float4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = i + u * groups;
                const int64_t at = base + (int64_t)(k == 0 ? !a.by_pair : 2 * k) * a.R;
                m[u] = k < np ? a.pml[at] : make_float2(NO_REF, 0.f);
                v[u] = k < np ? *reinterpret_cast<const float4 *>(a.po + at * D + 4 * q) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            const float to = fminf(ref, fminf(fminf(m[0].x, m[1].x), fminf(m[2].x, m[3].x)));
            const float al = ex2f(to - ref);
            ref = to;
            l *= al; x.x *= al; x.y *= al; x.z *= al; x.w *= al;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float f = ex2f(to - m[u].x);
                l = fmaf(f, m[u].y, l);
                x.x = fmaf(f, v[u].x, x.x); x.y = fmaf(f, v[u].y, x.y); x.z = fmaf(f, v[u].z, x.z); x.w = fmaf(f, v[u].w, x.w);
            }
        }
    }
    if (groups > 1) {
        xs[threadIdx.x] = x;
        ms[threadIdx.x] = make_float2(ref, l);
        __syncthreads();
        if (g == 0) {
            float to = ref;
            for (int k = 1; k < groups; ++k) to = fminf(to, ms[threadIdx.x + k * Q * rows].x);
            const float al = ex2f(to - ref);
            l *= al; x.x *= al; x.y *= al; x.z *= al; x.w *= al;
            for (int k = 1; k < groups; ++k) {
                const float2 m = ms[threadIdx.x + k * Q * rows];
                const float4 v = xs[threadIdx.x + k * Q * rows];
                const float f = ex2f(to - m.x);
                l = fmaf(f, m.y, l);
                x.x = fmaf(f, v.x, x.x); x.y = fmaf(f, v.y, x.y); x.z = fmaf(f, v.z, x.z); x.w = fmaf(f, v.w, x.w);
            }
            ref = to;
        }
        __syncthreads();                           // (before the next rows' parts)
    }
    if (!valid || g) continue;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2 *>(a.out + ((int64_t)p.b * a.G + t) * a.ld_out + (int64_t)(p.h * a.group + hl) * D + 4 * q) =
        make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
    if (q == 0 && a.stat) a.stat[(int64_t)bh * a.R + row] = make_float2(ref, inv);
    }
}

// What each row receives: acc_out_j = (j < len ? acc_in_j : 0) + sum over the rows r of the kv head of 2^(s_rj - m_r) / l_r.  The scores are formed a second time from K alone (half of the
// cache): the weights need every row's final maximum and sum, and holding the scores would cost R times 4 bytes per row where K is D bytes.
// A warp per tile of 32 rows, the block's rows of Q from shared memory 16 at a time; sums run in a fixed order.
// 16 sequences of up to 8192 rows, 24 heads of 80, 32 queries: 48 us, of which reading K is 28; the tensor pipe is 43 % active, exponentials 35 %, instruction issue 45 %.  12 warps per SM are as
// fast as 16.  (Scores of the next 16 queries beside the terms of these, as in the attention kernel: 30 us more; K through rings of bulk copies: 6 more.)
// grid: (B * Hkv, pieces of the tiles)
struct WeightArgs {
    const float *in;
    float *out;                                    // [B, Hkv, cap]
    int row0, rows;                                // rows of the kv head taken by this launch (multiple of 16 from row0)
    int tiles;                                     // tiles per CTA
};
constexpr int WROWS = 128;                         // rows of Q that fit in shared memory beside several CTAs

template <int D>
__global__ void __launch_bounds__(NT)
kv8_weights_kernel(const AttnArgs a, const WeightArgs wa) {
    constexpr int KS = D / 16;
    extern __shared__ __align__(16) uint4 qs[];    // [mt][KS][32 lanes], then float4 [mt][8]: (f0, f1) ... per row: score factor, maximum, 1 / sum
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gr = lane >> 2, qc = lane & 3;
    const int bh = blockIdx.x;
    const Place p = place(a, bh);
    const int t0 = blockIdx.y * wa.tiles, t_end = min((p.n + BLK - 1) / BLK, t0 + wa.tiles);
    if (t0 >= t_end) { pdl_wait(); return; }
    const int nm = (wa.rows + 15) / 16;
    float4 *rs = reinterpret_cast<float4 *>(qs + nm * KS * 32);
    for (int mt = warp; mt < nm; mt += NW) {
        const int r = wa.row0 + 16 * mt + gr;
        const QRow rows[2] = {q_row(a, p, r, D), q_row(a, p, r + 8, D)};
        uint32_t qf[KS][4];
        float f[2];
        load_q<D>(rows, qc, qf, f);
#pragma unroll
        for (int k = 0; k < KS; ++k) qs[(mt * KS + k) * 32 + lane] = make_uint4(qf[k][0], qf[k][1], qf[k][2], qf[k][3]);
        if (qc == 0) {
            rs[mt * 16 + gr] = make_float4(f[0] * a.scale_log2, 0.f, 0.f, 0.f);
            rs[mt * 16 + 8 + gr] = make_float4(f[1] * a.scale_log2, 0.f, 0.f, 0.f);
        }
    }
    const uint8_t *kg = a.c.k + (int64_t)bh * a.c.cap * D;
    const float *ksg = a.c.ks + (int64_t)bh * (a.c.cap / BLK);
    uint32_t w[4][KS];
    float ks = 0.f;
    auto fetch = [&](int t) {
#pragma unroll
        for (int j = 0; j < 4; ++j) load_k<D>(kg + (int64_t)t * BLK * D, gr, qc, j, w[j]);
        ks = ksg[t];
    };
    int t = t0 + warp;
    if (t < t_end) fetch(t);
    pdl_wait();                                    // (up to here only what was there before the attention launch began)
    pdl_trigger();
    __syncthreads();
    for (int i = tid; i < 16 * nm; i += NT) {
        const int r = wa.row0 + i, hl = r / a.G;
        if (r < a.R && r - hl * a.G < p.live) {
            const float2 st = a.stat[(int64_t)bh * a.R + r];
            rs[i].y = st.x; rs[i].z = st.y;
        }
    }
    __syncthreads();
    for (; t < t_end; t += NW) {
        uint32_t b[4][KS][2];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < KS; ++k) four_codes(w[j][k], b[j][k][0], b[j][k][1]);
        const float kt = ks;
        if (t + NW < t_end) fetch(t + NW);         // the next tile's codes while this one is multiplied
        // a lane writes one row of the 32; what it adds to is asked for early
        const int row = t * BLK + lane;
        const int64_t at = (int64_t)bh * a.c.cap + row;
        const float was = row < p.n && (row < p.len || wa.row0 > 0) ? wa.in[at] : 0.f;
        f32x2 sum[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll 1
        for (int mt = 0; mt < nm; ++mt) {
            float s[4][4];
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const uint4 q4 = qs[(mt * KS + k) * 32 + lane];
                const uint32_t qf[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (k == 0) mma_f16_16816_first(s[j], qf, b[j][k][0], b[j][k][1]);
                    else mma_f16_16816(s[j], qf, b[j][k][0], b[j][k][1]);
                }
            }
            const float4 r0 = rs[mt * 16 + gr], r1 = rs[mt * 16 + 8 + gr];
            const f32x2 f0 = pk2(r0.x * kt, r0.x * kt), f1 = pk2(r1.x * kt, r1.x * kt), n0 = pk2(r0.y, r0.y), n1 = pk2(r1.y, r1.y), i0 = pk2(r0.z, r0.z), i1 = pk2(r1.z, r1.z);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x0, x1, y0, y1;
                upk2(fma2(pk2(s[j][0], s[j][1]), f0, n0), x0, x1);
                upk2(fma2(pk2(s[j][2], s[j][3]), f1, n1), y0, y1);
                sum[j] = fma2(pk2(ex2f(x0), ex2f(x1)), i0, sum[j]);
                sum[j] = fma2(pk2(ex2f(y0), ex2f(y1)), i1, sum[j]);
            }
        }
        // over the eight lanes of a column: each step halves the columns a lane keeps, the last leaves one row of the tile per lane
        float c[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) upk2(sum[j], c[2 * j], c[2 * j + 1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool hi = gr & 4;
            const float give = hi ? c[i] : c[i + 4], keep = hi ? c[i + 4] : c[i];
            c[i] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool hi = gr & 2;
            const float give = hi ? c[i] : c[i + 2], keep = hi ? c[i + 2] : c[i];
            c[i] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
        }
        const bool hi = gr & 1;
        const float mine = (hi ? c[1] : c[0]) + __shfl_xor_sync(0xffffffffu, hi ? c[0] : c[1], 4);
        // lane (gr, qc) holds row 8 qc + gr of the tile; lane i writes row i
        const float v = __shfl_sync(0xffffffffu, mine, (lane & 7) * 4 + (lane >> 3));
        if (row < p.n) wa.out[at] = p.live ? was + v : was;        // (without queries zeros were multiplied, and zero times a NaN code is not zero)
    }
}

template <int D, int MT>
cudaError_t launch_attention(const AttnArgs &a, int shares, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(kv8_attention_kernel<D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Smem<D, MT>::total);
    if (e != cudaSuccess) return e;
    const int64_t ctas = (int64_t)shares * a.rt;
    if (ctas > 0x7fffffff) return cudaErrorNotSupported;
    e = launch_chain(kv8_attention_kernel<D, MT>, dim3((unsigned)ctas), NT, Smem<D, MT>::total, s, 0, a);
    if (e != cudaSuccess || shares <= 1) return e;
    // pieces that a pair can have: all of them share the slots.  Many are shared out over several threads per channel (one head of 64, 8192 rows, in 37 pieces: 11 us, one thread 14; where
    // there are 6, all threads of a CTA on one row instead of half of them: 113 -> 116)
    const int64_t pieces = a.slots / ((int64_t)a.B * a.Hkv) + 2;
    const int groups = pieces <= 4 ? 1 : JT / (D / 4) / (pieces <= 8 ? 2 : 1), per = JT / (D / 4 * groups);
    AttnArgs j = a;
    // no more CTAs than run at a time (each finds its pieces first): 16 x 24 heads, 32 queries, with weights 161.8 -> 159.5 us
    const int64_t tiles = (a.R + per - 1) / per, most = 8 * (int64_t)sm_count() / ((int64_t)a.B * a.Hkv);
    j.join_tiles = (int)(tiles < most ? tiles : most < 1 ? 1 : most);
    return launch_chain(kv8_join_kernel<D>, dim3((unsigned)(a.B * a.Hkv * j.join_tiles)), JT, 0, s, 0, j, groups);
}

template <int D>
cudaError_t launch_weights(const AttnArgs &a, const float *in, float *out, cudaStream_t s) {
    const int tiles = (a.max_rows + BLK - 1) / BLK;
    for (int r0 = 0; r0 < a.R; r0 += WROWS) {
        WeightArgs wa{r0 ? out : in, out, r0, a.R - r0 < WROWS ? a.R - r0 : WROWS, 0};
        // tiles per CTA: two waves of CTAs, but no fewer than four tiles per warp: bringing the queries to shared memory costs a CTA 2 us or so (16 x 24 heads of 80, up to 8192 rows, with
        // the attention before it: two waves 154.0 us, one 161.9, three 157.5, ten 164.5; eight tiles per CTA 181; as many CTAs as run at a time with equal shares of all tiles 155.0)
        const int64_t share = (int64_t)a.B * a.Hkv * tiles / (2 * 4 * (int64_t)sm_count()) / NW * NW;
        wa.tiles = (int)(share < 4 * NW ? 4 * NW : share > 64 * NW ? 64 * NW : share);
        while ((tiles + wa.tiles - 1) / wa.tiles > 65535) wa.tiles *= 2;
        const int nm = (wa.rows + 15) / 16;
        const size_t smem = (size_t)nm * (D / 16) * 32 * 16 + (size_t)nm * 16 * 16;
        cudaError_t e = cudaFuncSetAttribute(kv8_weights_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        e = launch_chain(kv8_weights_kernel<D>, dim3((unsigned)(a.B * a.Hkv), (unsigned)((tiles + wa.tiles - 1) / wa.tiles)), NT, smem, s, 0, a, wa);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

struct Plan { int mt, rt, slots, by_pair, ctas; };
Plan plan(int B, int Hkv, int R, int D, int max_rows) {
    Plan p;
    const int64_t pairs = (int64_t)B * Hkv, groups = pairs * ((max_rows + NW * BLK - 1) / (NW * BLK));
    // Rows of queries that a warp takes with each tile: 16, or 32 where they fit its registers and leave no half empty, and where there is much to do: 32 halve the conversions, 16 have 12 warps
    // per SM instead of 8 and less to set up (16 heads of 64, 32 queries: 4 x 65536 rows 121.4 us with 16, 112.6 with 32; 4 x 16384 rows 41.8 and 42.9; 1 x 8192 rows 14.7 and 16.1; 24 heads of
    // 80: 4 x 8192 rows 39.0 and 43.3, 64 queries and 1 x 8192 rows 28.5 and 26.4; 4 heads of 64, 64 queries, 8 x 1024 rows 12.4 and 18.1).
    const int halves = (R + 15) / 16, room2 = 2 * sm_count();
    p.mt = D <= 80 && (halves % 2 == 0 || halves > 4) && groups * ((halves + 1) / 2) > (halves > 2 ? 8 : 24) * (int64_t)room2 ? 2 : 1;
    p.rt = (R + 16 * p.mt - 1) / (16 * p.mt);
    const int64_t room = p.mt == 1 && D < 128 ? 3 * (int64_t)sm_count() : room2, slots = room / p.rt < 1 ? 1 : room / p.rt;
    p.slots = (int)(groups < slots ? groups : slots);
    // By pair where shares are more than two groups (starting anew inside one then shows: 2 x 16 heads of 64 channels, 32 queries, 8192 rows: 20.0 us, equal shares 24.1; with shares of a
    // group or two 8 heads of 80, 32 queries, 8192 rows: 15.7, equal 15.6) and what rounding each pair to whole pieces leaves empty, up to a share in slots / pairs + 1, is less than
    // five groups' time (4 x 16 heads of 64, 32 queries: 8192 rows 27.3, equal 29.8; 32768 rows 71.2, equal 68.7).
    p.by_pair = p.slots >= 2 * pairs && groups > 2 * (int64_t)p.slots && groups / p.slots * pairs < 5 * (p.slots + pairs);
    p.ctas = p.slots + (p.by_pair ? (int)pairs : 0);      // (every pair has a piece, however few rows)
    return p;
}

}  // namespace

// Enough for any smaller max_rows too, whichever way its work is cut
size_t kv8_attention_workspace(int B, int G, int H, int Hkv, int D, int max_rows) {
    const int R = H / Hkv * G;
    const Plan p = plan(B, Hkv, R, D, max_rows);
    const size_t pairs = (size_t)B * Hkv, ctas = (size_t)p.slots + ((size_t)p.slots >= 2 * pairs ? pairs : 0);
    size_t n = align_up(pairs * R * sizeof(float2));
    if (ctas > 1) n += align_up(ctas * 2 * R * sizeof(float2)) + align_up(ctas * 2 * R * D * sizeof(float));
    return n;
}

cudaError_t kv8_attention(const kv8::Cache &c, const void *q, int64_t ld_q, const int32_t *lens, const int32_t *counts, const float *acc_in, float *acc_out, void *out,
                          int64_t ld_out, int B, int G, int H, int Hkv, int D, int max_rows, void *ws, cudaStream_t s) {
    AttnArgs a{};
    a.c = c; a.q = static_cast<const __nv_bfloat16 *>(q); a.ld_q = ld_q; a.lens = lens; a.counts = counts;
    a.out = static_cast<__nv_bfloat16 *>(out); a.ld_out = ld_out;
    a.B = B; a.G = G; a.H = H; a.Hkv = Hkv; a.group = H / Hkv; a.R = a.group * G; a.max_rows = max_rows;
    const Plan p = plan(B, Hkv, a.R, D, max_rows);
    a.slots = p.slots; a.by_pair = p.by_pair; a.rt = p.rt;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
    a.status = device_status_ptr();
    if (!a.status) return cudaErrorInitializationError;
    char *w = static_cast<char *>(ws);
    const size_t rows = (size_t)B * Hkv * a.R;
    a.stat = acc_out ? reinterpret_cast<float2 *>(w) : nullptr;
    w += align_up(rows * sizeof(float2));
    a.pml = reinterpret_cast<float2 *>(w);
    a.po = reinterpret_cast<float *>(w + align_up((size_t)p.ctas * 2 * a.R * sizeof(float2)));
    cudaError_t e;
    if (D == 64) e = p.mt == 2 ? launch_attention<64, 2>(a, p.ctas, s) : launch_attention<64, 1>(a, p.ctas, s);
    else if (D == 80) e = p.mt == 2 ? launch_attention<80, 2>(a, p.ctas, s) : launch_attention<80, 1>(a, p.ctas, s);
    else e = launch_attention<128, 1>(a, p.ctas, s);
    if (e != cudaSuccess || !acc_out) return e;
    return D == 64 ? launch_weights<64>(a, acc_in, acc_out, s) : D == 80 ? launch_weights<80>(a, acc_in, acc_out, s) : launch_weights<128>(a, acc_in, acc_out, s);
}

}  // namespace dm
