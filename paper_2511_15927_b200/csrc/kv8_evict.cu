// Rows with little accumulated attention weight leave the 8-bit cache (per sequence and kv head), the others move up, in order, into another cache.
// Two launches.
// The choice: one CTA per (sequence, head) finds the keep-th largest weight: counts of the weights' bits (as whole numbers in their order) in 4096 equal steps of the interval
// that they span, then of the step that holds it, and so on until 32 or fewer are left, which are ranked (whole numbers, so the order of additions does not matter).  It writes the kept rows'
// numbers in ascending order.  Bound by latencies and, with long sequences, by counting in shared memory (4.7 clocks per 32 weights): 27 us for 8 x 24 heads of up to 32768 rows,
// in two waves of CTAs since the weights that a CTA keeps fill the SM's registers.
// The move: one warp per block of 32 kept rows, for K and for V; it finds the new block's scale and brings the codes to it, in f16.  Bound by memory: V's
// channel-major blocks are read whole as soon as one of their rows stays; where 8000 of up to 32768 rows stay in 8 x 24 heads of 80 channels the move takes 129 us and both launches 155.
// One sequence, 16 heads of 64, 2048 of 8192 rows stay: 12 us, latencies.
// Attention without positions does not see where a row lies, so the kept rows need no numbers of their own.
#include "kv8.cuh"
#include "tc_ptx.cuh"

namespace dm {
namespace {

using namespace kv8;

struct EvictArgs {
    Cache src, dst;
    const float *acc_in;
    float *acc_out;                                // [B, Hkv, dst.cap]
    const int32_t *lens_in;
    int32_t *lens_out;
    int32_t *rows;                                 // [B * Hkv, keep] kept rows, -1 behind the last: the caller's array, or the workspace
    int B, H, max_rows, keep, recent;
};

constexpr int CT = 1024, BINS = 4 * CT;

// larger weight, larger key; NaN below everything (0), the two zeros alike
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ int rows_of(const EvictArgs &a, int b) { return min(min(max(a.lens_in[b], 0), a.src.cap), a.max_rows); }

// exclusive prefix sum over the CTA; *total: the sum.  Both halves of a 64-bit word (two counters) at once, or one 32-bit counter.
template <typename U> __device__ __forceinline__ U cta_prefix(U v, U *part, U *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    U x = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const U y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();
    if (lane == 31) part[warp] = x;
    __syncthreads();
    U s = part[lane];                              // (every warp adds up the warps' sums for itself)
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const U y = __shfl_up_sync(0xffffffffu, s, off);
        if (lane >= off) s += y;
    }
    *total = __shfl_sync(0xffffffffu, s, 31);
    const U before = __shfl_sync(0xffffffffu, s, warp ? warp - 1 : 0);
    return x - v + (warp ? before : U(0));
}

// grid: B * Hkv.  HELD = 32: a thread keeps the keys of its up to 32 rows in registers; HELD = 0, beyond 32768 rows: the weights are read again in every pass (8 x 24 heads of up to 32768
// rows: 19 us more).
template <int HELD>
__global__ void __launch_bounds__(CT)
kv8_choose_kernel(const EvictArgs a) {
    __shared__ __align__(16) uint32_t hist[BINS];
    __shared__ unsigned long long part[CT / 32];
    __shared__ uint32_t part32[CT / 32], low[CT / 32], found[3], few[32], fews;
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bh = blockIdx.x, b = bh / a.H;
    const int n = rows_of(a, b), kept = min(n, a.keep);
    const float *acc = a.acc_in + (int64_t)bh * a.src.cap;
    int32_t *rows = a.rows + (int64_t)bh * a.keep;
    if (bh == b * a.H && tid == 0) a.lens_out[b] = kept;
    for (int i = kept + tid; i < a.keep; i += CT) rows[i] = -1;
    if (n <= a.keep) {
        for (int i = tid; i < n; i += CT) rows[i] = i;
        return;
    }
    // Recent rows have a key above all others, rows behind the last one the lowest: they come last among equals, so neither needs a question of its own below.
    constexpr uint32_t RECENT = 0xffffffffu;
    const int old = n - a.recent;
    auto key_at = [&](int i) { return i >= n ? 0u : i >= old ? RECENT : key_of(acc[i]); };
    const int per = (n + CT - 1) / CT, first = warp * 32 * per + lane;           // HELD: a warp has 32 per consecutive rows, a lane every 32nd of them
    uint32_t key[HELD ? HELD : 1], mn = RECENT, mx = 0;
    if (HELD) {
        float x[HELD ? HELD : 1];
#pragma unroll
        for (int q = 0; q < HELD; ++q) x[HELD ? q : 0] = q < per && first + 32 * q < old ? __ldg(acc + first + 32 * q) : 0.f;
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            const int i = first + 32 * q;
            if (q < per) {
                const uint32_t k = key_of(x[HELD ? q : 0]);
                key[HELD ? q : 0] = i < old ? k : i < n ? RECENT : 0u;
                if (i < old) { mn = min(mn, k); mx = max(mx, k); }
            }
        }
    } else {
        for (int i = tid; i < old; i += CT) {
            const uint32_t k = key_of(acc[i]);
            mn = min(mn, k); mx = max(mx, k);
        }
    }
    mn = __reduce_min_sync(0xffffffffu, mn); mx = __reduce_max_sync(0xffffffffu, mx);
    if (lane == 0) { low[warp] = mn; part32[warp] = mx; }
    __syncthreads();
    // The left-th largest key of the old rows lies in [lo, lo + span].  Each pass counts what lies there in 4096 equal steps.  The first interval is what the keys really span: the leading
    // bits of all of them taken as steps would put weights of one magnitude into a handful of counters, and counting into one address is one lane at a time.
    uint32_t lo = __reduce_min_sync(0xffffffffu, low[lane]), span = __reduce_max_sync(0xffffffffu, part32[lane]) - lo;
    int left = a.keep - a.recent;
    // The keys in the interval.  Held ones are first marked, without a branch for each: after the first pass they are few.
    auto each = [&](bool many, auto f) {
        if (!HELD) {
            for (int i = tid; i < old; i += CT) {
                const uint32_t k = key_of(acc[i]);
                if (k - lo <= span) f(k);
            }
        } else if (many) {
#pragma unroll
            for (int q = 0; q < HELD; ++q) {
                if (q >= per) break;
                if (key[HELD ? q : 0] - lo <= span) f(key[HELD ? q : 0]);
            }
        } else {
            uint32_t in = 0;
#pragma unroll
            for (int q = 0; q < HELD; ++q) {
                if (q >= per) break;
                in |= key[HELD ? q : 0] - lo <= span ? 1u << q : 0u;
            }
            for (; in; in &= in - 1) {
                const int i = first + 32 * (__ffs(in) - 1);
                if (i < old) f(key_of(acc[i]));    // (from L2 again: registers have no index)
            }
        }
    };
    if (left == 0) { lo = RECENT - 1; span = 0; }  // none but the recent rows are above that, and no row is equal to it
    if (tid == 0) fews = 0;
    for (bool first_pass = true; span > 0; first_pass = false) {
        const int bits = 32 - __clz(span), shift = max(bits - 12, 0);
        reinterpret_cast<uint4 *>(hist)[tid] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        each(first_pass, [&](uint32_t k) { atomicAdd(&hist[(k - lo) >> shift], 1u); });
        __syncthreads();
        // steps from the top: thread i owns the four from 4095 - 4 i down
        const uint4 h = reinterpret_cast<const uint4 *>(hist)[CT - 1 - tid];
        const uint32_t c[4] = {h.w, h.z, h.y, h.x};
        uint32_t total, before = cta_prefix(c[0] + c[1] + c[2] + c[3], part32, &total);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (before < (uint32_t)left && before + c[k] >= (uint32_t)left) {
                found[0] = BINS - 1 - (4 * tid + k); found[1] = left - before; found[2] = c[k];
            }
            before += c[k];
        }
        __syncthreads();
        lo += found[0] << shift;
        span = (1u << shift) - 1;
        left = (int)found[1];                      // how many of the keys of that step are still to be taken
        const int in_step = (int)found[2];         // (the counters themselves are cleared by whoever is first in the next pass)
        if (span > 0 && in_step <= 32) {           // few: every warp ranks them for itself
            each(false, [&](uint32_t k) { few[atomicAdd(&fews, 1u) & 31] = k; });
            __syncthreads();
            const int m = min((int)fews, 32);      // (rows behind the last one may have been counted with NaN, the lowest key; the left-th largest is a real one all the same)
            const uint32_t mine = few[lane];
            int larger = 0, alike = 0;
#pragma unroll 4
            for (int i = 0; i < m; ++i) {
                const uint32_t k = few[i];
                larger += k > mine; alike += k == mine;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, lane < m && larger < left && larger + alike >= left);
            lo = __shfl_sync(0xffffffffu, mine, __ffs(hit) - 1);
            left -= __shfl_sync(0xffffffffu, larger, __ffs(hit) - 1);
            break;
        }
    }
    const uint32_t prefix = lo;
    // kept: key above the threshold, or equal to it and among the first `left` such rows: keep of them.  (The bound on the place holds whatever becomes of the weights meanwhile: ones that somebody
    // changes between two passes give wrong rows, not a wrong access.)
    if (HELD) {
        uint32_t g = 0, e = 0;                     // bit q: row first + 32 q is above, is equal
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            if (q >= per) break;
            g |= (key[HELD ? q : 0] > prefix ? 1u : 0u) << q;
            e |= (key[HELD ? q : 0] == prefix ? 1u : 0u) << q;
        }
        uint32_t total;                            // two counts of at most 32768 in a word
        const unsigned lower = (1u << lane) - 1;
        const uint32_t before = __shfl_sync(0xffffffffu, cta_prefix((uint32_t)__popc(g) << 16 | __popc(e), part32, &total), 0);
        if ((total & 0xffffu) > (uint32_t)left) {  // ties that do not all stay: in the rows' order
            uint32_t eq = before & 0xffffu;
            for (int q = 0; q < per; ++q) {
                const unsigned eb = __ballot_sync(0xffffffffu, (e >> q) & 1);
                if (eq + __popc(eb & lower) >= (uint32_t)left) e &= ~(1u << q);
                eq += __popc(eb);
            }
        }
        g |= e;
        uint32_t at = (before >> 16) + min(before & 0xffffu, (uint32_t)left);
#pragma unroll 8
        for (int q = 0; q < per; ++q) {
            const bool stays = (g >> q) & 1;
            const unsigned gb = __ballot_sync(0xffffffffu, stays);
            const uint32_t to = at + __popc(gb & lower);
            if (stays && to < (uint32_t)a.keep) rows[to] = first + 32 * q;
            at += __popc(gb);
        }
        return;
    }
    uint32_t above = 0, equal = 0;                 // rows so far
    for (int base = 0; base < n; base += CT * 4) {
        const int i0 = base + tid * 4;
        uint32_t g = 0, e = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t k = key_at(i0 + q);
            g |= (k > prefix ? 1u : 0u) << q;
            e |= (k == prefix ? 1u : 0u) << q;
        }
        unsigned long long total;
        const unsigned long long before = cta_prefix((unsigned long long)__popc(g) << 32 | __popc(e), part, &total);
        uint32_t na = above + (uint32_t)(before >> 32), ne = equal + (uint32_t)before;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool ge = (g >> q) & 1, eq = (e >> q) & 1;
            const uint32_t to = na + min(ne, (uint32_t)left);
            if ((ge || (eq && ne < (uint32_t)left)) && to < (uint32_t)a.keep) rows[to] = i0 + q;
            na += ge; ne += eq;
        }
        above += (uint32_t)(total >> 32); equal += (uint32_t)total;
    }
}

// Codes of another scale: code' = round(code f), f = old scale / new scale = 2^k.  In f16, where code f is exact down to 2^-24 (an e4m3 code ends at 2^-9) for k of -24 to 15; below
// that the code becomes zero (f = 0), above it (a row whose codes were all but zero) two factors are needed.
__device__ __forceinline__ uint32_t f16_pow2(float f) {                    // f16 bits of 2^min(k, 15), 0 below 2^-24; twice
    return __half_as_ushort(__float2half_rn(fminf(f, 32768.f))) * 0x10001u;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {    // a NaN gives way to the other
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t codes_of(uint32_t h) {                 // two codes in the low half
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(h));
    return c;
}
__device__ __forceinline__ float top_f16x2(uint32_t h) {                   // larger of two non-negative f16 (0 for NaN)
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    return fmaxf(fmaxf(v.x, v.y), 0.f);
}

// grid: ceil(B * Hkv * dst blocks / MW): a warp per block of 32 kept rows.
// V: a lane per kept row.  The blocks that the rows come from are copied to shared memory whole (one bulk copy each, up to NSB at a time, a multiple of 32 bytes apart so that
// four of them lie in different banks), a lane then picks its row's byte of channel after channel, and 32 lanes write the 32 bytes of a channel.
// K, whose rows are read as they lie, is done while the first of these copies are on their way.
// Three copies at a time leave shared memory and registers for six CTAs per SM (8 x 24 heads of 80, 8000 of up to 32768 rows: 155.7 us with the choice, four and five CTAs 172, two 157.3; seven CTAs of 72
// registers 173; 24000 rows: 262 and 294).
constexpr int MW = 4, NSB = 3;
template <int D>
__global__ void __launch_bounds__(MW * 32, D == 128 ? 4 : 6)
kv8_move_kernel(const EvictArgs a, int blocks, int *status) {
    constexpr unsigned ALL = 0xffffffffu;
    constexpr uint32_t SLOT = D * BLK + 32;
    extern __shared__ __align__(128) uint8_t sm[];
    __shared__ uint64_t bars[MW];
    __shared__ int abort_word;
    volatile int *abort_flag = &abort_word;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) *abort_flag = 0;
    if (lane == 0) tc::mbar_init(&bars[warp], 1);
    tc::mbar_fence_init();
    __syncthreads();
    const int64_t w = (int64_t)blockIdx.x * MW + warp;
    const int j = (int)(w % blocks), bh = min((int)(w / blocks), a.B * a.H - 1), b = bh / a.H;
    const int kept = min(rows_of(a, b), a.keep), n = min(BLK, kept - j * BLK);
    pdl_wait();                                    // (the choice; lengths were there before it)
    pdl_trigger();
    if (w >= (int64_t)a.B * a.H * blocks || n <= 0) return;
    const int64_t sb = (int64_t)bh * (a.src.cap / BLK), db = (int64_t)bh * (a.dst.cap / BLK) + j;
    // (lanes behind the last row repeat it; the bound holds for all that the choice writes, and keeps weights that somebody changes meanwhile from becoming wrong accesses)
    const int row = (int)min((unsigned)a.rows[(int64_t)bh * a.keep + j * BLK + min(lane, n - 1)], (unsigned)(a.src.cap - 1));
    // source blocks in order: this lane's row is the first of its block, and the blocks' number up to here
    const int blk = row / BLK, blk_before = __shfl_up_sync(ALL, blk, 1);
    const bool head = lane == 0 || blk != blk_before;
    const unsigned heads = __ballot_sync(ALL, head);
    const int nth = __popc(heads & ((2u << lane) - 1)) - 1, nb = __popc(heads);
    uint8_t *slots = sm + warp * (NSB * SLOT);
    auto fetch = [&](int b0) {
        if (lane == 0) tc::mbar_expect_tx(&bars[warp], min(NSB, nb - b0) * (D * BLK));
        __syncwarp();                              // (also: the bytes of the round before have been picked)
        if (head && nth >= b0 && nth < b0 + NSB) tc::bulk_load(slots + (nth - b0) * SLOT, a.src.v + (sb + blk) * (D * BLK), D * BLK, &bars[warp]);
    };
    fetch(0);
    const float ksc = a.src.ks[sb + blk], vsc = a.src.vs[sb + blk];
    if (lane < n) a.acc_out[(int64_t)bh * a.dst.cap + j * BLK + lane] = a.acc_in[(int64_t)bh * a.src.cap + row];
    {
        // K: a row is D bytes, pieces of 16 over the lanes
        constexpr int U = D / 16;
        uint4 c[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + 32 * i, r = u / U, rr = __shfl_sync(ALL, row, r);
            c[i] = __ldg(reinterpret_cast<const uint4 *>(a.src.k + ((int64_t)bh * a.src.cap + rr) * D) + (u - r * U));
        }
        uint32_t h[U][8];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint32_t q[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[i][2 * k] = f16x2_of(q[k]); h[i][2 * k + 1] = f16x2_of(q[k] >> 16);
                m = max_f16x2(m, h[i][2 * k] & 0x7fff7fffu);
                m = max_f16x2(m, h[i][2 * k + 1] & 0x7fff7fffu);
            }
            top = fmaxf(top, top_f16x2(m) * __shfl_sync(ALL, ksc, (lane + 32 * i) / U));
        }
#pragma unroll
        for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, off));
        const float s = scale_of(top), f = ksc * inverse_pow2(s);
        if (lane == 0) a.dst.ks[db] = s;
        const bool far = __any_sync(ALL, f > 32768.f);
        uint8_t *o = a.dst.k + db * BLK * D;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + 32 * i, r = u / U;
            const float fr = __shfl_sync(ALL, f, r);
            const uint32_t g = f16_pow2(fr), g2 = f16_pow2(fr > 32768.f ? fr * 0x1p-15f : 1.f);
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t x = mul_f16x2(h[i][2 * k], g), y = mul_f16x2(h[i][2 * k + 1], g);
                if (far) { x = mul_f16x2(x, g2); y = mul_f16x2(y, g2); }
                q[k] = codes_of(x) | codes_of(y) << 16;
            }
            if (r < n) *(reinterpret_cast<uint4 *>(o + r * D) + (u - r * U)) = make_uint4(q[0], q[1], q[2], q[3]);
        }
    }
    uint32_t h[D / 2];                             // this lane's row of V, two channels a register, in f16
    uint32_t phase = 0;
    for (int b0 = 0; b0 < nb; b0 += NSB) {
        if (b0) fetch(b0);
        if (!tc::mbar_wait_warp(&bars[warp], phase, abort_flag, status)) {
            tc::mbar_wait_quiet(&bars[warp], phase, 1000000ull);       // (the copies in flight)
            return;
        }
        phase ^= 1;
        const uint8_t *p = slots + (nth - b0) * SLOT + row % BLK;
        if (nth >= b0 && nth < b0 + NSB) {
#pragma unroll
            for (int c = 0; c < D / 2; ++c) h[c] = f16x2_of((uint32_t)p[2 * c * BLK] | (uint32_t)p[(2 * c + 1) * BLK] << 8);
        }
        __syncwarp();
    }
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < D / 2; ++c) m = max_f16x2(m, h[c] & 0x7fff7fffu);
    float top = top_f16x2(m) * vsc;
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, off));
    const float s = scale_of(top), f = vsc * inverse_pow2(s);
    if (lane == 0) a.dst.vs[db] = s;
    const uint32_t g = f16_pow2(f);
    if (__any_sync(ALL, f > 32768.f)) {
        const uint32_t g2 = f16_pow2(f > 32768.f ? f * 0x1p-15f : 1.f);
#pragma unroll
        for (int c = 0; c < D / 2; ++c) h[c] = mul_f16x2(h[c], g2);
    }
    if (lane < n) {
        uint8_t *o = a.dst.v + db * D * BLK + lane;
#pragma unroll
        for (int c = 0; c < D / 2; ++c) {
            const uint32_t q = codes_of(mul_f16x2(h[c], g));
            o[2 * c * BLK] = (uint8_t)q;
            o[(2 * c + 1) * BLK] = (uint8_t)(q >> 8);
        }
    }
}

template <int D>
cudaError_t launch_move(const EvictArgs &a, int blocks, int64_t ctas, int *status, cudaStream_t s) {
    constexpr int smem = MW * NSB * (D * BLK + 32);
    cudaError_t e = cudaFuncSetAttribute(kv8_move_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_chain(kv8_move_kernel<D>, dim3((unsigned)ctas), MW * 32, smem, s, 0, a, blocks, status);
}

}  // namespace

size_t kv8_evict_workspace(int B, int H, int keep) { return align_up((size_t)B * H * keep * sizeof(int32_t)); }

cudaError_t kv8_evict(const kv8::Cache &src, const kv8::Cache &dst, const float *acc_in, float *acc_out, const int32_t *lens_in, int32_t *lens_out, int32_t *rows_out, int B,
                      int H, int D, int max_rows, int keep, int recent, void *ws, cudaStream_t s) {
    EvictArgs a{src, dst, acc_in, acc_out, lens_in, lens_out, rows_out ? rows_out : static_cast<int32_t *>(ws), B, H, max_rows, keep, recent};
    const int blocks = ((keep < max_rows ? keep : max_rows) + BLK - 1) / BLK;
    const int64_t ctas = ((int64_t)B * H * blocks + MW - 1) / MW;
    if (ctas > 0x7fffffff) return cudaErrorNotSupported;
    cudaError_t e = launch_chain(max_rows <= 32 * CT ? kv8_choose_kernel<32> : kv8_choose_kernel<0>, dim3((unsigned)(B * H)), CT, 0, s, 0, a);
    if (e != cudaSuccess || blocks == 0) return e;
    int *status = device_status_ptr();
    if (!status) return cudaErrorInitializationError;
    return D == 64 ? launch_move<64>(a, blocks, ctas, status, s) : D == 80 ? launch_move<80>(a, blocks, ctas, status, s) : launch_move<128>(a, blocks, ctas, status, s);
}

}  // namespace dm
