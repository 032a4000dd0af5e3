// Rows with little accumulated attention weight leave the 8-bit cache (per sequence and kv head), the others move up, in order, into another cache.
// Two launches.  The choice: one CTA per (sequence, head) finds the keep-th largest weight with a radix selection (three passes over the weights, 11 bits each, counted in shared
// memory; whole numbers, so the order of the additions does not matter) and writes the kept rows' numbers in ascending order.  The move: one warp per block of 32 kept
// rows, for K and for V; it finds the new block's scale from the codes' largest bytes (e4m3 orders like its bits) and copies codes, converting only
// those whose scale changes.  Attention without positions does not see where a row lies, so the kept rows need no numbers of their own.
// The choice is bound by latency, the move by memory.
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
    int32_t *rows;                                 // [B * Hkv, keep] kept rows (workspace)
    int32_t *rows_out;                             // the same for the caller, -1 behind the last, or NULL
    int B, H, max_rows, keep, recent;
};

constexpr int CT = 1024, BINS = 2048;

// larger weight, larger key; NaN below everything (0), the two zeros alike
__device__ __forceinline__ uint32_t key_of(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ int rows_of(const EvictArgs &a, int b) { return min(min(max(a.lens_in[b], 0), a.src.cap), a.max_rows); }

// exclusive prefix sum over the CTA; *total: the sum.  Both halves of a 64-bit word (two counters) at once.
__device__ __forceinline__ unsigned long long cta_prefix(unsigned long long v, unsigned long long *part, unsigned long long *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long x = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();
    if (lane == 31) part[warp] = x;
    __syncthreads();
    if (warp == 0) {
        unsigned long long s = part[lane];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const unsigned long long y = __shfl_up_sync(0xffffffffu, s, off);
            if (lane >= off) s += y;
        }
        part[lane] = s;
    }
    __syncthreads();
    *total = part[CT / 32 - 1];
    return x - v + (warp ? part[warp - 1] : 0ull);
}

// grid: B * Hkv
__global__ void __launch_bounds__(CT)
kv8_choose_kernel(const EvictArgs a) {
    __shared__ uint32_t hist[BINS];
    __shared__ unsigned long long part[CT / 32];
    __shared__ uint32_t found[2];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, bh = blockIdx.x, b = bh / a.H;
    const int n = rows_of(a, b), kept = min(n, a.keep);
    const float *acc = a.acc_in + (int64_t)bh * a.src.cap;
    int32_t *rows = a.rows + (int64_t)bh * a.keep, *out = a.rows_out ? a.rows_out + (int64_t)bh * a.keep : nullptr;
    if (bh == b * a.H && tid == 0) a.lens_out[b] = kept;
    if (out)
        for (int i = kept + tid; i < a.keep; i += CT) out[i] = -1;
    if (n <= a.keep) {
        for (int i = tid; i < n; i += CT) { rows[i] = i; if (out) out[i] = i; }
        return;
    }
    const int old = n - min(a.recent, a.keep), want = a.keep - (n - old);        // rows that compete, and how many of them stay
    // the want-th largest key: 11, 11 and 10 bits
    uint32_t prefix = 0, mask = 0;
    int left = want;                               // how many of the keys that agree with the prefix are still to be taken
    if (want > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < BINS; i += CT) hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < old; i += CT) {
                const uint32_t k = key_of(acc[i]);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
            // bins from the top: thread i owns bins BINS - 1 - 2 i and the one below
            const uint32_t c0 = hist[BINS - 1 - 2 * tid], c1 = hist[BINS - 2 - 2 * tid];
            unsigned long long total;
            const uint32_t before = (uint32_t)cta_prefix((unsigned long long)c0 + c1, part, &total);
            if (before < (uint32_t)left && before + c0 >= (uint32_t)left) { found[0] = BINS - 1 - 2 * tid; found[1] = left - before; }
            else if (before + c0 < (uint32_t)left && before + c0 + c1 >= (uint32_t)left) { found[0] = BINS - 2 - 2 * tid; found[1] = left - before - c0; }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= ((1u << bits) - 1) << shift;
            left = (int)found[1];
            __syncthreads();
        }
    }
    // kept: key above the threshold, or equal to it and among the first `left` such rows, or recent
    uint32_t above = 0, equal = 0;                 // rows so far
    for (int base = 0; base < n; base += CT * 4) {
        const int i0 = base + tid * 4;
        uint32_t g = 0, e = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = i0 + q;
            if (i >= n) continue;
            const uint32_t k = i < old && want > 0 ? key_of(acc[i]) : 0u;
            if (i >= old || (want > 0 && k > prefix)) g |= 1u << q;
            else if (want > 0 && k == prefix) e |= 1u << q;
        }
        unsigned long long total;
        const unsigned long long before = cta_prefix((unsigned long long)__popc(g) << 32 | __popc(e), part, &total);
        uint32_t na = above + (uint32_t)(before >> 32), ne = equal + (uint32_t)before;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool ge = (g >> q) & 1, eq = (e >> q) & 1;
            if (ge || (eq && ne < (uint32_t)left)) {
                const uint32_t at = na + min(ne, (uint32_t)left);
                rows[at] = i0 + q;
                if (out) out[at] = i0 + q;
            }
            na += ge; ne += eq;
        }
        above += (uint32_t)(total >> 32); equal += (uint32_t)total;
    }
}

// largest byte of (w & 0x7f..) over four codes, the NaN code counting as 0
__device__ __forceinline__ uint32_t top_codes(uint32_t w) {
    const uint32_t m = w & 0x7f7f7f7fu;
    return m & ~__vcmpeq4(m, 0x7f7f7f7fu);
}
// four codes from scale s to s / ratio ... code' = round(code * f), f = old scale / new scale
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
    const float2 a = decode2(w), b = decode2(w >> 16);
    return encode2(a.x * f, a.y * f) | encode2(b.x * f, b.y * f) << 16;
}
__device__ __forceinline__ float code_value(uint32_t c) { return decode2(c).x; }

constexpr int MW = 8;
// grid: ceil(B * Hkv * dst blocks * 2 / MW): a warp per block of 32 kept rows and side
template <int D>
__global__ void __launch_bounds__(MW * 32)
kv8_move_kernel(const EvictArgs a, int blocks) {
    constexpr unsigned ALL = 0xffffffffu;
    const int lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    int64_t w = (int64_t)blockIdx.x * MW + (threadIdx.x >> 5);
    if (w >= (int64_t)a.B * a.H * blocks * 2) return;
    const int side = (int)(w & 1);
    w >>= 1;
    const int j = (int)(w % blocks), bh = (int)(w / blocks), b = bh / a.H;
    const int kept = min(rows_of(a, b), a.keep), n = min(BLK, kept - j * BLK);
    if (n <= 0) return;
    const int64_t sb = (int64_t)bh * (a.src.cap / BLK), db = (int64_t)bh * (a.dst.cap / BLK) + j;
    const int row = a.rows[(int64_t)bh * a.keep + j * BLK + min(lane, n - 1)];       // (lanes behind the last row repeat it)
    const float sc = (side ? a.src.vs : a.src.ks)[sb + row / BLK];
    if (!side) {
        // K: a row is D bytes, pieces of 16 over the lanes
        if (lane < n) a.acc_out[(int64_t)bh * a.dst.cap + j * BLK + lane] = a.acc_in[(int64_t)bh * a.src.cap + row];
        constexpr int U = D / 16;
        uint4 c[U];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + 32 * i, r = u / U;
            const int rr = __shfl_sync(ALL, row, r);
            const float rs = __shfl_sync(ALL, sc, r);
            c[i] = __ldg(reinterpret_cast<const uint4 *>(a.src.k + ((int64_t)bh * a.src.cap + rr) * D) + (u - r * U));
            uint32_t m = __vmaxu4(__vmaxu4(top_codes(c[i].x), top_codes(c[i].y)), __vmaxu4(top_codes(c[i].z), top_codes(c[i].w)));
            m = max(max(m & 0xff, (m >> 8) & 0xff), max((m >> 16) & 0xff, m >> 24));
            top = fmaxf(top, code_value(m) * rs);
        }
#pragma unroll
        for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, off));
        const float s = scale_of(top), inv = inverse_pow2(s);
        if (lane == 0) a.dst.ks[db] = s;
        uint8_t *o = a.dst.k + db * BLK * D;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = lane + 32 * i, r = u / U;
            const float f = __shfl_sync(ALL, sc, r) * inv;
            if (f != 1.f) c[i] = make_uint4(rescale4(c[i].x, f), rescale4(c[i].y, f), rescale4(c[i].z, f), rescale4(c[i].w, f));
            if (r < n) *(reinterpret_cast<uint4 *>(o + r * D) + (u - r * U)) = c[i];
        }
        return;
    }
    // V: a lane per channel; of each source block its 32 bytes, squeezed to the kept ones
    const int blk = row / BLK;
    float top = 0.f;
    for (unsigned todo = n == 32 ? ALL : (1u << n) - 1; todo;) {
        const int l = __ffs(todo) - 1, sbk = __shfl_sync(ALL, blk, l);
        const unsigned mine = __ballot_sync(ALL, blk == sbk) & todo;
        const unsigned rows = __reduce_or_sync(ALL, (mine >> lane) & 1 ? 1u << (row % BLK) : 0u);
        const float rs = __shfl_sync(ALL, sc, l);
        todo &= ~mine;
        uint32_t m = 0;
#pragma unroll
        for (int c = lane; c < D; c += 32) {
            const uint4 *p = reinterpret_cast<const uint4 *>(a.src.v + ((sb + sbk) * D + c) * BLK);
            const uint4 x = __ldg(p), y = __ldg(p + 1);
            const uint32_t q[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t nib = (rows >> (4 * i)) & 15u, keepers = ((nib * 0x00204081u) & 0x01010101u) * 0xffu;
                m = __vmaxu4(m, top_codes(q[i]) & keepers);
            }
        }
        m = max(max(m & 0xff, (m >> 8) & 0xff), max((m >> 16) & 0xff, m >> 24));
        top = fmaxf(top, code_value(m) * rs);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, off));
    const float s = scale_of(top), inv = inverse_pow2(s);
    if (lane == 0) a.dst.vs[db] = s;
#pragma unroll 1
    for (int c0 = 0; c0 < D; c0 += 32) {
        const int c = c0 + lane;
        uint32_t w8[8];
        unsigned long long buf = 0;                // bytes squeezed so far that make no whole word yet (at most 3 + 4)
        int have = 0, words = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) w8[i] = 0;
        for (unsigned todo = n == 32 ? ALL : (1u << n) - 1; todo;) {
            const int l = __ffs(todo) - 1, sbk = __shfl_sync(ALL, blk, l);
            const unsigned mine = __ballot_sync(ALL, blk == sbk) & todo;
            const unsigned rows = __reduce_or_sync(ALL, (mine >> lane) & 1 ? 1u << (row % BLK) : 0u);
            const float f = __shfl_sync(ALL, sc, l) * inv;
            todo &= ~mine;
            uint4 x = make_uint4(0, 0, 0, 0), y = x;
            if (c < D) {
                const uint4 *p = reinterpret_cast<const uint4 *>(a.src.v + ((sb + sbk) * D + c) * BLK);
                x = __ldg(p); y = __ldg(p + 1);
            }
            const uint32_t q[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t nib = (rows >> (4 * i)) & 15u;
                if (!nib) continue;
                // the selector that moves the kept bytes of a word down: nibble b holds the position of the b-th set bit
                uint32_t sel = 0, cnt = 0;
#pragma unroll
                for (int bit = 0; bit < 4; ++bit)
                    if ((nib >> bit) & 1) { sel |= bit << (4 * cnt); ++cnt; }
                uint32_t v = f == 1.f ? q[i] : rescale4(q[i], f);
                v = __byte_perm(v, 0, sel) & (cnt == 4 ? ALL : (1u << (8 * cnt)) - 1);
                buf |= (unsigned long long)v << (8 * have);
                have += cnt;
                if (have >= 4) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) if (k == words) w8[k] = (uint32_t)buf;
                    ++words; buf >>= 32; have -= 4;
                }
            }
        }
        if (have) {
#pragma unroll
            for (int k = 0; k < 8; ++k) if (k == words) w8[k] = (uint32_t)buf;
        }
        if (c >= D) continue;
        uint8_t *o = a.dst.v + (db * D + c) * BLK;
        if (n == BLK) {
            reinterpret_cast<uint4 *>(o)[0] = make_uint4(w8[0], w8[1], w8[2], w8[3]);
            reinterpret_cast<uint4 *>(o)[1] = make_uint4(w8[4], w8[5], w8[6], w8[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) if (i < n) o[i] = (uint8_t)(w8[i >> 2] >> (8 * (i & 3)));
        }
    }
}

}  // namespace

size_t kv8_evict_workspace(int B, int H, int keep) { return align_up((size_t)B * H * keep * sizeof(int32_t)); }

cudaError_t kv8_evict(const kv8::Cache &src, const kv8::Cache &dst, const float *acc_in, float *acc_out, const int32_t *lens_in, int32_t *lens_out, int32_t *rows_out, int B,
                      int H, int D, int max_rows, int keep, int recent, void *ws, cudaStream_t s) {
    EvictArgs a{src, dst, acc_in, acc_out, lens_in, lens_out, static_cast<int32_t *>(ws), rows_out, B, H, max_rows, keep, recent};
    const int blocks = ((keep < max_rows ? keep : max_rows) + BLK - 1) / BLK;
    const int64_t ctas = ((int64_t)B * H * blocks * 2 + MW - 1) / MW;
    if (ctas > 0x7fffffff) return cudaErrorNotSupported;
    cudaError_t e = launch_chain(kv8_choose_kernel, dim3((unsigned)(B * H)), CT, 0, s, 0, a);
    if (e != cudaSuccess || blocks == 0) return e;
    auto kern = D == 64 ? kv8_move_kernel<64> : D == 80 ? kv8_move_kernel<80> : kv8_move_kernel<128>;
    return launch_chain(kern, dim3((unsigned)ctas), MW * 32, 0, s, 0, a, blocks);
}

}  // namespace dm
