// Rows with little accumulated attention weight leave the 8-bit cache (per sequence and kv head), the others move up, in order, into another cache.
// Two launches.  The choice: one CTA per (sequence, head) finds the keep-th largest weight with a radix selection (three passes over the weights, 11 bits each, counted in shared
// memory; whole numbers, so the order of the additions does not matter; weights stay in registers) and writes the kept rows' numbers in ascending order.  The move: one warp per block of 32 kept
// rows, for K and for V; it finds the new block's scale and brings the codes to it, in f16.  Attention without positions does not see where a row lies, so the kept rows need no numbers of their own.
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

// grid: B * Hkv.  HELD: a thread keeps the keys of its up to 32 consecutive rows in registers (sequences of up to 32768 rows), and after the first pass the few that share the
// threshold's bin are all that is looked at; otherwise the weights are read again in every pass.
constexpr int HELD_ROWS = 32 * CT, LIST = 4096;
template <bool HELD>
__global__ void __launch_bounds__(CT)
kv8_choose_kernel(const EvictArgs a) {
    __shared__ uint32_t hist[BINS];
    __shared__ unsigned long long part[CT / 32];
    __shared__ uint32_t found[2], listed;
    __shared__ uint32_t list[HELD ? LIST : 1];
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
    const int per = ((n + CT - 1) / CT + 3) / 4 * 4, first = tid * per;          // this thread's rows (HELD)
    uint32_t key[HELD ? 32 : 1];
    if (HELD) {
        const bool wide = (reinterpret_cast<uintptr_t>(acc) & 15u) == 0;
#pragma unroll
        for (int q = 0; q < 32; q += 4) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            const int i = first + q;
            if (q < per && i < old) {
                if (wide && i + 4 <= old) x = __ldg(reinterpret_cast<const float4 *>(acc + i));
                else { x.x = acc[i]; if (i + 1 < old) x.y = acc[i + 1]; if (i + 2 < old) x.z = acc[i + 2]; if (i + 3 < old) x.w = acc[i + 3]; }
            }
            key[HELD ? q : 0] = key_of(x.x); key[HELD ? q + 1 : 0] = key_of(x.y); key[HELD ? q + 2 : 0] = key_of(x.z); key[HELD ? q + 3 : 0] = key_of(x.w);
        }
    }
    // the want-th largest key: 11, 11 and 10 bits
    uint32_t prefix = 0, mask = 0;
    int left = want;                               // how many of the keys that agree with the prefix are still to be taken
    int list_n = -1;                               // keys in the list; -1: there is none
    if (want > 0) {
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < BINS; i += CT) hist[i] = 0;
            if (tid == 0 && pass == 0) listed = 0;
            __syncthreads();
            auto count = [&](uint32_t k) {
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
            };
            if (HELD && list_n >= 0) {
                for (int i = tid; i < list_n; i += CT) count(list[HELD ? i : 0]);
            } else if (HELD) {
#pragma unroll
                for (int q = 0; q < 32; ++q) {
                    if (q >= per) break;
                    if (first + q < old) count(key[HELD ? q : 0]);
                }
            } else {
                for (int i = tid; i < old; i += CT) count(key_of(acc[i]));
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
            const uint32_t in_bin = hist[found[0]];
            __syncthreads();
            if (HELD && pass == 0 && in_bin <= LIST) {
#pragma unroll
                for (int q = 0; q < 32; ++q) {
                    if (q >= per) break;
                    if (first + q < old && (key[HELD ? q : 0] & mask) == prefix) list[HELD ? atomicAdd(&listed, 1u) : 0] = key[HELD ? q : 0];
                }
                list_n = (int)in_bin;
                __syncthreads();
            }
        }
    }
    // kept: key above the threshold, or equal to it and among the first `left` such rows, or recent
    if (HELD) {
        uint32_t g = 0, e = 0;
#pragma unroll
        for (int q = 0; q < 32; ++q) {
            if (q >= per) break;
            const int i = first + q;
            if (i < n && (i >= old || (want > 0 && key[HELD ? q : 0] > prefix))) g |= 1u << q;
            else if (i < old && want > 0 && key[HELD ? q : 0] == prefix) e |= 1u << q;
        }
        unsigned long long total;
        const unsigned long long before = cta_prefix((unsigned long long)__popc(g) << 32 | __popc(e), part, &total);
        // of the equal ones here the first `take` stay
        const int ne = (int)(uint32_t)before, take = min(max(left - ne, 0), __popc(e));
        uint32_t at = (uint32_t)(before >> 32) + min(ne, left);
        for (int k = __popc(e); k > take; --k) e &= ~(0x80000000u >> __clz(e));
        for (uint32_t m = g | e; m; m &= m - 1, ++at) {
            const int i = first + __ffs(m) - 1;
            rows[at] = i;
            if (out) out[at] = i;
        }
        return;
    }
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

// grid: ceil(B * Hkv * dst blocks * 2 / MW): a warp per block of 32 kept rows and side.
// V: a lane per kept row.  The blocks that the rows come from are copied to shared memory whole (one bulk copy each, up to NSB at a time, a multiple of 32 bytes apart so that
// four of them lie in different banks), a lane then picks its row's byte of channel after channel, and 32 lanes write the 32 bytes of a channel.
constexpr int MW = 4, NSB = 4;
template <int D>
__global__ void __launch_bounds__(MW * 32)
kv8_move_kernel(const EvictArgs a, int blocks, int *status) {
    constexpr unsigned ALL = 0xffffffffu;
    constexpr uint32_t SLOT = D * BLK + 32;
    extern __shared__ __align__(128) uint8_t sm[];
    __shared__ uint64_t bars[MW];
    __shared__ int abort_word;
    volatile int *abort_flag = &abort_word;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    pdl_trigger();
    if (threadIdx.x == 0) *abort_flag = 0;
    if (lane == 0) tc::mbar_init(&bars[warp], 1);
    tc::mbar_fence_init();
    __syncthreads();
    int64_t w = (int64_t)blockIdx.x * MW + warp;
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
            top = fmaxf(top, top_f16x2(m) * __shfl_sync(ALL, sc, (lane + 32 * i) / U));
        }
#pragma unroll
        for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, off));
        const float s = scale_of(top), f = sc * inverse_pow2(s);
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
        return;
    }
    uint8_t *slots = sm + warp * (NSB * SLOT);
    const int blk = row / BLK, blk_before = __shfl_up_sync(ALL, blk, 1);
    // source blocks in order: this lane's row is the first of its block, and the blocks' number up to here
    const bool head = lane == 0 || blk != blk_before;
    const unsigned heads = __ballot_sync(ALL, head);
    const int nth = __popc(heads & ((2u << lane) - 1)) - 1, nb = __popc(heads);
    uint32_t h[D / 2];                             // this lane's row, two channels a register, in f16
    uint32_t phase = 0;
    for (int b0 = 0; b0 < nb; b0 += NSB) {
        const bool here = nth >= b0 && nth < b0 + NSB;
        if (lane == 0) tc::mbar_expect_tx(&bars[warp], min(NSB, nb - b0) * (D * BLK));
        __syncwarp();                              // (also: the bytes of the round before have been picked)
        if (here && head) tc::bulk_load(slots + (nth - b0) * SLOT, a.src.v + (sb + blk) * (D * BLK), D * BLK, &bars[warp]);
        if (!tc::mbar_wait(&bars[warp], phase, abort_flag, status)) {
            tc::mbar_wait_quiet(&bars[warp], phase, 1000000ull);       // (the copies in flight)
            return;
        }
        phase ^= 1;
        const uint8_t *p = slots + (nth - b0) * SLOT + row % BLK;
        if (here) {
#pragma unroll
            for (int c = 0; c < D / 2; ++c) h[c] = f16x2_of((uint32_t)p[2 * c * BLK] | (uint32_t)p[(2 * c + 1) * BLK] << 8);
        }
        __syncwarp();
    }
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < D / 2; ++c) m = max_f16x2(m, h[c] & 0x7fff7fffu);
    float top = top_f16x2(m) * sc;
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(ALL, top, off));
    const float s = scale_of(top), f = sc * inverse_pow2(s);
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
    EvictArgs a{src, dst, acc_in, acc_out, lens_in, lens_out, static_cast<int32_t *>(ws), rows_out, B, H, max_rows, keep, recent};
    const int blocks = ((keep < max_rows ? keep : max_rows) + BLK - 1) / BLK;
    const int64_t ctas = ((int64_t)B * H * blocks * 2 + MW - 1) / MW;
    if (ctas > 0x7fffffff) return cudaErrorNotSupported;
    cudaError_t e = launch_chain(max_rows <= HELD_ROWS ? kv8_choose_kernel<true> : kv8_choose_kernel<false>, dim3((unsigned)(B * H)), CT, 0, s, 0, a);
    if (e != cudaSuccess || blocks == 0) return e;
    int *status = device_status_ptr();
    if (!status) return cudaErrorInitializationError;
    return D == 64 ? launch_move<64>(a, blocks, ctas, status, s) : D == 80 ? launch_move<80>(a, blocks, ctas, status, s) : launch_move<128>(a, blocks, ctas, status, s);
}

}  // namespace dm
