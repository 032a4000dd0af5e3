// New rows into the 8-bit key/value cache.  A CTA per (sequence, head, few consecutive blocks of 32 rows), a thread per row and 8 channels of K and of V: what it holds of the
// next block is on its way while the present one's maxima are found (one reduction instruction per warp, one word of shared memory per side), scaled and rounded.  V's
// codes turn channel-major on the way out: 4 x 4 bytes by two exchanges between the lanes of a quad, whole words through shared memory.
// Bound by memory: a row and head is D values read and D bytes written; 4 x 8191 rows, 24 heads of 80, bf16: 75 us = 5.0 TB/s, 16 x 4096: 140 us = 5.4; the SM's pipes are 67 % busy, the
// barriers of a block's maxima the largest wait.  A single token's 16 x 16 heads: 4 us, latency.
#include "kv8.cuh"
#include "tc_ptx.cuh"

namespace dm {
namespace {

using namespace kv8;

struct AppendArgs {
    Cache c;
    const void *kn, *vn;                 // [B * G] rows of pitch ld, heads side by side
    int64_t ld;
    const int32_t *lens, *counts;
    int B, G, H, blocks;                 // blocks: per sequence, as many as G rows can touch
};

template <typename T> struct Piece;      // 8 values of one row
template <> struct Piece<__nv_bfloat16> {
    uint4 r;
    __device__ __forceinline__ void zero() { r = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = __ldg(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {       // values of codes: four significant bits, exact in bf16 (scales reach down to 2^-100)
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
        r = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ uint32_t top() const {                // bits of the largest magnitude; NaN are passed over
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
        __nv_bfloat162 m = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i])));
        const uint32_t b = *reinterpret_cast<const uint32_t *>(&m);
        return max(b << 16, b & 0xffff0000u);
    }
};
template <> struct Piece<float> {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    __device__ __forceinline__ void load(const float *p) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(p)), b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v[i];
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[i];
    }
    __device__ __forceinline__ uint32_t top() const {
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
        return __float_as_uint(m);
    }
};
constexpr uint32_t INF_BITS = 0x7f800000u;
template <typename T> __device__ __forceinline__ uint32_t finite_top(const Piece<T> &p) {
    float x[8], m = 0.f;
    p.get(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fabsf(x[i]) < INFINITY ? fmaxf(m, fabsf(x[i])) : m;
    return __float_as_uint(m);
}
// codes of the 8 values; NaN become the NaN code by themselves, infinities where the caller has seen some
template <typename T> __device__ __forceinline__ uint2 codes_of(const Piece<T> &p, float inv, bool infinite) {
    float x[8];
    p.get(x);
    uint32_t q[4];
    if (infinite) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = encode2(x[2 * i] * inv, x[2 * i + 1] * inv);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint16_t c;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(x[2 * i + 1] * inv), "f"(x[2 * i] * inv));
            q[i] = c;
        }
    }
    return make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
}
// 4 x 4 bytes over the lanes of a quad: lane i has row i's bytes of channels 0..3 and receives channel i's of rows 0..3
__device__ __forceinline__ uint32_t quad_transpose(uint32_t w, int lane) {
    const uint32_t x = __shfl_xor_sync(0xffffffffu, w, 2);
    w = __byte_perm(w, x, lane & 2 ? 0x3276 : 0x5410);
    const uint32_t y = __shfl_xor_sync(0xffffffffu, w, 1);
    return __byte_perm(w, y, lane & 1 ? 0x3715 : 0x6240);
}

// grid: (B * H, runs of `per` blocks); 4 D threads
template <typename T, int D>
__global__ void __launch_bounds__(4 * D)
kv8_append_kernel(const AppendArgs a, int per) {
    constexpr int U = D / 8, VP = 9;               // pieces per row; words per channel in shared memory: the quads of a warp hit 16 banks twice
    __shared__ uint32_t tile[2][D * VP], tops[2][2];
    const int tid = threadIdx.x, lane = tid & 31;
    const int rq = tid / (4 * U), c = (tid - rq * 4 * U) >> 2, r = 4 * rq + (tid & 3);       // this thread's row quad, piece and row
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H;
    const int len = min(max(a.lens[b], 0), a.c.cap), cnt = a.counts ? min(max(a.counts[b], 0), a.G) : a.G, end = min(len + cnt, a.c.cap);
    const int jb0 = blockIdx.y * per, j0 = len / BLK + jb0, j1 = end <= len ? j0 : min(j0 + per, (end + BLK - 1) / BLK);
    if (j0 >= j1) return;                          // nothing of this call falls into these blocks
    const int64_t bh = (int64_t)b * a.H + h, blk0 = bh * (a.c.cap / BLK);
    // this thread's row and 8 channels of the first block (a row before `len` is not read there), then 32 rows on at a time
    int row = j0 * BLK + r;
    const int64_t at0 = ((int64_t)b * a.G + (row - len)) * a.ld + h * D + 8 * c, step = BLK * a.ld;
    const T *kp = static_cast<const T *>(a.kn) + at0, *vp = static_cast<const T *>(a.vn) + at0;
    uint8_t *ko = a.c.k + (bh * a.c.cap + row) * D + 8 * c, *vo = a.c.v + (blk0 + j0) * D * BLK;
    Piece<T> k, v, k2, v2;
    k.zero(); v.zero();
    if (row >= len) {
        if (row < end) { k.load(kp); v.load(vp); }
    } else {                                       // a committed row of a half-full block
        const float ks = a.c.ks[blk0 + j0], vs = a.c.vs[blk0 + j0];
        const uint2 q = *reinterpret_cast<const uint2 *>(ko);
        const uint8_t *p = vo + 8 * c * BLK + r;
        float x[8], y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 d = decode2((e < 2 ? q.x : q.y) >> (16 * (e & 1)));
            x[2 * e] = d.x * ks; x[2 * e + 1] = d.y * ks;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = decode2(p[e * BLK]).x * vs;
        k.set(x); v.set(y);
    }
    if (tid < 4) (&tops[0][0])[tid] = 0;
    __syncthreads();
    for (int j = j0, buf = 0; j < j1; ++j, buf ^= 1) {
        k2.zero(); v2.zero();
        kp += step; vp += step;
        if (j + 1 < j1 && row + BLK < end) { k2.load(kp); v2.load(vp); }
        const uint32_t kt = __reduce_max_sync(0xffffffffu, k.top()), vt = __reduce_max_sync(0xffffffffu, v.top());
        if (lane == 0) { atomicMax(&tops[buf][0], kt); atomicMax(&tops[buf][1], vt); }
        __syncthreads();
        uint32_t ktop = tops[buf][0], vtop = tops[buf][1];
        if (tid < 2) tops[buf ^ 1][tid] = 0;       // (last read before the barrier, next written behind the one below)
        const bool infinite = ktop >= INF_BITS || vtop >= INF_BITS;
        if (infinite) {                            // the same again over what is finite
            __syncthreads();
            if (tid < 2) tops[buf][tid] = 0;
            __syncthreads();
            const uint32_t kf = __reduce_max_sync(0xffffffffu, finite_top(k)), vf = __reduce_max_sync(0xffffffffu, finite_top(v));
            if (lane == 0) { atomicMax(&tops[buf][0], kf); atomicMax(&tops[buf][1], vf); }
            __syncthreads();
            ktop = tops[buf][0]; vtop = tops[buf][1];
        }
        const int rows = min(BLK, end - j * BLK);
        const float ks = scale_of(__uint_as_float(ktop)), vs = scale_of(__uint_as_float(vtop));
        if (tid == 0) { a.c.ks[blk0 + j] = ks; a.c.vs[blk0 + j] = vs; }
        const uint2 kq = codes_of(k, inverse_pow2(ks), infinite), vq = codes_of(v, inverse_pow2(vs), infinite);
        if (row < end) *reinterpret_cast<uint2 *>(ko) = kq;
        const int ch = 8 * c + (tid & 3);
        tile[buf][ch * VP + rq] = quad_transpose(vq.x, lane);
        tile[buf][(ch + 4) * VP + rq] = quad_transpose(vq.y, lane);
        __syncthreads();
        if (rows == BLK) {
            if (tid < 2 * D) {                     // 16 rows of a channel
                const uint32_t *p = &tile[buf][(tid >> 1) * VP + (tid & 1) * 4];
                reinterpret_cast<uint4 *>(vo)[tid] = make_uint4(p[0], p[1], p[2], p[3]);
            }
        } else if (tid < 4 * D) {                  // rows behind the last one stay as they were
            for (int i = tid; i < D * rows; i += 4 * D) {
                const int oc = i / rows, orow = i - oc * rows;
                vo[oc * BLK + orow] = (uint8_t)(tile[buf][oc * VP + (orow >> 2)] >> (8 * (orow & 3)));
            }
        }
        k = k2; v = v2;
        row += BLK; ko += BLK * D; vo += BLK * D;
    }
}

template <typename T>
cudaError_t launch(const AppendArgs &a, int D, cudaStream_t s) {
    const int64_t pairs = (int64_t)a.B * a.H;
    // blocks per CTA: as many as leave some eight CTAs per SM, so that the next block's loads overlap this one's work (4 x 24 heads of 8191 rows: one block each 109 us, four 79, eight 75,
    // 16 73, 32 77; with four CTAs per SM 4 x 16 heads of 8192 rows 40 -> 44)
    int64_t per = pairs * a.blocks / (8 * (int64_t)tc::sm_count());
    per = per < 1 ? 1 : per > 8 ? 8 : per;
    while ((a.blocks + per - 1) / per > 65535) ++per;
    auto kern = D == 64 ? kv8_append_kernel<T, 64> : D == 80 ? kv8_append_kernel<T, 80> : kv8_append_kernel<T, 128>;
    return launch_chain(kern, dim3((unsigned)pairs, (unsigned)((a.blocks + per - 1) / per)), 4 * D, 0, s, 0, a, (int)per);
}

}  // namespace

cudaError_t kv8_append(const kv8::Cache &c, const void *k_new, const void *v_new, int64_t ld, const int32_t *lens, const int32_t *counts, int dtype, int B,
                       int G, int H, int D, cudaStream_t s) {
    AppendArgs a{c, k_new, v_new, ld, lens, counts, B, G, H, (2 * (BLK - 1) + G) / BLK};
    return dtype == DM_BF16 ? launch<__nv_bfloat16>(a, D, s) : launch<float>(a, D, s);
}

}  // namespace dm
