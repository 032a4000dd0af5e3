// New rows into the 8-bit key/value cache.  One warp per (sequence, head, block of 32 rows, K or V): it reads the block's rows (new ones from the
// projection's output, committed ones of a half-full block from the cache), finds the scale with a butterfly of maxima and writes codes and scale.  The
// blocks do not depend on each other, and nothing is read twice.  Bound by memory: a row and head is D values read and D bytes written.
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

constexpr int AW = 8;                    // warps per CTA

template <typename T> struct Piece;      // 8 values of one row
template <> struct Piece<__nv_bfloat16> {
    uint4 r;
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
};
template <> struct Piece<float> {
    float v[8];
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
};

// grid: ceil(B * H * blocks * 2 / AW)
template <typename T, int D>
__global__ void __launch_bounds__(AW * 32)
kv8_append_kernel(const AppendArgs a) {
    constexpr int U = D / 8, N = U;                // pieces per row, and per lane: 32 rows of U pieces over 32 lanes
    constexpr int VP = 36;                         // pitch of a channel's 32 bytes in shared memory: four lanes of a row hit four banks
    __shared__ __align__(16) uint8_t tile[AW][D * VP];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    int64_t w = (int64_t)blockIdx.x * AW + warp;
    if (w >= (int64_t)a.B * a.H * a.blocks * 2) return;
    const int side = (int)(w & 1);
    w >>= 1;
    const int h = (int)(w % a.H);                  // heads next to each other: their columns of a row are too
    w /= a.H;
    const int jb = (int)(w % a.blocks), b = (int)(w / a.blocks);
    const int len = min(max(a.lens[b], 0), a.c.cap), cnt = a.counts ? min(max(a.counts[b], 0), a.G) : a.G, end = min(len + cnt, a.c.cap);
    const int j = len / BLK + jb, r0 = j * BLK;
    if (r0 >= end || end <= len) return;           // nothing of this call falls into the block
    const int rows = min(BLK, end - r0), old = max(0, len - r0);
    const int64_t bh = (int64_t)b * a.H + h, blk = bh * (a.c.cap / BLK) + j;
    uint8_t *codes = side ? a.c.v + blk * D * BLK : a.c.k + (bh * a.c.cap + r0) * D;
    float *scale = (side ? a.c.vs : a.c.ks) + blk;
    const T *src = static_cast<const T *>(side ? a.vn : a.kn) + h * D;

    Piece<T> x[N];
    const float was = old ? *scale : 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = lane + 32 * i, r = u / U, c = (u - r * U) * 8;
        const float zero[8] = {};
        if (r >= old && r < rows) x[i].load(src + ((int64_t)b * a.G + (r0 + r - len)) * a.ld + c);
        else x[i].set(zero);
        if (r < old) {
            float v[8];
            if (side) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = decode2(codes[(c + e) * BLK + r]).x * was;
            } else {
                const uint2 q = *reinterpret_cast<const uint2 *>(codes + r * D + c);
                const uint32_t qw[2] = {q.x, q.y};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 d = decode2(qw[e >> 1] >> (16 * (e & 1)));
                    v[2 * e] = d.x * was; v[2 * e + 1] = d.y * was;
                }
            }
            x[i].set(v);
        }
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[8];
        x[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) { const float m = fabsf(v[e]); top = m < INFINITY ? fmaxf(top, m) : top; }
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const float s = scale_of(top), inv = inverse_pow2(s);
    if (lane == 0) *scale = s;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int u = lane + 32 * i, r = u / U, c = (u - r * U) * 8;
        float v[8];
        x[i].get(v);
        const uint32_t q0 = encode2(v[0] * inv, v[1] * inv) | encode2(v[2] * inv, v[3] * inv) << 16;
        const uint32_t q1 = encode2(v[4] * inv, v[5] * inv) | encode2(v[6] * inv, v[7] * inv) << 16;
        if (side) {
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[warp][(c + e) * VP + r] = (uint8_t)((e < 4 ? q0 : q1) >> (8 * (e & 3)));
        } else if (r < rows) {
            *reinterpret_cast<uint2 *>(codes + r * D + c) = make_uint2(q0, q1);
        }
    }
    if (!side) return;
    __syncwarp();                                  // (also: every lane has read the committed rows' codes)
    if (rows == BLK) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {         // 16 rows of a channel per lane
            const int u = lane + 32 * i, c = u >> 1, r = (u & 1) * 16;
            const uint32_t *p = reinterpret_cast<const uint32_t *>(&tile[warp][c * VP + r]);
            *reinterpret_cast<uint4 *>(codes + c * BLK + r) = make_uint4(p[0], p[1], p[2], p[3]);
        }
    } else {                                       // rows behind the last one stay as they were
        for (int c = 0; c < D; ++c)
            if (lane < rows) codes[c * BLK + lane] = tile[warp][c * VP + lane];
    }
}

template <typename T>
cudaError_t launch(const AppendArgs &a, int D, cudaStream_t s) {
    const int64_t ctas = ((int64_t)a.B * a.H * a.blocks * 2 + AW - 1) / AW;
    if (ctas > 0x7fffffff) return cudaErrorNotSupported;
    auto kern = D == 64 ? kv8_append_kernel<T, 64> : D == 80 ? kv8_append_kernel<T, 80> : kv8_append_kernel<T, 128>;
    return launch_chain(kern, dim3((unsigned)ctas), AW * 32, 0, s, 0, a);
}

}  // namespace

cudaError_t kv8_append(const kv8::Cache &c, const void *k_new, const void *v_new, int64_t ld, const int32_t *lens, const int32_t *counts, int dtype, int B,
                       int G, int H, int D, cudaStream_t s) {
    AppendArgs a{c, k_new, v_new, ld, lens, counts, B, G, H, (2 * (BLK - 1) + G) / BLK};
    return dtype == DM_BF16 ? launch<__nv_bfloat16>(a, D, s) : launch<float>(a, D, s);
}

}  // namespace dm
