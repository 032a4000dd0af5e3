// What a step reads off its logits, one pass over each row: the log probability of a given token, the entropy of the distribution, and its most likely tokens.
//   S = sum 2^(x L - M), T = sum 2^(x L - M) (x L - M)  with L = log2(e) and M near the largest x L
//   log p_t = ln 2 ((x_t L - M) - log2 S),   H = ln 2 (log2 S - T / S)
// Each thread keeps (M, S, T) of its own; M follows its maximum only when that has grown by more than 3, so that the running sums are seldom rescaled and no term exceeds e^3.
// The k most likely tokens: the k-th largest of 32 group maxima is a lower bound of the k-th largest value, so only threads whose own maximum reaches it are gone through a
// second time (the row is still in L2), and of their values only those at or above the bound, a little more than k as a rule, are ranked, by value and then by id.
// A CTA takes a row; with few rows a cluster of up to eight shares one and the first of them joins the shares through distributed shared memory.
// Bound by reading the logits, with bf16 close to what exponentials and instruction issue allow as well.
#include <cstddef>

#include "dm_internal.h"
#include "tc_ptx.cuh"

namespace dm {
namespace {

using namespace tc;

constexpr int NT = 256, CAP = 2048, KMAX = 32;
constexpr unsigned ALL = 0xffffffffu;
constexpr float L2E = 1.4426950408889634f, LN2 = 0.6931471805599453f, BIG = 1.2676506e30f, FAR = 1048576.f;      // 2^100, 2^20
constexpr float GROWTH = 3.f;

struct ScoreArgs {
    const void *x;
    int64_t ld;
    int rows, vocab, exclude, k;
    const int32_t *tokens;
    float *logprob, *entropy;
    int32_t *ids;
    float *lps;
};

template <typename T> struct Vec;                  // 16 bytes of a row
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    uint4 r;
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void range(float &lo, float &hi) const {     // NaN are passed over
        const __nv_bfloat162 *p = reinterpret_cast<const __nv_bfloat162 *>(&r);
        const __nv_bfloat162 h = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])), l = __hmin2(__hmin2(p[0], p[1]), __hmin2(p[2], p[3]));
        hi = fmaxf(__low2float(h), __high2float(h));
        lo = fminf(__low2float(l), __high2float(l));
    }
    __device__ __forceinline__ void set(int e, float v) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&r);
        const uint32_t b = __float_as_uint(v) >> 16;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i == e) w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | b << 16 : (w[i >> 1] & 0xffff0000u) | b;
    }
};
template <> struct Vec<float> {
    static constexpr int N = 4;
    uint4 r;
    __device__ __forceinline__ void get(float (&x)[4]) const {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
    __device__ __forceinline__ void range(float &lo, float &hi) const {
        float x[4];
        get(x);
        hi = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        lo = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    }
    __device__ __forceinline__ void set(int e, float v) {
        uint32_t *w = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i == e) w[i] = __float_as_uint(v);
    }
};
template <typename T> __device__ __forceinline__ float as_float(T v);
template <> __device__ __forceinline__ float as_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// A row as 16-byte pieces: piece i holds ids [i N - off, i N - off + N), of which those outside [0, vocab) and the excluded one read as -infinity
template <typename T> struct Row {
    static constexpr int N = Vec<T>::N;
    const T *p;
    int off, vocab, exclude, pieces;
    __device__ __forceinline__ Row(const ScoreArgs &a, int row) {
        p = static_cast<const T *>(a.x) + (int64_t)row * a.ld;
        off = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
        vocab = a.vocab; exclude = a.exclude;
        pieces = (off + vocab + N - 1) / N;
    }
    __device__ __forceinline__ int id(int i) const { return i * N - off; }
    __device__ __forceinline__ Vec<T> load(int i) const {
        Vec<T> v;
        const int id0 = id(i);
        if (id0 >= 0 && id0 + N <= vocab) {
            v.r = __ldg(reinterpret_cast<const uint4 *>(p + id0));
        } else {
            v.r = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < N; ++e) v.set(e, id0 + e >= 0 && id0 + e < vocab ? as_float(p[id0 + e]) : -INFINITY);
        }
        if ((unsigned)(exclude - id0) < (unsigned)N) v.set(exclude - id0, -INFINITY);
        return v;
    }
};

// S and T of what a thread has seen, relative to X: a value that it has seen (-infinity: none yet).  The exponents' reference is X log2(e) rounded once, everywhere the same number
// (one FMA per exponent), except where X is so far from zero that this rounding would shift them by more than a tenth.
struct Sums { float X, S, T; };
__device__ __forceinline__ bool ordinary(float X) { return fabsf(X) <= FAR; }
__device__ __forceinline__ float delta(float x, float X) { return ordinary(X) ? fmaf(x, L2E, -(X * L2E)) : (x - X) * L2E; }
__device__ __forceinline__ float move_by(float from, float to) {          // log2 of what sums relative to `from` are multiplied with
    return ordinary(from) && ordinary(to) ? __fsub_rn(from * L2E, to * L2E) : (from - to) * L2E;
}
__device__ __forceinline__ void move_ref(Sums &s, float X) {
    if (s.S != 0.f) {                              // (NaN goes on)
        const float d = move_by(s.X, X), f = ex2f(d);
        s.T = f == 0.f ? 0.f : (s.T + s.S * d) * f;
        s.S *= f;
    }
    s.X = X;
}
template <typename T> __device__ __forceinline__ void take(const Vec<T> &v, Sums &s, float &top) {
    float lo, hi;
    v.range(lo, hi);
    top = fmaxf(top, hi);
    if (hi > s.X + GROWTH) move_ref(s, hi);
    float x[Vec<T>::N];
    v.get(x);
    if (lo >= -BIG && ordinary(s.X)) {
        const float M = s.X * L2E;
#pragma unroll
        for (int e = 0; e < Vec<T>::N; ++e) {
            const float d = fmaf(x[e], L2E, -M), p = ex2f(d);
            s.S += p;
            s.T = fmaf(p, d, s.T);
        }
    } else {                                       // masked ids, or values far from zero
#pragma unroll
        for (int e = 0; e < Vec<T>::N; ++e) {
            if (x[e] == -INFINITY) continue;
            const float d = delta(x[e], s.X), p = ex2f(d);
            s.S += p;
            if (!(p == 0.f)) s.T = fmaf(p, d, s.T);
        }
    }
}

struct Share {                                     // what a CTA of a cluster hands over
    Sums s;
    int n;                                         // candidates: its k most likely ids, or fewer
    float val[KMAX];
    int id[KMAX];
};

__device__ __forceinline__ bool better(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// k-th largest of 32 values, one per lane
__device__ __forceinline__ float kth_of_warp(float v, int k) {
    int rank = 0;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float w = __shfl_sync(ALL, v, j);
        rank += w > v || (w == v && j < lane);
    }
    return __shfl_sync(ALL, v, __ffs(__ballot_sync(ALL, rank == k - 1)) - 1);
}

// grid: rows * C, cluster C
template <typename T>
__global__ void __launch_bounds__(NT, 4)
token_scores_kernel(const ScoreArgs a, int C) {
    __shared__ float red[3][NT / 32], gmax[32], cval[CAP];
    __shared__ int cid[CAP];
    __shared__ int count, fresh;
    __shared__ float pick_v[NT / 32];
    __shared__ int pick_i[NT / 32];
    __shared__ Share mine;
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row = blockIdx.x / C, part = blockIdx.x - row * C;
    const Row<T> r(a, row);
    const int per = (r.pieces + C - 1) / C, i0 = part * per, i1 = min(r.pieces, i0 + per);
    const int tok = a.tokens ? a.tokens[row] : -1;
    const bool known = tok >= 0 && tok < a.vocab && tok != a.exclude;
    const float xt = known && part == 0 ? as_float(r.p[tok]) : -INFINITY;

    Sums s{-INFINITY, 0.f, 0.f};
    float top = -INFINITY;
    constexpr int U = 4;
    for (int i = i0 + tid; i < i1; i += U * NT) {
        Vec<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) if (i + u * NT < i1) v[u] = r.load(i + u * NT);
#pragma unroll
        for (int u = 0; u < U; ++u) if (i + u * NT < i1) take(v[u], s, top);
    }
    // one reference for the CTA, then plain sums
    float X = s.X;
#pragma unroll
    for (int off = 16; off; off >>= 1) X = fmaxf(X, __shfl_xor_sync(ALL, X, off));
    float g = top;
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) g = fmaxf(g, __shfl_xor_sync(ALL, g, off));
    if (lane == 0) red[0][warp] = X;
    if ((lane & 7) == 0) gmax[tid >> 3] = g;
    if (tid == 0) count = 0;
    __syncthreads();
    X = red[0][0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w) X = fmaxf(X, red[0][w]);
    move_ref(s, X);
#pragma unroll
    for (int off = 16; off; off >>= 1) { s.S += __shfl_xor_sync(ALL, s.S, off); s.T += __shfl_xor_sync(ALL, s.T, off); }
    if (lane == 0) { red[1][warp] = s.S; red[2][warp] = s.T; }

    // candidates
    if (a.k > 0) {
        float bound = kth_of_warp(gmax[lane], a.k);
        unsigned hot = __ballot_sync(ALL, top >= bound && top > -INFINITY);
        while (hot) {                              // this thread's pieces over the warp's lanes
            const int l = __ffs(hot) - 1;
            hot &= hot - 1;
            for (int i = i0 + warp * 32 + l + lane * NT; i < i1; i += 32 * NT) {
                float x[Vec<T>::N];
                r.load(i).get(x);
#pragma unroll
                for (int e = 0; e < Vec<T>::N; ++e)
                    if (x[e] >= bound && x[e] > -INFINITY) {
                        const int at = atomicAdd(&count, 1);
                        if (at < CAP) { cval[at] = x[e]; cid[at] = r.id(i) + e; }
                    }
            }
        }
        __syncthreads();
        int n = count;
        if (n <= CAP) {
            // many of them (few groups, or ties): the bound once more, from the candidates' own group maxima
            while (n > NT) {
                float v = -INFINITY;
                for (int i = tid; i < n; i += NT) v = fmaxf(v, cval[i]);
#pragma unroll
                for (int off = 1; off < 8; off <<= 1) v = fmaxf(v, __shfl_xor_sync(ALL, v, off));
                __syncthreads();
                if ((lane & 7) == 0) gmax[tid >> 3] = v;
                if (tid == 0) fresh = 0;
                __syncthreads();
                bound = kth_of_warp(gmax[lane], a.k);
                float kv[CAP / NT];
                int ki[CAP / NT];
#pragma unroll
                for (int q = 0; q < CAP / NT; ++q) {
                    const int i = tid + q * NT;
                    kv[q] = i < n ? cval[i] : -INFINITY;
                    ki[q] = i < n ? cid[i] : 0;
                }
                __syncthreads();
#pragma unroll
                for (int q = 0; q < CAP / NT; ++q)
                    if (tid + q * NT < n && kv[q] >= bound) { const int at = atomicAdd(&fresh, 1); cval[at] = kv[q]; cid[at] = ki[q]; }
                __syncthreads();
                const int m = fresh;
                if (m == n) break;                 // all the same
                n = m;
            }
            for (int i = tid; i < n; i += NT) {
                const float v = cval[i];
                const int id = cid[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += better(cval[j], cid[j], v, id);
                if (rank < a.k) { mine.val[rank] = v; mine.id[rank] = id; }
            }
            if (tid == 0) mine.n = min(n, a.k);
        } else {                                   // more values than room at or above the bound, most of them equal: one by one
            float lv = INFINITY;
            int li = -1, q = 0;
            for (; q < a.k; ++q) {
                float bv = -INFINITY;
                int bi = 0x7fffffff;
                for (int i = i0 + tid; i < i1; i += NT) {
                    float x[Vec<T>::N];
                    r.load(i).get(x);
#pragma unroll
                    for (int e = 0; e < Vec<T>::N; ++e) {
                        const int id = r.id(i) + e;
                        if (x[e] > -INFINITY && better(lv, li, x[e], id) && better(x[e], id, bv, bi)) { bv = x[e]; bi = id; }
                    }
                }
#pragma unroll
                for (int off = 16; off; off >>= 1) {
                    const float ov = __shfl_xor_sync(ALL, bv, off);
                    const int oi = __shfl_xor_sync(ALL, bi, off);
                    if (better(ov, oi, bv, bi)) { bv = ov; bi = oi; }
                }
                __syncthreads();
                if (lane == 0) { pick_v[warp] = bv; pick_i[warp] = bi; }
                __syncthreads();
                lv = pick_v[0]; li = pick_i[0];
#pragma unroll
                for (int w = 1; w < NT / 32; ++w) if (better(pick_v[w], pick_i[w], lv, li)) { lv = pick_v[w]; li = pick_i[w]; }
                if (lv == -INFINITY) break;
                if (tid == 0) { mine.val[q] = lv; mine.id[q] = li; }
            }
            if (tid == 0) mine.n = q;
        }
    }
    __syncthreads();
    if (tid == 0) {
        Sums t{X, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) { t.S += red[1][w]; t.T += red[2][w]; }
        mine.s = t;
        if (a.k == 0) mine.n = 0;
    }
    if (C > 1) {
        cluster_sync();                            // every CTA's share is there
        if (part == 0 && warp == 0) {
            // one warp joins: the sums in the order of the shares, then the candidates one by one off the shares' sorted lists, a lane per share
            Sums t{-INFINITY, 0.f, 0.f};
            const uint32_t theirs = cluster_addr(&mine, min(lane, C - 1));
            auto f32 = [&](uint32_t at) { float v; asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory"); return v; };
            auto s32 = [&](uint32_t at) { int v; asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory"); return v; };
            Sums q{f32(theirs), f32(theirs + 4), f32(theirs + 8)};
            const int have = lane < C ? s32(theirs + (uint32_t)offsetof(Share, n)) : 0;
            float XX = lane < C ? q.X : -INFINITY;
#pragma unroll
            for (int off = 16; off; off >>= 1) XX = fmaxf(XX, __shfl_xor_sync(ALL, XX, off));
            move_ref(q, XX);
            t.X = XX;
            for (int k = 0; k < C; ++k) { t.S += __shfl_sync(ALL, q.S, k); t.T += __shfl_sync(ALL, q.T, k); }
            int at = 0;
            float v = have > 0 ? f32(theirs + (uint32_t)offsetof(Share, val)) : -INFINITY;
            int id = have > 0 ? s32(theirs + (uint32_t)offsetof(Share, id)) : 0x7fffffff, n = 0;
            for (; n < a.k; ++n) {
                float bv = v;
                int bi = id;
#pragma unroll
                for (int off = 16; off; off >>= 1) {
                    const float ov = __shfl_xor_sync(ALL, bv, off);
                    const int oi = __shfl_xor_sync(ALL, bi, off);
                    if (better(ov, oi, bv, bi)) { bv = ov; bi = oi; }
                }
                if (bv == -INFINITY) break;
                if (lane == 0) { cval[n] = bv; cid[n] = bi; }
                if (id == bi) {
                    ++at;
                    v = at < have ? f32(theirs + (uint32_t)offsetof(Share, val) + 4 * at) : -INFINITY;
                    id = at < have ? s32(theirs + (uint32_t)offsetof(Share, id) + 4 * at) : 0x7fffffff;
                }
            }
            __syncwarp();
            for (int i = lane; i < n; i += 32) { mine.val[i] = cval[i]; mine.id[i] = cid[i]; }
            if (lane == 0) { mine.s = t; mine.n = n; }
        }
        cluster_sync();                            // the shares have been read
        if (part != 0) return;
    } else {
        __syncthreads();
    }
    const Sums t = mine.s;
    const float ls = log2f(t.S);
    if (tid == 0) {
        if (a.logprob) a.logprob[row] = t.S != t.S ? t.S : xt == -INFINITY ? -INFINITY : (delta(xt, t.X) - ls) * LN2;
        if (a.entropy) { const float h = (ls - t.T / t.S) * LN2; a.entropy[row] = t.S == 0.f || h < 0.f ? 0.f : h; }
    }
    for (int i = tid; i < a.k; i += NT) {
        const bool there = i < mine.n;
        if (a.ids) a.ids[(int64_t)row * a.k + i] = there ? mine.id[i] : -1;
        if (a.lps) a.lps[(int64_t)row * a.k + i] = t.S != t.S ? t.S : there ? (delta(mine.val[i], t.X) - ls) * LN2 : -INFINITY;
    }
}

}  // namespace

cudaError_t token_scores(const void *logits, int64_t ld, int dtype, int rows, int vocab, int exclude, int k, const int32_t *tokens, float *logprob, float *entropy,
                         int32_t *ids, float *lps, cudaStream_t s) {
    ScoreArgs a{logits, ld, rows, vocab, exclude, k, tokens, logprob, entropy, ids, lps};
    int C = 1;          // enough CTAs for the GPU, none with less than 4096 ids
    while (C < 8 && (int64_t)rows * C * 2 <= 4 * sm_count() && vocab / (C * 2) >= 4096) C *= 2;
    if ((int64_t)rows * C > 0x7fffffff) return cudaErrorNotSupported;
    auto kern = dtype == DM_BF16 ? token_scores_kernel<__nv_bfloat16> : token_scores_kernel<float>;
    return launch_chain(kern, dim3((unsigned)(rows * C)), NT, 0, s, C, a, C);
}

}  // namespace dm
