// What a step reads off its logits, one pass over each row: the log probability of a given token, the entropy of the distribution, and its most likely tokens.
//   S = sum 2^(x L - M), T = sum 2^(x L - M) (x L - M)  with L = log2(e) and M near the largest x L
//   log p_t = ln 2 ((x_t L - M) - log2 S),   H = ln 2 (log2 S - T / S)
// Each thread keeps (M, S, T) of its own; M follows its maximum only when that has grown by more than 3, so that the running sums are seldom rescaled and no term exceeds e^3 (e^4 with bf16, where
// the limit that the growth is held against is itself a bf16 value).
// The k most likely tokens: a lower bound of the k-th largest of the threads' maxima is one of the k-th largest value, so only threads whose own maximum reaches it have
// anything to give: the round of loads that held it is read again (all of the thread's rounds where a second one reaches the bound too), and the values at or above the
// bound, a little more than k as a rule, are ranked, by value and then by id.
// A CTA takes a row; with few rows a cluster of up to eight shares one and the first of them joins the shares through distributed shared memory.
// Bound by reading the logits, with bf16 close to what exponentials and instruction issue allow as well: 8192 rows of 50257 bf16 with eight alternatives
// 148 us = 5.6 TB/s (the floor 126) among others in a captured graph, one call from Python 174; the exponentials' pipe is 70 % busy, and what is done once per row at its end (a bound, the rounds
// read again, ranks) is not hidden.  32 rows of 50304 fp32: 7.2 us in a graph, 9.6 from Python, latencies.
#include <cstddef>

#include "dm_internal.h"
#include "tc_ptx.cuh"

namespace dm {
namespace {

using namespace tc;

constexpr int CAP = 2048, KMAX = 32;
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

// 16 bytes of a row.  floor(): no value below -2^100 (an exponential of it is 0 all the same, but 0 times -infinity is not); NaN stay.
// above(): whether some value is larger than the threshold made by limit_of(); NaN are not.
template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    typedef __nv_bfloat162 Top;                    // running maxima, of even and odd ids
    uint4 r;
    __device__ __forceinline__ const __nv_bfloat162 *pairs() const { return reinterpret_cast<const __nv_bfloat162 *>(&r); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void floored(f32x2 (&x)[4]) const {
        const __nv_bfloat162 lo = __float2bfloat162_rn(-BIG);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __hmax2_nan(pairs()[i], lo);
            x[i] = bf2_to_f2(*reinterpret_cast<const uint32_t *>(&v));
        }
    }
    __device__ __forceinline__ void clear() { r = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }      // nothing but -infinity
    __device__ __forceinline__ Top top() const { return __hmax2(__hmax2(pairs()[0], pairs()[1]), __hmax2(pairs()[2], pairs()[3])); }
    static __device__ __forceinline__ Top none() { return __float2bfloat162_rn(-INFINITY); }
    static __device__ __forceinline__ Top larger(Top a, Top b) { return __hmax2(a, b); }
    static __device__ __forceinline__ float value(Top a) { return fmaxf(__low2float(a), __high2float(a)); }
    static __device__ __forceinline__ Top limit_of(float x) { return __float2bfloat162_rn(x); }
    static __device__ __forceinline__ bool above(Top a, Top limit) { return __hgt2_mask(a, limit) != 0u; }
    static __device__ __forceinline__ bool reaches(Top a, Top least) { return __hge2_mask(a, least) != 0u; }
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
    typedef float Top;
    uint4 r;
    __device__ __forceinline__ void get(float (&x)[4]) const {
        x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
    }
    __device__ __forceinline__ void floored(f32x2 (&x)[2]) const {
        float v[4];
        get(v);
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(v[i]) : "f"(-BIG));
        x[0] = pk2(v[0], v[1]); x[1] = pk2(v[2], v[3]);
    }
    __device__ __forceinline__ void clear() { r = make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    __device__ __forceinline__ Top top() const {
        float x[4];
        get(x);
        return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    }
    static __device__ __forceinline__ Top none() { return -INFINITY; }
    static __device__ __forceinline__ Top larger(Top a, Top b) { return fmaxf(a, b); }
    static __device__ __forceinline__ float value(Top a) { return fmaxf(a, -INFINITY); }
    static __device__ __forceinline__ Top limit_of(float x) { return x; }
    static __device__ __forceinline__ bool above(Top a, Top limit) { return a > limit; }
    static __device__ __forceinline__ bool reaches(Top a, Top least) { return a >= least; }
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
// log p of a value x from the reference and ls = log2 S.  Far from zero in natural units: x log2(e) ends where |x| = 2.4e38.  Not above 0, which a certain id's may round to.
__device__ __forceinline__ float log_p(float x, float X, float ls) {
    const float v = ordinary(X) && ordinary(x) ? (delta(x, X) - ls) * LN2 : (x - X) - ls * LN2;
    return v > 0.f ? 0.f : v;
}
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
// What a thread carries from piece to piece.  M2 = (-X log2(e), twice), or zeros while X is no ordinary number: a piece that then comes to the ordinary way holds nothing but masked ids or NaN.
template <typename T> struct Running {
    typedef Vec<T> V;
    Sums s{-INFINITY, 0.f, 0.f};
    f32x2 S2 = 0ull, T2 = 0ull, M2 = 0ull;
    typename V::Top limit = V::none();
    // the largest round maximum, that round's first piece (~piece: an end of the row), and the largest of the other rounds'
    float best = -INFINITY, second = -INFINITY;
    int where = 0;
    __device__ __forceinline__ void remember(float t, int from) {
        second = fmaxf(second, fminf(best, t));
        if (t > best) { best = t; where = from; }
    }
    __device__ __forceinline__ void flush() {
        float lo, hi;
        upk2(S2, lo, hi); s.S += lo + hi;
        upk2(T2, lo, hi); s.T += lo + hi;
        S2 = T2 = 0ull;
    }
    // values above the limit, the largest of them in t: the reference follows.  False: it is far from zero, and the pieces are to be taken value by value.
    __device__ __forceinline__ bool follow(typename V::Top t) {
        flush();
        const float hi = V::value(t);
        if (hi > s.X + GROWTH) move_ref(s, hi);
        const bool usual = ordinary(s.X);
        limit = usual ? V::limit_of(s.X + GROWTH) : V::none();
        const float M = usual ? -(s.X * L2E) : 0.f;
        M2 = pk2(M, M);
        return usual;
    }
    __device__ __forceinline__ void take(const V &v) {
        f32x2 x[V::N / 2];
        v.floored(x);
        const f32x2 L2 = pk2(L2E, L2E);
#pragma unroll
        for (int e = 0; e < V::N / 2; ++e) {
            const f32x2 d = fma2(x[e], L2, M2);
            float lo, hi;
            upk2(d, lo, hi);
            const f32x2 p = pk2(ex2f(lo), ex2f(hi));
            S2 = add2(S2, p);
            T2 = fma2(p, d, T2);
        }
    }
    __device__ __forceinline__ void take_far(const V &v) {
        float x[V::N];
        v.get(x);
#pragma unroll
        for (int e = 0; e < V::N; ++e) {
            if (x[e] == -INFINITY) continue;
            const float d = delta(x[e], s.X), p = ex2f(d);
            s.S += p;
            if (!(p == 0.f)) s.T = fmaf(p, d, s.T);
        }
    }
};

struct Share {                                     // what a CTA of a cluster hands over
    Sums s;
    int n;                                         // candidates: its k most likely ids, or fewer
    float val[KMAX];
    int id[KMAX];
};

__device__ __forceinline__ bool better(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// 32 values, one per lane, the largest first
__device__ __forceinline__ float sorted(float v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size *= 2)
#pragma unroll
        for (int off = size / 2; off; off /= 2) {
            const float w = __shfl_xor_sync(ALL, v, off);
            const bool down = (lane & size) == 0 || size == 32, lower = (lane & off) == 0;
            v = down == lower ? fmaxf(v, w) : fminf(v, w);
        }
    return v;
}
// A lower bound of the k-th largest (k <= 32) of one value per thread, from sorted warps: k / warps of each warp's are at or above the smallest of their (k / warps)-th, and k of one
// warp's at or above its k-th.  About twice k of the values reach it.  `ends`: room for two values per warp; read after the next barrier by bound_of_cta.
template <int NT> __device__ __forceinline__ void bound_of_warp(float v, int k, float (&ends)[2][NT / 32]) {
    v = sorted(v);
    const int lane = threadIdx.x & 31, part = (k + NT / 32 - 1) / (NT / 32);
    if (lane == part - 1) ends[0][threadIdx.x >> 5] = v;
    if (lane == k - 1) ends[1][threadIdx.x >> 5] = v;
}
template <int NT> __device__ __forceinline__ float bound_of_cta(const float (&ends)[2][NT / 32]) {
    float lo = ends[0][0], hi = ends[1][0];
#pragma unroll
    for (int w = 1; w < NT / 32; ++w) { lo = fminf(lo, ends[0][w]); hi = fmaxf(hi, ends[1][w]); }
    return fmaxf(lo, hi);
}

// grid: rows * C, cluster C.  U: pieces on a thread's way at a time, a round; the SM's other warps add up meanwhile
template <typename T, int NT, int U>
__global__ void __launch_bounds__(NT, (U * Vec<T>::N > 40 ? 896 : 1024) / NT)
token_scores_kernel(const ScoreArgs a, int C) {
    __shared__ float red[3][NT / 32], ends[2][NT / 32], cval[CAP];
    __shared__ int hot[NT], full[NT], hots, fulls;
    __shared__ int cid[CAP];
    __shared__ int count, fresh;
    __shared__ float pick_v[NT / 32];
    __shared__ int pick_i[NT / 32];
    __shared__ float final_val[KMAX];
    __shared__ int final_id[KMAX], joined;
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

    typedef Vec<T> V;
    Running<T> run;
    // pieces [f0, f1) lie wholly inside the row, thread t has every NT-th of them from f0 + t; those at the row's ends are thread 0's and 32's
    const int f0 = max(i0, r.off ? 1 : 0), f1 = min(i1, (r.off + r.vocab) / V::N);
    const int edge0 = i0 < f0 && i0 < i1 ? i0 : -1, edge1 = f1 < i1 && i1 - 1 >= f0 ? i1 - 1 : -1;
    {
        int ex = r.exclude >= 0 && r.exclude < r.vocab ? (r.off + r.exclude) / V::N : -1;
        if (ex < f0 || (ex - f0) % NT != tid) ex = -1 << 30;       // the excluded id is another thread's, or nobody's
        int i = f0 + tid;
        const uint4 *p = reinterpret_cast<const uint4 *>(r.p - r.off) + i;
        int edge = tid == 0 ? edge0 : tid == 32 ? edge1 : -1;
        // thread 0 asks for what lies two rounds on (or one, where they are longer): the rounds' own loads then come from L2 (170 -> 162 us)
        constexpr int AHEAD = (U * V::N > 32 ? 1 : 2) * U * NT;
#pragma unroll 1
        for (; i < f1 || edge >= 0; i += U * NT, p += U * NT) {
            if (tid == 0 && i + AHEAD < f1)
                asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p + AHEAD), "r"(min(f1 - i - AHEAD, U * NT) * 16) : "memory");
            V v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u * NT < f1) v[u].r = __ldg(p + u * NT);
                else v[u].clear();
            }
            int from = i, place = i;
            if ((unsigned)(ex - i) < (unsigned)(U * NT)) {
#pragma unroll
                for (int u = 0; u < U; ++u) if (i + u * NT == ex) v[u].set(r.exclude - r.id(ex), -INFINITY);
            }
            if (i >= f1) { v[0] = r.load(edge); from = edge; place = ~edge; edge = -1; }        // the last round of the two threads that have one
            typename V::Top t = v[0].top();
#pragma unroll
            for (int u = 1; u < U; ++u) t = V::larger(t, v[u].top());
            run.remember(V::value(t), place);
            if (V::above(t, run.limit) && !run.follow(t)) {
#pragma unroll 1
                for (int u = 0; u < U; ++u)
                    if (u == 0 || (place >= 0 && from + u * NT < f1)) run.take_far(r.load(from + u * NT));      // (a round at an end of the row is one piece: what follows that is other threads')
                continue;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) run.take(v[u]);
        }
        run.flush();
    }
    Sums s = run.s;
    const float top = run.best;
    // one reference for the CTA, then plain sums
    float X = s.X;
#pragma unroll
    for (int off = 16; off; off >>= 1) X = fmaxf(X, __shfl_xor_sync(ALL, X, off));
    if (lane == 0) red[0][warp] = X;
    if (tid == 0) { count = 0; hots = 0; fulls = 0; }
    if (a.k > 0) bound_of_warp<NT>(top, a.k, ends);
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
        float bound = bound_of_cta<NT>(ends);
        const typename V::Top least = V::limit_of(bound);          // exact: it is one of the row's values
        auto look = [&](const V &v, int id) {
            float x[V::N];
            v.get(x);
#pragma unroll
            for (int e = 0; e < V::N; ++e)
                if (x[e] >= bound && x[e] > -INFINITY && id + e != r.exclude) {
                    const int at = atomicAdd(&count, 1);
                    if (at < CAP) { cval[at] = x[e]; cid[at] = id + e; }
                }
        };
        const uint4 *base = reinterpret_cast<const uint4 *>(r.p - r.off);
        if (top >= bound && top > -INFINITY) {
            if (run.where >= 0 && run.second < bound) {
                hot[atomicAdd(&hots, 1)] = run.where;
            } else {                               // an end of the row, or a second round
                full[atomicAdd(&fulls, 1)] = tid;
                const int edge = tid == 0 ? edge0 : tid == 32 ? edge1 : -1;
                if (edge >= 0) look(r.load(edge), r.id(edge));
            }
        }
        __syncthreads();
        // the pieces in question, shared out over all threads: one more memory latency for all of them together
        const int one = hots * U, each = (f1 - f0 + NT - 1) / NT, all = one + (f1 > f0 ? fulls * each : 0);
#pragma unroll 1
        for (int j0 = tid; j0 < all; j0 += 2 * NT) {
            V v[2];
            int at[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int j = j0 + u * NT, k = j - one, h = k / max(each, 1);
                at[u] = j >= all ? f1 : j < one ? hot[j / U] + j % U * NT : f0 + full[h] + (k - h * each) * NT;
                if (at[u] < f1) v[u].r = __ldg(base + at[u]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) if (at[u] < f1 && V::reaches(v[u].top(), least)) look(v[u], r.id(at[u]));
        }
        __syncthreads();
        int n = count;
        if (n <= CAP) {
            // many of them (few threads with values, or ties): the bound once more, from the threads' maxima over the candidates
            while (n > NT) {
                float v = -INFINITY;
                for (int i = tid; i < n; i += NT) v = fmaxf(v, cval[i]);
                if (tid == 0) fresh = 0;
                bound_of_warp<NT>(v, a.k, ends);
                __syncthreads();
                bound = bound_of_cta<NT>(ends);
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
                __syncthreads();                   // (read by all before it is cleared again)
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
        if (part == 0) {
            // the sums in the order of the shares; all candidates at once, a thread each (at most 8 x 32)
            auto f32 = [&](uint32_t at) { float v; asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory"); return v; };
            auto s32 = [&](uint32_t at) { int v; asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at) : "memory"); return v; };
            const int share = a.k ? tid / a.k : C, q = tid - share * a.k;
            const uint32_t theirs = cluster_addr(&mine, min(share, C - 1)), lanes = cluster_addr(&mine, min(lane, C - 1));
            const int have = s32(theirs + (uint32_t)offsetof(Share, n));
            const float v = f32(theirs + (uint32_t)offsetof(Share, val) + 4 * min(q, KMAX - 1));
            const int id = s32(theirs + (uint32_t)offsetof(Share, id) + 4 * min(q, KMAX - 1));
            Sums one{f32(lanes), f32(lanes + 4), f32(lanes + 8)};
            const bool there = share < C && q < have;
            if (tid < C * a.k) { cval[tid] = there ? v : -INFINITY; cid[tid] = there ? id : 0x7fffffff; }
            float XX = one.X;
#pragma unroll
            for (int off = 16; off; off >>= 1) XX = fmaxf(XX, __shfl_xor_sync(ALL, XX, off));
            move_ref(one, XX);
            Sums t{XX, 0.f, 0.f};
            for (int k = 0; k < C; ++k) { t.S += __shfl_sync(ALL, one.S, k); t.T += __shfl_sync(ALL, one.T, k); }
            if (tid == 0) joined = 0;
            __syncthreads();                       // (and: this CTA's own share has been read by its threads)
            if (there) {
                int rank = 0;
                for (int k = 0; k < C * a.k; ++k) rank += better(cval[k], cid[k], v, id);
                if (rank < a.k) { final_val[rank] = v; final_id[rank] = id; atomicAdd(&joined, 1); }
            }
            __syncthreads();
            if (tid < KMAX) { mine.val[tid] = final_val[tid]; mine.id[tid] = final_id[tid]; }
            if (tid == 0) { mine.s = t; mine.n = joined; }
        }
        cluster_sync();                            // the shares have been read
        if (part != 0) return;
    }
    __syncthreads();
    const Sums t = mine.s;
    const float ls = log2f(t.S);
    if (tid == 0) {
        if (a.logprob) a.logprob[row] = t.S != t.S ? t.S : xt == -INFINITY ? -INFINITY : log_p(xt, t.X, ls);
        if (a.entropy) { const float h = (ls - t.T / t.S) * LN2; a.entropy[row] = t.S == 0.f || h < 0.f ? 0.f : h; }
    }
    for (int i = tid; i < a.k; i += NT) {
        const bool there = i < mine.n;
        if (a.ids) a.ids[(int64_t)row * a.k + i] = there ? mine.id[i] : -1;
        if (a.lps) a.lps[(int64_t)row * a.k + i] = t.S != t.S ? t.S : there ? log_p(mine.val[i], t.X, ls) : -INFINITY;
    }
}

}  // namespace

cudaError_t token_scores(const void *logits, int64_t ld, int dtype, int rows, int vocab, int exclude, int k, const int32_t *tokens, float *logprob, float *entropy,
                         int32_t *ids, float *lps, cudaStream_t s) {
    ScoreArgs a{logits, ld, rows, vocab, exclude, k, tokens, logprob, entropy, ids, lps};
    int C = 1;          // enough CTAs for the GPU, none with less than 4096 ids
    while (C < 8 && (int64_t)rows * C * 2 <= 4 * sm_count() && vocab / (C * 2) >= 4096) C *= 2;
    if ((int64_t)rows * C > 0x7fffffff) return cudaErrorNotSupported;
    // Many rows: 128 threads each, what is done once per row costs fewer warps (8192 rows of 50257 bf16, rounds of 4: 160 us, with 256 threads 195); few: 256, which are sooner through
    // their share (32 rows of 50304 fp32: 7.2 us, with 128 threads 7.8; one CTA per row instead of a cluster: 12.4)
    const int nt = C == 1 ? 128 : 256;
    typedef void (*Kernel)(const ScoreArgs, int);
    Kernel kern = nt == 128 ? token_scores_kernel<float, 128, 8> : token_scores_kernel<float, 256, 8>;
    if (dtype == DM_BF16 && nt == 256) kern = token_scores_kernel<__nv_bfloat16, 256, 4>;
    if (dtype == DM_BF16 && nt == 128) {
        // The length of a round by what all rounds of a row's four warps cost: its pieces, filled or not, and about one more (50257 ids, 49 or 50 pieces per thread: rounds of 7 147.8 us, 5 152.2,
        // 6 155.0, 4 159.4; 32000 ids: 7 111.7, 4 115.1; 20000 rows of 1000 ids: 4 86.5, 5 92.6)
        auto cost = [&](int u) {
            int rounds = 0;
            for (int w = 0; w < 4; ++w) rounds += ((vocab / 8 - 32 * w + 127) / 128 + u - 1) / u;
            return rounds * (u + 1);
        };
        int u = 4;
        for (int v = 5; v <= 7; ++v) if (cost(v) <= cost(u)) u = v;
        kern = u == 4 ? token_scores_kernel<__nv_bfloat16, 128, 4> : u == 5 ? token_scores_kernel<__nv_bfloat16, 128, 5>
             : u == 6 ? token_scores_kernel<__nv_bfloat16, 128, 6> : token_scores_kernel<__nv_bfloat16, 128, 7>;
    }
    return launch_chain(kern, dim3((unsigned)(rows * C)), nt, 0, s, C, a, C);
}

}  // namespace dm
