// deco_token_logprobs / deco_token_logprobs_grad: log probabilities of given tokens under rows of
// logits, with entropy, log-sum-exp and the largest alternatives, and the gradient of all of them.
//
// Forward: one pass over the logits.  With c = scale * log2(e) a thread keeps, for the entries
// it has seen, the maximum m, s = sum 2^t and q = sum 2^t t with t = x c - S, where S is m c rounded.
// A larger maximum multiplies s by f = 2^(S_old - S_new) and turns q into f (q + (S_old - S_new) s): the
// difference of the rounded numbers, against which the sums were taken, so that what rounding
// did to S is in no result, however far from 0 the logits are.  At the end of the row
// entropy = ln2 (log2 s - q / s),  logprob = ln2 (t_target - log2 s)  and
// lse = m scale + ln2 (log2 s - (m c - S)).
//
// A row is one CTA's work, or a cluster's of 2, 4 or 8 CTAs, each with a contiguous part of it,
// where the rows alone would leave most of the device idle; the parts are joined through
// distributed shared memory, so there is no workspace and no second launch.
//
// What bounds it: one exponential per logit takes as long as reading two bytes of it from memory (16 a cycle
// and SM against 44 bytes a nanosecond), and the other instructions about as long again, so the pass works on
// pairs of logits (fma and add of two fp32 numbers at once) and has no bounds check inside a row.  8192 rows of
// 50257 bf16: 160 us, 5.2 TB/s, exponential units 76 % busy.  Short calls are bounded by their chain of
// barriers: 6 us for one row of 32000 with 20 alternatives on eight CTAs.
//
// Alternatives: a thread's maximum over its entries is known when the pass ends.  The k-th largest of 64
// groups' maxima is a bound which at least k entries reach and few more than k do; only threads
// whose maximum reaches it have their entries read again (from L2), 32 granules at a time by their warp.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>

#include "deco.h"

namespace cg = cooperative_groups;

namespace {

constexpr int NT = 256;                  // threads of a CTA
constexpr int WARPS = NT / 32;
constexpr int UNROLL = 2;                // 16-byte loads of a thread per batch; one more batch is in flight
constexpr int GRAD_UNROLL = 4;           // granules of a thread in the gradient
constexpr int GROUPS = 64;               // groups of threads whose maxima bound the alternatives
constexpr int MAX_TOP = DECO_LOGPROBS_MAX_TOP;
constexpr int LIST = 1024;               // candidates kept for the alternatives
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
// The streaming path treats entries below FLOOR as FLOOR, with weight 0 (masks of -inf, of the
// type's lowest value, of -1e10 ...).  That is exact for rows whose maximum m has |m c| < SPAN and
// scales in [SCALE_LO, SCALE_HI]: then (FLOOR - m) c < -2^20, and a weight of the maximum, 2^(m c - S), lies
// within 2^(1/16) of 1.  All other rows, and rows with a NaN, take the slow path.  While a thread
// has seen nothing above FAR / c (masked entries alone) it sums against 0, so that they all have weight 0, as they
// have in a row of this path: S may be -2^32 there, and its rounding would make weights of 2^128.
constexpr float FLOOR = -0x1p30f;
constexpr float SPAN = 0x1p20f;
constexpr float FAR = -4.f * SPAN;       // of m c
constexpr float SCALE_LO = 0x1p-8f, SCALE_HI = 0x1p8f;

static_assert(GROUPS >= 2 * MAX_TOP, "the bound needs more groups than alternatives");
static_assert(NT % GROUPS == 0 && NT >= MAX_TOP * 8, "merge of eight parts in one go");

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// Total order of the alternatives: descending value, then ascending index.  +0 and -0 have one
// key, all NaNs another above every number.
__device__ __forceinline__ uint32_t order_key(float x)
{
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    if (k == 0xFFFFFFFFu) return __uint_as_float(0x7FC00000u);
    return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t item_key(float x, uint32_t idx)
{
    return (static_cast<uint64_t>(order_key(x)) << 32) | (0xFFFFFFFFu - idx);
}

// Two fp32 numbers in one register pair.
__device__ __forceinline__ uint64_t pair(float a, float b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void unpair(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t ex2_2(uint64_t v)
{
    float a, b;
    unpair(v, a, b);
    return pair(ex2(a), ex2(b));
}

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int E = 4;
    template <bool NC> __device__ static float get(const float *p) { return NC ? __ldg(p) : *p; }
    // clamp at FLOOR (NaN stays) and return the largest entry (NaN ignored)
    __device__ static float clamp_max(uint32_t (&w)[4])
    {
        float m = FLOOR;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = max_nan(__uint_as_float(w[i]), FLOOR);
            w[i] = __float_as_uint(x);
            m = fmaxf(m, x);
        }
        return m;
    }
    __device__ static float at(const uint32_t (&w)[4], int e) { return __uint_as_float(w[e]); }
    __device__ static uint64_t two(const uint32_t (&w)[4], int i) { return pair(at(w, 2 * i), at(w, 2 * i + 1)); }
    // the same for an e that is not known to the compiler
    __device__ static float pick(const uint32_t (&w)[4], int e)
    {
        const uint32_t a = e & 1 ? w[1] : w[0], b = e & 1 ? w[3] : w[2];
        return __uint_as_float(e & 2 ? b : a);
    }
    static constexpr uint32_t NEG_INF = 0xFF800000u;
    __device__ static void put(uint32_t (&w)[4], int e, float x) { w[e] = __float_as_uint(x); }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int E = 8;
    template <bool NC> __device__ static float get(const __nv_bfloat16 *p)
    {
        const unsigned short *b = reinterpret_cast<const unsigned short *>(p);
        const uint32_t u = NC ? __ldg(b) : *b;
        return __uint_as_float(u << 16);
    }
    __device__ static float clamp_max(uint32_t (&w)[4])
    {
        const uint32_t fl = __float_as_uint(FLOOR);
        const uint32_t f2 = fl | (fl >> 16);
        uint32_t m2 = f2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(w[i]) : "r"(w[i]), "r"(f2));
            asm("max.bf16x2 %0, %1, %2;" : "=r"(m2) : "r"(m2), "r"(w[i]));
        }
        return fmaxf(__uint_as_float(m2 << 16), __uint_as_float(m2 & 0xFFFF0000u));
    }
    __device__ static float at(const uint32_t (&w)[4], int e)
    {
        return __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    __device__ static uint64_t two(const uint32_t (&w)[4], int i) { return pair(at(w, 2 * i), at(w, 2 * i + 1)); }
    __device__ static float pick(const uint32_t (&w)[4], int e)
    {
        const uint32_t a = e & 2 ? w[1] : w[0], b = e & 2 ? w[3] : w[2], c = e & 4 ? b : a;
        return __uint_as_float(e & 1 ? c & 0xFFFF0000u : c << 16);
    }
    static constexpr uint32_t NEG_INF = 0xFF80FF80u;
    __device__ static void put(uint32_t (&w)[4], int e, float x)
    {
        const uint32_t b = __float_as_uint(x) >> 16;
        w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xFFFFu) | (b << 16) : (w[e >> 1] & 0xFFFF0000u) | b;
    }
};

// A row seen in 16-byte granules of memory: granule v holds the entries v E - lead .. v E - lead + E - 1,
// of which those in [0, vocab) exist.  NC: nothing writes the row while the kernel runs.
template <typename T, bool NC>
struct Row {
    const T *p;
    uint32_t vocab, lead, granules;
    __device__ Row(const T *p_, uint32_t vocab_) : p(p_), vocab(vocab_)
    {
        constexpr uint32_t E = Elem<T>::E;
        lead = static_cast<uint32_t>((reinterpret_cast<uintptr_t>(p_) & 15u) / sizeof(T));
        granules = static_cast<uint32_t>((static_cast<uint64_t>(vocab_) + lead + E - 1) / E);
    }
    // granules v .. v + n - 1 lie inside the row and below end
    __device__ __forceinline__ bool inside(uint32_t v, uint32_t n, uint32_t end) const
    {
        return v > 0 && v + n <= end && v + n < granules;
    }
    __device__ __forceinline__ const T *at(uint32_t v) const { return p + (static_cast<int64_t>(v) * Elem<T>::E - lead); }
    // a whole granule
    __device__ __forceinline__ static void load_at(const T *q, uint32_t (&w)[4])
    {
        if (NC) {
            asm("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(q));
        } else {
            const uint4 x = *reinterpret_cast<const uint4 *>(q);
            w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        }
    }
    // entries of granule v; those that do not exist read as -inf
    __device__ __forceinline__ void load(uint32_t v, uint32_t end, uint32_t (&w)[4]) const
    {
        constexpr int E = Elem<T>::E;
        const int64_t first = static_cast<int64_t>(v) * E - lead;
        if (v < end && first >= 0 && first + E <= vocab) {
            load_at(p + first, w);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Elem<T>::NEG_INF;
        if (v >= end) return;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (first + e >= 0 && first + e < vocab) Elem<T>::put(w, e, Elem<T>::template get<NC>(p + first + e));
    }
};

struct Part {                            // softmax statistics of some entries, against S = m c rounded
    float m, s, q;
};
// (shift, to: S of a.m and of m)
__device__ __forceinline__ void raise(Part &a, float shift, float m, float to)
{
    const float d = shift - to, f = ex2(d);
    a.q = f * __fmaf_rn(d, a.s, a.q);
    a.s = f * a.s;
    a.m = m;
}
// The statistics of the first `width` lanes together (width a power of two; the lanes beyond repeat them),
// in every lane: their maximum first, so that each is raised once.
__device__ __forceinline__ Part join_lanes(Part a, float c, uint32_t width)
{
    float m = a.m;
    for (uint32_t o = 1; o < width; o *= 2) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    raise(a, __fmul_rn(a.m, c), m, __fmul_rn(m, c));
    for (uint32_t o = 1; o < width; o *= 2) {
        a.s += __shfl_xor_sync(0xFFFFFFFFu, a.s, o);
        a.q += __shfl_xor_sync(0xFFFFFFFFu, a.q, o);
    }
    return a;
}

struct Shared {
    Part part[WARPS];
    Part cta;                            // this CTA's part of the row
    int fast;
    alignas(16) float tmax[NT];
    float bound;
    uint32_t n_list;
    uint64_t list[LIST];                 // item keys of the entries that reach the bound
    uint64_t top[MAX_TOP];               // this CTA's alternatives, sorted; 0: none
    uint64_t merged[MAX_TOP * 8];
    uint64_t final_top[MAX_TOP];
    uint32_t warp_u32[WARPS];
};

// The k-th largest of the GROUPS group maxima (thread t is of group t mod GROUPS): at least k
// entries are not below it.  Every thread returns the bound.
__device__ float group_bound(Shared &sh, float tm, uint32_t k)
{
    const int t = threadIdx.x;
    sh.tmax[t] = tm;
    __syncthreads();
    float g = 0.f;
    if (t < GROUPS) {
        g = sh.tmax[t];
#pragma unroll
        for (int o = GROUPS; o < NT; o += GROUPS) g = fmaxf(g, sh.tmax[t + o]);
    }
    __syncthreads();
    if (t < GROUPS) sh.tmax[t] = g;
    __syncthreads();
    if (t < GROUPS) {
        uint32_t rank = 0;
#pragma unroll
        for (int j = 0; j < GROUPS; j += 4) {
            const float4 o = *reinterpret_cast<const float4 *>(sh.tmax + j);
            rank += (o.x > g || (o.x == g && j < t)) ? 1u : 0u;
            rank += (o.y > g || (o.y == g && j + 1 < t)) ? 1u : 0u;
            rank += (o.z > g || (o.z == g && j + 2 < t)) ? 1u : 0u;
            rank += (o.w > g || (o.w == g && j + 3 < t)) ? 1u : 0u;
        }
        if (rank == k - 1) sh.bound = g;
    }
    __syncthreads();
    return sh.bound;
}

// Fill out[have .. want) with the largest entries of [lo, hi) whose order key is below `below`,
// by descending value and ascending index: per distinct value one pass that finds it and one,
// ended early, that collects its indices in order.  For what the candidate list cannot hold.
template <typename T>
__device__ void top_by_passes(Shared &sh, const T *row, uint32_t lo, uint32_t hi, uint64_t below,
                              uint32_t have, uint32_t want, uint64_t *out)
{
    const int t = threadIdx.x, lane = t & 31, wid = t >> 5;
    while (have < want) {
        uint32_t best = 0;
        bool found = false;
        for (uint64_t j = static_cast<uint64_t>(lo) + t; j < hi; j += NT) {
            const uint32_t k = order_key(Elem<T>::template get<true>(row + j));
            if (k < below && (!found || k > best)) { best = k; found = true; }
        }
        // order keys of numbers and NaN are never 0 (that would be a NaN's bit pattern)
        best = __reduce_max_sync(0xFFFFFFFFu, found ? best : 0u);
        if (lane == 0) sh.warp_u32[wid] = best;
        __syncthreads();
        best = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) best = max(best, sh.warp_u32[w]);
        __syncthreads();
        if (best == 0) break;                                    // nothing left
        for (uint64_t base = lo; base < hi && have < want; base += NT) {
            const uint64_t j = base + t;
            const bool hit = j < hi && order_key(Elem<T>::template get<true>(row + j)) == best;
            const uint32_t b = __ballot_sync(0xFFFFFFFFu, hit);
            if (lane == 0) sh.warp_u32[wid] = __popc(b);
            __syncthreads();
            uint32_t before = 0, total = 0;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const uint32_t n = sh.warp_u32[w];
                before += w < wid ? n : 0u;
                total += n;
            }
            const uint32_t at = have + before + __popc(b & ((1u << lane) - 1u));
            if (hit && at < want)
                out[at] = (static_cast<uint64_t>(best) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(j));
            have += total;
            __syncthreads();
        }
        below = best;
    }
    for (uint32_t i = have + t; i < want; i += NT) out[i] = 0;
    __syncthreads();
}

// out[0 .. k) = the k largest of keys[0 .. n) in descending order (distinct keys; 0 fills up)
__device__ void rank_into(const uint64_t *keys, uint32_t n, uint32_t k, uint64_t *out)
{
    for (uint32_t i = threadIdx.x; i < k; i += NT)
        if (i >= n) out[i] = 0;
    for (uint32_t i = threadIdx.x; i < n; i += NT) {
        const uint64_t a = keys[i];
        uint32_t rank = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) rank += keys[j] > a ? 1u : 0u;
        if (rank < k) out[rank] = a;
    }
    __syncthreads();
}

struct Args {
    const void *logits;
    uint64_t row_stride;
    uint32_t vocab, top;
    const int64_t *targets;
    float scale;
    int slow;                            // every row by the slow path (extreme scale)
    float *logprob, *entropy, *lse;
    uint32_t *top_idx;
    float *top_logprob;
};

template <typename T, bool TOP, bool SPLIT>
__global__ void __launch_bounds__(NT)
logprobs_kernel(const Args a)
{
    constexpr int E = Elem<T>::E;
    __shared__ Shared sh;
    const int t = threadIdx.x, lane = t & 31, wid = t >> 5;
    uint32_t parts = 1, part = 0;
    uint64_t r = blockIdx.x;
    if (SPLIT) {
        parts = cg::this_cluster().num_blocks();
        part = cg::this_cluster().block_rank();
        r = blockIdx.x / parts;
    }
    const T *row = static_cast<const T *>(a.logits) + r * a.row_stride;
    const Row<T, true> R(row, a.vocab);
    const uint32_t v0 = static_cast<uint32_t>(static_cast<uint64_t>(R.granules) * part / parts);
    const uint32_t v1 = static_cast<uint32_t>(static_cast<uint64_t>(R.granules) * (part + 1) / parts);
    const float c = a.scale * LOG2E;

    // the target's logit, wanted at the end
    int64_t tgt = -1;
    float x_tgt = 0.f;
    if (t == 0 && part == 0 && a.targets) {
        tgt = a.targets[r];
        if (tgt >= 0 && tgt < a.vocab) x_tgt = Elem<T>::template get<true>(row + tgt);
    }

    // ---- one pass over this CTA's granules
    Part my = {FLOOR, 0.f, 0.f};
    if (TOP && t == 0) sh.n_list = 0;
    uint32_t w[UNROLL][4];
    if (!a.slow) {
        // the next batch of a thread is under way while it works on one
        uint32_t next[UNROLL][4];
        auto fetch = [&](uint32_t vb) {
            if (R.inside(vb, NT * UNROLL, v1)) {
                const T *q = R.at(vb + t);
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) R.load_at(q + u * NT * E, next[u]);
            } else {
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) R.load(vb + u * NT + t, v1, next[u]);
            }
        };
        fetch(v0);
        const uint64_t c2 = pair(c, c);
        float mc = __fmul_rn(my.m, c);
        for (uint32_t vb = v0; vb < v1; vb += NT * UNROLL) {
            float bm = FLOOR;
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[u][i] = next[u][i];
                bm = fmaxf(bm, Elem<T>::clamp_max(w[u]));
            }
            if (vb + NT * UNROLL < v1) fetch(vb + NT * UNROLL);
            if (bm > my.m) {
                const float to = __fmul_rn(bm, c);
                raise(my, mc, bm, to);
                mc = to;
            }
            const float from = mc < FAR ? 0.f : -mc;             // masked entries alone so far: weights 0
            const uint64_t shift = pair(from, from);
            uint64_t s = pair(my.s, 0.f), q = pair(my.q, 0.f);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int i = 0; i < E / 2; ++i) {
                    const uint64_t tt = fma2(Elem<T>::two(w[u], i), c2, shift);
                    const uint64_t p = ex2_2(tt);
                    s = add2(s, p);
                    q = fma2(p, tt, q);
                }
            float s1, q1;
            unpair(s, my.s, s1);
            unpair(q, my.q, q1);
            my.s += s1;
            my.q += q1;
        }
    }

    // ---- alternatives of this CTA's part
    if (TOP && !a.slow) {
        const uint32_t k = a.top;
        const float bound = group_bound(sh, my.m, k);
        // the entries of the threads that reach it
        auto list_hits = [&](const uint32_t (&g)[4], uint32_t v) {
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = Elem<T>::at(g, e);
                hits |= x >= bound && x > FLOOR ? 1u << e : 0u;
            }
            for (; hits; hits &= hits - 1) {
                const int e = __ffs(hits) - 1;
                const uint32_t at = atomicAdd(&sh.n_list, 1u);
                if (at < LIST) sh.list[at] = item_key(Elem<T>::pick(g, e), v * E + e - R.lead);
            }
        };
        const bool one_batch = v1 - v0 <= NT * UNROLL;           // a thread still holds all of its own
        if (one_batch && v1 > v0 && my.m >= bound) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) list_hits(w[u], v0 + u * NT + t);
        }
        constexpr int AT_ONCE = 4;                               // of these threads, so that their reads overlap
        for (uint32_t who = __ballot_sync(0xFFFFFFFFu, !one_batch && my.m >= bound && my.m > FLOOR); who;) {
            uint32_t first[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                first[j] = who ? v0 + wid * 32 + __ffs(who) - 1 + lane * NT : v1;
                who &= who - 1;
            }
            for (uint32_t step = 0; v0 + step < v1; step += 32 * NT) {
                uint32_t g[AT_ONCE][4];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) R.load(first[j] + step, v1, g[j]);
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) list_hits(g[j], first[j] + step);
            }
        }
        __syncthreads();
        const uint32_t lo = v0 == 0 ? 0u : v0 * E - R.lead;
        const uint32_t hi = v1 == R.granules ? a.vocab : v1 * E - R.lead;
        const uint32_t listed = sh.n_list, want = min(k, hi - lo);
        if (listed > LIST) {                                     // ties without end, or one thread's entries above all others
            top_by_passes<T>(sh, row, lo, hi, 1ull << 32, 0, want, sh.top);
        } else {
            rank_into(sh.list, listed, k, sh.top);
            if (listed < want)                                   // fewer than k entries above FLOOR
                top_by_passes<T>(sh, row, lo, hi, listed ? sh.top[listed - 1] >> 32 : 1ull << 32, listed, want, sh.top);
        }
        for (uint32_t i = t; i < k; i += NT)
            if (i >= hi - lo) sh.top[i] = 0;
    }

    // ---- this CTA's statistics
    my = join_lanes(my, c, 32);
    if (lane == 0) sh.part[wid] = my;
    __syncthreads();
    Part all = {};
    if (wid == 0) all = join_lanes(sh.part[lane & (WARPS - 1)], c, WARPS);
    const uint64_t *top = sh.top;
    if (SPLIT) {
        cg::cluster_group cl = cg::this_cluster();
        if (t == 0) sh.cta = all;
        cl.sync();
        if (part == 0) {
            if (wid == 0) {
                // lane o: part o's statistics (lanes from `parts` on repeat them)
                all = join_lanes(cl.map_shared_rank(&sh, lane & (parts - 1))->cta, c, parts);
            }
            if (TOP) {
                const uint32_t n = parts * a.top;
                for (uint32_t i = t; i < n; i += NT)
                    sh.merged[i] = cl.map_shared_rank(&sh, i / a.top)->top[i % a.top];
            }
        }
        cl.sync();                                               // the others may leave
        if (part != 0) return;
        if (TOP) {
            // sorted lists: an entry's place is its place in its own list and the number of larger ones in the others
            const uint32_t n = parts * a.top;
            for (uint32_t i = t; i < n; i += NT) {
                const uint64_t x = sh.merged[i];
                const uint32_t own = i / a.top;
                uint32_t rank = i - own * a.top;
#pragma unroll
                for (uint32_t o = 0; o < 8; ++o) {
                    if (o >= parts || o == own) continue;
                    uint32_t n_larger = 0;                       // binary search in a descending list
#pragma unroll
                    for (uint32_t step = MAX_TOP; step > 0; step /= 2)
                        if (n_larger + step <= a.top && sh.merged[o * a.top + n_larger + step - 1] > x) n_larger += step;
                    rank += n_larger;
                }
                if (x != 0 && rank < a.top) sh.final_top[rank] = x;     // (0: an empty place; vocab >= top entries exist)
            }
            __syncthreads();
            top = sh.final_top;
        }
    }

    // ---- the row's results
    // warp 0 holds the statistics; the slow path takes every warp
    if (t == 0) sh.fast = !a.slow && fabsf(all.m * c) < SPAN && all.s < INFINITY;
    __syncthreads();
    const bool fast = sh.fast != 0;
    if (fast && wid != 0) return;
    float lse, entropy, lp, zm, zs, logz;
    bool empty = false;
    if (fast) {
        zs = c;
        zm = __fmul_rn(all.m, c);
        logz = log2f(all.s);
        lse = __fmaf_rn(all.m, a.scale, LN2 * (logz - __fmaf_rn(all.m, c, -zm)));
        entropy = fmaxf(LN2 * (logz - __fdiv_rn(all.q, all.s)), 0.f);
    } else {
        // NaN, infinities, rows of masked entries only, extreme scales: two plain passes of the
        // row by this CTA, maximum first.  (scale and differences apart, so that nothing overflows early.)
        float m = -INFINITY;
        bool nan = false;
        for (uint64_t j = t; j < a.vocab; j += NT) {
            const float x = Elem<T>::template get<true>(row + j);
            m = fmaxf(m, x);
            nan |= x != x;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        nan = __syncthreads_or(nan);
        if (lane == 0) sh.part[wid].m = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) m = fmaxf(m, sh.part[w].m);
        __syncthreads();
        empty = !nan && m == -INFINITY;
        nan |= m == INFINITY;
        float s = 0.f, q = 0.f;
        if (!nan && !empty)
            for (uint64_t j = t; j < a.vocab; j += NT) {
                const float d = fmaxf((Elem<T>::template get<true>(row + j) - m) * a.scale, -1e30f);
                const float p = expf(d);
                s += p;
                q = __fmaf_rn(p, d, q);
            }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
        }
        if (lane == 0) { sh.part[wid].s = s; sh.part[wid].q = q; }
        __syncthreads();
        s = q = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { s += sh.part[w].s; q += sh.part[w].q; }
        const float bad = __uint_as_float(0x7FC00000u);
        zs = a.scale;
        zm = m;                                                  // subtracted before the scale
        logz = logf(s);
        lse = nan ? bad : empty ? -INFINITY : __fmaf_rn(m, a.scale, logz);
        entropy = nan ? bad : empty ? 0.f : fmaxf(logz - __fdiv_rn(q, s), 0.f);
        if (nan) logz = bad;
        if (TOP) {
            top_by_passes<T>(sh, row, 0, a.vocab, 1ull << 32, 0, a.top, sh.top);
            top = sh.top;
        }
    }
    auto log_p = [&](float x) {
        if (empty) return -INFINITY;
        if (fast && x < FLOOR) return (x - all.m) * a.scale - LN2 * logz;   // x c might overflow
        if (fast) return LN2 * (__fmaf_rn(x, zs, -zm) - logz);
        return (x - zm) * zs - logz;
    };
    if (t == 0) {
        if (tgt < 0) lp = 0.f;
        else if (tgt >= a.vocab) lp = __uint_as_float(0x7FC00000u);
        else lp = log_p(x_tgt);
        if (a.logprob) a.logprob[r] = lp;
        if (a.entropy) a.entropy[r] = entropy;
        if (a.lse) a.lse[r] = lse;
    }
    if (TOP)
        for (uint32_t i = t; i < a.top; i += NT) {               // (top <= 32: warp 0)
            const uint32_t idx = 0xFFFFFFFFu - static_cast<uint32_t>(top[i]);
            a.top_idx[r * a.top + i] = idx;
            a.top_logprob[r * a.top + i] = log_p(key_value(static_cast<uint32_t>(top[i] >> 32)));
        }
}

// ------------------------------------------------------------------------------ gradient

struct GradArgs {
    const void *logits;
    void *grad;
    uint64_t row_stride, grad_stride;
    uint32_t vocab, top, chunks;
    const int64_t *targets;
    float scale;
    float c, c_rest;                     // scale log2(e) rounded, and c / scale - LOG2E (a division per thread cost 12 %)
    const float *lse, *entropy, *g_logprob, *g_entropy;
    const uint32_t *top_idx;
    const float *g_top;
};

template <typename T> __device__ __forceinline__ void put_entry(T *p, float x);
template <> __device__ __forceinline__ void put_entry<float>(float *p, float x) { *p = x; }
template <> __device__ __forceinline__ void put_entry<__nv_bfloat16>(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }

// The g's of the token idx: the target's, and those of this warp's alternatives, lane i holding the i-th
__device__ __forceinline__ float own_gradient(uint32_t idx, uint32_t tgt, float g_t, float g_i, uint32_t top)
{
    float own = (idx != 0xFFFFFFFFu && idx == tgt) ? g_t : 0.f;
    for (uint32_t j = 0; j < top; ++j) {
        const uint32_t oj = __shfl_sync(0xFFFFFFFFu, idx, j);
        const float gj = __shfl_sync(0xFFFFFFFFu, g_i, j);
        if (oj == idx) own += gj;
    }
    return own;
}

// Rows with |lse| log2(e) >= SPAN or an infinite lse: masked by finite values alone, logits of 10^6 and more,
// nothing but -inf.  An fp32 number of that size does not hold the log of the number of tokens (at -10^9
// its spacing is 64), so exp(z - lse) may be 1 for every one of them.  One CTA does the whole row, in
// three plain passes like the forward's slow path: maximum, sum, gradient.  (All others of the row leave it alone, so it
// may be done in place.)  8192 x 50257 bf16, all rows of this kind: 980 us, against 284 with lse.
template <typename T>
struct WholeRow {
    const T *row;
    T *out;
    uint32_t vocab;
    float scale;
    uint32_t tgt;
    float g_t, total, g_h, h;
    uint32_t top, idx;                   // of this lane's alternative
    float g_i;
};
template <typename T>
__device__ __noinline__ void grad_anew(const WholeRow<T> w)
{
    __shared__ float part[WARPS];
    const int t = threadIdx.x, lane = t & 31, wid = t >> 5;
    auto at = [&](uint64_t j) { return Elem<T>::template get<false>(w.row + j); };
    const float x_i = w.idx != 0xFFFFFFFFu ? at(w.idx) : 0.f;    // (read before the first barrier)
    float m = -INFINITY;
    for (uint64_t j = t; j < w.vocab; j += NT) m = fmaxf(m, at(j));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if (lane == 0) part[wid] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) m = fmaxf(m, part[i]);
    __syncthreads();
    if (m == -INFINITY) {
        for (uint64_t j = t; j < w.vocab; j += NT) put_entry<T>(w.out + j, 0.f);
        return;
    }
    auto below_max = [&](float x) { return max_nan((x - m) * w.scale, -1e30f); };
    float s = 0.f;
    for (uint64_t j = t; j < w.vocab; j += NT) s += expf(below_max(at(j)));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) part[wid] = s;
    __syncthreads();
    s = 0.f;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) s += part[i];
    const float logz = logf(s);
    auto gradient = [&](float x, float own) {
        const float d = max_nan(below_max(x) - logz, -1e6f);
        return w.scale * (own - expf(d) * __fmaf_rn(w.g_h, d + w.h, w.total));
    };
    for (uint64_t j = t; j < w.vocab; j += NT) put_entry<T>(w.out + j, gradient(at(j), j == w.tgt ? w.g_t : 0.f));
    if (w.top) {
        __syncthreads();
        if (wid == 0) {
            const float own = own_gradient(w.idx, w.tgt, w.g_t, w.g_i, w.top);
            if (w.idx != 0xFFFFFFFFu) put_entry<T>(w.out + w.idx, gradient(x_i, own));
        }
    }
}

// One CTA per chunk of a row: entries are read and written once, 16 bytes at a time, with the softmax
// from the saved lse.  The target's term is added by the thread that holds its granule.  The
// alternatives' entries are few: warp 0 reads their logits first (the gradient may lie in the
// logits' place) and writes them over at the end, the terms of equal tokens added in a fixed order.
// ENT: there is a gradient of the entropy.
// Bound by memory: 8192 rows of 50257 bf16 in 290 us, 5.7 TB/s (when four granules per thread took 296, two took
// 340 and eight 304).
template <typename T, int U, bool ENT>
__global__ void __launch_bounds__(NT)
logprobs_grad_kernel(const GradArgs a)
{
    constexpr int E = Elem<T>::E;
    const int t = threadIdx.x, lane = t & 31;
    const uint64_t r = blockIdx.x / a.chunks;
    const uint32_t chunk = blockIdx.x % a.chunks;
    const T *row = static_cast<const T *>(a.logits) + r * a.row_stride;
    T *out = static_cast<T *>(a.grad) + r * a.grad_stride;
    const Row<T, false> R(row, a.vocab);
    const uint64_t v0 = static_cast<uint64_t>(chunk) * (NT * U);
    const uint32_t end = R.granules;
    if (v0 >= end) return;

    const float lse = a.lse[r];
    const int64_t tgt64 = a.g_logprob ? a.targets[r] : -1;
    const float bad = __uint_as_float(0x7FC00000u);
    const float g_t = tgt64 < 0 ? 0.f : tgt64 >= a.vocab ? bad : a.g_logprob[r];
    const uint32_t tgt = tgt64 < 0 || tgt64 >= a.vocab ? 0xFFFFFFFFu : static_cast<uint32_t>(tgt64);
    const float g_h = a.g_entropy ? a.g_entropy[r] : 0.f;
    const float h = a.g_entropy ? a.entropy[r] : 0.f;
    float total = g_t;
    uint32_t idx = 0xFFFFFFFFu;
    float g_i = 0.f;
    if (a.top) {
        if (lane < static_cast<int>(a.top)) {
            idx = a.top_idx[r * a.top + lane];
            if (idx < a.vocab) g_i = a.g_top[r * a.top + lane];
            else idx = 0xFFFFFFFFu;
        }
        float s = g_i;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        total += s;
    }
    // In full, for any scale: d = log p.
    auto careful = [&](float x, float own_g) {
        const float d = max_nan(__fmaf_rn(x, a.scale, -lse), -1e6f);
        const float p = ex2(d * LOG2E);
        const float u = p * __fmaf_rn(g_h, d + h, total);
        return a.scale * (own_g - u);
    };
    // For lse and scale in the usual range: p = f 2^t, t = x c - L, where L is lse log2(e) rounded and
    // f = 2^-rest.  rest is what lse / scale times c, c as rounded, has over L: an error of c then acts on
    // x - lse / scale, which is small where p is not, instead of on x and lse apart.
    // log p + entropy = ln2 t + (entropy - ln2 rest).  So an entry is
    // 2^t (A t + B), or 2^t B without the entropy's term; logits below FLOOR count as FLOOR there (p = 0).
    const float c = a.c, big = lse * LOG2E;
    const float rest = __fmaf_rn(lse, LOG2E, -big) + lse * a.c_rest;
    const float f = -a.scale * ex2(-rest);
    const float coef_a = f * g_h * LN2, coef_b = f * __fmaf_rn(g_h, h - LN2 * rest, total);
    const bool in_span = fabsf(big) < SPAN;
    if (!in_span && lse == lse) {                                // (a NaN goes on, and into every entry)
        if (chunk == 0)
            grad_anew<T>({row, out, a.vocab, a.scale, tgt, g_t, total, g_h, h, a.top, idx, g_i});
        return;
    }
    const bool usual = in_span && a.scale >= SCALE_LO && a.scale <= SCALE_HI;
    // the alternatives in this chunk
    float x_i = 0.f;
    bool mine = false;
    if (a.top && t < 32) {
        const uint64_t v = (static_cast<uint64_t>(idx) + R.lead) / E;
        mine = idx != 0xFFFFFFFFu && v >= v0 && v < v0 + NT * U;
        if (mine) x_i = Elem<T>::template get<false>(row + idx);
    }
    if (a.top) __syncthreads();
    const uint32_t vt = tgt == 0xFFFFFFFFu ? 0xFFFFFFFFu : static_cast<uint32_t>((static_cast<uint64_t>(tgt) + R.lead) / E);
    const bool same_phase = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    uint32_t w[U][4];
    const uint32_t vb = static_cast<uint32_t>(v0);
    const bool whole = R.inside(vb, NT * U, end);
    if (whole) {
        const T *q = R.at(vb + t);
#pragma unroll
        for (int u = 0; u < U; ++u) R.load_at(q + u * NT * E, w[u]);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) R.load(vb + u * NT + t, end, w[u]);
    }
    const uint64_t c2 = pair(c, c), shift = pair(-big, -big), a2 = pair(coef_a, coef_a), b2 = pair(coef_b, coef_b);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t v = vb + u * NT + t;
        if (!whole && v >= end) continue;
        uint64_t y[E / 2];
        if (usual) {
            if (ENT) Elem<T>::clamp_max(w[u]);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const uint64_t tt = fma2(Elem<T>::two(w[u], i), c2, shift);
                const uint64_t p = ex2_2(tt);
                y[i] = mul2(p, ENT ? fma2(tt, a2, b2) : b2);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) y[i] = pair(careful(Elem<T>::at(w[u], 2 * i), 0.f), careful(Elem<T>::at(w[u], 2 * i + 1), 0.f));
        }
        const int64_t first = static_cast<int64_t>(v) * E - R.lead;
        if (v == vt) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float y0, y1;
                unpair(y[i], y0, y1);
                y0 += first + 2 * i == tgt ? a.scale * g_t : 0.f;
                y1 += first + 2 * i + 1 == tgt ? a.scale * g_t : 0.f;
                y[i] = pair(y0, y1);
            }
        }
        if (same_phase && (whole || (first >= 0 && first + E <= a.vocab))) {
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float y0, y1;
                unpair(y[i], y0, y1);
                if (E == 4) {
                    o[2 * i % 4] = __float_as_uint(y0);
                    o[(2 * i + 1) % 4] = __float_as_uint(y1);
                } else {
                    const __nv_bfloat162 b = __floats2bfloat162_rn(y0, y1);
                    o[i] = *reinterpret_cast<const uint32_t *>(&b);
                }
            }
            asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};"
                         :: "l"(out + first), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float yy[2];
                unpair(y[i], yy[0], yy[1]);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int64_t e = first + 2 * i + j;
                    if (e >= 0 && e < a.vocab) put_entry<T>(out + e, yy[j]);
                }
            }
        }
    }
    if (a.top) {
        __syncthreads();
        if (t < 32) {
            const float own = own_gradient(idx, tgt, g_t, g_i, a.top);
            if (mine) put_entry<T>(out + idx, careful(x_i, own));
        }
    }
}

int sm_count()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 0;
    return n;
}

template <typename T, bool TOP>
cudaError_t launch_forward(const Args &a, uint64_t rows, uint32_t parts, cudaStream_t s)
{
    if (parts == 1) {
        logprobs_kernel<T, TOP, false><<<static_cast<unsigned>(rows), NT, 0, s>>>(a);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * parts));
    cfg.blockDim = dim3(NT);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = parts;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, logprobs_kernel<T, TOP, true>, a);
    if (err != cudaSuccess) cudaGetLastError();                  // (pending, it would be taken for the next call's)
    return err;
}

template <typename T>
void launch_grad(const GradArgs &a, unsigned grid, bool small, cudaStream_t s)
{
    const bool ent = a.g_entropy != nullptr;
    if (small && ent) logprobs_grad_kernel<T, 1, true><<<grid, NT, 0, s>>>(a);
    else if (small) logprobs_grad_kernel<T, 1, false><<<grid, NT, 0, s>>>(a);
    else if (ent) logprobs_grad_kernel<T, GRAD_UNROLL, true><<<grid, NT, 0, s>>>(a);
    else logprobs_grad_kernel<T, GRAD_UNROLL, false><<<grid, NT, 0, s>>>(a);
}

bool bad_shape(const void *logits, int32_t dtype, uint64_t rows, uint32_t vocab, uint64_t stride, float scale)
{
    const uintptr_t unit = dtype == DECO_F32 ? 4 : 2;
    return !logits || (dtype != DECO_F32 && dtype != DECO_BF16) || vocab == 0 || vocab > 0x7FFFFFFFu ||
           rows >= (1ull << 28) || stride < vocab || stride > (1ull << 40) || !(scale > 0.f) || scale > 3.0e38f ||
           (reinterpret_cast<uintptr_t>(logits) & (unit - 1)) != 0;
}

// an address that is no multiple of its entries' size would fault on the device (NULL is fine)
bool misaligned(std::initializer_list<const void *> words, const int64_t *targets)
{
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return true;
    return (reinterpret_cast<uintptr_t>(targets) & 7u) != 0;
}

}  // namespace

extern "C" deco_status deco_token_logprobs(const void *logits, int32_t dtype, uint64_t rows, uint32_t vocab,
                                           uint64_t row_stride, const int64_t *targets, float scale,
                                           float *logprob, float *entropy, float *lse, uint32_t top,
                                           uint32_t *top_idx, float *top_logprob, void *stream)
{
    if (top > DECO_LOGPROBS_MAX_TOP) return DECO_ERR_CAPACITY;
    if (top > vocab || (logprob && !targets)) return DECO_ERR_INVALID_ARG;
    if (rows == 0) return DECO_OK;
    if (bad_shape(logits, dtype, rows, vocab, row_stride, scale)) return DECO_ERR_INVALID_ARG;
    if (top && (!top_idx || !top_logprob)) return DECO_ERR_INVALID_ARG;
    if (!logprob && !entropy && !lse && !top) return DECO_ERR_INVALID_ARG;
    if (misaligned({logprob, entropy, lse, top_idx, top_logprob}, targets)) return DECO_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms == 0) return DECO_ERR_CUDA;
    Args a = {};
    a.logits = logits;
    a.row_stride = row_stride;
    a.vocab = vocab;
    a.top = top;
    a.targets = logprob ? targets : nullptr;
    a.scale = scale;
    a.slow = !(scale >= SCALE_LO && scale <= SCALE_HI);
    a.logprob = logprob;
    a.entropy = entropy;
    a.lse = lse;
    a.top_idx = top_idx;
    a.top_logprob = top_logprob;
    // (Measured, one row of 32000 bf16: 9.6 us a call with eight parts, 10.2 with one; 64 rows of 50257 f32: 12.3 and
    // 15.8; 1999 rows, which already fill the device: 53 with one part, 93 with two.)
    // A row is split while the CTAs do not fill the device and every part still has half a batch
    // of loads for each of its threads.
    const uint64_t batch = static_cast<uint64_t>(NT) * UNROLL * (dtype == DECO_F32 ? 4 : 8);
    uint32_t parts = 1;
    while (parts < 8 && rows * parts * 2 <= 4ull * sms && vocab >= parts * batch) parts *= 2;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t err;
    if (dtype == DECO_F32)
        err = top ? launch_forward<float, true>(a, rows, parts, s) : launch_forward<float, false>(a, rows, parts, s);
    else
        err = top ? launch_forward<__nv_bfloat16, true>(a, rows, parts, s)
                  : launch_forward<__nv_bfloat16, false>(a, rows, parts, s);
    return err == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}

extern "C" deco_status deco_token_logprobs_grad(const void *logits, int32_t dtype, uint64_t rows, uint32_t vocab,
                                                uint64_t row_stride, const int64_t *targets, float scale,
                                                const float *lse, const float *entropy, const float *g_logprob,
                                                const float *g_entropy, uint32_t top, const uint32_t *top_idx,
                                                const float *g_top, void *grad, uint64_t grad_row_stride,
                                                void *stream)
{
    if (top > DECO_LOGPROBS_MAX_TOP) return DECO_ERR_CAPACITY;
    if (rows == 0) return DECO_OK;
    if (bad_shape(logits, dtype, rows, vocab, row_stride, scale) ||
        bad_shape(grad, dtype, rows, vocab, grad_row_stride, scale))
        return DECO_ERR_INVALID_ARG;
    if (!lse || (g_logprob && !targets) || (g_entropy && !entropy) || (top && (!top_idx || !g_top)))
        return DECO_ERR_INVALID_ARG;
    if (misaligned({lse, entropy, g_logprob, g_entropy, top_idx, g_top}, targets)) return DECO_ERR_INVALID_ARG;
    if (grad == logits && grad_row_stride != row_stride) return DECO_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms == 0) return DECO_ERR_CUDA;
    GradArgs a = {};
    a.logits = logits;
    a.grad = grad;
    a.row_stride = row_stride;
    a.grad_stride = grad_row_stride;
    a.vocab = vocab;
    a.top = top;
    a.targets = targets;
    a.scale = scale;
    a.c = scale * LOG2E;
    a.c_rest = static_cast<float>(static_cast<double>(a.c) / scale - static_cast<double>(LOG2E));
    a.lse = lse;
    a.entropy = entropy;
    a.g_logprob = g_logprob;
    a.g_entropy = g_entropy;
    a.top_idx = top_idx;
    a.g_top = g_top;
    // Short calls take one granule per thread, so that they spread over more SMs.
    const uint64_t per = dtype == DECO_F32 ? 4 : 8;
    const uint64_t granules = (static_cast<uint64_t>(vocab) + 2 * per - 2) / per;
    const bool small = rows * granules <= 4ull * sms * NT * GRAD_UNROLL;
    const uint64_t span = static_cast<uint64_t>(NT) * (small ? 1 : GRAD_UNROLL);
    const uint64_t chunks = (granules + span - 1) / span;
    if (rows * chunks > 0x7FFFFFFFull) return DECO_ERR_INVALID_ARG;
    a.chunks = static_cast<uint32_t>(chunks);
    const unsigned grid = static_cast<unsigned>(rows * chunks);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == DECO_F32) launch_grad<float>(a, grid, small, s);
    else launch_grad<__nv_bfloat16>(a, grid, small, s);
    return cudaGetLastError() == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}
