// deco_layernorm, deco_layernorm_grad, deco_pack8, deco_unpack8: layer norm with its gradient, and
// activations put away in 8 bits.
//
// All four are bound by memory.  A row belongs to a group of warps.  A thread owns the same columns of every row of its
// group: item i of thread t holds the V columns from (i * threads + t) * V.  V = 8 where every row of every
// array starts on 16 bytes and the width is a multiple of 8 (16-byte accesses), V = 1 otherwise (any alignment, any
// stride; consecutive lanes hold consecutive columns).  Either way a block of 32 columns lies in one warp.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "deco.h"
#include "deco_packed8.h"

namespace {

using deco::BLOCK8;

constexpr uint32_t FULL = 0xFFFFFFFFu;

// ----------------------------------------------------------------------------- entries

// `n` consecutive entries as fp32: V = 8 with 16-byte accesses, V = 1 with one of the entry's size.
template <int V> __device__ __forceinline__ void get(const float *p, float (&v)[V])
{
    if (V == 1) {
        v[0] = *p;
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const float4 w = reinterpret_cast<const float4 *>(p)[i];
            v[4 * i] = w.x; v[4 * i + 1] = w.y; v[4 * i + 2] = w.z; v[4 * i + 3] = w.w;
        }
    }
}
template <int V> __device__ __forceinline__ void get(const __nv_bfloat16 *p, float (&v)[V])
{
    if (V == 1) {
        v[0] = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const unsigned short *>(p)) << 16);
    } else {
        const uint4 w = *reinterpret_cast<const uint4 *>(p);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
        }
    }
}
template <int V> __device__ __forceinline__ void put(float *p, const float (&v)[V])
{
    if (V == 1) {
        *p = v[0];
    } else {
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            reinterpret_cast<float4 *>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    }
}
template <int V> __device__ __forceinline__ void put(__nv_bfloat16 *p, const float (&v)[V])
{
    if (V == 1) {
        *p = __float2bfloat16_rn(v[0]);
    } else {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    }
}
__device__ __forceinline__ float rounded(float x, const float *) { return x; }
__device__ __forceinline__ float rounded(float x, const __nv_bfloat16 *) { return __bfloat162float(__float2bfloat16_rn(x)); }

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

// --------------------------------------------------------------------- 8-bit checkpoints

// Exponent byte of a block whose largest magnitude has the bits `top` (sign cleared): the smallest b >= 1 for
// which the magnitude, over 2^(b - 127), still rounds to at most 127.  With magnitude = f 2^(E - 127), f in [1, 2), that is b = E - 6,
// and one more from f = 127.5 / 64 on: there adding 2^16 to the bits carries into E.  255: a NaN or an infinity.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top)
{
    if (top >= 0x7F800000u) return 255u;
    const int b = static_cast<int>((top + 0x10000u) >> 23) - 6;
    return static_cast<uint32_t>(b < 1 ? 1 : b);
}
__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Store V entries (0 beyond the row's end) of a row's checkpoint; the warp together, `in` where there is something to
// store.  Products with a power of two are exact, so each code is rounded once.
template <int V>
__device__ __forceinline__ void put_packed(int8_t *codes, uint8_t *exps, uint32_t col, bool in, const float (&v)[V])
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) top = max(top, in ? magnitude_bits(v[j]) : 0u);
    if (V == 1) {
        top = __reduce_max_sync(FULL, top);
    } else {
        top = max(top, __shfl_xor_sync(FULL, top, 1));
        top = max(top, __shfl_xor_sync(FULL, top, 2));
    }
    if (!in) return;
    const uint32_t b = exponent_byte(top);
    const float inv = b == 255u ? 0.f : __uint_as_float((254u - b) << 23);
    // 64 of the largest step are 2^128, which is no fp32 number: 63 are kept there
    const int most = b == 249u ? 63 : 127;
    uint32_t q[V];
#pragma unroll
    for (int j = 0; j < V; ++j)                          // (a block that stands for NaN has codes of 0)
        q[j] = static_cast<uint32_t>(b == 255u ? 0 : max(-most, min(most, __float2int_rn(v[j] * inv)))) & 0xFFu;
    if (V == 1) {
        codes[col] = static_cast<int8_t>(q[0]);
    } else {
        uint32_t w[V / 4 + 1];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) w[i] = q[4 * i] | q[4 * i + 1] << 8 | q[4 * i + 2] << 16 | q[4 * i + 3] << 24;
        *reinterpret_cast<uint2 *>(codes + col) = make_uint2(w[0], w[1 % (V / 4 + 1)]);
    }
    if (col % BLOCK8 == 0) exps[col / BLOCK8] = static_cast<uint8_t>(b);
}

__device__ __forceinline__ float step_of(uint32_t b) { return __uint_as_float(b == 255u ? 0x7FC00000u : b << 23); }

// V entries of a row's checkpoint.
template <int V>
__device__ __forceinline__ void get_packed(const int8_t *codes, const uint8_t *exps, uint32_t col, float (&v)[V])
{
    const float step = step_of(exps[col / BLOCK8]);
    if (V == 1) {
        v[0] = static_cast<float>(codes[col]) * step;
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(codes + col);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t u = j < 4 ? w.x : w.y;
            v[j] = static_cast<float>(static_cast<int>(u << (24 - 8 * (j & 3))) >> 24) * step;
        }
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(256)
pack_kernel(const T *x, uint64_t stride, uint32_t cols, uint32_t chunks, uint64_t units, int8_t *codes, uint8_t *exps)
{
    // a unit is 32 * V consecutive columns of a row, a warp's
    const uint64_t unit = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (unit >= units) return;
    const uint64_t row = unit / chunks;
    const uint32_t col = static_cast<uint32_t>(unit - row * chunks) * (32 * V) + (threadIdx.x & 31) * V;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = 0.f;
    if (col < cols) get<V>(x + row * stride + col, v);
    put_packed<V>(codes + row * blocks * BLOCK8, exps + row * blocks, col, col < blocks * BLOCK8, v);
}

template <typename T, int V>
__global__ void __launch_bounds__(256)
unpack_kernel(const int8_t *codes, const uint8_t *exps, uint32_t cols, uint32_t chunks, uint64_t units, T *y, uint64_t stride)
{
    const uint64_t unit = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (unit >= units) return;
    const uint64_t row = unit / chunks;
    const uint32_t col = static_cast<uint32_t>(unit - row * chunks) * (32 * V) + (threadIdx.x & 31) * V;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    if (col >= cols) return;
    float v[V];
    get_packed<V>(codes + row * blocks * BLOCK8, exps + row * blocks, col, v);
    put<V>(y + row * stride + col, v);
}

// ------------------------------------------------------------------------------ layer norm

struct NormArgs {
    const void *x, *add;
    void *sum, *y;
    uint64_t x_stride, add_stride, sum_stride, y_stride, rows;
    const float *weight, *bias;
    float *mean, *rstd;
    int8_t *codes;
    uint8_t *exps;
    float eps;
    uint32_t cols, warps;                // warps of a row's group
};

// Statistics of the entries of some warp: count, mean, sum of squared deviations from it.
struct Moments {
    float n, mean, m2;
};

// Of a group of `warps` warps from their own, in every thread.  Means are joined as differences from the first, so that a
// common offset of the row costs no digits.
__device__ __forceinline__ Moments join(const Moments *m, uint32_t warps)
{
    const float base = m[0].mean;
    float n = 0.f, sum = 0.f;
    for (uint32_t w = 0; w < warps; ++w) {
        n += m[w].n;
        sum = __fmaf_rn(m[w].n, m[w].mean - base, sum);
    }
    const float off = sum / n;
    float m2 = 0.f;
    for (uint32_t w = 0; w < warps; ++w) {
        const float d = m[w].mean - base - off;
        m2 += __fmaf_rn(m[w].n * d, d, m[w].m2);
    }
    return {n, base + off, m2};
}

// One pass: the row stays in registers between its statistics and its output.  Deviations are summed from the warp's own
// mean, and what rounding did to that mean is taken back by their sum.
template <typename T, int V, int ITEMS, bool ADD, bool KEEP>
__global__ void __launch_bounds__(1024)
norm_kernel(const NormArgs a)
{
    __shared__ Moments moments[32];
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, group = wid / a.warps;
    const uint32_t threads = a.warps * 32, t = threadIdx.x - group * threads, cols = a.cols;
    const uint64_t row = static_cast<uint64_t>(blockIdx.x) * ((blockDim.x >> 5) / a.warps) + group;
    const bool live = row < a.rows;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *add = static_cast<const T *>(a.add) + row * a.add_stride;
    T *sum = static_cast<T *>(a.sum) + row * a.sum_stride;
    float v[ITEMS][V];
    float s = 0.f, n = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t col = (i * threads + t) * V;
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] = 0.f;
        if (live && col < cols) get<V>(x + col, v[i]);
    }
    if (ADD) {
        float w[ITEMS][V];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t col = (i * threads + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) w[i][j] = 0.f;
            if (live && col < cols) get<V>(add + col, w[i]);
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t col = (i * threads + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = rounded(v[i][j] + w[i][j], x);
            if (live && col < cols && a.sum) put<V>(sum + col, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t c0 = (i * threads + t - lane) * V;        // the warp's first column
        if (c0 < cols) n += static_cast<float>(min(cols - c0, 32u * V));
#pragma unroll
        for (int j = 0; j < V; ++j) s += v[i][j];
    }
    const float m = warp_sum(s) / fmaxf(n, 1.f);
    float d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        if ((i * threads + t) * V < cols) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = v[i][j] - m;
                d1 += d;
                d2 = __fmaf_rn(d, d, d2);
            }
        }
    }
    d1 = warp_sum(d1);
    d2 = warp_sum(d2);
    const float rest = d1 / fmaxf(n, 1.f);
    const float m2 = __fmaf_rn(-d1, rest, d2);
    Moments mo = {n, m + rest, m2 < 0.f ? 0.f : m2};             // (a NaN stays)
    if (a.warps > 1) {
        if (lane == 0) moments[wid] = mo;
        __syncthreads();
        mo = join(moments + group * a.warps, a.warps);
    }
    const float rstd = 1.f / sqrtf(mo.m2 / mo.n + a.eps);
    if (live && t == 0) {
        if (a.mean) a.mean[row] = mo.mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t col = (i * threads + t) * V;
        if (KEEP) put_packed<V>(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col, live && col < blocks * BLOCK8, v[i]);
        if (!live || col >= cols) continue;
        float w[V], b[V], o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            w[j] = 1.f;
            b[j] = 0.f;
        }
        if (a.weight) get<V>(a.weight + col, w);
        if (a.bias) get<V>(a.bias + col, b);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = __fmaf_rn((v[i][j] - mo.mean) * rstd, w[j], b[j]);
        put<V>(y + col, o);
    }
}

// Rows that do not fit the registers of 1024 threads: one CTA a row, which reads it once for its sum, once for its
// deviations and once for the output (the second and third time from the caches).
template <typename T>
__global__ void __launch_bounds__(1024)
norm_wide_kernel(const NormArgs a)
{
    __shared__ Moments moments[32];
    const uint32_t t = threadIdx.x, lane = t & 31, wid = t >> 5, cols = a.cols;
    const uint64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *add = a.add ? static_cast<const T *>(a.add) + row * a.add_stride : nullptr;
    T *sum = a.sum ? static_cast<T *>(a.sum) + row * a.sum_stride : nullptr;
    auto value = [&](uint32_t col) {
        float v[1], w[1];
        get<1>(x + col, v);
        if (!add) return v[0];
        get<1>(add + col, w);
        return rounded(v[0] + w[0], x);
    };
    // the sum may be stored over x or add: the output pass stores it, entry by entry
    float s = 0.f, n = 0.f;
    for (uint32_t col = t; col < cols; col += 1024) s += value(col);
    for (uint32_t c0 = wid * 32; c0 < cols; c0 += 1024) n += static_cast<float>(min(cols - c0, 32u));
    const float m = warp_sum(s) / n;
    float d1 = 0.f, d2 = 0.f;
    for (uint32_t col = t; col < cols; col += 1024) {
        const float d = value(col) - m;
        d1 += d;
        d2 = __fmaf_rn(d, d, d2);
    }
    d1 = warp_sum(d1);
    d2 = warp_sum(d2);
    const float rest = d1 / n;
    const float m2 = __fmaf_rn(-d1, rest, d2);
    if (lane == 0) moments[wid] = {n, m + rest, m2 < 0.f ? 0.f : m2};
    __syncthreads();
    const Moments mo = join(moments, 32);
    const float rstd = 1.f / sqrtf(mo.m2 / mo.n + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[row] = mo.mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    for (uint32_t col = t; col - lane < cols; col += 1024) {
        float v[1] = {0.f};
        if (col < cols) v[0] = value(col);
        if (a.codes) put_packed<1>(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col, col < blocks * BLOCK8, v);
        if (col >= cols) continue;
        if (sum) put<1>(sum + col, v);
        const float o[1] = {__fmaf_rn((v[0] - mo.mean) * rstd, a.weight ? a.weight[col] : 1.f, a.bias ? a.bias[col] : 0.f)};
        put<1>(y + col, o);
    }
}

// ---------------------------------------------------------------------------- its gradient

struct NormGradArgs {
    const void *x, *dy, *add;
    void *dx;
    const int8_t *codes;                 // x as a checkpoint, or null
    const uint8_t *exps;
    uint64_t x_stride, dy_stride, add_stride, dx_stride, rows;
    const float *mean, *rstd, *weight;
    float *parts;                        // [part][2][cols]: sums of dy xhat and of dy over some rows; null: not wanted
    float *c;                            // [rows][2] (wide rows)
    uint32_t cols, warps;
};

constexpr int E = 8;                     // entries of a row that a thread holds

template <typename T, int V>
__device__ __forceinline__ void get_row(const NormGradArgs &a, const void *base, uint64_t stride, uint64_t row, uint32_t t,
                                        uint32_t threads, float (&v)[E])
{
    const T *p = static_cast<const T *>(base) + row * stride;
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const uint32_t col = (i * threads + t) * V;
        float w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = 0.f;
        if (col < a.cols) get<V>(p + col, w);
#pragma unroll
        for (int j = 0; j < V; ++j) v[i * V + j] = w[j];
    }
}
template <typename T, int V, bool PACKED>
__device__ __forceinline__ void get_x(const NormGradArgs &a, uint64_t row, uint32_t t, uint32_t threads, float (&v)[E])
{
    if (!PACKED) {
        get_row<T, V>(a, a.x, a.x_stride, row, t, threads, v);
        return;
    }
    const uint32_t blocks = (a.cols + BLOCK8 - 1) / BLOCK8;
#pragma unroll
    for (int i = 0; i < E / V; ++i) {
        const uint32_t col = (i * threads + t) * V;
        float w[V];
#pragma unroll
        for (int j = 0; j < V; ++j) w[j] = 0.f;
        if (col < a.cols) get_packed<V>(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col, w);
#pragma unroll
        for (int j = 0; j < V; ++j) v[i * V + j] = w[j];
    }
}

// xhat = (x - mean) rstd, g = dy w;  dx = rstd (g - mean g - xhat mean(g xhat)) (+ add).  A group takes every
// (groups)th row, and each thread sums dy xhat and dy of its own columns over its rows in registers; the groups of
// a CTA are joined in shared memory in their order, the CTAs by sum_parts_kernel in theirs: the same bits every time.
template <typename T, int V, bool PACKED, bool ADD>
__global__ void __launch_bounds__(1024)
norm_grad_kernel(const NormGradArgs a)
{
    extern __shared__ float joined[];                            // [2][threads * E] of a row's group; groups > 1
    __shared__ float2 sums[2][32];
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, group = wid / a.warps, groups = (blockDim.x >> 5) / a.warps;
    const uint32_t threads = a.warps * 32, t = threadIdx.x - group * threads, cols = a.cols;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float w[E], dw[E], db[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const uint32_t col = V == 1 ? e * threads + t : t * V + e;
        w[e] = a.weight && col < cols ? a.weight[col] : 1.f;
        dw[e] = db[e] = 0.f;
    }
    const float inv = 1.f / static_cast<float>(cols);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * groups;
    uint32_t parity = 0;
    for (uint64_t row = static_cast<uint64_t>(blockIdx.x) * groups + group; row < a.rows; row += step) {
        float x[E], dy[E];
        get_x<T, V, PACKED>(a, row, t, threads, x);
        get_row<T, V>(a, a.dy, a.dy_stride, row, t, threads, dy);
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t col = V == 1 ? e * threads + t : t * V + e;
            x[e] = col < cols ? (x[e] - mean) * rstd : 0.f;
            dw[e] = __fmaf_rn(dy[e], x[e], dw[e]);
            db[e] += dy[e];
            dy[e] *= w[e];
            s1 += dy[e];
            s2 = __fmaf_rn(dy[e], x[e], s2);
        }
        s1 = warp_sum(s1);
        s2 = warp_sum(s2);
        if (a.warps > 1) {
            if (lane == 0) sums[parity][wid] = make_float2(s1, s2);
            asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "r"(threads) : "memory");
            s1 = s2 = 0.f;
            for (uint32_t i = 0; i < a.warps; ++i) {
                const float2 p = sums[parity][group * a.warps + i];
                s1 += p.x;
                s2 += p.y;
            }
            parity ^= 1;                                         // (a warp may be one row ahead of the group's others)
        }
        const float c1 = s1 * inv, c2 = s2 * inv;
        if (ADD) {
            float r[E];
            get_row<T, V>(a, a.add, a.add_stride, row, t, threads, r);
#pragma unroll
            for (int e = 0; e < E; ++e) dy[e] = __fmaf_rn(__fmaf_rn(-x[e], c2, dy[e] - c1), rstd, r[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) dy[e] = __fmaf_rn(-x[e], c2, dy[e] - c1) * rstd;
        }
        T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
#pragma unroll
        for (int i = 0; i < E / V; ++i) {
            const uint32_t col = (i * threads + t) * V;
            float o[V];
#pragma unroll
            for (int j = 0; j < V; ++j) o[j] = dy[i * V + j];
            if (col < cols) put<V>(dx + col, o);
        }
    }
    if (!a.parts) return;
    float *part = a.parts + static_cast<uint64_t>(blockIdx.x) * 2 * cols;
    if (groups == 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t col = V == 1 ? e * threads + t : t * V + e;
            if (col >= cols) continue;
            part[col] = dw[e];
            part[cols + col] = db[e];
        }
        return;
    }
    for (uint32_t g = 0; g < groups; ++g) {
        if (group == g) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t at = e * threads + t;
                joined[at] = g ? joined[at] + dw[e] : dw[e];
                joined[E * threads + at] = g ? joined[E * threads + at] + db[e] : db[e];
            }
        }
        __syncthreads();
    }
    for (uint32_t at = threadIdx.x; at < E * threads; at += blockDim.x) {
        const uint32_t e = at / threads, tt = at - e * threads, col = V == 1 ? at : tt * V + e;
        if (col >= cols) continue;
        part[col] = joined[at];
        part[cols + col] = joined[E * threads + at];
    }
}

// Rows of more columns than a CTA's threads can hold, in two launches.  First c = (mean g, mean(g xhat)) of each row ...
template <typename T, bool PACKED>
__global__ void __launch_bounds__(1024)
norm_grad_rows_kernel(const NormGradArgs a)
{
    __shared__ float2 sums[32];
    const uint64_t row = blockIdx.x;
    const uint32_t blocks = (a.cols + BLOCK8 - 1) / BLOCK8;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (uint32_t col = threadIdx.x; col < a.cols; col += 1024) {
        float x[1], dy[1];
        if (PACKED) get_packed<1>(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col, x);
        else get<1>(static_cast<const T *>(a.x) + row * a.x_stride + col, x);
        get<1>(static_cast<const T *>(a.dy) + row * a.dy_stride + col, dy);
        const float g = a.weight ? dy[0] * a.weight[col] : dy[0];
        s1 += g;
        s2 = __fmaf_rn(g, (x[0] - mean) * rstd, s2);
    }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = make_float2(s1, s2);
    __syncthreads();
    if (threadIdx.x < 32) {
        s1 = warp_sum(sums[threadIdx.x].x);
        s2 = warp_sum(sums[threadIdx.x].y);
        if (threadIdx.x == 0) {
            a.c[2 * row] = s1 / static_cast<float>(a.cols);
            a.c[2 * row + 1] = s2 / static_cast<float>(a.cols);
        }
    }
}
// ... then dx and the sums over rows, a thread a column and a CTA every gridDim.y-th row.
template <typename T, bool PACKED>
__global__ void __launch_bounds__(256)
norm_grad_columns_kernel(const NormGradArgs a)
{
    const uint32_t col = blockIdx.x * 256 + threadIdx.x, blocks = (a.cols + BLOCK8 - 1) / BLOCK8;
    if (col >= a.cols) return;
    const float w = a.weight ? a.weight[col] : 1.f;
    float dw = 0.f, db = 0.f;
#pragma unroll 4
    for (uint64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float x[1], dy[1], r[1] = {0.f};
        if (PACKED) get_packed<1>(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col, x);
        else get<1>(static_cast<const T *>(a.x) + row * a.x_stride + col, x);
        get<1>(static_cast<const T *>(a.dy) + row * a.dy_stride + col, dy);
        if (a.add) get<1>(static_cast<const T *>(a.add) + row * a.add_stride + col, r);
        const float h = (x[0] - mean) * rstd;
        dw = __fmaf_rn(dy[0], h, dw);
        db += dy[0];
        const float o[1] = {__fmaf_rn(__fmaf_rn(-h, a.c[2 * row + 1], dy[0] * w - a.c[2 * row]), rstd, r[0])};
        put<1>(static_cast<T *>(a.dx) + row * a.dx_stride + col, o);
    }
    if (!a.parts) return;
    float *part = a.parts + static_cast<uint64_t>(blockIdx.y) * 2 * a.cols;
    part[col] = dw;
    part[a.cols + col] = db;
}

// Sum of the parts in their order, 32 columns a CTA: 8 warps take every eighth part each and are joined in order.
template <typename G>
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float *parts, uint32_t n, uint32_t cols, G *dweight, G *dbias, int accumulate)
{
    __shared__ float s[8][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    G *out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    float v = 0.f;
    if (col < cols) {
        const float *p = parts + (blockIdx.y ? cols : 0) + col;
#pragma unroll 8
        for (uint32_t i = wid; i < n; i += 8) v += p[static_cast<uint64_t>(i) * 2 * cols];
    }
    s[wid][lane] = v;
    __syncthreads();
    if (wid == 0 && col < cols) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += s[i][lane];
        float old[1] = {0.f};
        if (accumulate) get<1>(out + col, old);
        const float o[1] = {old[0] + v};
        put<1>(out + col, o);
    }
}

// ------------------------------------------------------------------------------------ host

constexpr uint32_t MAX_ENTRIES = 32;                             // of a row in a thread's registers, forward
constexpr uint32_t CTAS = 296;                                   // two of 512 threads on each of 148 SMs
constexpr uint64_t MAX_ROWS = 1ull << 28;
constexpr uint32_t MAX_COLS = 1u << 24;
constexpr uint64_t MAX_STRIDE = 1ull << 40;

uint32_t unit_of(int32_t dtype) { return dtype == DECO_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == DECO_F32 || d == DECO_BF16; }
bool aligned_to(const void *p, uintptr_t unit) { return (reinterpret_cast<uintptr_t>(p) & (unit - 1)) == 0; }

struct Rows {                            // rows of an argument; null: not given
    const void *p;
    uint64_t stride;
};
bool bad_rows(const Rows &r, int32_t dtype, uint32_t cols)
{
    return r.p && (r.stride < cols || r.stride > MAX_STRIDE || !aligned_to(r.p, unit_of(dtype)));
}
// 16-byte accesses: all rows start on 16 bytes
bool wide_rows(std::initializer_list<Rows> all, int32_t dtype, uint32_t cols)
{
    if (cols % 8) return false;
    for (const Rows &r : all)
        if (r.p && (!aligned_to(r.p, 16) || r.stride * unit_of(dtype) % 16)) return false;
    return true;
}
bool bad_packed(const int8_t *codes, const uint8_t *exps) { return !codes || !exps || !aligned_to(codes, 16); }
bool same_start(const Rows &a, const Rows &b) { return a.p && a.p == b.p && a.stride != b.stride; }

deco_status result() { return cudaGetLastError() == cudaSuccess ? DECO_OK : DECO_ERR_CUDA; }

template <typename T, int V, bool ADD, bool KEEP>
void launch_norm_items(const NormArgs &a, uint32_t items, unsigned grid, unsigned block, cudaStream_t s)
{
    if (items <= 8) norm_kernel<T, V, 8 / V, ADD, KEEP><<<grid, block, 0, s>>>(a);
    else if (items <= 16) norm_kernel<T, V, 16 / V, ADD, KEEP><<<grid, block, 0, s>>>(a);
    else norm_kernel<T, V, 32 / V, ADD, KEEP><<<grid, block, 0, s>>>(a);
}
template <typename T, int V>
void launch_norm(const NormArgs &a, uint32_t items, unsigned grid, unsigned block, cudaStream_t s)
{
    if (a.add && a.codes) launch_norm_items<T, V, true, true>(a, items, grid, block, s);
    else if (a.add) launch_norm_items<T, V, true, false>(a, items, grid, block, s);
    else if (a.codes) launch_norm_items<T, V, false, true>(a, items, grid, block, s);
    else launch_norm_items<T, V, false, false>(a, items, grid, block, s);
}

template <typename T, int V>
void launch_grad(const NormGradArgs &a, unsigned grid, unsigned block, size_t smem, cudaStream_t s)
{
    if (a.codes && a.add) norm_grad_kernel<T, V, true, true><<<grid, block, smem, s>>>(a);
    else if (a.codes) norm_grad_kernel<T, V, true, false><<<grid, block, smem, s>>>(a);
    else if (a.add) norm_grad_kernel<T, V, false, true><<<grid, block, smem, s>>>(a);
    else norm_grad_kernel<T, V, false, false><<<grid, block, smem, s>>>(a);
}
template <typename T>
void launch_grad_wide(const NormGradArgs &a, uint32_t parts, cudaStream_t s)
{
    const dim3 grid((a.cols + 255) / 256, parts);
    if (a.codes) {
        norm_grad_rows_kernel<T, true><<<static_cast<unsigned>(a.rows), 1024, 0, s>>>(a);
        norm_grad_columns_kernel<T, true><<<grid, 256, 0, s>>>(a);
    } else {
        norm_grad_rows_kernel<T, false><<<static_cast<unsigned>(a.rows), 1024, 0, s>>>(a);
        norm_grad_columns_kernel<T, false><<<grid, 256, 0, s>>>(a);
    }
}

// How a gradient's rows are shared out.
struct GradPlan {
    bool wide;                           // more columns than the threads of a CTA hold
    uint32_t warps, groups, parts;
    uint64_t bytes() const { return c_floats * 4 + part_floats * 4; }
    uint64_t c_floats, part_floats;
};
GradPlan grad_plan(uint64_t rows, uint32_t cols)
{
    GradPlan p = {};
    p.warps = (cols + 32 * E - 1) / (32 * E);
    p.wide = p.warps > 32;
    if (p.wide) {
        // the columns alone make cols / 256 CTAs: rows are cut so that eight CTAs stand on an SM
        const uint64_t across = (cols + 255) / 256;
        p.parts = static_cast<uint32_t>(std::min<uint64_t>(rows, std::max<uint64_t>(1, 4 * CTAS / across)));
        p.c_floats = 2 * rows;
    } else {
        p.groups = std::min<uint32_t>(8, std::max<uint32_t>(1, 16 / p.warps));
        p.parts = static_cast<uint32_t>(std::min<uint64_t>((rows + p.groups - 1) / p.groups, CTAS));
    }
    p.part_floats = 2ull * p.parts * cols;
    return p;
}

template <typename G>
cudaError_t launch_sum(const float *parts, uint32_t n, uint32_t cols, void *dweight, void *dbias, int accumulate, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((cols + 31) / 32, 2);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const cudaError_t err = cudaLaunchKernelEx(&cfg, sum_parts_kernel<G>, parts, n, cols, static_cast<G *>(dweight),
                                               static_cast<G *>(dbias), accumulate);
    if (err != cudaSuccess) cudaGetLastError();                  // (pending, it would be taken for the next call's)
    return err;
}

}  // namespace

extern "C" deco_status deco_layernorm(const void *x, int32_t dtype, uint64_t rows, uint32_t cols, uint64_t x_stride,
                                      const void *add, uint64_t add_stride, void *sum, uint64_t sum_stride,
                                      const float *weight, const float *bias, float eps, void *y, uint64_t y_stride,
                                      float *mean, float *rstd, int8_t *codes, uint8_t *exponents, void *stream)
{
    if (!is_dtype(dtype) || cols == 0 || cols > MAX_COLS || rows >= MAX_ROWS || !(eps > 0.f) || eps > 3.0e38f)
        return DECO_ERR_INVALID_ARG;
    if (rows == 0) return DECO_OK;
    const Rows rx = {x, x_stride}, ra = {add, add_stride}, rs = {sum, sum_stride}, ry = {y, y_stride};
    if (!x || !y || (sum && !add) || sum == y) return DECO_ERR_INVALID_ARG;
    if (bad_rows(rx, dtype, cols) || bad_rows(ra, dtype, cols) || bad_rows(rs, dtype, cols) || bad_rows(ry, dtype, cols))
        return DECO_ERR_INVALID_ARG;
    if (same_start(ry, rx) || same_start(ry, ra) || same_start(rs, rx) || same_start(rs, ra)) return DECO_ERR_INVALID_ARG;
    for (const float *p : {weight, bias, static_cast<const float *>(mean), static_cast<const float *>(rstd)})
        if (!aligned_to(p, 4)) return DECO_ERR_INVALID_ARG;
    if ((codes || exponents) && bad_packed(codes, exponents)) return DECO_ERR_INVALID_ARG;
    NormArgs a = {};
    a.x = x; a.add = add; a.sum = sum; a.y = y;
    a.x_stride = x_stride; a.add_stride = add_stride; a.sum_stride = sum_stride; a.y_stride = y_stride;
    a.rows = rows;
    a.cols = cols;
    a.weight = weight;
    a.bias = bias;
    a.eps = eps;
    a.mean = mean;
    a.rstd = rstd;
    a.codes = codes;
    a.exps = exponents;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cols > 1024 * MAX_ENTRIES) {
        if (dtype == DECO_F32) norm_wide_kernel<float><<<static_cast<unsigned>(rows), 1024, 0, s>>>(a);
        else norm_wide_kernel<__nv_bfloat16><<<static_cast<unsigned>(rows), 1024, 0, s>>>(a);
        return result();
    }
    const bool wide = wide_rows({rx, ra, rs, ry}, dtype, cols) && aligned_to(weight, 16) && aligned_to(bias, 16);
    // A warp alone needs no barrier: rows of up to 1024 columns are one warp's each, 8 rows a CTA.
    a.warps = (cols + 32 * MAX_ENTRIES - 1) / (32 * MAX_ENTRIES);
    const uint32_t items = (cols + a.warps * 32 - 1) / (a.warps * 32);
    const uint32_t groups = std::max<uint32_t>(1, 8 / a.warps), block = groups * a.warps * 32;
    const unsigned grid = static_cast<unsigned>((rows + groups - 1) / groups);
    if (dtype == DECO_F32) {
        if (wide) launch_norm<float, 8>(a, items, grid, block, s);
        else launch_norm<float, 1>(a, items, grid, block, s);
    } else {
        if (wide) launch_norm<__nv_bfloat16, 8>(a, items, grid, block, s);
        else launch_norm<__nv_bfloat16, 1>(a, items, grid, block, s);
    }
    return result();
}

extern "C" uint64_t deco_layernorm_grad_workspace(uint64_t rows, uint32_t cols)
{
    if (rows == 0 || rows >= MAX_ROWS || cols == 0 || cols > MAX_COLS) return 0;
    return grad_plan(rows, cols).bytes();
}

extern "C" deco_status deco_layernorm_grad(const void *x, int32_t dtype, uint64_t rows, uint32_t cols, uint64_t x_stride,
                                           const int8_t *codes, const uint8_t *exponents, const float *mean,
                                           const float *rstd, const float *weight, const void *dy, uint64_t dy_stride,
                                           const void *add, uint64_t add_stride, void *dx, uint64_t dx_stride,
                                           void *dweight, void *dbias, int32_t grad_dtype, int32_t accumulate,
                                           void *workspace, uint64_t workspace_bytes, void *stream)
{
    if (!is_dtype(dtype) || !is_dtype(grad_dtype) || cols == 0 || cols > MAX_COLS || rows >= MAX_ROWS)
        return DECO_ERR_INVALID_ARG;
    if (!aligned_to(dweight, unit_of(grad_dtype)) || !aligned_to(dbias, unit_of(grad_dtype))) return DECO_ERR_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto sum = [&](const float *parts, uint32_t n) {
        return grad_dtype == DECO_F32 ? launch_sum<float>(parts, n, cols, dweight, dbias, accumulate, s)
                                      : launch_sum<__nv_bfloat16>(parts, n, cols, dweight, dbias, accumulate, s);
    };
    if (rows == 0) {                                             // sums of nothing
        if ((!dweight && !dbias) || accumulate) return DECO_OK;
        return sum(nullptr, 0) == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
    }
    const Rows rx = {x, x_stride}, rg = {dy, dy_stride}, ra = {add, add_stride}, rd = {dx, dx_stride};
    if (!dy || !dx || !mean || !rstd || !x == !codes) return DECO_ERR_INVALID_ARG;
    if (bad_rows(rx, dtype, cols) || bad_rows(rg, dtype, cols) || bad_rows(ra, dtype, cols) || bad_rows(rd, dtype, cols))
        return DECO_ERR_INVALID_ARG;
    if (same_start(rd, rx) || same_start(rd, rg) || same_start(rd, ra)) return DECO_ERR_INVALID_ARG;
    for (const float *p : {mean, rstd, weight})
        if (!aligned_to(p, 4)) return DECO_ERR_INVALID_ARG;
    if ((codes || exponents) && bad_packed(codes, exponents)) return DECO_ERR_INVALID_ARG;
    const GradPlan plan = grad_plan(rows, cols);
    const bool sums = dweight || dbias;
    if (sums || plan.wide) {
        if (!workspace || !aligned_to(workspace, 16)) return DECO_ERR_INVALID_ARG;
        if (workspace_bytes < plan.bytes()) return DECO_ERR_CAPACITY;
    }
    NormGradArgs a = {};
    a.x = x; a.dy = dy; a.add = add; a.dx = dx;
    a.codes = codes; a.exps = exponents;
    a.x_stride = x_stride; a.dy_stride = dy_stride; a.add_stride = add_stride; a.dx_stride = dx_stride;
    a.rows = rows;
    a.cols = cols;
    a.mean = mean;
    a.rstd = rstd;
    a.weight = weight;
    a.c = static_cast<float *>(workspace);
    a.parts = sums ? static_cast<float *>(workspace) + plan.c_floats : nullptr;
    a.warps = plan.warps;
    if (plan.wide) {
        if (dtype == DECO_F32) launch_grad_wide<float>(a, plan.parts, s);
        else launch_grad_wide<__nv_bfloat16>(a, plan.parts, s);
    } else {
        const unsigned block = plan.groups * plan.warps * 32;
        const size_t smem = sums && plan.groups > 1 ? 2ull * plan.warps * 32 * E * sizeof(float) : 0;    // (16 KB at most)
        const bool wide = wide_rows({rx, rg, ra, rd}, dtype, cols);
        if (dtype == DECO_F32) {
            if (wide) launch_grad<float, 8>(a, plan.parts, block, smem, s);
            else launch_grad<float, 1>(a, plan.parts, block, smem, s);
        } else {
            if (wide) launch_grad<__nv_bfloat16, 8>(a, plan.parts, block, smem, s);
            else launch_grad<__nv_bfloat16, 1>(a, plan.parts, block, smem, s);
        }
    }
    const deco_status st = result();
    if (st != DECO_OK || !sums) return st;
    return sum(a.parts, plan.parts) == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}

extern "C" deco_status deco_pack8(const void *x, int32_t dtype, uint64_t rows, uint32_t cols, uint64_t x_stride,
                                  int8_t *codes, uint8_t *exponents, void *stream)
{
    if (!is_dtype(dtype) || cols == 0 || cols > MAX_COLS || rows >= MAX_ROWS) return DECO_ERR_INVALID_ARG;
    if (rows == 0) return DECO_OK;
    const Rows rx = {x, x_stride};
    if (!x || bad_rows(rx, dtype, cols) || bad_packed(codes, exponents)) return DECO_ERR_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool wide = wide_rows({rx}, dtype, cols);
    const uint32_t chunks = (cols + (wide ? 255 : 31)) / (wide ? 256 : 32);
    const uint64_t units = rows * chunks;
    if ((units + 7) / 8 > 0x7FFFFFFFull) return DECO_ERR_INVALID_ARG;
    const unsigned grid = static_cast<unsigned>((units + 7) / 8);
    const float *f = static_cast<const float *>(x);
    const __nv_bfloat16 *h = static_cast<const __nv_bfloat16 *>(x);
    if (dtype == DECO_F32) {
        if (wide) pack_kernel<float, 8><<<grid, 256, 0, s>>>(f, x_stride, cols, chunks, units, codes, exponents);
        else pack_kernel<float, 1><<<grid, 256, 0, s>>>(f, x_stride, cols, chunks, units, codes, exponents);
    } else {
        if (wide) pack_kernel<__nv_bfloat16, 8><<<grid, 256, 0, s>>>(h, x_stride, cols, chunks, units, codes, exponents);
        else pack_kernel<__nv_bfloat16, 1><<<grid, 256, 0, s>>>(h, x_stride, cols, chunks, units, codes, exponents);
    }
    return result();
}

extern "C" deco_status deco_unpack8(const int8_t *codes, const uint8_t *exponents, uint64_t rows, uint32_t cols,
                                    void *y, int32_t dtype, uint64_t y_stride, void *stream)
{
    if (!is_dtype(dtype) || cols == 0 || cols > MAX_COLS || rows >= MAX_ROWS) return DECO_ERR_INVALID_ARG;
    if (rows == 0) return DECO_OK;
    const Rows ry = {y, y_stride};
    if (!y || bad_rows(ry, dtype, cols) || bad_packed(codes, exponents)) return DECO_ERR_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool wide = wide_rows({ry}, dtype, cols);
    const uint32_t chunks = (cols + (wide ? 255 : 31)) / (wide ? 256 : 32);
    const uint64_t units = rows * chunks;
    if ((units + 7) / 8 > 0x7FFFFFFFull) return DECO_ERR_INVALID_ARG;
    const unsigned grid = static_cast<unsigned>((units + 7) / 8);
    float *f = static_cast<float *>(y);
    __nv_bfloat16 *h = static_cast<__nv_bfloat16 *>(y);
    if (dtype == DECO_F32) {
        if (wide) unpack_kernel<float, 8><<<grid, 256, 0, s>>>(codes, exponents, cols, chunks, units, f, y_stride);
        else unpack_kernel<float, 1><<<grid, 256, 0, s>>>(codes, exponents, cols, chunks, units, f, y_stride);
    } else {
        if (wide) unpack_kernel<__nv_bfloat16, 8><<<grid, 256, 0, s>>>(codes, exponents, cols, chunks, units, h, y_stride);
        else unpack_kernel<__nv_bfloat16, 1><<<grid, 256, 0, s>>>(codes, exponents, cols, chunks, units, h, y_stride);
    }
    return result();
}
