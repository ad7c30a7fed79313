// deco_layernorm, deco_layernorm_grad, deco_pack8, deco_unpack8: layer norm with its gradient, and
// activations put away in 8 bits.
//
// All four are bound by memory; at 16 bits there are six entries a cycle and SM to be dealt with, so arithmetic goes by pairs of
// fp32 numbers.  A row belongs to a group of warps, each with 32 N consecutive columns of every row, N a thread's.  Where every
// row of every array starts on 16 bytes a thread's are granules of 16 bytes (V = 4 or 8 entries), and an access of the warp
// 512 consecutive bytes (two granules side by side in a thread made fp32 rows 1.7 times slower: every 32-byte sector is
// asked for twice); with V = 1 (any alignment, any stride) it is 32 consecutive entries.  Either way the places of a
// thread's entries are constants apart, and a block of 32 columns lies in one warp.
//
// Measured at 32768 x 2048 (of the copy rate, 6.54 TB/s): norm of bf16 rows 65 us (63 %), with residual 102 (80 %), with residual and
// checkpoint 109 (85 %), of fp32 rows 93 (88 %); gradient of bf16 rows 76 us (81 %), with residual 89 (92 %), from the checkpoint with
// residual 96 (75 %), of fp32 rows 132 (93 %); packing bf16 39 us (79 %), fp32 54 (96 %), taking back bf16 35 (89 %).  Where it is
// not memory, no limit is reached: issue slots are 60 to 70 % busy, a quarter of the warps there.  Rows that do not start on 16 bytes, 65536 x 1001 bf16: norm 105 us (38 %),
// gradient 125 (48 %), packing 126 (24 %): an instruction an entry for each access, and for a code and its block's maximum.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>
#include <type_traits>

#include "deco.h"
#include "deco_packed8.h"
#include "deco_pairs.h"

namespace {

using namespace deco::pairs;
using deco::BLOCK8;
using deco::converted;

constexpr uint32_t FULL = 0xFFFFFFFFu;
constexpr int THREADS = 512;             // of a CTA whose groups go from row to row
constexpr uint32_t MAX_COLS_HELD = THREADS * 16;                 // of a row whose entries a CTA's threads hold

// ----------------------------------------------------------------------------- entries

__device__ __forceinline__ float get1(const float *p) { return *p; }
__device__ __forceinline__ float get1(const __nv_bfloat16 *p)
{
    return __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const unsigned short *>(p)) << 16);
}
__device__ __forceinline__ void put1(float *p, float v) { *p = v; }
__device__ __forceinline__ void put1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float rounded(float x, const float *) { return x; }
__device__ __forceinline__ float rounded(float x, const __nv_bfloat16 *) { return __bfloat162float(__float2bfloat16_rn(x)); }

// The entries of 16 bytes, as pairs.
template <typename T> constexpr int VEC = 16 / sizeof(T);
__device__ __forceinline__ void pairs_of(const uint4 &w, uint64_t *v, const float *)
{
    v[0] = pair(__uint_as_float(w.x), __uint_as_float(w.y));
    v[1] = pair(__uint_as_float(w.z), __uint_as_float(w.w));
}
__device__ __forceinline__ void pairs_of(const uint4 &w, uint64_t *v, const __nv_bfloat16 *)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void put_granule(float *p, const uint64_t *v)
{
    float4 f;
    unpair(v[0], f.x, f.y);
    unpair(v[1], f.z, f.w);
    *reinterpret_cast<float4 *>(p) = f;
}
__device__ __forceinline__ void put_granule(__nv_bfloat16 *p, const uint64_t *v)
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        unpair(v[i], a, b);
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        u[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

// N entries of a row that a thread owns, in pairs: pair i holds entries 2 i and 2 i + 1 of the thread.  Columns beyond the row
// read as 0 and are not stored.
template <int V, int N>
struct Own {
    uint32_t cols, first, mask;          // the thread's first column; a bit for each of its entries that exists
    __device__ __forceinline__ Own(uint32_t cols_, uint32_t t) : cols(cols_), first(t / 32 * (32 * N) + t % 32 * V), mask(0)
    {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col(e) < cols) mask |= 1u << e;
    }
    static __device__ __forceinline__ constexpr uint32_t offset(int e) { return e / V * (32 * V) + e % V; }
    __device__ __forceinline__ uint32_t col(int e) const { return first + offset(e); }
    __device__ __forceinline__ bool has(int e) const { return mask >> e & 1; }
    template <typename T> __device__ __forceinline__ void load(const T *row, uint64_t (&v)[N / 2]) const
    {
        static_assert(V == 1, "granules come through the ring");
        const T *p = row + first;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            v[i] = pair(has(2 * i) ? get1(p + offset(2 * i)) : 0.f, has(2 * i + 1) ? get1(p + offset(2 * i + 1)) : 0.f);
    }
    template <typename T> __device__ __forceinline__ void store(T *row, const uint64_t (&v)[N / 2]) const
    {
        T *p = row + first;
        if (V > 1) {
#pragma unroll
            for (int e = 0; e < N; e += V)
                if (has(e)) put_granule(p + offset(e), v + e / 2);
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                float a, b;
                unpair(v[i], a, b);
                if (has(2 * i)) put1(p + offset(2 * i), a);
                if (has(2 * i + 1)) put1(p + offset(2 * i + 1), b);
            }
        }
    }
    // pair i of an array of fp32 numbers per column
    __device__ __forceinline__ uint64_t per_column(const float *p, float otherwise, int i) const
    {
        if (!p) return pair(otherwise, otherwise);
        return pair(has(2 * i) ? p[col(2 * i)] : otherwise, has(2 * i + 1) ? p[col(2 * i + 1)] : otherwise);
    }
    // how many of the warp's entries exist
    __device__ __forceinline__ float of_warp() const
    {
        const uint32_t begin = first - threadIdx.x % 32 * V;
        return begin < cols ? static_cast<float>(min(cols - begin, 32u * N)) : 0.f;
    }
};

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}
__device__ __forceinline__ float both(uint64_t v)
{
    float a, b;
    unpair(v, a, b);
    return a + b;
}
__device__ __forceinline__ uint64_t twice(float a) { return pair(a, a); }

// Steps of a group that a thread has asked for ahead (16-byte accesses), in units of shared memory that are its alone.
constexpr int AHEAD = 3;

__device__ __forceinline__ void copy_async(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
}
template <int BYTES> __device__ __forceinline__ void copy_async_small(uint32_t to, const void *from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" :: "r"(to), "l"(from), "n"(BYTES) : "memory");
}
// Four numbers of an array per column, on 16 bytes.
__device__ __forceinline__ uint4 quad_of(const float *p, uint32_t col, bool has, float otherwise)
{
    const uint32_t o = __float_as_uint(otherwise);
    return p && has ? __ldg(reinterpret_cast<const uint4 *>(p + col)) : make_uint4(o, o, o, o);
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

// x / 2^(b - 127) to the nearest integer, as the lowest byte: the product with a power of two is exact, and the sum with
// 1.5 * 2^23 rounds it to an integer, ties to even, whose two's complement its lowest bits are.
constexpr float TO_INTEGER = 12582912.f;
__device__ __forceinline__ float inverse_step(uint32_t b) { return __uint_as_float((254u - b) << 23); }
// Of the largest step, 64 are 2^128, which is no fp32 number: 63 are kept there.
__device__ __forceinline__ float kept(float x, uint32_t b)
{
    const float most = 63.f * 0x1p122f;
    return b == 249u ? fmaxf(-most, fminf(most, x)) : x;
}

// Checkpoint of V consecutive entries a thread owns of a row; the warp together, `in` where there is something to store (entries
// beyond the row's end are 0).
template <int V>
__device__ __forceinline__ void put_packed_granule(int8_t *codes, uint8_t *exps, uint32_t col, bool in, const uint64_t *v)
{
    float f[V];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        unpair(v[i], f[2 * i], f[2 * i + 1]);
        top = max(top, max(magnitude_bits(f[2 * i]), magnitude_bits(f[2 * i + 1])));
    }
    top = in ? top : 0u;
#pragma unroll
    for (int o = 1; o < 32 / V; o *= 2) top = max(top, __shfl_xor_sync(FULL, top, o));
    if (!in) return;
    const uint32_t b = exponent_byte(top);
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = 0;            // (a block that stands for NaN has codes of 0)
    if (b < 250u) {
        const uint64_t inv = twice(inverse_step(b)), magic = twice(TO_INTEGER);
        uint32_t q[V];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            float x, y;
            unpair(fma2(b == 249u ? pair(kept(f[2 * i], b), kept(f[2 * i + 1], b)) : v[i], inv, magic), x, y);
            q[2 * i] = __float_as_uint(x);
            q[2 * i + 1] = __float_as_uint(y);
        }
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            w[i] = __byte_perm(__byte_perm(q[4 * i], q[4 * i + 1], 0x0040), __byte_perm(q[4 * i + 2], q[4 * i + 3], 0x0040), 0x5410);
    }
    if (V == 8) *reinterpret_cast<uint2 *>(codes + col) = make_uint2(w[0], w[V / 4 - 1]);
    else *reinterpret_cast<uint32_t *>(codes + col) = w[0];
    if (col % BLOCK8 == 0) exps[col / BLOCK8] = static_cast<uint8_t>(b);
}
__device__ __forceinline__ void put_packed1(int8_t *codes, uint8_t *exps, uint32_t col, bool in, float v)
{
    const uint32_t b = exponent_byte(__reduce_max_sync(FULL, in ? magnitude_bits(v) : 0u));
    if (!in) return;
    codes[col] = b < 250u ? static_cast<int8_t>(__float_as_uint(__fmaf_rn(kept(v, b), inverse_step(b), TO_INTEGER))) : int8_t(0);
    if (col % BLOCK8 == 0) exps[col / BLOCK8] = static_cast<uint8_t>(b);
}
template <int V, int N>
__device__ __forceinline__ void put_packed(const Own<V, N> &own, int8_t *codes, uint8_t *exps, const uint64_t (&v)[N / 2])
{
    const uint32_t end = (own.cols + BLOCK8 - 1) / BLOCK8 * BLOCK8;
    if constexpr (V > 1) {
#pragma unroll
        for (int e = 0; e < N; e += V) put_packed_granule<V>(codes, exps, own.col(e), own.col(e) < end, v + e / 2);
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            float a, b;
            unpair(v[i], a, b);
            put_packed1(codes, exps, own.col(2 * i), own.col(2 * i) < end, a);
            put_packed1(codes, exps, own.col(2 * i + 1), own.col(2 * i + 1) < end, b);
        }
    }
}

__device__ __forceinline__ float step_of(uint32_t b) { return __uint_as_float(b == 255u ? 0x7FC00000u : b << 23); }
__device__ __forceinline__ float get_packed1(const int8_t *codes, const uint8_t *exps, uint32_t col)
{
    return static_cast<float>(codes[col]) * step_of(exps[col / BLOCK8]);
}
// Four codes and their exponent byte as pairs of fp32 numbers.  A code with its sign bit turned, in the place of the lowest
// byte of 2^23, is 2^23 + 128 + code.
__device__ __forceinline__ void values4(uint32_t codes, uint32_t b, uint64_t *v)
{
    const uint64_t step = twice(step_of(b)), off = twice(-8388736.f);
    const uint32_t w = codes ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float x = __uint_as_float(__byte_perm(w, 0x4B000000u, i ? 0x7542 : 0x7540));
        const float y = __uint_as_float(__byte_perm(w, 0x4B000000u, i ? 0x7543 : 0x7541));
        v[i] = mul2(add2(pair(x, y), off), step);
    }
}

// A warp takes 32 N consecutive columns of ROWS rows, so that four granules (or 16 entries) of a thread are under way together.
// (32768 x 2048 bf16: 63 us to pack with one granule, 39 with four.)
template <int V, int G> constexpr int PACK_ROWS = (V > 1 ? 4 : 16) / G;
struct Part {
    uint64_t row;
    uint32_t chunk;
    bool any;
    __device__ __forceinline__ Part(uint64_t row_groups, uint32_t chunks, uint32_t rows)
    {
        const uint64_t unit = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5), units = row_groups * chunks;
        any = unit < units;
        const uint64_t group = units <= 0xFFFFFFFFull ? static_cast<uint32_t>(unit) / chunks : unit / chunks;
        chunk = static_cast<uint32_t>(unit - group * chunks);
        row = group * rows;
    }
};

template <typename T, int V, int G>
__global__ void __launch_bounds__(256)
pack_kernel(const T *x, uint64_t rows, uint64_t stride, uint32_t cols, uint64_t row_groups, uint32_t chunks, int8_t *codes, uint8_t *exps)
{
    constexpr int N = V * G, R = PACK_ROWS<V, G>;
    const Part part(row_groups, chunks, R);
    if (!part.any) return;
    const Own<V, N> own(cols, part.chunk * 32 + (threadIdx.x & 31));
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    uint4 w[R][G];
    uint64_t v[R][N / 2];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const T *p = x + (part.row + r) * stride;
        const bool live = part.row + r < rows;
        if constexpr (V > 1) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                w[r][g] = make_uint4(0, 0, 0, 0);
                if (live && own.has(V * g)) w[r][g] = *reinterpret_cast<const uint4 *>(p + own.col(V * g));
            }
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) v[r][i] = 0;
            if (live) own.load(p, v[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (part.row + r >= rows) return;
        if constexpr (V > 1) {
#pragma unroll
            for (int g = 0; g < G; ++g) pairs_of(w[r][g], v[r] + V / 2 * g, x);
        }
        put_packed(own, codes + (part.row + r) * blocks * BLOCK8, exps + (part.row + r) * blocks, v[r]);
    }
}

__device__ __forceinline__ void put_values(float *p, uint2 codes, uint32_t b)
{
    uint64_t v[2];
    values4(codes.x, b, v);
    put_granule(p, v);
}
__device__ __forceinline__ void put_values(__nv_bfloat16 *p, uint2 codes, uint32_t b)
{
    *reinterpret_cast<uint4 *>(p) = converted(codes.x, codes.y, deco::bf16_step(b) * 0x10001u);
}

template <typename T, int V, int G>
__global__ void __launch_bounds__(256)
unpack_kernel(const int8_t *codes, const uint8_t *exps, uint64_t rows, uint32_t cols, uint64_t row_groups, uint32_t chunks, T *y,
              uint64_t stride)
{
    constexpr int N = V * G, R = PACK_ROWS<V, G>;
    const Part part(row_groups, chunks, R);
    if (!part.any) return;
    const Own<V, N> own(cols, part.chunk * 32 + (threadIdx.x & 31));
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    uint2 c[R][G];
    uint32_t e[R][G];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int8_t *p = codes + (part.row + r) * blocks * BLOCK8 + own.first;
        const uint8_t *q = exps + (part.row + r) * blocks + own.first / BLOCK8;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            c[r][g] = make_uint2(0, 0);
            e[r][g] = 0;
            if (part.row + r >= rows || !own.has(V * g)) continue;
            if (V == 8) c[r][g] = *reinterpret_cast<const uint2 *>(p + own.offset(V * g));
            else if (V == 4) c[r][g].x = *reinterpret_cast<const uint32_t *>(p + own.offset(V * g));
            else c[r][g].x = static_cast<uint32_t>(static_cast<int>(p[own.offset(g)]));
            e[r][g] = q[own.offset(V * g) / BLOCK8];             // (32 V columns on are whole blocks on)
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        T *p = y + (part.row + r) * stride + own.first;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (part.row + r >= rows || !own.has(V * g)) continue;
            if constexpr (V > 1) put_values(p + own.offset(V * g), c[r][g], e[r][g]);
            else put1(p + own.offset(g), static_cast<float>(static_cast<int>(c[r][g].x)) * step_of(e[r][g]));
        }
    }
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
    float eps, inv_cols;
    uint32_t cols, warps;                // warps of a row's group
};

// Statistics of the entries of some warp: count, mean (as a number and what is left of it), sum of squared deviations from it.
struct __align__(16) Moments {
    float n, mean, rest, m2;
};

// Of a group of `warps` warps (up to WIDTH) from their own, in every thread; the warp together.  Means are joined as differences from
// the first, so that a common offset of the row costs no digits.
template <int WIDTH>
__device__ __forceinline__ Moments join(const Moments *m, uint32_t warps, float inv_cols)
{
    const uint32_t i = threadIdx.x & (WIDTH - 1);
    const float base = m[0].mean;
    const Moments a = i < warps ? m[i] : Moments{0.f, base, 0.f, 0.f};
    const float d = a.mean - base + a.rest;
    float sum = a.n * d;
#pragma unroll
    for (int o = 1; o < WIDTH; o *= 2) sum += __shfl_xor_sync(FULL, sum, o);
    const float off = sum * inv_cols, e = d - off;
    float m2 = __fmaf_rn(a.n * e, e, a.m2);
#pragma unroll
    for (int o = 1; o < WIDTH; o *= 2) m2 += __shfl_xor_sync(FULL, m2, o);
    return {0.f, base + off, 0.f, m2};
}
__device__ __forceinline__ float reciprocal(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// One step of Newton's method on the approximate root's reciprocal: within 2 roundings.
__device__ __forceinline__ float root_reciprocal(float v)
{
    const float y = rsqrtf(v);
    return __fmaf_rn(0.5f * y, __fmaf_rn(-v * y, y, 1.f), y);
}
// Of a warp's entries in pairs, `n` of them: those beyond the row are 0 and counted out by `mask` (a bit a pair's entry).
template <int N>
__device__ __forceinline__ Moments warp_moments(const uint64_t (&v)[N / 2], float n, bool whole, uint32_t mask)
{
    uint64_t s = 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) s = add2(s, v[i]);
    const float inv = reciprocal(fmaxf(n, 1.f)), m = warp_sum(both(s)) * inv;
    const uint64_t mm = twice(-m);
    uint64_t d1 = 0, d2 = 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        uint64_t d = add2(v[i], mm);
        if (!whole) {
            float p, q;
            unpair(d, p, q);
            d = pair(mask >> (2 * i) & 1 ? p : 0.f, mask >> (2 * i + 1) & 1 ? q : 0.f);
        }
        d1 = add2(d1, d);
        d2 = fma2(d, d, d2);
    }
    const float t1 = warp_sum(both(d1)), t2 = warp_sum(both(d2)), rest = t1 * inv, m2 = __fmaf_rn(-t1, rest, t2);
    return {n, m, rest, m2 < 0.f ? 0.f : m2};                    // (a NaN stays)
}

// One pass: a row stays in registers between its statistics and its output.  Deviations are summed from the warp's own mean,
// and what rounding did to that mean is taken back by their sum.  Every group goes from row to row; what keeps memory busy
// between a row's arrival and its output are the copies of the group's next rows, in shared memory that is each thread's alone.
template <typename T, bool ADD, bool KEEP, int E>
__global__ void __launch_bounds__(THREADS, E == 8 ? 2 : 1)
norm_kernel(const NormArgs a)
{
    constexpr int V = VEC<T>, A = AHEAD, U = ADD ? 2 : 1, G = E / V;
    extern __shared__ uint4 ring[];                              // [A][G][U][thread]
    __shared__ Moments moments[2][THREADS / 32];                 // (a warp may be one row ahead of the group's others)
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, group = wid / a.warps, groups = (blockDim.x >> 5) / a.warps;
    const uint32_t threads = a.warps * 32, t = threadIdx.x - group * threads, cols = a.cols, all = blockDim.x;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    const Own<V, E> own(cols, t);
    // (with V = 4 a warp reads weights and bias as consecutive bytes from the cache, which leaves registers)
    uint64_t w[E / 2], b[E / 2];
#pragma unroll
    for (int i = 0; V == 8 && i < E / 2; ++i) {
        w[i] = own.per_column(a.weight, 1.f, i);
        b[i] = own.per_column(a.bias, 0.f, i);
    }
    const float n = own.of_warp();
    const bool whole = n == 32.f * E;
    uint4 *mine = ring + threadIdx.x;
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(mine));
    // (columns beyond the last stay 0 in the ring)
    for (uint32_t u = 0; u < A * G * U; ++u) mine[u * all] = make_uint4(0, 0, 0, 0);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * groups;
    uint64_t row = static_cast<uint64_t>(blockIdx.x) * groups + group, next = row;
    const T *x_next = static_cast<const T *>(a.x) + row * a.x_stride, *add_next = static_cast<const T *>(a.add) + row * a.add_stride;
    T *y = static_cast<T *>(a.y) + row * a.y_stride, *sum = static_cast<T *>(a.sum) + row * a.sum_stride;
    auto ask = [&](uint32_t s) {
        if (next < a.rows) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t at = to + (s * G + g) * U * all * 16;
                if (!own.has(V * g)) continue;
                copy_async(at, x_next + own.col(V * g));
                if (ADD) copy_async(at + all * 16, add_next + own.col(V * g));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        next += step;
        x_next += step * a.x_stride;
        if (ADD) add_next += step * a.add_stride;
    };
#pragma unroll
    for (int s = 0; s < A; ++s) ask(s);
    uint32_t parity = 0, s = 0;
    for (; row < a.rows; row += step) {
        asm volatile("cp.async.wait_group %0;" :: "n"(A - 1) : "memory");
        uint64_t v[E / 2];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint4 *q = mine + (s * G + g) * U * all;
            pairs_of(*q, v + V / 2 * g, y);
            if (ADD) {
                uint64_t r[V / 2];
                pairs_of(q[all], r, y);
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    float f, h;
                    unpair(add2(v[V / 2 * g + i], r[i]), f, h);
                    v[V / 2 * g + i] = pair(rounded(f, y), rounded(h, y));
                }
            }
        }
        ask(s);
        s = s + 1 == A ? 0 : s + 1;
        if (ADD) {
            if (a.sum) own.store(sum, v);
            sum += step * a.sum_stride;
        }
        Moments mo = warp_moments<E>(v, n, whole, own.mask);
        float mean = mo.mean + mo.rest;
        if (a.warps > 1) {
            if (lane == 0) moments[parity][wid] = mo;
            asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "r"(threads) : "memory");
            mo = join<THREADS / 32>(moments[parity] + group * a.warps, a.warps, a.inv_cols);
            mean = mo.mean;
            parity ^= 1;
        }
        const float rstd = root_reciprocal(__fmaf_rn(mo.m2, a.inv_cols, a.eps));
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (KEEP) put_packed(own, a.codes + row * blocks * BLOCK8, a.exps + row * blocks, v);
        const uint64_t mm = twice(-mean), rr = twice(rstd);
#pragma unroll
        for (int i = 0; V == 4 && i < E / 4; ++i) {
            pairs_of(quad_of(a.weight, own.col(4 * i), own.has(4 * i), 1.f), w + 2 * i, static_cast<const float *>(nullptr));
            pairs_of(quad_of(a.bias, own.col(4 * i), own.has(4 * i), 0.f), b + 2 * i, static_cast<const float *>(nullptr));
        }
#pragma unroll
        for (int i = 0; i < E / 2; ++i) v[i] = fma2(mul2(add2(v[i], mm), rr), w[i], b[i]);
        own.store(y, v);
        y += step * a.y_stride;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// The same for rows and columns of any alignment: what keeps memory busy is the number of warps.
template <typename T, bool ADD, bool KEEP, int E>
__global__ void __launch_bounds__(THREADS, E == 8 ? 2 : 1)
norm_any_kernel(const NormArgs a)
{
    __shared__ Moments moments[2][THREADS / 32];
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, group = wid / a.warps, groups = (blockDim.x >> 5) / a.warps;
    const uint32_t threads = a.warps * 32, t = threadIdx.x - group * threads, blocks = (a.cols + BLOCK8 - 1) / BLOCK8;
    const Own<1, E> own(a.cols, t);
    uint64_t w[E / 2], b[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        w[i] = own.per_column(a.weight, 1.f, i);
        b[i] = own.per_column(a.bias, 0.f, i);
    }
    const float n = own.of_warp();
    const bool whole = n == 32.f * E;
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * groups;
    uint32_t parity = 0;
    for (uint64_t row = static_cast<uint64_t>(blockIdx.x) * groups + group; row < a.rows; row += step) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        uint64_t v[E / 2];
        own.load(x, v);
        if (ADD) {
            uint64_t r[E / 2];
            own.load(static_cast<const T *>(a.add) + row * a.add_stride, r);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float p, q;
                unpair(add2(v[i], r[i]), p, q);
                v[i] = pair(rounded(p, x), rounded(q, x));
            }
            if (a.sum) own.store(static_cast<T *>(a.sum) + row * a.sum_stride, v);
        }
        Moments mo = warp_moments<E>(v, n, whole, own.mask);
        float mean = mo.mean + mo.rest;
        if (a.warps > 1) {
            if (lane == 0) moments[parity][wid] = mo;
            asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "r"(threads) : "memory");
            mo = join<THREADS / 32>(moments[parity] + group * a.warps, a.warps, a.inv_cols);
            mean = mo.mean;
            parity ^= 1;
        }
        const float rstd = root_reciprocal(__fmaf_rn(mo.m2, a.inv_cols, a.eps));
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (KEEP) put_packed(own, a.codes + row * blocks * BLOCK8, a.exps + row * blocks, v);
        const uint64_t mm = twice(-mean), rr = twice(rstd);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) v[i] = fma2(mul2(add2(v[i], mm), rr), w[i], b[i]);
        own.store(static_cast<T *>(a.y) + row * a.y_stride, v);
    }
}

// Rows of more columns than that: one CTA a row, which reads it once for its sum, once for its
// deviations and once for the output (the second and third time from the caches), an entry an access.  (8192 x 12288 bf16: 430 us,
// 0.94 TB/s; 4096 x 16384: 264.)
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
        const float v = get1(x + col);
        return add ? rounded(v + get1(add + col), x) : v;
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
    if (lane == 0) moments[wid] = {n, m, rest, m2 < 0.f ? 0.f : m2};
    __syncthreads();
    const Moments mo = join<32>(moments, 32, a.inv_cols);
    const float rstd = root_reciprocal(__fmaf_rn(mo.m2, a.inv_cols, a.eps));
    if (t == 0) {
        if (a.mean) a.mean[row] = mo.mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    for (uint32_t col = t; col - lane < cols; col += 1024) {
        const float v = col < cols ? value(col) : 0.f;
        if (a.codes) put_packed1(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col, col < blocks * BLOCK8, v);
        if (col >= cols) continue;
        if (sum) put1(sum + col, v);
        put1(y + col, __fmaf_rn((v - mo.mean) * rstd, a.weight ? a.weight[col] : 1.f, a.bias ? a.bias[col] : 0.f));
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


template <typename T> constexpr int GRAD_AHEAD = VEC<T> == 8 ? 3 : 2;    // (what fits shared memory, twice with 8 entries)

// What a thread knows of its columns, over the rows of its group.
template <int E> struct Columns {
    uint64_t dw[E / 2], db[E / 2];
};
struct GroupSums {
    float2 s[2][THREADS / 32];           // (a warp may be one row ahead of the group's others)
};

// A row's x and dy of the thread's columns in pairs -> in x xhat, in dy g, and -mean g and -mean(g xhat).
template <int E, typename W>
__device__ __forceinline__ void means(Columns<E> &c, W weight, uint64_t (&x)[E / 2], uint64_t (&dy)[E / 2], float mean, float rstd,
                                      float inv, GroupSums &sums, uint32_t parity, uint32_t group, uint32_t warps, uint64_t &c1, uint64_t &c2)
{
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint64_t mm = twice(-mean), rr = twice(rstd);
    uint64_t p1 = 0, p2 = 0;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
        x[i] = mul2(add2(x[i], mm), rr);
        c.dw[i] = fma2(dy[i], x[i], c.dw[i]);
        c.db[i] = add2(c.db[i], dy[i]);
        dy[i] = mul2(dy[i], weight(i));
        p1 = add2(p1, dy[i]);
        p2 = fma2(dy[i], x[i], p2);
    }
    float s1 = warp_sum(both(p1)), s2 = warp_sum(both(p2));
    if (warps > 1) {
        if (lane == 0) sums.s[parity][wid] = make_float2(s1, s2);
        asm volatile("bar.sync %0, %1;" :: "r"(1 + group), "r"(warps * 32) : "memory");
        const uint32_t i = lane & (THREADS / 32 - 1);
        const float2 p = i < warps ? sums.s[parity][group * warps + i] : make_float2(0.f, 0.f);
        s1 = p.x;
        s2 = p.y;
#pragma unroll
        for (int o = 1; o < THREADS / 32; o *= 2) {
            s1 += __shfl_xor_sync(FULL, s1, o);
            s2 += __shfl_xor_sync(FULL, s2, o);
        }
    }
    c1 = twice(-s1 * inv);
    c2 = twice(-s2 * inv);
}

// The groups' sums over their rows, joined in shared memory in the groups' order, as the CTA's part.
template <int V, int E>
__device__ __forceinline__ void put_part(const NormGradArgs &a, const Columns<E> &c, const Own<V, E> &own, uint32_t t, uint32_t threads,
                                         uint32_t group, uint32_t groups, float *joined)
{
    const uint32_t cols = a.cols;
    float *part = a.parts + static_cast<uint64_t>(blockIdx.x) * 2 * cols;
    for (uint32_t g = 0; g < groups; ++g) {
        if (group == g) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t at = e * threads + t;
                float x, y, dw, db;
                unpair(c.dw[e / 2], x, y);
                dw = e & 1 ? y : x;
                unpair(c.db[e / 2], x, y);
                db = e & 1 ? y : x;
                if (g) {
                    dw += joined[at];
                    db += joined[E * threads + at];
                }
                if (g + 1 < groups) {
                    joined[at] = dw;
                    joined[E * threads + at] = db;
                } else if (own.has(e)) {
                    part[own.col(e)] = dw;
                    part[cols + own.col(e)] = db;
                }
            }
        }
        if (g + 1 < groups) __syncthreads();
    }
}

// xhat = (x - mean) rstd, g = dy w;  dx = rstd (g - mean g - xhat mean(g xhat)) (+ add).  A group goes from row to
// row, and each thread sums dy xhat and dy of its own columns over its rows in registers; the groups of
// a CTA are joined in their order, the CTAs by sum_parts_kernel in theirs: the same bits every time.  What keeps memory
// busy between a row's arrival and its result are the copies of the group's next rows.
template <typename T, bool PACKED, bool ADD, int E>
__global__ void __launch_bounds__(THREADS, E == 8 ? 2 : 1)
norm_grad_kernel(const NormGradArgs a)
{
    constexpr int V = VEC<T>, A = GRAD_AHEAD<T>, U = ADD ? 3 : 2, G = E / V;
    extern __shared__ uint4 ring[];                              // [A][G][U][thread], weights [E / 4][thread] if V = 8; then the groups' sums
    __shared__ GroupSums sums;
    const uint32_t wid = threadIdx.x >> 5, group = wid / a.warps, groups = (blockDim.x >> 5) / a.warps;
    const uint32_t threads = a.warps * 32, t = threadIdx.x - group * threads, cols = a.cols, all = blockDim.x;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Own<V, E> own(cols, t);
    Columns<E> c;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) c.dw[i] = c.db[i] = 0;
    const float inv = 1.f / static_cast<float>(cols);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * groups;
    uint4 *mine = ring + threadIdx.x, *weights = mine + A * G * U * all;
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(mine));
    uint64_t row = static_cast<uint64_t>(blockIdx.x) * groups + group, next = row;
    // (columns beyond the last stay 0 in the ring)
    for (uint32_t u = 0; u < A * G * U; ++u) mine[u * all] = make_uint4(0, 0, 0, 0);
    // (with V = 4 a warp reads the weights as consecutive bytes from the cache; with V = 8 it would not)
#pragma unroll
    for (int i = 0; V == 8 && i < E / 4; ++i) {
        const uint64_t p[2] = {own.per_column(a.weight, 1.f, 2 * i), own.per_column(a.weight, 1.f, 2 * i + 1)};
        weights[i * all] = *reinterpret_cast<const uint4 *>(p);
    }
    uint32_t exps[A][G];                                         // of rows ahead
    float mean[A], rstd[A];
    auto ask = [&](int s) {
        if (next < a.rows) {
            mean[s] = __ldg(a.mean + next);
            rstd[s] = __ldg(a.rstd + next);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t col = own.col(V * g), at = to + (s * G + g) * U * all * 16;
                if (!own.has(V * g)) continue;
                if (PACKED) {
                    copy_async_small<V>(at, a.codes + next * blocks * BLOCK8 + col);
                    exps[s][g] = __ldg(a.exps + next * blocks + col / BLOCK8);
                } else {
                    copy_async(at, static_cast<const T *>(a.x) + next * a.x_stride + col);
                }
                copy_async(at + all * 16, static_cast<const T *>(a.dy) + next * a.dy_stride + col);
                if (ADD) copy_async(at + 2 * all * 16, static_cast<const T *>(a.add) + next * a.add_stride + col);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        next += step;
    };
#pragma unroll
    for (int s = 0; s < A; ++s) {
#pragma unroll
        for (int g = 0; g < G; ++g) exps[s][g] = 0;
        mean[s] = rstd[s] = 0.f;
        ask(s);
    }
    uint32_t parity = 0;
    while (row < a.rows) {
#pragma unroll
        for (int s = 0; s < A; ++s) {
            if (row >= a.rows) break;
            asm volatile("cp.async.wait_group %0;" :: "n"(A - 1) : "memory");
            uint64_t x[E / 2], dy[E / 2], c1, c2;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint4 *q = mine + (s * G + g) * U * all;
                if (PACKED) {
                    const uint2 codes = *reinterpret_cast<const uint2 *>(q);
                    values4(codes.x, exps[s][g], x + V / 2 * g);
                    if (V == 8) values4(codes.y, exps[s][g], x + V / 2 * g + 2);
                } else {
                    pairs_of(*q, x + V / 2 * g, static_cast<const T *>(nullptr));
                }
                pairs_of(q[all], dy + V / 2 * g, static_cast<const T *>(nullptr));
            }
            const uint64_t rr = twice(rstd[s]);
            uint64_t w[E / 2];
#pragma unroll
            for (int i = 0; i < E / 4; ++i) {
                const uint4 q = V == 8 ? weights[i * all] : quad_of(a.weight, own.col(4 * i), own.has(4 * i), 1.f);
                w[2 * i] = pair(__uint_as_float(q.x), __uint_as_float(q.y));
                w[2 * i + 1] = pair(__uint_as_float(q.z), __uint_as_float(q.w));
            }
            T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
            means<E>(c, [&](int i) { return w[i]; }, x, dy, mean[s], rstd[s], inv, sums, parity, group, a.warps, c1, c2);
            parity ^= 1;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                uint64_t add[V / 2];
                if (ADD) pairs_of(mine[((s * G + g) * U + 2) * all], add, static_cast<const T *>(nullptr));
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    const int k = V / 2 * g + i;
                    const uint64_t h = fma2(x[k], c2, add2(dy[k], c1));
                    x[k] = ADD ? fma2(h, rr, add[i]) : mul2(h, rr);
                }
                if (own.has(V * g)) put_granule(dx + own.col(V * g), x + V / 2 * g);
            }
            ask(s);
            row += step;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!a.parts) return;
    __syncthreads();
    put_part<V, E>(a, c, own, t, threads, group, groups, reinterpret_cast<float *>(ring));
}

// The same for rows and columns of any alignment.
template <typename T, bool PACKED, bool ADD, int E>
__global__ void __launch_bounds__(THREADS, E == 8 ? 2 : 1)
norm_grad_any_kernel(const NormGradArgs a)
{
    extern __shared__ float joined[];                            // [2][threads * E] of a row's group; groups > 1
    __shared__ GroupSums sums;
    const uint32_t wid = threadIdx.x >> 5, group = wid / a.warps, groups = (blockDim.x >> 5) / a.warps;
    const uint32_t threads = a.warps * 32, t = threadIdx.x - group * threads, cols = a.cols;
    const uint32_t blocks = (cols + BLOCK8 - 1) / BLOCK8;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Own<1, E> own(cols, t);
    Columns<E> c;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) c.dw[i] = c.db[i] = 0;
    const float inv = 1.f / static_cast<float>(cols);
    const uint64_t step = static_cast<uint64_t>(gridDim.x) * groups;
    uint32_t parity = 0;
    for (uint64_t row = static_cast<uint64_t>(blockIdx.x) * groups + group; row < a.rows; row += step) {
        uint64_t x[E / 2], dy[E / 2], c1, c2;
        if (PACKED) {
            const int8_t *codes = a.codes + row * blocks * BLOCK8 + own.first;
            const uint8_t *exps = a.exps + row * blocks + own.first / BLOCK8;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float v[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int e = 2 * i + k;                     // (entry e is in the thread's block e: 32 columns on)
                    v[k] = own.has(e) ? static_cast<float>(codes[own.offset(e)]) * step_of(exps[e]) : 0.f;
                }
                x[i] = pair(v[0], v[1]);
            }
        } else {
            own.load(static_cast<const T *>(a.x) + row * a.x_stride, x);
        }
        own.load(static_cast<const T *>(a.dy) + row * a.dy_stride, dy);
        const float mean = a.mean[row], rstd = a.rstd[row];
        means<E>(c, [&](int i) { return own.per_column(a.weight, 1.f, i); }, x, dy, mean, rstd, inv, sums, parity, group, a.warps, c1, c2);
        parity ^= 1;
        const uint64_t rr = twice(rstd);
        uint64_t add[E / 2];
        if (ADD) own.load(static_cast<const T *>(a.add) + row * a.add_stride, add);
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const uint64_t g = fma2(x[i], c2, add2(dy[i], c1));
            x[i] = ADD ? fma2(g, rr, add[i]) : mul2(g, rr);
        }
        own.store(static_cast<T *>(a.dx) + row * a.dx_stride, x);
    }
    if (!a.parts) return;
    put_part<1, E>(a, c, own, t, threads, group, groups, joined);
}

// Rows of more columns than a CTA's threads can hold, in two launches, x and dy read twice.  (8192 x 12288 bf16: 362 us, 1.67 TB/s;
// 4096 x 16384: 244.)  First c = (mean g, mean(g xhat)) of each row ...
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
        const float x = PACKED ? get_packed1(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col)
                               : get1(static_cast<const T *>(a.x) + row * a.x_stride + col);
        const float dy = get1(static_cast<const T *>(a.dy) + row * a.dy_stride + col), g = a.weight ? dy * a.weight[col] : dy;
        s1 += g;
        s2 = __fmaf_rn(g, (x - mean) * rstd, s2);
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
        const float x = PACKED ? get_packed1(a.codes + row * blocks * BLOCK8, a.exps + row * blocks, col)
                               : get1(static_cast<const T *>(a.x) + row * a.x_stride + col);
        const float dy = get1(static_cast<const T *>(a.dy) + row * a.dy_stride + col);
        const float r = a.add ? get1(static_cast<const T *>(a.add) + row * a.add_stride + col) : 0.f;
        const float h = (x - mean) * rstd;
        dw = __fmaf_rn(dy, h, dw);
        db += dy;
        put1(static_cast<T *>(a.dx) + row * a.dx_stride + col,
             __fmaf_rn(__fmaf_rn(-h, a.c[2 * row + 1], dy * w - a.c[2 * row]), rstd, r));
    }
    if (!a.parts) return;
    float *part = a.parts + static_cast<uint64_t>(blockIdx.y) * 2 * a.cols;
    part[col] = dw;
    part[a.cols + col] = db;
}

// Sum of the parts in their order, 32 columns a CTA: 32 warps take every 32nd part each and are joined in order.
template <typename G>
__global__ void __launch_bounds__(1024)
sum_parts_kernel(const float *parts, uint32_t n, uint32_t cols, G *dweight, G *dbias, int accumulate)
{
    __shared__ float s[32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    G *out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    float v = 0.f;
    if (col < cols) {
        const float *p = parts + (blockIdx.y ? cols : 0) + col;
#pragma unroll 5
        for (uint32_t i = wid; i < n; i += 32) v += p[static_cast<uint64_t>(i) * 2 * cols];
    }
    s[lane][wid] = v;
    __syncthreads();
    v = warp_sum(s[wid][lane]);                                  // warp w: column w of the 32
    const uint32_t c = blockIdx.x * 32 + wid;
    if (lane == 0 && c < cols) put1(out + c, accumulate ? get1(out + c) + v : v);
}

// ------------------------------------------------------------------------------------ host

constexpr uint32_t SMS = 148;
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
// 16-byte accesses: all rows start on 16 bytes and have whole granules
bool wide_rows(std::initializer_list<Rows> all, int32_t dtype, uint32_t cols)
{
    if (cols * unit_of(dtype) % 16) return false;
    for (const Rows &r : all)
        if (r.p && (!aligned_to(r.p, 16) || r.stride * unit_of(dtype) % 16)) return false;
    return true;
}
bool bad_packed(const int8_t *codes, const uint8_t *exps) { return !codes || !exps || !aligned_to(codes, 16); }
// Rows of one buffer that do not lie over one another.  (One row has no distance to the next.)
bool askew(const Rows &a, const Rows &b, uint64_t rows) { return rows > 1 && a.p && a.p == b.p && a.stride != b.stride; }

deco_status result() { return cudaGetLastError() == cudaSuccess ? DECO_OK : DECO_ERR_CUDA; }

// How rows are shared out among groups of warps that go from row to row.  Entries of a row that a thread holds: 8 (two CTAs of 512
// threads an SM) or more (one).  A warp spends about 100 instructions on a row whatever its share is, which 16-bit rows cannot
// afford for 8 entries (32768 x 2048 bf16, gradient with residual: 111 us with 8, 91 with 16; fp32: 134 and 141); a
// row of one warp needs no barrier (65536 x 768 bf16 forward: 57 us with 16, 39 with 24; the gradient has no registers for
// 24, and of 8192 rows 8 entries, three warps, make 22 us, 16 and two 25; more rows of 513 to 768 columns were not
// measured).  As many groups as 512 threads make, but few rows are spread over the device.
struct Spread {
    uint32_t entries, warps, groups, ctas;
};
Spread spread(uint64_t rows, uint32_t cols, int32_t dtype, bool wide, bool gradient)
{
    Spread p = {};
    if (cols > MAX_COLS_HELD) return p;                          // (too many)
    if (!wide) p.entries = cols <= THREADS * 8 ? 8 : 16;
    else if (dtype == DECO_F32) p.entries = cols <= 256 || cols > 512 ? (cols <= THREADS * 8 ? 8 : 16) : 16;
    else if (gradient) p.entries = cols <= 256 || (cols > 512 && cols <= 768) ? 8 : 16;
    else p.entries = cols <= 256 ? 8 : cols > 512 && cols <= 768 ? 24 : 16;
    p.warps = (cols + 32 * p.entries - 1) / (32 * p.entries);
    const uint64_t most = p.entries == 8 ? 2 * SMS : SMS, groups = p.warps == 1 ? 16 : std::min<uint64_t>(8, THREADS / 32 / p.warps);
    p.groups = static_cast<uint32_t>(std::min<uint64_t>(groups, (rows + most - 1) / most));
    p.ctas = static_cast<uint32_t>(std::min<uint64_t>((rows + p.groups - 1) / p.groups, most));
    return p;
}

// A kernel's shared memory, once per device.
template <auto KERNEL>
cudaError_t allow(size_t bytes)
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err == cudaSuccess && dev >= 0 && dev < 64 && (done.load() >> dev & 1)) return cudaSuccess;
    if (err == cudaSuccess) err = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (err != cudaSuccess) cudaGetLastError();                  // (pending, it would be taken for the next call's)
    else if (dev >= 0 && dev < 64) done.fetch_or(1ull << dev);
    return err;
}

template <typename T, bool ADD, bool KEEP, int E>
cudaError_t launch_norm_as(const NormArgs &a, const Spread &p, cudaStream_t s)
{
    constexpr size_t BYTES = 16ull * AHEAD * (ADD ? 2 : 1) * (E / VEC<T>);                           // a thread's
    static_assert(BYTES * THREADS <= (E == 8 ? 110 : 224) * 1024, "a CTA's shared memory");
    const cudaError_t err = allow<norm_kernel<T, ADD, KEEP, E>>(BYTES * THREADS);
    if (err != cudaSuccess) return err;
    const unsigned block = p.groups * p.warps * 32;
    norm_kernel<T, ADD, KEEP, E><<<p.ctas, block, BYTES * block, s>>>(a);
    return cudaGetLastError();
}
template <typename T, bool ADD, bool KEEP>
cudaError_t launch_norm_rows(NormArgs a, bool wide, cudaStream_t s)
{
    const Spread p = spread(a.rows, a.cols, sizeof(T) == 4 ? DECO_F32 : DECO_BF16, wide, false);
    a.warps = p.warps;
    if (!wide) {
        const unsigned block = p.groups * p.warps * 32;
        if (p.entries == 8) norm_any_kernel<T, ADD, KEEP, 8><<<p.ctas, block, 0, s>>>(a);
        else norm_any_kernel<T, ADD, KEEP, 16><<<p.ctas, block, 0, s>>>(a);
        return cudaGetLastError();
    }
    if (p.entries == 8) return launch_norm_as<T, ADD, KEEP, 8>(a, p, s);
    if constexpr (sizeof(T) == 2) {
        if (p.entries == 24) return launch_norm_as<T, ADD, KEEP, 24>(a, p, s);
    }
    return launch_norm_as<T, ADD, KEEP, 16>(a, p, s);
}
template <typename T>
cudaError_t launch_norm(const NormArgs &a, bool wide, cudaStream_t s)
{
    if (a.add && a.codes) return launch_norm_rows<T, true, true>(a, wide, s);
    if (a.add) return launch_norm_rows<T, true, false>(a, wide, s);
    if (a.codes) return launch_norm_rows<T, false, true>(a, wide, s);
    return launch_norm_rows<T, false, false>(a, wide, s);
}

template <typename T, bool PACKED, bool ADD, int E>
cudaError_t launch_grad_as(const NormGradArgs &a, bool wide, unsigned grid, unsigned block, cudaStream_t s)
{
    const size_t joined = block > a.warps * 32 ? 2ull * a.warps * 32 * E * sizeof(float) : 0;       // (at most 32 KB)
    if (!wide) {
        norm_grad_any_kernel<T, PACKED, ADD, E><<<grid, block, joined, s>>>(a);
        return cudaGetLastError();
    }
    constexpr size_t BYTES = 16ull * (GRAD_AHEAD<T> * (ADD ? 3 : 2) * (E / VEC<T>) + (VEC<T> == 8 ? E / 4 : 0));     // a thread's
    static_assert(BYTES * THREADS <= (E == 8 ? 112 : 224) * 1024, "a CTA's shared memory");
    const cudaError_t err = allow<norm_grad_kernel<T, PACKED, ADD, E>>(BYTES * THREADS);
    if (err != cudaSuccess) return err;
    norm_grad_kernel<T, PACKED, ADD, E><<<grid, block, std::max(joined, BYTES * block), s>>>(a);
    return cudaGetLastError();
}
template <typename T, bool PACKED, bool ADD>
cudaError_t launch_grad_rows(const NormGradArgs &a, uint32_t entries, bool wide, unsigned grid, unsigned block, cudaStream_t s)
{
    return entries == 8 ? launch_grad_as<T, PACKED, ADD, 8>(a, wide, grid, block, s) : launch_grad_as<T, PACKED, ADD, 16>(a, wide, grid, block, s);
}
template <typename T>
cudaError_t launch_grad(const NormGradArgs &a, uint32_t entries, bool wide, unsigned grid, unsigned block, cudaStream_t s)
{
    if (a.codes && a.add) return launch_grad_rows<T, true, true>(a, entries, wide, grid, block, s);
    if (a.codes) return launch_grad_rows<T, true, false>(a, entries, wide, grid, block, s);
    if (a.add) return launch_grad_rows<T, false, true>(a, entries, wide, grid, block, s);
    return launch_grad_rows<T, false, false>(a, entries, wide, grid, block, s);
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

// Granules of a row that a thread of the packing kernels takes: as many as leave few lanes empty.  V = 1: 8 entries.
template <typename F>
deco_status by_shape(uint32_t vec, uint64_t rows, uint32_t cols, F launch)
{
    const auto chunks = [&](uint32_t g) { return (cols + 32 * vec * g - 1) / (32 * vec * g); };
    const auto fits = [&](uint32_t g) { return static_cast<uint64_t>(chunks(g)) * (32 * vec * g) * 8 <= static_cast<uint64_t>(cols) * 9; };
    const uint32_t g = vec == 1 ? 8 : fits(4) ? 4 : fits(2) ? 2 : 1, together = (vec > 1 ? 4 : 16) / g;
    const uint64_t row_groups = (rows + together - 1) / together, ctas = (row_groups * chunks(g) + 7) / 8;
    if (ctas > 0x7FFFFFFFull) return DECO_ERR_INVALID_ARG;
    const unsigned grid = static_cast<unsigned>(ctas);
    const auto with = [&](auto v) {
        if (g == 4) launch(v, std::integral_constant<int, 4>(), row_groups, chunks(g), grid);
        else if (g == 2) launch(v, std::integral_constant<int, 2>(), row_groups, chunks(g), grid);
        else launch(v, std::integral_constant<int, 1>(), row_groups, chunks(g), grid);
    };
    if (vec == 8) with(std::integral_constant<int, 8>());
    else if (vec == 4) with(std::integral_constant<int, 4>());
    else launch(std::integral_constant<int, 1>(), std::integral_constant<int, 8>(), row_groups, chunks(g), grid);
    return result();
}

// How a gradient's rows are shared out.
struct GradPlan {
    bool wide;                           // more columns than the threads of a CTA hold
    uint32_t entries, warps, groups, parts;
    uint64_t bytes() const { return c_floats * 4 + part_floats * 4; }
    uint64_t c_floats, part_floats;
};
GradPlan grad_plan(uint64_t rows, uint32_t cols, int32_t dtype, bool aligned)
{
    GradPlan p = {};
    const Spread q = spread(rows, cols, dtype, aligned, true);
    p.wide = q.entries == 0;
    if (p.wide) {
        // the columns alone make cols / 256 CTAs: rows are cut so that eight CTAs stand on an SM
        const uint64_t across = (cols + 255) / 256;
        p.parts = static_cast<uint32_t>(std::min<uint64_t>(rows, std::max<uint64_t>(1, 8 * SMS / across)));
        p.c_floats = 2 * rows;
    } else {
        p.entries = q.entries;
        p.warps = q.warps;
        p.groups = q.groups;
        p.parts = q.ctas;
    }
    p.part_floats = 2ull * p.parts * cols;
    return p;
}

template <typename G>
cudaError_t launch_sum(const float *parts, uint32_t n, uint32_t cols, void *dweight, void *dbias, int accumulate, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((cols + 31) / 32, 2);
    cfg.blockDim = dim3(1024);
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
    if (askew(ry, rx, rows) || askew(ry, ra, rows) || askew(rs, rx, rows) || askew(rs, ra, rows)) return DECO_ERR_INVALID_ARG;
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
    a.inv_cols = 1.f / static_cast<float>(cols);
    a.mean = mean;
    a.rstd = rstd;
    a.codes = codes;
    a.exps = exponents;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cols > MAX_COLS_HELD) {
        if (dtype == DECO_F32) norm_wide_kernel<float><<<static_cast<unsigned>(rows), 1024, 0, s>>>(a);
        else norm_wide_kernel<__nv_bfloat16><<<static_cast<unsigned>(rows), 1024, 0, s>>>(a);
        return result();
    }
    const bool wide = wide_rows({rx, ra, rs, ry}, dtype, cols) && aligned_to(weight, 16) && aligned_to(bias, 16);
    const cudaError_t err = dtype == DECO_F32 ? launch_norm<float>(a, wide, s) : launch_norm<__nv_bfloat16>(a, wide, s);
    return err == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}

extern "C" uint64_t deco_layernorm_grad_workspace(uint64_t rows, uint32_t cols)
{
    if (rows == 0 || rows >= MAX_ROWS || cols == 0 || cols > MAX_COLS) return 0;
    uint64_t most = 0;                                           // of all types and alignments
    for (const int32_t dtype : {DECO_F32, DECO_BF16})
        for (const bool aligned : {false, true}) most = std::max(most, grad_plan(rows, cols, dtype, aligned).bytes());
    return most;
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
    if (askew(rd, rx, rows) || askew(rd, rg, rows) || askew(rd, ra, rows)) return DECO_ERR_INVALID_ARG;
    for (const float *p : {mean, rstd, weight})
        if (!aligned_to(p, 4)) return DECO_ERR_INVALID_ARG;
    if ((codes || exponents) && bad_packed(codes, exponents)) return DECO_ERR_INVALID_ARG;
    const bool aligned = wide_rows({rx, rg, ra, rd}, dtype, cols) && aligned_to(weight, 16);
    const GradPlan plan = grad_plan(rows, cols, dtype, aligned);
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
        const cudaError_t err = dtype == DECO_F32 ? launch_grad<float>(a, plan.entries, aligned, plan.parts, block, s)
                                                  : launch_grad<__nv_bfloat16>(a, plan.entries, aligned, plan.parts, block, s);
        if (err != cudaSuccess) return DECO_ERR_CUDA;
    }
    if (plan.wide && result() != DECO_OK) return DECO_ERR_CUDA;
    if (!sums) return DECO_OK;
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
    return by_shape(wide ? 16 / unit_of(dtype) : 1, rows, cols, [&](auto v, auto g, uint64_t row_groups, uint32_t chunks, unsigned grid) {
        constexpr int V = decltype(v)::value, G = decltype(g)::value;
        if constexpr (V != 8)
            if (dtype == DECO_F32)
                pack_kernel<float, V, G><<<grid, 256, 0, s>>>(static_cast<const float *>(x), rows, x_stride, cols, row_groups, chunks, codes, exponents);
        if constexpr (V != 4)
            if (dtype == DECO_BF16)
                pack_kernel<__nv_bfloat16, V, G><<<grid, 256, 0, s>>>(static_cast<const __nv_bfloat16 *>(x), rows, x_stride, cols, row_groups,
                                                                     chunks, codes, exponents);
    });
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
    return by_shape(wide ? 16 / unit_of(dtype) : 1, rows, cols, [&](auto v, auto g, uint64_t row_groups, uint32_t chunks, unsigned grid) {
        constexpr int V = decltype(v)::value, G = decltype(g)::value;
        if constexpr (V != 8)
            if (dtype == DECO_F32)
                unpack_kernel<float, V, G><<<grid, 256, 0, s>>>(codes, exponents, rows, cols, row_groups, chunks, static_cast<float *>(y), y_stride);
        if constexpr (V != 4)
            if (dtype == DECO_BF16)
                unpack_kernel<__nv_bfloat16, V, G><<<grid, 256, 0, s>>>(codes, exponents, rows, cols, row_groups, chunks,
                                                                       static_cast<__nv_bfloat16 *>(y), y_stride);
    });
}
