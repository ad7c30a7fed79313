// deco_orth_*: orthogonalised update directions by Newton-Schulz products.
//
// For a matrix Y [rows][cols] with short side m and long side n:  X = Y / (|Y|_F + eps), then per step
//     A = X X^T   (X^T X where rows > cols),   P = a + b A + c A^2,   X <- P X   (X P).
// All matrices of a group go through a step together, in three launches: one list of output tiles
// spans matrices of every shape.  A and P are symmetric: only blocks on and below the diagonal are
// computed and the others are their mirror images.  X is kept in the orientation of Y, so nothing
// is ever transposed in memory: the tensor cores take an operand with either of its dimensions
// consecutive, and one 64 x 64 box loads both kinds.
//
// Numbers.  Operands are fp16, X scaled by 2^14, A by 2^13, P by 2^12: |X| <= 2.5 and |P| <= 15 in the spectral
// norm (checked for the coefficients in deco_orth_init), so every entry stays below 65504, and entries
// down to 3.7e-9 (A: 7.5e-9, P: 1.5e-8) keep all 11 bits.  Sums are fp32.  X is carried as hi + lo, two fp16 numbers; the
// product reads hi, and a lo is added to it.  Without lo, rounding X to 11 bits would put noise of 2^-12 |X|
// into directions in which Y has nothing, and five steps amplify those 485 times (a rank-1 matrix
// came out 15 % wrong); noise that enters through A or P stays in the row and
// column space of X and is not amplified.  The last step needs no lo: it amplifies 3.4 times.
//
// The rounding of A and P themselves reaches the result through b A and c A^2, which nearly cancel.
// Over many singular values these errors average out (1.3e-3 of the norm at a short side of 512, against
// 1.7e-3 of the rounding to bf16), over few they do not (up to 8e-3 at short sides below 16).  So
// matrices up to FULL_SIDE are multiplied in full, hi and lo of both operands (22 bits), and
// those up to WIDE_P_SIDE with P as hi + lo (1.5e-3 -> 1.2e-3 at 160).  Eight of 256 x 2048: 206 us with, 191
// without; eight of 128 x 4000: 225 and 208; twelve of 4000 x 100, the worst found: 318 and 262.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <functional>
#include <new>
#include <queue>
#include <vector>

#include "deco_internal.h"

namespace {

constexpr float X_SCALE = 16384.f, A_SCALE = 8192.f, P_SCALE = 4096.f;      // of X, A and P in fp16
constexpr float XX_TO_A = A_SCALE / (X_SCALE * X_SCALE), A_TO_P = P_SCALE / A_SCALE, AA_TO_P = A_TO_P / A_SCALE;
constexpr float INV_X_SCALE = 1.f / X_SCALE, INV_P_SCALE = 1.f / P_SCALE;
constexpr double MAX_SIGMA = 2.5, MAX_P = 15.0;
constexpr uint32_t MAX_STEPS = 16;

// ------------------------------------------------------------------ tables in device memory

struct Mat {
    uint64_t offset, stride;             // in the flat vectors
    uint32_t rows, cols;
    uint32_t ldx, lda;                   // entries between rows of X and of A, P
    __half *hi[2], *lo[2];               // X and the next X
    __half *a, *p, *a_lo, *p_lo;         // (a_lo, p_lo where the precision asks for them)
    uint32_t m, n;                       // short and long side
    uint32_t tall;                       // rows > cols
    uint32_t precision;                  // see Precision
    uint32_t spread;                     // rows not back to back
    uint32_t piece0, pieces;             // partial sums of squares
    float scale;                         // s of deco_orth_scale
};

// Consecutive entries of the flat vector that one CTA takes in: of one matrix, or of none.
struct Piece {
    uint64_t offset;
    uint32_t count;
    uint32_t slot;                       // of the partial sum; NO_SLOT: none wanted
};
// Rows of a matrix whose rows are not back to back.
struct RowPiece {
    uint32_t mat, row0, rows, slot;
};
// Rows [row0, row0 + rows) of a matrix that one CTA converts.
struct ConvertPiece {
    uint32_t mat, row0, rows, col0;
};
struct alignas(16) Tile {
    uint32_t mat;
    uint16_t tm, tn;
    uint16_t part, parts;                // of the sum over k (GRAM)
    uint32_t slot;                       // where the parts' sums go, parts > 1
    uint32_t k;                          // length of the sum; k, tall and precision as in the matrix's entry: what the
    uint16_t tall, precision;            // loading thread needs is one read away
    uint32_t unused[2];
};
static_assert(sizeof(Tile) == 32, "two 16-byte reads");

// Which operands of a matrix's products are carried as hi + lo.
enum Precision { PLAIN = 0, WIDE_P = 1, FULL = 2 };
constexpr uint32_t FULL_SIDE = 128, WIDE_P_SIDE = 256;
// A matrix's tensor maps: boxes of 64 x 64 for the operands; from BOX32 on the same with boxes of
// 32 rows for the epilogue; and A and P in boxes of 64 rows by 32 for mirror images.
enum Map { MAP_X = 0 /* hi, lo, next hi, next lo */, MAP_A = 4 /* hi, lo */, MAP_P = 6 /* hi, lo */, BOX32 = 8,
           MIRROR_A = 16, MIRROR_P = 18 /* hi, lo */, MAPS = 20 };

constexpr uint32_t NO_SLOT = 0xFFFFFFFFu;
constexpr uint32_t PIECE = 16384;
constexpr int INGEST_THREADS = 256;

// ------------------------------------------------------------------------- taking in

template <typename T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

template <int THREADS>
__device__ double block_sum(double v)
{
    __shared__ double s[THREADS / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v += s[w];
    __syncthreads();
    return v;
}

__device__ __forceinline__ float4 read4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 read4(const __nv_bfloat16 *p)
{
    const uint2 w = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xFFFF0000u));
}
__device__ __forceinline__ float4 scaled(float4 v, float w) { return make_float4(w * v.x, w * v.y, w * v.z, w * v.w); }

// What a pass takes in: an input vector, a momentum buffer, or both.
template <typename T>
struct Source {
    const T *in;                         // null: the momentum buffer holds the direction already
    float *mom;                          // null: no momentum
    float weight;                        // of the input
    float mu;
    int nesterov;
    __device__ __forceinline__ float input(uint64_t i) const { return in ? weight * to_f<T>(in[i]) : 0.f; }
    // whether entries i .. i + 3 can be read at once from every array there is
    __device__ __forceinline__ bool wide(uint64_t i) const
    {
        return (reinterpret_cast<uintptr_t>(in + i) & (4 * sizeof(T) - 1)) * (in != nullptr) == 0 &&
               (reinterpret_cast<uintptr_t>(mom + i) & 15u) * (mom != nullptr) == 0;
    }
    __device__ __forceinline__ float4 input4(uint64_t i) const { return in ? scaled(read4(in + i), weight) : make_float4(0, 0, 0, 0); }
    __device__ __forceinline__ float4 direction4(uint64_t i) const
    {
        if (!mom) return input4(i);
        const float4 m = read4(mom + i);
        if (!nesterov) return m;
        const float4 x = input4(i);
        return make_float4(__fmaf_rn(mu, m.x, x.x), __fmaf_rn(mu, m.y, x.y), __fmaf_rn(mu, m.z, x.z), __fmaf_rn(mu, m.w, x.w));
    }
    // the direction at entry i, the momentum having been updated
    __device__ __forceinline__ float direction(uint64_t i) const
    {
        if (!mom) return input(i);
        const float m = mom[i];
        return nesterov ? __fmaf_rn(mu, m, input(i)) : m;
    }
};

// M <- mu M + in over a piece, and the sum of squares of the direction in double (it neither overflows nor
// loses small entries).  Bound by memory: 12 bytes an entry with fp32 input and momentum.
template <typename T>
__global__ void __launch_bounds__(INGEST_THREADS)
ingest_kernel(const Piece *pieces, const Source<T> src, double *partial)
{
    constexpr int FLIGHT = 4;            // 16-byte reads of a thread under way
    const Piece p = pieces[blockIdx.x];
    const bool update = src.mom && src.in;
    double sum = 0;
    auto take = [&](float y) { sum = __fma_rn(static_cast<double>(y), static_cast<double>(y), sum); };
    auto single = [&](uint64_t i) {
        if (!update) return take(src.direction(i));
        const float x = src.input(i), m = __fmaf_rn(src.mu, src.mom[i], x);
        src.mom[i] = m;
        take(src.nesterov ? __fmaf_rn(src.mu, m, x) : m);
    };
    // entries before the first place where every array is aligned (none of them aligned together: all)
    uint32_t head = 0;
    while (head < 4 && head < p.count && !src.wide(p.offset + head)) ++head;
    if (head == 4) head = p.count;
    const uint32_t quads = (p.count - head) / 4;
    for (uint32_t j = threadIdx.x; j < head; j += INGEST_THREADS) single(p.offset + j);
    for (uint32_t j = head + 4 * quads + threadIdx.x; j < p.count; j += INGEST_THREADS) single(p.offset + j);
    const uint64_t first = p.offset + head;
    for (uint32_t q0 = threadIdx.x; q0 < quads; q0 += INGEST_THREADS * FLIGHT) {
        float4 x[FLIGHT], m[FLIGHT];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            const uint32_t q = q0 + f * INGEST_THREADS;
            if (q >= quads) continue;
            x[f] = src.input4(first + 4ull * q);
            if (src.mom) m[f] = read4(src.mom + first + 4ull * q);
        }
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            const uint32_t q = q0 + f * INGEST_THREADS;
            if (q >= quads) continue;
            float4 y = x[f];
            if (src.mom) {
                if (update) {
                    m[f] = make_float4(__fmaf_rn(src.mu, m[f].x, x[f].x), __fmaf_rn(src.mu, m[f].y, x[f].y),
                                       __fmaf_rn(src.mu, m[f].z, x[f].z), __fmaf_rn(src.mu, m[f].w, x[f].w));
                    *reinterpret_cast<float4 *>(src.mom + first + 4ull * q) = m[f];
                }
                y = !src.nesterov ? m[f]
                                  : make_float4(__fmaf_rn(src.mu, m[f].x, x[f].x), __fmaf_rn(src.mu, m[f].y, x[f].y),
                                                __fmaf_rn(src.mu, m[f].z, x[f].z), __fmaf_rn(src.mu, m[f].w, x[f].w));
            }
            take(y.x);
            take(y.y);
            take(y.z);
            take(y.w);
        }
    }
    if (p.slot == NO_SLOT) return;
    sum = block_sum<INGEST_THREADS>(sum);
    if (threadIdx.x == 0) partial[p.slot] = sum;
}

// The same sum for rows that are not back to back (their momentum has been updated already).
template <typename T>
__global__ void __launch_bounds__(INGEST_THREADS)
ingest_rows_kernel(const RowPiece *pieces, const Mat *mats, const Source<T> src, double *partial)
{
    const RowPiece p = pieces[blockIdx.x];
    const Mat &M = mats[p.mat];
    double sum = 0;
    for (uint32_t r = 0; r < p.rows; ++r)
        for (uint32_t j = threadIdx.x; j < M.cols; j += INGEST_THREADS) {
            const double y = src.direction(M.offset + (p.row0 + r) * M.stride + j);
            sum = __fma_rn(y, y, sum);
        }
    sum = block_sum<INGEST_THREADS>(sum);
    if (threadIdx.x == 0) partial[p.slot] = sum;
}

constexpr uint32_t CONVERT_COLS = 2048;

// X = Y / (|Y|_F + eps) as hi + lo.  Every CTA adds up its matrix's partial sums itself, in the
// same order.  The quotient is formed in double: |Y|_F may lie outside the range of fp32.
template <typename T>
__global__ void __launch_bounds__(INGEST_THREADS)
convert_kernel(const ConvertPiece *pieces, const Mat *mats, const Source<T> src, const double *partial, float eps)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const ConvertPiece p = pieces[blockIdx.x];
    const Mat &M = mats[p.mat];
    double sum = 0;
    for (uint32_t i = threadIdx.x; i < M.pieces; i += INGEST_THREADS) sum += partial[M.piece0 + i];
    const double inv = static_cast<double>(X_SCALE) / (sqrt(block_sum<INGEST_THREADS>(sum)) + static_cast<double>(eps));
    const bool plain = inv > 1e-30 && inv < 1e30;                // the factor itself is an fp32 number
    const float inv32 = static_cast<float>(inv);
    // 8 columns at a time: rows of X start on 16 bytes, and their length is rounded up to 8
    const uint32_t w = min(M.cols - p.col0, CONVERT_COLS), units = (w + 7) / 8;
    for (uint32_t e = threadIdx.x; e < p.rows * units; e += INGEST_THREADS) {
        const uint32_t r = p.row0 + e / units, c = p.col0 + (e % units) * 8;
        const uint64_t from = M.offset + r * M.stride + c, to = static_cast<uint64_t>(r) * M.ldx + c;
        float y[8];
        if (c + 8 <= M.cols && src.wide(from)) {
            const float4 a = src.direction4(from), b = src.direction4(from + 4);
            y[0] = a.x; y[1] = a.y; y[2] = a.z; y[3] = a.w;
            y[4] = b.x; y[5] = b.y; y[6] = b.z; y[7] = b.w;
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) y[j] = c + j < M.cols ? src.direction(from + j) : 0.f;
        }
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                x[k] = plain ? y[2 * j + k] * inv32 : static_cast<float>(static_cast<double>(y[2 * j + k]) * inv);
            const __half2 h = __floats2half2_rn(x[0], x[1]);
            const float2 back = __half22float2(h);
            const __half2 l = __floats2half2_rn(x[0] - back.x, x[1] - back.y);
            hi[j] = *reinterpret_cast<const uint32_t *>(&h);
            lo[j] = *reinterpret_cast<const uint32_t *>(&l);
        }
        *reinterpret_cast<uint4 *>(M.hi[0] + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4 *>(M.lo[0] + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// --------------------------------------------------------------- products on the tensor cores

enum Phase { GRAM = 0, POLY = 1, APPLY = 2 };
enum Target { NEXT_X = 0, OUT_BF16 = 1, PARAMS = 2 };

constexpr int BK = 64;                   // k per stage: 128 bytes, one swizzle row
constexpr int STAGES = 5;                // (four, and a third staging box per warp, were slower for pairs)
constexpr uint32_t OPERAND_BYTES = 128 * BK * 2;
constexpr uint32_t STAGE_BYTES = 2 * OPERAND_BYTES;
constexpr int FIRST_EPI_WARP = 4;        // warps 0: loads, 1: mma, 2: tensor memory
constexpr int EPI_WARPS = 8;             // two per quarter of the tensor memory's lanes, each half of the columns
constexpr int GEMM_THREADS = 32 * (FIRST_EPI_WARP + EPI_WARPS);
constexpr int CHUNK = 64;                // columns an epilogue warp takes at a time
constexpr uint32_t CHUNK_BYTES = 32 * CHUNK * 2;
constexpr uint32_t PART_FLOATS = 128 * 128;
constexpr uint32_t STAGING_BYTES = 2 * CHUNK_BYTES;      // of a warp
constexpr size_t GEMM_SMEM = STAGES * STAGE_BYTES + EPI_WARPS * STAGING_BYTES + 1024;

struct GemmArgs {
    const Mat *mats;
    const CUtensorMap *maps;             // [mat][MAPS]
    const Tile *tiles;
    const uint32_t *starts;              // [CTAs or pairs + 1]
    float *part_sums;                    // [slot][PART_FLOATS]
    uint32_t *arrived;                   // [slot][EPI_WARPS]: parts of a tile that are done, in its first slot
    int src;                             // which X holds the current iterate
    int read_lo, write_lo;
    float a, b, c;
    // last step
    __nv_bfloat16 *out;
    float *params;
    float lr, decay;                     // params <- params * decay - lr * s * X
    uint32_t *status;
};

struct __align__(8) Control {
    uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2], staged[EPI_WARPS];
    uint32_t tmem;
    volatile uint32_t abort;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
// the same shared-memory address in CTA 0 of the pair
__device__ __forceinline__ uint32_t leader_addr(uint32_t a)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(a));
    return r;
}

__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_addr(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(smem_addr(b)), "r"(bytes) : "memory");
}
template <int CG>
__device__ __forceinline__ void bar_arrive_leader(uint64_t *b)
{
    if (CG == 1)
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_addr(b)) : "memory");
    else
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(leader_addr(smem_addr(b))) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t *b, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_addr(b)), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait: false once the limit has passed or another role has given up; the first to give
// up leaves DECO_ERR_TIMEOUT in the status word.
__device__ __noinline__ bool bar_wait_slow(uint64_t *b, uint32_t parity, volatile uint32_t *abort, uint32_t *status)
{
    constexpr long long LIMIT = 4000000000ll;                    // clock cycles: about 2 s
    const long long t0 = clock64();
    while (!bar_try(b, parity)) {
        if (*abort) return false;
        if (clock64() - t0 > LIMIT) {
            *abort = 1;
            atomicExch(status, static_cast<uint32_t>(DECO_ERR_TIMEOUT));
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity, volatile uint32_t *abort, uint32_t *status)
{
    return bar_try(b, parity) || bar_wait_slow(b, parity, abort, status);
}

__device__ __forceinline__ void map_acquire(const CUtensorMap *map)
{
    asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;" :: "l"(map) : "memory");
}
// Box at (x, y) into this CTA's shared memory; its bytes are counted by the barrier at `bar`, which
// with CG = 2 is the leading CTA's.
template <int CG>
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, uint32_t bar)
{
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, int32_t x, int32_t y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];"
                 :: "l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}

// Shared-memory descriptor of an operand with 128-byte swizzle.  k consecutive: groups of 8 rows are
// 1024 bytes apart.  Outer dimension consecutive: 64 of it form a row, 8 k's are 1024 bytes
// apart, the next 64 of the outer dimension 8192.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, bool mn_major)
{
    uint64_t d = (addr >> 4) & 0x3FFFu;
    d |= static_cast<uint64_t>(mn_major ? 8192 >> 4 : 1) << 16;
    d |= static_cast<uint64_t>(1024 >> 4) << 32;
    d |= 1ull << 46;
    d |= 2ull << 61;
    return d;
}

template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrive at the barrier (with CG = 2: in both CTAs) once the products issued so far are done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];"
                     :: "r"(smem_addr(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     :: "r"(smem_addr(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]),
                   "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]),
                   "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]),
                   "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts16(uint32_t a, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Four 8 x 8 pieces of 2-byte numbers, transposed, and back to memory: lane l passes row l % 8 of piece l / 8.
__device__ __forceinline__ void transposed(uint32_t from, uint32_t (&v)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(from) : "memory");
}
__device__ __forceinline__ void store_pieces(uint32_t to, const uint32_t (&v)[4])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};"
                 :: "r"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ float2 half2_at(const uint4 &v, int i)
{
    const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
    return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}
template <typename H2> __device__ __forceinline__ uint32_t bits(H2 h) { return *reinterpret_cast<const uint32_t *>(&h); }

// What a tile of a phase reads: the sum over `passes` pairs of operands, pair i being
// (a + lo of a if i is in a_lo, b + lo of b if i is in b_lo), over k in [0, k) each.
struct Operands {
    const CUtensorMap *a, *b;
    bool a_mn, b_mn;                     // outer dimension consecutive in memory
    uint32_t k, passes, a_lo, b_lo;
    __device__ __forceinline__ const CUtensorMap *map_a(uint32_t i) const { return a + ((a_lo >> i) & 1); }
    __device__ __forceinline__ const CUtensorMap *map_b(uint32_t i) const { return b + ((b_lo >> i) & 1); }
    // blocks of BK in all passes, and where a part of them starts
    __device__ __forceinline__ uint32_t blocks() const { return passes * ((k + BK - 1) / BK); }
    __device__ __forceinline__ uint32_t start(uint32_t part, uint32_t parts) const { return blocks() * part / parts; }
};
template <Phase P>
__device__ __forceinline__ Operands operands(const GemmArgs &g, const Tile &tl)
{
    const CUtensorMap *at = g.maps + static_cast<uint64_t>(tl.mat) * MAPS;
    const CUtensorMap *x = at + MAP_X + 2 * g.src, *am = at + MAP_A, *pm = at + MAP_P;
    const uint32_t full = tl.precision == FULL;
    const bool tall = tl.tall != 0;
    // hi hi, hi lo, lo hi
    if (P == GRAM) return {x, x, tall, tall, tl.k, full ? 3u : 1u, 4, 2};
    if (P == POLY) return {am, am, false, false, tl.k, full ? 3u : 1u, 4, 2};
    // (P, X): hi hi, lo hi, hi lo
    const uint32_t passes = 1u + tl.precision;
    if (tall) return {x, pm, false, false, tl.k, passes, 4, 2};
    return {pm, x, false, true, tl.k, passes, 2, 4};
}

// A CTA (CG = 1: tiles of 128 x 128) or a pair of CTAs (CG = 2: 256 x 256, each CTA half of the rows of
// the tile and of either operand) works through the tiles; the epilogue of a tile runs beside
// the products of the next.
//
// Epilogue.  A warp takes 32 rows by 64 columns at a time.  What the formula adds to the product (A, or
// X's lo) comes as a box into the warp's own staging memory, loaded while the tile's products still run;
// a thread owns a row there, as in tensor memory, and puts the result in the place of the input;
// a box store writes it back.  Rows lie 128 bytes apart in the staging memory with their 16-byte units
// permuted as the box copies do it, so the row-wise accesses meet no bank conflicts.  A block's mirror
// image is transposed in 8 x 8 pieces in registers and stored as a box too: 2-byte stores
// straight to global memory made the products of A with itself 1.4 times slower.
//
// What bounds it: an SM takes in about 51 bytes of operands a cycle, 620 to 640 cycles for the 64 k on which the
// tensor cores work 512, so they are busy 80 % of the cycles with the epilogue left out and 61 % with it (A and
// X P of a decoder block, k = 5632 and 2048; 33 to 38 % at k = 768, where a tile's epilogue is as long as its
// products).  On four decoder blocks, launches one at a time and one triangle of A and P counted: A 1.20, P 1.06,
// X P 1.25 PFLOP/s, together 1.20; one block: 1.09, 0.80, 1.25, together 1.11.
template <int CG, Phase P, Target T>
__global__ void __launch_bounds__(GEMM_THREADS, 1)
gemm_kernel(const GemmArgs g)
{
    constexpr int SIDE = 128 * CG;
    extern __shared__ uint8_t raw[];
    __shared__ Control ctl;
    const uint32_t stages = (smem_addr(raw) + 1023) & ~1023u;
    const int wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if (CG == 2) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const uint32_t first = g.starts[blockIdx.x / CG], end = g.starts[blockIdx.x / CG + 1];

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            bar_init(&ctl.full[s], 1);
            bar_init(&ctl.empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(&ctl.acc_full[s], 1);
            bar_init(&ctl.acc_empty[s], EPI_WARPS * CG);
        }
        for (int w = 0; w < EPI_WARPS; ++w) bar_init(&ctl.staged[w], 1);
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == 2) {
        if (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                         :: "r"(smem_addr(&ctl.tmem)), "r"(2 * SIDE) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                         :: "r"(smem_addr(&ctl.tmem)), "r"(2 * SIDE) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        }
    }
    // Tensor maps lie in global memory, where the host has put them, perhaps over those of an earlier handle: a
    // block has to acquire each before its first use (600 cycles; all threads at once, and
    // while the launch before this one ends).
    for (uint32_t e = threadIdx.x; e < (end - first) * MAPS; e += GEMM_THREADS) {
        const uint32_t t = first + e / MAPS, mat = g.tiles[t].mat;
        if (t == first || g.tiles[t - 1].mat != mat) map_acquire(g.maps + static_cast<uint64_t>(mat) * MAPS + e % MAPS);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = ctl.tmem;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // The results of the launch before this one are read behind this, in the roles that read any: what they need
    // to know of their first tile is on hand by then.
    auto results_of_before = []() { asm volatile("griddepcontrol.wait;" ::: "memory"); };

    if (wid == 0) {
        if (lane == 0) {
            // This thread's loop is what the tensor cores wait for (a division in it cost 5 % of a large pass):
            // addresses and coordinates are carried along.
            uint32_t s = 0, parity = 1;
            const uint32_t full0 = smem_addr(ctl.full), bar0 = CG == 1 ? full0 : leader_addr(full0);
            bool ok = true;
            Tile next = g.tiles[first];
            for (uint32_t t = first; ok && t < end; ++t) {
                const Tile tl = next;
                if (t + 1 < end) next = g.tiles[t + 1];          // (there when this tile is done)
                const Operands op = operands<P>(g, tl);
                const int32_t ra = tl.tm * SIDE + rank * 128, rb = tl.tn * SIDE + rank * 128;
                const uint32_t per_pass = (op.k + BK - 1) / BK;
                const uint32_t b0 = op.start(tl.part, tl.parts), b1 = op.start(tl.part + 1, tl.parts);
                uint32_t pass = b0 / per_pass;
                int32_t k = static_cast<int32_t>((b0 - pass * per_pass) * BK);
                const CUtensorMap *ma = op.map_a(pass), *mb = op.map_b(pass);
                // an operand's 128 entries come as two boxes of 64 x 64, side by side in its outer dimension
                const int32_t a_out = op.a_mn ? 64 : 0, b_out = op.b_mn ? 64 : 0;
                if (t == first) results_of_before();
                for (uint32_t b = b0; b < b1; ++b) {
                    if (k >= static_cast<int32_t>(op.k)) {
                        k = 0;
                        pass += 1;
                        ma = op.map_a(pass);
                        mb = op.map_b(pass);
                    }
                    if (!bar_wait(&ctl.empty[s], parity, &ctl.abort, g.status)) { ok = false; break; }
                    if (rank == 0) bar_expect(&ctl.full[s], CG * STAGE_BYTES);
                    const uint32_t bar = bar0 + s * 8, st = stages + s * STAGE_BYTES;
                    const int32_t ax = op.a_mn ? ra : k, ay = op.a_mn ? k : ra, bx = op.b_mn ? rb : k, by = op.b_mn ? k : rb;
                    load_box<CG>(st, ma, ax, ay, bar);
                    load_box<CG>(st + OPERAND_BYTES / 2, ma, ax + a_out, ay + 64 - a_out, bar);
                    load_box<CG>(st + OPERAND_BYTES, mb, bx, by, bar);
                    load_box<CG>(st + OPERAND_BYTES + OPERAND_BYTES / 2, mb, bx + b_out, by + 64 - b_out, bar);
                    k += BK;
                    if (++s == STAGES) {
                        s = 0;
                        parity ^= 1;
                    }
                }
            }
            // Every copy has landed before a CTA leaves: in the normal course the products and so the
            // epilogue have waited for all of them; after a wait that ran out they get some time here.
            if (ctl.abort) {
                const long long t0 = clock64();
                while (clock64() - t0 < 20000000ll) {}
            }
        }
    } else if (wid == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t s = 0, parity = 0, n = 0;
            bool ok = true;
            Tile next = g.tiles[first];
            for (uint32_t t = first; ok && t < end; ++t, ++n) {
                const Tile tl = next;
                if (t + 1 < end) next = g.tiles[t + 1];
                const Operands op = operands<P>(g, tl);
                const uint32_t as = n & 1;
                if (!bar_wait(&ctl.acc_empty[as], ((n >> 1) & 1) ^ 1, &ctl.abort, g.status)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                // fp16 operands, fp32 sums, N and M, which dimension is consecutive
                const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(op.a_mn) << 15) |
                                       (static_cast<uint32_t>(op.b_mn) << 16) | ((SIDE >> 3) << 17) | ((SIDE >> 4) << 24);
                const uint32_t sa = op.a_mn ? 2048 >> 4 : 32 >> 4, sb = op.b_mn ? 2048 >> 4 : 32 >> 4;
                const uint64_t desc_a = operand_desc(stages, op.a_mn), desc_b = operand_desc(stages + OPERAND_BYTES, op.b_mn);
                const uint32_t blocks = op.start(tl.part + 1, tl.parts) - op.start(tl.part, tl.parts), acc = tmem + as * SIDE;
                for (uint32_t k = 0; k < blocks; ++k) {
                    if (!bar_wait(&ctl.full[s], parity, &ctl.abort, g.status)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = desc_a + s * (STAGE_BYTES >> 4), db = desc_b + s * (STAGE_BYTES >> 4);
#pragma unroll
                    for (uint32_t q = 0; q < BK / 16; ++q) mma<CG>(acc, da + q * sa, db + q * sb, idesc, (k | q) != 0);
                    mma_commit<CG>(&ctl.empty[s]);
                    if (++s == STAGES) {
                        s = 0;
                        parity ^= 1;
                    }
                }
                if (ok) mma_commit<CG>(&ctl.acc_full[as]);
            }
        }
    } else if (wid >= FIRST_EPI_WARP) {
        const int ew = wid - FIRST_EPI_WARP, quad = wid & 3, side = ew >> 2;
        // POLY adds A to the product and APPLY X's lo: these come in, and go out, through one box, what else goes out
        // through the other
        const uint32_t staging = stages + STAGES * STAGE_BYTES + ew * STAGING_BYTES;
        const uint32_t hi_buf = staging + (P == APPLY ? CHUNK_BYTES : 0), lo_buf = staging + (P == APPLY ? 0 : CHUNK_BYTES);
        const uint32_t my_row = lane * 128, perm = lane & 7;
        constexpr uint32_t CHUNKS = SIDE / 2 / CHUNK;            // of this warp, per tile
        uint32_t n = 0, loads = 0;
        bool ok = true;
        for (uint32_t t = first; ok && t < end; ++t, ++n) {
            const Tile tl = g.tiles[t];
            const Mat &M = g.mats[tl.mat];
            const uint32_t as = n & 1;
            const uint32_t rows = P == APPLY ? M.rows : M.m, cols = P == APPLY ? M.cols : M.m;
            const uint32_t r0 = tl.tm * SIDE + rank * 128 + quad * 32, r = r0 + lane;
            const uint32_t c_first = tl.tn * SIDE + side * (SIDE / 2);
            const bool full = M.precision == FULL;
            // POLY adds A (lo with full precision), APPLY adds lo of X unless the products did
            const bool in_hi = P == POLY, in_lo = P == POLY ? full : P == APPLY ? g.read_lo && !full : false;
            const bool out_lo = P == GRAM ? full : P == POLY ? M.precision != PLAIN : g.write_lo || full;
            const bool fetches = in_hi || in_lo;
            const bool live = r0 < rows;
            const CUtensorMap *maps = g.maps + static_cast<uint64_t>(tl.mat) * MAPS + BOX32;
            const CUtensorMap *in_map = maps + (P == POLY ? MAP_A : MAP_X + 2 * g.src);
            const CUtensorMap *out_map = maps + (P == GRAM ? MAP_A : P == POLY ? MAP_P : MAP_X + 2 * (g.src ^ 1));
            const uint32_t chunks = !live || c_first >= cols ? 0 : min(CHUNKS, (cols - c_first + CHUNK - 1) / CHUNK);
            auto fetch = [&](uint32_t c0) {                      // lane 0: the chunk's input, once the staging memory is free
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                bar_expect(&ctl.staged[ew], in_hi && in_lo ? 2 * CHUNK_BYTES : CHUNK_BYTES);
                const uint32_t bar = smem_addr(&ctl.staged[ew]);
                if (in_hi) load_box<1>(hi_buf, in_map, c0, r0, bar);
                if (in_lo) load_box<1>(lo_buf, in_map + 1, c0, r0, bar);
            };
            if (t == first) results_of_before();
            if (fetches && chunks && lane == 0) fetch(c_first);
            ok = bar_wait(&ctl.acc_full[as], (n >> 1) & 1, &ctl.abort, g.status);
            if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
            for (uint32_t ch = 0; ch < chunks; ++ch) {
                const uint32_t c0 = c_first + ch * CHUNK;
                const uint32_t acc_at = tmem + (static_cast<uint32_t>(quad * 32) << 16) + as * SIDE + side * (SIDE / 2) + ch * CHUNK;
                const bool split = P == GRAM && CG == 1 && tl.parts > 1;
                float4 *sums = nullptr;
                if (split) {
                    // A part's sums are left in memory; the warp that comes last of its tile's parts adds them up, in
                    // the order of the parts whoever it is, and goes on with the total.
                    sums = reinterpret_cast<float4 *>(g.part_sums + static_cast<uint64_t>(tl.slot) * PART_FLOATS + ew * 2048) + lane;
                    float4 *mine = sums + static_cast<uint64_t>(tl.part) * (PART_FLOATS / 4);
#pragma unroll
                    for (uint32_t h = 0; h < 2; ++h) {
                        uint32_t v[32];
                        __syncwarp();
                        tmem_load32(acc_at + h * 32, v);
#pragma unroll
                        for (uint32_t u = 0; u < 8; ++u)
                            __stcg(mine + (h * 8 + u) * 32, make_float4(__uint_as_float(v[4 * u]), __uint_as_float(v[4 * u + 1]),
                                                                        __uint_as_float(v[4 * u + 2]), __uint_as_float(v[4 * u + 3])));
                    }
                    __threadfence();
                    __syncwarp();
                    uint32_t before = 0;
                    uint32_t *count = g.arrived + static_cast<uint64_t>(tl.slot) * EPI_WARPS + ew;
                    if (lane == 0) before = atomicAdd(count, 1u);
                    before = __shfl_sync(0xFFFFFFFFu, before, 0);
                    if (before + 1 != tl.parts) continue;
                    if (lane == 0) *count = 0;                   // for the next launch
                    __threadfence();
                }
                if (fetches) {
                    if (ch && lane == 0) fetch(c0);
                    ok = bar_wait(&ctl.staged[ew], loads & 1, &ctl.abort, g.status);
                    if (!__all_sync(0xFFFFFFFFu, ok)) { ok = false; break; }
                    loads += 1;
                }
#pragma unroll
                for (uint32_t h = 0; h < 2; ++h) {
                    uint32_t v[32];
                    if (!split) {
                        __syncwarp();
                        tmem_load32(acc_at + h * 32, v);
                    } else {
#pragma unroll
                        for (uint32_t u = 0; u < 8; ++u) {
                            float4 a = make_float4(0, 0, 0, 0);
                            for (uint32_t q = 0; q < tl.parts; ++q) {
                                const float4 x = __ldcg(sums + static_cast<uint64_t>(q) * (PART_FLOATS / 4) + (h * 8 + u) * 32);
                                a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
                            }
                            v[4 * u] = __float_as_uint(a.x);
                            v[4 * u + 1] = __float_as_uint(a.y);
                            v[4 * u + 2] = __float_as_uint(a.z);
                            v[4 * u + 3] = __float_as_uint(a.w);
                        }
                    }
                    if (h == 0 && !fetches) {                    // the boxes written next may still be on their way out
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        __syncwarp();
                    }
#pragma unroll
                    for (uint32_t u = 0; u < 4; ++u) {
                        const uint32_t at = my_row + (((h * 4 + u) ^ perm) << 4);
                        uint4 ih = make_uint4(0, 0, 0, 0), il = ih;
                        if (in_hi) ih = lds16(hi_buf + at);
                        if (in_lo) il = lds16(lo_buf + at);
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 a = half2_at(ih, i), b = half2_at(il, i);
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const float acc = __uint_as_float(v[u * 8 + 2 * i + j]);
                                const float in = j ? a.y + b.y : a.x + b.x;
                                float y;
                                if (P == GRAM) y = acc * XX_TO_A;
                                else if (P == POLY) y = __fmaf_rn(g.c * AA_TO_P, acc, (g.b * A_TO_P) * in);
                                else y = __fmaf_rn(g.a, in, acc * INV_P_SCALE);
                                if (P == POLY && c0 + h * 32 + u * 8 + 2 * i + j == r) y += g.a * P_SCALE;
                                x[2 * i + j] = y;
                            }
                        }
                        if (T == NEXT_X) {
                            uint32_t oh[4], ol[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const __half2 hh = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                                const float2 back = __half22float2(hh);
                                oh[i] = bits(hh);
                                ol[i] = bits(__floats2half2_rn(x[2 * i] - back.x, x[2 * i + 1] - back.y));
                            }
                            sts16(hi_buf + at, make_uint4(oh[0], oh[1], oh[2], oh[3]));
                            if (out_lo) sts16(lo_buf + at, make_uint4(ol[0], ol[1], ol[2], ol[3]));
                        } else if (T == OUT_BF16) {
                            const float s = M.scale * INV_X_SCALE;
                            uint32_t o[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[i] = bits(__floats2bfloat162_rn(s * x[2 * i], s * x[2 * i + 1]));
                            sts16(hi_buf + at, make_uint4(o[0], o[1], o[2], o[3]));
                        } else {
                            const float s = M.scale * INV_X_SCALE;
                            uint32_t o[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(s * x[i]);
                            sts16(hi_buf + at, make_uint4(o[0], o[1], o[2], o[3]));
                            sts16(lo_buf + at, make_uint4(o[4], o[5], o[6], o[7]));
                        }
                    }
                }
                if (T == NEXT_X) {
                    const bool mirror = P != APPLY && tl.tm != tl.tn;
                    const CUtensorMap *image = maps - BOX32 + (P == GRAM ? MIRROR_A : MIRROR_P);
                    // row c of the mirror image is 64 bytes, its 16-byte units permuted; four 8 x 8 pieces at a time
                    auto piece_at = [&](uint32_t u) {
                        const uint32_t c = u * 8 + (lane & 7);
                        return c * 64 + (((lane >> 3) ^ ((c >> 1) & 3)) << 4);
                    };
                    if (mirror && !out_lo) {                     // through the half that lo does not need
                        __syncwarp();
#pragma unroll
                        for (uint32_t u = 0; u < 8; ++u) {
                            uint32_t v[4];
                            transposed(hi_buf + my_row + ((u ^ perm) << 4), v);
                            store_pieces(lo_buf + piece_at(u), v);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        store_box(out_map, c0, r0, hi_buf);
                        if (out_lo) store_box(out_map + 1, c0, r0, lo_buf);
                        if (mirror && !out_lo) store_box(image, r0, c0, lo_buf);
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                    if (mirror && out_lo) {                      // each half once more, when its box is on its way
#pragma unroll 1
                        for (uint32_t which = 0; which < 2; ++which) {
                            const uint32_t buf = which ? lo_buf : hi_buf;
                            uint32_t v[8][4];
                            __syncwarp();
#pragma unroll
                            for (uint32_t u = 0; u < 8; ++u) transposed(buf + my_row + ((u ^ perm) << 4), v[u]);
                            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                            __syncwarp();
#pragma unroll
                            for (uint32_t u = 0; u < 8; ++u) store_pieces(buf + piece_at(u), v[u]);
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                            __syncwarp();
                            if (lane == 0) {
                                store_box(image + which, r0, c0, buf);
                                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                            }
                        }
                    }
                } else if (T == OUT_BF16) {
                    // rows of the flat vector: 8 lanes write 128 bytes of one, whatever its alignment allows
                    __syncwarp();
                    __nv_bfloat16 *base = g.out + M.offset + c0;
                    const bool wide = ((reinterpret_cast<uintptr_t>(base) & 15u) | (M.stride & 7u)) == 0;
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) {
                        const uint32_t rr = i * 4 + (lane >> 3), q = lane & 7;
                        if (r0 + rr >= rows || c0 + q * 8 >= cols) continue;
                        const uint4 o = lds16(hi_buf + rr * 128 + ((q ^ (rr & 7)) << 4));
                        __nv_bfloat16 *p = base + (r0 + rr) * M.stride + q * 8;
                        if (wide && c0 + q * 8 + 8 <= cols) {
                            *reinterpret_cast<uint4 *>(p) = o;
                        } else {
                            const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                            for (uint32_t j = 0; j < 8; ++j)
                                if (c0 + q * 8 + j < cols)
                                    reinterpret_cast<unsigned short *>(p)[j] = static_cast<unsigned short>(w[j >> 1] >> (16 * (j & 1)));
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                } else {
                    __syncwarp();
                    float *base = g.params + M.offset + c0;
                    const bool wide = ((reinterpret_cast<uintptr_t>(base) & 15u) | (M.stride & 3u)) == 0;
#pragma unroll 4
                    for (uint32_t i = 0; i < 16; ++i) {
                        const uint32_t rr = i * 2 + (lane >> 4), q = lane & 15;
                        if (r0 + rr >= rows || c0 + q * 4 >= cols) continue;
                        const uint4 o = lds16((q & 1 ? lo_buf : hi_buf) + rr * 128 + (((q >> 1) ^ (rr & 7)) << 4));
                        const float y[4] = {__uint_as_float(o.x), __uint_as_float(o.y), __uint_as_float(o.z), __uint_as_float(o.w)};
                        float *p = base + (r0 + rr) * M.stride + q * 4;
                        if (wide && c0 + q * 4 + 4 <= cols) {
                            float4 x = *reinterpret_cast<float4 *>(p);
                            x.x = __fmaf_rn(-g.lr, y[0], g.decay * x.x);
                            x.y = __fmaf_rn(-g.lr, y[1], g.decay * x.y);
                            x.z = __fmaf_rn(-g.lr, y[2], g.decay * x.z);
                            x.w = __fmaf_rn(-g.lr, y[3], g.decay * x.w);
                            *reinterpret_cast<float4 *>(p) = x;
                        } else {
#pragma unroll
                            for (uint32_t j = 0; j < 4; ++j)
                                if (c0 + q * 4 + j < cols) p[j] = __fmaf_rn(-g.lr, y[j], g.decay * p[j]);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive_leader<CG>(&ctl.acc_empty[as]);
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    if (wid == 2) {
        if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(2 * SIDE));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(2 * SIDE));
    }
}

// ------------------------------------------------------------- short sides: one launch for it all

// Matrices with a short side of at most FULL_SIDE whose entries fit the shared memory of a cluster go
// through all steps in one launch.  The long side is cut into tiles of 128, dealt to the cluster's CTAs;
// a CTA keeps its part of X, hi and lo, as rows along the long side.  Per step it forms its part of
// A (products over its tiles); in a cluster the parts are added through distributed shared memory, every CTA adding
// up its share of the entries and handing the sums to all, in a fixed order, and then makes P and the
// products with its own part by itself.  All products are taken in full (hi hi + hi lo + lo hi).  What bounds this
// kernel is the chain of products and epilogues, each waiting for the one before it, not bytes.  64 x 147, one
// CTA, 36 us a pass; cycles of a step: A 2640 and its epilogue 510, A^2 1050, P 1050, X P 1940, X 1450, together 8900
// (23 us in five steps; the rest is the launch, the norm and the writing).  64 x 1000, a cluster of four: 12300, of
// which 3500 are the exchange of A's parts with its two cluster barriers.  128 x 128: 10900.  The 17 launches of
// the general way took 111 us for 64 x 147.

constexpr int NARROW_THREADS = 512;
constexpr uint32_t NARROW_TILE_LIMIT = 5;        // tiles of 128 per CTA at short sides up to 64
constexpr uint32_t NARROW_MAX_CLUSTER = 8;

struct NarrowArgs {
    const Mat *mats;
    const uint32_t *list;                // matrices, one per cluster
    float coef[3 * MAX_STEPS];
    uint32_t steps;
    float eps;
    __nv_bfloat16 *out;
    float *params;
    float lr, decay;
    uint32_t *status;
};

struct NarrowControl {
    uint64_t done;
    double sum;
    uint32_t tmem;
    volatile uint32_t abort;
};

// (All lanes of a warp must come to an .aligned instruction together, whatever loop they leave before it.)
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t a, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 peer_load(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void peer_store(uint32_t a, uint4 v)
{
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[2][8])
{
    uint32_t u[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
                   "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i >> 3][i & 7] = __uint_as_float(u[i]);
}
// 8 numbers as hi and lo fp16
__device__ __forceinline__ void split8(const float (&x)[8], uint4 &hi, uint4 &lo)
{
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 a = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        const float2 back = __half22float2(a);
        h[i] = bits(a);
        l[i] = bits(__floats2half2_rn(x[2 * i] - back.x, x[2 * i + 1] - back.y));
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void join8(uint4 hi, uint4 lo, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = half2_at(hi, i), b = half2_at(lo, i);
        x[2 * i] = a.x + b.x;
        x[2 * i + 1] = a.y + b.y;
    }
}

// Shared memory, each part 1024-byte aligned: X hi, X lo (64 columns of the short side per block: rows of
// 128 bytes, tiles * 128 of them), then A or P hi, lo (blocks of 128 rows), then this CTA's part of A in fp32.
struct NarrowLayout {
    uint32_t blocks, x_block, x, ab, part, total;
    __host__ __device__ NarrowLayout(uint32_t side, uint32_t tiles)
    {
        blocks = side <= 64 ? 1 : 2;
        x_block = tiles * 128 * 128;
        x = blocks * x_block;
        ab = blocks * 128 * 128;
        part = side * side * 4;
        total = 2 * x + 2 * ab + part + 1024;
    }
};

// Dynamic shared memory is rounded up to this, so that an SM never holds two of these CTAs: each takes all of
// the tensor memory, and CTAs of two clusters waiting for each other's would wait for good.
constexpr uint32_t NARROW_MIN_SMEM = 120 * 1024;

// Smallest power of two of CTAs, at most NARROW_MAX_CLUSTER, that leaves each at most two tiles (one, where shared
// memory holds no more; with the largest cluster up to NARROW_TILE_LIMIT).  A second tile costs a CTA 2400 cycles
// a step (64 x 256 against 64 x 128), a cluster's exchange 3500.
uint32_t narrow_cluster(uint32_t m, uint32_t n)
{
    uint32_t c = 1;
    while (c < NARROW_MAX_CLUSTER && c * (m <= 64 ? 256 : 128) < n) c *= 2;
    return c;
}
uint32_t narrow_tiles(uint32_t m, uint32_t n)
{
    const uint32_t c = narrow_cluster(m, n);
    return ((n + 127) / 128 + c - 1) / c;
}
bool is_narrow(uint32_t m, uint32_t n) { return m <= FULL_SIDE && narrow_tiles(m, n) <= (m <= 64 ? NARROW_TILE_LIMIT : 1); }

// C: CTAs per matrix
template <typename T, uint32_t C>
__global__ void __launch_bounds__(NARROW_THREADS, 1)
narrow_kernel(const NarrowArgs g, const Source<T> src)
{
    extern __shared__ uint8_t raw[];
    __shared__ NarrowControl ctl;
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31, quad = wid & 3, part_of = wid >> 2;
    const uint32_t rank = C == 1 ? 0 : blockIdx.x % C;
    const Mat &M = g.mats[g.list[blockIdx.x / C]];
    const uint32_t m = M.m, n = M.n, side = (m + 15) & ~15u;
    const bool tall = M.tall;
    const uint32_t all_tiles = (n + 127) / 128, per = (all_tiles + C - 1) / C;
    const uint32_t tile0 = min(rank * per, all_tiles), tiles = min(per, all_tiles - tile0);
    const uint32_t j0 = tile0 * 128, count = min(n - min(n, j0), tiles * 128);       // this CTA's share of the long side
    const NarrowLayout L(side, per);
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t x_hi = base, x_lo = x_hi + L.x, ab_hi = x_lo + L.x, ab_lo = ab_hi + L.ab, part = ab_lo + L.ab;

    if (tid == 0) {
        bar_init(&ctl.done, 1);
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == 0) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_addr(&ctl.tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }

    // ---- momentum and norm
    auto place = [&](uint32_t i, uint32_t j) { return M.offset + (tall ? j * M.stride + i : i * M.stride + j); };
    const bool update = src.mom && src.in && !M.spread;
    // X starts as zeros: what lies beyond the matrix stays zero
    for (uint32_t b = tid * 16; b < 2 * L.x + 2 * L.ab; b += NARROW_THREADS * 16) sts16(base + b, make_uint4(0, 0, 0, 0));
    __syncthreads();
    // Not before the tensor memory is taken: a dependent launch with tensor memory of its own could
    // come to hold columns here that the allocation above waits for, while it waits for this launch.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // A warp per row of memory (short rows: several), many entries of a lane under way.  The entries wait
    // in the places of their hi and lo for the norm, upper and lower half of the fp32 number.
    const uint32_t fast = tall ? m : count, slow = tall ? count : m;
    const uint64_t origin = M.offset + (tall ? j0 * M.stride : j0);
    uint32_t width = 1;                                          // lanes of a row
    while (width < 32 && width < fast) width *= 2;
    const uint32_t rows_at_once = NARROW_THREADS / width;
    auto spot = [&](uint32_t q, uint32_t p) {
        const uint32_t i = tall ? p : q, j = tall ? q : p;
        return (i >> 6) * L.x_block + j * 128 + ((((i & 63) >> 3) ^ (j & 7)) << 4) + (i & 7) * 2;
    };
    double sum = 0;
    constexpr uint32_t ROWS = 4, COLS = 4;                       // under way: rows and pieces of a row
    for (uint32_t q0 = tid / width; q0 < slow; q0 += rows_at_once * ROWS)
        for (uint32_t p0 = tid % width; p0 < fast; p0 += width * COLS) {
            float x[ROWS][COLS], mo[ROWS][COLS];
#pragma unroll
            for (uint32_t u = 0; u < ROWS; ++u)
#pragma unroll
                for (uint32_t v = 0; v < COLS; ++v) {
                    const uint32_t q = q0 + u * rows_at_once, p = p0 + v * width;
                    const bool there = q < slow && p < fast;
                    const uint64_t at = origin + q * M.stride + p;
                    x[u][v] = there ? src.input(at) : 0.f;
                    mo[u][v] = there && src.mom ? src.mom[at] : 0.f;
                }
#pragma unroll
            for (uint32_t u = 0; u < ROWS; ++u)
#pragma unroll
                for (uint32_t v = 0; v < COLS; ++v) {
                    const uint32_t q = q0 + u * rows_at_once, p = p0 + v * width;
                    if (q >= slow || p >= fast) continue;
                    float y = x[u][v];
                    if (src.mom) {
                        float mom = mo[u][v];
                        if (update) {
                            mom = __fmaf_rn(src.mu, mom, y);
                            src.mom[origin + q * M.stride + p] = mom;
                        }
                        y = src.nesterov ? __fmaf_rn(src.mu, mom, y) : mom;
                    }
                    sum = __fma_rn(static_cast<double>(y), static_cast<double>(y), sum);
                    const uint32_t at = spot(q, p), w = __float_as_uint(y);
                    asm volatile("st.shared.b16 [%0], %1;" :: "r"(x_hi + at), "h"(static_cast<unsigned short>(w >> 16)) : "memory");
                    asm volatile("st.shared.b16 [%0], %1;" :: "r"(x_lo + at), "h"(static_cast<unsigned short>(w)) : "memory");
                }
        }
    sum = block_sum<NARROW_THREADS>(sum);
    if (tid == 0) ctl.sum = sum;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = ctl.tmem;
    if (C > 1) {
        cluster_sync();
        sum = 0;
        for (uint32_t o = 0; o < C; ++o) {
            double s;
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(s) : "r"(peer_addr(smem_addr(&ctl.sum), o)) : "memory");
            sum += s;
        }
    }
    const double inv = static_cast<double>(X_SCALE) / (sqrt(sum) + static_cast<double>(g.eps));
    const uint32_t units = side / 8;                             // 8 columns each
    for (uint32_t e = tid; e < count * units; e += NARROW_THREADS) {
        const uint32_t u = e / count, j = e - u * count;
        const uint32_t at = (u >> 3) * L.x_block + j * 128 + (((u & 7) ^ (j & 7)) << 4);
        const uint4 a = lds16(x_hi + at), b = lds16(x_lo + at);
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = static_cast<float>(static_cast<double>(__uint_as_float((aw[i] << 16) | (bw[i] & 0xFFFFu))) * inv);
            x[2 * i + 1] = static_cast<float>(static_cast<double>(__uint_as_float((aw[i] & 0xFFFF0000u) | (bw[i] >> 16))) * inv);
        }
        uint4 hi, lo;
        split8(x, hi, lo);
        sts16(x_hi + at, hi);
        sts16(x_lo + at, lo);
    }

    // ---- steps
    uint32_t phase = 0;
    bool ok = true;
    // every thread's writes to the operands, then the products of thread 0, then everyone waits for them
    auto products = [&](auto issue) {
        __syncwarp();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        if (tid == 0) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            issue();
            mma_commit<1>(&ctl.done);
        }
        __syncwarp();
        ok = ok && bar_wait(&ctl.done, phase & 1, &ctl.abort, g.status);
        phase += 1;
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    const uint32_t row_tmem = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t d_apply = 128;                                // columns 0 .. 127: A, A^2;  from 128: products with X
    const uint32_t groups = side / 16;                           // 16 columns each: what a warp takes at a time
    const uint32_t i_row = quad * 32 + lane;                     // this thread's row of A and P
    const uint32_t idesc = (1u << 4) | ((side >> 3) << 17) | ((128 >> 4) << 24);
    // A's operands have the short side consecutive; with one block of it, rows beyond repeat the first
    const uint64_t lbo = static_cast<uint64_t>(L.blocks == 2 ? L.x_block >> 4 : 0) << 16;
    const uint64_t gram_hi = (operand_desc(x_hi, false) & ~(0x3FFFull << 16)) | lbo;
    const uint64_t gram_lo = (operand_desc(x_lo, false) & ~(0x3FFFull << 16)) | lbo;
    const uint64_t ap_hi = operand_desc(ab_hi, false), ap_lo = operand_desc(ab_lo, false);
    auto unit_at = [&](uint32_t u, uint32_t row, uint32_t block) { return (u >> 3) * block + row * 128 + (((u & 7) ^ (row & 7)) << 4); };
#pragma unroll 1
    for (uint32_t st = 0; st < g.steps; ++st) {
        const float ca = g.coef[3 * st], cb = g.coef[3 * st + 1], cc = g.coef[3 * st + 2];
        products([&]() {
#pragma unroll 4
            for (uint32_t k = 0; k < tiles * 8; ++k) {
                mma<1>(tmem, gram_hi + k * 128, gram_hi + k * 128, idesc | (3u << 15), k);
                mma<1>(tmem, gram_hi + k * 128, gram_lo + k * 128, idesc | (3u << 15), 1);
                mma<1>(tmem, gram_lo + k * 128, gram_hi + k * 128, idesc | (3u << 15), 1);
            }
        });
        for (uint32_t q = part_of; q < groups; q += NARROW_THREADS / 128) {
            float v[2][8] = {};
            __syncwarp();
            if (tiles) tmem_load16(row_tmem + q * 16, v);
            if (i_row >= side) continue;
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                const uint32_t u = q * 2 + k;
                if (C == 1) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[k][e] *= XX_TO_A;
                    uint4 hi, lo;
                    split8(v[k], hi, lo);
                    sts16(ab_hi + unit_at(u, i_row, 128 * 128), hi);
                    sts16(ab_lo + unit_at(u, i_row, 128 * 128), lo);
                } else {
                    // 16-byte units of a row permuted within groups of 4: few bank conflicts between rows
                    const uint32_t perm = i_row & 3, at = part + i_row * side * 4;
#pragma unroll
                    for (uint32_t e = 0; e < 2; ++e)
                        sts16(at + (((2 * u + e) ^ perm) << 4),
                              make_uint4(__float_as_uint(v[k][4 * e]), __float_as_uint(v[k][4 * e + 1]),
                                         __float_as_uint(v[k][4 * e + 2]), __float_as_uint(v[k][4 * e + 3])));
                }
            }
        }
        if (C > 1) {
            cluster_sync();
            // This CTA's share: side * units / C pieces of 8 entries, back to back, so that a warp reads and
            // writes consecutive memory of one CTA at a time; the parts are added in the CTAs' order.
            const uint32_t share = side * units / C;
            for (uint32_t e = rank * share + tid; e < (rank + 1) * share; e += NARROW_THREADS) {
                const uint32_t i = e / units, u = e - i * units, perm = i & 3;
                float4 a[C], b[C];
#pragma unroll
                for (uint32_t o = 0; o < C; ++o) {
                    const uint32_t p = peer_addr(part + i * side * 4, o);
                    a[o] = peer_load(p + (((2 * u) ^ perm) << 4));
                    b[o] = peer_load(p + (((2 * u + 1) ^ perm) << 4));
                }
                float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (uint32_t o = 0; o < C; ++o) {
                    v[0] += a[o].x; v[1] += a[o].y; v[2] += a[o].z; v[3] += a[o].w;
                    v[4] += b[o].x; v[5] += b[o].y; v[6] += b[o].z; v[7] += b[o].w;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= XX_TO_A;
                uint4 hi, lo;
                split8(v, hi, lo);
                const uint32_t to = unit_at(u, i, 128 * 128);
#pragma unroll
                for (uint32_t o = 0; o < C; ++o) {
                    peer_store(peer_addr(ab_hi + to, o), hi);
                    peer_store(peer_addr(ab_lo + to, o), lo);
                }
            }
            cluster_sync();                                      // (the readers' fence comes with the products)
        }
        // A^2, then P in the place of A
        products([&]() {
#pragma unroll 2
            for (uint32_t k = 0; k < groups; ++k) {
                const uint64_t d = static_cast<uint64_t>((k >> 2) * (128 * 128 >> 4) + (k & 3) * 2);
                mma<1>(tmem, ap_hi + d, ap_hi + d, idesc, k);
                mma<1>(tmem, ap_hi + d, ap_lo + d, idesc, 1);
                mma<1>(tmem, ap_lo + d, ap_hi + d, idesc, 1);
            }
        });
        for (uint32_t q = part_of; q < groups; q += NARROW_THREADS / 128) {
            float v[2][8];
            __syncwarp();
            tmem_load16(row_tmem + q * 16, v);
            if (i_row >= side) continue;
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                const uint32_t u = q * 2 + k, at = unit_at(u, i_row, 128 * 128);
                float x[8];
                join8(lds16(ab_hi + at), lds16(ab_lo + at), x);
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) {
                    x[e] = __fmaf_rn(cc * AA_TO_P, v[k][e], (cb * A_TO_P) * x[e]);
                    if (u * 8 + e == i_row) x[e] += ca * P_SCALE;
                }
                uint4 hi, lo;
                split8(x, hi, lo);
                sts16(ab_hi + at, hi);
                sts16(ab_lo + at, lo);
            }
        }
        // X P, tile by tile
        products([&]() {
            for (uint32_t t = 0; t < tiles; ++t) {
                const uint64_t xh = operand_desc(x_hi + t * (128 * 128), false), xl = operand_desc(x_lo + t * (128 * 128), false);
#pragma unroll 2
                for (uint32_t k = 0; k < groups; ++k) {
                    const uint64_t dx = static_cast<uint64_t>((k >> 2) * (L.x_block >> 4) + (k & 3) * 2);
                    const uint64_t dp = static_cast<uint64_t>((k >> 2) * (128 * 128 >> 4) + (k & 3) * 2);
                    mma<1>(tmem + d_apply + t * side, xh + dx, ap_hi + dp, idesc, k);
                    mma<1>(tmem + d_apply + t * side, xh + dx, ap_lo + dp, idesc, 1);
                    mma<1>(tmem + d_apply + t * side, xl + dx, ap_hi + dp, idesc, 1);
                }
            }
        });
        const bool last = st + 1 == g.steps;
        const float last_scale = M.scale * (INV_X_SCALE * INV_P_SCALE);
        for (uint32_t w = part_of; w < tiles * groups; w += NARROW_THREADS / 128) {
            const uint32_t t = w / groups, q = w - t * groups;
            float v[2][8];
            __syncwarp();
            tmem_load16(row_tmem + d_apply + t * side + q * 16, v);
            const uint32_t j = t * 128 + i_row;
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                const uint32_t u = q * 2 + k;
                if (!last) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[k][e] *= INV_P_SCALE;
                    uint4 hi, lo;
                    split8(v[k], hi, lo);
                    const uint32_t at = unit_at(u, j, L.x_block);
                    sts16(x_hi + at, hi);
                    sts16(x_lo + at, lo);
                } else if (j < count) {
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) {
                        const uint32_t i = u * 8 + e;
                        if (i >= m) break;
                        const uint64_t p = place(i, j0 + j);
                        if (g.params) g.params[p] = __fmaf_rn(-g.lr, last_scale * v[k][e], g.decay * g.params[p]);
                        else g.out[p] = __float2bfloat16_rn(last_scale * v[k][e]);
                    }
                }
            }
        }
    }
    __syncwarp();
    // the launch before this one may still run: its results are this one's to be waited for as well
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (C > 1) cluster_sync();
    if (wid == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512));
}

// ------------------------------------------------------------------- server update's own parts

// M <- mu M
__global__ void __launch_bounds__(INGEST_THREADS)
decay_kernel(float *m, uint64_t d, float mu)
{
    for (uint64_t i = blockIdx.x * static_cast<uint64_t>(INGEST_THREADS) + threadIdx.x; i < d;
         i += static_cast<uint64_t>(gridDim.x) * INGEST_THREADS)
        m[i] *= mu;
}

// M <- M + weight S for an aggregate kept as pairs (each index at most once)
__global__ void __launch_bounds__(INGEST_THREADS)
add_pairs_kernel(float *m, uint64_t d, const deco_pair *s, uint64_t positions, float weight, uint32_t *status)
{
    for (uint64_t i = blockIdx.x * static_cast<uint64_t>(INGEST_THREADS) + threadIdx.x; i < positions;
         i += static_cast<uint64_t>(gridDim.x) * INGEST_THREADS) {
        const deco_pair p = s[i];
        if (p.idx == DECO_NO_INDEX) continue;
        if (p.idx >= d) {
            atomicExch(status, static_cast<uint32_t>(DECO_ERR_DEVICE_CHECK));
            continue;
        }
        m[p.idx] = __fmaf_rn(weight, p.val, m[p.idx]);
    }
}

// x <- x decay - lr M for the entries of no matrix
__global__ void __launch_bounds__(INGEST_THREADS)
rest_kernel(const Piece *pieces, float *params, const float *m, float lr, float decay)
{
    const Piece p = pieces[blockIdx.x];
    for (uint32_t j = threadIdx.x; j < p.count; j += INGEST_THREADS) {
        const uint64_t i = p.offset + j;
        params[i] = __fmaf_rn(-lr, m[i], decay * params[i]);
    }
}

// ------------------------------------------------------------------------------------- host

// Work of one launch: where in the handle's list, how much, and by how many CTAs each.
struct Span {
    uint32_t first, count, cg;
    uint32_t starts, lanes;              // gemm_kernel: lane l takes tiles starts[l] .. starts[l + 1] - 1 of the launch
};
struct Group {
    uint32_t convert0, n_convert;        // in the handle's list
    Span phase[3];                       // GRAM, POLY, APPLY
};

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        ok = cudaGetDevice(&prev) == cudaSuccess && (prev == dev || cudaSetDevice(dev) == cudaSuccess);
    }
    ~DeviceGuard()
    {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                             const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                             CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_function()
{
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
        return nullptr;
    return reinterpret_cast<EncodeFn>(fn);
}

// A row-major fp16 matrix in boxes of 64 or 32 columns; outside of it zeros are read and nothing is written.
bool encode(EncodeFn fn, CUtensorMap *map, void *base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_cols,
            uint32_t box_rows)
{
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {ld * 2};
    const cuuint32_t box[2] = {box_cols, box_rows}, step[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
              box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

// The polynomials, in order, on [0, 1]: largest singular value met and largest |a + b t + c t^2| on the way.
bool coefficients_fit(const float *coef, uint32_t steps)
{
    double top = 1.0;
    for (uint32_t i = 0; i < steps; ++i) {
        const double a = coef[3 * i], b = coef[3 * i + 1], c = coef[3 * i + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || top > MAX_SIGMA) return false;
        // ends, extrema of x (a + b x^2 + c x^4): a + 3 b t + 5 c t^2 = 0, and of a + b t + c t^2: t = -b / 2c
        double at[5] = {0, top, 0, 0, 0};
        const double disc = 9 * b * b - 20 * a * c;
        if (c != 0 && disc >= 0) {
            const double t1 = (-3 * b + sqrt(disc)) / (10 * c), t2 = (-3 * b - sqrt(disc)) / (10 * c);
            if (t1 > 0) at[2] = sqrt(t1);
            if (t2 > 0) at[3] = sqrt(t2);
        } else if (c == 0 && b != 0 && -a / (3 * b) > 0) {
            at[2] = sqrt(-a / (3 * b));
        }
        if (c != 0 && -b / (2 * c) > 0) at[4] = sqrt(-b / (2 * c));
        double next = 0;
        for (double x : at) {
            if (x > top) continue;
            const double t = x * x, p = a + b * t + c * t * t;
            if (fabs(p) > MAX_P) return false;
            next = std::max(next, fabs(x * p));
        }
        top = next;
    }
    return true;                                                 // the last iterate is not an operand
}

}  // namespace

struct deco_orth {
    uint64_t d = 0;
    int device = 0;
    uint32_t steps = 5;
    std::vector<float> coef;
    float eps = 1e-7f, mu = 0.f;
    int nesterov = 0;
    bool strided = false;                // some matrix's rows are not back to back
    uint32_t sms = 0;
    std::vector<Group> groups;
    std::vector<Span> narrow;            // matrices of narrow_kernel, by cluster size
    uint32_t narrow_smem = 0;
    // where there are matrices of both kinds, narrow_kernel runs beside gemm_kernel
    cudaStream_t side = nullptr;
    cudaEvent_t fork = nullptr, join = nullptr;
    uint32_t n_pieces = 0, n_rest = 0, n_row_pieces = 0;
    // device memory
    uint8_t *workspace = nullptr;
    Mat *mats = nullptr;
    CUtensorMap *maps = nullptr;
    Piece *pieces = nullptr;             // of the matrices, then of the rest
    RowPiece *row_pieces = nullptr;
    ConvertPiece *convert = nullptr;
    Tile *tiles = nullptr;
    uint32_t *starts = nullptr, *narrow_list = nullptr;
    float *part_sums = nullptr;
    uint32_t *arrived = nullptr;
    double *partial = nullptr;
    uint32_t *status = nullptr;
    uint64_t device_bytes = 0, launches = 0;
};

namespace {

void release(deco_orth *h)
{
    if (h->side) cudaStreamDestroy(h->side);
    if (h->fork) cudaEventDestroy(h->fork);
    if (h->join) cudaEventDestroy(h->join);
    cudaFree(h->workspace);
    cudaFree(h->mats);
    cudaFree(h->maps);
    cudaFree(h->pieces);
    cudaFree(h->row_pieces);
    cudaFree(h->convert);
    cudaFree(h->tiles);
    cudaFree(h->starts);
    cudaFree(h->part_sums);
    cudaFree(h->arrived);
    cudaFree(h->narrow_list);
    cudaFree(h->partial);
    cudaFree(h->status);
    delete h;
}

template <typename T>
bool upload(deco_orth *h, T **dst, const std::vector<T> &v)
{
    const size_t bytes = sizeof(T) * std::max<size_t>(v.size(), 1);
    if (cudaMalloc(reinterpret_cast<void **>(dst), bytes) != cudaSuccess) return false;
    h->device_bytes += bytes;
    return v.empty() || cudaMemcpy(*dst, v.data(), sizeof(T) * v.size(), cudaMemcpyHostToDevice) == cudaSuccess;
}

void add_pieces(std::vector<Piece> &out, uint64_t lo, uint64_t hi, uint32_t *slot)
{
    for (uint64_t at = lo; at < hi; at += PIECE)
        out.push_back({at, static_cast<uint32_t>(std::min<uint64_t>(PIECE, hi - at)), slot ? (*slot)++ : NO_SLOT});
}

uint64_t span_end(const deco_matrix &m, uint64_t stride) { return m.offset + (m.rows - 1ull) * stride + m.cols; }

// Matrices inside [0, d) that share no entry.  Spans may interleave only as columns of rows of one length.
bool layout_ok(uint64_t d, const std::vector<deco_matrix> &ms)
{
    for (const deco_matrix &m : ms) {
        if (m.rows == 0 || m.cols == 0 || m.rows >= (1u << 20) || m.cols >= (1u << 20) || m.row_stride < m.cols) return false;
        if (m.offset > d || m.row_stride > (1ull << 40) || span_end(m, m.row_stride) > d) return false;
    }
    std::vector<uint32_t> order(ms.size());
    for (uint32_t i = 0; i < ms.size(); ++i) order[i] = i;
    std::sort(order.begin(), order.end(), [&](uint32_t x, uint32_t y) { return ms[x].offset < ms[y].offset; });
    std::vector<uint32_t> open;                                  // earlier matrices whose spans may reach on
    for (uint32_t i : order) {
        const deco_matrix &b = ms[i];
        std::vector<uint32_t> still;
        for (uint32_t j : open) {
            const deco_matrix &a = ms[j];
            if (span_end(a, a.row_stride) <= b.offset) continue;
            still.push_back(j);
            if (a.row_stride != b.row_stride) return false;
            const uint64_t s = a.row_stride, ca = a.offset % s, cb = b.offset % s;
            if (ca + a.cols > s || cb + b.cols > s) return false;
            if (ca < cb + b.cols && cb < ca + a.cols) {
                // same columns: rows must not meet
                const uint64_t ra = a.offset / s, rb = b.offset / s;
                if (ra < rb + b.rows && rb < ra + a.rows) return false;
            }
        }
        still.push_back(i);
        open.swap(still);
    }
    return true;
}

uint32_t passes(const Mat &M, int phase) { return phase == APPLY ? 1 + M.precision : M.precision == FULL ? 3 : 1; }

// Clock cycles of a tile of k products deep (for comparing ways to cut the work, not exact).  An SM takes in 40 to 50 bytes of operands a cycle, 4 a row and
// k: with 256 rows per CTA either way that is 10 to 13 cycles for each k of a tile, where the products take 4
// (one CTA) or 8 (a pair); measured 13 for a lone CTA, 9 to 10 with all SMs at work on pairs of
// CTAs.  Then the ends that do not overlap.
// Parts of a sum are worth their join from some length on: MIN_PART of k takes 9000 cycles, the join of four 5000.
constexpr uint32_t MAX_PARTS = 8, MIN_PART = 512;
double tile_cost(uint32_t cg, uint32_t k) { return cg == 1 ? 9.0 * k + 3000 : 10.0 * k + 4500; }

deco_status plan(deco_orth *h, const std::vector<deco_matrix> &ms, int scale, uint64_t cap, uint32_t tile_ctas)
{
    const EncodeFn enc = encode_function();
    if (!enc) return DECO_ERR_CUDA;
    const uint32_t n = static_cast<uint32_t>(ms.size());
    std::vector<Mat> mats(n);
    std::vector<uint64_t> bytes(n);
    std::vector<uint32_t> wide;                                  // matrices that go through gemm_kernel
    for (uint32_t i = 0; i < n; ++i) {
        Mat &M = mats[i];
        const deco_matrix &q = ms[i];
        M.offset = q.offset;
        M.stride = q.row_stride;
        M.rows = q.rows;
        M.cols = q.cols;
        M.tall = q.rows > q.cols;
        M.m = std::min(q.rows, q.cols);
        M.n = std::max(q.rows, q.cols);
        M.ldx = static_cast<uint32_t>(round_up(q.cols, 8));
        M.lda = static_cast<uint32_t>(round_up(M.m, 8));
        M.precision = M.m <= FULL_SIDE ? FULL : M.m <= WIDE_P_SIDE ? WIDE_P : PLAIN;
        M.spread = q.row_stride != q.cols && q.rows > 1;
        const double r = q.rows, c = q.cols;
        M.scale = scale == DECO_ORTH_SCALE_SPECTRAL ? static_cast<float>(sqrt(std::max(1.0, r / c)))
                : scale == DECO_ORTH_SCALE_RMS      ? static_cast<float>(0.2 * sqrt(std::max(r, c)))
                                                    : 1.f;
        if (is_narrow(M.m, M.n)) continue;
        bytes[i] = (M.precision == FULL ? 4 : 3) * round_up(2ull * M.rows * M.ldx, 256) +
                   (2 + M.precision) * round_up(2ull * M.m * M.lda, 256);
        wide.push_back(i);
    }
    std::vector<uint32_t> narrow_list;
    for (uint32_t c = NARROW_MAX_CLUSTER; c >= 1; c /= 2) {
        Span span = {static_cast<uint32_t>(narrow_list.size()), 0, c, 0, 0};
        for (uint32_t i = 0; i < n; ++i)
            if (is_narrow(mats[i].m, mats[i].n) && narrow_cluster(mats[i].m, mats[i].n) == c) {
                narrow_list.push_back(i);
                const NarrowLayout L((mats[i].m + 15) & ~15u, narrow_tiles(mats[i].m, mats[i].n));
                h->narrow_smem = std::max(h->narrow_smem, std::max(L.total, NARROW_MIN_SMEM));
            }
        span.count = static_cast<uint32_t>(narrow_list.size()) - span.first;
        if (span.count) h->narrow.push_back(span);
    }
    // groups, in order, of what fits the workspace
    std::vector<uint32_t> group_of(n, NO_SLOT);
    uint64_t used = 0, most = 0;
    uint32_t groups = 0;
    for (uint32_t i : wide) {
        if (groups == 0 || used + bytes[i] > cap) {
            groups += 1;
            used = 0;
        }
        group_of[i] = groups - 1;
        used += bytes[i];
        most = std::max(most, used);
    }
    if (most) {
        if (cudaMalloc(reinterpret_cast<void **>(&h->workspace), most) != cudaSuccess) return DECO_ERR_OOM;
        h->device_bytes += most;
        if (cudaMemset(h->workspace, 0, most) != cudaSuccess) return DECO_ERR_CUDA;
    }
    std::vector<CUtensorMap> maps(static_cast<uint64_t>(MAPS) * n);
    uint64_t at = 0;
    uint32_t placed = NO_SLOT;
    for (uint32_t i : wide) {
        if (group_of[i] != placed) at = 0;
        placed = group_of[i];
        Mat &M = mats[i];
        const uint64_t xb = round_up(2ull * M.rows * M.ldx, 256), ab = round_up(2ull * M.m * M.lda, 256);
        auto take = [&](uint64_t b) { __half *p = reinterpret_cast<__half *>(h->workspace + at); at += b; return p; };
        M.hi[0] = take(xb);
        M.hi[1] = take(xb);
        M.lo[0] = take(xb);
        // where only the epilogue touches lo, each entry is read and written by the same tile: one copy does
        M.lo[1] = M.precision == FULL ? take(xb) : M.lo[0];
        M.a = take(ab);
        M.p = take(ab);
        M.p_lo = M.precision >= WIDE_P ? take(ab) : nullptr;
        M.a_lo = M.precision == FULL ? take(ab) : nullptr;
        CUtensorMap *map = &maps[static_cast<uint64_t>(MAPS) * i];
        bool ok = true;
        auto both = [&](int which, __half *p, uint32_t rows, uint32_t cols, uint32_t ld) {
            ok = ok && (!p || (encode(enc, map + which, p, rows, cols, ld, 64, 64) &&
                               encode(enc, map + BOX32 + which, p, rows, cols, ld, 64, 32)));
        };
        for (int k = 0; k < 2; ++k) {
            both(MAP_X + 2 * k, M.hi[k], M.rows, M.cols, M.ldx);
            both(MAP_X + 2 * k + 1, M.lo[k], M.rows, M.cols, M.ldx);
        }
        both(MAP_A, M.a, M.m, M.m, M.lda);
        both(MAP_A + 1, M.a_lo, M.m, M.m, M.lda);
        both(MAP_P, M.p, M.m, M.m, M.lda);
        both(MAP_P + 1, M.p_lo, M.m, M.m, M.lda);
        __half *mirrored[4] = {M.a, M.a_lo, M.p, M.p_lo};
        for (int k = 0; k < 4; ++k)
            ok = ok && (!mirrored[k] || encode(enc, map + MIRROR_A + k, mirrored[k], M.m, M.m, M.lda, 32, 64));
        if (!ok) return DECO_ERR_CUDA;
    }
    // pieces: matrices whose rows are back to back, in order of their place; then everything else
    std::vector<uint32_t> order(n);
    for (uint32_t i = 0; i < n; ++i) order[i] = i;
    std::sort(order.begin(), order.end(), [&](uint32_t x, uint32_t y) { return mats[x].offset < mats[y].offset; });
    std::vector<Piece> pieces, rest;
    std::vector<RowPiece> row_pieces;
    uint32_t slot = 0;
    uint64_t end = 0;
    for (uint32_t i : order) {
        Mat &M = mats[i];
        if (M.spread) continue;
        add_pieces(rest, end, M.offset, nullptr);
        end = M.offset + static_cast<uint64_t>(M.rows) * M.cols;
        if (group_of[i] == NO_SLOT) continue;                    // narrow_kernel takes its own in
        M.piece0 = slot;
        add_pieces(pieces, M.offset, end, &slot);
        M.pieces = slot - M.piece0;
    }
    add_pieces(rest, end, h->d, nullptr);
    for (uint32_t i : order) {
        Mat &M = mats[i];
        if (!M.spread) continue;
        h->strided = true;
        if (group_of[i] == NO_SLOT) continue;
        M.piece0 = slot;
        const uint32_t per = std::max(1u, PIECE / M.cols);
        for (uint32_t r = 0; r < M.rows; r += per) row_pieces.push_back({i, r, std::min(per, M.rows - r), slot++});
        M.pieces = slot - M.piece0;
    }
    h->n_pieces = static_cast<uint32_t>(pieces.size());
    h->n_rest = static_cast<uint32_t>(rest.size());
    h->n_row_pieces = static_cast<uint32_t>(row_pieces.size());
    pieces.insert(pieces.end(), rest.begin(), rest.end());
    // tiles and convert pieces of each group, the longest products first
    std::vector<Tile> tiles;
    std::vector<ConvertPiece> convert;
    std::vector<uint32_t> starts;
    uint32_t part_slots = 0;
    for (uint32_t g = 0; g < groups; ++g) {
        Group G = {};
        G.convert0 = static_cast<uint32_t>(convert.size());
        std::vector<uint32_t> by;
        for (uint32_t i : wide) {
            if (group_of[i] != g) continue;
            by.push_back(i);
            const Mat &M = mats[i];
            for (uint32_t c = 0; c < M.cols; c += CONVERT_COLS) {
                const uint32_t per = std::max(1u, PIECE / std::min(M.cols - c, CONVERT_COLS));
                for (uint32_t r = 0; r < M.rows; r += per) convert.push_back({i, r, std::min(per, M.rows - r), c});
            }
        }
        G.n_convert = static_cast<uint32_t>(convert.size()) - G.convert0;
        for (int phase = 0; phase < 3; ++phase) {
            // longest products first, and the tile size under which the busiest CTA is done first
            auto depth = [&](uint32_t i) { return (phase == GRAM ? mats[i].n : mats[i].m) * passes(mats[i], phase); };
            std::stable_sort(by.begin(), by.end(), [&](uint32_t x, uint32_t y) { return depth(x) > depth(y); });
            double best = 0;
            std::vector<std::vector<Tile>> chosen;
            uint32_t best_slots = 0;
            // one CTA per tile, the sums of GRAM in up to MAX_PARTS parts, or a pair of CTAs per tile
            for (uint32_t way = 1; way <= (phase == GRAM ? 2 * MAX_PARTS : 2u); way *= 2) {
                const uint32_t cg = way == 2 ? 2 : 1, most_parts = way <= 2 ? 1 : way / 2, side = 128 * cg;
                if (tile_ctas != 0 && tile_ctas != cg) continue;
                auto blocks = [&](uint32_t v) { return (v + side - 1) / side; };
                // every tile, the longest first, to the lane that is free first
                std::vector<std::vector<Tile>> lanes(h->sms / cg);
                typedef std::pair<double, uint32_t> Load;
                std::priority_queue<Load, std::vector<Load>, std::greater<Load>> free;
                for (uint32_t l = 0; l < lanes.size(); ++l) free.push({0.0, l});
                double cost = 0;
                uint32_t slots = 0;
                for (uint32_t i : by) {
                    const Mat &M = mats[i];
                    const uint32_t nr = blocks(phase == APPLY ? M.rows : M.m), nc = blocks(phase == APPLY ? M.cols : M.m);
                    const uint32_t parts = std::max(1u, std::min(most_parts, depth(i) / MIN_PART));
                    for (uint32_t r = 0; r < nr; ++r)
                        for (uint32_t c = 0; c < (phase == APPLY ? nc : r + 1); ++c) {
                            for (uint32_t q = 0; q < parts; ++q) {
                                const Load at = free.top();
                                const double until = at.first + tile_cost(cg, depth(i) / parts) + (parts > 1 ? 2500 + 700 * parts : 0);
                                free.pop();
                                lanes[at.second].push_back({i, static_cast<uint16_t>(r), static_cast<uint16_t>(c),
                                                            static_cast<uint16_t>(q), static_cast<uint16_t>(parts), slots,
                                                            phase == GRAM ? M.n : M.m, static_cast<uint16_t>(M.tall),
                                                            static_cast<uint16_t>(M.precision), {0, 0}});
                                free.push({until, at.second});
                                cost = std::max(cost, until);
                            }
                            slots += parts > 1 ? parts : 0;
                        }
                }
                if (chosen.empty() || cost < best) {
                    best = cost;
                    best_slots = slots;
                    chosen.swap(lanes);
                    G.phase[phase].cg = cg;
                }
            }
            part_slots = std::max(part_slots, best_slots);
            Span &span = G.phase[phase];
            span.first = static_cast<uint32_t>(tiles.size());
            span.starts = static_cast<uint32_t>(starts.size());
            span.count = span.lanes = 0;
            for (const std::vector<Tile> &l : chosen) {
                if (l.empty()) continue;
                starts.push_back(span.count);
                tiles.insert(tiles.end(), l.begin(), l.end());
                span.count += static_cast<uint32_t>(l.size());
                span.lanes += 1;
            }
            starts.push_back(span.count);
        }
        h->groups.push_back(G);
    }
    std::vector<double> partial(slot, 0.0);
    std::vector<uint32_t> status(1, 0u), arrived(static_cast<size_t>(part_slots) * EPI_WARPS, 0u);
    if (part_slots) {
        const uint64_t part_bytes = static_cast<uint64_t>(part_slots) * PART_FLOATS * sizeof(float);
        if (cudaMalloc(reinterpret_cast<void **>(&h->part_sums), part_bytes) != cudaSuccess) return DECO_ERR_OOM;
        h->device_bytes += part_bytes;
    }
    if (!upload(h, &h->mats, mats) || !upload(h, &h->maps, maps) || !upload(h, &h->pieces, pieces) ||
        !upload(h, &h->row_pieces, row_pieces) || !upload(h, &h->convert, convert) || !upload(h, &h->tiles, tiles) ||
        !upload(h, &h->starts, starts) || !upload(h, &h->narrow_list, narrow_list) ||
        !upload(h, &h->arrived, arrived) || !upload(h, &h->partial, partial) || !upload(h, &h->status, status))
        return DECO_ERR_OOM;
    if (!h->narrow.empty() && !h->groups.empty() &&
        (cudaStreamCreateWithFlags(&h->side, cudaStreamNonBlocking) != cudaSuccess ||
         cudaEventCreateWithFlags(&h->fork, cudaEventDisableTiming) != cudaSuccess ||
         cudaEventCreateWithFlags(&h->join, cudaEventDisableTiming) != cudaSuccess))
        return DECO_ERR_CUDA;
    // the copies above may still be under way; the handle's first pass may come on any stream
    return cudaDeviceSynchronize() == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}

// What a launch returned.  An error is this pass's alone: left pending in the runtime, it would be taken for the
// next pass's, which would stop behind its update of the momentum.
cudaError_t launched(deco_orth *h, cudaError_t err)
{
    if (err == cudaSuccess) h->launches += 1;
    else cudaGetLastError();
    return err;
}

// Launched so that its start may overlap the end of the launch before it (the kernels wait for its results).
template <typename... A>
cudaError_t launch_after(deco_orth *h, void (*kernel)(A...), uint32_t grid, uint32_t threads, size_t smem, uint32_t cluster,
                         cudaStream_t s, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return launched(h, cudaLaunchKernelEx(&cfg, kernel, args...));
}

template <Phase P, Target T>
cudaError_t launch_gemm(deco_orth *h, GemmArgs g, const Span &span, cudaStream_t s)
{
    g.tiles = h->tiles + span.first;
    g.starts = h->starts + span.starts;
    const uint32_t grid = span.lanes * span.cg;
    return span.cg == 1 ? launch_after(h, gemm_kernel<1, P, T>, grid, GEMM_THREADS, GEMM_SMEM, 1, s, g)
                        : launch_after(h, gemm_kernel<2, P, T>, grid, GEMM_THREADS, GEMM_SMEM, 2, s, g);
}

template <typename T, uint32_t C>
cudaError_t launch_narrow(deco_orth *h, const NarrowArgs &a, const Source<T> &src, uint32_t count, bool first, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(count * C);
    cfg.blockDim = dim3(NARROW_THREADS);
    cfg.dynamicSmemBytes = h->narrow_smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    // the launches of one pass may run side by side; the first waits for what comes before the pass
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = first ? 1 : 2;
    return launched(h, cudaLaunchKernelEx(&cfg, narrow_kernel<T, C>, a, src));
}

template <typename T>
bool allow_narrow_smem()
{
    const int most = 227 * 1024;
    auto set = [&](void (*k)(const NarrowArgs, const Source<T>)) {
        cudaFuncAttributes fa;
        return cudaFuncGetAttributes(&fa, k) == cudaSuccess &&
               cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, most - static_cast<int>(fa.sharedSizeBytes)) == cudaSuccess;
    };
    return set(narrow_kernel<T, 1>) && set(narrow_kernel<T, 2>) && set(narrow_kernel<T, 4>) && set(narrow_kernel<T, 8>);
}

template <Phase P, Target T>
bool allow_smem()
{
    return cudaFuncSetAttribute(gemm_kernel<1, P, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(GEMM_SMEM)) == cudaSuccess &&
           cudaFuncSetAttribute(gemm_kernel<2, P, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(GEMM_SMEM)) == cudaSuccess;
}

// Everything behind the taking in: short sides on stream ns, the rest on stream s.
template <typename T>
cudaError_t run_matrices(deco_orth *h, const Source<T> &src, __nv_bfloat16 *out, float *params, float lr, float decay,
                         cudaStream_t s, cudaStream_t ns)
{
    cudaError_t err = cudaSuccess;
    NarrowArgs na = {};
    na.mats = h->mats;
    std::copy(h->coef.begin(), h->coef.end(), na.coef);
    na.steps = h->steps;
    na.eps = h->eps;
    na.out = out;
    na.params = params;
    na.lr = lr;
    na.decay = decay;
    na.status = h->status;
    for (const Span &q : h->narrow) {
        if (err != cudaSuccess) return err;
        na.list = h->narrow_list + q.first;
        const bool first = &q == &h->narrow.front();
        err = q.cg == 8   ? launch_narrow<T, 8>(h, na, src, q.count, first, ns)
              : q.cg == 4 ? launch_narrow<T, 4>(h, na, src, q.count, first, ns)
              : q.cg == 2 ? launch_narrow<T, 2>(h, na, src, q.count, first, ns)
                          : launch_narrow<T, 1>(h, na, src, q.count, first, ns);
    }
    for (const Group &G : h->groups) {
        if (err != cudaSuccess) return err;
        err = launch_after(h, convert_kernel<T>, G.n_convert, INGEST_THREADS, 0, 1, s,
                           static_cast<const ConvertPiece *>(h->convert + G.convert0), static_cast<const Mat *>(h->mats),
                           src, static_cast<const double *>(h->partial), h->eps);
        GemmArgs g = {};
        g.mats = h->mats;
        g.maps = h->maps;
        g.status = h->status;
        g.part_sums = h->part_sums;
        g.arrived = h->arrived;
        g.out = out;
        g.params = params;
        g.lr = lr;
        g.decay = decay;
        for (uint32_t i = 0; i < h->steps && err == cudaSuccess; ++i) {
            const bool last = i + 1 == h->steps;
            g.src = i & 1;
            g.read_lo = !last || h->steps == 1;                  // (see the numbers above)
            g.write_lo = i + 2 < h->steps;
            g.a = h->coef[3 * i];
            g.b = h->coef[3 * i + 1];
            g.c = h->coef[3 * i + 2];
            err = launch_gemm<GRAM, NEXT_X>(h, g, G.phase[GRAM], s);
            if (err == cudaSuccess) err = launch_gemm<POLY, NEXT_X>(h, g, G.phase[POLY], s);
            if (err != cudaSuccess) break;
            err = !last    ? launch_gemm<APPLY, NEXT_X>(h, g, G.phase[APPLY], s)
                : params   ? launch_gemm<APPLY, PARAMS>(h, g, G.phase[APPLY], s)
                           : launch_gemm<APPLY, OUT_BF16>(h, g, G.phase[APPLY], s);
        }
    }
    return err;
}

// The whole pass over what `src` describes; params: the server update's target instead of out.
template <typename T>
cudaError_t run_pass(deco_orth *h, const Source<T> &src, __nv_bfloat16 *out, float *params, float lr, float decay,
                     cudaStream_t s)
{
    const uint32_t taken = h->n_pieces + (src.mom && src.in ? h->n_rest : 0);
    if (taken) {
        ingest_kernel<T><<<taken, INGEST_THREADS, 0, s>>>(h->pieces, src, h->partial);
        h->launches += 1;
    }
    if (h->n_row_pieces) {
        ingest_rows_kernel<T><<<h->n_row_pieces, INGEST_THREADS, 0, s>>>(h->row_pieces, h->mats, src, h->partial);
        h->launches += 1;
    }
    cudaError_t err = cudaGetLastError();
    if (!h->side || err != cudaSuccess) return err != cudaSuccess ? err : run_matrices(h, src, out, params, lr, decay, s, s);
    // The handle's own stream starts where the caller's has got to, and the caller's waits for it at the end, also
    // when a launch in between has failed: what did start writes the caller's buffers.
    err = cudaEventRecord(h->fork, s);
    if (err == cudaSuccess) err = cudaStreamWaitEvent(h->side, h->fork, 0);
    if (err != cudaSuccess) return err;
    err = run_matrices(h, src, out, params, lr, decay, s, h->side);
    cudaError_t joined = cudaEventRecord(h->join, h->side);
    if (joined == cudaSuccess) joined = cudaStreamWaitEvent(s, h->join, 0);
    return err != cudaSuccess ? err : joined;
}

}  // namespace

extern "C" deco_status deco_orth_init(deco_orth **out, uint64_t d, const deco_matrix *matrices, uint32_t n_matrices,
                                      const deco_orth_options *opt)
try {
    if (!out || d == 0 || d > (1ull << 40) || (n_matrices && !matrices) || n_matrices > (1u << 24)) return DECO_ERR_INVALID_ARG;
    deco_orth_options o = {};
    if (opt) o = *opt;
    for (uint32_t r : o.reserved)
        if (r) return DECO_ERR_INVALID_ARG;
    const uint32_t steps = o.steps ? o.steps : 5;
    if (steps > MAX_STEPS || !(o.eps >= 0.f) || o.eps > 1e30f || !(o.momentum >= 0.f && o.momentum < 1.f) ||
        o.scale < DECO_ORTH_SCALE_NONE || o.scale > DECO_ORTH_SCALE_RMS || o.tile_ctas > 2)
        return DECO_ERR_INVALID_ARG;
    std::vector<float> coef(3 * steps);
    const float standard[3] = {3.4445f, -4.7750f, 2.0315f};
    for (uint32_t i = 0; i < 3 * steps; ++i) coef[i] = o.coef ? o.coef[i] : standard[i % 3];
    if (!coefficients_fit(coef.data(), steps)) return DECO_ERR_INVALID_ARG;
    std::vector<deco_matrix> ms(matrices, matrices + n_matrices);
    for (deco_matrix &m : ms)
        if (m.row_stride == 0 || m.rows == 1) m.row_stride = m.row_stride ? std::max<uint64_t>(m.row_stride, m.cols) : m.cols;
    if (!layout_ok(d, ms)) return DECO_ERR_INVALID_ARG;
    DeviceGuard guard(o.device);
    if (!guard.ok) return DECO_ERR_CUDA;
    int sms = 0;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, o.device) != cudaSuccess) return DECO_ERR_CUDA;
    if (!allow_smem<GRAM, NEXT_X>() || !allow_smem<POLY, NEXT_X>() || !allow_smem<APPLY, NEXT_X>() ||
        !allow_smem<APPLY, OUT_BF16>() || !allow_smem<APPLY, PARAMS>() || !allow_narrow_smem<float>() ||
        !allow_narrow_smem<__nv_bfloat16>())
        return DECO_ERR_CUDA;
    deco_orth *h = new deco_orth;
    deco_status st = DECO_ERR_OOM;
    try {
        h->d = d;
        h->device = o.device;
        h->steps = steps;
        h->coef = coef;
        h->eps = o.eps > 0.f ? o.eps : 1e-7f;
        h->mu = o.momentum;
        h->nesterov = o.nesterov != 0;
        h->sms = static_cast<uint32_t>(sms);
        st = plan(h, ms, o.scale, o.workspace_bytes ? o.workspace_bytes : 2ull << 30, o.tile_ctas);
    } catch (...) {
    }
    if (st != DECO_OK) {
        cudaGetLastError();
        release(h);
        return st;
    }
    *out = h;
    return DECO_OK;
} catch (...) {
    return DECO_ERR_OOM;
}

extern "C" void deco_orth_destroy(deco_orth *h)
{
    if (!h) return;
    DeviceGuard guard(h->device);
    cudaDeviceSynchronize();
    release(h);
}

extern "C" deco_status deco_orth_run(deco_orth *h, const void *in, int32_t in_dtype, float *momentum, void *out, void *stream)
{
    if (!h || !in || !out || (in_dtype != DECO_F32 && in_dtype != DECO_BF16)) return DECO_ERR_INVALID_ARG;
    const uintptr_t unit = in_dtype == DECO_F32 ? 3 : 1;
    if ((reinterpret_cast<uintptr_t>(in) & unit) || (reinterpret_cast<uintptr_t>(momentum) & 3) ||
        (reinterpret_cast<uintptr_t>(out) & 1))
        return DECO_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok) return DECO_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(out);
    cudaError_t err;
    if (in_dtype == DECO_F32)
        err = run_pass(h, Source<float>{static_cast<const float *>(in), momentum, 1.f, h->mu, h->nesterov}, o, nullptr, 0.f, 0.f, s);
    else
        err = run_pass(h, Source<__nv_bfloat16>{static_cast<const __nv_bfloat16 *>(in), momentum, 1.f, h->mu, h->nesterov}, o,
                       nullptr, 0.f, 0.f, s);
    return err == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}

deco_status deco::orth_update(deco_orth *h, const deco_ctx *c, const Slot &slot, const deco_pair *data, float *momentum,
                              float weight_decay, cudaStream_t s)
{
    const float weight = 1.f / static_cast<float>(c->n_total);
    const float decay = 1.f - c->lr * weight_decay;
    Source<float> src = {nullptr, momentum, weight, h->mu, 0};
    if (slot.dense) {
        src.in = reinterpret_cast<const float *>(data);
    } else {
        const unsigned grid = h->sms * 8;
        decay_kernel<<<grid, INGEST_THREADS, 0, s>>>(momentum, h->d, h->mu);
        add_pairs_kernel<<<grid, INGEST_THREADS, 0, s>>>(momentum, h->d, data, slot.positions, weight, h->status);
        h->launches += 2;
    }
    cudaError_t err = run_pass(h, src, nullptr, c->params, c->lr, decay, s);
    if (err == cudaSuccess && h->n_rest) {
        rest_kernel<<<h->n_rest, INGEST_THREADS, 0, s>>>(h->pieces + h->n_pieces, c->params, momentum, c->lr, decay);
        h->launches += 1;
        err = cudaGetLastError();
    }
    return err == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}

bool deco::orth_fits(const deco_orth *h, const deco_ctx *c)
{
    return h->d == c->d && h->device == c->device && !h->strided && !h->nesterov;
}

extern "C" deco_status deco_orth_get_stats(deco_orth *h, void *stream, deco_orth_stats *out)
{
    if (!h || !out) return DECO_ERR_INVALID_ARG;
    DeviceGuard guard(h->device);
    if (!guard.ok) return DECO_ERR_CUDA;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint32_t status = 0;
    if (cudaMemcpyAsync(&status, h->status, sizeof(status), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
        cudaStreamSynchronize(s) != cudaSuccess)
        return DECO_ERR_CUDA;
    out->device_bytes = h->device_bytes;
    out->launches = h->launches;
    out->groups = static_cast<uint32_t>(h->groups.size());
    out->device_status = status;
    return status ? DECO_ERR_DEVICE_CHECK : DECO_OK;
}
