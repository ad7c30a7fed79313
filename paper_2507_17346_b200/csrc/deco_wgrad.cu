// deco_weight_grad8: the weight gradient of a linear layer whose input was put away in 8 bits,
//     dW[o][i] = sum_t dY[t][o] X[t][i],   db[o] = sum_t dY[t][o],
// on the tensor cores.  X's entries, 8-bit integers times a power of two, are bf16 numbers, so the products are exact and
// X is never written out: box copies bring codes (a byte an entry) into shared memory, twelve warps make bf16 of them
// (five instructions for two) and put them in the place of the operand, while dY comes as it is.  Both operands have
// their outer dimension consecutive, 128-byte swizzle.
//
// fp32 dY is taken as the sum of bf16 numbers, hi + mid + lo (24 bits).  Where the result is bf16 hi + mid do: they leave out up
// to 2^-17 of a term, 2^-8 of what the result's own rounding may take, and save a third of the products.  They are split by a
// launch before; the same launch lays out bf16 rows that do not start on 16 bytes.
//
// db.  Sixteen columns of ones behind a CTA's columns of X in shared memory make it one more column of the
// product, for an eighth of the tensor cores' time in the tiles of the first columns, and no second pass over dY.
//
// Sums.  The tensor cores' fp32 sums are cut off, not rounded: over 8192 products the result is 9e-6 off (in the 2-norm), over
// 512 5e-7, and sums of one sign lose up to 2^-23 for every 16 products.  So the accumulators are emptied every CHUNK (fp32 results)
// or LONG_CHUNK (bf16) blocks of 64 tokens into registers, where sums are rounded; the two accumulators take turns, and the products go on.
// lo's and mid's products of a chunk come before hi's, while the sum is still small.
//
// Shares.  The blocks of all tiles in a row, cut into equal ranges, one per worker (a CTA or a pair): where whole tiles
// would leave too many idle, a worker begins and ends inside tiles.  Parts of a tile are left in the workspace, and whoever
// comes last adds them up, in their order whoever it is: the same bits every time.
//
// What bounds it (8192 x 5632 x 2048 bf16, 166 us, 1.14 PFLOP/s; tensor cores busy 70 % of the cycles): shared memory.  64 tokens of a pair's
// tile take each SM 23 KB of copies in, 8 KB of codes and steps read and 14 KB of bf16 written to convert, and 32 KB read by
// the tensor cores: 77 KB, 600 cycles at 128 bytes a cycle, where the products take 448 to 512; 640 are measured, 476 without
// conversion and copies.  In a loop the power cap is next: clocks fall to 1.5 GHz.  Short sums (8192 x 2304 x 768, 44 us): the products
// of a worker's one part 43 thousand cycles, and its end 17 to 21 thousand more if it comes last: sums to tensor memory 2.7, the part
// to memory 3 to 4, the fence 2 to 3, the other part in and the result out the rest.  Few tokens (64 x 6000 x 6000 bf16, 33 us,
// 2.2 TB/s written): instructions of the eight warps that write the result, 1000 cycles for sixteen columns.  Leaving out the stores
// alone saves nothing, shorter code does: 32 bytes a store took 41 us, one entry a store 64 (by single CTAs).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "deco.h"
#include "deco_packed8.h"
#include "deco_tensor.h"

namespace {

using namespace deco::tensor;
using deco::BLOCK8;
using deco::bf16_step;
using deco::converted;

constexpr int BK = 64;                   // tokens per stage
constexpr uint32_t TILE_M = 128;         // of dY's columns, a CTA's
constexpr uint32_t MAX_H = 112, MAX_HALF = 128;  // of X's columns, a CTA's; with those of ones
constexpr uint32_t ONES = 16;            // columns of ones, a CTA's
constexpr uint32_t SLAB = BK * 128;      // 64 columns of an operand
constexpr uint32_t OPERAND = 2 * SLAB;
// Codes of a block, tokens an odd number of 16 bytes apart (no bank conflicts), and per token the steps of up to eight times
// 16 columns, in bf16.
constexpr uint32_t CODE_BYTES = BK * MAX_H, STEP_BYTES = BK * 16, RAW_BYTES = CODE_BYTES + STEP_BYTES;
// Warps: eight empty the accumulators; twelve convert, four a block; one loads dY, one multiplies, one loads X.
constexpr int SUM_WARPS = 8, CONVERT_WARPS = 12, TEAM_WARPS = 4, TEAMS = CONVERT_WARPS / TEAM_WARPS;
constexpr uint32_t FIRST_CONVERT = SUM_WARPS, LOAD = FIRST_CONVERT + CONVERT_WARPS, MULTIPLY = LOAD + 1, LOAD_X = LOAD + 2;
constexpr int THREADS = 32 * (SUM_WARPS + CONVERT_WARPS + 4);
// Stages of dY, of X as bf16, of X as codes and steps.  The rings of X are multiples of the teams: every buffer is always
// the same team's, which so sees each of its phases.  (A wait for a phase after one that only others have waited for could
// take an older one's parity for it.)
constexpr int A_STAGES = 4, X_STAGES = 2 * TEAMS;
// Registers: a launch gives 768 threads 80 each (61440).  256 threads hold 128 sums each, the others need few:
// 256 * 168 + 384 * 32 + 128 * 48 = 61440.
constexpr int SUM_REGISTERS = 168, CONVERT_REGISTERS = 32, OTHER_REGISTERS = 48;
constexpr uint32_t STAGING_BYTES = 32 * 16 * 4;      // of a warp: 32 rows, 16 columns
constexpr size_t SMEM = A_STAGES * OPERAND + X_STAGES * (OPERAND + RAW_BYTES) + SUM_WARPS * STAGING_BYTES + 1024;
// Blocks an accumulator takes before it is emptied; LONG_CHUNK where the result is bf16: 2048 tokens' sums are cut off by at most
// 2^-16 a plane, far below half a unit of bf16, 2^-9 to 2^-8.  (8192 x 5632 x 2048 bf16 with 8, 16, 32, 64 and all 128 blocks:
// 172, 168, 166, 165 and 164 us; 0.02, 0.04, 0.08, 0.16 and 0.30 % of the entries are rounded otherwise than the exact sum.)
constexpr uint32_t CHUNK = 8, LONG_CHUNK = 32;
constexpr uint32_t SMS = 148;
constexpr uint32_t MIN_BLOCKS = 8;       // a worker's share, if tiles have to be cut for it
constexpr uint32_t PART_BLOCKS = 2, CUT_BLOCKS = 8;      // what cutting a tile costs: a part, and at all

// A tile is CG * 128 columns of dY by CG * h of X, h a multiple of 16.  A CTA (of a pair) makes the operand of h of the
// product's columns and, in tiles that sum db too, of 16 of ones behind them.
struct Args {
    const uint4 *steps;                  // [tile column's share of a CTA][k_blocks * BK] tokens: of eight times 16 columns, in bf16
    uint32_t out, cols;
    uint32_t h, code_pitch, tiles_n, k_blocks;
    uint32_t planes, plane_rows, chunk;
    uint32_t workers;                    // CTAs or pairs
    uint32_t grain;                      // ranges are whole numbers of so many blocks: 1, or k_blocks (whole tiles)
    uint64_t grains;
    void *dw, *db;
    int transposed, accumulate, wide;    // wide: not transposed, and each row of dw starts on 32 bytes
    float *slots;                        // [worker][2][CG][columns of a tile's product][TILE_M]: parts of tiles
    uint32_t *arrived;                   // [tile][CG][SUM_WARPS]: how many of a tile's parts are there
    // where a worker's range of blocks begins
    __host__ __device__ __forceinline__ uint64_t begin(uint32_t worker) const { return grains * worker / workers * grain; }
};

struct __align__(8) Control {
    uint64_t a_full[A_STAGES], a_empty[A_STAGES], b_full[X_STAGES], b_empty[X_STAGES];
    uint64_t raw_full[X_STAGES], raw_empty[X_STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem;
    volatile uint32_t abort;
};

// A worker's blocks in their order: segments of tiles, in them chunks, in those planes (the smallest first), in those blocks of
// tokens.  Every second segment goes from its last tokens to its first, so that it begins with what the last one has just
// brought into L2.  Either function may end the walk by false.
template <typename S, typename B>
__device__ __forceinline__ void walk(const Args &g, uint32_t worker, S segment, B block)
{
    const uint64_t end = g.begin(worker + 1);
    bool back = false;
    for (uint64_t u = g.begin(worker); u < end; back = !back) {
        const uint32_t tile = static_cast<uint32_t>(u / g.k_blocks);
        const uint32_t first = static_cast<uint32_t>(u - static_cast<uint64_t>(tile) * g.k_blocks);
        const uint32_t last = static_cast<uint32_t>(min(static_cast<uint64_t>(g.k_blocks), first + (end - u)));
        if (!segment(tile)) return;
        for (uint32_t c0 = first; c0 < last;) {
            const uint32_t c1 = min(c0 + g.chunk, last);
            for (uint32_t plane = g.planes; plane-- > 0;)
                for (uint32_t k = c0; k < c1; ++k)
                    if (!block(back ? first + last - 1 - k : k, plane)) return;
            c0 = c1;
        }
        u += last - first;
    }
}

// The worker whose range holds block u.
__device__ __forceinline__ uint32_t owner(const Args &g, uint64_t u)
{
    uint32_t w = static_cast<uint32_t>(u / g.grain * g.workers / g.grains);
    while (g.begin(w + 1) <= u) ++w;
    while (g.begin(w) > u) --w;
    return w;
}

// Columns of a tile's product: `width` of them, of which `in` belong to X, as column `col` of the tile.
template <int CG>
struct Columns {
    uint32_t h, half, width;
    bool ones;
    __device__ Columns(const Args &g, uint32_t nt) : h(g.h), ones(g.db && nt == 0)
    {
        half = h + (ones ? ONES : 0);
        width = CG * half;
    }
    __device__ bool in(uint32_t n) const { return n < h || (CG == 2 && n >= half && n < half + h); }
    __device__ uint32_t col(uint32_t n) const { return CG == 2 && n >= half ? n - half + h : n; }
};

template <typename G> __device__ __forceinline__ float grad_at(const G *p);
template <> __device__ __forceinline__ float grad_at<float>(const float *p) { return *p; }
template <> __device__ __forceinline__ float grad_at<__nv_bfloat16>(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put_grad(float *p, float v) { *p = v; }
__device__ __forceinline__ void put_grad(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
template <typename G> __device__ __forceinline__ void store_grad(void *base, uint64_t at, float v, int accumulate)
{
    G *p = static_cast<G *>(base) + at;
    put_grad(p, accumulate ? grad_at<G>(p) + v : v);
}

// Sixteen entries side by side, from 32 bytes' boundary on.
__device__ __forceinline__ void load_wide(const void *p, uint32_t *w)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void store_wide(void *p, const uint32_t *w)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void load16(const float *p, float *v)
{
    uint32_t w[16];
    load_wide(p, w);
    load_wide(p + 8, w + 8);
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void load16(const __nv_bfloat16 *p, float *v)
{
    uint32_t w[8];
    load_wide(p, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void store16(float *p, const float *v)
{
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(v[j]);
    store_wide(p, w);
    store_wide(p + 8, w + 8);
}
__device__ __forceinline__ void store16(__nv_bfloat16 *p, const float *v)
{
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const __nv_bfloat162 two = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t *>(&two);
    }
    store_wide(p, w);
}

// Where the 8 columns from 8 c on of token k lie in an operand's stage.
__device__ __forceinline__ uint32_t unit_offset(uint32_t k, uint32_t c)
{
    return (c >> 3) * SLAB + k * 128 + (((c & 7) ^ (k & 7)) << 4);
}

template <int CG, typename G>
__global__ void __launch_bounds__(THREADS, 1)
wgrad_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap code_map, const Args g)
{
    constexpr uint32_t SIDE = CG * 64;           // columns of the product, a warp's
    extern __shared__ uint8_t raw[];
    __shared__ Control ctl;
    const uint32_t a_at = (smem_addr(raw) + 1023) & ~1023u, b_at = a_at + A_STAGES * OPERAND, raws = b_at + X_STAGES * OPERAND;
    const uint32_t wid = threadIdx.x >> 5, lane = threadIdx.x & 31, worker = blockIdx.x / CG;
    uint32_t rank = 0;
    if (CG == 2) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    if (threadIdx.x == 0) {
        for (int s = 0; s < A_STAGES; ++s) {
            bar_init(&ctl.a_full[s], 1);
            bar_init(&ctl.a_empty[s], 1);
        }
        for (int s = 0; s < X_STAGES; ++s) {
            bar_init(&ctl.b_full[s], CG * TEAM_WARPS);
            bar_init(&ctl.b_empty[s], 1);
            bar_init(&ctl.raw_full[s], 1);
            bar_init(&ctl.raw_empty[s], TEAM_WARPS);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(&ctl.acc_full[s], 1);
            bar_init(&ctl.acc_empty[s], CG * SUM_WARPS);
        }
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (wid == MULTIPLY) tmem_alloc<CG>(&ctl.tmem, 512);
    if (g.db && threadIdx.x < BK)                                // the columns of ones, which nothing overwrites
        for (int s = 0; s < X_STAGES; ++s)
            for (uint32_t c = 0; c < ONES / 8; ++c)
                sts16(b_at + s * OPERAND + unit_offset(threadIdx.x, g.h / 8 + c),
                      make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u));
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) {
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = ctl.tmem;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (wid >= LOAD) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(OTHER_REGISTERS));
        if (wid == LOAD) {
            uint32_t s = 0, parity = 1;
            int32_t x = 0;
            const uint32_t full0 = smem_addr(ctl.a_full), bar0 = CG == 1 ? full0 : leader_addr(full0);
            walk(g, worker,
                 [&](uint32_t tile) {
                     x = ((tile / g.tiles_n) * CG + rank) * TILE_M;
                     return true;
                 },
                 [&](uint32_t k, uint32_t plane) {
                     if (!bar_wait_warp(&ctl.a_empty[s], parity, &ctl.abort)) return false;
                     if (lane == 0) {
                         const uint32_t st = a_at + s * OPERAND, bar = bar0 + s * 8;
                         const int32_t y = plane * g.plane_rows + k * BK;
                         if (rank == 0) bar_expect(&ctl.a_full[s], CG * OPERAND);
                         load_box<CG>(st, &map, x, y, bar);
                         load_box<CG>(st + SLAB, &map, x + 64, y, bar);
                     }
                     if (++s == A_STAGES) {
                         s = 0;
                         parity ^= 1;
                     }
                     return true;
                 });
            if (ctl.abort) {                                     // copies under way get time to land
                const long long t0 = clock64();
                while (clock64() - t0 < 20000000ll) {}
            }
        } else if (wid == MULTIPLY && rank == 0) {
            // This warp's loop is what the tensor cores wait for: it runs with all lanes, so that the descriptors can stay in
            // uniform registers, and one lane issues.
            const bool issues = elected();
            uint32_t sa = 0, pa = 0, sb = 0, pb = 0, n = 0;
            const uint64_t desc_a = operand_desc(a_at, true), desc_b = operand_desc(b_at, true);
            bool ok = true;
            const uint64_t end = g.begin(worker + 1);
            for (uint64_t u = g.begin(worker); ok && u < end;) {    // (as walk does; all blocks of a chunk are alike here)
                const uint32_t tile = static_cast<uint32_t>(u / g.k_blocks);
                const uint32_t first = static_cast<uint32_t>(u - static_cast<uint64_t>(tile) * g.k_blocks);
                const uint32_t last = static_cast<uint32_t>(min(static_cast<uint64_t>(g.k_blocks), first + (end - u)));
                u += last - first;
                const Columns<CG> c(g, tile % g.tiles_n);
                // bf16 operands, fp32 sums, outer dimensions consecutive, N and M
                const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((c.width >> 3) << 17) |
                                       ((CG * TILE_M >> 4) << 24);
                for (uint32_t c0 = first; ok && c0 < last; c0 += g.chunk, ++n) {
                    const uint32_t blocks = (min(c0 + g.chunk, last) - c0) * g.planes, acc = tmem + (n & 1) * 256;
                    ok = bar_wait_warp(&ctl.acc_empty[n & 1], ((n >> 1) & 1) ^ 1, &ctl.abort);
#pragma unroll 1
                    for (uint32_t b = 0; ok && b < blocks; ++b) {
                        // (both at once: a wait that need not wait takes 70 cycles)
                        const bool a_there = bar_try_cta(&ctl.a_full[sa], pa), b_there = bar_try_cta(&ctl.b_full[sb], pb);
                        ok = __all_sync(0xFFFFFFFFu, (a_there || bar_wait_cta(&ctl.a_full[sa], pa, &ctl.abort)) &&
                                                         (b_there || bar_wait_cta(&ctl.b_full[sb], pb, &ctl.abort)));
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        if (issues && ok) {
                            const uint64_t da = desc_a + sa * (OPERAND >> 4), db = desc_b + sb * (OPERAND >> 4);
#pragma unroll
                            for (uint32_t q = 0; q < BK / 16; ++q)
                                mma<CG>(acc, da + q * (2048 >> 4), db + q * (2048 >> 4), idesc, b | q);
                            mma_commit<CG>(&ctl.a_empty[sa]);
                            mma_commit<CG>(&ctl.b_empty[sb]);
                        }
                        if (++sa == A_STAGES) {
                            sa = 0;
                            pa ^= 1;
                        }
                        if (++sb == X_STAGES) {
                            sb = 0;
                            pb ^= 1;
                        }
                    }
                    if (issues && ok) mma_commit<CG>(&ctl.acc_full[n & 1]);
                }
            }
        } else if (wid == LOAD_X) {
            uint32_t s = 0, parity = 1, j = 0;
            walk(g, worker,
                 [&](uint32_t tile) {
                     j = (tile % g.tiles_n) * CG + rank;
                     return true;
                 },
                 [&](uint32_t k, uint32_t) {
                     if (!bar_wait_warp(&ctl.raw_empty[s], parity, &ctl.abort)) return false;
                     if (lane == 0) {
                         const uint32_t to = raws + s * RAW_BYTES, bar = smem_addr(&ctl.raw_full[s]);
                         bar_expect(&ctl.raw_full[s], BK * g.code_pitch + STEP_BYTES);
                         load_box<1>(to, &code_map, j * g.h, k * BK, bar);
                         load_bytes(to + CODE_BYTES, g.steps + (static_cast<uint64_t>(j) * g.k_blocks + k) * BK, STEP_BYTES, bar);
                     }
                     if (++s == X_STAGES) {
                         s = 0;
                         parity ^= 1;
                     }
                     return true;
                 });
        }
    } else if (wid >= FIRST_CONVERT) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(CONVERT_REGISTERS));
        // A team of four warps converts every third block, a thread half a token's units, eight codes each.  No bank conflicts:
        // rows of codes are an odd number of 16 bytes apart, and of eight lanes that store at a time the tokens are all even or all odd.
        const uint32_t team = (wid - FIRST_CONVERT) / TEAM_WARPS, half = lane & 1;
        const uint32_t token = ((wid - FIRST_CONVERT) % TEAM_WARPS) * 16 + (lane >> 4) * 8 + ((lane >> 1) & 3) * 2 + ((lane >> 3) & 1);
        const uint32_t per_row = g.h / 16;
        const uint64_t u0 = g.begin(worker), u1 = g.begin(worker + 1);
        const uint32_t to0 = b_at + unit_offset(token, half), from0 = raws + token * g.code_pitch + half * 8;
        uint32_t r = team, parity = 0;                           // the team's two buffers take turns
        for (uint64_t left = (u1 - u0) * g.planes, n = team; n < left; n += TEAMS) {
            const uint32_t from = from0 + r * RAW_BYTES, to = to0 + r * OPERAND;
            if (!bar_wait_warp(&ctl.raw_full[r], parity, &ctl.abort)) break;
            const uint4 st = lds16(raws + r * RAW_BYTES + CODE_BYTES + token * 16);
            const uint32_t step[4] = {st.x, st.y, st.z, st.w};
            uint2 code = lds8(from);
            if (!bar_wait_warp(&ctl.b_empty[r], parity ^ 1, &ctl.abort)) break;
#pragma unroll
            for (uint32_t c = 0; c < MAX_H / 16; ++c) {
                if (c >= per_row) break;
                const uint2 now = code;
                if (c + 1 < MAX_H / 16) code = lds8(from + (c + 1) * 16);
                const uint32_t twice = __byte_perm(step[c >> 1], 0, c & 1 ? 0x3232 : 0x1010);
                // (unit 2 c + half of the row lies at that exclusive-or token: the permutation of the row's first, turned)
                sts16((to ^ ((2 * c & 7) << 4)) + (c >> 2) * SLAB, converted(now.x, now.y, twice));
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                bar_arrive(&ctl.raw_empty[r]);
                bar_arrive_leader_cta<CG>(&ctl.b_full[r]);
            }
            r += TEAMS;
            if (r >= X_STAGES) {
                r -= X_STAGES;
                parity ^= 1;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(SUM_REGISTERS));
        const uint32_t quad = wid & 3, side = wid >> 2;          // lanes of the tensor memory, half of the columns
        float sum[SIDE];                                         // this warp's half of the columns, a row a thread
        uint32_t n = 0;
        bool dead = false;                                       // a wait has run out, NaN from here on
        const uint64_t end = g.begin(worker + 1);
        for (uint64_t u = g.begin(worker); u < end;) {           // (as walk does)
            const uint32_t tile = static_cast<uint32_t>(u / g.k_blocks), nt = tile % g.tiles_n, mt = (tile / g.tiles_n) * CG + rank;
            const uint32_t first = static_cast<uint32_t>(u - static_cast<uint64_t>(tile) * g.k_blocks);
            const uint32_t last = static_cast<uint32_t>(min(static_cast<uint64_t>(g.k_blocks), first + (end - u)));
            u += last - first;
            const Columns<CG> c(g, nt);
            const uint32_t mine = c.width > side * SIDE ? min(SIDE, c.width - side * SIDE) : 0;      // of this warp's columns
            const uint32_t lanes = tmem + ((quad * 32) << 16) + side * SIDE;
            const bool several = first + g.chunk < last;
#pragma unroll
            for (uint32_t j = 0; j < SIDE; ++j) sum[j] = 0.f;
            auto done = [&]() {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive_leader_cta<CG>(&ctl.acc_empty[n & 1]);
                n += 1;
            };
            for (uint32_t c0 = first;;) {
                if (!dead) dead = !bar_wait_warp(&ctl.acc_full[n & 1], (n >> 1) & 1, &ctl.abort);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (several) {
#pragma unroll
                    for (uint32_t p = 0; p < SIDE; p += 16) {
                        if (p >= mine) break;
                        uint32_t v[16];
                        tmem_load16(lanes + (n & 1) * 256 + p, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[p + j] += __uint_as_float(v[j]);
                    }
                }
                c0 += g.chunk;
                if (c0 >= last) break;
                done();
            }
            // The segment is complete.  Its sums go back to where its last chunk's were: from there a short loop can take them.
            const uint32_t acc = lanes + (n & 1) * 256;
            if (several) {
#pragma unroll
                for (uint32_t p = 0; p < SIDE; p += 16)
                    if (p < mine) tmem_store16(acc + p, sum + p);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            }
            const bool whole = last - first == g.k_blocks;
            const uint64_t top = static_cast<uint64_t>(tile) * g.k_blocks;
            const uint32_t a = whole ? worker : owner(g, top), b = whole ? worker : owner(g, top + g.k_blocks - 1);
            // (a range in which the tile begins has it in the second slot, one that begins inside the tile in the first)
            auto slot = [&](uint32_t w) {
                return g.slots + ((w * 2ull + (w == a)) * CG + rank) * (CG * MAX_HALF * TILE_M) + side * SIDE * TILE_M + quad * 32 + lane;
            };
            bool out = true;
            if (!whole) {
                float *to = slot(worker);
#pragma unroll 1
                for (uint32_t p = 0; p < mine; p += 16) {
                    uint32_t v[16];
                    tmem_load16(acc + p, v);
#pragma unroll
                    for (uint32_t j = 0; j < 16; ++j) __stcg(to + (p + j) * TILE_M, dead ? __uint_as_float(0x7FC00000u) : __uint_as_float(v[j]));
                }
                __threadfence();
                __syncwarp();
                uint32_t before = 0;
                if (lane == 0) before = atomicAdd(g.arrived + (static_cast<uint64_t>(tile) * CG + rank) * SUM_WARPS + wid, 1u);
                out = __shfl_sync(0xFFFFFFFFu, before, 0) == b - a;
                __threadfence();
            }
            // (Short code: what runs once per segment waits for its instructions longer than for anything else.)
            const bool two = b - a == 1;
            const float *other = slot(worker == a ? b : a);
            uint32_t thread;                                     // (so that nothing made of it takes a register before)
            asm volatile("mov.u32 %0, %%tid.x;" : "=r"(thread));
            const uint32_t l = thread & 31;
            float4 *const staging = reinterpret_cast<float4 *>(raw + (raws - smem_addr(raw)) + X_STAGES * RAW_BYTES + (thread >> 5) * STAGING_BYTES);
            const uint32_t col0 = nt * CG * g.h, o0 = mt * TILE_M + quad * 32, o = o0 + l;
            // sixteen columns from the tile's p-th on, this lane's row of them in x
            auto put = [&](uint32_t p, float (&x)[16]) {
                const uint32_t n0 = side * SIDE + p, col = col0 + c.col(n0);
                if (dead) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = __uint_as_float(0x7FC00000u);
                }
                if (c.ones && n0 == c.h) {                                           // (the columns of ones are all alike)
                    if (o < g.out) store_grad<G>(g.db, o, x[0], g.accumulate);
                    return;
                }
                if (!c.in(n0)) return;
                if (g.wide && col + 16 <= g.cols) {              // a lane writes its row's sixteen entries
                    G *const to = static_cast<G *>(g.dw) + static_cast<uint64_t>(o) * g.cols + col;
                    if (o < g.out) {
                        if (g.accumulate) {
                            float old[16];
                            load16(to, old);
#pragma unroll
                            for (int j = 0; j < 16; ++j) x[j] = old[j] + x[j];
                        }
                        store16(to, x);
                    }
                    return;
                }
                // Where this lane's sixteen entries go, `valid` of them, `step` apart: with `transposed` one of each of the sixteen
                // columns, else sixteen rows' of one of them.
                uint64_t at, step;
                uint32_t valid = 0;
                if (g.transposed) {
                    at = static_cast<uint64_t>(col) * g.out + o;
                    step = g.out;
                    if (o < g.out) valid = g.cols - min(col, g.cols);
                } else {
                    const uint32_t mine_col = col + (l & 15), row = o0 + (l >> 4);
                    at = static_cast<uint64_t>(row) * g.cols + mine_col;
                    step = 2ull * g.cols;
                    if (mine_col < g.cols && row < g.out) valid = (g.out - row + 1) / 2;
                    // through shared memory, so that neighbouring lanes write neighbouring entries (a row's four units of 16 bytes at
                    // their numbers exclusive-or half the row's)
                    __syncwarp();
#pragma unroll
                    for (uint32_t q = 0; q < 4; ++q)
                        staging[l * 4 + (q ^ ((l >> 1) & 3))] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                    __syncwarp();
                    const float *from = reinterpret_cast<const float *>(staging) + (l >> 4) * 16 + (l & 3);
#pragma unroll
                    for (uint32_t q = 0; q < 16; ++q) x[q] = from[q * 32 + (((l >> 2) ^ q) & 3) * 4];
                }
                G *const to = static_cast<G *>(g.dw) + at;
                if (g.accumulate) {
                    float old[16];
#pragma unroll
                    for (uint32_t j = 0; j < 16; ++j) old[j] = j < valid ? grad_at<G>(to + j * step) : 0.f;
#pragma unroll
                    for (uint32_t j = 0; j < 16; ++j) x[j] = old[j] + x[j];
                }
#pragma unroll
                for (uint32_t j = 0; j < 16; ++j)
                    if (j < valid) put_grad(to + j * step, x[j]);
            };
            if (two && out) {                                    // (the other part's a step ahead)
                float next[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) next[j] = __ldcg(other + j * TILE_M);
#pragma unroll 1
                for (uint32_t p = 0; p < mine; p += 16) {
                    uint32_t v[16];
                    float x[16];
                    tmem_load16(acc + p, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] = next[j] + __uint_as_float(v[j]);     // (0 + a) + b in whichever order
                    if (p + 16 < mine) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) next[j] = __ldcg(other + (p + 16 + j) * TILE_M);
                    }
                    put(p, x);
                }
                out = false;
            }
#pragma unroll 1
            for (uint32_t p = 0; out && p < mine; p += 16) {
                uint32_t v[16];
                float x[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] = 0.f;
                tmem_load16(acc + p, v);
                if (whole) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[j] += __uint_as_float(v[j]);
                } else {
#pragma unroll 1
                    for (uint32_t w = a; w <= b; w += 4) {       // (four parts' reads under way together)
                        float y[4][16];
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k) {
                            const float *part = slot(w + k) + p * TILE_M;
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                y[k][j] = w + k == worker ? __uint_as_float(v[j]) : w + k <= b ? __ldcg(part + j * TILE_M) : 0.f;
                        }
#pragma unroll
                        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
                            for (int j = 0; j < 16; ++j) x[j] += y[k][j];
                    }
                }
                put(p, x);
            }
            done();
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2) {                                               // (the pair's barriers are used until both are done)
        asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    if (wid == MULTIPLY) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free<CG>(tmem, 512);
    }
}

// What the products need besides dY and codes, by one launch.
//   Steps of X as bf16, 16 bytes per token and CTA's share of a tile's columns (0 beyond the last token).
//   The parts' counters at 0.
//   dY, where it cannot be read as it is, as bf16 rows that start on 16 bytes, in planes of which each holds what the ones
//   before it left; rows beyond the last are 0.  (8192 x 5632 fp32 in three planes: 77 us, 6.0 TB/s.)
struct PrepareArgs {
    const uint8_t *exps;
    uint32_t rows, blocks8, h, shares, tokens;
    uint4 *steps;
    uint32_t *counters, n_counters;
    uint32_t step_blocks, plane_blocks_x, plane_blocks_y;        // blocks of threads for the steps; for the planes
    const void *dy;
    uint64_t stride;
    uint32_t out, pitch, planes;
    __nv_bfloat16 *to;
};
template <typename T>
__global__ void __launch_bounds__(256)
prepare_kernel(const PrepareArgs a)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (blockIdx.x < a.step_blocks) {
        const uint32_t first = blockIdx.x * 256 + threadIdx.x, all = a.step_blocks * 256;
        for (uint32_t i = first; i < a.n_counters; i += all) a.counters[i] = 0;
        // (neighbouring threads take neighbouring shares of a token, whose bytes lie side by side)
        const uint64_t n = static_cast<uint64_t>(a.shares) * a.tokens;
        for (uint64_t i = first; i < n; i += all) {
            const uint32_t t = static_cast<uint32_t>(i / a.shares), j = static_cast<uint32_t>(i - static_cast<uint64_t>(t) * a.shares);
            uint32_t e[5];
#pragma unroll
            for (uint32_t q = 0; q < 5; ++q) {
                const uint32_t b = j * a.h / BLOCK8 + q;
                e[q] = t < a.rows && b < a.blocks8 ? bf16_step(a.exps[static_cast<uint64_t>(t) * a.blocks8 + b]) : 0u;
            }
            // a share begins at a block of 32 columns or in its middle
            uint32_t o[4];
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) o[u] = e[u] | ((j * a.h) & 16 ? e[u + 1] : e[u]) << 16;
            a.steps[static_cast<uint64_t>(j) * a.tokens + t] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        return;
    }
    __shared__ __align__(16) uint16_t staged[8][256];
    const uint32_t block = blockIdx.x - a.step_blocks, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t warp_col = (block % a.plane_blocks_x * 8 + wid) * 256, col = warp_col + lane * 8;
    if (warp_col >= a.pitch) return;
    for (uint32_t row = block / a.plane_blocks_x; row < a.tokens; row += a.plane_blocks_y) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.stride;
        uint4 *to = reinterpret_cast<uint4 *>(a.to + static_cast<uint64_t>(row) * a.pitch + col);
        if (sizeof(T) == 2) {
            // through shared memory: lanes read neighbouring entries and write eight
            const uint16_t *p = reinterpret_cast<const uint16_t *>(dy);
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                const uint32_t c = warp_col + j * 32 + lane;
                staged[wid][j * 32 + lane] = row < a.rows && c < a.out ? p[c] : uint16_t(0);
            }
            __syncwarp();
            if (col < a.pitch) *to = *reinterpret_cast<const uint4 *>(&staged[wid][lane * 8]);
            __syncwarp();
            continue;
        }
        if (col >= a.pitch) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = row < a.rows && col + j < a.out ? static_cast<float>(dy[col + j]) : 0.f;
        for (uint32_t p = 0; p < a.planes; ++p) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = v[j];
                const bool number = fabsf(x) <= 3.402823466e38f;
                // (a number that would round to infinity: the largest bf16 number, and the rest in the next plane)
                float h = __bfloat162float(__float2bfloat16_rn(x));
                if (number && fabsf(h) > 3.402823466e38f) h = copysignf(__uint_as_float(0x7F7F0000u), x);
                v[j] = number ? x - h : 0.f;
                w[j] = __float_as_uint(h) >> 16;
            }
            to[static_cast<uint64_t>(p) * a.tokens * a.pitch / 8] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
}

// ------------------------------------------------------------------------------------ host

constexpr uint64_t MAX_ROWS = 1ull << 28;
constexpr uint32_t MAX_COLS = 1u << 24;
constexpr uint64_t MAX_STRIDE = 1ull << 40;

bool aligned_to(const void *p, uintptr_t unit) { return (reinterpret_cast<uintptr_t>(p) & (unit - 1)) == 0; }
bool is_dtype(int32_t d) { return d == DECO_F32 || d == DECO_BF16; }

struct Plan {
    uint32_t planes;                     // 0: dY is read where it is
    uint32_t plane_rows, pitch;
    uint32_t cg, h, tiles_n, tiles_m, k_blocks, workers, grain;
    uint64_t tiles;
    bool cut;                            // tiles may lie in more than one range
    uint64_t plane_bytes() const { return 2ull * planes * plane_rows * pitch; }
    uint64_t slot_bytes() const { return cut ? 2ull * workers * cg * cg * MAX_HALF * TILE_M * 4 : 0; }
    uint64_t counters() const { return cut ? tiles * cg * SUM_WARPS : 0; }
    uint64_t step_bytes() const { return 16ull * tiles_n * cg * k_blocks * BK; }
    uint64_t bytes() const { return plane_bytes() + step_bytes() + slot_bytes() + 4 * counters(); }
};
Plan make_plan(const void *dy, int32_t dtype, uint64_t rows, uint32_t out, uint64_t stride, uint32_t cols, int32_t grad_dtype)
{
    Plan p = {};
    if (dtype == DECO_F32) p.planes = grad_dtype == DECO_F32 ? 3 : 2;
    else if (!aligned_to(dy, 16) || stride % 8 || stride >= (1ull << 39)) p.planes = 1;      // (what box copies can address)
    p.pitch = (out + 7) / 8 * 8;
    p.k_blocks = static_cast<uint32_t>((rows + BK - 1) / BK);
    // Pairs of CTAs read half as much per product, and begin and end half as many tiles; small results are left to single CTAs, whose
    // tiles are a quarter.  (Single and pairs, us: 64 x 4096 x 3000, 864 tiles of one block, 17 and 20; 64 x 6000 x 6000, 2538,
    // 38 and 33; 300 x 2500 x 2500 from fp32, 460 of 15, 34 and 26.  4000 x 777 x 600 from fp32, 42 of 189, goes by pairs too and
// loses by it: 42 and 47.)
    const uint64_t area = static_cast<uint64_t>((out + TILE_M - 1) / TILE_M) * ((cols + MAX_H - 1) / MAX_H);
    p.cg = area * p.k_blocks * std::max<uint32_t>(1, p.planes) >= 4 * SMS * MIN_BLOCKS || area >= 8 * SMS ? 2 : 1;
    const uint32_t most = p.cg * MAX_H, unit = 16 * p.cg;
    p.tiles_n = (cols + most - 1) / most;
    p.h = ((cols + p.tiles_n - 1) / p.tiles_n + unit - 1) / unit * 16;
    p.tiles_m = (out + p.cg * TILE_M - 1) / (p.cg * TILE_M);
    p.tiles = static_cast<uint64_t>(p.tiles_m) * p.tiles_n;
    // How long the worker with most to do takes, in blocks: with whole tiles, with tiles in q equal parts, or with all blocks dealt
    // out evenly, wherever that cuts tiles; whoever is last adds up a tile's parts, each as long as some blocks.
    const uint64_t most_workers = SMS / p.cg, kb = p.k_blocks, units = p.tiles * kb;
    uint64_t best = (p.tiles + most_workers - 1) / most_workers * kb;
    uint32_t parts = 1;
    for (uint32_t q = 2; q <= 64 && (kb + q - 1) / q >= MIN_BLOCKS; ++q) {
        const uint64_t cost = (p.tiles * q + most_workers - 1) / most_workers * ((kb + q - 1) / q) + PART_BLOCKS * (q - 1) + CUT_BLOCKS;
        if (cost < best) {
            best = cost;
            parts = q;
        }
    }
    const uint64_t even_workers = std::min(most_workers, std::max<uint64_t>(1, units / MIN_BLOCKS));
    const uint64_t even_blocks = (units + even_workers - 1) / even_workers, even_parts = (kb + even_blocks - 1) / even_blocks + 1;
    p.cut = parts > 1;
    p.grain = static_cast<uint32_t>((kb + parts - 1) / parts);
    if (even_blocks + PART_BLOCKS * (even_parts - 1) + CUT_BLOCKS < best) {
        p.cut = true;
        p.grain = 1;
        p.workers = static_cast<uint32_t>(even_workers);
    } else {
        p.k_blocks = p.grain * parts;                            // (blocks beyond the last are zeros)
        p.workers = static_cast<uint32_t>(std::min(p.tiles * parts, most_workers));
    }
    p.plane_rows = p.k_blocks * BK;
    return p;
}

// Boxes of `box_cols` columns and BK rows; outside of the matrix zeros are read.
bool box_map(EncodeFn fn, CUtensorMap *map, CUtensorMapDataType type, const void *base, uint64_t cols, uint64_t rows,
             uint64_t row_bytes, uint32_t box_cols, CUtensorMapSwizzle swizzle)
{
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {row_bytes};
    const cuuint32_t box[2] = {box_cols, BK}, step[2] = {1, 1};
    return fn(map, type, 2, const_cast<void *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, typename G>
bool allow()
{
    return cudaFuncSetAttribute(wgrad_kernel<CG, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(SMEM)) == cudaSuccess;
}
// the kernels' shared memory, once per device
bool allow_shared_memory()
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) {
        cudaGetLastError();                                      // (pending, it would be taken for the next call's)
        return false;
    }
    if (dev < 64 && (done.load() >> dev & 1)) return true;
    if (!allow<1, float>() || !allow<1, __nv_bfloat16>() || !allow<2, float>() || !allow<2, __nv_bfloat16>()) {
        cudaGetLastError();
        return false;
    }
    if (dev < 64) done.fetch_or(1ull << dev);
    return true;
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), uint32_t cluster, dim3 grid, unsigned block, size_t smem, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
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
    const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (err != cudaSuccess) cudaGetLastError();                  // (pending, it would be taken for the next call's)
    return err;
}

template <int CG, typename G>
cudaError_t launch_all(const CUtensorMap &map, const CUtensorMap &code_map, const Args &a, const Plan &p, cudaStream_t s)
{
    return launch(wgrad_kernel<CG, G>, CG, dim3(p.workers * CG), THREADS, SMEM, s, map, code_map, a);
}

}  // namespace

extern "C" uint64_t deco_weight_grad8_workspace(const void *dy, int32_t dtype, uint64_t rows, uint32_t out,
                                                uint64_t dy_stride, uint32_t cols, int32_t grad_dtype)
{
    if (rows == 0 || rows >= MAX_ROWS || out == 0 || out > MAX_COLS || cols == 0 || cols > MAX_COLS) return 0;
    return make_plan(dy, dtype, rows, out, dy_stride, cols, grad_dtype).bytes();
}

extern "C" deco_status deco_weight_grad8(const void *dy, int32_t dtype, uint64_t rows, uint32_t out, uint64_t dy_stride,
                                         const int8_t *codes, const uint8_t *exponents, uint32_t cols, void *dw, void *db,
                                         int32_t grad_dtype, int32_t transposed, int32_t accumulate, void *workspace,
                                         uint64_t workspace_bytes, void *stream)
{
    if (!is_dtype(dtype) || !is_dtype(grad_dtype) || rows >= MAX_ROWS || out == 0 || out > MAX_COLS || cols == 0 ||
        cols > MAX_COLS)
        return DECO_ERR_INVALID_ARG;
    const uint32_t gsize = grad_dtype == DECO_F32 ? 4 : 2;
    if (!dw || !aligned_to(dw, gsize) || !aligned_to(db, gsize)) return DECO_ERR_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (rows == 0) {                                             // sums of nothing
        if (accumulate) return DECO_OK;
        if (cudaMemsetAsync(dw, 0, static_cast<uint64_t>(out) * cols * gsize, s) != cudaSuccess ||
            (db && cudaMemsetAsync(db, 0, static_cast<uint64_t>(out) * gsize, s) != cudaSuccess)) {
            cudaGetLastError();
            return DECO_ERR_CUDA;
        }
        return DECO_OK;
    }
    if (!dy || !aligned_to(dy, dtype == DECO_F32 ? 4 : 2) || dy_stride < out || dy_stride > MAX_STRIDE) return DECO_ERR_INVALID_ARG;
    if (!codes || !exponents || !aligned_to(codes, 16)) return DECO_ERR_INVALID_ARG;
    const Plan p = make_plan(dy, dtype, rows, out, dy_stride, cols, grad_dtype);
    if (p.tiles * p.cg * SUM_WARPS > 0x7FFFFFFFull || static_cast<uint64_t>(p.planes) * p.plane_rows > 0x7FFFFFFFull)
        return DECO_ERR_INVALID_ARG;
    if (!workspace || !aligned_to(workspace, 16)) return DECO_ERR_INVALID_ARG;
    if (workspace_bytes < p.bytes()) return DECO_ERR_CAPACITY;
    const EncodeFn encode = encode_function();
    if (!encode || !allow_shared_memory()) return DECO_ERR_CUDA;
    const void *operand = p.planes ? workspace : dy;
    const uint64_t pitch = (cols + BLOCK8 - 1) / BLOCK8 * static_cast<uint64_t>(BLOCK8);
    // (as a box, so it may reach into the next tile's columns)
    const uint32_t code_pitch = p.h / 16 % 2 ? p.h : p.h + 16;
    CUtensorMap map, code_map;
    if (!box_map(encode, &map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, operand, out, p.planes ? static_cast<uint64_t>(p.planes) * p.plane_rows : rows,
                 2 * (p.planes ? p.pitch : dy_stride), 64, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !box_map(encode, &code_map, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, pitch, rows, pitch, code_pitch, CU_TENSOR_MAP_SWIZZLE_NONE))
        return DECO_ERR_CUDA;
    Args a = {};
    a.out = out;
    a.cols = cols;
    a.h = p.h;
    a.code_pitch = code_pitch;
    a.tiles_n = p.tiles_n;
    a.k_blocks = p.k_blocks;
    a.planes = std::max<uint32_t>(1, p.planes);
    a.plane_rows = p.plane_rows;
    a.chunk = grad_dtype == DECO_F32 ? CHUNK : LONG_CHUNK;
    a.workers = p.workers;
    a.grain = p.grain;
    a.grains = p.tiles * (p.k_blocks / p.grain);
    a.dw = dw;
    a.db = db;
    a.transposed = transposed != 0;
    a.accumulate = accumulate != 0;
    a.wide = !transposed && aligned_to(dw, 32) && cols % (32 / gsize) == 0;
    uint8_t *room = static_cast<uint8_t *>(workspace) + p.plane_bytes();
    uint4 *steps = reinterpret_cast<uint4 *>(room);
    a.steps = steps;
    a.slots = reinterpret_cast<float *>(room + p.step_bytes());
    a.arrived = reinterpret_cast<uint32_t *>(room + p.step_bytes() + p.slot_bytes());
    PrepareArgs b = {};
    b.exps = exponents;
    b.rows = static_cast<uint32_t>(rows);
    b.blocks8 = static_cast<uint32_t>(pitch / BLOCK8);
    b.h = p.h;
    b.shares = p.tiles_n * p.cg;
    b.tokens = p.plane_rows;
    b.steps = steps;
    b.counters = a.arrived;
    b.n_counters = static_cast<uint32_t>(p.counters());
    const uint64_t records = static_cast<uint64_t>(b.shares) * p.plane_rows;
    b.step_blocks = static_cast<uint32_t>(std::min<uint64_t>(8 * SMS, (records + 255) / 256));
    if (p.planes) {
        b.dy = dy;
        b.stride = dy_stride;
        b.out = out;
        b.pitch = p.pitch;
        b.planes = p.planes;
        b.to = static_cast<__nv_bfloat16 *>(workspace);
        b.plane_blocks_x = (p.pitch + 2047) / 2048;
        b.plane_blocks_y = std::min<uint32_t>(p.plane_rows, std::max<uint32_t>(1, 16 * SMS / b.plane_blocks_x));
    }
    const unsigned blocks = b.step_blocks + b.plane_blocks_x * b.plane_blocks_y;
    if (dtype == DECO_F32) prepare_kernel<float><<<blocks, 256, 0, s>>>(b);
    else prepare_kernel<__nv_bfloat16><<<blocks, 256, 0, s>>>(b);
    if (cudaGetLastError() != cudaSuccess) return DECO_ERR_CUDA;
    const bool f32 = grad_dtype == DECO_F32;
    const cudaError_t err = p.cg == 2 ? (f32 ? launch_all<2, float>(map, code_map, a, p, s) : launch_all<2, __nv_bfloat16>(map, code_map, a, p, s))
                                      : (f32 ? launch_all<1, float>(map, code_map, a, p, s) : launch_all<1, __nv_bfloat16>(map, code_map, a, p, s));
    return err == cudaSuccess ? DECO_OK : DECO_ERR_CUDA;
}
