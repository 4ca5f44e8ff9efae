// Linear layer on 8-bit floating point operands with a scale for each block of 128 along the reduction, on the tensor cores.
//
//   y[m][k] = act( sum_b sx[b][m] * sw[b][k / wb] * ( sum_{c in block b} x[m][c] * w[k][c] ) + bias[k] ),  wb = 128 or 1
//
// The tensor core sums the 128 products of a block; the scales differ from block to block, so a block's sums have to leave the
// tensor memory and be added up in registers: acc += (sx * sw) * t, in fp32.  Slices are extents of the tensor maps: the first K
// rows and C columns of the stored weights, zeros beyond.
//
// Three forms, by the size of the call (the rule stands at the launch): pairs of blocks on tiles of 256 x 256, single blocks on tiles of
// 128 x 128, and for few rows, or few tiles and a long reduction, tiles of 128 rows of w whose reduction a cluster shares.
//
// What bounds the large form (8192^3, 579 us, 1.90 PFLOP/s at some 1.55 GHz under the power cap; 574 to 594 from call to call): the way of a
// block's sums through the warps.  The MMAs of a block take 512 clocks; with the sums left out a block takes 745 (operand copies and MMAs share the port of shared
// memory, and each accumulator passes from hand to hand), with them 1030: a wait, four loads of the tensor memory and 64 packed
// multiply-adds are a chain that two warps a scheduler do not hide.  Measured instead (same call, 598 us then): sixteen warps of 64 columns
// 602 us; tiles of 256 x 192 with twelve warps that read all their columns first 610 us; 256 x 160 with three accumulators 676 us; two teams
// of warps on alternate blocks of 256 x 128 tiles 935 us; scalar multiply-adds 595 us.
#include "sgs_tc.cuh"

#include <algorithm>

namespace sgs {
namespace {

constexpr int F8_BLOCK = 128;                       // reduction steps of a scale, of a pipeline stage and of a 128-byte swizzle row
constexpr int F8_A_BYTES = TILE_M * F8_BLOCK;
constexpr int F8_SUM_WARPS = 8, F8_THREADS = 128 + 32 * F8_SUM_WARPS;
constexpr int F8_RING = 160 * 1024;                 // operand stages
constexpr int F8_AHEAD = 4;                         // blocks whose scales travel together; two such sets are in shared memory or on their way
constexpr int F8_OUT = 2048;                        // an output box of a warp: 32 rows x 64 bytes

struct F8Params {
    CUtensorMap tmX, tmW, tmY;
    const float *sx, *sw, *bias;
    void *y;
    int *status;
    long long ldsx, ldsw, ldy;
    int M, K, C, blocks;        // blocks of the reduction
    int m_tiles, n_tiles;
    int act, y_bf16;
    int bulk_y;                 // columns of y that the copy unit may write: all where rows end on 16 bytes (it cuts boxes off there, not at the column)
    uint32_t formats;           // operand formats at their places in the instruction descriptor
    int withhold;               // test of the time-out path: a block of the reduction whose w is not copied (else -1)
    unsigned long long limit_ns;  // of a wait
};

template <int CTAS> __device__ __forceinline__ void umma_f8_if(uint32_t on, uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    if (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate), "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate), "r"(on)
            : "memory");
}
// Commit of the MMAs issued so far; of a pair's to the barrier at this place in both blocks.
template <int CTAS> __device__ __forceinline__ void commit_if(uint32_t on, uint32_t bar) {
    if (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
            "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}" ::"r"(bar), "r"(on), "h"((uint16_t)3) : "memory");
    else umma_commit_if(on, bar);
}
// Copy of a tile into this block's shared memory; `bar` may be the pair's first block's.
template <int CTAS> __device__ __forceinline__ void tma_load_2d_if(uint32_t on, uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    if (CTAS == 2)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];\n\t}"
            ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
            ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(on)
            : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ uint32_t block_addr(uint32_t saddr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
    return r;
}
// Arrival at a barrier of either block, behind tensor-memory loads alone.  (A release at cluster scope waits for all of the thread's
// memory operations: 1000 to 1700 clocks here, three times a block's MMAs.)
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory"); }
__device__ __forceinline__ void pair_sync() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }
template <int CTAS> __device__ __forceinline__ void f8_tmem_alloc(uint32_t *dst, uint32_t cols) {
    if (CTAS == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else tmem_alloc(dst, cols);
}
template <int CTAS> __device__ __forceinline__ void f8_tmem_dealloc(uint32_t addr, uint32_t cols) {
    if (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
    else tmem_dealloc(addr, cols);
}
__device__ __forceinline__ void copy_float(float *dst, const float *src, bool in) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
}
// Bounded wait of a converged warp, as mbar_wait but in few instructions and without a jump where the phase is complete: the warps that
// add up wait twice in some 300 instructions.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, volatile int *abort_flag, unsigned long long limit_ns) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    unsigned long long t0 = 0;
#pragma unroll 1
    for (uint32_t n = 1; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); n++) {
        if (n & 255) continue;
        const unsigned long long t = global_ns();
        if (!t0) t0 = t;
        if (__any_sync(0xffffffffu, *abort_flag || t - t0 > limit_ns)) { *abort_flag = 1; return false; }
    }
    return true;
}
// Waits for this warp's tensor-memory loads; the values named are the ones that they bring.
__device__ __forceinline__ void tmem_ld_wait32(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                   "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]),
                   "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 ::"memory");
}

// One output row's `n` consecutive columns o[0..] (n at most N), where the copy unit cannot write them: rows of y that do not start or, in the last columns, do not end on 16 bytes.
template <int N> __device__ __forceinline__ void store_row(const F8Params &p, long long at, const float *o, int n) {
#pragma unroll
    for (int j = 0; j < N; j++)
        if (j < n) {
            if (p.y_bf16) static_cast<__nv_bfloat16 *>(p.y)[at + j] = __float2bfloat16_rn(o[j]);
            else static_cast<float *>(p.y)[at + j] = o[j];
        }
}

// A tile is 128 rows of x a block (lanes of the tensor memory) x BN rows of w (columns); CTAS = 2: the blocks of a cluster of two share
// a tile of 256 rows, each holds its rows of x and half of the rows of w, and the first one issues the MMAs for both.
// Warp 0 loads, warp 1 issues, warp 2 brings the scales, warps 4..11 add up: a quadrant of the lanes and half of the columns each.  512 / BN accumulators: the
// tensor core sums a block into one while the warps take another, and into the next tile's while they write this one's.
template <int CTAS, int BN, bool W_ROWS>
__global__ void __launch_bounds__(F8_THREADS, 1) linear_f8_kernel(const __grid_constant__ F8Params p) {
    constexpr int B_ROWS = BN / CTAS, STAGE = F8_A_BYTES + B_ROWS * F8_BLOCK, STAGES = F8_RING / STAGE, NACC = 512 / BN, COLS = BN / 2;
    struct Shared {
        alignas(16) float row_scale[2][TILE_M][F8_AHEAD];                                   // a thread reads its row's of a set at once
        alignas(16) float col_scale[2][W_ROWS ? F8_AHEAD : 2][W_ROWS ? BN : F8_AHEAD];       // W_ROWS: [block][column], else [half of the columns][block]
        alignas(16) float bias[BN];
        alignas(8) uint64_t full[STAGES], empty[STAGES], acc_full[NACC], acc_empty[NACC], sc_full[2], sc_empty[2];
        uint32_t tmem_base;
        int abort;
    };
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem + F8_RING + F8_SUM_WARPS * 2 * F8_OUT);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = CTAS == 2 ? (int)(blockIdx.x & 1) : 0, group = (int)blockIdx.x / CTAS, groups = (int)gridDim.x / CTAS;
    volatile int *abort_flag = &sh.abort;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; s++) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int i = 0; i < NACC; i++) { mbar_init(&sh.acc_full[i], 1); mbar_init(&sh.acc_empty[i], F8_SUM_WARPS * CTAS); }
        for (int i = 0; i < 2; i++) { mbar_init(&sh.sc_full[i], 32); mbar_init(&sh.sc_empty[i], F8_SUM_WARPS); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) f8_tmem_alloc<CTAS>(&sh.tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    if (CTAS == 2) pair_sync();
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t ring = smem_u32(smem);
    const int blocks = p.blocks, tiles = p.m_tiles * p.n_tiles;
    // Tiles go by strips of 8 along the rows: the tiles at work at a time share what they read of both operands.
    auto place = [&](int tile, int *m0, int *f0) {
        const int strip = 8 * p.n_tiles, g = tile / strip, rest = tile - g * strip, wide = min(8, p.m_tiles - 8 * g);
        *m0 = ((8 * g + rest % wide) * CTAS + rank) * TILE_M;
        *f0 = rest / wide * BN;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0) {
            const uint32_t on = elect_one(), full0 = CTAS == 2 ? block_addr(smem_u32(sh.full), 0) : smem_u32(sh.full), first = rank == 0 ? on : 0;
            int s = 0;
            uint32_t phase = 1;  // (the first pass over the ring finds it empty)
            bool ok = true;
            for (int tile = group; ok && tile < tiles; tile += groups) {
                int m0, f0;
                place(tile, &m0, &f0);
                for (int b = 0; b < blocks; b++) {
                    if (!warp_wait(&sh.empty[s], phase, abort_flag, p.limit_ns)) { ok = false; break; }
                    const uint32_t sa = ring + (uint32_t)(s * STAGE), fb = full0 + (uint32_t)(s * 8);
                    if (rank == 0) mbar_expect_tx_if(first, smem_u32(&sh.full[s]), STAGE * CTAS);
                    tma_load_2d_if<CTAS>(on, sa, &p.tmX, fb, b * F8_BLOCK, m0);
                    if (b != p.withhold) tma_load_2d_if<CTAS>(on, sa + F8_A_BYTES, &p.tmW, fb, b * F8_BLOCK, f0 + rank * B_ROWS);
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                }
            }
        } else if (warp == 1 && rank == 0) {
            const uint32_t on = elect_one(), d_tmem = uniform(tmem_base), empty0 = smem_u32(sh.empty), acc0 = smem_u32(sh.acc_full);
            // instruction descriptor: fp32 accumulator at bit 4, operand formats at bits 7 / 10, N >> 3 at bit 17, M >> 4 at bit 24
            const uint32_t idesc = (1u << 4) | p.formats | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(TILE_M * CTAS >> 4) << 24);
            int s = 0, a = 0;
            uint32_t phase = 0, acc_phase = 1;
            bool ok = true;
            for (int tile = group; ok && tile < tiles; tile += groups)
                for (int b = 0; b < blocks; b++) {
                    if (!warp_wait(&sh.acc_empty[a], acc_phase, abort_flag, p.limit_ns) ||
                        !warp_wait(&sh.full[s], phase, abort_flag, p.limit_ns)) { ok = false; break; }
                    tc_fence_after();
                    const int steps = min(4, (p.C - b * F8_BLOCK + 31) / 32);
                    const uint32_t sa = ring + (uint32_t)(s * STAGE);
                    const uint64_t da = smem_desc_sw128(sa), db = smem_desc_sw128(sa + F8_A_BYTES);
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        if (q < steps) umma_f8_if<CTAS>(on, d_tmem + (uint32_t)(a * BN), da + (uint64_t)(2 * q), db + (uint64_t)(2 * q), idesc, q > 0 ? 1u : 0u);
                    commit_if<CTAS>(on, empty0 + (uint32_t)(s * 8));
                    commit_if<CTAS>(on, acc0 + (uint32_t)(a * 8));
                    if (++s == STAGES) { s = 0; phase ^= 1; }
                    if (++a == NACC) { a = 0; acc_phase ^= 1; }
                }
        } else if (warp == 2) {
            // scales: two sets of four blocks ahead of their use, without a register (a load just before the block that needs it took as
            // long as two blocks' MMAs); zeros beyond the operands
            int i = 0;
            uint32_t phase = 1;
            bool ok = true;
            for (int tile = group; ok && tile < tiles; tile += groups) {
                int m0, f0;
                place(tile, &m0, &f0);
                for (int b0 = 0; b0 < blocks; b0 += F8_AHEAD) {
                    if (!warp_wait(&sh.sc_empty[i], phase, abort_flag, p.limit_ns)) { ok = false; break; }
#pragma unroll
                    for (int k = 0; k < F8_AHEAD; k++) {
                        if (b0 + k >= blocks) break;
                        const float *sx = p.sx + (long long)(b0 + k) * p.ldsx, *sw = p.sw + (long long)(b0 + k) * p.ldsw;
#pragma unroll
                        for (int j = 0; j < TILE_M; j += 32) copy_float(&sh.row_scale[i][j + lane][k], sx + min(m0 + j + lane, p.M - 1), m0 + j + lane < p.M);
                        if (W_ROWS) {
#pragma unroll
                            for (int j = 0; j < BN; j += 32) copy_float(&sh.col_scale[i][W_ROWS ? k : 0][j + lane], sw + min(f0 + j + lane, p.K - 1), f0 + j + lane < p.K);
                        } else if (lane < 2) copy_float(&sh.col_scale[i][lane][W_ROWS ? 0 : k], sw + min(f0 + lane * COLS, p.K - 1) / 128, true);
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sh.sc_full[i])) : "memory");
                    if ((i ^= 1) == 0) phase ^= 1;
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int quad = warp & 3, half = warp >> 3;  // (a warp reads the 32 lanes of its number modulo 4)
        const int c0 = half * COLS, ht = (warp & 3) * 32 + lane;  // first column of the half, thread of it
        const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)c0;
        const uint32_t out0 = ring + F8_RING + (uint32_t)((warp - 4) * 2 * F8_OUT);
        const uint32_t drained0 = CTAS == 2 ? block_addr(smem_u32(sh.acc_empty), 0) : smem_u32(sh.acc_empty);
        auto half_sync = [&] {
            if (half) asm volatile("bar.sync 2, 128;" ::: "memory");
            else asm volatile("bar.sync 1, 128;" ::: "memory");
        };
        int a = 0, parts = 0, i = 0;  // accumulator, output boxes written, scales
        uint32_t acc_phase = 0, sc_phase = 0;
        for (int tile = group; tile < tiles; tile += groups) {
            int m0, f0;
            place(tile, &m0, &f0);
            const int m = m0 + quad * 32 + lane, fc = f0 + c0;
            const float my_bias = p.bias && ht < COLS ? ld_act(p.bias + min(fc + ht, p.K - 1)) : 0.f;
            float2 acc[COLS / 2];
#pragma unroll
            for (int j = 0; j < COLS / 2; j++) acc[j] = make_float2(0.f, 0.f);
            // The tensor memory is read a chunk of 32 columns ahead, over the end of a block too: while the last chunk is added up, the
            // next block's first one is on its way.  (After a wait that ran out the warps leave the loop and meet the others at the
            // barriers below.)
            uint32_t v[2][32];
            float rs[F8_AHEAD];
            bool ok = warp_wait(&sh.acc_full[a], acc_phase, abort_flag, p.limit_ns);
            tc_fence_after();
            if (ok) tmem_ld32(taddr + (uint32_t)(a * BN), v[0]);
            // (four blocks written out where registers allow: 1024x4096x4096, 29.9 us and 24.8; the pairs' kernel spills, 607 us at 8192^3)
#pragma unroll(CTAS == 1 ? F8_AHEAD : 1)
            for (int b = 0; ok && b < blocks; b++) {
                const int k = b % F8_AHEAD;
                if (k == 0) {
                    if (!(ok = warp_wait(&sh.sc_full[i], sc_phase, abort_flag, p.limit_ns))) break;
                    const float4 x4 = *reinterpret_cast<const float4 *>(sh.row_scale[i][quad * 32 + lane]);
                    rs[0] = x4.x; rs[1] = x4.y; rs[2] = x4.z; rs[3] = x4.w;
                    if (!W_ROWS) {
                        const float4 w4 = *reinterpret_cast<const float4 *>(sh.col_scale[i][half]);
                        rs[0] *= w4.x; rs[1] *= w4.y; rs[2] *= w4.z; rs[3] *= w4.w;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.sc_empty[i]);
                    }
                }
                const float *cs = sh.col_scale[i][W_ROWS ? k : 0] + c0;
                const float f = rs[0];
                rs[0] = rs[1]; rs[1] = rs[2]; rs[2] = rs[3];
                const float2 s2 = make_float2(f, f);
                // the columns' scales, four loads of shared memory ahead in the pairs' kernel (4096 x 2048 over 8197, us: 109.5, one by one
                // 114.3, eight ahead spill, 130; single blocks, 512 x 4096 x 4096: 20.1 ahead, 19.6 one by one)
                constexpr bool EARLY = W_ROWS && CTAS == 2;
                float4 c[4];
                if (EARLY) {
#pragma unroll
                    for (int t = 0; t < 4; t++) c[t] = *reinterpret_cast<const float4 *>(cs + 4 * t);
                }
#pragma unroll
                for (int j0 = 0; j0 < COLS; j0 += 32) {
                    uint32_t (&w)[32] = v[(j0 / 32) & 1], (&next)[32] = v[(j0 / 32 + 1) & 1];
                    tmem_ld_wait32(w);
                    if (j0 + 32 < COLS) tmem_ld32(taddr + (uint32_t)(a * BN + j0 + 32), next);
                    else {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if (CTAS == 1) mbar_arrive(&sh.acc_empty[a]);
                            else arrive_at(drained0 + (uint32_t)(a * 8));
                        }
                        if (++a == NACC) { a = 0; acc_phase ^= 1; }
                        if (b + 1 < blocks) {
                            ok = warp_wait(&sh.acc_full[a], acc_phase, abort_flag, p.limit_ns);
                            tc_fence_after();
                            tmem_ld32(taddr + (uint32_t)(a * BN), next);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        float2 g0 = s2, g1 = s2;
                        if (W_ROWS) {
                            const float4 e = EARLY ? c[j / 2 % 4] : *reinterpret_cast<const float4 *>(cs + j0 + 2 * j);
                            if (EARLY && j0 + 2 * j + 16 < COLS) c[j / 2 % 4] = *reinterpret_cast<const float4 *>(cs + j0 + 2 * j + 16);
                            g0 = __fmul2_rn(s2, make_float2(e.x, e.y));
                            g1 = __fmul2_rn(s2, make_float2(e.z, e.w));
                        }
                        acc[j0 / 2 + j] = __ffma2_rn(make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1])), g0, acc[j0 / 2 + j]);
                        acc[j0 / 2 + j + 1] = __ffma2_rn(make_float2(__uint_as_float(w[2 * j + 2]), __uint_as_float(w[2 * j + 3])), g1, acc[j0 / 2 + j + 1]);
                    }
                }
                if (k == F8_AHEAD - 1 || b == blocks - 1) {
                    if (W_ROWS) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.sc_empty[i]);
                    }
                    if ((i ^= 1) == 0) sc_phase ^= 1;
                }
            }
            if (!ok) {  // a wait ran out: no load of the tensor memory may be under way into registers that are used for something else now
                tmem_ld_wait32(v[0]);
                tmem_ld_wait32(v[1]);
            }
            // ---- bias, activation, one rounding, output
            half_sync();  // (all have read the last tile's)
            if (ht < COLS) sh.bias[c0 + ht] = my_bias;
            half_sync();
#pragma unroll
            for (int j = 0; j < COLS / 2; j++) acc[j] = __fadd2_rn(acc[j], *reinterpret_cast<const float2 *>(&sh.bias[c0 + 2 * j]));
            if (p.act == ACT_RELU) {
#pragma unroll
                for (int j = 0; j < COLS / 2; j++) { acc[j].x = acc[j].x < 0.f ? 0.f : acc[j].x; acc[j].y = acc[j].y < 0.f ? 0.f : acc[j].y; }
            } else if (p.act == ACT_HSWISH) {
#pragma unroll
                for (int j = 0; j < COLS / 2; j++) { acc[j].x = act_fn(acc[j].x, ACT_HSWISH); acc[j].y = act_fn(acc[j].y, ACT_HSWISH); }
            }
            if (*abort_flag) continue;
            if (p.bulk_y >= min(fc + COLS, p.K)) {
                // through shared memory in boxes of 32 rows x 64 bytes (64-byte swizzle) and out by the copy unit, which leaves out what lies
                // beyond the output; two boxes a warp, one being filled while the other is read
                const bool rows_in = m0 + quad * 32 < p.M;
                const uint32_t line = (uint32_t)lane * 64, swz = ((uint32_t)lane >> 1) & 3;
                auto box = [&](const uint4 (&q)[4], int col) {
                    if (fc + col >= p.K || !rows_in) return;
                    const uint32_t buf = out0 + (uint32_t)(parts & 1) * F8_OUT;
                    if (lane == 0 && parts >= 2) bulk_wait_read<1>();
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 4; j++) sts128(buf + line + (((uint32_t)j ^ swz) << 4), q[j]);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_2d(&p.tmY, buf, fc + col, m0 + quad * 32);
                        bulk_commit();
                    }
                    parts++;
                };
                if (p.y_bf16) {
#pragma unroll
                    for (int col = 0; col < COLS; col += 32) {
                        uint4 q[4];
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&q[j]);
#pragma unroll
                            for (int i = 0; i < 4; i++) h[i] = __float22bfloat162_rn(acc[col / 2 + 4 * j + i]);
                        }
                        box(q, col);
                    }
                } else {
#pragma unroll
                    for (int col = 0; col < COLS; col += 16) {
                        uint4 q[4];
#pragma unroll
                        for (int j = 0; j < 4; j++)
                            q[j] = make_uint4(__float_as_uint(acc[col / 2 + 2 * j].x), __float_as_uint(acc[col / 2 + 2 * j].y), __float_as_uint(acc[col / 2 + 2 * j + 1].x),
                                              __float_as_uint(acc[col / 2 + 2 * j + 1].y));
                        box(q, col);
                    }
                }
            } else if (m < p.M) store_row<COLS>(p, (long long)m * p.ldy + fc, reinterpret_cast<const float *>(acc), min(COLS, p.K - fc));
        }
        if (lane == 0) bulk_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (sh.abort) {  // a wait ran out: report, let copies in flight land, then release the tensor memory
        if (threadIdx.x == 0) atomicExch(p.status, 1);
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (CTAS == 2) pair_sync();  // (the other block's MMAs read this one's shared memory, its warps signal this one's barriers)
    if (warp == 1) { tc_fence_after(); f8_tmem_dealloc<CTAS>(tmem_base, 512); }
}

// Few rows of x: the rows of w take the lanes (128 a block), up to N rows of x the columns, and the blocks of a cluster share the
// reduction, whose parts meet in distributed shared memory, in the order of c.  What bounds such a call is w's bytes: 16 KB of them a
// stage, two thread blocks an SM (one row, 8192 filters, 4096 channels: 9.3 us, 3.6 TB/s; 16384 x 8192: 25.7 us, 5.2 TB/s; the weights of
// several calls in turn, 268 MB in all; the rest is the way in and out: launch, first copies, the cluster's two meetings).  Blocks that share an SM hold 256 columns of tensor memory at most
// each, and kernels that fit beside them the rest: no allocation waits for another block's, which a cluster whose blocks wait for each
// other could not afford.  Warp 0 loads, 1 issues, 2 brings the scales, warps 4..7 add up, a quadrant of the lanes each.
constexpr int F8_SPLIT_THREADS = 256, F8_SPLIT_RING = 96 * 1024;
struct F8Split {
    int parts, part_blocks;  // blocks of a cluster; blocks of the reduction that each of them takes (the last may have fewer)
};
template <int N, bool W_ROWS>
__global__ void __launch_bounds__(F8_SPLIT_THREADS, 2) linear_f8_split_kernel(const __grid_constant__ F8Params p, const F8Split q) {
    static_assert(N <= 64, "two blocks an SM: registers, shared memory and 256 columns of tensor memory each");
    constexpr int STAGE = F8_A_BYTES + N * F8_BLOCK, STAGES = F8_SPLIT_RING / STAGE, NACC = N <= 32 ? 8 : 256 / N;
    struct Shared {
        alignas(16) float w_scale[2][W_ROWS ? TILE_M : 1][F8_AHEAD];
        alignas(16) float x_scale[2][F8_AHEAD][N];
        alignas(8) uint64_t full[STAGES], empty[STAGES], acc_full[NACC], acc_empty[NACC], sc_full[2], sc_empty[2];
        uint32_t tmem_base;
        int abort;
    };
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared &sh = *reinterpret_cast<Shared *>(smem + F8_SPLIT_RING);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile int *abort_flag = &sh.abort;
    const int f0 = (int)blockIdx.x * TILE_M, n0 = (int)blockIdx.y * N, part = (int)blockIdx.z;
    const int b_first = part * q.part_blocks, blocks = min(q.part_blocks, p.blocks - b_first);  // (1 at least)
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; s++) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], 1); }
        for (int i = 0; i < NACC; i++) { mbar_init(&sh.acc_full[i], 1); mbar_init(&sh.acc_empty[i], 4); }
        for (int i = 0; i < 2; i++) { mbar_init(&sh.sc_full[i], 32); mbar_init(&sh.sc_empty[i], 4); }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&sh.tmem_base, NACC * N);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t ring = smem_u32(smem);
    float2 acc[N / 2];
    if (warp == 0) {
        const uint32_t on = elect_one(), full0 = smem_u32(sh.full);
        int s = 0;
        uint32_t phase = 1;
        for (int b = 0; b < blocks; b++) {
            if (!warp_wait(&sh.empty[s], phase, abort_flag, p.limit_ns)) break;
            const uint32_t sa = ring + (uint32_t)(s * STAGE), fb = full0 + (uint32_t)(s * 8);
            mbar_expect_tx_if(on, fb, STAGE);
            if (b_first + b != p.withhold) tma_load_2d_if<1>(on, sa, &p.tmW, fb, (b_first + b) * F8_BLOCK, f0);
            tma_load_2d_if<1>(on, sa + F8_A_BYTES, &p.tmX, fb, (b_first + b) * F8_BLOCK, n0);
            if (++s == STAGES) { s = 0; phase ^= 1; }
        }
    } else if (warp == 1) {
        const uint32_t on = elect_one(), d_tmem = uniform(tmem_base), empty0 = smem_u32(sh.empty), acc0 = smem_u32(sh.acc_full);
        const int n_mma = min(N, (p.M - n0 + 15) & ~15);
        const uint32_t idesc = (1u << 4) | p.formats | ((uint32_t)(n_mma >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
        int s = 0, a = 0;
        uint32_t phase = 0, acc_phase = 1;
        for (int b = 0; b < blocks; b++) {
            if (!warp_wait(&sh.acc_empty[a], acc_phase, abort_flag, p.limit_ns) || !warp_wait(&sh.full[s], phase, abort_flag, p.limit_ns)) break;
            tc_fence_after();
            const int steps = min(4, (p.C - (b_first + b) * F8_BLOCK + 31) / 32);
            const uint32_t sa = ring + (uint32_t)(s * STAGE);
            const uint64_t da = smem_desc_sw128(sa), db = smem_desc_sw128(sa + F8_A_BYTES);
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (k < steps) umma_f8_if<1>(on, d_tmem + (uint32_t)(a * N), da + (uint64_t)(2 * k), db + (uint64_t)(2 * k), idesc, k > 0 ? 1u : 0u);
            umma_commit_if(on, empty0 + (uint32_t)(s * 8));
            umma_commit_if(on, acc0 + (uint32_t)(a * 8));
            if (++s == STAGES) { s = 0; phase ^= 1; }
            if (++a == NACC) { a = 0; acc_phase ^= 1; }
        }
    } else if (warp == 2) {
        int i = 0;
        uint32_t phase = 1;
        for (int b0 = 0; b0 < blocks; b0 += F8_AHEAD) {
            if (!warp_wait(&sh.sc_empty[i], phase, abort_flag, p.limit_ns)) break;
#pragma unroll
            for (int k = 0; k < F8_AHEAD; k++) {
                if (b0 + k >= blocks) break;
                const float *sx = p.sx + (long long)(b_first + b0 + k) * p.ldsx, *sw = p.sw + (long long)(b_first + b0 + k) * p.ldsw;
#pragma unroll
                for (int j = 0; j < N; j += 32)
                    if (N >= 32 || lane < N) copy_float(&sh.x_scale[i][k][j + lane], sx + min(n0 + j + lane, p.M - 1), n0 + j + lane < p.M);
                if (W_ROWS) {
#pragma unroll
                    for (int j = 0; j < TILE_M; j += 32) copy_float(&sh.w_scale[i][W_ROWS ? j + lane : 0][k], sw + min(f0 + j + lane, p.K - 1), f0 + j + lane < p.K);
                } else if (lane == 0) copy_float(&sh.w_scale[i][0][k], sw + blockIdx.x, true);
            }
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sh.sc_full[i])) : "memory");
            if ((i ^= 1) == 0) phase ^= 1;
        }
    } else if (warp >= 4) {
        const int quad = warp & 3, l = quad * 32 + lane;
        const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16);
#pragma unroll
        for (int j = 0; j < N / 2; j++) acc[j] = make_float2(0.f, 0.f);
        int a = 0, i = 0;
        uint32_t acc_phase = 0, sc_phase = 0;
        bool ok = true;
        float4 w4;
        for (int b = 0; b < blocks; b++) {
            const int k = b % F8_AHEAD;
            if (k == 0) {
                ok = ok && warp_wait(&sh.sc_full[i], sc_phase, abort_flag, p.limit_ns);
                w4 = *reinterpret_cast<const float4 *>(sh.w_scale[i][W_ROWS ? l : 0]);
            }
            if (ok && (ok = warp_wait(&sh.acc_full[a], acc_phase, abort_flag, p.limit_ns))) {
                const float f = k & 2 ? (k & 1 ? w4.w : w4.z) : (k & 1 ? w4.y : w4.x);
                const float2 f2 = make_float2(f, f);
                tc_fence_after();
#pragma unroll
                for (int j0 = 0; j0 < N; j0 += 32) {
                    uint32_t v[32];
                    if (N >= 32) tmem_ld32(taddr + (uint32_t)(a * N + j0), v);
                    else {
                        tmem_ld16(taddr + (uint32_t)(a * N), v);
#pragma unroll
                        for (int j = 16; j < 32; j++) v[j] = 0;
                    }
                    tmem_ld_wait32(v);
                    if (j0 + 32 >= N) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.acc_empty[a]);
                    }
#pragma unroll
                    for (int j = 0; j < (N < 32 ? N : 32); j += 4) {
                        const float4 c = *reinterpret_cast<const float4 *>(&sh.x_scale[i][k][j0 + j]);
                        float2 &a0 = acc[(j0 + j) / 2], &a1 = acc[(j0 + j) / 2 + 1];
                        a0 = __ffma2_rn(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), __fmul2_rn(f2, make_float2(c.x, c.y)), a0);
                        a1 = __ffma2_rn(make_float2(__uint_as_float(v[j + 2]), __uint_as_float(v[j + 3])), __fmul2_rn(f2, make_float2(c.z, c.w)), a1);
                    }
                }
            }
            if (++a == NACC) { a = 0; acc_phase ^= 1; }
            if (k == F8_AHEAD - 1) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.sc_empty[i]);
                if ((i ^= 1) == 0) sc_phase ^= 1;
            }
        }
        // the sums: [row of x][lane], in the operand stages (all of this block's MMAs have read theirs)
        if (ok) {
            float *sums = reinterpret_cast<float *>(smem) + l;
#pragma unroll
            for (int j = 0; j < N; j++) sums[j * TILE_M] = j & 1 ? acc[j / 2].y : acc[j / 2].x;
        }
        if (q.parts == 1) asm volatile("bar.sync 1, 128;" ::: "memory");
    }
    if (q.parts > 1) pair_sync();  // (every thread of every block of the cluster)
    // A warp takes a row, a lane four features.  (One feature a lane and its columns written out, 64 stores behind their branches were read
    // once each from a cold instruction cache: 64 x 320 x 360 took 9.1 us, 5.5 so.)
    if (warp >= 4 && !*abort_flag) {
        const int f = f0 + lane * 4, rows = min(N, p.M - n0), size = p.y_bf16 ? 2 : 4;
        const bool whole = f + 4 <= p.K && ((reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)(p.ldy * size)) & (uintptr_t)(4 * size - 1)) == 0;
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; i++) bias[i] = p.bias && f + i < p.K ? ld_act(p.bias + f + i) : 0.f;
        auto put = [&](int n, const float (&sum)[4]) {
            float o[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                o[i] = sum[i] + bias[i];
                if (p.act == ACT_RELU) o[i] = o[i] < 0.f ? 0.f : o[i];
                else if (p.act == ACT_HSWISH) o[i] = act_fn(o[i], ACT_HSWISH);
            }
            const long long at = (long long)(n0 + n) * p.ldy + f;
            if (p.y_bf16) {
                __nv_bfloat16 *y = static_cast<__nv_bfloat16 *>(p.y) + at;
                __nv_bfloat162 h[2] = {__floats2bfloat162_rn(o[0], o[1]), __floats2bfloat162_rn(o[2], o[3])};
                if (whole) *reinterpret_cast<uint2 *>(y) = *reinterpret_cast<uint2 *>(h);
                else
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (f + i < p.K) y[i] = __float2bfloat16_rn(o[i]);
            } else {
                float *y = static_cast<float *>(p.y) + at;
                if (whole) *reinterpret_cast<float4 *>(y) = make_float4(o[0], o[1], o[2], o[3]);
                else
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (f + i < p.K) y[i] = o[i];
            }
        };
        if (q.parts == 1) {
            const float4 *sums = reinterpret_cast<const float4 *>(smem) + lane;
#pragma unroll 4
            for (int n = warp - 4; n < rows; n += 4) {
                const float4 v = sums[n * (TILE_M / 4)];
                put(n, {v.x, v.y, v.z, v.w});
            }
        } else {
#pragma unroll 1
            for (int n = part + (warp - 4) * q.parts; n < rows; n += 4 * q.parts) {
                float v[8][4], sum[4] = {0.f, 0.f, 0.f, 0.f};  // all parts are asked for before the first is used
#pragma unroll
                for (int s = 0; s < 8; s++)
                    if (s < q.parts)
                        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                     : "=f"(v[s][0]), "=f"(v[s][1]), "=f"(v[s][2]), "=f"(v[s][3])
                                     : "r"(block_addr(ring + (uint32_t)(n * TILE_M + lane * 4) * 4, (uint32_t)s)) : "memory");
                    else v[s][0] = v[s][1] = v[s][2] = v[s][3] = 0.f;
#pragma unroll
                for (int s = 0; s < 8; s++)
#pragma unroll
                    for (int i = 0; i < 4; i++) sum[i] += v[s][i];
                put(n, sum);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (sh.abort) {  // as above
        if (threadIdx.x == 0) atomicExch(p.status, 1);
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (q.parts > 1) pair_sync();  // (nobody leaves while another block may still read its sums)
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, NACC * N); }
}

template <int N, bool W_ROWS> cudaError_t launch_split(F8Params &p, const LinearF8Args &a, DeviceBits &done, cudaStream_t st) {
    constexpr int SMEM = F8_SPLIT_RING + 2 * F8_AHEAD * ((W_ROWS ? TILE_M : 1) + N) * 4 + 512;
    if (!tc_encode_bytes(&p.tmX, a.x, (uint64_t)a.C, (uint64_t)a.M, (uint64_t)a.ldx, N) || !tc_encode_bytes(&p.tmW, a.w, (uint64_t)a.C, (uint64_t)a.K, (uint64_t)a.ldw, TILE_M))
        return cudaErrorInvalidValue;
    p.formats = ((uint32_t)(a.w_e5m2 ? 1 : 0) << 7) | ((uint32_t)(a.x_e5m2 ? 1 : 0) << 10);
    cudaError_t e = smem_limit_once(linear_f8_split_kernel<N, W_ROWS>, SMEM, done);
    if (e != cudaSuccess) return e;
    const unsigned filters = (unsigned)((a.K + TILE_M - 1) / TILE_M), rows = (unsigned)((a.M + N - 1) / N);
    F8Split q;
    q.parts = 1;
    // (one row, 8192 x 4096: 9.2 us with 4 parts, 10.0 with 2, 12.8 with 8)
    while (q.parts < 8 && (long long)filters * rows * q.parts < sm_count() && p.blocks >= 4 * q.parts) q.parts *= 2;
    q.part_blocks = (p.blocks + q.parts - 1) / q.parts;
    while ((q.parts - 1) * q.part_blocks >= p.blocks) q.parts--;  // (no block without a share; any number makes a cluster)
    return launch_pdl(linear_f8_split_kernel<N, W_ROWS>, dim3(filters, rows, (unsigned)q.parts), dim3(F8_SPLIT_THREADS), SMEM, st, (unsigned)q.parts, p, q);
}

DeviceBits g_set[10];

template <int CTAS, int BN, bool W_ROWS> cudaError_t launch_tiles(F8Params &p, const LinearF8Args &a, DeviceBits &done, cudaStream_t st) {
    constexpr int SMEM = F8_RING + F8_SUM_WARPS * 2 * F8_OUT + 2 * F8_AHEAD * (TILE_M + (W_ROWS ? BN : 2)) * 4 + BN * 4 + 512;
    static_assert(SMEM <= 227 * 1024, "shared memory");
    if (!tc_encode_bytes(&p.tmX, a.x, (uint64_t)a.C, (uint64_t)a.M, (uint64_t)a.ldx, TILE_M) ||
        !tc_encode_bytes(&p.tmW, a.w, (uint64_t)a.C, (uint64_t)a.K, (uint64_t)a.ldw, BN / CTAS))
        return cudaErrorInvalidValue;
    p.m_tiles = (a.M + TILE_M * CTAS - 1) / (TILE_M * CTAS);
    p.n_tiles = (a.K + BN - 1) / BN;
    cudaError_t e = smem_limit_once(linear_f8_kernel<CTAS, BN, W_ROWS>, SMEM, done);
    if (e != cudaSuccess) return e;
    const long long groups = std::min<long long>((long long)p.m_tiles * p.n_tiles, sm_count() / CTAS);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * CTAS));
    cfg.blockDim = dim3(F8_THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, linear_f8_kernel<CTAS, BN, W_ROWS>, p);
}

}  // namespace

cudaError_t launch_linear_f8(const LinearF8Args &a, int device, cudaStream_t st) {
    F8Params p = {};
    p.sx = a.sx; p.sw = a.sw; p.bias = a.bias; p.y = a.y; p.status = tc_status_word(device);
    p.ldsx = a.ldsx; p.ldsw = a.ldsw; p.ldy = a.ldy;
    p.M = a.M; p.K = a.K; p.C = a.C; p.blocks = (a.C + F8_BLOCK - 1) / F8_BLOCK;
    p.act = a.act; p.y_bf16 = a.y_bf16; p.withhold = a.withhold; p.limit_ns = a.limit_ns ? a.limit_ns : WAIT_LIMIT_NS;
    const size_t pitch = (size_t)a.ldy * (a.y_bf16 ? 2 : 4);
    const int unit = a.y_bf16 ? 8 : 4;  // elements of 16 bytes
    if (((reinterpret_cast<uintptr_t>(a.y) | pitch) & 15) == 0 && tc_encode_output(&p.tmY, a.y, (uint64_t)a.K, (uint64_t)a.M, pitch, a.y_bf16, 4 * unit, 32))
        p.bulk_y = a.K / unit * unit;
    p.formats = ((uint32_t)(a.x_e5m2 ? 1 : 0) << 7) | ((uint32_t)(a.w_e5m2 ? 1 : 0) << 10);
    const long long tiles = (long long)((a.M + 127) / 128) * ((a.K + 127) / 128);
    // Few rows split the reduction over clusters.  So do more than 32 where the tiles of 128 x 128 would leave three SMs in four idle and the
    // reduction is long enough to pay for the meeting (split and in tiles, us: 128 x 4096 x 4096 10.8 and 13.4, 300 x 1000 x 8192 14.0 and
    // 22.0; with 64 tiles 256 x 4096 x 4096, which the split form reads w four times for, 15.2 and 13.4, and 64 x 8192 x 4096, which it would
    // read once, 12.2 and 13.6; 128 x 4096 x 1024 6.9 and 6.0, 64 x 320 x 640 6.6 and 4.9).
    if (a.M <= 16) return a.w_rows ? launch_split<16, true>(p, a, g_set[4], st) : launch_split<16, false>(p, a, g_set[5], st);
    if (a.M <= 32) return a.w_rows ? launch_split<32, true>(p, a, g_set[6], st) : launch_split<32, false>(p, a, g_set[7], st);
    if (tiles * 4 <= sm_count() && p.blocks > 8) return a.w_rows ? launch_split<64, true>(p, a, g_set[8], st) : launch_split<64, false>(p, a, g_set[9], st);
    // Pairs of SMs take a tile of 256 x 256 in 1.6 times the time that one takes for 128 x 128 (4096 long: 16.5 us more for each wave, and
    // 10.2): they win where they need that many fewer waves.  1024 x 4096, one wave and two, 22.1 and 23.9 us; 1280 x 4096, two and three,
    // 39.0 and 33.4; 512 x 4096, one and one, 21.4 and 13.9; 50176 x 64, 256 long, three and three, 11.7 and 9.1; 12544 x 408, 512 long, two
    // and three, 12.6 and 10.6.  (Both count whole tiles: of 408 filters' fourth one 24 are in use.)
    const long long sms = sm_count(), pair_tiles = (long long)((a.M + 255) / 256) * ((a.K + 255) / 256);
    const long long waves = (tiles + sms - 1) / sms, pair_waves = (pair_tiles + sms / 2 - 1) / (sms / 2);
    const bool pairs = 8 * pair_waves <= 5 * waves;
    if (a.w_rows) return pairs ? launch_tiles<2, 256, true>(p, a, g_set[0], st) : launch_tiles<1, 128, true>(p, a, g_set[1], st);
    return pairs ? launch_tiles<2, 256, false>(p, a, g_set[2], st) : launch_tiles<1, 128, false>(p, a, g_set[3], st);
}

}  // namespace sgs
