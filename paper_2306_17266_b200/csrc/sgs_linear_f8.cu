// Linear layer on 8-bit floating point operands with a scale for each block of 128 along the reduction, on the tensor cores.
//
//   y[m][k] = act( sum_b sx[b][m] * sw[b][k / wb] * ( sum_{c in block b} x[m][c] * w[k][c] ) + bias[k] ),  wb = 128 or 1
//
// The tensor core sums the 128 products of a block; the scales differ from block to block, so a block's sums have to leave the
// tensor memory and be added up in registers: acc += (sx * sw) * t, in fp32.  Slices are extents of the tensor maps: the first K
// rows and C columns of the stored weights, zeros beyond.
#include "sgs_tc.cuh"

#include <algorithm>

namespace sgs {
namespace {

constexpr int F8_BLOCK = 128;                       // reduction steps of a scale, of a pipeline stage and of a 128-byte swizzle row
constexpr int F8_A_BYTES = TILE_M * F8_BLOCK;
constexpr int F8_SUM_WARPS = 8, F8_THREADS = 64 + 32 * F8_SUM_WARPS;

struct F8Params {
    CUtensorMap tmX, tmW;
    const float *sx, *sw, *bias;
    void *y;
    int *status;
    long long ldsx, ldsw, ldy;
    int M, K, C, blocks;        // blocks of the reduction
    int m_tiles, n_tiles;
    int act, y_bf16, vec_y;     // vec_y: 16-byte stores allowed
    uint32_t formats;           // operand formats at their places in the instruction descriptor
};

__device__ __forceinline__ void umma_f8_if(uint32_t on, uint32_t tmem_d, uint64_t desc_a, uint64_t desc_b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d), "l"(desc_a), "l"(desc_b), "r"(idesc), "r"(accumulate), "r"(on)
        : "memory");
}
__device__ __forceinline__ void tma_load_2d_if(uint32_t on, uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n\t}"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(on)
        : "memory");
}

// One output row's `n` consecutive columns o[0..] (n at most N).
template <int N> __device__ __forceinline__ void store_row(const F8Params &p, long long at, const float *o, int n) {
    if (p.y_bf16) {
        __nv_bfloat16 *y = static_cast<__nv_bfloat16 *>(p.y) + at;
#pragma unroll
        for (int j = 0; j < N; j += 8) {
            if (p.vec_y && j + 8 <= n) {
                uint4 v;
                __nv_bfloat162 *b = reinterpret_cast<__nv_bfloat162 *>(&v);
#pragma unroll
                for (int i = 0; i < 4; i++) b[i] = __floats2bfloat162_rn(o[j + 2 * i], o[j + 2 * i + 1]);
                *reinterpret_cast<uint4 *>(y + j) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (j + i < n) y[j + i] = __float2bfloat16_rn(o[j + i]);
            }
        }
    } else {
        float *y = static_cast<float *>(p.y) + at;
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            if (p.vec_y && j + 4 <= n) *reinterpret_cast<float4 *>(y + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
            else {
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (j + i < n) y[j + i] = o[j + i];
            }
        }
    }
}

// A tile of 128 rows of x (lanes of the tensor memory) x BN rows of w (columns).  Warp 0 loads, warp 1 issues, eight warps add up:
// a quadrant of the lanes and half of the columns each.  Two accumulators: the tensor core sums a block into one while the
// warps take the other.
template <int BN, bool W_ROWS>
__global__ void __launch_bounds__(F8_THREADS, 1) linear_f8_kernel(const __grid_constant__ F8Params p, const int stages) {
    constexpr int STAGE = F8_A_BYTES + BN * F8_BLOCK, COLS = BN / 2, CHUNK = 32;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[TC_MAX_STAGES], empty_bar[TC_MAX_STAGES], acc_full[2], acc_empty[2];
    __shared__ __align__(16) float col_scale[W_ROWS ? 2 : 1][W_ROWS ? BN : 4];
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_s;
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    volatile int *abort_flag = &abort_s;
    const int mt = (int)(blockIdx.x % (unsigned)p.m_tiles), nt = (int)(blockIdx.x / (unsigned)p.m_tiles);
    const int m0 = mt * TILE_M, f0 = nt * BN;
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; s++) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        for (int i = 0; i < 2; i++) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], F8_SUM_WARPS); }
        abort_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(&tmem_base_s, 2 * BN);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_s;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t ring = smem_u32(smem);
    const int blocks = p.blocks;

    if (warp == 0) {
        const uint32_t on = elect_one(), full0 = smem_u32(full_bar);
        int s = 0;
        uint32_t phase = 0;
        for (int b = 0; b < blocks; b++) {
            if (b >= stages && !__all_sync(0xffffffffu, mbar_wait(&empty_bar[s], phase ^ 1, abort_flag))) break;
            const uint32_t sa = ring + (uint32_t)(s * STAGE), fb = full0 + (uint32_t)(s * 8);
            mbar_expect_tx_if(on, fb, STAGE);
            tma_load_2d_if(on, sa, &p.tmX, fb, b * F8_BLOCK, m0);
            tma_load_2d_if(on, sa + F8_A_BYTES, &p.tmW, fb, b * F8_BLOCK, f0);
            if (++s == stages) { s = 0; phase ^= 1; }
        }
    } else if (warp == 1) {
        const uint32_t on = elect_one(), d_tmem = uniform(tmem_base), empty0 = smem_u32(empty_bar), acc0 = smem_u32(acc_full);
        const int n_mma = min(BN, (p.K - f0 + 15) & ~15);
        // instruction descriptor: fp32 accumulator at bit 4, operand formats at bits 7 / 10, N >> 3 at bit 17, M >> 4 at bit 24
        const uint32_t idesc = (1u << 4) | p.formats | ((uint32_t)(n_mma >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
        int s = 0;
        uint32_t phase = 0;
        for (int b = 0; b < blocks; b++) {
            const int a = b & 1;
            if (b >= 2 && !__all_sync(0xffffffffu, mbar_wait(&acc_empty[a], (uint32_t)((b >> 1) - 1) & 1, abort_flag))) break;
            if (!__all_sync(0xffffffffu, mbar_wait(&full_bar[s], phase, abort_flag))) break;
            tc_fence_after();
            const int steps = min(4, (p.C - b * F8_BLOCK + 31) / 32);
            const uint32_t sa = ring + (uint32_t)(s * STAGE);
            const uint64_t da = smem_desc_sw128(sa), db = smem_desc_sw128(sa + F8_A_BYTES);
#pragma unroll
            for (int q = 0; q < 4; q++)
                if (q < steps) umma_f8_if(on, d_tmem + (uint32_t)(a * BN), da + (uint64_t)(2 * q), db + (uint64_t)(2 * q), idesc, q > 0 ? 1u : 0u);
            umma_commit_if(on, empty0 + (uint32_t)(s * 8));
            umma_commit_if(on, acc0 + (uint32_t)(a * 8));
            if (++s == stages) { s = 0; phase ^= 1; }
        }
    } else {
        const int quad = warp & 3, half = warp >= 6 ? 1 : 0;  // (a warp reads the 32 lanes of its number modulo 4)
        const int m = m0 + quad * 32 + lane, c0 = half * COLS;
        const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)c0;
        const float *sx = p.sx + min(m, p.M - 1);
        // columns of this half lie in one block of 128 rows of w
        const float *sw = W_ROWS ? p.sw : p.sw + min(f0 + c0, p.K - 1) / 128;
        const int ht = (warp - 2) % 4 * 32 + lane;  // thread of the half
        const int my_col = min(f0 + c0 + ht, p.K - 1);
        float2 acc[COLS / 2];
#pragma unroll
        for (int j = 0; j < COLS / 2; j++) acc[j] = make_float2(0.f, 0.f);
        float next_x = ld_act(sx), next_w = W_ROWS ? (ht < COLS ? ld_act(sw + my_col) : 0.f) : ld_act(sw);
        for (int b = 0; b < blocks; b++) {
            const int a = b & 1;
            const float cur_x = next_x, cur_w = next_w;
            if (b + 1 < blocks) {
                next_x = ld_act(sx + (long long)(b + 1) * p.ldsx);
                if (W_ROWS) { if (ht < COLS) next_w = ld_act(sw + (long long)(b + 1) * p.ldsw + my_col); }
                else next_w = ld_act(sw + (long long)(b + 1) * p.ldsw);
            }
            if (W_ROWS) {
                if (ht < COLS) col_scale[a][c0 + ht] = cur_w;
                if (half) asm volatile("bar.sync 2, 128;" ::: "memory");
                else asm volatile("bar.sync 1, 128;" ::: "memory");
            }
            // (after a wait that ran out the warps still go through all steps: the others meet them at the barrier above)
            if (!__all_sync(0xffffffffu, mbar_wait(&acc_full[a], (uint32_t)(b >> 1) & 1, abort_flag))) continue;
            tc_fence_after();
            const float2 s2 = W_ROWS ? make_float2(cur_x, cur_x) : make_float2(cur_x * cur_w, cur_x * cur_w);
#pragma unroll
            for (int j0 = 0; j0 < COLS; j0 += CHUNK) {
                uint32_t v[CHUNK];
                tmem_ld32(taddr + (uint32_t)(a * BN + j0), v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < CHUNK / 2; j++) {
                    float2 f = s2;
                    if (W_ROWS) f = __fmul2_rn(s2, *reinterpret_cast<const float2 *>(&col_scale[a][c0 + j0 + 2 * j]));
                    acc[j0 / 2 + j] = __ffma2_rn(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), f, acc[j0 / 2 + j]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[a]);
        }
        if (!*abort_flag && m < p.M) {
            const int n = min(COLS, p.K - f0 - c0);
#pragma unroll
            for (int j = 0; j < COLS / 2; j++) {
                if (2 * j >= n) break;
                if (p.bias) {
                    acc[j].x += ld_act(p.bias + f0 + c0 + 2 * j);
                    if (2 * j + 1 < n) acc[j].y += ld_act(p.bias + f0 + c0 + 2 * j + 1);
                }
                acc[j].x = act_fn(acc[j].x, p.act);
                acc[j].y = act_fn(acc[j].y, p.act);
            }
            if (n > 0) store_row<COLS>(p, (long long)m * p.ldy + f0 + c0, reinterpret_cast<const float *>(acc), n);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (abort_s) {  // a wait ran out: report, let copies in flight land, then release the tensor memory
        if (threadIdx.x == 0) atomicExch(p.status, 1);
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 2000000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 1) { tc_fence_after(); tmem_dealloc(tmem_base, 2 * BN); }
}

DeviceBits g_set[4];

template <int BN, bool W_ROWS> cudaError_t launch_tiles(F8Params &p, const LinearF8Args &a, DeviceBits &done, cudaStream_t st) {
    constexpr int STAGE = F8_A_BYTES + BN * F8_BLOCK, STAGES = std::min(192 * 1024 / STAGE, TC_MAX_STAGES);
    if (!tc_encode_bytes(&p.tmX, a.x, (uint64_t)a.C, (uint64_t)a.M, (uint64_t)a.ldx, TILE_M) ||
        !tc_encode_bytes(&p.tmW, a.w, (uint64_t)a.C, (uint64_t)a.K, (uint64_t)a.ldw, BN))
        return cudaErrorInvalidValue;
    p.m_tiles = (a.M + TILE_M - 1) / TILE_M;
    p.n_tiles = (a.K + BN - 1) / BN;
    cudaError_t e = smem_limit_once(linear_f8_kernel<BN, W_ROWS>, STAGES * STAGE + 1024, done);
    if (e != cudaSuccess) return e;
    return launch_pdl(linear_f8_kernel<BN, W_ROWS>, dim3((unsigned)(p.m_tiles * p.n_tiles)), dim3(F8_THREADS), STAGES * STAGE + 1024, st, 1, p, STAGES);
}

}  // namespace

cudaError_t launch_linear_f8(const LinearF8Args &a, int device, cudaStream_t st) {
    F8Params p = {};
    p.sx = a.sx; p.sw = a.sw; p.bias = a.bias; p.y = a.y; p.status = tc_status_word(device);
    p.ldsx = a.ldsx; p.ldsw = a.ldsw; p.ldy = a.ldy;
    p.M = a.M; p.K = a.K; p.C = a.C; p.blocks = (a.C + F8_BLOCK - 1) / F8_BLOCK;
    p.act = a.act; p.y_bf16 = a.y_bf16;
    p.vec_y = ((reinterpret_cast<uintptr_t>(a.y) | (size_t)a.ldy * (a.y_bf16 ? 2 : 4)) & 15) == 0;
    p.formats = ((uint32_t)(a.x_e5m2 ? 1 : 0) << 7) | ((uint32_t)(a.w_e5m2 ? 1 : 0) << 10);
    const bool wide = a.K > 128 && (long long)((a.M + 127) / 128) * ((a.K + 255) / 256) >= sm_count();
    if (a.w_rows) return wide ? launch_tiles<256, true>(p, a, g_set[0], st) : launch_tiles<128, true>(p, a, g_set[1], st);
    return wide ? launch_tiles<256, false>(p, a, g_set[2], st) : launch_tiles<128, false>(p, a, g_set[3], st);
}

}  // namespace sgs
