// Operators on logits: the k largest of every row, and the distillation loss against a teacher's top logits with its gradient.
#include "sgs_internal.h"
#include "sgs_pdl.cuh"

#include <algorithm>

namespace sgs {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_huge_valf();

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float *p, float v) { *p = v; }
__device__ __forceinline__ void from_float(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// ---------------------------------------------------------------------------------------------
// Top logits.  A logit's rank is that of its 64-bit word: an order-preserving key of the value above the complement of its index, so
// that no two words are equal, larger values come first and of equal values (-0 and 0 are) the lower index.  NaN is the largest.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);  // (-0 becomes 0)
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int TOP_THREADS = 1024, TOP_CAP = 1024;

template <typename T> __global__ void __launch_bounds__(TOP_THREADS) top_logits_kernel(const T *z, float *values, int *index, int V, int k, long long ldz, long long ldt) {
    __shared__ uint64_t cand[TOP_CAP];
    __shared__ int n_cand;
    __shared__ int hist[256];
    __shared__ uint64_t prefix_s;
    __shared__ int want_s;
    pdl_launch_dependents();
    pdl_wait();
    const T *row = z + (long long)blockIdx.x * ldz;
    const int t = threadIdx.x;
    // The k-th largest of the threads' own maxima is a lower bound of the k-th largest logit.
    uint32_t most = 0;
    for (int i = t; i < V; i += TOP_THREADS) most = max(most, key_of(to_float(ld_act(row + i))));
    uint32_t least = 0;
    if (V > TOP_CAP)
        for (int b = 31; b >= 0; b--) {
            const uint32_t trial = least | (1u << b);
            if (__syncthreads_count(most >= trial) >= k) least = trial;
        }
    if (t == 0) n_cand = 0;
    __syncthreads();
    for (int i = t; i < V; i += TOP_THREADS) {
        const uint32_t key = key_of(to_float(ld_act(row + i)));
        if (key >= least) {
            const int at = atomicAdd(&n_cand, 1);  // (any order: the ranks below do not depend on it)
            if (at < TOP_CAP) cand[at] = (uint64_t)key << 32 | (uint32_t)~i;
        }
    }
    __syncthreads();
    int n = n_cand;
    if (n > TOP_CAP) {
        // Too many candidates (many equal values): the k-th largest word itself, eight bits at a time.
        uint64_t prefix = 0;
        int want = k;
        for (int shift = 56; shift >= 0; shift -= 8) {
            if (t < 256) hist[t] = 0;
            __syncthreads();
            for (int i0 = 0; i0 < V; i0 += TOP_THREADS) {
                const int i = i0 + t;
                int digit = -1;
                if (i < V) {
                    const uint64_t w = (uint64_t)key_of(to_float(ld_act(row + i))) << 32 | (uint32_t)~i;
                    if (shift == 56 || (w >> (shift + 8)) == (prefix >> (shift + 8))) digit = (int)(w >> shift) & 255;
                }
                const unsigned same = __match_any_sync(0xffffffffu, digit);
                if (digit >= 0 && (int)(__ffs(same) - 1) == (t & 31)) atomicAdd(&hist[digit], __popc(same));
            }
            __syncthreads();
            if (t == 0) {
                int d = 255, left = want;
                while (d > 0 && hist[d] < left) left -= hist[d--];
                prefix_s = prefix | (uint64_t)d << shift;
                want_s = left;
            }
            __syncthreads();
            prefix = prefix_s;
            want = want_s;
        }
        if (t == 0) n_cand = 0;
        __syncthreads();
        for (int i = t; i < V; i += TOP_THREADS) {
            const uint64_t w = (uint64_t)key_of(to_float(ld_act(row + i))) << 32 | (uint32_t)~i;
            if (w >= prefix) cand[atomicAdd(&n_cand, 1)] = w;  // (exactly k of them)
        }
        __syncthreads();
        n = n_cand;
    }
    if (t < n) {
        const uint64_t w = cand[t];
        int rank = 0;
        for (int i = 0; i < n; i++) rank += cand[i] > w;
        if (rank < k) {
            const int i = (int)~(uint32_t)w;
            values[(long long)blockIdx.x * ldt + rank] = to_float(ld_act(row + i));
            index[(long long)blockIdx.x * ldt + rank] = i;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Distillation
// ---------------------------------------------------------------------------------------------
constexpr int DIS_THREADS = 512;

template <typename Op> __device__ __forceinline__ float block_reduce(float v, float *buf, Op op) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = buf[0];
    for (int i = 1; i < (int)(blockDim.x >> 5); i++) v = op(v, buf[i]);
    return v;
}
__device__ __forceinline__ float fmax_op(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float add_op(float a, float b) { return a + b; }

template <typename T> struct DisParams {
    const T *z;
    T *dz;
    const float *teacher, *row_scale;
    const int *index;
    float *loss, *stat;
    int V, k, backward;
    long long ldz, lddz, ldt;
    float inv_t, temperature, grad_scale;
};

template <typename T> __global__ void __launch_bounds__(DIS_THREADS) distill_kernel(const DisParams<T> p) {
    __shared__ float buf[32];
    __shared__ int at[DISTILL_TOP_MAX];
    __shared__ float prob[DISTILL_TOP_MAX], zl[DISTILL_TOP_MAX];
    pdl_launch_dependents();
    pdl_wait();
    const int t = threadIdx.x, V = p.V, k = p.k;
    const long long r = blockIdx.x;
    const T *row = p.z + r * p.ldz;
    const float a = p.inv_t * LOG2E;
    // the teacher's distribution over the slots in use
    float tmax = NEG_INF;
    bool used_any = false, nan_any = false;
    for (int j = t; j < k; j += DIS_THREADS) {
        int i = ld_act(p.index + r * p.ldt + j);
        const float v = ld_act(p.teacher + r * p.ldt + j);
        if (i < 0 || i >= V || v == NEG_INF) i = -1;
        at[j] = i;
        prob[j] = v;
        if (i >= 0) { tmax = fmaxf(tmax, v); used_any = true; nan_any |= v != v; }
    }
    const bool used = __syncthreads_or(used_any);
    (void)nan_any;
    tmax = block_reduce(tmax, buf, fmax_op);
    if (tmax == NEG_INF) tmax = 0.f;  // (all NaN)
    float tsum = 0.f;
    for (int j = t; j < k; j += DIS_THREADS) {
        const float e = at[j] >= 0 ? exp2f((prob[j] - tmax) * a) : 0.f;
        zl[j] = at[j] >= 0 ? to_float(ld_act(row + at[j])) : 0.f;
        tsum += e;
    }
    tsum = block_reduce(tsum, buf, add_op);
    // the student's statistics
    float zmax = NEG_INF, logsum;
    if (p.backward) {
        zmax = ld_act(p.stat + 2 * r);
        logsum = ld_act(p.stat + 2 * r + 1);
    } else {
        for (int i = t; i < V; i += DIS_THREADS) zmax = fmaxf(zmax, to_float(ld_act(row + i)));
        zmax = block_reduce(zmax, buf, fmax_op);
        const float base = zmax == NEG_INF ? 0.f : zmax;
        float s = 0.f;
        for (int i = t; i < V; i += DIS_THREADS) s += exp2f((to_float(ld_act(row + i)) - base) * a);
        logsum = logf(block_reduce(s, buf, add_op));
    }
    const float base = zmax == NEG_INF ? 0.f : zmax, off = zmax == NEG_INF ? 0.f : logsum;
    const float log_tsum = logf(tsum);
    if (!p.backward) {
        float loss = 0.f;
        for (int j = t; j < k; j += DIS_THREADS)
            if (at[j] >= 0) {
                // T (log p - log q), with differences of logits as they are: masks of the type's lowest value do not overflow
                const float term = (prob[j] - tmax) - (zl[j] - base) + p.temperature * (off - log_tsum);
                const float pj = exp2f((prob[j] - tmax) * a) / tsum;
                if (!(pj <= 0.f)) loss += pj * term;
            }
        loss = block_reduce(loss, buf, add_op);
        if (t == 0) {
            p.loss[r] = used ? loss * p.temperature : 0.f;
            if (p.stat) { p.stat[2 * r] = zmax; p.stat[2 * r + 1] = logsum; }
        }
    }
    if (!p.dz) return;
    __syncthreads();
    for (int j = t; j < k; j += DIS_THREADS) prob[j] = at[j] >= 0 ? exp2f((prob[j] - tmax) * a) / tsum : 0.f;
    T *out = p.dz + r * p.lddz;
    const float c = used ? p.grad_scale * p.temperature * (p.row_scale ? ld_act(p.row_scale + r) : 1.f) : 0.f;
    const float off2 = off * LOG2E;
    if (c == 0.f) {
        for (int i = t; i < V; i += DIS_THREADS) from_float(out + i, 0.f);
        return;
    }
    for (int i = t; i < V; i += DIS_THREADS) from_float(out + i, c * exp2f((to_float(ld_act(row + i)) - base) * a - off2));
    __syncthreads();
    for (int j = t; j < k; j += DIS_THREADS) {
        if (at[j] < 0) continue;
        float sum = 0.f;
        for (int i = 0; i < k; i++) sum += at[i] == at[j] ? prob[i] : 0.f;
        from_float(out + at[j], c * (exp2f((zl[j] - base) * a - off2) - sum));
    }
}

template <typename T> cudaError_t launch_distill_type(const DistillArgs &a, cudaStream_t st) {
    DisParams<T> p;
    p.z = static_cast<const T *>(a.z); p.dz = static_cast<T *>(a.dz);
    p.teacher = a.teacher; p.row_scale = a.row_scale; p.index = a.index; p.loss = a.loss; p.stat = a.stat;
    p.V = a.classes; p.k = a.top; p.backward = a.backward; p.ldz = a.ldz; p.lddz = a.lddz; p.ldt = a.ldt;
    p.inv_t = 1.f / a.temperature; p.temperature = a.temperature; p.grad_scale = a.grad_scale;
    return launch_pdl(distill_kernel<T>, dim3((unsigned)a.rows), dim3(DIS_THREADS), 0, st, 1, p);
}

}  // namespace

cudaError_t launch_top_logits(const TopArgs &a, cudaStream_t st) {
    if (a.bf16)
        return launch_pdl(top_logits_kernel<__nv_bfloat16>, dim3((unsigned)a.rows), dim3(TOP_THREADS), 0, st, 1, static_cast<const __nv_bfloat16 *>(a.z), a.values,
                          a.index, a.classes, a.top, a.ldz, a.ldt);
    return launch_pdl(top_logits_kernel<float>, dim3((unsigned)a.rows), dim3(TOP_THREADS), 0, st, 1, static_cast<const float *>(a.z), a.values, a.index,
                      a.classes, a.top, a.ldz, a.ldt);
}

cudaError_t launch_distill(const DistillArgs &a, cudaStream_t st) {
    return a.bf16 ? launch_distill_type<__nv_bfloat16>(a, st) : launch_distill_type<float>(a, st);
}

}  // namespace sgs
