// Operators on logits: the k largest of every row, and the distillation loss against a teacher's top logits with its gradient.
//
// Both read rows of some thousand to some hundred thousand logits and are bound by bytes where there are many rows and by a chain of
// latencies where there are few.  Hence for both: a row is one block's, or the blocks of a cluster take contiguous parts of it and meet
// through distributed shared memory where the rows alone do not fill the GPU; copies of 16 bytes into shared memory run ahead of their
// use, from the first aligned element of a row on (rows of an odd pitch start anywhere); and a second pass reads a row again instead of
// keeping it: two blocks an SM are between their passes with 39 MB of rows of 128 KB, which stay in the 126 MB L2 (four blocks an SM, and
// what they write, do not: 2048 x 65536 bf16 takes 121 us then, 113 with two).
// Measured (B200): top 64 of 512 x 131071 bf16 32.4 us (4.1 TB/s), fp32 52.7 us (5.1 TB/s), top 32 of 8192 x 1000 fp32 39 us; loss and
// gradient of 2048 x 65536 bf16 113 us (4.8 TB/s of what has to be read and written; 110 where a sixteenth of the rows have no list), fp32
// 200 us (5.4 TB/s); the loss alone 50 and 84 us; the gradient of 1000 x 100008 bf16 72.4 us (5.5 TB/s); the loss of 64 x 1000 fp32 3.2 us.
#include "sgs_internal.h"
#include "sgs_pdl.cuh"

#include <algorithm>
#include <cmath>

namespace sgs {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_huge_valf();

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_float(float *p, float v) { *p = v; }
__device__ __forceinline__ void from_float(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// 16 bytes of a row.
template <typename T> struct Vec { static constexpr int N = 16 / (int)sizeof(T); };
__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[4]) {
    v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
}
__device__ __forceinline__ void unpack(const uint4 &q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; j++) { v[2 * j] = __uint_as_float(w[j] << 16); v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint4 q;
    __nv_bfloat162 *b = reinterpret_cast<__nv_bfloat162 *>(&q);
#pragma unroll
    for (int j = 0; j < 4; j++) b[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
    return q;
}

// How a row of V elements splits: `head` elements up to the first 16-byte boundary, vectors, the rest; the vectors are divided among
// the blocks of the cluster, the head and the rest (fewer than two vectors together) belong to block 0.
struct Split {
    int head, first, last, edges;  // vectors first .. last - 1 are this block's
    long long tail;                // first element behind the vectors
    __device__ long long edge(int e) const { return e < head ? e : tail + (e - head); }
};
template <typename T> __device__ __forceinline__ Split split_row(const T *row, int V, int part, int parts) {
    constexpr int N = Vec<T>::N;
    Split s;
    s.head = min(V, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T));
    const int n = (V - s.head) / N;
    s.first = (int)((long long)n * part / parts);
    s.last = (int)((long long)n * (part + 1) / parts);
    s.tail = s.head + (long long)n * N;
    s.edges = part == 0 ? s.head + (int)(V - s.tail) : 0;
    return s;
}

// Calls f(vector, its number) for this thread's vectors first + t, first + t + TEAM ...  Copies into a ring of the thread's own places in
// shared memory run six to eight vectors ahead: enough bytes under way for HBM's latency (two blocks of 512 threads: 128 KB an SM), which
// registers do not hold, and nothing to wait for but the thread's own copies.
constexpr int STREAM_STAGES = 4, STREAM_PAIR = 2, STREAM_RING = STREAM_STAGES * STREAM_PAIR;  // stages of two vectors
template <bool LAST_USE> __device__ __forceinline__ void copy16(uint32_t dst, const uint4 *src, uint64_t policy) {  // LAST_USE: with an L2 policy
    if (LAST_USE) asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
    else asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
template <int TEAM, int BLOCK, bool LAST_USE = false, typename F> __device__ __forceinline__ void stream(uint4 *ring_, const uint4 *vec, int first, int last, int t, F f) {
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ring_ + threadIdx.x);
    constexpr uint32_t STAGE = STREAM_PAIR * BLOCK * 16;
    int ahead = first + t;  // next vector to ask for
    uint64_t policy = 0;
    if (LAST_USE) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    auto ask = [&](uint32_t at) {
#pragma unroll
        for (int u = 0; u < STREAM_PAIR; u++)
            if (ahead + u * TEAM < last) copy16<LAST_USE>(at + u * BLOCK * 16, vec + ahead + u * TEAM, policy);
        asm volatile("cp.async.commit_group;" ::: "memory");
        ahead += STREAM_PAIR * TEAM;
    };
#pragma unroll
    for (int d = 0; d < STREAM_STAGES - 1; d++) ask(ring + d * STAGE);
    uint32_t at = ring, free_ = ring + (STREAM_STAGES - 1) * STAGE;
    for (int i = first + t; i < last; i += STREAM_PAIR * TEAM) {
        ask(free_);  // (its vectors were used in the last step)
        asm volatile("cp.async.wait_group %0;" ::"n"(STREAM_STAGES - 1) : "memory");
        uint4 q[STREAM_PAIR];
#pragma unroll
        for (int u = 0; u < STREAM_PAIR; u++)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q[u].x), "=r"(q[u].y), "=r"(q[u].z), "=r"(q[u].w) : "r"(at + u * BLOCK * 16) : "memory");
#pragma unroll
        for (int u = 0; u < STREAM_PAIR; u++)
            if (i + u * TEAM < last) f(q[u], i + u * TEAM);
        free_ = at;
        at = at == ring + (STREAM_STAGES - 1) * STAGE ? ring : at + STAGE;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---- clusters along z ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_addr(const void *p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 peer_ld2(uint32_t a) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void peer_st64(uint32_t a, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }

// Blocks a row: as many as give every SM two blocks, but none less than `least` bytes.
int parts_for(long long rows, double row_bytes, double least) {
    int parts = 1;
    while (parts < 8 && rows * parts < 2ll * sm_count() && row_bytes / (2 * parts) >= least) parts *= 2;
    return parts;
}

// ---------------------------------------------------------------------------------------------
// Top logits.  A logit's rank is that of its 64-bit word: an order-preserving key of the value above the complement of its index, so
// that no two words are equal, larger values come first and of equal values (-0 and 0 are) the lower index.  NaN is the largest.
//
// A row (or part) in two passes: the k-th largest of the threads' own maxima bounds the k-th largest logit from below, and few more
// than k logits reach it; these are collected, from the threads whose maximum does, and ranked by counting.  Rows where too many reach
// it (many equal values) find the k-th largest word eight bits at a time.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);  // (-0 becomes 0)
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }  // (NaN: 0x7fffffff)
__device__ __forceinline__ uint64_t word_of(float v, uint32_t i) { return (uint64_t)key_of(v) << 32 | (uint32_t)~i; }
// Maximum that is NaN if one operand is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float vec_max(const uint4 &q, const float *) {
    return max_nan(max_nan(__uint_as_float(q.x), __uint_as_float(q.y)), max_nan(__uint_as_float(q.z), __uint_as_float(q.w)));
}
__device__ __forceinline__ float vec_max(const uint4 &q, const __nv_bfloat16 *) {
    const uint32_t m = max_nan2(max_nan2(q.x, q.y), max_nan2(q.z, q.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}

constexpr int TOP_CAP = 1024;
struct TopParams {
    const void *z;
    float *values;
    int *index;
    int V, k, parts;
    long long ldz, ldt;
};

template <typename T, int THREADS> __global__ void __launch_bounds__(THREADS, 1024 / THREADS) top_logits_kernel(const TopParams p) {
    constexpr int N = Vec<T>::N;
    extern __shared__ uint4 ring[];
    uint64_t *joined = reinterpret_cast<uint64_t *>(ring);  // block 0, when the row has been read: the parts' words
    __shared__ uint64_t cand[TOP_CAP];
    __shared__ int n_cand, n_hot, want_s, hot[THREADS];
    __shared__ uint2 range[THREADS / 32];
    __shared__ uint32_t prefix_s;
    __shared__ int hist[256];
    const int t = threadIdx.x, part = (int)blockIdx.z, k = p.k;
    pdl_launch_dependents();
    pdl_wait();
    const T *row = static_cast<const T *>(p.z) + (long long)blockIdx.x * p.ldz;
    const Split s = split_row(row, p.V, part, p.parts);
    const uint4 *vec = reinterpret_cast<const uint4 *>(row + s.head);
    // Calls f(vector, its first element) for this thread's vectors, f1(value, element) for its share of the edges.
    auto walk = [&](auto f, auto f1) {
        stream<THREADS, THREADS>(ring, vec, s.first, s.last, t, [&](const uint4 &q, int i) { f(q, (uint32_t)(s.head + i * N)); });
        if (t < s.edges) { const long long e = s.edge(t); f1(to_float(ld_act(row + e)), (uint32_t)e); }
    };
    // Short rows, where vectors would leave threads without any logit: element by element.  (A row that a cluster shares is never short.)
    const bool brief = p.parts == 1 && p.V <= 2 * N * THREADS;
    auto each = [&](auto f1) {
        for (int i = t; i < p.V; i += THREADS) f1(to_float(ld_act(row + i)), (uint32_t)i);
    };
    uint32_t most = 0;  // largest key (0: below every key)
    int top_vec = -1;   // the vector that has it
    float second = NEG_INF;  // largest of the thread's other vectors
    if (brief) each([&](float v, uint32_t) { most = max(most, key_of(v)); });
    else {
        float m = NEG_INF;
        stream<THREADS, THREADS>(ring, vec, s.first, s.last, t, [&](const uint4 &q, int i) {
            const float v = vec_max(q, (const T *)nullptr);
            const bool up = top_vec < 0 || !(v <= m);  // (the first; larger, or NaN)
            second = max_nan(second, up ? m : v);
            m = up ? v : m;
            top_vec = up ? i : top_vec;
        });
        most = max(key_of(m), key_of(second));  // (a NaN may be behind the second)
    }
    // A bound that a few more than k of the maxima reach will do: halve the range of the maxima until one is found.
    uint32_t least = 0;
    {
        const uint32_t lo1 = __reduce_min_sync(0xffffffffu, most), hi1 = __reduce_max_sync(0xffffffffu, most);
        if ((t & 31) == 0) range[t >> 5] = make_uint2(lo1, hi1);
        __syncthreads();
        uint32_t lo = 0xffffffffu, hi = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 32; i++) { lo = min(lo, range[i].x); hi = max(hi, range[i].y); }
        const int enough = k + k / 4 + 8;
        if (THREADS >= k && __syncthreads_count(most > 0) >= k) {
            least = lo;  // (all reach it)
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo) / 2 + 1;
                const int count = __syncthreads_count(most >= mid);
                if (count >= k) {
                    lo = least = mid;
                    if (count <= enough) break;
                } else hi = mid - 1;
            }
        }
    }
    if (t == 0) n_cand = n_hot = 0;
    __syncthreads();
    auto take = [&](float v, uint32_t i) {
        const uint32_t key = key_of(v);
        if (key >= least && *(volatile int *)&n_cand <= TOP_CAP) {  // (more than enough are counted no further)
            const int at = atomicAdd(&n_cand, 1);  // (any order: the ranks below do not depend on it)
            if (at < TOP_CAP) cand[at] = (uint64_t)key << 32 | (uint32_t)~i;
        }
    };
    if (brief) each(take);
    else {
        // Of the threads whose maximum reaches the bound most have one vector that does: it is read again; where another one does too, all
        // of the thread's are, a warp a thread's.
        auto look = [&](const uint4 &q, int i) {
            float v[N];
            unpack(q, v);
#pragma unroll
            for (int j = 0; j < N; j++) take(v[j], (uint32_t)(s.head + (long long)i * N + j));
        };
        if (most >= least) {
            if (key_of(second) >= least) hot[atomicAdd(&n_hot, 1)] = t;  // (any order, as above)
            else look(ld_act(vec + top_vec), top_vec);
        }
        __syncthreads();
        const int rescans = n_hot;
        for (int h = t >> 5; h < rescans; h += THREADS / 32)
            for (int i = s.first + hot[h] + (t & 31) * THREADS; i < s.last; i += 32 * THREADS) {
                const uint4 q = ld_act(vec + i);
                if (key_of(vec_max(q, (const T *)nullptr)) >= least) look(q, i);
            }
        if (t < s.edges) { const long long e = s.edge(t); take(to_float(ld_act(row + e)), (uint32_t)e); }
    }
    __syncthreads();
    int n = n_cand;
    // (Ranks cost the square, the way below some passes over the row: of 1000 zeros it takes 37 us for 512 rows and k = 64, ranking them all 151.)
    if (n > (brief ? min(TOP_CAP, 2 * k + 256) : TOP_CAP)) {
        // The k-th largest key itself, eight bits at a time; then the larger ones in any order and as many of its equals as are wanted, by
        // their index.
        constexpr int LOW = sizeof(T) == 2 ? 16 : 0;  // (a bf16's key has its lower half from its sign)
        uint32_t prefix = 0;
        int want = k;  // of the keys that begin with prefix
        for (int shift = 24; shift >= LOW; shift -= 8) {
            for (int i = t; i < 256; i += THREADS) hist[i] = 0;
            __syncthreads();
            // (rows come here for values that repeat: the thread keeps the counts of its last two digits)
            int d0 = -1, n0 = 0, d1 = -1, n1 = 0;
            auto tally = [&](float v, uint32_t) {
                const uint32_t key = key_of(v);
                if (shift < 24 && (key >> (shift + 8)) != (prefix >> (shift + 8))) return;
                const int d = (int)(key >> shift) & 255;
                if (d == d0) n0++;
                else if (d == d1) n1++;
                else {
                    if (n1) atomicAdd(&hist[d1], n1);
                    d1 = d0; n1 = n0;
                    d0 = d; n0 = 1;
                }
            };
            if (brief) each(tally);
            else
                walk([&](const uint4 &q, uint32_t i) {
                    float v[N];
                    unpack(q, v);
#pragma unroll
                    for (int j = 0; j < N; j++) tally(v[j], i + j);
                }, tally);
            if (n0) atomicAdd(&hist[d0], n0);
            if (n1) atomicAdd(&hist[d1], n1);
            __syncthreads();
            if (t == 0) {
                int d = 255, left = want;
                while (d > 0 && hist[d] < left) left -= hist[d--];
                prefix_s = prefix | (uint32_t)d << shift;
                want_s = left;
            }
            __syncthreads();
            prefix = prefix_s;
            want = want_s;
        }
        if (t == 0) n_cand = 0;
        __syncthreads();
        auto keep = [&](float v, uint32_t i) {
            if (key_of(v) >> LOW > prefix >> LOW) cand[atomicAdd(&n_cand, 1)] = word_of(v, i);  // (k - want of them)
        };
        if (brief) each(keep);
        else
            walk([&](const uint4 &q, uint32_t i) {
                if (key_of(vec_max(q, (const T *)nullptr)) >> LOW <= prefix >> LOW) return;
                float v[N];
                unpack(q, v);
#pragma unroll
                for (int j = 0; j < N; j++) keep(v[j], i + j);
            }, keep);
        // this block's elements in the order of their index: its share of the head, its vectors, its share of the rest
        const long long head = part == 0 ? s.head : 0, middle = head + (long long)(s.last - s.first) * N, all = middle + (part == 0 ? p.V - s.tail : 0);
        int found = 0;
        for (long long j0 = 0; j0 < all && found < want; j0 += THREADS) {
            const long long j = j0 + t, i = j < head ? j : j < middle ? s.head + (long long)s.first * N + (j - head) : s.tail + (j - middle);
            const float v = j < all ? to_float(ld_act(row + i)) : 0.f;
            const bool same = j < all && key_of(v) >> LOW == prefix >> LOW;
            const unsigned lanes = __ballot_sync(0xffffffffu, same);
            __syncthreads();  // (the last round's counts have been read)
            if ((t & 31) == 0) hist[t >> 5] = __popc(lanes);
            __syncthreads();
            int at = found + __popc(lanes & ((1u << (t & 31)) - 1));
#pragma unroll
            for (int w = 0; w < THREADS / 32; w++) {
                if (w < t >> 5) at += hist[w];
                found += hist[w];
            }
            if (same && at < want) cand[k - want + at] = word_of(v, (uint32_t)i);
        }
        __syncthreads();
        n = k;
    }
    float *values = p.values + (long long)blockIdx.x * p.ldt;
    int *index = p.index + (long long)blockIdx.x * p.ldt;
    auto write = [&](int rank, uint64_t w) {
        values[rank] = value_of((uint32_t)(w >> 32));
        index[rank] = (int)~(uint32_t)w;
    };
    if (p.parts == 1) {
        for (int c = t; c < n; c += THREADS) {
            const uint64_t w = cand[c];
            int rank = 0;
            for (int i = 0; i < n; i++) rank += cand[i] > w;
            if (rank < k) write(rank, w);
        }
        return;
    }
    if (part == 0)
        for (int c = t; c < p.parts * k; c += THREADS) joined[c] = 0;  // (no logit's word)
    cluster_arrive();
    cluster_wait();
    for (int c = t; c < n; c += THREADS) {
        const uint64_t w = cand[c];
        int rank = 0;
        for (int i = 0; i < n; i++) rank += cand[i] > w;
        if (rank < k) peer_st64(peer_addr(&joined[part * k + rank], 0), w);
    }
    cluster_arrive();
    cluster_wait();
    if (part) return;
    for (int c = t; c < p.parts * k; c += THREADS) {
        const uint64_t w = joined[c];
        // own part's words are sorted: the rank there is known, of another part's it is the number of larger ones
        int rank = c % k;
        if (!w) continue;
        for (int q = 0; q < p.parts; q++) {
            if (q == c / k) continue;
            int lo = 0, hi = k;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (joined[q * k + mid] > w) lo = mid + 1;
                else hi = mid;
            }
            rank += lo;
        }
        if (rank < k) write(rank, w);
    }
}

// ---------------------------------------------------------------------------------------------
// Distillation.  One pass keeps a running maximum and a sum of exponentials relative to it, a second writes the gradient.
// ---------------------------------------------------------------------------------------------
// 2^x; results below the normal range are 0.
__device__ __forceinline__ float pow2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// (largest, sum of 2^(a (v - largest))) of two sets; of an empty set or one of -infinities: (-infinity, 0).
__device__ __forceinline__ float2 join(float2 p, float2 q, float a) {
    const float m = fmaxf(p.x, q.x), b = m == NEG_INF ? 0.f : m;
    return make_float2(m, p.y * pow2((p.x - b) * a) + q.y * pow2((q.x - b) * a));
}
// The same of all values of a warp: largest first, then the sums relative to it.
__device__ __forceinline__ float2 warp_join(float2 v, float a) {
    float m = v.x;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float s = v.y * pow2((v.x - (m == NEG_INF ? 0.f : m)) * a);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return make_float2(m, s);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The largest of a vector's elements, NaN left out.
__device__ __forceinline__ float vec_most(const uint4 &q, const float *) {
    return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
}
__device__ __forceinline__ float vec_most(const uint4 &q, const __nv_bfloat16 *) {
    auto two = [](uint32_t x, uint32_t y) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
        return r;
    };
    const uint32_t m = two(two(q.x, q.y), two(q.z, q.w));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}

struct DisParams {
    const void *z;
    void *dz;
    const float *teacher, *row_scale;
    const int *index;
    float *loss, *stat;
    int V, k, backward, parts, table;  // table: places of the table of classes, a power of two
    long long ldz, lddz, ldt;
    float inv_t, temperature;
    float grad_factor[3];  // their product is grad_scale * temperature, which may leave fp32's range where its product with a row's scale does not
};

// A team of TEAM threads takes a row (or a cluster's part of one): a block, or for short rows a warp, eight to a block.
//
// What costs time besides the bytes is the chain of one row: list, row, two reductions, gradient.  So the list and the row's scale are
// asked for before the row is streamed and looked at behind it, the loss is summed behind the gradient, and the sums over slots that name
// the same class are formed by the threads that own the slots while the others write.
template <typename T, int TEAM, int BLOCK> __global__ void __launch_bounds__(BLOCK, 1024 / BLOCK) distill_kernel(const DisParams p, const int rows) {
    constexpr int N = Vec<T>::N, TEAMS = BLOCK / TEAM, SLOTS = TEAM == 32 ? 4 : DISTILL_TOP_MAX / TEAM;
    // a row's slots: (class, probability), class -1: not in use; then, for long lists, a table of the classes named, which tells whether one is
    // named twice
    extern __shared__ uint4 ring[];
    float2 *lists = reinterpret_cast<float2 *>(ring + BLOCK * STREAM_RING);
    __shared__ int twice[TEAMS];
    __shared__ float4 joined[BLOCK / 32];
    __shared__ float sums[BLOCK / 32];
    __shared__ __align__(8) float2 mine;
    const int t = (int)threadIdx.x % TEAM, team = (int)threadIdx.x / TEAM, V = p.V, k = p.k, part = (int)blockIdx.z;
    const long long r = (long long)blockIdx.x * TEAMS + team;
    pdl_launch_dependents();
    pdl_wait();
    if (TEAM == 32 && r >= rows) return;
    auto sync = [&] {
        if (TEAM == 32) __syncwarp();
        else __syncthreads();
    };
    float2 *list = lists + team * (k + p.table / 2);
    int *table = reinterpret_cast<int *>(list + k);
    if (p.table) {
        for (int j = t; j < p.table; j += TEAM) table[j] = -1;
        if (t == 0) twice[team] = 0;
        sync();
    }
    const T *row = static_cast<const T *>(p.z) + r * p.ldz;
    const float a = p.inv_t * LOG2E;
    const Split s = split_row(row, V, part, p.parts);
    const uint4 *vec = reinterpret_cast<const uint4 *>(row + s.head);
    int at[SLOTS];
    float tv[SLOTS], zl[SLOTS];
#pragma unroll
    for (int q = 0; q < SLOTS; q++) {
        const bool in = t + q * TEAM < k;
        at[q] = in ? ld_act(p.index + r * p.ldt + t + q * TEAM) : -1;
        tv[q] = in ? ld_act(p.teacher + r * p.ldt + t + q * TEAM) : NEG_INF;
    }
    const float row_scale = p.dz && p.row_scale ? ld_act(p.row_scale + r) : 1.f;
    float2 stud = make_float2(NEG_INF, 0.f), kept = make_float2(NEG_INF, 0.f);
    if (p.backward) kept = make_float2(ld_act(p.stat + 2 * r), ld_act(p.stat + 2 * r + 1));
    else {
        // (two elements an instruction where there is one for that)
        const float2 a2 = make_float2(a, a);
        float m = NEG_INF;
        float2 sum = make_float2(0.f, 0.f);
        auto raise = [&](float most) {  // the largest of the next elements
            if (most > m) {
                const float f = pow2((m - most) * a);
                sum.x *= f; sum.y *= f;
                m = most;
            }
            return m == NEG_INF ? 0.f : -m;
        };
        stream<TEAM, BLOCK>(ring, vec, s.first, s.last, t, [&](const uint4 &q, int) {
            float v[N];
            unpack(q, v);
            const float b = raise(vec_most(q, (const T *)nullptr));
            const float2 b2 = make_float2(b, b);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const float2 x = __fmul2_rn(__fadd2_rn(make_float2(v[j], v[j + 1]), b2), a2);
                sum = __fadd2_rn(sum, make_float2(pow2(x.x), pow2(x.y)));
            }
        });
        if (t < s.edges) {
            const float v = to_float(ld_act(row + s.edge(t))), b = raise(v == v ? v : NEG_INF);
            sum.x += pow2((v + b) * a);
        }
        stud = make_float2(m, sum.x + sum.y);
    }
    // the teacher's list (every block of the row reads it)
    float2 teach = make_float2(NEG_INF, 0.f);
#pragma unroll
    for (int q = 0; q < SLOTS; q++) {
        if (at[q] < 0 || at[q] >= V || tv[q] == NEG_INF) at[q] = -1;
        zl[q] = at[q] >= 0 ? to_float(ld_act(row + at[q])) : 0.f;
        if (at[q] < 0) continue;
        teach = join(teach, make_float2(tv[q] == tv[q] ? tv[q] : NEG_INF, tv[q] == tv[q] ? 1.f : tv[q]), a);
        if (p.table)
            for (int h = (int)((unsigned)at[q] * 40503u) & (p.table - 1);; h = (h + 1) & (p.table - 1)) {  // (never full: it has at least twice as many places as slots)
                const int there = atomicCAS(&table[h], -1, at[q]);
                if (there == at[q]) twice[team] = 1;
                if (there == -1 || there == at[q]) break;
            }
    }
    stud = warp_join(stud, a);
    teach = warp_join(teach, a);
    if (TEAM > 32) {
        if ((t & 31) == 0) joined[t >> 5] = make_float4(stud.x, stud.y, teach.x, teach.y);
        __syncthreads();
        const float4 j = (t & 31) < TEAM / 32 ? joined[t & 31] : make_float4(NEG_INF, 0.f, NEG_INF, 0.f);
        stud = warp_join(make_float2(j.x, j.y), a);
        teach = warp_join(make_float2(j.z, j.w), a);
    }
    const bool used = !(teach.x == NEG_INF && teach.y == 0.f);  // (a sum of NaN is one: slots are in use)
    const bool meet = TEAM > 32 && p.parts > 1 && !p.backward;
    if (meet) {
        if (t == 0) mine = stud;
        cluster_arrive();
        cluster_wait();
        stud = (t & 31) < p.parts ? peer_ld2(peer_addr(&mine, t & 31)) : make_float2(NEG_INF, 0.f);
        stud = warp_join(stud, a);
        cluster_arrive();  // (nobody leaves before all have read: the wait is at the end)
    }
    // The running maximum leaves NaN out, the sum does not.  A row is empty where its sum is 0, not where the largest of its numbers is minus
    // infinity: beside that there may be a NaN.
    const float zmax = p.backward ? kept.x : stud.x, logsum = p.backward ? kept.y : logf(stud.y);
    const float base = zmax == NEG_INF ? 0.f : zmax, off = logsum == NEG_INF ? 0.f : logsum;
    const float tmax = teach.x == NEG_INF ? 0.f : teach.x, tsum = teach.y;
    const float c = used ? row_scale * p.grad_factor[0] * p.grad_factor[1] * p.grad_factor[2] : 0.f, off2 = off * LOG2E;
    float loss = 0.f;
    const float log_tsum = logf(tsum);
#pragma unroll
    for (int q = 0; q < SLOTS; q++) {
        if (t + q * TEAM >= k) continue;
        const float pj = at[q] >= 0 ? pow2((tv[q] - tmax) * a) / tsum : 0.f;
        // T (log p - log q), with differences of logits as they are: masks of the type's lowest value do not overflow
        if (at[q] >= 0 && !(pj <= 0.f)) loss += pj * ((tv[q] - tmax) - (zl[q] - base) + p.temperature * (off - log_tsum));
        if (p.dz) list[t + q * TEAM] = make_float2(__int_as_float(at[q]), pj);
    }
    if (p.dz) {
        T *out = static_cast<T *>(p.dz) + r * p.lddz;
        sync();
        // the named classes of this part: q less the probability of all slots with that class, rounded once, written behind the others
        const long long e0 = s.head + (long long)s.first * N, e1 = s.head + (long long)s.last * N;
        float named[SLOTS];
#pragma unroll
        for (int q = 0; q < SLOTS; q++) {
            const int i = at[q];
            if (!((i >= e0 && i < e1) || (part == 0 && i >= 0 && (i < s.head || i >= s.tail)))) at[q] = -1;
            named[q] = 0.f;
            if (at[q] < 0 || c == 0.f) continue;
            float sum = list[t + q * TEAM].y;
            if (!p.table || twice[team]) {
                sum = 0.f;
                for (int l = 0; l < k; l++) sum += __float_as_int(list[l].x) == i ? list[l].y : 0.f;
            }
            named[q] = c * (pow2((zl[q] - base) * a - off2) - sum);
        }
        // fp32 rows: what is read for the last time and what is written make way in L2 for the rows between their passes (2048 x 65536: 239 us,
        // 200 with it; bf16 rows, half as many bytes in L2, take 113 and 131 us)
        constexpr bool FIRST_OUT = sizeof(T) == 4;
        const bool same = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
        const float2 a2 = make_float2(a, a), base2 = make_float2(-base, -base), less2 = make_float2(-off2, -off2), c2 = make_float2(c, c);
        auto store = [&](int i, const float (&v)[N]) {
            T *dst = out + s.head + (long long)i * N;
            if (same && FIRST_OUT) __stcs(reinterpret_cast<uint4 *>(dst), pack(v));
            else if (same) *reinterpret_cast<uint4 *>(dst) = pack(v);
            else {
#pragma unroll
                for (int j = 0; j < N; j++) from_float(dst + j, v[j]);
            }
        };
        if (c != 0.f)
            stream<TEAM, BLOCK, FIRST_OUT>(ring, vec, s.first, s.last, t, [&](const uint4 &q, int i) {
                float v[N];
                unpack(q, v);
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float2 x = __ffma2_rn(__fadd2_rn(make_float2(v[j], v[j + 1]), base2), a2, less2);
                    const float2 g = __fmul2_rn(make_float2(pow2(x.x), pow2(x.y)), c2);
                    v[j] = g.x; v[j + 1] = g.y;
                }
                store(i, v);
            });
        else {
            const float zeros[N] = {};
            for (int i = s.first + t; i < s.last; i += TEAM) store(i, zeros);
        }
        if (t < s.edges) {
            const long long e = s.edge(t);
            from_float(out + e, c != 0.f ? c * pow2((to_float(ld_act(row + e)) - base) * a - off2) : 0.f);
        }
        sync();
#pragma unroll
        for (int q = 0; q < SLOTS; q++)
            if (at[q] >= 0) from_float(out + at[q], named[q]);
    }
    if (!p.backward && part == 0) {
        loss = warp_sum(loss);
        if (TEAM > 32) {
            if ((t & 31) == 0) sums[t >> 5] = loss;
            __syncthreads();
            if (t < 32) loss = warp_sum(t < TEAM / 32 ? sums[t] : 0.f);
        }
        if (t == 0) {
            p.loss[r] = used ? loss * p.temperature : 0.f;
            if (p.stat) {
                p.stat[2 * r] = logsum == logsum || zmax == -NEG_INF ? zmax : logsum;  // (NaN in a row with a NaN)
                p.stat[2 * r + 1] = logsum;
            }
        }
    }
    if (meet) cluster_wait();
}

template <typename T, int TEAM, int BLOCK> cudaError_t launch_distill_blocks(const DisParams &p, dim3 grid, unsigned list, int rows, cudaStream_t st) {
    constexpr unsigned RING = BLOCK * STREAM_RING * 16, LISTS = (TEAM == 32 ? 8 * 128 : DISTILL_TOP_MAX) * 16;  // (a slot and its places in the table)
    static DeviceBits done;
    cudaError_t e = smem_limit_once(distill_kernel<T, TEAM, BLOCK>, RING + LISTS, done);
    if (e != cudaSuccess) return e;
    return launch_pdl(distill_kernel<T, TEAM, BLOCK>, grid, dim3(BLOCK), RING + list, st, (unsigned)p.parts, p, rows);
}
template <typename T> cudaError_t launch_distill_type(DisParams &p, int rows, double bytes, cudaStream_t st) {
    // Lists of up to 128 slots are compared with each other outright (64 of 4096 classes, 16384 rows: 69 us, 99 with the table; 1000 of
    // 1000, 64 rows: 44 us, 5.2 with it).
    p.table = 0;
    if (p.dz && p.k > 128)
        for (p.table = 2; p.table < 2 * p.k; p.table *= 2) {}
    const unsigned list = (unsigned)(p.k * 8 + p.table * 4);
    // Short rows, and many of them: a warp each (loss and gradient of 16384 x 4096 bf16: 69 us, 166 with a block a row; the loss of 16384 x 1000
    // fp32: 20.5 and 100 us).
    if (bytes <= 8192 && p.k <= 128 && rows >= 8 * sm_count()) {
        constexpr int TEAMS = 256 / 32;
        p.parts = 1;
        return launch_distill_blocks<T, 32, 256>(p, dim3((unsigned)(((long long)rows + TEAMS - 1) / TEAMS)), TEAMS * list, rows, st);
    }
    // Blocks of 256 threads keep four rows of an SM at work, which serves the loss alone; with a gradient the rows between their two
    // passes have to stay in L2 together with what is written: blocks of 512, two rows an SM (2048 x 65536 bf16: 121 and 113 us; the loss
    // alone 50 and 60 us).
    const dim3 grid((unsigned)rows, 1, (unsigned)p.parts);
    if (p.dz && bytes / p.parts > 16384) return launch_distill_blocks<T, 512, 512>(p, grid, list, rows, st);
    return launch_distill_blocks<T, 256, 256>(p, grid, list, rows, st);
}

template <typename T> cudaError_t launch_top_type(const TopParams &p, int rows, double bytes, cudaStream_t st) {
    const dim3 grid((unsigned)rows, 1, (unsigned)p.parts);
    if (bytes <= 16384 && p.k <= 64 && rows >= 2 * sm_count())  // (rows that are read element by element need no ring)
        return launch_pdl(top_logits_kernel<T, 128>, grid, dim3(128), p.V <= 2 * Vec<T>::N * 128 ? 0 : 128 * STREAM_RING * 16, st, 1, p);
    static_assert(512 * STREAM_RING * 16 >= 8 * TOP_LOGITS_MAX * 8, "the parts' words");
    static DeviceBits done;
    cudaError_t e = smem_limit_once(top_logits_kernel<T, 512>, 512 * STREAM_RING * 16, done);
    if (e != cudaSuccess) return e;
    return launch_pdl(top_logits_kernel<T, 512>, grid, dim3(512), 512 * STREAM_RING * 16, st, (unsigned)p.parts, p);
}

}  // namespace

cudaError_t launch_top_logits(const TopArgs &a, cudaStream_t st) {
    TopParams p;
    p.z = a.z; p.values = a.values; p.index = a.index; p.V = a.classes; p.k = a.top; p.ldz = a.ldz; p.ldt = a.ldt;
    const double bytes = (double)a.classes * (a.bf16 ? 2 : 4);
    // (a cluster's two meetings cost as much as 64 KB of a row: 64 x 32768 bf16 takes 6.7 us with a block a row, 9.2 with two)
    p.parts = parts_for(a.rows, bytes, 65536);
    // Many short rows: blocks of 128 threads, eight an SM (8192 x 1000 fp32: 126 us with 512 threads, 39 with 128; 64 x 1000: 4.4 and 5.5 us).
    return a.bf16 ? launch_top_type<__nv_bfloat16>(p, a.rows, bytes, st) : launch_top_type<float>(p, a.rows, bytes, st);
}

cudaError_t launch_distill(const DistillArgs &a, cudaStream_t st) {
    DisParams p;
    p.z = a.z; p.dz = a.dz; p.teacher = a.teacher; p.row_scale = a.row_scale; p.index = a.index; p.loss = a.loss; p.stat = a.stat;
    p.V = a.classes; p.k = a.top; p.backward = a.backward; p.ldz = a.ldz; p.lddz = a.lddz; p.ldt = a.ldt;
    p.inv_t = 1.f / a.temperature; p.temperature = a.temperature;
    // (a number of fp32's precision and powers of two, all of them above 1 or all below: a row's scale comes to the product without leaving the
    // range on the way; multiplied in 64 bits by every thread a row of 65536 takes 0.7 % longer)
    int e;
    p.grad_factor[0] = (float)std::frexp((double)a.grad_scale * a.temperature, &e);  // (e from -297 to 256)
    for (int i = 0; i < 3; i++) {
        const int part = std::max(-100, std::min(100, e));
        p.grad_factor[i] = std::ldexp(i ? 1.f : p.grad_factor[0], part);
        e -= part;
    }
    const double bytes = (double)a.classes * (a.bf16 ? 2 : 4);
    p.parts = parts_for(a.rows, bytes, 16384);
    return a.bf16 ? launch_distill_type<__nv_bfloat16>(p, a.rows, bytes, st) : launch_distill_type<float>(p, a.rows, bytes, st);
}

}  // namespace sgs
