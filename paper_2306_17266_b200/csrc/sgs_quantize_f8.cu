// Block quantisation to 8-bit floating point: the codes of a matrix and of its transpose, from one read of it.
//
//   scale(B) = 2^e,  e = max(-126, ceil(log2(amax(B) / FMAX)))      amax: the largest finite magnitude of block B
//   code(x)  = nearest(x / scale(B)), ties to even;  NaN and infinities become NaN
//
// B is 128 elements along the reduction (a row's, or in the transposed output a column's), or a square of 128 x 128.  FMAX is
// 448 = 1.75 * 2^8 (e4m3) or 57344 = 1.75 * 2^15 (e5m2), so e follows from the exponent and mantissa bits of amax alone, without
// a logarithm or a division, and x / scale is exact: a code is rounded once, from x itself.
//
// What bounds it: bytes.  A block of 256 threads takes a tile of 128 x 128: a thread holds 8 columns of 8 neighbouring rows, 16
// threads a row, so the largest of a row is a shuffle among 16 lanes, and the 8 codes of a column and thread are one 8-byte word
// of the transposed tile, which goes through shared memory (16 KB, units of 8 bytes swizzled by the column group: neither the
// writes nor the 16-byte reads meet in a bank) so that the transposed codes leave in rows of 128 bytes too.
// Measured (B200, 8192 x 8192, row-wise / transposed / both from one read, us): bf16 32.3 / 37.6 / 58.6 (6.3, 5.4, 4.7 TB/s), fp32 62.0 / 60.5 /
// 95.3 (5.5, 5.6, 4.3 TB/s); with blocks of 128 x 128 bf16 34.4 / 34.5 / 47.0, fp32 58.8 / 55.5 / 64.5 (6.2 TB/s).  Both sides at once are not
// held by one unit (integer pipe 59 %, DRAM 49 %, shared memory 48 %): a block has one tile, whose load, exchange of maxima, codes and
// transpose follow each other; without the columns' maxima, with blocks of 128 x 128, it is a fifth faster.
#include "sgs_internal.h"
#include "sgs_pdl.cuh"

#include <cuda_fp8.h>

namespace sgs {
namespace {

constexpr uint32_t INF_BITS = 0x7f800000u;

// Power-of-two scale of a block whose largest finite magnitude has the bits `amax`: exponent field of the scale.
__device__ __forceinline__ int scale_field(uint32_t amax, int top) {
    const int e = (int)(amax >> 23) - 127 - top + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, -126) + 127;
}
__device__ __forceinline__ float scale_of(int field) { return __uint_as_float((uint32_t)field << 23); }
__device__ __forceinline__ float inverse_of(int field) { return __uint_as_float((uint32_t)(254 - field) << 23); }

template <bool E5M2> __device__ __forceinline__ uint32_t codes2(float lo, float hi) {
    uint16_t r;
    if (E5M2) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool E5M2> __device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) { return codes2<E5M2>(a, b) | codes2<E5M2>(c, d) << 16; }

// 8 consecutive elements of a row as they lie in memory, zeros from `n` on: the tiles stay in this form in registers (half the
// registers for bf16), and the largest magnitude of two bf16 is one 16-bit SIMD maximum.
template <typename T> struct Eight;
template <> struct Eight<float> {
    uint32_t w[8];
    __device__ __forceinline__ float at(int j) const { return __uint_as_float(w[j]); }
    __device__ __forceinline__ uint32_t most() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) m = max(m, w[j] & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ void set_nan() {
#pragma unroll
        for (int j = 0; j < 8; j++) w[j] = (w[j] & 0x7fffffffu) >= INF_BITS ? 0x7fc00000u : w[j];
    }
    __device__ __forceinline__ uint32_t most_finite() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) m = max(m, (w[j] & 0x7fffffffu) >= INF_BITS ? 0u : w[j] & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ void load(const float *p, int n, bool vec) {
        if (vec && n >= 8) {
            const uint4 a = ld_act(reinterpret_cast<const uint4 *>(p)), b = ld_act(reinterpret_cast<const uint4 *>(p) + 1);
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) w[j] = j < n ? __float_as_uint(ld_act(p + j)) : 0u;
        }
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ float at(int j) const { return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16); }
    static __device__ __forceinline__ uint32_t wide(uint32_t m) { return max(m & 0xffff0000u, m << 16); }
    __device__ __forceinline__ uint32_t most() const {
        return wide(__vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu)));
    }
    __device__ __forceinline__ void set_nan() {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t odd = __vcmpgeu2(w[j] & 0x7fff7fffu, 0x7f807f80u);
            w[j] = (w[j] & ~odd) | (0x7fc07fc0u & odd);
        }
    }
    __device__ __forceinline__ uint32_t most_finite() const {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t v = w[j] & 0x7fff7fffu;
            m = __vmaxu2(m, v & ~__vcmpgeu2(v, 0x7f807f80u));
        }
        return wide(m);
    }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, int n, bool vec) {
        if (vec && n >= 8) {
            const uint4 q = ld_act(reinterpret_cast<const uint4 *>(p));
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
                w[j] = (2 * j < n ? (uint32_t)ld_act(reinterpret_cast<const unsigned short *>(p) + 2 * j) : 0u) |
                       (2 * j + 1 < n ? (uint32_t)ld_act(reinterpret_cast<const unsigned short *>(p) + 2 * j + 1) << 16 : 0u);
        }
    }
};
// The largest magnitudes of each of the 8 columns of some rows.
template <typename T> struct EightMax;
template <> struct EightMax<float> {
    uint32_t m[8] = {};
    __device__ __forceinline__ void add(const Eight<float> &e) {
#pragma unroll
        for (int j = 0; j < 8; j++) m[j] = max(m[j], e.w[j] & 0x7fffffffu);
    }
    __device__ __forceinline__ void add_finite(const Eight<float> &e) {
#pragma unroll
        for (int j = 0; j < 8; j++) m[j] = max(m[j], (e.w[j] & 0x7fffffffu) >= INF_BITS ? 0u : e.w[j] & 0x7fffffffu);
    }
    __device__ __forceinline__ uint32_t bits(int j) const { return m[j]; }
};
template <> struct EightMax<__nv_bfloat16> {
    uint32_t m[4] = {};
    __device__ __forceinline__ void add(const Eight<__nv_bfloat16> &e) {
#pragma unroll
        for (int j = 0; j < 4; j++) m[j] = __vmaxu2(m[j], e.w[j] & 0x7fff7fffu);
    }
    __device__ __forceinline__ void add_finite(const Eight<__nv_bfloat16> &e) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t v = e.w[j] & 0x7fff7fffu;
            m[j] = __vmaxu2(m[j], v & ~__vcmpgeu2(v, 0x7f807f80u));
        }
    }
    __device__ __forceinline__ uint32_t bits(int j) const { return j & 1 ? m[j >> 1] & 0xffff0000u : m[j >> 1] << 16; }
};
// `n` of the bytes of one or two words.
__device__ __forceinline__ void store_bytes(uint8_t *p, uint32_t lo, uint32_t hi, int n) {
#pragma unroll
    for (int j = 0; j < 8; j++)
        if (j < n) p[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
}

struct QuantParams {
    const void *x;
    uint8_t *q, *qt;
    float *scale, *scale_t;
    long long ldx, ldq, ldqt, lds, ldst;
    int rows, cols, col_tiles;
    int vec_x, vec_q, vec_qt;  // 16-byte (q: 8-byte) accesses allowed
};

template <typename T, bool E5M2> __device__ __forceinline__ uint2 codes8(const Eight<T> &e, float inv) {
    return make_uint2(codes4<E5M2>(e.at(0) * inv, e.at(1) * inv, e.at(2) * inv, e.at(3) * inv), codes4<E5M2>(e.at(4) * inv, e.at(5) * inv, e.at(6) * inv, e.at(7) * inv));
}
// Largest of each of R rows over the 16 threads that hold them; a thread is left with one row's, row_of(l) (16 / R threads hold the same).
// The first exchanges halve what a thread still has: R + log2(16 / R) - 1 shuffles in place of 4 R.
template <int R> __device__ __forceinline__ uint32_t rows_max(uint32_t (&m)[R], int l) {
    int o = 8;
#pragma unroll
    for (int n = R / 2; n >= 1; n /= 2, o /= 2) {
        const bool high = l & o;
#pragma unroll
        for (int i = 0; i < n; i++) {
            const uint32_t send = high ? m[i] : m[i + n], keep = high ? m[i + n] : m[i];
            m[i] = max(keep, __shfl_xor_sync(0xffffffffu, send, o));
        }
    }
    for (; o; o /= 2) m[0] = max(m[0], __shfl_xor_sync(0xffffffffu, m[0], o));
    return m[0];
}
template <int R> __device__ __forceinline__ int row_of(int l) { return l / (16 / R); }

// Row-wise codes alone, a scale per 128 elements: 16 threads take a block of each of four neighbouring rows; nothing is shared.
constexpr int QROWS = 4;
template <typename T, bool E5M2> __global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantParams p) {
    constexpr int TOP = E5M2 ? 15 : 8;
    const int t = threadIdx.x, l = t & 15, g = t >> 4;
    const int ct = (int)(blockIdx.x % (unsigned)p.col_tiles), rt = (int)(blockIdx.x / (unsigned)p.col_tiles);
    const int r0 = rt * (16 * QROWS) + QROWS * g, c0 = ct * 128 + 8 * l;
    const int n = min(8, p.cols - c0);
    pdl_launch_dependents();
    pdl_wait();
    Eight<T> v[QROWS];
#pragma unroll
    for (int i = 0; i < QROWS; i++) {
        const bool in = r0 + i < p.rows && n > 0;
        v[i].load(static_cast<const T *>(p.x) + (in ? (long long)(r0 + i) * p.ldx + c0 : 0), in ? n : 0, p.vec_x);
    }
    uint32_t m[QROWS];
#pragma unroll
    for (int i = 0; i < QROWS; i++) m[i] = v[i].most();
    uint32_t a = rows_max<QROWS>(m, l);
    if (__any_sync(0xffffffffu, a >= INF_BITS)) {  // (rare; for both half-warps, whose shuffles are one instruction)
#pragma unroll
        for (int i = 0; i < QROWS; i++) {
            m[i] = v[i].most_finite();
            v[i].set_nan();
        }
        a = rows_max<QROWS>(m, l);
    }
    const int field = scale_field(a, TOP), mine = row_of<QROWS>(l);
    if (l % (16 / QROWS) == 0 && r0 + mine < p.rows) p.scale[(long long)ct * p.lds + r0 + mine] = scale_of(field);
    const float own = inverse_of(field);
#pragma unroll
    for (int i = 0; i < QROWS; i++) {
        const uint2 q = codes8<T, E5M2>(v[i], __shfl_sync(0xffffffffu, own, (t & 16) + i * (16 / QROWS)));
        if (r0 + i < p.rows && n > 0) {
            uint8_t *dst = p.q + (long long)(r0 + i) * p.ldq + c0;
            if (p.vec_q && n == 8) *reinterpret_cast<uint2 *>(dst) = q;
            else store_bytes(dst, q.x, q.y, n);
        }
    }
}

template <typename T, bool E5M2, bool SQUARE, bool ROWS, bool TRANSPOSED>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 2) quantize_f8_kernel(const QuantParams p) {
    __shared__ __align__(16) uint8_t tile[TRANSPOSED ? 128 * 128 : 16];
    __shared__ uint32_t col_max[TRANSPOSED && !SQUARE ? 16 : 1][128];
    __shared__ uint32_t warp_max[8];
    constexpr int TOP = E5M2 ? 15 : 8;
    const int t = threadIdx.x, l = t & 15, g = t >> 4;  // columns 8 l .., rows 8 g ..
    const int ct = (int)(blockIdx.x % (unsigned)p.col_tiles), rt = (int)(blockIdx.x / (unsigned)p.col_tiles);
    const int r0 = rt * 128 + 8 * g, c0 = ct * 128 + 8 * l;
    const int n = min(8, p.cols - c0);  // (may be negative)
    pdl_launch_dependents();
    pdl_wait();
    Eight<T> v[8];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const bool in = r0 + i < p.rows && n > 0;
        v[i].load(static_cast<const T *>(p.x) + (in ? (long long)(r0 + i) * p.ldx + c0 : 0), in ? n : 0, p.vec_x);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) most = max(most, v[i].most());
    // A tile with a NaN or an infinity (rare): they become NaN, and the scales are those of the other elements.
    const bool odd = __syncthreads_or(most >= INF_BITS);
    if (odd) {
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            most = max(most, v[i].most_finite());
            v[i].set_nan();
        }
    }
    int square = 0;
    if (SQUARE) {
        most = __reduce_max_sync(0xffffffffu, most);
        if ((t & 31) == 0) warp_max[t >> 5] = most;
        __syncthreads();
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) most = max(most, warp_max[i]);
        square = scale_field(most, TOP);
        if (t == 0) {
            if (ROWS) p.scale[(long long)ct * p.lds + rt] = scale_of(square);
            if (TRANSPOSED) p.scale_t[(long long)rt * p.ldst + ct] = scale_of(square);
        }
    }
    if (TRANSPOSED && !SQUARE) {
        EightMax<T> cm;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (odd) cm.add_finite(v[i]);
            else cm.add(v[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; j += 4)
            *reinterpret_cast<uint4 *>(&col_max[g][8 * l + j]) = make_uint4(cm.bits(j), cm.bits(j + 1), cm.bits(j + 2), cm.bits(j + 3));
        __syncthreads();
        if (t < 128) {
            uint32_t a = 0;
#pragma unroll
            for (int i = 0; i < 16; i++) a = max(a, col_max[i][t]);
            const int field = scale_field(a, TOP);
            if (ct * 128 + t < p.cols) p.scale_t[(long long)rt * p.ldst + ct * 128 + t] = scale_of(field);
            col_max[0][t] = (uint32_t)(254 - field) << 23;
        }
    }
    if (ROWS) {
        float own = inverse_of(square);
        if (!SQUARE) {
            uint32_t m[8];
#pragma unroll
            for (int i = 0; i < 8; i++) m[i] = odd ? v[i].most_finite() : v[i].most();
            const int field = scale_field(rows_max<8>(m, l), TOP), mine = row_of<8>(l);
            if (l % 2 == 0 && r0 + mine < p.rows) p.scale[(long long)ct * p.lds + r0 + mine] = scale_of(field);
            own = inverse_of(field);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint2 q = codes8<T, E5M2>(v[i], SQUARE ? own : __shfl_sync(0xffffffffu, own, (t & 16) + 2 * i));
            if (r0 + i < p.rows && n > 0) {
                uint8_t *dst = p.q + (long long)(r0 + i) * p.ldq + c0;
                if (p.vec_q && n == 8) *reinterpret_cast<uint2 *>(dst) = q;
                else store_bytes(dst, q.x, q.y, n);
            }
        }
    }
    if (TRANSPOSED) {
        if (!SQUARE) __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float inv = SQUARE ? inverse_of(square) : __uint_as_float(col_max[0][8 * l + j]);
            const uint32_t lo = codes4<E5M2>(v[0].at(j) * inv, v[1].at(j) * inv, v[2].at(j) * inv, v[3].at(j) * inv);
            const uint32_t hi = codes4<E5M2>(v[4].at(j) * inv, v[5].at(j) * inv, v[6].at(j) * inv, v[7].at(j) * inv);
            *reinterpret_cast<uint2 *>(tile + (8 * l + j) * 128 + ((g ^ l) * 8)) = make_uint2(lo, hi);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int c = (t >> 3) + 32 * i, k = t & 7, s = c >> 3;  // column, 16-byte piece, its swizzle
            const uint4 w = *reinterpret_cast<const uint4 *>(tile + c * 128 + (((2 * k) ^ s) & ~1) * 8);
            const uint4 u = s & 1 ? make_uint4(w.z, w.w, w.x, w.y) : w;
            const int row = rt * 128 + 16 * k, m = min(16, p.rows - row);
            if (ct * 128 + c < p.cols && m > 0) {
                uint8_t *dst = p.qt + (long long)(ct * 128 + c) * p.ldqt + row;
                if (p.vec_qt && m == 16) *reinterpret_cast<uint4 *>(dst) = u;
                else { store_bytes(dst, u.x, u.y, m); store_bytes(dst + 8, u.z, u.w, m - 8); }
            }
        }
    }
}

template <typename T, bool E5M2, bool SQUARE> cudaError_t launch_sides(const QuantParams &p, unsigned blocks, cudaStream_t st) {
    if (p.q && p.qt) return launch_pdl(quantize_f8_kernel<T, E5M2, SQUARE, true, true>, dim3(blocks), dim3(256), 0, st, 1, p);
    if (p.q) {
        if constexpr (SQUARE) return launch_pdl(quantize_f8_kernel<T, E5M2, true, true, false>, dim3(blocks), dim3(256), 0, st, 1, p);
        else return launch_pdl(quantize_rows_kernel<T, E5M2>, dim3((unsigned)((long long)p.col_tiles * ((p.rows + 16 * QROWS - 1) / (16 * QROWS)))), dim3(256), 0, st, 1, p);
    }
    return launch_pdl(quantize_f8_kernel<T, E5M2, SQUARE, false, true>, dim3(blocks), dim3(256), 0, st, 1, p);
}
template <typename T> cudaError_t launch_type(const QuantParams &p, int e5m2, int square, unsigned blocks, cudaStream_t st) {
    if (e5m2) return square ? launch_sides<T, true, true>(p, blocks, st) : launch_sides<T, true, false>(p, blocks, st);
    return square ? launch_sides<T, false, true>(p, blocks, st) : launch_sides<T, false, false>(p, blocks, st);
}

}  // namespace

cudaError_t launch_quantize_f8(const QuantF8Args &a, cudaStream_t st) {
    QuantParams p;
    p.x = a.x; p.q = static_cast<uint8_t *>(a.q); p.qt = static_cast<uint8_t *>(a.qt); p.scale = a.scale; p.scale_t = a.scale_t;
    p.ldx = a.ldx; p.ldq = a.ldq; p.ldqt = a.ldqt; p.lds = a.lds; p.ldst = a.ldst;
    p.rows = a.rows; p.cols = a.cols; p.col_tiles = (a.cols + 127) / 128;
    const size_t eb = a.bf16 ? 2 : 4;
    p.vec_x = ((reinterpret_cast<uintptr_t>(a.x) | (size_t)a.ldx * eb) & 15) == 0;
    p.vec_q = ((reinterpret_cast<uintptr_t>(a.q) | (size_t)a.ldq) & 7) == 0;
    p.vec_qt = ((reinterpret_cast<uintptr_t>(a.qt) | (size_t)a.ldqt) & 15) == 0;
    const unsigned blocks = (unsigned)((long long)p.col_tiles * ((a.rows + 127) / 128));
    return a.bf16 ? launch_type<__nv_bfloat16>(p, a.e5m2, a.square, blocks, st) : launch_type<float>(p, a.e5m2, a.square, blocks, st);
}

}  // namespace sgs
