// 8-bit values with a power-of-two scale per block of 128: x ~ q * 2^e, q in e4m3, e the least with
// max |x| <= 448 * 2^e over the block.  A power of two costs e4m3 no precision (its steps are relative) and leaves one rounding,
// that of q: what x / 2^e loses in fp32 lies far below q's smallest step, and q * 2^e is exact (in bf16 from 2^-124 on).
//
// A block of 256 threads takes a tile of 128 x 128 elements into registers, 8 rows by 8 columns per thread, so that one
// read serves both layouts: maxima along the rows need 16 lanes, along the columns the block; values along the rows leave
// directly, eight bytes per thread; the transposed ones are turned in 16 KB of shared memory, whose 8-byte units are
// XORed with the column's group so that neither the writes nor the reads meet a bank conflict.
// 2 bytes read and 1 or 2 written per bf16 element: HBM is the bound.
#include "dense_common.cuh"

namespace tppo {
namespace {

constexpr int kQTile = 128, kQThreads = 256;

struct QuantArgs {
    const void* x; int64_t ldx, M, K;
    uint8_t* q; int64_t ldq; float* scale; int64_t lds;
    uint8_t* qt; int64_t ldqt; float* scale_t; int64_t ldst;
    int32_t* status;
    int64_t k_tiles;
    int32_t vec;              // rows of x start on 16-byte boundaries
};

// Exponent of the scale of a block whose largest magnitude is `top` (448 = 1.75 * 2^8).
__device__ __forceinline__ int scale_exponent(float top) {
    const uint32_t b = __float_as_uint(top);
    const int e = int(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return top == 0.f ? 0 : e < -126 ? -126 : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(uint32_t(127 + e) << 23); }

// Two values as e4m3, lo in the low byte.
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// A thread's 8 x 8 elements as loaded (32 registers of bf16, 64 of fp32), magnitudes as bit patterns, which order
// like the numbers: their maxima take one packed instruction per two bf16 elements, and a NaN or infinity shows in them.
// N words that start `offset` bytes (a multiple of 2) into a 16-byte piece, from the pieces they touch.
template <int N>
__device__ __forceinline__ void quant_align(const uint32_t (&in)[N + 4], int offset, uint32_t* out) {
    uint32_t a[N + 2], b[N + 1];
#pragma unroll
    for (int i = 0; i < N + 2; ++i) a[i] = offset & 8 ? in[i + 2] : in[i];
#pragma unroll
    for (int i = 0; i < N + 1; ++i) b[i] = offset & 4 ? a[i + 1] : a[i];
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = __funnelshift_r(b[i], b[i + 1], (offset & 2) * 8);
}
// Eight elements at p, of which the first `cols` belong to the row (0 for the others), from whole 16-byte pieces: a piece
// with one of them in it is mapped, whatever else it holds.
template <class T>
__device__ __forceinline__ void quant_read(const T* p, int cols, uint32_t* out) {
    constexpr int N = 8 * sizeof(T) / 4;
    const int offset = int(reinterpret_cast<uintptr_t>(p) & 15), bytes = cols < 8 ? cols * int(sizeof(T)) : 4 * N;
    const uint4* g = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) - offset);
    uint32_t in[N + 4];
#pragma unroll
    for (int i = 0; i < N / 4 + 1; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (bytes > 0 && 16 * i < offset + bytes) v = g[i];
        in[4 * i] = v.x; in[4 * i + 1] = v.y; in[4 * i + 2] = v.z; in[4 * i + 3] = v.w;
    }
    quant_align<N>(in, offset, out);
    if (cols < 8) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int left = bytes - 4 * i;               // bytes of word i that count
            out[i] = left >= 4 ? out[i] : left == 2 ? out[i] & 0xffffu : 0u;
        }
    }
}
template <class T> struct QuantTile;
template <> struct QuantTile<bf16_bits> {
    uint32_t w[8][4];
    static constexpr uint32_t kInfinity = 0x7f80;
    __device__ __forceinline__ void load(int i, const bf16_bits* p, int cols, bool vec) {
        if (cols >= 8 && vec) {
            const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
            w[i][0] = v.x; w[i][1] = v.y; w[i][2] = v.z; w[i][3] = v.w;
        } else {
            quant_read(p, cols, w[i]);
        }
    }
    __device__ __forceinline__ float get(int i, int j) const { return j % 2 ? bf16_hi(w[i][j / 2]) : bf16_lo(w[i][j / 2]); }
    __device__ __forceinline__ void clear_bad() {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if ((w[i][j] & 0x7f80u) == 0x7f80u) w[i][j] &= 0xffff0000u;
                if ((w[i][j] & 0x7f800000u) == 0x7f800000u) w[i][j] &= 0xffffu;
            }
    }
    // Largest magnitudes of the columns, and of the thread.
    __device__ __forceinline__ uint32_t columns(uint32_t (&top)[8]) const {
        uint32_t all = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i][j] & 0x7fff7fffu);
            top[2 * j] = m & 0xffffu;
            top[2 * j + 1] = m >> 16;
            all = __vmaxu2(all, m);
        }
        return max(all & 0xffffu, all >> 16);
    }
    // ... of the rows, over the 16 lanes that share them
    __device__ __forceinline__ void rows(uint32_t (&top)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t m[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                m[k] = __vmaxu2(__vmaxu2(w[i + k][0] & 0x7fff7fffu, w[i + k][1] & 0x7fff7fffu),
                                __vmaxu2(w[i + k][2] & 0x7fff7fffu, w[i + k][3] & 0x7fff7fffu));
                m[k] = __vmaxu2(m[k], m[k] >> 16);
            }
            uint32_t both = (m[0] & 0xffffu) | m[1] << 16;
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, o));
            top[i] = both & 0xffffu;
            top[i + 1] = both >> 16;
        }
    }
    static __device__ __forceinline__ float magnitude(uint32_t bits) { return __uint_as_float(bits << 16); }
};
template <> struct QuantTile<float> {
    float v[8][8];
    static constexpr uint32_t kInfinity = 0x7f800000;
    __device__ __forceinline__ void load(int i, const float* p, int cols, bool vec) {
        if (cols >= 8 && vec) {
            load_vec<8>(p, v[i]);
        } else {
            uint32_t w[8];
            quant_read(p, cols, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = __uint_as_float(w[j]);
        }
    }
    __device__ __forceinline__ float get(int i, int j) const { return v[i][j]; }
    __device__ __forceinline__ void clear_bad() {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!is_finite(v[i][j])) v[i][j] = 0;
    }
    __device__ __forceinline__ uint32_t bits(int i, int j) const { return __float_as_uint(v[i][j]) & 0x7fffffffu; }
    __device__ __forceinline__ uint32_t columns(uint32_t (&top)[8]) const {
        uint32_t all = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top[j] = max(top[j], bits(i, j));
            all = max(all, top[j]);
        }
        return all;
    }
    __device__ __forceinline__ void rows(uint32_t (&top)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            top[i] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top[i] = max(top[i], bits(i, j));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
        }
    }
    static __device__ __forceinline__ float magnitude(uint32_t bits) { return __uint_as_float(bits); }
};

template <class T, bool SQUARE>
__global__ void __launch_bounds__(kQThreads, sizeof(T) == 2 ? 4 : 2) fp8_quantize_kernel(const QuantArgs a) {
    __shared__ __align__(16) uint8_t turned[kQTile * kQTile];
    __shared__ __align__(16) uint32_t tops[8][kQTile];
    __shared__ __align__(16) float inverse[kQTile];
    pdl_launch();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, piece = lane & 15;
    const int64_t mb = blockIdx.x / a.k_tiles, kb = blockIdx.x % a.k_tiles;
    const int64_t r0 = mb * kQTile + warp * 16 + half * 8, c0 = kb * kQTile + piece * 8;
    const int rows = int(a.M - r0 < 8 ? a.M - r0 : 8), cols = int(a.K - c0 < 8 ? a.K - c0 : 8);      // may be negative
    QuantTile<T> x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.load(i, static_cast<const T*>(a.x) + (r0 + i) * a.ldx + c0, i < rows ? cols : 0, a.vec);
    uint32_t top[8];
    uint32_t most = x.columns(top);
    if (most >= QuantTile<T>::kInfinity) {
        x.clear_bad();
        most = x.columns(top);
        if (a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    }
    // column maxima over the block: only what is transposed needs them
    const bool columns = !SQUARE && a.qt;
    if (columns) {
#pragma unroll
        for (int j = 0; j < 8; ++j) top[j] = max(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16));
        if (half == 0) {
            *reinterpret_cast<uint4*>(&tops[warp][piece * 8]) = make_uint4(top[0], top[1], top[2], top[3]);
            *reinterpret_cast<uint4*>(&tops[warp][piece * 8 + 4]) = make_uint4(top[4], top[5], top[6], top[7]);
        }
    }
    int e_tile = 0;
    if (SQUARE) {
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) tops[warp][0] = most;
        __syncthreads();
        for (int w = 0; w < 8; ++w) most = max(most, tops[w][0]);
        e_tile = scale_exponent(QuantTile<T>::magnitude(most));
        if (threadIdx.x == 0) {
            if (a.q) a.scale[mb * a.lds + kb] = power_of_two(e_tile);
            if (a.qt) a.scale_t[kb * a.ldst + mb] = power_of_two(e_tile);
        }
    } else if (columns) {
        __syncthreads();
        if (threadIdx.x < kQTile) {
            uint32_t t = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) t = max(t, tops[w][threadIdx.x]);
            const int e = scale_exponent(QuantTile<T>::magnitude(t));
            inverse[threadIdx.x] = power_of_two(-e);
            const int64_t c = kb * kQTile + threadIdx.x;
            if (c < a.K) a.scale_t[mb * a.ldst + c] = power_of_two(e);
        }
    }
    if (a.q) {
        if (!SQUARE) x.rows(top);
        float mine = 0;                                   // lane `piece` of the half keeps the scale of row `piece`
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = SQUARE ? e_tile : scale_exponent(QuantTile<T>::magnitude(top[i]));
            if (piece == i) mine = power_of_two(e);
            const float inv = power_of_two(-e);
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_e4m3x2(x.get(i, 2 * j) * inv, x.get(i, 2 * j + 1) * inv);
            if (i < rows && cols > 0) {
                uint8_t* p = a.q + (r0 + i) * a.ldq + c0;
                if (cols == 8) {
                    *reinterpret_cast<uint2*>(p) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < cols) p[j] = uint8_t(w[j / 2] >> (j % 2 * 8));
                }
            }
        }
        if (!SQUARE && piece < rows) a.scale[kb * a.lds + r0 + piece] = mine;
    }
    if (!a.qt) return;
    if (columns) __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float inv = SQUARE ? power_of_two(-e_tile) : inverse[piece * 8 + j];
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_e4m3x2(x.get(2 * i, j) * inv, x.get(2 * i + 1, j) * inv);
        const int unit = (warp * 2 + half) ^ piece;
        *reinterpret_cast<uint2*>(turned + (piece * 8 + j) * kQTile + unit * 8) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
    __syncthreads();
    // 16 bytes of a column: two units, exchanged where the column's group is odd
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int col = it * 32 + int(threadIdx.x >> 3), pair = threadIdx.x & 7, g = col >> 3;
        uint4 w = *reinterpret_cast<const uint4*>(turned + col * kQTile + (pair ^ (g >> 1)) * 16);
        if (g & 1) w = make_uint4(w.z, w.w, w.x, w.y);
        const int64_t c = kb * kQTile + col, m = mb * kQTile + pair * 16;
        if (c >= a.K || m >= a.M) continue;
        uint8_t* p = a.qt + c * a.ldqt + m;
        if (m + 16 <= a.M) {
            *reinterpret_cast<uint4*>(p) = w;
        } else {
            const uint32_t part[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (m + i < a.M) p[i] = uint8_t(part[i / 4] >> (i % 4 * 8));
        }
    }
}

}  // namespace
}  // namespace tppo

TPPO_API int tppo_fp8_quantize(const void* x, int32_t dtype, int64_t ldx, int64_t M, int64_t K, int32_t block, void* q, int64_t ldq,
                               float* scale, int64_t lds, void* qt, int64_t ldqt, float* scale_t, int64_t ldst, int32_t* status,
                               void* stream) {
    using namespace tppo;
    if (M < 0 || K < 0 || (dtype != TPPO_BF16 && dtype != TPPO_F32) || (block != TPPO_FP8_ROWS && block != TPPO_FP8_SQUARE))
        return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || K > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    if (!aligned(status, 4)) return TPPO_ERR_INVALID_ARG;
    if (M == 0 || K == 0) return TPPO_OK;
    const int64_t mb = (M + kQTile - 1) / kQTile, kb = (K + kQTile - 1) / kQTile;
    const bool rows = block == TPPO_FP8_ROWS;
    if (!x || ldx < K || !aligned(x, dtype == TPPO_F32 ? 4 : 2) || (q == nullptr) != (scale == nullptr) || (qt == nullptr) != (scale_t == nullptr))
        return TPPO_ERR_INVALID_ARG;
    // rows of one element's height need no stride
    if (q && (!aligned(q, 16) || ldq < K || (M > 1 && ldq % 16) || !aligned(scale, 4) || lds < (rows ? M : kb)))
        return TPPO_ERR_INVALID_ARG;
    if (qt && (!aligned(qt, 16) || ldqt < M || (K > 1 && ldqt % 16) || !aligned(scale_t, 4) || ldst < (rows ? K : mb)))
        return TPPO_ERR_INVALID_ARG;
    if (mb * kb > 0x7fffffff) return TPPO_ERR_UNSUPPORTED;
    if (!q && !qt) return TPPO_OK;
    QuantArgs a{x, ldx, M, K, static_cast<uint8_t*>(q), ldq, scale, lds, static_cast<uint8_t*>(qt), ldqt, scale_t, ldst, status, kb,
                rows_aligned(x, ldx, dtype == TPPO_F32 ? 4 : 2)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid(unsigned(mb * kb)), threads(kQThreads);
    if (dtype == TPPO_F32) {
        TPPO_CUDA_CHECK(rows ? launch_dense(fp8_quantize_kernel<float, false>, grid, threads, 0, s, a)
                             : launch_dense(fp8_quantize_kernel<float, true>, grid, threads, 0, s, a));
    } else {
        TPPO_CUDA_CHECK(rows ? launch_dense(fp8_quantize_kernel<bf16_bits, false>, grid, threads, 0, s, a)
                             : launch_dense(fp8_quantize_kernel<bf16_bits, true>, grid, threads, 0, s, a));
    }
    return TPPO_OK;
}
