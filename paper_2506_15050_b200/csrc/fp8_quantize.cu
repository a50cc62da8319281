// 8-bit values with a power-of-two scale per block of 128: x ~ q * 2^e, q in e4m3, e the least with
// max |x| <= 448 * 2^e over the block.  A power of two costs e4m3 no precision (its steps are relative), makes x / 2^e and
// q * 2^e exact, and leaves one rounding, that of q.
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

template <class T, bool SQUARE>
__global__ void __launch_bounds__(kQThreads) fp8_quantize_kernel(const QuantArgs a) {
    __shared__ __align__(16) uint8_t turned[kQTile * kQTile];
    __shared__ float tops[8][kQTile];
    __shared__ __align__(16) float inverse[kQTile];
    pdl_launch();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = lane >> 4, piece = lane & 15;
    const int64_t mb = blockIdx.x / a.k_tiles, kb = blockIdx.x % a.k_tiles;
    const int64_t r0 = mb * kQTile + warp * 16 + half * 8, c0 = kb * kQTile + piece * 8;
    const int rows = int(a.M - r0 < 8 ? a.M - r0 : 8), cols = int(a.K - c0 < 8 ? a.K - c0 : 8);      // may be negative
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const T* p = static_cast<const T*>(a.x) + (r0 + i) * a.ldx + c0;
        if (i < rows && cols == 8 && a.vec) {
            load_vec<8>(p, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = i < rows && j < cols ? load_f32(p + j) : 0.f;
        }
    }
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!is_finite(v[i][j])) { v[i][j] = 0; bad = true; }
    if (bad && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);

    int e_tile = 0;
    if (SQUARE) {
        float top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[i][j]));
        top = warp_max(top);
        if (lane == 0) tops[warp][0] = top;
        __syncthreads();
        for (int w = 0; w < 8; ++w) top = fmaxf(top, tops[w][0]);
        e_tile = scale_exponent(top);
        if (threadIdx.x == 0) {
            if (a.q) a.scale[mb * a.lds + kb] = power_of_two(e_tile);
            if (a.qt) a.scale_t[kb * a.ldst + mb] = power_of_two(e_tile);
        }
    }
    if (a.q) {
        float mine = 0;                                   // lane `piece` of the half keeps the scale of row `piece`
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int e = e_tile;
            if (!SQUARE) {
                float top = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[i][j]));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                e = scale_exponent(top);
                if (piece == i) mine = power_of_two(e);
            }
            const float inv = power_of_two(-e);
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack_e4m3x2(v[i][2 * j] * inv, v[i][2 * j + 1] * inv);
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
    if (!SQUARE) {
        float top[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top[j] = fmaxf(top[j], fabsf(v[i][j]));
            top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16));
        }
        if (half == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) tops[warp][piece * 8 + j] = top[j];
        }
        __syncthreads();
        if (threadIdx.x < kQTile) {
            float t = 0;
            for (int w = 0; w < 8; ++w) t = fmaxf(t, tops[w][threadIdx.x]);
            const int e = scale_exponent(t);
            inverse[threadIdx.x] = power_of_two(-e);
            const int64_t c = kb * kQTile + threadIdx.x;
            if (c < a.K) a.scale_t[mb * a.ldst + c] = power_of_two(e);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float inv = SQUARE ? power_of_two(-e_tile) : inverse[piece * 8 + j];
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_e4m3x2(v[2 * i][j] * inv, v[2 * i + 1][j] * inv);
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
