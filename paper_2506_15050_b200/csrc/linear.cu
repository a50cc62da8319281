// Matrix product with bias, activation and residual in its epilogue, and its backward pass:
//     z = x W + bias,   y = act(z) + residual
//     dz = dy * act'(z),   dx = dz W^T,   dweight = x^T dz,   dbias = sum over rows of dz
// x [M, K], W [K, N] (the LM-head weight's layout) and the kept pre-activation z are bf16; products
// are accumulated in fp32 on the tensor cores and everything up to the one rounding of y is fp32.
//
// dz is the one intermediate that is rounded: both gradients contract it on the tensor cores, so it
// is formed once, in bf16 like the operand it meets, by a kernel that also sums dbias from the
// unrounded values.  (The error of dx and dweight against 64 bits goes from 1.7e-3, their own rounding, to
// 2.3e-3; carrying dz in two bf16 parts would double the products.  The narrow backward kernel keeps fp32.
// Without an activation and with an aligned bf16 dy that kernel writes nothing and dy itself is the operand.)
//
// Large outputs are tensor bound and take the persistent kernel; a handful of columns is no work for tensor
// cores and takes the narrow kernels, both ways; few rows, or few columns, are bound
// by reading the weight (or x) once and take the split kernel, which spreads the contraction over a
// cluster -- see dense_gemm.cuh.  TMA wants 16-byte aligned rows: operands whose row length or base
// does not allow that are first copied into the workspace with a padded row stride.
//   16384 x 5120 x 5120: the bare product 600 us (1430 TFLOP/s, the sustained cuBLAS rate: power bound), with
//   bias, gelu_tanh, residual and a kept z 750-810 us; backward 1490-1550 us, of which dz 109 (one call behind the
//   other, SM clock at the power cap).
//   1 x 5120 x 5120: 12.8 us a call, replayed 12.2 with weights that come from HBM (4.3 TB/s with the launch's start
//   and end) and 8.7 with one that stays in L2.
#include "dense_gemm.cuh"

namespace tppo {
namespace {

// Activations and slopes in a dozen instructions each: the backward pass evaluates one slope per six
// bytes it moves, and with the library's expf, erff and division it is bound by them (247 us for
// 16384 x 5120 elements where 77 us of traffic is the floor).  ex2 and the reciprocal are the hardware's
// approximations (2^-22 resp. 1 ulp); forming exp(t) as 2^(t log2 e) adds |t| 2^-24.
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / (1 + exp(-t)): 0 and 1 far out, where ex2 overflows or vanishes.
__device__ __forceinline__ float sigmoid(float t) { return rcp(1.f + ex2(-kLog2e * t)); }
// Phi(z) and the density e = exp(-z^2 / 2).  With t = 1 / (1 + 0.304 |z|) the quotient Phi(-|z|) / (e t) is
// smooth and stays between 0.12 and 0.5 from t = 1 down to t = 0, so a polynomial in t holds the lower tail
// relative to itself: degree 7, fitted here by weighted least squares to the least maximum, 8.6e-8 up to
// |z| = 13.2, where e leaves fp32's normal range.  (Five coefficients bounded only absolutely, at 1.5e-7, left
// gelu 1e-2 of itself off at z = -8.)  In fp32 the polynomial is within 6 roundings, e within 1.5 z^2 + 4.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    e = ex2(-0.5f * kLog2e * z * z);
    const float t = rcp(fmaf(0.304f, fabsf(z), 1.f));
    float q = fmaf(t, 0.03682147f, -0.155148894f);
    q = fmaf(t, q, 0.191937312f);
    q = fmaf(t, q, -0.0429043546f);
    q = fmaf(t, q, 0.123437144f);
    q = fmaf(t, q, 0.102457002f);
    q = fmaf(t, q, 0.122165337f);
    q = fmaf(t, q, 0.12123502f);
    const float tail = t * q * e;
    return z < 0.f ? tail : 1.f - tail;
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == TPPO_ACT_RELU) return fmaxf(z, 0.f);
    if constexpr (ACT == TPPO_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    if constexpr (ACT == TPPO_ACT_GELU_TANH)          // 0.5 (1 + tanh u) = sigmoid(2u)
        return z * sigmoid(z * fmaf(1.59576912160573071f * 0.044715f, z * z, 1.59576912160573071f));
    if constexpr (ACT == TPPO_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == TPPO_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    // the slopes below have reached 0 and 1 at |z| = 100; powers of a larger z would overflow
    z = fminf(fmaxf(z, -100.f), 100.f);
    if constexpr (ACT == TPPO_ACT_GELU) {
        float e;
        const float phi = normal_cdf(z, e);
        return fmaf(z * 0.39894228040143268f, e, phi);
    }
    if constexpr (ACT == TPPO_ACT_GELU_TANH) {
        constexpr float k = 1.59576912160573071f;
        const float z2 = z * z, p = sigmoid(z * fmaf(k * 0.044715f, z2, k));
        return fmaf(z * fmaf(-p, p, p), fmaf(k * 3.f * 0.044715f, z2, k), p);
    }
    if constexpr (ACT == TPPO_ACT_SILU) {
        const float p = sigmoid(z);
        return fmaf(z, fmaf(-p, p, p), p);
    }
    return 1.f;
}
template <int ACT>
__device__ __forceinline__ void act_values(const float (&z)[8], float (&o)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = act_value<ACT>(z[i]);
}
template <int ACT>
__device__ __forceinline__ void act_slopes(const float (&z)[8], float (&o)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = act_slope<ACT>(z[i]);
}
// One (uniform) branch per eight elements: inside the loop it would cost more than the arithmetic, and
// the eight chains of arithmetic would not overlap.
__device__ __forceinline__ void act_values(int act, const float (&z)[8], float (&o)[8]) {
    switch (act) {
        case TPPO_ACT_RELU: act_values<TPPO_ACT_RELU>(z, o); break;
        case TPPO_ACT_GELU: act_values<TPPO_ACT_GELU>(z, o); break;
        case TPPO_ACT_GELU_TANH: act_values<TPPO_ACT_GELU_TANH>(z, o); break;
        case TPPO_ACT_SILU: act_values<TPPO_ACT_SILU>(z, o); break;
        default: act_values<TPPO_ACT_NONE>(z, o);
    }
}
__device__ __forceinline__ void act_slopes(int act, const float (&z)[8], float (&o)[8]) {
    switch (act) {
        case TPPO_ACT_RELU: act_slopes<TPPO_ACT_RELU>(z, o); break;
        case TPPO_ACT_GELU: act_slopes<TPPO_ACT_GELU>(z, o); break;
        case TPPO_ACT_GELU_TANH: act_slopes<TPPO_ACT_GELU_TANH>(z, o); break;
        case TPPO_ACT_SILU: act_slopes<TPPO_ACT_SILU>(z, o); break;
        default: act_slopes<TPPO_ACT_NONE>(z, o);
    }
}

// `count` (1..8) elements from v; one 16-byte store where the row allows it.
__device__ __forceinline__ void put8(bf16_bits* p, const float (&v)[8], int count, bool vec) {
    if (vec && count == 8) { store_vec<8>(p, v); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) store_f32(p + i, v[i]);
}
__device__ __forceinline__ void put8(float* p, const float (&v)[8], int count, bool vec) {
    if (vec && count == 8) { store_vec<8>(p, v); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = v[i];
}
template <class T>
__device__ __forceinline__ void get8(const T* p, float (&v)[8], int count, bool vec) {
    if (vec && count == 8) { load_vec<8>(p, v); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < count ? load_f32(p + i) : 0.f;
}

__device__ __forceinline__ void widen8(const uint4& w, float (&v)[8]) {
    v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}

// Whether all eight are finite and at most `top`: the largest magnitude as bits, where a NaN is larger than
// everything -- a tree of three levels instead of eight comparisons that wait for one another.
__device__ __forceinline__ bool all_within(const float (&v)[8], float top) {
    uint32_t m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) m[i] = __float_as_uint(v[i]) & 0x7fffffffu;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < o; ++i) m[i] = max(m[i], m[i + o]);
    return m[0] <= __float_as_uint(top);
}

// Forward epilogue.
struct EpiLinear {
    const void* bias; int32_t bias_f32;
    const bf16_bits* residual; int64_t ldr;
    void* y; int64_t ldy; int32_t y_f32;
    bf16_bits* pre; int64_t ldp;
    int64_t M; int32_t N; int32_t act;
    int32_t vec_y, vec_r, vec_p, vec_b;
    int32_t* status;

    static constexpr bool kRows = true;
    struct Loads { uint4 r; };                    // the residual, where one 16-byte load fetches it

    __device__ __forceinline__ bool outside(int64_t m, int n) const { return m >= M || n >= N; }
    __device__ __forceinline__ bool fast(int64_t m, int n) const { return residual && vec_r && m < M && n + 8 <= N; }
    __device__ __forceinline__ void load(int64_t m, int n, Loads& l) const {
        if (fast(m, n)) l.r = *reinterpret_cast<const uint4*>(residual + m * ldr + n);
    }
    __device__ __forceinline__ bool by_rows() const { return !vec_y; }
    __device__ __forceinline__ void put(int64_t m, int n, float v) const {
        if (outside(m, n)) return;
        if (y_f32) static_cast<float*>(y)[m * ldy + n] = v;
        else store_f32(static_cast<bf16_bits*>(y) + m * ldy + n, v);
    }
    // What a lane's eight columns share down the rows.
    struct Cursor { float b[8]; const bf16_bits* r; bf16_bits* pre; char* y; int rows, count; };
    __device__ __forceinline__ void open(Cursor& c, int64_t m, int n) const {
        c.count = min(8, N - n);
        c.rows = c.count > 0 && m < M ? int(min(M - m, int64_t(64))) : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) c.b[i] = 0.f;
        if (c.rows == 0) return;
        if (bias) {
            if (bias_f32) get8(static_cast<const float*>(bias) + n, c.b, c.count, vec_b);
            else get8(static_cast<const bf16_bits*>(bias) + n, c.b, c.count, vec_b);
        }
        c.r = residual + m * ldr + n;
        c.pre = pre + m * ldp + n;
        c.y = static_cast<char*>(y) + (m * ldy + n) * (y_f32 ? 4 : 2);
    }
    __device__ __forceinline__ void fetch(const Cursor& c, int it, Loads& l) const {
        if (residual && vec_r && it * 8 < c.rows && c.count == 8) l.r = *reinterpret_cast<const uint4*>(c.r + it * 8 * ldr);
    }
    // v: the sums in, y out; stores the pre-activation, and y with STORE
    template <bool STORE>
    __device__ __forceinline__ void finish(const Cursor& c, int it, float (&v)[8], const Loads& l) const {
        if (it * 8 >= c.rows) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += c.b[i];
        float o[8];
        act_values(act, v, o);
        if (residual) {
            float r[8];
            if (vec_r && c.count == 8) widen8(l.r, r);
            else get8(c.r + it * 8 * ldr, r, c.count, false);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] += r[i];
        }
        // z and y that are not finite, or leave the range of the type they are stored in, are written 0
        // (without a stored z only relu hides a z that is not finite)
        const float top = y_f32 ? kFltMax : kBf16Max, ztop = pre ? kBf16Max : kFltMax;
        bool fine = all_within(o, top);
        if (pre || act == TPPO_ACT_RELU) fine = fine && all_within(v, ztop);
        if (!fine) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool zok = fabsf(v[i]) <= ztop, ok = zok && fabsf(o[i]) <= top;
                if (!zok) v[i] = 0.f;
                if (!ok) o[i] = 0.f;
                bad |= !ok && i < c.count;
            }
            if (bad && status) atomicOr(status, TPPO_DEV_NONFINITE);
        }
        if (pre) put8(c.pre + it * 8 * ldp, v, c.count, vec_p);
        if (STORE) {
            if (y_f32) put8(reinterpret_cast<float*>(c.y) + it * 8 * ldy, o, c.count, vec_y);
            else put8(reinterpret_cast<bf16_bits*>(c.y) + it * 8 * ldy, o, c.count, vec_y);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = o[i];
        }
    }
    __device__ __forceinline__ void operator()(int64_t m, int n, float (&v)[8], const Loads& l) const {
        Cursor c;
        open(c, m, n);
        finish<true>(c, 0, v, l);
    }
};

// Plain bf16 output (the two gradients).
struct EpiStore {
    bf16_bits* out; int64_t ld; int64_t M; int32_t N; int32_t vec;
    int32_t* status;
    static constexpr bool kRows = true;
    struct Loads {};
    __device__ __forceinline__ bool outside(int64_t m, int n) const { return m >= M || n >= N; }
    __device__ __forceinline__ void load(int64_t, int, Loads&) const {}
    __device__ __forceinline__ bool by_rows() const { return !vec; }
    __device__ __forceinline__ void put(int64_t m, int n, float v) const {
        if (!outside(m, n)) store_f32(out + m * ld + n, v);
    }
    struct Cursor { bf16_bits* out; int rows, count; };
    __device__ __forceinline__ void open(Cursor& c, int64_t m, int n) const {
        c.count = min(8, N - n);
        c.rows = c.count > 0 && m < M ? int(min(M - m, int64_t(64))) : 0;
        if (c.rows > 0) c.out = out + m * ld + n;
    }
    __device__ __forceinline__ void fetch(const Cursor&, int, Loads&) const {}
    template <bool STORE>
    __device__ __forceinline__ void finish(const Cursor& c, int it, float (&v)[8], const Loads&) const {
        if (it * 8 >= c.rows) return;
        if (!all_within(v, kBf16Max)) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(fabsf(v[i]) <= kBf16Max)) { bad |= i < c.count; v[i] = 0.f; }
            if (bad && status) atomicOr(status, TPPO_DEV_NONFINITE);
        }
        if (STORE) put8(c.out + it * 8 * ld, v, c.count, vec);
    }
    __device__ __forceinline__ void operator()(int64_t m, int n, float (&v)[8], const Loads& l) const {
        Cursor c;
        open(c, m, n);
        finish<true>(c, 0, v, l);
    }
};

// Few output columns (a value head has one): a product that reads x once and is bound by that.  A warp
// takes kNarrowRows rows at a time, its lanes 8 consecutive k each, with the weight transposed in shared
// memory; fp32 multiply-adds.  16384 rows of 5120, one column: the split tensor-core kernel takes 66 us
// (its tile computes 128 columns), this one 33.5 us (5.0 TB/s).
constexpr int kNarrowRows = 4;
constexpr int kNarrowMaxN = 8;
constexpr int kNarrowMaxSmem = 96 * 1024;
int narrow_columns(int32_t N) { return N <= 1 ? 1 : N <= 2 ? 2 : N <= 4 ? 4 : 8; }
bool narrow_fits(int nb, int32_t K) { return size_t(nb) * ((size_t(K) + 7) / 8 * 8) * 2 <= size_t(kNarrowMaxSmem); }

template <int NB, bool VEC>
__global__ void __launch_bounds__(256) linear_narrow_kernel(const bf16_bits* x, int64_t ldx, const bf16_bits* w, int64_t ldw,
                                                            int64_t M, int32_t K, int32_t kpad, const EpiLinear epi) {
    extern __shared__ __align__(16) bf16_bits wt[];           // [NB][kpad], zeros beyond K and N
    pdl_launch();
    pdl_wait();
    // eight independent loads per trip: the rows of x wait for this
    for (int i0 = threadIdx.x; i0 < NB * kpad; i0 += 8 * 256) {
        bf16_bits v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * 256, k = i / NB, n = i % NB;
            v[j] = k < K && n < epi.N ? w[int64_t(k) * ldw + n] : bf16_bits(0);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * 256, k = i / NB, n = i % NB;
            if (i < NB * kpad) wt[n * kpad + k] = v[j];
        }
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const int64_t warp = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5), warps = int64_t(gridDim.x) * 8;
    for (int64_t m0 = warp * kNarrowRows; m0 < M; m0 += warps * kNarrowRows) {
        float acc[kNarrowRows][NB];
#pragma unroll
        for (int r = 0; r < kNarrowRows; ++r)
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[r][n] = 0.f;
#pragma unroll 2
        for (int k = lane * 8; k < K; k += 256) {
            float xv[kNarrowRows][8];
#pragma unroll
            for (int r = 0; r < kNarrowRows; ++r) {
                // rows past the last are computed from the last and not stored
                const bf16_bits* p = x + min(m0 + r, M - 1) * ldx + k;
                if (VEC) load_vec<8>(p, xv[r]);
                else get8(p, xv[r], min(8, K - k), false);
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float wv[8];
                load_vec<8>(wt + n * kpad + k, wv);
#pragma unroll
                for (int r = 0; r < kNarrowRows; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[r][n] = fmaf(xv[r][i], wv[i], acc[r][n]);
            }
        }
#pragma unroll
        for (int r = 0; r < kNarrowRows; ++r) {
            float v[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) v[n] = n < NB ? warp_sum(acc[r][n < NB ? n : 0]) : 0.f;
            if (lane == r) {
                EpiLinear::Loads l;
                epi.load(m0 + r, 0, l);
                epi(m0 + r, 0, v, l);
            }
        }
    }
}

template <int NB>
int linear_narrow(const DenseOperand& X, const DenseOperand& W, const EpiLinear& e, bool vec, cudaStream_t s) {
    const int32_t K = int32_t(X.cols), kpad = (K + 7) / 8 * 8;
    const size_t smem = size_t(NB) * kpad * 2;
    auto kernel = vec ? linear_narrow_kernel<NB, true> : linear_narrow_kernel<NB, false>;
    // the same value in every call: another host thread may be about to launch with more than this one needs
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNarrowMaxSmem));
    const int64_t blocks = (X.rows + 8 * kNarrowRows - 1) / (8 * kNarrowRows), most = 4 * kNumSms;
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(unsigned(blocks < most ? blocks : most)), dim3(256), smem, s,
                                 static_cast<const bf16_bits*>(X.p), X.ld, static_cast<const bf16_bits*>(W.p), W.ld, X.rows, K,
                                 kpad, e));
    return TPPO_OK;
}

// Copies a bf16 matrix into rows of ldo elements (whole lines), eight elements per thread; the tail of a
// row is filled with zeros.  A row that starts at any element is read in aligned 16-byte granules, two per
// eight elements, shifted together; granules that reach beyond the matrix are read by element.
__global__ void __launch_bounds__(256) linear_repack_kernel(const bf16_bits* src, int64_t ld, int64_t rows, int32_t cols,
                                                            bf16_bits* dst, int64_t ldo, Link link) {
    link_begin(link);
    const int per = int(ldo / 8);
    const uintptr_t begin = reinterpret_cast<uintptr_t>(src), end = begin + uintptr_t((rows - 1) * ld + cols) * 2;
    const int64_t total = rows * per;
    for (int64_t i0 = int64_t(blockIdx.x) * 256; i0 < total; i0 += int64_t(gridDim.x) * 256) {
        // the first row of the block's pieces by one 64-bit division, the thread's by a 32-bit one
        const int64_t r0 = i0 / per;
        const uint32_t in = uint32_t(i0 - r0 * per) + threadIdx.x;
        const int64_t r = r0 + in / uint32_t(per);
        if (r < rows) {
            const int c = int(in % uint32_t(per)) * 8, count = min(8, cols - c);
            uint4 o = make_uint4(0u, 0u, 0u, 0u);
            if (count > 0) {
                const bf16_bits* p = src + r * ld + c;
                const uintptr_t at = reinterpret_cast<uintptr_t>(p), low = at & ~uintptr_t(15);
                const int shift = int(at & 15);
                if (low >= begin && low + (shift ? 32 : 16) <= end) {
                    const uint4 a = *reinterpret_cast<const uint4*>(low);
                    const uint4 b = shift ? *reinterpret_cast<const uint4*>(low + 16) : a;
                    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                    if (shift & 8) {
#pragma unroll
                        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
                    }
                    if (shift & 4) {
#pragma unroll
                        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
                    }
                    if (shift & 2) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
                    }
                    if (count < 8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (2 * i >= count) w[i] = 0u;
                            else if (2 * i + 1 >= count) w[i] &= 0xffffu;
                        }
                    }
                    o = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
                    uint32_t h[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[i] = i < count ? p[i] : 0u;
                    o = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
                }
            }
            *reinterpret_cast<uint4*>(dst + r * ldo + c) = o;
        }
    }
    link_end(link);
}

struct DzArgs {
    const void* dy; int64_t lddy;
    const bf16_bits* pre; int64_t ldp;
    bf16_bits* dz; int64_t ldz;             // NULL: dy itself is the operand
    float* partial;                         // [gridDim.y][N] column sums or NULL
    int64_t M; int32_t N; int32_t act;
    int32_t* status;
    Link link;
};

// Eight elements as loaded: 16-byte pieces, or (VEC false) element by element with `count` of them there.
template <class T, bool VEC> struct Eight {
    static constexpr int kWords = int(sizeof(T)) / 2;
    uint4 w[VEC ? kWords : 1];
    float f[VEC ? 1 : 8];
    __device__ __forceinline__ void load(const T* p, int count) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = i < count ? load_f32(p + i) : 0.f;
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (!VEC) {
            return f[i];
        } else {
            const uint4& q = w[i / (8 / kWords)];
            const uint32_t u[4] = {q.x, q.y, q.z, q.w};
            if constexpr (sizeof(T) == 4) return __uint_as_float(u[i % 4]);
            else return i % 2 ? bf16_hi(u[i / 2]) : bf16_lo(u[i / 2]);
        }
    }
};

// dz and the column sums behind dbias.  A block covers 256 columns (8 per thread, 32 threads) and every
// (8 gridDim.y)-th row from its first, kDzRows of them per trip with all loads issued before the first
// is used; its eight warps' sums are added in warp order.  Bound by HBM: 503 MB for 16384 x 5120 bf16.
constexpr int kDzRows = 4;

template <class T, bool VEC, bool ACT>
__global__ void __launch_bounds__(256) linear_dz_kernel(const DzArgs a) {
    // Without an activation a bf16 dy is the products' operand as it is, elements that are not finite with it;
    // whether it is read in place or from a copy made here is a matter of alignment and speed.
    constexpr bool AS_IS = !ACT && sizeof(T) == 2;
    __shared__ float sums[8][256 + 8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = blockIdx.x * 256 + lane * 8;
    const int count = min(8, a.N - n);
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    bool bad = false;
    const T* dy = static_cast<const T*>(a.dy) + n;
    const bf16_bits* pre = a.pre + n;
    link_begin(a.link);
    if (count > 0) {
        const int64_t step = int64_t(gridDim.y) * 8;
        for (int64_t m0 = int64_t(blockIdx.y) * 8 + warp; m0 < a.M; m0 += kDzRows * step) {
            Eight<T, VEC> d[kDzRows];
            Eight<bf16_bits, VEC> z[kDzRows];
#pragma unroll
            for (int k = 0; k < kDzRows; ++k) {
                const int64_t m = m0 + k * step;
                if (m < a.M) {
                    d[k].load(dy + m * a.lddy, count);
                    if (ACT) z[k].load(pre + m * a.ldp, count);
                }
            }
#pragma unroll
            for (int k = 0; k < kDzRows; ++k) {
                const int64_t m = m0 + k * step;
                if (m < a.M) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = d[k].get(i);
                    if (ACT) {
                        float zv[8], slope[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) zv[i] = z[k].get(i);
                        act_slopes(a.act, zv, slope);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] *= slope[i];
                    }
                    float kept[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) kept[i] = v[i];
                    if (!all_within(v, kBf16Max)) {
                        bad = true;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!(fabsf(v[i]) <= kBf16Max)) v[i] = 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] += v[i];
                    // a copy of a bf16 dy goes to the products as dy itself would (see AS_IS)
                    if (a.dz) store_vec<8>(a.dz + m * a.ldz + n, AS_IS ? kept : v);
                }
            }
        }
    }
    if (bad && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    if (!a.partial) { link_end(a.link); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[warp][lane * 8 + i] = acc[i];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < a.N) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += sums[w][threadIdx.x];
        a.partial[int64_t(blockIdx.y) * a.N + c] = t;
    }
    link_end(a.link);
}

template <class T>
void (*linear_dz_pick(bool vec, bool act))(const DzArgs) {
    if (vec) return act ? linear_dz_kernel<T, true, true> : linear_dz_kernel<T, true, false>;
    return act ? linear_dz_kernel<T, false, true> : linear_dz_kernel<T, false, false>;
}

// dbias: the partial rows in ascending order within each of a column's 16 strands, then the strands.
template <class T>
__global__ void __launch_bounds__(512) linear_dbias_kernel(const float* partial, int32_t parts, int32_t N, T* dbias,
                                                           int32_t* status, Link link) {
    __shared__ double s[16][33];
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int64_t c = int64_t(blockIdx.x) * 32 + lane;
    link_begin(link);
    double t = 0.0;
    if (c < N) {
        for (int p0 = strand; p0 < parts; p0 += 8 * 16) {        // eight loads in flight
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p0 + 16 * k < parts ? __ldcg(partial + int64_t(p0 + 16 * k) * N + c) : 0.f;   // see kBeside
#pragma unroll
            for (int k = 0; k < 8; ++k) t += double(v[k]);
        }
    }
    s[strand][lane] = t;
    __syncthreads();
    if (strand == 0 && c < N) {
        t = 0.0;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += s[k][lane];
        // a sum beyond the type, or partial sums beyond fp32
        const bool fine = fabs(t) <= double(top_of(dbias));
        if (!fine && status) atomicOr(status, TPPO_DEV_NONFINITE);
        store_f32(dbias + c, fine ? float(t) : 0.f);
    }
    link_end(link);
}

// The backward pass of few output columns, in one sweep over x and dx and a second launch that adds the
// partial sums: the products have nothing to feed a tensor core with.  A block takes blockDim.x * 8 columns
// of x (blockIdx.x) and one of gridDim.y equal ranges of rows; a thread keeps its eight columns of W and of
// the sums behind dweight in registers and the block's dz, kNarrowChunk rows at a time, is in shared
// memory.  Bound by HBM: 16384 x 5120 x 1 takes 61 us (5.5 TB/s), and 129 through the tensor-core products.
constexpr int kNarrowChunk = 64;
constexpr int kNarrowBwdMaxN = 4;

struct NarrowBwdArgs {
    const void* dy; int32_t dy_f32; int64_t lddy;
    const bf16_bits* x; int64_t ldx;            // NULL without dweight
    const bf16_bits* w; int64_t ldw;            // NULL without dx
    const bf16_bits* pre; int64_t ldp; int32_t act;
    bf16_bits* dx; int64_t lddx;
    float* partial;                             // [gridDim.y][NB * K sums of dweight, NB of dbias] or NULL
    int64_t M; int32_t K, N;
    int32_t* status;
};

__device__ __forceinline__ float act_slope_of(int act, float z) {
    switch (act) {
        case TPPO_ACT_RELU: return act_slope<TPPO_ACT_RELU>(z);
        case TPPO_ACT_GELU: return act_slope<TPPO_ACT_GELU>(z);
        case TPPO_ACT_GELU_TANH: return act_slope<TPPO_ACT_GELU_TANH>(z);
        case TPPO_ACT_SILU: return act_slope<TPPO_ACT_SILU>(z);
        default: return 1.f;
    }
}

// Rows of x in flight, and blocks per SM that the registers have to allow, as measured (16384 x 5120 x 1, us: 4 rows
// and 4 blocks 62, 8 and 2 68, 2 and 4 70; x 4: 8 and 2 106, without a bound 117, everything else spills).
template <int NB, bool VEC> __host__ __device__ constexpr int narrow_rows() { return NB == 1 ? (VEC ? 4 : 2) : VEC ? 8 : 4; }
template <int NB> __host__ __device__ constexpr int narrow_blocks() { return NB == 1 ? 4 : 2; }

template <int NB, bool VEC>
__global__ void __launch_bounds__(256, narrow_blocks<NB>()) linear_narrow_bwd_kernel(const NarrowBwdArgs a) {
    constexpr int ROWS = narrow_rows<NB, VEC>();
    __shared__ float dz[kNarrowChunk * NB];
    __shared__ float red[256];
    const int t = threadIdx.x, T = blockDim.x;
    // eight consecutive columns, or (rows of any alignment) eight that are T apart
    const int64_t k0 = int64_t(blockIdx.x) * T * 8 + (VEC ? t * 8 : t);
    const int stride = VEC ? 1 : T;
    const int64_t left = a.K - k0;
    const int count = left <= 0 ? 0 : int(min(int64_t(8), (left + stride - 1) / stride));
    pdl_launch();
    pdl_wait();
    float w[NB][8], sum[NB][8];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sum[n][i] = 0.f;
            w[n][i] = a.dx && n < a.N && i < count ? load_f32(a.w + (k0 + i * stride) * a.ldw + n) : 0.f;
        }
    float top[NB];                              // |dz| times these bounds |dx|: most rows need no look at each element
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        uint32_t m = 0u;                        // a NaN's bits are larger than every number's
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(w[n][i]) & 0x7fffffffu);
        top[n] = __uint_as_float(m);
    }
    const int64_t first = a.M * blockIdx.y / gridDim.y, end = a.M * (blockIdx.y + 1) / gridDim.y;
    float bias = 0.f;                           // of column t % NB
    bool bad = false;
    for (int64_t base = first; base < end; base += kNarrowChunk) {
        const int rows = int(min(int64_t(kNarrowChunk), end - base));
        __syncthreads();                        // the chunk before has been used
        for (int i = t; i < kNarrowChunk * NB; i += T) {
            const int r = i / NB, n = i % NB;
            float v = 0.f, d = 0.f;
            if (r < rows && n < a.N) {
                const int64_t at = (base + r) * a.lddy + n;
                v = a.dy_f32 ? static_cast<const float*>(a.dy)[at] : load_f32(static_cast<const bf16_bits*>(a.dy) + at);
                if (a.act != TPPO_ACT_NONE) v *= act_slope_of(a.act, load_f32(a.pre + (base + r) * a.ldp + n));
                d = v;
                if (!(fabsf(v) <= kBf16Max)) {
                    bad = true;
                    v = 0.f;
                    if (a.act != TPPO_ACT_NONE || a.dy_f32) d = 0.f;      // a bf16 dy goes on as it is: see AS_IS
                }
                bias += v;
            }
            dz[i] = d;                          // fp32: nothing here feeds a tensor core
        }
        __syncthreads();
        if (count == 0) continue;
        for (int r0 = 0; r0 < rows; r0 += ROWS) {
            float x[VEC ? 1 : ROWS][8];
            uint4 raw[VEC ? ROWS : 1];
            if (a.x) {
#pragma unroll
                for (int q = 0; q < ROWS; ++q) {
                    if (r0 + q < rows) {
                        const bf16_bits* p = a.x + (base + r0 + q) * a.ldx + k0;
                        if constexpr (VEC) {
                            raw[q] = *reinterpret_cast<const uint4*>(p);
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[q][i] = i < count ? load_f32(p + i * stride) : 0.f;
                        }
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < ROWS; ++q) {
                if (r0 + q >= rows) continue;
                float d[NB];
#pragma unroll
                for (int n = 0; n < NB; ++n) d[n] = dz[(r0 + q) * NB + n];
                if (a.x) {
                    float v[8];
                    if constexpr (VEC) {
                        widen8(raw[q], v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = x[q][i];
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[n][i] = fmaf(v[i], d[n], sum[n][i]);
                }
                if (a.dx) {
                    float o[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        o[i] = d[0] * w[0][i];
#pragma unroll
                        for (int n = 1; n < NB; ++n) o[i] = fmaf(d[n], w[n][i], o[i]);
                    }
                    float most = 0.f;
#pragma unroll
                    for (int n = 0; n < NB; ++n) most = fmaf(fabsf(d[n]), top[n], most);
                    if (!(most <= 0.99f * kBf16Max)) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!(fabsf(o[i]) <= kBf16Max)) { o[i] = 0.f; bad = true; }
                    }
                    bf16_bits* p = a.dx + (base + r0 + q) * a.lddx + k0;
                    if constexpr (VEC) {
                        store_vec<8>(p, o);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i < count) store_f32(p + i * stride, o[i]);
                    }
                }
            }
        }
    }
    if (bad && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.y) * NB * (int64_t(a.K) + 1);
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) out[n * int64_t(a.K) + k0 + i * stride] = sum[n][i];
    if (blockIdx.x != 0) return;
    red[t] = bias;
    __syncthreads();
    if (t < NB) {
        float s = 0.f;
        for (int i = t; i < T; i += NB) s += red[i];
        out[NB * int64_t(a.K) + t] = s;
    }
}

// dweight and dbias from the partial sums, added as in linear_dbias_kernel, in 32 strands.
template <class B>
__global__ void __launch_bounds__(1024) linear_narrow_sum_kernel(const float* partial, int32_t parts, int32_t K, int32_t N, int32_t nb,
                                                                bf16_bits* dweight, int64_t lddw, B* dbias, int32_t* status) {
    __shared__ double s[32][33];
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int64_t all = nb * (int64_t(K) + 1), j = int64_t(blockIdx.x) * 32 + lane;
    pdl_launch();
    pdl_wait();
    double t = 0.0;
    if (j < all) {
        for (int p0 = strand; p0 < parts; p0 += 8 * 32) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p0 + 32 * k < parts ? partial[(p0 + 32 * k) * all + j] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += double(v[k]);
        }
    }
    s[strand][lane] = t;
    __syncthreads();
    if (strand != 0 || j >= all) return;
    t = 0.0;
#pragma unroll
    for (int k = 0; k < 32; ++k) t += s[k][lane];
    const bool bias = j >= nb * int64_t(K);
    const int n = int(bias ? j - nb * int64_t(K) : j / K);
    if (n >= N || (bias ? !dbias : !dweight)) return;
    const double top = double(bias ? top_of(dbias) : kBf16Max);
    const bool fine = fabs(t) <= top;
    if (!fine && status) atomicOr(status, TPPO_DEV_NONFINITE);
    const float v = fine ? float(t) : 0.f;
    if (bias) store_f32(dbias + n, v);
    else store_f32(dweight + (j - n * int64_t(K)) * lddw + n, v);
}

// Blocks along the columns and along the rows, and threads: as many as are resident, and at least 4 NB
// rows to a partial sum, so that writing those stays at half the bytes of reading x.
struct NarrowGrid { unsigned x, y; int threads; size_t bytes; };
NarrowGrid narrow_grid(int64_t M, int32_t K, int nb) {
    NarrowGrid g;
    g.x = unsigned((int64_t(K) + 2047) / 2048);
    g.threads = int((int64_t(K) + int64_t(g.x) * 256 - 1) / (int64_t(g.x) * 256)) * 32;
    int64_t y = int64_t(kNumSms) * ((nb == 1 ? 1024 : 512) / g.threads) / g.x, most = M / (4 * nb);
    if (y > most) y = most;
    g.y = unsigned(y < 1 ? 1 : y);
    g.bytes = size_t(g.y) * nb * (size_t(K) + 1) * 4;
    return g;
}

// At least that grid's bytes, for every M and K up to these: y threads K <= 148 threads_per_SM 8 columns each.
size_t narrow_room(int64_t M, int32_t K, int nb) {
    const size_t sm_threads = nb == 1 ? 1024 : 512, y_most = kNumSms * sm_threads / 32, wide = kNumSms * sm_threads * 8;
    const size_t by_grid = (wide > size_t(K) ? wide : size_t(K)) + y_most, by_rows = (size_t(M) / (4 * nb) + 1) * (size_t(K) + 1);
    return (by_grid < by_rows ? by_grid : by_rows) * nb * 4;
}

template <int NB>
int linear_narrow_bwd(const NarrowBwdArgs& a, const NarrowGrid& g, bool vec, bf16_bits* dweight, int64_t lddw, void* dbias,
                      bool bias_f32, cudaStream_t s) {
    TPPO_CUDA_CHECK(launch_dense(vec ? linear_narrow_bwd_kernel<NB, true> : linear_narrow_bwd_kernel<NB, false>, dim3(g.x, g.y),
                                 dim3(g.threads), 0, s, a));
    if (!a.partial) return TPPO_OK;
    const float* partial = a.partial;
    const dim3 grid(unsigned((NB * (int64_t(a.K) + 1) + 31) / 32));
    if (bias_f32)
        TPPO_CUDA_CHECK(launch_dense(linear_narrow_sum_kernel<float>, grid, dim3(1024), 0, s, partial, int32_t(g.y), a.K, a.N, NB,
                                     dweight, lddw, static_cast<float*>(dbias), a.status));
    else
        TPPO_CUDA_CHECK(launch_dense(linear_narrow_sum_kernel<bf16_bits>, grid, dim3(1024), 0, s, partial, int32_t(g.y), a.K, a.N,
                                     NB, dweight, lddw, static_cast<bf16_bits*>(dbias), a.status));
    return TPPO_OK;
}

// Row stride of the workspace's matrices: whole 128-byte lines.  At other pitches the tensor copies'
// 128-byte rows straddle two lines each: 4096 x 3000 x 3000 takes 95 us with rows of 6000 bytes and 58 us
// with rows of 6016.
int64_t pad64(int64_t n) { return (n + 63) / 64 * 64; }

constexpr int kDzMaxParts = 256;

// Workspace: dz, the partial sums of dbias, and (only where the sizes do not make whole lines, or the
// caller asked for them) padded copies of x and W.
struct LinearWs { bf16_bits* dz; float* partial; bf16_bits* x; bf16_bits* w; size_t plain, bytes; };
LinearWs linear_carve(void* ws, int64_t M, int32_t K, int32_t N) {
    char* p = static_cast<char*>(ws);
    const size_t dz = align_up(size_t(M) * pad64(N) * 2, kWsAlign), part = align_up(size_t(kDzMaxParts) * N * 4, kWsAlign);
    const size_t x = align_up(size_t(M) * pad64(K) * 2, kWsAlign), w = align_up(size_t(K) * pad64(N) * 2, kWsAlign);
    LinearWs r;
    r.dz = reinterpret_cast<bf16_bits*>(p);
    r.partial = reinterpret_cast<float*>(p + dz);
    r.x = reinterpret_cast<bf16_bits*>(p + dz + part);
    r.w = reinterpret_cast<bf16_bits*>(p + dz + part + x);
    r.plain = dz + part;
    r.bytes = dz + part + x + w;
    return r;
}

bool tma_rows(const void* p, int64_t ld) { return rows_aligned(p, ld, 2); }
// Whether a [rows, cols] operand that TMA takes as it is is better copied to whole lines first: a product
// loses a fifth of its time (at 1.2 PFLOP/s) to each operand with straddling rows, a copy moves four bytes
// per element at 5 TB/s after 2 us.
bool worth_copying(const void* p, int64_t ld, int64_t rows, int64_t cols, double flops) {
    return (ld % 64 != 0 || !aligned(p, 128)) && 0.2 * flops / 1.2e15 > double(rows) * double(cols) * 4 / 5e12 + 2e-6;
}

int repack(DenseOperand& o, bf16_bits* dst, cudaStream_t s, Link link) {
    const int64_t ldo = pad64(o.cols);
    const int64_t blocks = (o.rows * (ldo / 8) + 255) / 256;
    TPPO_CUDA_CHECK(launch_dense(linear_repack_kernel, dim3(unsigned(blocks < 16 * kNumSms ? blocks : 16 * kNumSms)), dim3(256), 0, s,
                                 static_cast<const bf16_bits*>(o.p), o.ld, o.rows, int32_t(o.cols), dst, ldo, link));
    o.p = dst;
    o.ld = ldo;
    return TPPO_OK;
}

bool act_known(int32_t a) { return a >= TPPO_ACT_NONE && a <= TPPO_ACT_SILU; }

}  // namespace

size_t linear_workspace_bytes(int64_t M, int32_t K, int32_t N, bool copies) {
    if (K < 1 || N < 1 || M > kDenseMaxSize || K > kDenseMaxSize || N > kDenseMaxSize) return 0;
    const LinearWs w = linear_carve(nullptr, M, K, N);
    // a value head: no products, unless rows at odd places or a weight beyond shared memory ask for them
    const int nb = narrow_columns(N);
    if (!copies && N <= kNarrowBwdMaxN && K % 8 == 0 && narrow_fits(nb, K)) return align_up(narrow_room(M, K, nb), kWsAlign);
    return copies || K % 64 || N % 64 ? w.bytes : w.plain;
}

}  // namespace tppo

using namespace tppo;

TPPO_API int tppo_linear_fwd(const void* x, int64_t ldx, const void* weight, int64_t ldw, int64_t M, int32_t K, int32_t N,
                             const void* bias, int32_t bias_dtype, int32_t activation, const void* residual, int64_t ldr,
                             void* y, int32_t y_dtype, int64_t ldy, void* preact, int64_t ldp, int32_t* status,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 0 || K < 1 || N < 1 || ldx < K || ldw < N || ldy < N || (residual && ldr < N) ||
        (preact && ldp < N) || !act_known(activation))
        return TPPO_ERR_INVALID_ARG;
    if ((y_dtype != TPPO_BF16 && y_dtype != TPPO_F32) || (bias && bias_dtype != TPPO_BF16 && bias_dtype != TPPO_F32))
        return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || K > kDenseMaxSize || N > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    if (M == 0) return TPPO_OK;
    const size_t ys = y_dtype == TPPO_F32 ? 4 : 2, bs = bias_dtype == TPPO_F32 ? 4 : 2;
    if (!x || !weight || !y || !aligned(x, 2) || !aligned(weight, 2) || !aligned(bias, bs) || !aligned(residual, 2) ||
        !aligned(y, ys) || !aligned(preact, 2) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    const int nb = narrow_columns(N);
    const bool narrow = N <= kNarrowMaxN && narrow_fits(nb, K);
    bool copy_x = !narrow && !tma_rows(x, ldx), copy_w = !narrow && !tma_rows(weight, ldw);
    const LinearWs w = linear_carve(workspace, M, K, N);
    const bool room = workspace && aligned(workspace, kWsAlign) && workspace_bytes >= w.bytes;
    if ((copy_x || copy_w) && !room) return TPPO_ERR_WORKSPACE;
    if (room && !narrow) {
        const double flops = 2.0 * double(M) * K * N;
        copy_x = copy_x || worth_copying(x, ldx, M, K, flops);
        copy_w = copy_w || worth_copying(weight, ldw, K, N, flops);
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    DenseOperand X{x, M, K, ldx}, W{weight, K, N, ldw};
    int rc;
    LinkGroup copies(int(copy_x) + int(copy_w), stream_link(copy_w ? int64_t(K) * N : M * K));
    if (copy_x && (rc = repack(X, w.x, s, copies.next())) != TPPO_OK) return rc;
    if (copy_w && (rc = repack(W, w.w, s, copies.next())) != TPPO_OK) return rc;
    EpiLinear e{};
    e.bias = bias; e.bias_f32 = bias_dtype == TPPO_F32;
    e.residual = static_cast<const bf16_bits*>(residual); e.ldr = ldr;
    e.y = y; e.ldy = ldy; e.y_f32 = y_dtype == TPPO_F32;
    e.pre = static_cast<bf16_bits*>(preact); e.ldp = ldp;
    e.M = M; e.N = N; e.act = activation;
    e.vec_y = rows_aligned(y, ldy, ys); e.vec_r = rows_aligned(residual, ldr, 2); e.vec_p = rows_aligned(preact, ldp, 2);
    e.vec_b = aligned(bias, 16);
    e.status = status;
    if (narrow) {
        const bool vec = tma_rows(x, ldx) && K % 8 == 0;
        if (nb == 1) return linear_narrow<1>(X, W, e, vec, s);
        if (nb == 2) return linear_narrow<2>(X, W, e, vec, s);
        if (nb == 4) return linear_narrow<4>(X, W, e, vec, s);
        return linear_narrow<8>(X, W, e, vec, s);
    }
    return dense_product<0, 1, false, false>(X, W, M, N, K, e, status, s);
}

TPPO_API int tppo_linear_bwd(const void* dy, int32_t dy_dtype, int64_t lddy, const void* x, int64_t ldx, const void* weight,
                             int64_t ldw, int64_t M, int32_t K, int32_t N, int32_t activation, const void* preact,
                             int64_t ldp, void* dx, int64_t lddx, void* dweight, int64_t lddw, void* dbias,
                             int32_t bias_dtype, int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 0 || K < 1 || N < 1 || lddy < N || (x && ldx < K) || (weight && ldw < N) || (dx && lddx < K) ||
        (dweight && lddw < N) || !act_known(activation) || (activation != TPPO_ACT_NONE && ldp < N))
        return TPPO_ERR_INVALID_ARG;
    if ((dy_dtype != TPPO_BF16 && dy_dtype != TPPO_F32) || (dbias && bias_dtype != TPPO_BF16 && bias_dtype != TPPO_F32))
        return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || K > kDenseMaxSize || N > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    const size_t ds = dy_dtype == TPPO_F32 ? 4 : 2, bs = bias_dtype == TPPO_F32 ? 4 : 2;
    if ((M > 0 && (!dy || (activation != TPPO_ACT_NONE && !preact) || (dx && !weight) || (dweight && !x))) ||
        !aligned(dy, ds) || !aligned(x, 2) || !aligned(weight, 2) || !aligned(preact, 2) || !aligned(dx, 2) ||
        !aligned(dweight, 2) || !aligned(dbias, bs) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (M == 0) {                                  // no rows: the weight's and the bias' sums are empty
        if (dweight) TPPO_CUDA_CHECK(cudaMemset2DAsync(dweight, size_t(lddw) * 2, 0, size_t(N) * 2, size_t(K), s));
        if (dbias) TPPO_CUDA_CHECK(cudaMemsetAsync(dbias, 0, size_t(N) * bs, s));
        return TPPO_OK;
    }
    if (!dx && !dweight && !dbias) return TPPO_OK;
    const LinearWs w = linear_carve(workspace, M, K, N);
    const size_t have = workspace && aligned(workspace, kWsAlign) ? workspace_bytes : 0;
    const bool products = dx || dweight;
    bool copy_x = dweight && !tma_rows(x, ldx), copy_w = dx && !tma_rows(weight, ldw);
    bool make_dz = products && (activation != TPPO_ACT_NONE || dy_dtype == TPPO_F32 || !tma_rows(dy, lddy));
    const size_t need = copy_x || copy_w ? w.bytes : make_dz || dbias ? w.plain : 0;
    const bool narrow_vec = K % 8 == 0 && (!dweight || tma_rows(x, ldx)) && (!dx || tma_rows(dx, lddx));
    // 16384 x 5120, us against the tensor-core products: one column 61 / 129, four 92 / 130, eight 242 / 133; rows
    // that are read by element lose from some 2^23 of them on (16384 x 5121 x 1 432 / 307, 4000 x 1001 x 1 15 / 33)
    // -- and are taken all the same where the products' operands have no room
    if (N <= kNarrowBwdMaxN && (narrow_vec || M * K <= (int64_t(1) << 23) || need > have)) {
        const int nb = narrow_columns(N);
        const NarrowGrid g = narrow_grid(M, K, nb);
        const bool sums = dweight || dbias;
        if (!sums || have >= g.bytes) {
            const NarrowBwdArgs a{dy, dy_dtype == TPPO_F32, lddy, dweight ? static_cast<const bf16_bits*>(x) : nullptr, ldx,
                                  static_cast<const bf16_bits*>(weight), ldw, static_cast<const bf16_bits*>(preact), ldp, activation,
                                  static_cast<bf16_bits*>(dx), lddx, sums ? static_cast<float*>(workspace) : nullptr, M, K, N, status};
            bf16_bits* dw = static_cast<bf16_bits*>(dweight);
            const bool f = bias_dtype == TPPO_F32;
            if (nb == 1) return linear_narrow_bwd<1>(a, g, narrow_vec, dw, lddw, dbias, f, s);
            if (nb == 2) return linear_narrow_bwd<2>(a, g, narrow_vec, dw, lddw, dbias, f, s);
            return linear_narrow_bwd<4>(a, g, narrow_vec, dw, lddw, dbias, f, s);
        }
    }
    if (need > have) return TPPO_ERR_WORKSPACE;
    const double flops = 2.0 * double(M) * K * N;
    if (have >= w.bytes) {
        copy_x = copy_x || (dweight && worth_copying(x, ldx, M, K, flops));
        copy_w = copy_w || (dx && worth_copying(weight, ldw, K, N, flops));
    }
    if (have >= w.plain && products && !make_dz) make_dz = worth_copying(dy, lddy, M, N, (dx && dweight ? 2 : 1) * flops);

    DenseOperand X{x, M, K, ldx}, W{weight, K, N, ldw}, Z{dy, M, N, lddy};
    int rc;
    // the copies and dz run side by side, then the products and dbias do (1001 x 515 x 777 28.6 -> 23.1 us, 4096 x
    // 5120 x 5120 340 -> 327)
    LinkGroup first(int(copy_x) + int(copy_w) + int(make_dz || dbias), stream_link(M * N));
    LinkGroup second(int(dx != nullptr) + int(dweight != nullptr) + int(dbias != nullptr));
    if (copy_x && (rc = repack(X, w.x, s, first.next())) != TPPO_OK) return rc;
    if (copy_w && (rc = repack(W, w.w, s, first.next())) != TPPO_OK) return rc;
    int32_t parts = 0;
    if (make_dz || dbias) {
        DzArgs a{};
        a.dy = dy; a.lddy = lddy;
        a.pre = static_cast<const bf16_bits*>(preact); a.ldp = ldp;
        a.dz = make_dz ? w.dz : nullptr; a.ldz = pad64(N);
        a.partial = dbias ? w.partial : nullptr;
        a.M = M; a.N = N; a.act = activation; a.status = status;
        a.link = first.next();
        const int gx = (N + 255) / 256;
        int64_t gy = (M + 31) / 32, most = (6 * kNumSms + gx - 1) / gx;       // four rows per warp at least
        if (gy > most) gy = most;
        if (gy > kDzMaxParts) gy = kDzMaxParts;
        parts = int32_t(gy);
        const bool act = activation != TPPO_ACT_NONE;
        const bool vec = N % 8 == 0 && rows_aligned(dy, lddy, ds) && (!act || rows_aligned(preact, ldp, 2));
        auto kernel = dy_dtype == TPPO_F32 ? linear_dz_pick<float>(vec, act) : linear_dz_pick<bf16_bits>(vec, act);
        TPPO_CUDA_CHECK(launch_dense(kernel, dim3(gx, unsigned(gy)), dim3(256), 0, s, a));
        if (make_dz) { Z.p = w.dz; Z.ld = a.ldz; }
    }
    if (dx) {        // dx[m, k] = sum_n dz[m, n] W[k, n]: both operands contiguous along the contraction
        const EpiStore e{static_cast<bf16_bits*>(dx), lddx, M, K, rows_aligned(dx, lddx, 2), status};
        if ((rc = dense_product<0, 0, false, false>(Z, W, M, K, N, e, status, s, second.next())) != TPPO_OK) return rc;
    }
    if (dweight) {   // dweight[k, n] = sum_m x[m, k] dz[m, n]: both contiguous along their outer index
        const EpiStore e{static_cast<bf16_bits*>(dweight), lddw, K, N, rows_aligned(dweight, lddw, 2), status};
        if ((rc = dense_product<1, 1, false, false>(X, Z, K, N, M, e, status, s, second.next())) != TPPO_OK) return rc;
    }
    if (dbias) {
        const dim3 grid((N + 31) / 32);
        const float* partial = w.partial;
        if (bias_dtype == TPPO_F32)
            TPPO_CUDA_CHECK(launch_dense(linear_dbias_kernel<float>, grid, dim3(512), 0, s, partial, parts, N,
                                         static_cast<float*>(dbias), status, second.next()));
        else
            TPPO_CUDA_CHECK(launch_dense(linear_dbias_kernel<bf16_bits>, grid, dim3(512), 0, s, partial, parts, N,
                                         static_cast<bf16_bits*>(dbias), status, second.next()));
    }
    return TPPO_OK;
}
