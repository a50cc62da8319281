// Orthogonalised update of a weight matrix: momentum, normalisation and Newton-Schulz products.
//     momentum = mu * momentum + grad,   U = grad + mu * momentum (Nesterov) or momentum
//     X = U / (|U|_F + eps);  `steps` times:  A = X X^T,  B = b A + c A^2,  X = a X + B X
//     update = scale * X
// from the smaller side: with more rows than columns A = X^T X and X = a X + X B.
//
// The products run on the tensor cores, in fp16 with fp32 accumulation.  fp16 because bf16's 8 bits
// leave an error of 1 % of the result's norm after five steps and fp16's 11 bits 0.15 %, at the same
// rate; every operand is bounded (singular values of X stay below 1.21, of A below 1.45, of B below
// 2.81) and is stored times 2^13, which puts its largest possible element at 2.3e4 and keeps elements
// down to 2^-27 normal.  Two more choices keep the rounding harmless:
//   - X itself is carried in fp32 and enters a X from there; only the product's operand is rounded.  A
//     rounding error of X in a direction of small singular value would be amplified 3.4 times per step
//     (485 times in all); as an operand of B X it is not, because B nearly vanishes on those
//     directions.  For a matrix of low rank plus noise the error of the result falls from 3.5e-2 to
//     6e-4.
//   - In the last three steps A is near the identity, so its diagonal holds most of its rounding error
//     and B's diagonal that of B X.  There both diagonals are kept apart in fp32:
//         A = D + O:  A^2 = D^2 + DO + OD + O^2,   B X = diag(B) X + (B - diag(B)) X
//     with the diagonal's share of B X taken from the fp32 X (error 1.5e-3 -> 7e-4 of the norm).  In
//     the first steps that would feed the operand's rounding to the small directions again, so they
//     take plain A and B -- except for matrices of at most 64 on the smaller side, whose diagonal weighs
//     more than their spectrum.
//
// Work: A and A^2 are symmetric, so the persistent kernel computes the tiles of the lower triangle and
// mirrors them: m^2 n + m^3 + 2 m^2 n flop per step for an m x n matrix, m <= n, instead of
// 4 m^2 n + 2 m^3.  Large matrices are tensor bound, under the power cap; small ones are a chain of
// three launches per step and two before, each the programmatic dependent of the one before.
//   five steps: 5120 x 5120 2760-2980 us (900-970 TFLOP/s of the work above; SM clock at the power cap),
//   4096 x 4096 1280, 2048 x 2048 327, 256 x 1024 78 (seventeen launches).
#include <cuda_fp16.h>

#include "dense_gemm.cuh"

namespace tppo {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kScale = 8192.f, kUnscale = 1.f / 8192.f;        // 2^13 on every stored operand
constexpr int kMuonThreads = 256;
constexpr int kMuonMaxBlocks = 8 * kNumSms;

typedef uint16_t f16_bits;

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 unpack_f16x2(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// Eight stored operand elements: value * 2^13 in fp16 (rows of workspace matrices are padded, so the
// eight always exist).
__device__ __forceinline__ void store_operand(f16_bits* p, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_f16x2(v[0] * kScale, v[1] * kScale), pack_f16x2(v[2] * kScale, v[3] * kScale),
                   pack_f16x2(v[4] * kScale, v[5] * kScale), pack_f16x2(v[6] * kScale, v[7] * kScale));
}
__device__ __forceinline__ void widen_operand(const uint4& w, float (&v)[8]) {
    const float2 a = unpack_f16x2(w.x), b = unpack_f16x2(w.y), c = unpack_f16x2(w.z), d = unpack_f16x2(w.w);
    v[0] = a.x * kUnscale; v[1] = a.y * kUnscale; v[2] = b.x * kUnscale; v[3] = b.y * kUnscale;
    v[4] = c.x * kUnscale; v[5] = c.y * kUnscale; v[6] = d.x * kUnscale; v[7] = d.y * kUnscale;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    double t = 0.0;
    for (int w = 0; w < kMuonThreads / 32; ++w) t += red[w];
    return t;
}

struct PrepareArgs {
    const void* grad; int64_t ldg;
    float* momentum; int64_t ldm;              // NULL: U = grad
    float mu; int32_t nesterov;
    float* x32;                                // U, [R, ldx]
    double* partial;                           // [gridDim.x] sums of squares
    int64_t R; int32_t C; int64_t ldx;
    int32_t* status;
};

// Momentum and U.  A warp takes 32 * VEC consecutive elements of a row (VEC 8 where rows are aligned, else
// 1); a gradient or momentum element that is not finite counts as 0.  14 bytes move per element of a
// bf16 gradient, and nothing else bounds it.
template <class T, int VEC>
__global__ void __launch_bounds__(kMuonThreads) muon_prepare_kernel(const PrepareArgs a) {
    __shared__ double red[kMuonThreads / 32];
    pdl_launch();
    pdl_wait();
    constexpr int kRun = VEC == 1 ? 4 : 1;       // 32-element runs per trip: loads in flight
    const int lane = threadIdx.x & 31;
    const uint32_t per = uint32_t((a.C + 32 * VEC * kRun - 1) / (32 * VEC * kRun));
    const int64_t warps = int64_t(gridDim.x) * (kMuonThreads / 32), total = a.R * per;
    double sum = 0.0;
    bool bad = false;
    for (int64_t i = int64_t(blockIdx.x) * (kMuonThreads / 32) + (threadIdx.x >> 5); i < total; i += warps) {
        const int64_t r = i / per;
        const int c0 = int(uint32_t(i - r * per)) * 32 * VEC * kRun + lane * VEC;
        float g[kRun][VEC], m[kRun][VEC];
        float* pm = a.momentum + r * a.ldm;
#pragma unroll
        for (int q = 0; q < kRun; ++q) {
            const int c = c0 + q * 32;
            if (c < a.C) {
                load_vec<VEC>(static_cast<const T*>(a.grad) + r * a.ldg + c, g[q]);
                if (a.momentum) load_vec<VEC>(pm + c, m[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < kRun; ++q) {
            const int c = c0 + q * 32;
            if (c < a.C) {
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    if (!is_finite(g[q][k])) { g[q][k] = 0.f; bad = true; }
                if (a.momentum) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        m[q][k] = fmaf(a.mu, m[q][k], g[q][k]);
                        if (!is_finite(m[q][k])) { m[q][k] = 0.f; bad = true; }
                        g[q][k] = a.nesterov ? fmaf(a.mu, m[q][k], g[q][k]) : m[q][k];
                        if (!is_finite(g[q][k])) { g[q][k] = 0.f; bad = true; }
                    }
                    store_vec<VEC>(pm + c, m[q]);
                }
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < VEC; ++k) s = fmaf(g[q][k], g[q][k], s);
                // fp32 squares under- or overflow far from 1; those few go in fp64
                double wide = double(s);
                if (!(s > 1e-30f && s < 1e30f)) {
                    wide = 0.0;
#pragma unroll
                    for (int k = 0; k < VEC; ++k) wide += double(g[q][k]) * double(g[q][k]);
                }
                sum += wide;
                store_vec<VEC>(a.x32 + r * a.ldx + c, g[q]);
            }
        }
    }
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
    if (bad && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
}

// X's first operand U / (|U| + eps); every block adds the partial sums in the same order.  The first step
// multiplies U by `inverse` again, so that U itself need not be written once more -- but where that
// factor nears the ends of fp32's range the quotient is taken in fp64 and U replaced by it.
__global__ void __launch_bounds__(kMuonThreads) muon_normalise_kernel(const double* partial, int32_t parts, float eps,
                                                                      float* x32, f16_bits* x16, float* inverse,
                                                                      int64_t vectors, Link link) {
    __shared__ double red[kMuonThreads / 32];
    link_begin(link);
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kMuonThreads) s += partial[i];
    const double norm = sqrt(block_sum(s, red)) + double(eps);
    const double inv = norm > 0.0 ? 1.0 / norm : 0.0;
    const bool far = norm > 0.0 && !(inv > 1e-30 && inv < 1e30);
    const float f = far ? 1.f : float(inv);
    if (blockIdx.x == 0 && threadIdx.x == 0) *inverse = f;
    for (int64_t i = int64_t(blockIdx.x) * kMuonThreads + threadIdx.x; i < vectors; i += int64_t(gridDim.x) * kMuonThreads) {
        float v[8];
        load_vec<8>(x32 + i * 8, v);
        if (far) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = float(double(v[k]) * inv);
            store_vec<8>(x32 + i * 8, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= f;
        }
        store_operand(x16 + i * 8, v);
    }
}

// A = X X^T.  With `diag` its diagonal goes there and the stored operand has zeros instead.
struct EpiA {
    f16_bits* out; int64_t ld; int32_t m; float* diag;
    static constexpr bool kRows = false;
    struct Loads {};
    struct Cursor { f16_bits* out; int rows, off; };       // off: row - first column
    __device__ __forceinline__ bool outside(int64_t r, int c) const { return r >= m || c >= m; }
    __device__ __forceinline__ void load(int64_t, int, Loads&) const {}
    __device__ __forceinline__ void open(Cursor& k, int64_t r, int c) const {
        k.rows = outside(r, c) ? 0 : int(m - r);
        k.out = out + r * ld + c;
        k.off = int(r) - c;
    }
    __device__ __forceinline__ void fetch(const Cursor&, int, Loads&) const {}
    template <bool STORE>
    __device__ __forceinline__ void finish(const Cursor& k, int it, float (&v)[8], const Loads&) const {
        if (it * 8 >= k.rows) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= kUnscale * kUnscale;
        const int on = k.off + it * 8;            // where the row meets the diagonal
        if (diag && on >= 0 && on < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i == on) { diag[m - k.rows + it * 8] = v[i]; v[i] = 0.f; }
        }
        store_operand(k.out + it * 8 * ld, v);
    }
    __device__ __forceinline__ void operator()(int64_t r, int c, float (&v)[8], const Loads& l) const {
        Cursor k;
        open(k, r, c);
        finish<true>(k, 0, v, l);
    }
};

// B = b A + c A^2, from the accumulated square of the stored A.
struct EpiB {
    const f16_bits* a; f16_bits* out; int64_t ld; int32_t m; const float* diag_a; float* diag_b;
    static constexpr bool kRows = false;
    struct Loads { uint4 a; float d; };
    struct Cursor { float f[8]; int64_t at; int rows, off; };
    __device__ __forceinline__ bool outside(int64_t r, int c) const { return r >= m || c >= m; }
    __device__ __forceinline__ void open(Cursor& k, int64_t r, int c) const {
        k.rows = outside(r, c) ? 0 : int(m - r);
        k.at = r * ld + c;
        k.off = int(r) - c;
#pragma unroll
        for (int i = 0; i < 8; ++i) k.f[i] = kNsB;
        if (diag_a && k.rows > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < m) k.f[i] = fmaf(kNsC, diag_a[c + i], kNsB);
        }
    }
    __device__ __forceinline__ void fetch(const Cursor& k, int it, Loads& l) const {
        if (it * 8 >= k.rows) return;
        l.a = *reinterpret_cast<const uint4*>(a + k.at + it * 8 * ld);
        l.d = diag_a ? diag_a[m - k.rows + it * 8] : 0.f;
    }
    __device__ __forceinline__ void load(int64_t r, int c, Loads& l) const {
        if (outside(r, c)) return;
        l.a = *reinterpret_cast<const uint4*>(a + r * ld + c);
        l.d = diag_a ? diag_a[r] : 0.f;
    }
    template <bool STORE>
    __device__ __forceinline__ void finish(const Cursor& k, int it, float (&v)[8], const Loads& l) const {
        if (it * 8 >= k.rows) return;
        float o[8];
        widen_operand(l.a, o);
        const int on = k.off + it * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float sq = kNsC * (v[i] * (kUnscale * kUnscale));
            v[i] = fmaf(fmaf(kNsC, l.d, k.f[i]), o[i], sq);
            if (diag_a && i == on) {
                diag_b[m - k.rows + it * 8] = fmaf(fmaf(kNsC, l.d, kNsB), l.d, sq);
                v[i] = 0.f;
            }
        }
        store_operand(out + k.at + it * 8 * ld, v);
    }
    __device__ __forceinline__ void operator()(int64_t r, int c, float (&v)[8], const Loads& l) const {
        Cursor k;
        open(k, r, c);
        finish<true>(k, 0, v, l);
    }
};

// X = a X + B X (RIGHT: a X + X B), or the update in the last step.
template <bool RIGHT>
struct EpiX {
    float* x32; f16_bits* x16; int64_t ldx;
    const float* inverse;                      // first step: x32 holds U
    const float* diag_b;
    bf16_bits* update; int64_t ldu; int32_t vec_u; float scale;
    int64_t R; int32_t C;
    static constexpr bool kRows = false;
    struct Loads { float4 lo, hi; };
    // what a lane's eight columns share down the rows
    struct Cursor { float f[8]; float norm; int64_t at; bf16_bits* update; const float* diag; int rows, count; };
    __device__ __forceinline__ void open(Cursor& k, int64_t r, int c) const {
        k.count = min(8, C - c);
        k.rows = k.count > 0 && r < R ? int(min(R - r, int64_t(64))) : 0;
        if (k.rows == 0) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) k.f[i] = kNsA + (RIGHT && diag_b && i < k.count ? diag_b[c + i] : 0.f);
        k.norm = inverse ? *inverse : 1.f;
        k.at = r * ldx + c;
        k.update = update + r * ldu + c;
        k.diag = !RIGHT && diag_b ? diag_b + r : nullptr;
    }
    __device__ __forceinline__ void fetch(const Cursor& k, int it, Loads& l) const {
        if (it * 8 >= k.rows) return;
        const float4* p = reinterpret_cast<const float4*>(x32 + k.at + it * 8 * ldx);
        l.lo = p[0];
        l.hi = p[1];
    }
    template <bool STORE>
    __device__ __forceinline__ void finish(const Cursor& k, int it, float (&v)[8], const Loads& l) const {
        if (it * 8 >= k.rows) return;
        const float x[8] = {l.lo.x, l.lo.y, l.lo.z, l.lo.w, l.hi.x, l.hi.y, l.hi.z, l.hi.w};
        const float row = k.diag ? k.diag[it * 8] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(k.f[i] + row, x[i] * k.norm, v[i] * (kUnscale * kUnscale));
        if (update) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= scale;
            bf16_bits* p = k.update + it * 8 * ldu;
            if (vec_u && k.count == 8) {
                store_vec<8>(p, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < k.count) store_f32(p + i, v[i]);
            }
        } else {
            const int64_t at = k.at + it * 8 * ldx;
            store_vec<8>(x32 + at, v);
            store_operand(x16 + at, v);
        }
    }
    __device__ __forceinline__ bool outside(int64_t r, int c) const { return r >= R || c >= C; }
    __device__ __forceinline__ void load(int64_t r, int c, Loads& l) const {
        if (outside(r, c)) return;
        const float4* p = reinterpret_cast<const float4*>(x32 + r * ldx + c);
        l.lo = p[0];
        l.hi = p[1];
    }
    __device__ __forceinline__ void operator()(int64_t r, int c, float (&v)[8], const Loads& l) const {
        Cursor k;
        open(k, r, c);
        finish<true>(k, 0, v, l);
    }
};

struct MuonWs {
    float* x32; f16_bits* x16[2]; f16_bits* a; f16_bits* b;
    float* diag_a; float* diag_b; float* inverse; double* partial;
    int64_t ldx, lda;
    size_t bytes;
};
MuonWs muon_carve(void* ws, int64_t R, int32_t C) {
    MuonWs w;
    const int64_t m = R < C ? R : C;
    // rows of whole 128-byte lines: at a pitch of 6000 bytes the tensor copies' 128-byte rows straddle two
    // lines each, and the products of a 3000 x 3000 matrix take 2.3 times as long
    w.ldx = (int64_t(C) + 63) / 64 * 64;
    w.lda = (m + 63) / 64 * 64;
    char* p = static_cast<char*>(ws);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* q = p + at;
        at += align_up(bytes, kWsAlign);
        return q;
    };
    w.x32 = reinterpret_cast<float*>(take(size_t(R) * w.ldx * 4));
    w.x16[0] = reinterpret_cast<f16_bits*>(take(size_t(R) * w.ldx * 2));
    w.x16[1] = reinterpret_cast<f16_bits*>(take(size_t(R) * w.ldx * 2));
    w.a = reinterpret_cast<f16_bits*>(take(size_t(m) * w.lda * 2));
    w.b = reinterpret_cast<f16_bits*>(take(size_t(m) * w.lda * 2));
    w.diag_a = reinterpret_cast<float*>(take(size_t(m) * 4));
    w.diag_b = reinterpret_cast<float*>(take(size_t(m) * 4));
    w.inverse = reinterpret_cast<float*>(take(4));
    w.partial = reinterpret_cast<double*>(take(kMuonMaxBlocks * sizeof(double)));
    w.bytes = at;
    return w;
}

template <class T>
int muon_prepare(const PrepareArgs& a, bool vec, int* parts, cudaStream_t s) {
    const int run = vec ? 32 * 8 : 32 * 4;        // elements per warp and trip
    const int64_t blocks = (a.R * ((a.C + run - 1) / run) + kMuonThreads / 32 - 1) / (kMuonThreads / 32);
    *parts = int(blocks < kMuonMaxBlocks ? blocks : kMuonMaxBlocks);
    auto kernel = vec ? muon_prepare_kernel<T, 8> : muon_prepare_kernel<T, 1>;
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(unsigned(*parts)), dim3(kMuonThreads), 0, s, a));
    return TPPO_OK;
}

}  // namespace

size_t muon_workspace_bytes(int64_t R, int32_t C) {
    return R < 1 || C < 1 || R > kDenseMaxSize || C > kDenseMaxSize ? 0 : muon_carve(nullptr, R, C).bytes;
}

}  // namespace tppo

using namespace tppo;

TPPO_API int tppo_muon_orthogonalize(const void* grad, int32_t grad_dtype, int64_t ldg, float* momentum, int64_t ldm,
                                     int64_t R, int32_t C, float mu, int32_t nesterov, float eps, int32_t steps, float scale,
                                     void* update, int64_t ldu, int32_t* status, void* workspace, size_t workspace_bytes,
                                     void* stream) {
    if (R < 0 || C < 1 || ldg < C || ldu < C || (momentum && ldm < C) || steps < 1 || steps > 16 ||
        !(eps >= 0.f) || !is_finite_host(eps) || !(fabsf(scale) <= 1e38f) || (momentum && !is_finite_host(mu)) ||
        (grad_dtype != TPPO_BF16 && grad_dtype != TPPO_F32))
        return TPPO_ERR_INVALID_ARG;
    if (R > kDenseMaxSize || C > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    if (R == 0) return TPPO_OK;
    const size_t gs = grad_dtype == TPPO_F32 ? 4 : 2;
    if (!grad || !update || !aligned(grad, gs) || !aligned(update, 2) || !aligned(momentum, 4) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    const MuonWs w = muon_carve(workspace, R, C);
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < w.bytes) return TPPO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool right = R > C;
    const int64_t m = right ? C : R;

    const PrepareArgs pa{grad, ldg, momentum, ldm, mu, nesterov, w.x32, w.partial, R, C, w.ldx, status};
    const bool vec = C % 8 == 0 && aligned(grad, 16) && (ldg * int64_t(gs)) % 16 == 0 &&
                     (!momentum || (aligned(momentum, 16) && ldm % 4 == 0));
    int parts = 0;
    int rc = grad_dtype == TPPO_F32 ? muon_prepare<float>(pa, vec, &parts, s) : muon_prepare<bf16_bits>(pa, vec, &parts, s);
    if (rc != TPPO_OK) return rc;
    const int64_t vectors = R * w.ldx / 8, blocks = (vectors + kMuonThreads - 1) / kMuonThreads;
    TPPO_CUDA_CHECK(launch_dense(muon_normalise_kernel, dim3(unsigned(blocks < kMuonMaxBlocks ? blocks : kMuonMaxBlocks)),
                                 dim3(kMuonThreads), 0, s, static_cast<const double*>(w.partial), int32_t(parts), eps,
                                 w.x32, w.x16[0], w.inverse, vectors,
                                 stream_link(R * w.ldx)));
    for (int32_t k = 0; k < steps; ++k) {
        const DenseOperand X{w.x16[k % 2], R, C, w.ldx}, A{w.a, m, m, w.lda}, B{w.b, m, m, w.lda};
        const bool apart = m <= 64 || k >= steps - 3, last = k == steps - 1;
        const EpiA ea{w.a, w.lda, int32_t(m), apart ? w.diag_a : nullptr};
        const EpiB eb{w.a, w.b, w.lda, int32_t(m), apart ? w.diag_a : nullptr, w.diag_b};
        if (right) rc = dense_product<1, 1, true, true>(X, X, m, m, R, ea, status, s);
        else rc = dense_product<0, 0, true, true>(X, X, m, m, C, ea, status, s);
        if (rc == TPPO_OK) rc = dense_product<0, 0, true, true>(A, A, m, m, m, eb, status, s);
        if (rc != TPPO_OK) return rc;
        bf16_bits* out = last ? static_cast<bf16_bits*>(update) : nullptr;
        const int32_t vec_u = aligned(update, 16) && ldu % 8 == 0;
        const float* inverse = k == 0 ? w.inverse : nullptr;
        const float* diag_b = apart ? w.diag_b : nullptr;
        if (right) {
            const EpiX<true> ex{w.x32, w.x16[(k + 1) % 2], w.ldx, inverse, diag_b, out, ldu, vec_u, scale, R, C};
            rc = dense_product<0, 0, true, false>(X, B, R, C, m, ex, status, s);
        } else {
            const EpiX<false> ex{w.x32, w.x16[(k + 1) % 2], w.ldx, inverse, diag_b, out, ldu, vec_u, scale, R, C};
            rc = dense_product<0, 1, true, false>(B, X, R, C, m, ex, status, s);
        }
        if (rc != TPPO_OK) return rc;
    }
    return TPPO_OK;
}
