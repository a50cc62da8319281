// Forward pass of the residual join; see residual_norm.cuh.
#include "residual_norm.cuh"

namespace tppo {
namespace {

template <class T, int E, bool GATED, bool SHIFT>
__global__ void __launch_bounds__(join_threads(E), 1) join_fwd_kernel(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef JoinThread<T, E, SHIFT, join_fwd_regs(E), kFwdIn> Thread;
    constexpr int VEC = Thread::VEC, CH = Thread::CH;
    Thread th(a, smem);
    pdl_launch();
    pdl_wait();
    for (int s = 0; s < a.stages; ++s) th.fetch(a, th.row + s * th.step, th.stage_at(a, s));
    th.load_params(a, smem);
    __syncthreads();
    const bool post = a.norms & TPPO_NORM_POST, pre = a.norms & TPPO_NORM_PRE;
    const float inv = 1.f / float(a.N);
    int turn = 0;
    uint32_t stage = th.stage_at(a, 0);
    for (int64_t r = th.row; r < a.M; r += th.step) {
        th.land(a, stage);
        float r1 = 1.f, s[1];
        bool good = true;
        if (post) {
            float q[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!th.k.any(c)) continue;
                float z[VEC];
                join_piece<T>(th.at(a, stage, kZ, c), z);
#pragma unroll
                for (int i = 0; i < VEC; ++i) q[i & 1] = fmaf(z[i], z[i], q[i & 1]);
            }
            s[0] = q[0] + q[1];
            th.sum(s);
            r1 = join_rstd(s[0], inv, a.eps, good);
        }
        float h[CH][VEC], q[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!th.k.any(c)) continue;
            float z[VEC], g[VEC];
            join_piece<T>(th.at(a, stage, kZ, c), z);
            join_piece<T>(th.at(a, stage, kRes, c), h[c]);
            th.post(a, c, g);
            if (GATED) {
                float w[VEC];
                join_piece<T>(th.at(a, stage, kGate, c), w);
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[c][i] = fmaf(z[i] * r1, g[i], a.alpha * h[c][i]);
            if (pre) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) q[i & 1] = fmaf(h[c][i], h[c][i], q[i & 1]);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) q[i & 1] += fabsf(h[c][i]);
            }
        }
        th.fetch(a, r + a.stages * th.step, stage);
        if (++turn == a.stages) turn = 0;
        stage = th.stage_at(a, turn);
        s[0] = q[0] + q[1];
        th.sum(s);
        const float r2 = pre ? join_rstd(s[0], inv, a.eps, good) : 1.f;
        good = good && is_finite(s[0]);
        if (th.t == 0) {
            if (a.r_post) a.r_post[r] = good ? r1 : 0.f;
            if (a.r_pre) a.r_pre[r] = good ? r2 : 0.f;
            if (!good && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
        }
        T *ho = th.out(a, 0, r), *no = th.out(a, 1, r);
        if (!good) {                                      // the same for the whole group
            th.store_zeros(ho);
            if (pre) th.store_zeros(no);
            continue;
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!th.k.any(c)) continue;
            join_store<T>(th.k, c, ho, h[c]);
            if (pre) {
                float g[VEC];
                th.pre(a, c, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] *= h[c][i] * r2;
                join_store<T>(th.k, c, no, g);
            }
        }
    }
}

// ---- any length and alignment: one block per row, swept once per sum -----------------------------------------
template <class T>
__global__ void __launch_bounds__(kJoinAnyThreads) join_fwd_any_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float red[32];
    pdl_launch();
    pdl_wait();
    const bool post = a.norms & TPPO_NORM_POST, pre = a.norms & TPPO_NORM_PRE;
    const float inv = 1.f / float(a.N);
    for (int64_t r = blockIdx.x; r < a.M; r += gridDim.x) {
        const T* z = static_cast<const T*>(a.in[kZ]) + r * a.ld[kZ];
        const T* res = static_cast<const T*>(a.in[kRes]) + r * a.ld[kRes];
        const T* gate = a.in[kGate] ? static_cast<const T*>(a.in[kGate]) + r * a.ld[kGate] : nullptr;
        T* ho = static_cast<T*>(a.out[0]) + r * a.ldo[0];
        T* no = pre ? static_cast<T*>(a.out[1]) + r * a.ldo[1] : nullptr;
        float r1 = 1.f, s[1] = {0.f};
        bool good = true;
        if (post) {
#pragma unroll 4
            for (int c = threadIdx.x; c < a.N; c += kJoinAnyThreads) s[0] = fmaf(load_f32(z + c), load_f32(z + c), s[0]);
            block_sums(s, red);
            r1 = join_rstd(s[0], inv, a.eps, good);
        }
        auto join = [&](int c) {
            float g = param(a.gate_row, c, a.p32) * param(a.gamma_post, c, a.p32);
            if (gate) g *= load_f32(gate + c);
            return fmaf(load_f32(z + c) * r1, g, a.alpha * load_f32(res + c));
        };
        s[0] = 0;
#pragma unroll 4
        for (int c = threadIdx.x; c < a.N; c += kJoinAnyThreads) {
            const float h = join(c);
            s[0] = pre ? fmaf(h, h, s[0]) : s[0] + fabsf(h);
        }
        block_sums(s, red);
        const float r2 = pre ? join_rstd(s[0], inv, a.eps, good) : 1.f;
        good = good && is_finite(s[0]);
        if (threadIdx.x == 0) {
            if (a.r_post) a.r_post[r] = good ? r1 : 0.f;
            if (a.r_pre) a.r_pre[r] = good ? r2 : 0.f;
            if (!good && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
        }
        // h or n may be z or residual: an element is read before it is written, by the same thread
#pragma unroll 4
        for (int c = threadIdx.x; c < a.N; c += kJoinAnyThreads) {
            const float h = join(c);
            store_f32(ho + c, good ? h : 0.f);
            if (pre) store_f32(no + c, good ? h * r2 * param(a.gamma_pre, c, a.p32) : 0.f);
        }
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
template <class T, int E>
int launch_fwd(const JoinArgs& a, const JoinPlan& p, cudaStream_t s) {
    auto kernel = a.in[kGate] ? (p.shift ? join_fwd_kernel<T, E, true, true> : join_fwd_kernel<T, E, true, false>)
                              : (p.shift ? join_fwd_kernel<T, E, false, true> : join_fwd_kernel<T, E, false, false>);
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kJoinSmem));
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(p.grid), dim3(a.T * a.groups), p.smem, s, a));
    return TPPO_OK;
}
template <class T>
int run_fwd(JoinArgs& a, bool same, cudaStream_t s) {
    constexpr int vec = Join<T>::VEC;
    JoinPlan p;
    if (same) {
        const int64_t width = join_width(a, p, vec);
        join_choose(a, p, {8, 16, 40, 32}, vec, width, false);
    }
    switch (p.E) {
        case 8: return launch_fwd<T, 8>(a, p, s);
        case 16: return launch_fwd<T, 16>(a, p, s);
        case 32: return launch_fwd<T, 32>(a, p, s);
        case 40: return launch_fwd<T, 40>(a, p, s);
    }
    const int grid = int(a.M < kJoinAnyBlocks ? a.M : kJoinAnyBlocks);
    TPPO_CUDA_CHECK(launch_dense(join_fwd_any_kernel<T>, dim3(grid), dim3(kJoinAnyThreads), 0, s, a));
    return TPPO_OK;
}

}  // namespace
}  // namespace tppo

TPPO_API int tppo_residual_norm_fwd(const void* z, int64_t ldz, const void* residual, int64_t ldr, const void* gate, int64_t ldg,
                                    int32_t dtype, int64_t M, int32_t N, const void* gamma_post, const void* gamma_pre,
                                    int32_t param_dtype, float alpha, float eps, int32_t norms, void* h, int64_t ldh, void* n, int64_t ldn,
                                    float* rstd_post, float* rstd_pre, int32_t* status, void* stream) {
    using namespace tppo;
    if (M < 0 || N < 1 || !type_ok(dtype) || !type_ok(param_dtype) || (norms & ~3) || !is_finite_host(alpha) || !(eps >= 0.f) ||
        !is_finite_host(eps))
        return TPPO_ERR_INVALID_ARG;
    const bool post = norms & TPPO_NORM_POST, pre = norms & TPPO_NORM_PRE;
    const bool full = gate && ldg != 0;
    if ((n != nullptr) != pre && M > 0) return TPPO_ERR_INVALID_ARG;
    if ((gamma_post && !post) || (gamma_pre && !pre) || (rstd_post && !post) || (rstd_pre && !pre)) return TPPO_ERR_INVALID_ARG;
    if (ldz < N || ldr < N || ldh < N || (pre && ldn < N) || (full && ldg < N)) return TPPO_ERR_INVALID_ARG;
    const size_t e = size_of(dtype), pe = size_of(param_dtype);
    if (!aligned(z, e) || !aligned(residual, e) || !aligned(h, e) || !aligned(n, e) || !aligned(gate, full ? e : pe) ||
        !aligned(gamma_post, pe) || !aligned(gamma_pre, pe) || !aligned(rstd_post, 4) || !aligned(rstd_pre, 4) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    if (M > 0 && (!z || !residual || !h)) return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || N > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    if (M == 0) return TPPO_OK;
    JoinArgs a{};
    a.in[kZ] = z; a.in[kRes] = residual; a.in[kGate] = full ? gate : nullptr;
    a.ld[kZ] = ldz; a.ld[kRes] = ldr; a.ld[kGate] = ldg;
    a.slot[kRes] = 1; a.slot[kGate] = 2;
    a.arrays = full ? 3 : 2;
    a.gate_row = full ? nullptr : gate;
    a.gamma_post = gamma_post; a.gamma_pre = gamma_pre; a.p32 = param_dtype == TPPO_F32;
    a.out[0] = h; a.out[1] = n; a.ldo[0] = ldh; a.ldo[1] = ldn;
    a.r_post = rstd_post; a.r_pre = rstd_pre; a.status = status;
    a.M = M; a.N = N; a.alpha = alpha; a.eps = eps; a.norms = norms;
    a.shift_step = int32_t(ldz % 16);
    a.one_ld = ldr == ldz && ldh == ldz && (!pre || ldn == ldz) && (!full || ldg == ldz);
    const bool same = same_start(z, ldz, residual, ldr, e) && same_start(z, ldz, a.in[kGate], ldg, e) && same_start(z, ldz, h, ldh, e) &&
                      same_start(z, ldz, n, ldn, e);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == TPPO_F32 ? run_fwd<float>(a, same, s) : run_fwd<bf16_bits>(a, same, s);
}
