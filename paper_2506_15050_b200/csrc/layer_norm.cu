// Layer norm over the rows of a matrix, forward and backward with the reduction of the weight's and
// the bias' gradients:
//     y  = (x - mean) * rstd * gamma + beta,      rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//     dx = rstd * (a - mean(a) - h * mean(a * h)),   h = (x - mean) * rstd,  a = dy * gamma
//     dgamma = sum_rows dy * h,   dbeta = sum_rows dy
// All arithmetic is fp32; the inputs are read once and the outputs rounded once.
//
// Both passes are bound by HBM (2 resp. 3 elements moved per element).  A row lives in the registers
// of a group of threads (one warp for short rows, up to a block for long ones), so mean and centred
// variance are two sweeps over registers, not over memory.  The backward kernel's groups walk the
// rows with a fixed stride and keep the gamma / beta sums of their columns in registers for the whole
// walk; each block writes one partial row to the workspace and a second kernel adds the partial rows
// in a fixed order, so the gradients do not depend on scheduling.  Rows longer than the registers of
// a block hold take kernels that read the row again from L2 instead.
#include "dense_common.cuh"

namespace tppo {
namespace {

constexpr int kNormMaxThreads = 1024;

struct NormFwdArgs {
    const void* x; const void* gamma; const void* beta; void* y;
    float* mean; float* rstd; int32_t* status;
    int64_t M; int32_t N; int64_t ldx, ldy; float eps;
    int32_t group;            // threads per row, a multiple of 32
};

// Sum over the group of `group` threads this thread belongs to.  A group of one warp needs no shared
// memory; otherwise every thread of the block calls this together (`red`: one float per warp).
__device__ __forceinline__ float group_sum(float v, int group, float* red) {
    v = warp_sum(v);
    if (group == 32) return v;
    const int warp = threadIdx.x >> 5, per = group >> 5, first = warp / per * per;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[warp] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return warp_sum(lane < per ? red[first + lane] : 0.f);
}
// Two sums at once.
__device__ __forceinline__ float2 group_sum2(float2 v, int group, float2* red) {
    v.x = warp_sum(v.x);
    v.y = warp_sum(v.y);
    if (group == 32) return v;
    const int warp = threadIdx.x >> 5, per = group >> 5, first = warp / per * per;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[warp] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const float2 w = lane < per ? red[first + lane] : make_float2(0.f, 0.f);
    return make_float2(warp_sum(w.x), warp_sum(w.y));
}

// Element c*group*VEC + t*VEC + i of the row sits in v[c][i] of the group's thread t.
template <class T, class P, int VEC, int CH>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_kernel(const NormFwdArgs a) {
    __shared__ float red[32];
    const int t = threadIdx.x % a.group;
    const int64_t r = int64_t(blockIdx.x) * (blockDim.x / a.group) + threadIdx.x / a.group;
    const bool have = r < a.M;                    // the last block may hold fewer rows
    const T* x = static_cast<const T*>(a.x) + (have ? r : 0) * a.ldx;
    float v[CH][VEC];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * a.group + t) * VEC;
        if (have && col < a.N) {
            load_vec<VEC>(x + col, v[c]);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[c][i];
        }
    }
    const float mean = group_sum(s, a.group, red) / float(a.N);
    s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * a.group + t) * VEC;
        if (have && col < a.N) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] -= mean;
                s = fmaf(v[c][i], v[c][i], s);
            }
        }
    }
    const float var = group_sum(s, a.group, red) / float(a.N);
    const float rstd = rsqrtf(var + a.eps);
    // a NaN or infinity in the row, or a variance outside fp32: no statistics, the row is written 0
    const bool good = is_finite(var) && is_finite(rstd);
    if (!have) return;
    if (t == 0) {
        if (a.mean) a.mean[r] = good ? mean : 0.f;
        if (a.rstd) a.rstd[r] = good ? rstd : 0.f;
        if (!good && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    }
    T* y = static_cast<T*>(a.y) + r * a.ldy;
    const P* gamma = static_cast<const P*>(a.gamma);
    const P* beta = static_cast<const P*>(a.beta);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * a.group + t) * VEC;
        if (col < a.N) {
            float g[VEC], b[VEC];
            if (gamma) load_vec<VEC>(gamma + col, g);
            if (beta) load_vec<VEC>(beta + col, b);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float h = v[c][i] * rstd;
                v[c][i] = good ? fmaf(h, gamma ? g[i] : 1.f, beta ? b[i] : 0.f) : 0.f;
            }
            store_vec<VEC>(y + col, v[c]);
        }
    }
}

// A row of any length: one block, three sweeps (the second and third are served by L2).
template <class T, class P>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_long_kernel(const NormFwdArgs a) {
    __shared__ float red[32];
    const int64_t r = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    float s = 0.f;
    for (int c = threadIdx.x; c < a.N; c += blockDim.x) s += load_f32(x + c);
    const float mean = group_sum(s, blockDim.x, red) / float(a.N);
    s = 0.f;
    for (int c = threadIdx.x; c < a.N; c += blockDim.x) {
        const float d = load_f32(x + c) - mean;
        s = fmaf(d, d, s);
    }
    const float var = group_sum(s, blockDim.x, red) / float(a.N);
    const float rstd = rsqrtf(var + a.eps);
    const bool good = is_finite(var) && is_finite(rstd);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = good ? mean : 0.f;
        if (a.rstd) a.rstd[r] = good ? rstd : 0.f;
        if (!good && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    }
    T* y = static_cast<T*>(a.y) + r * a.ldy;
    const P* gamma = static_cast<const P*>(a.gamma);
    const P* beta = static_cast<const P*>(a.beta);
    for (int c = threadIdx.x; c < a.N; c += blockDim.x) {
        const float h = (load_f32(x + c) - mean) * rstd;
        store_f32(y + c, good ? fmaf(h, gamma ? load_f32(gamma + c) : 1.f, beta ? load_f32(beta + c) : 0.f) : 0.f);
    }
}

struct NormBwdArgs {
    const void* dy; const void* x; const void* gamma;
    const float* mean; const float* rstd;
    void* dx; float* partial;      // [gridDim.x][2][N] (gamma sums, beta sums) or NULL
    int32_t* status;
    int64_t M; int32_t N; int64_t lddy, ldx, lddx;
    int32_t group;
};

template <class T, class P, int VEC, int CH>
__global__ void __launch_bounds__(CH * VEC >= 16 ? 512 : kNormMaxThreads) norm_bwd_kernel(const NormBwdArgs a) {
    extern __shared__ float cols[];               // [2][N], used when a block holds several groups
    __shared__ float2 red[32];
    const int t = threadIdx.x % a.group, grp = threadIdx.x / a.group, groups = blockDim.x / a.group;
    const P* gamma = static_cast<const P*>(a.gamma);
    const float inv_n = 1.f / float(a.N);
    float dg[CH][VEC], db[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dg[c][i] = db[c][i] = 0.f;
    const int64_t step = int64_t(gridDim.x) * groups;
    for (int64_t base = int64_t(blockIdx.x) * groups; base < a.M; base += step) {
        const int64_t r = base + grp;
        const bool have = r < a.M;
        const int64_t rr = have ? r : 0;
        const T* x = static_cast<const T*>(a.x) + rr * a.ldx;
        const T* dy = static_cast<const T*>(a.dy) + rr * a.lddy;
        const float rstd = have ? a.rstd[rr] : 0.f, mean = have ? a.mean[rr] : 0.f;
        float h[CH][VEC], d[CH][VEC], g[CH][VEC];
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * a.group + t) * VEC;
            if (have && col < a.N) {
                load_vec<VEC>(x + col, h[c]);
                load_vec<VEC>(dy + col, d[c]);
                if (gamma) load_vec<VEC>(gamma + col, g[c]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    if (!gamma) g[c][i] = 1.f;
                    h[c][i] = (h[c][i] - mean) * rstd;
                    const float av = d[c][i] * g[c][i];
                    s.x += av;
                    s.y = fmaf(av, h[c][i], s.y);
                }
            }
        }
        s = group_sum2(s, a.group, red);
        const float c1 = s.x * inv_n, c2 = s.y * inv_n;
        // rstd 0 marks a row without statistics; sums that are not finite come from a NaN or an
        // infinity in x or dy: neither kind contributes, its dx is 0
        const bool finite = is_finite(c1) && is_finite(c2) && is_finite(rstd);
        const bool good = finite && rstd != 0.f;
        if (!have) continue;
        if (!finite && t == 0 && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
        T* dx = a.dx ? static_cast<T*>(a.dx) + r * a.lddx : nullptr;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * a.group + t) * VEC;
            if (col < a.N) {
                float o[VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    if (good) {
                        dg[c][i] = fmaf(d[c][i], h[c][i], dg[c][i]);
                        db[c][i] += d[c][i];
                    }
                    o[i] = good ? rstd * (d[c][i] * g[c][i] - c1 - h[c][i] * c2) : 0.f;
                }
                if (dx) store_vec<VEC>(dx + col, o);
            }
        }
    }
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.x) * 2 * a.N;
    // the groups of a block add their columns one after the other: a fixed order
    for (int k = 0; k < groups; ++k) {
        if (grp == k) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * a.group + t) * VEC;
                if (col < a.N) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        float u = dg[c][i], w = db[c][i];
                        if (k > 0) { u += cols[col + i]; w += cols[a.N + col + i]; }
                        if (k < groups - 1) { cols[col + i] = u; cols[a.N + col + i] = w; }
                        else { out[col + i] = u; out[a.N + col + i] = w; }
                    }
                }
            }
        }
        if (groups > 1) __syncthreads();
    }
}

// Rows of any length: dx row by row; `row` keeps (c1, c2) and the row's flag for the column sums.
template <class T, class P>
__global__ void __launch_bounds__(kNormMaxThreads) norm_bwd_long_kernel(const NormBwdArgs a, float* row_flag) {
    __shared__ float2 red[32];
    const int64_t r = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
    const P* gamma = static_cast<const P*>(a.gamma);
    const float rstd = a.rstd[r], mean = a.mean[r];
    float2 s = make_float2(0.f, 0.f);
    for (int c = threadIdx.x; c < a.N; c += blockDim.x) {
        const float av = load_f32(dy + c) * (gamma ? load_f32(gamma + c) : 1.f);
        s.x += av;
        s.y = fmaf(av, (load_f32(x + c) - mean) * rstd, s.y);
    }
    s = group_sum2(s, blockDim.x, red);
    const float c1 = s.x / float(a.N), c2 = s.y / float(a.N);
    const bool finite = is_finite(c1) && is_finite(c2) && is_finite(rstd);
    const bool good = finite && rstd != 0.f;
    if (threadIdx.x == 0) {
        if (row_flag) row_flag[r] = good ? 1.f : 0.f;
        if (!finite && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    }
    if (!a.dx) return;
    T* dx = static_cast<T*>(a.dx) + r * a.lddx;
    for (int c = threadIdx.x; c < a.N; c += blockDim.x) {
        const float av = load_f32(dy + c) * (gamma ? load_f32(gamma + c) : 1.f);
        const float h = (load_f32(x + c) - mean) * rstd;
        store_f32(dx + c, good ? rstd * (av - c1 - h * c2) : 0.f);
    }
}

// Column sums of long rows: one thread per column, blockIdx.y takes every gridDim.y-th row.  Runs
// before the kernel above when dx overwrites dy, after it otherwise -- see the launcher.
template <class T>
__global__ void __launch_bounds__(256) norm_cols_kernel(const NormBwdArgs a, const float* row_flag) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.N) return;
    float dg = 0.f, db = 0.f;
    for (int64_t r = blockIdx.y; r < a.M; r += gridDim.y) {
        if (row_flag[r] == 0.f) continue;
        const float d = load_f32(static_cast<const T*>(a.dy) + r * a.lddy + c);
        const float h = (load_f32(static_cast<const T*>(a.x) + r * a.ldx + c) - a.mean[r]) * a.rstd[r];
        dg = fmaf(d, h, dg);
        db += d;
    }
    float* out = a.partial + int64_t(blockIdx.y) * 2 * a.N;
    out[c] = dg;
    out[a.N + c] = db;
}

// dgamma / dbeta = the sum of `parts` partial rows, in ascending order within each of the 8 strands of
// a column and then over the strands; fp64, rounded once.
template <class P>
__global__ void __launch_bounds__(256) norm_sum_kernel(const float* partial, int32_t parts, int32_t N, P* dgamma,
                                                       P* dbeta) {
    __shared__ double s[8][33];
    pdl_wait();
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int64_t j = int64_t(blockIdx.x) * 32 + lane;           // column of the [2N]-wide partial row
    double t = 0.0;
    if (j < 2 * int64_t(N))
        for (int p = strand; p < parts; p += 8) t += double(partial[int64_t(p) * 2 * N + j]);
    s[strand][lane] = t;
    __syncthreads();
    if (strand == 0 && j < 2 * int64_t(N)) {
        t = 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += s[k][lane];
        if (j < N) { if (dgamma) store_f32(dgamma + j, float(t)); }
        else if (dbeta) store_f32(dbeta + (j - N), float(t));
    }
}

// How a row of N elements is spread: vectors of `vec`, `ch` per thread, `group` threads.
struct NormPlan { int vec, ch, group, groups; };


// Smallest ch of the ladder whose group stays within `limit` threads; ch 0 when none does.
NormPlan norm_plan(int32_t N, int vec, const int* ladder, int rungs, int limit) {
    const int64_t nvec = (int64_t(N) + vec - 1) / vec;
    for (int k = 0; k < rungs; ++k) {
        const int64_t g = ((nvec + ladder[k] - 1) / ladder[k] + 31) / 32 * 32;
        if (g <= limit || (k == rungs - 1 && g <= kNormMaxThreads)) {
            const int group = int(g);
            const int groups = group >= 256 ? 1 : 256 / group;
            return {vec, ladder[k], group, groups};
        }
    }
    return {vec, 0, 0, 0};
}

bool rows_aligned(const void* p, int64_t ld, size_t esize) {
    return aligned(p, 16) && (ld * int64_t(esize)) % 16 == 0;
}

template <class T, class P, int VEC, int CH>
int norm_fwd_launch(const NormFwdArgs& a, const NormPlan& p, cudaStream_t s) {
    const int64_t blocks = (a.M + p.groups - 1) / p.groups;
    norm_fwd_kernel<T, P, VEC, CH><<<unsigned(blocks), p.group * p.groups, 0, s>>>(a);
    TPPO_CUDA_CHECK(cudaGetLastError());
    return TPPO_OK;
}

template <class T, class P>
int norm_fwd_typed(NormFwdArgs a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = a.N % V == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.y, a.ldy, sizeof(T)) &&
                     (!a.gamma || aligned(a.gamma, 16)) && (!a.beta || aligned(a.beta, 16));
    static const int ladder_v[] = {1, 2, 4}, ladder_s[] = {4, 16};
    const NormPlan p = vec ? norm_plan(a.N, V, ladder_v, 3, 320) : norm_plan(a.N, 1, ladder_s, 2, 512);
    a.group = p.group;
    if (p.ch == 0) {
        norm_fwd_long_kernel<T, P><<<unsigned(a.M), kNormMaxThreads, 0, s>>>(a);
        TPPO_CUDA_CHECK(cudaGetLastError());
        return TPPO_OK;
    }
    if (vec) {
        if (p.ch == 1) return norm_fwd_launch<T, P, V, 1>(a, p, s);
        if (p.ch == 2) return norm_fwd_launch<T, P, V, 2>(a, p, s);
        return norm_fwd_launch<T, P, V, 4>(a, p, s);
    }
    if (p.ch == 4) return norm_fwd_launch<T, P, 1, 4>(a, p, s);
    return norm_fwd_launch<T, P, 1, 16>(a, p, s);
}

constexpr int kNormMaxParts = 4 * kNumSms;

struct NormWs { float* partial; float* row_flag; size_t bytes; };
NormWs norm_carve(void* ws, int64_t M, int32_t N) {
    const size_t a = align_up(size_t(kNormMaxParts) * 2 * size_t(N) * 4, kWsAlign);
    const size_t b = align_up(size_t(M) * 4, kWsAlign);
    char* p = static_cast<char*>(ws);
    return {reinterpret_cast<float*>(p), reinterpret_cast<float*>(p + a), a + b};
}

template <class T, class P, int VEC, int CH>
int norm_bwd_launch(const NormBwdArgs& a, const NormPlan& p, int* parts, cudaStream_t s) {
    const int threads = p.group * p.groups;
    const int64_t rows = (a.M + p.groups - 1) / p.groups;
    const int per_sm = threads >= 1024 ? 1 : threads >= 512 ? 2 : 4;
    const int64_t most = int64_t(kNumSms) * per_sm;
    const int grid = int(rows < most ? rows : most);
    *parts = grid;
    const size_t smem = p.groups > 1 && a.partial ? size_t(a.N) * 8 : 0;
    norm_bwd_kernel<T, P, VEC, CH><<<grid, threads, smem, s>>>(a);
    TPPO_CUDA_CHECK(cudaGetLastError());
    return TPPO_OK;
}

template <class T, class P>
int norm_bwd_typed(NormBwdArgs a, P* dgamma, P* dbeta, float* row_flag, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = a.N % V == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.dy, a.lddy, sizeof(T)) &&
                     (!a.dx || rows_aligned(a.dx, a.lddx, sizeof(T))) && (!a.gamma || aligned(a.gamma, 16));
    // wide threads (16 sums or more of each kind) keep to 512 threads so that nothing spills
    static const int ladder_b[] = {1, 2}, ladder_f[] = {2, 4}, ladder_s[] = {4, 16};
    const NormPlan p = vec ? (V == 8 ? norm_plan(a.N, V, ladder_b, 2, 320) : norm_plan(a.N, V, ladder_f, 2, 320))
                           : norm_plan(a.N, 1, ladder_s, 2, 512);
    a.group = p.group;
    int rc = TPPO_OK, parts = 0;
    if (p.ch == 0 || (p.ch * p.vec >= 16 && p.group > 512)) {
        // the column sums read dy, which dx may overwrite: statistics and flags first, then the sums,
        // then dx
        NormBwdArgs b = a;
        if (a.partial) {
            b.dx = nullptr;
            norm_bwd_long_kernel<T, P><<<unsigned(a.M), kNormMaxThreads, 0, s>>>(b, row_flag);
            TPPO_CUDA_CHECK(cudaGetLastError());
            parts = int(a.M < 64 ? a.M : 64);
            norm_cols_kernel<T><<<dim3((a.N + 255) / 256, parts), 256, 0, s>>>(a, row_flag);
            TPPO_CUDA_CHECK(cudaGetLastError());
        }
        if (a.dx) {
            norm_bwd_long_kernel<T, P><<<unsigned(a.M), kNormMaxThreads, 0, s>>>(a, nullptr);
            TPPO_CUDA_CHECK(cudaGetLastError());
        }
    } else if (vec) {
        if (V == 8) rc = p.ch == 1 ? norm_bwd_launch<T, P, V, 1>(a, p, &parts, s) : norm_bwd_launch<T, P, V, 2>(a, p, &parts, s);
        else rc = p.ch == 2 ? norm_bwd_launch<T, P, V, 2>(a, p, &parts, s) : norm_bwd_launch<T, P, V, 4>(a, p, &parts, s);
    } else {
        rc = p.ch == 4 ? norm_bwd_launch<T, P, 1, 4>(a, p, &parts, s) : norm_bwd_launch<T, P, 1, 16>(a, p, &parts, s);
    }
    if (rc != TPPO_OK || !a.partial) return rc;
    TPPO_CUDA_CHECK(launch_dense(norm_sum_kernel<P>, dim3(unsigned((2 * int64_t(a.N) + 31) / 32)), dim3(256), 0, s, true,
                                 static_cast<const float*>(a.partial), int32_t(parts), a.N, dgamma, dbeta));
    return TPPO_OK;
}

bool type_known(int32_t t) { return t == TPPO_BF16 || t == TPPO_F32; }
size_t type_size(int32_t t) { return t == TPPO_BF16 ? 2 : 4; }

}  // namespace

size_t norm_workspace_bytes(int64_t M, int32_t N) { return N < 1 ? 0 : norm_carve(nullptr, M, N).bytes; }

}  // namespace tppo

using namespace tppo;

TPPO_API int tppo_layer_norm_fwd(const void* x, int32_t dtype, int64_t M, int32_t N, int64_t ldx, const void* gamma,
                                 const void* beta, int32_t param_dtype, float eps, void* y, int64_t ldy, float* mean,
                                 float* rstd, int32_t* status, void* stream) {
    if (M < 0 || N < 1 || M > 0x7fffffffll || ldx < N || ldy < N || !(eps >= 0.f) || !is_finite_host(eps))
        return TPPO_ERR_INVALID_ARG;
    if (!type_known(dtype) || ((gamma || beta) && !type_known(param_dtype))) return TPPO_ERR_INVALID_ARG;
    if (M == 0) return TPPO_OK;
    if (!x || !y) return TPPO_ERR_INVALID_ARG;
    const size_t es = type_size(dtype), ps = type_size(param_dtype);
    if (!aligned(x, es) || !aligned(y, es) || !aligned(gamma, ps) || !aligned(beta, ps) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    const NormFwdArgs a{x, gamma, beta, y, mean, rstd, status, M, N, ldx, ldy, eps, 0};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == TPPO_BF16)
        return param_dtype == TPPO_F32 ? norm_fwd_typed<bf16_bits, float>(a, s) : norm_fwd_typed<bf16_bits, bf16_bits>(a, s);
    return param_dtype == TPPO_F32 ? norm_fwd_typed<float, float>(a, s) : norm_fwd_typed<float, bf16_bits>(a, s);
}

TPPO_API int tppo_layer_norm_bwd(const void* dy, const void* x, int32_t dtype, int64_t M, int32_t N, int64_t lddy,
                                 int64_t ldx, const void* gamma, int32_t param_dtype, const float* mean,
                                 const float* rstd, void* dx, int64_t lddx, void* dgamma, void* dbeta, int32_t* status,
                                 void* workspace, size_t workspace_bytes, void* stream) {
    const bool params = dgamma || dbeta;
    if (M < 0 || N < 1 || M > 0x7fffffffll || lddy < N || ldx < N || (dx && lddx < N)) return TPPO_ERR_INVALID_ARG;
    if (!type_known(dtype) || ((gamma || params) && !type_known(param_dtype))) return TPPO_ERR_INVALID_ARG;
    if (M > 0 && (!dy || !x || !mean || !rstd)) return TPPO_ERR_INVALID_ARG;
    const size_t es = type_size(dtype), ps = type_size(param_dtype);
    if (!aligned(dy, es) || !aligned(x, es) || !aligned(dx, es) || !aligned(gamma, ps) || !aligned(dgamma, ps) ||
        !aligned(dbeta, ps) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    NormWs w = norm_carve(workspace, M, N);
    if (params && (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < w.bytes)) return TPPO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (M == 0) {                                  // no rows: the sums are empty
        if (dgamma) TPPO_CUDA_CHECK(cudaMemsetAsync(dgamma, 0, size_t(N) * ps, s));
        if (dbeta) TPPO_CUDA_CHECK(cudaMemsetAsync(dbeta, 0, size_t(N) * ps, s));
        return TPPO_OK;
    }
    if (!dx && !params) return TPPO_OK;
    const NormBwdArgs a{dy, x, gamma, mean, rstd, dx, params ? w.partial : nullptr, status, M, N, lddy, ldx, lddx, 0};
    if (dtype == TPPO_BF16) {
        if (param_dtype == TPPO_F32)
            return norm_bwd_typed<bf16_bits, float>(a, static_cast<float*>(dgamma), static_cast<float*>(dbeta), w.row_flag, s);
        return norm_bwd_typed<bf16_bits, bf16_bits>(a, static_cast<bf16_bits*>(dgamma), static_cast<bf16_bits*>(dbeta), w.row_flag, s);
    }
    if (param_dtype == TPPO_F32)
        return norm_bwd_typed<float, float>(a, static_cast<float*>(dgamma), static_cast<float*>(dbeta), w.row_flag, s);
    return norm_bwd_typed<float, bf16_bits>(a, static_cast<bf16_bits*>(dgamma), static_cast<bf16_bits*>(dbeta), w.row_flag, s);
}
