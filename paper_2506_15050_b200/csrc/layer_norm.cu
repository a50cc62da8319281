// Layer norm over the rows of a matrix, forward and backward with the reduction of the weight's and
// the bias' gradients:
//     y  = (x - mean) * rstd * gamma + beta,      rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//     dx = rstd * (a - mean(a) - h * mean(a * h)),   h = (x - mean) * rstd,  a = dy * gamma
//     dgamma = sum_rows dy * h,   dbeta = sum_rows dy
// All arithmetic is fp32; the inputs are read once and the outputs rounded once.
//
// Both passes are bound by HBM (2 resp. 3 elements moved per element).  Forward, a row lives in the
// registers of a few warps as the 16-byte pieces it was loaded in, so mean and centred variance are two
// sweeps over registers.  Backward, the sums of gamma and beta want few columns per thread, so a row is spread
// over a block; aligned rows are fed by bulk (TMA) copies through a shared-memory ring, which keeps
// ~100 KB per block in flight while the block goes from row to row with one barrier each, and other
// rows are loaded into registers some rows at a time.  Each block writes one partial row of column
// sums to the workspace and a second kernel adds them in a fixed order, so the gradients do not depend
// on scheduling.  Rows too long for either take kernels that read the row again from L2.
#include <type_traits>

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

// One 16-byte piece of a row as loaded, or one widened element (VEC 1).
template <class T, int VEC> struct Piece {
    uint4 w;
    __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ float get(int i) const {
        const uint32_t u = VEC == 8 ? (i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w) : (i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w);
        return VEC == 8 ? (i % 2 ? bf16_hi(u) : bf16_lo(u)) : __uint_as_float(u);
    }
};
template <class T> struct Piece<T, 1> {
    float w;
    __device__ __forceinline__ void load(const T* p) { w = load_f32(p); }
    __device__ __forceinline__ float get(int) const { return w; }
};

// VEC parameters, `otherwise` where there are none.
template <int VEC, class P>
__device__ __forceinline__ void load_params(const P* p, int col, float otherwise, float (&v)[VEC]) {
    if (p) { load_vec<VEC>(p + col, v); return; }
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = otherwise;
}

// Sum over the group of `group` threads this thread belongs to.  A group is one warp, or the whole
// block, whose threads then call this together (`red`: one float per warp).
__device__ __forceinline__ float group_sum(float v, int group, float* red) {
    v = warp_sum(v);
    if (group == 32) return v;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();                              // the previous sum has been read
    if (lane == 0) red[warp] = v;
    __syncthreads();
    return warp_sum(lane < (group >> 5) ? red[lane] : 0.f);
}

// Element (c * group + t) * VEC + i of the row sits in piece c of the group's thread t.
template <class T, class P, int VEC, int CH>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_kernel(const NormFwdArgs a) {
    __shared__ float red[32];
    pdl_launch();
    pdl_wait();
    const int t = threadIdx.x % a.group;
    const int64_t r = int64_t(blockIdx.x) * (blockDim.x / a.group) + threadIdx.x / a.group;
    const bool have = r < a.M;                    // the last block may hold fewer rows than warps
    const T* x = static_cast<const T*>(a.x) + (have ? r : 0) * a.ldx;
    Piece<T, VEC> raw[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * a.group + t) * VEC;
        if (have && col < a.N) raw[c].load(x + col);
    }
    // widened once: unpacking again in every sweep costs more issue slots than the arithmetic
    float v[CH][VEC], s[2] = {0.f, 0.f};            // two chains of additions
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (have && (c * a.group + t) * VEC < a.N) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] = raw[c].get(i);
                s[(c + i) & 1] = s[(c + i) & 1] + v[c][i];
            }
        }
    }
    const float mean = group_sum(s[0] + s[1], a.group, red) / float(a.N);
    s[0] = s[1] = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (have && (c * a.group + t) * VEC < a.N) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[c][i] = v[c][i] - mean;
                s[(c + i) & 1] = fmaf(v[c][i], v[c][i], s[(c + i) & 1]);
            }
        }
    }
    const float var = group_sum(s[0] + s[1], a.group, red) / float(a.N);
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
    if (!good) {
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0;
        for (int col = t * VEC; col < a.N; col += a.group * VEC) store_vec<VEC>(y + col, zero);
        return;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * a.group + t) * VEC;
        if (col < a.N) {
            float g[VEC], b[VEC];
            load_params<VEC>(gamma, col, 1.f, g);
            load_params<VEC>(beta, col, 0.f, b);
#pragma unroll
            for (int i = 0; i < VEC; ++i) b[i] = fmaf(v[c][i] * rstd, g[i], b[i]);
            store_vec<VEC>(y + col, b);
        }
    }
}

// A row of any length: one block, three sweeps (the second and third are served by L2).
template <class T, class P>
__global__ void __launch_bounds__(kNormMaxThreads) norm_fwd_long_kernel(const NormFwdArgs a) {
    __shared__ float red[32];
    pdl_launch();
    pdl_wait();
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
    int32_t stages;                // ring kernel
};

// The threads' share of one row.  With e = x - mean, k = sum(a e) / N * rstd^2 and q = -rstd sum(a) / N:
//     dx = rstd a + q - (rstd k) e,   dgamma += dy (e rstd),   dbeta += dy
// e is formed twice from the pieces instead of being kept in registers.
template <class T, class P, int VEC, int CH> struct NormRow {
    Piece<T, VEC> x[CH], d[CH];

    // (sum of a, sum of a * (x - mean))
    __device__ __forceinline__ float2 sums(const NormBwdArgs& a, int t, float mean) const {
        const P* gamma = static_cast<const P*>(a.gamma);
        float s[2] = {0.f, 0.f}, q[2] = {0.f, 0.f};      // two chains of additions each
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * a.group + t) * VEC;
            if (col < a.N) {
                float g[VEC];
                load_params<VEC>(gamma, col, 1.f, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float av = d[c].get(i) * g[i];
                    s[i & 1] += av;
                    q[i & 1] = fmaf(av, x[c].get(i) - mean, q[i & 1]);
                }
            }
        }
        return make_float2(s[0] + s[1], q[0] + q[1]);
    }
    __device__ __forceinline__ void finish(const NormBwdArgs& a, int t, int64_t r, float mean, float rstd, float c1, float c2, bool good,
                                           float (&dg)[CH][VEC], float (&db)[CH][VEC]) const {
        const P* gamma = static_cast<const P*>(a.gamma);
        T* dx = a.dx ? static_cast<T*>(a.dx) + r * a.lddx : nullptr;
        if (!good) {
            float zero[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) zero[i] = 0;
            if (dx)
                for (int col = t * VEC; col < a.N; col += a.group * VEC) store_vec<VEC>(dx + col, zero);
            return;
        }
        const float q = -rstd * c1, k = -rstd * c2;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * a.group + t) * VEC;
            if (col < a.N) {
                float g[VEC];
                load_params<VEC>(gamma, col, 1.f, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float dv = d[c].get(i), h = (x[c].get(i) - mean) * rstd;
                    dg[c][i] = fmaf(dv, h, dg[c][i]);
                    db[c][i] += dv;
                    g[i] = fmaf(dv * g[i], rstd, fmaf(h, k, q));
                }
                if (dx) store_vec<VEC>(dx + col, g);
            }
        }
    }
};

// Sums over a warp of V values per lane (V a power of two up to 8): lane l ends up with the total of
// value l % V.  Each of the first log2(V) exchanges halves the number of values.
template <int V>
__device__ __forceinline__ float warp_sum_many(float (&v)[V]) {
    const int lane = threadIdx.x & 31;
    int n = V;
#pragma unroll
    for (int o = 1; o < V; o <<= 1) {
        n >>= 1;
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            if (i < n) {
                // values are paired by the bit of their index that this exchange settles
                const float keep = up ? v[2 * i + 1] : v[2 * i], give = up ? v[2 * i] : v[2 * i + 1];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        }
    }
#pragma unroll
    for (int o = V; o < 32; o <<= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
}

// rstd 0 marks a row without statistics; sums that are not finite come from a NaN or an infinity in x
// or dy: neither kind contributes, its dx is 0.
__device__ __forceinline__ bool norm_row_good(float c1, float c2, float rstd, bool first, int32_t* status) {
    const bool finite = is_finite(c1) && is_finite(c2) && is_finite(rstd);
    if (!finite && first && status) atomicOr(status, TPPO_DEV_NONFINITE);
    return finite && rstd != 0.f;
}

// This thread's column sums into the block's partial row; the groups of a block add theirs one after
// the other: a fixed order.  `cols`: [2][N] shared floats, used with more than one group.
template <int VEC, int CH>
__device__ __forceinline__ void norm_put_partial(const NormBwdArgs& a, int t, int grp, int groups, float* cols,
                                                 const float (&dg)[CH][VEC], const float (&db)[CH][VEC]) {
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.x) * 2 * a.N;
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

// Rows of any alignment, ROWS of a group's rows at a time in registers.
template <class T, class P, int VEC, int CH, int ROWS>
__global__ void __launch_bounds__(512) norm_bwd_kernel(const NormBwdArgs a) {
    constexpr int VALUES = 2 * ROWS;
    extern __shared__ float cols[];
    __shared__ float red[2][16][VALUES];
    pdl_launch();
    pdl_wait();
    const int t = threadIdx.x % a.group, grp = threadIdx.x / a.group, groups = blockDim.x / a.group;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = a.group >> 5, first = warp / per * per;
    const float inv_n = 1.f / float(a.N);
    float dg[CH][VEC], db[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dg[c][i] = db[c][i] = 0;
    const int64_t step = int64_t(gridDim.x) * groups;
    int flip = 0;
    for (int64_t base = int64_t(blockIdx.x) * groups; base < a.M; base += step * ROWS, flip ^= 1) {
        const int64_t r0 = base + grp;
        NormRow<T, P, VEC, CH> row[ROWS];
        float mean[ROWS], rstd[ROWS], s[VALUES];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t r = r0 + k * step;
            mean[k] = rstd[k] = 0.f;
            if (r < a.M) {
                mean[k] = a.mean[r];
                rstd[k] = a.rstd[r];
                const T* x = static_cast<const T*>(a.x) + r * a.ldx;
                const T* dy = static_cast<const T*>(a.dy) + r * a.lddy;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const int col = (c * a.group + t) * VEC;
                    if (col < a.N) {
                        row[k].x[c].load(x + col);
                        row[k].d[c].load(dy + col);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            s[2 * k] = s[2 * k + 1] = 0.f;
            if (r0 + k * step < a.M) {
                const float2 v = row[k].sums(a, t, mean[k]);
                s[2 * k] = v.x;
                s[2 * k + 1] = v.y * rstd[k];
            }
        }
        float total = warp_sum_many<VALUES>(s);               // of value lane % VALUES
        if (per > 1) {
            // one barrier per trip (the groups of a block make the same number of them): the two halves
            // of `red` alternate
            if (lane < VALUES) red[flip][warp][lane] = total;
            __syncthreads();
            total = 0.f;
            for (int w = lane / VALUES; w < per; w += 32 / VALUES) total += red[flip][first + w][lane % VALUES];
#pragma unroll
            for (int o = VALUES; o < 32; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t r = r0 + k * step;
            const float c1 = __shfl_sync(0xffffffffu, total, 2 * k) * inv_n;
            const float c2 = __shfl_sync(0xffffffffu, total, 2 * k + 1) * inv_n;
            if (r < a.M) {
                const bool good = norm_row_good(c1, c2, rstd[k], t == 0, a.status);
                row[k].finish(a, t, r, mean[k], rstd[k], c1, c2, good, dg, db);
            }
        }
    }
    norm_put_partial<VEC, CH>(a, t, grp, groups, cols, dg, db);
}

// Aligned rows: a block per row, x and dy rows brought in by bulk copies `stages` rows ahead.
template <class T, class P, int VEC, int CH>
__global__ void __launch_bounds__(CH * VEC > 16 ? 512 : 640) norm_bwd_ring_kernel(const NormBwdArgs a) {
    extern __shared__ __align__(128) uint8_t ring[];     // [stages][x row, dy row], then one barrier per stage
    __shared__ float red[2][2][32];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, warps = blockDim.x >> 5;
    const uint32_t row_bytes = uint32_t(a.N) * sizeof(T), stage_bytes = 2 * row_bytes;
    const uint32_t base = ptx::smem_addr(ring), full = base + a.stages * stage_bytes;
    const float inv_n = 1.f / float(a.N);
    const int64_t step = gridDim.x;
    auto issue = [&](int64_t r, int s) {
        const uint32_t bar = full + 8 * s, at = base + s * stage_bytes;
        ptx::mbar_arrive_expect_tx(bar, stage_bytes);
        ptx::bulk_load(at, static_cast<const T*>(a.x) + r * a.ldx, row_bytes, bar);
        ptx::bulk_load(at + row_bytes, static_cast<const T*>(a.dy) + r * a.lddy, row_bytes, bar);
    };
    pdl_launch();
    pdl_wait();
    if (t == 0) {
        for (int s = 0; s < a.stages; ++s) ptx::mbar_init(full + 8 * s, 1);
        ptx::fence_mbar_init_cluster();
        for (int s = 0; s < a.stages && blockIdx.x + s * step < a.M; ++s) issue(blockIdx.x + s * step, s);
    }
    __syncthreads();
    float dg[CH][VEC], db[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) dg[c][i] = db[c][i] = 0;
    int stage = 0, flip = 0;
    uint32_t phase = 0;
    bool timed_out = false;
    float next_mean = a.mean[blockIdx.x], next_rstd = a.rstd[blockIdx.x];
    for (int64_t r = blockIdx.x; r < a.M; r += step, flip ^= 1) {
        const float mean = next_mean, rstd = next_rstd;
        if (r + step < a.M) { next_mean = a.mean[r + step]; next_rstd = a.rstd[r + step]; }
        // a wait that ran out is not repeated: the sums are then garbage, and flagged
        if (!timed_out) timed_out = !ptx::mbar_wait<false>(full + 8 * stage, phase);
        NormRow<T, P, VEC, CH> row;
        const uint8_t* at = ring + stage * stage_bytes;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * a.group + t) * VEC;
            if (col < a.N) {
                row.x[c].load(reinterpret_cast<const T*>(at) + col);
                row.d[c].load(reinterpret_cast<const T*>(at + row_bytes) + col);
            }
        }
        const float2 part = row.sums(a, t, mean);
        float s[2] = {part.x, part.y * rstd};
        const float mine = warp_sum_many<2>(s);
        if (lane < 2) red[flip][lane][warp] = mine;
        __syncthreads();                          // the partial sums are there, and the stage has been read
        if (t == 0 && r + a.stages * step < a.M) issue(r + a.stages * step, stage);
        if (++stage == a.stages) { stage = 0; phase ^= 1u; }
        float w[2] = {0.f, 0.f};
        if (lane < warps) { w[0] = red[flip][0][lane]; w[1] = red[flip][1][lane]; }
        const float total = warp_sum_many<2>(w);
        const float c1 = __shfl_sync(0xffffffffu, total, 0) * inv_n, c2 = __shfl_sync(0xffffffffu, total, 1) * inv_n;
        const bool good = norm_row_good(c1, c2, rstd, t == 0, a.status);
        row.finish(a, t, r, mean, rstd, c1, c2, good, dg, db);
    }
    if (timed_out && a.status) atomicOr(a.status, TPPO_DEV_WAIT_TIMEOUT);
    norm_put_partial<VEC, CH>(a, t, 0, 1, nullptr, dg, db);
}

// Rows of any length: dx and, in row_flag, which rows count in the column sums.
template <class T, class P>
__global__ void __launch_bounds__(kNormMaxThreads) norm_bwd_long_kernel(const NormBwdArgs a, float* row_flag) {
    __shared__ float red[32];
    pdl_launch();
    pdl_wait();
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
    const float c1 = group_sum(s.x, blockDim.x, red) / float(a.N), c2 = group_sum(s.y, blockDim.x, red) / float(a.N);
    const bool good = norm_row_good(c1, c2, rstd, threadIdx.x == 0, a.status);
    if (row_flag && threadIdx.x == 0) row_flag[r] = good ? 1.f : 0.f;
    if (!a.dx) return;
    T* dx = static_cast<T*>(a.dx) + r * a.lddx;
    for (int c = threadIdx.x; c < a.N; c += blockDim.x) {
        const float av = load_f32(dy + c) * (gamma ? load_f32(gamma + c) : 1.f);
        const float h = (load_f32(x + c) - mean) * rstd;
        store_f32(dx + c, good ? rstd * (av - c1 - h * c2) : 0.f);
    }
}

// Column sums of long rows: one thread per column, blockIdx.y takes every gridDim.y-th row.
template <class T>
__global__ void __launch_bounds__(256) norm_cols_kernel(const NormBwdArgs a, const float* row_flag) {
    pdl_launch();
    pdl_wait();
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

// dgamma / dbeta = the sum of `parts` partial rows, in ascending order within each of the 16 strands of
// a column and then over the strands; fp64, rounded once.
template <class P>
__global__ void __launch_bounds__(512) norm_sum_kernel(const float* partial, int32_t parts, int32_t N, P* dgamma,
                                                       P* dbeta) {
    __shared__ double s[16][33];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int64_t j = int64_t(blockIdx.x) * 32 + lane;           // column of the [2N]-wide partial row
    double t = 0.0;
    if (j < 2 * int64_t(N)) {
#pragma unroll 4
        for (int p = strand; p < parts; p += 16) t += double(partial[int64_t(p) * 2 * N + j]);
    }
    s[strand][lane] = t;
    __syncthreads();
    if (strand == 0 && j < 2 * int64_t(N)) {
        t = 0.0;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += s[k][lane];
        if (j < N) { if (dgamma) store_f32(dgamma + j, float(t)); }
        else if (dbeta) store_f32(dbeta + (j - N), float(t));
    }
}

bool rows_aligned(const void* p, int64_t ld, size_t esize) {
    return aligned(p, 16) && (ld * int64_t(esize)) % 16 == 0;
}

// Calls f.template operator()<CH>() with the smallest CH of the list that is at least `need`.
template <int... CH, class F>
int with_pieces(int need, F&& f) {
    int rc = TPPO_ERR_UNSUPPORTED;
    bool done = false;
    ((!done && need <= CH ? (done = true, rc = f(std::integral_constant<int, CH>())) : 0), ...);
    return rc;
}

template <class T, class P>
int norm_fwd_typed(NormFwdArgs a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = a.N % V == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.y, a.ldy, sizeof(T)) &&
                     (!a.gamma || aligned(a.gamma, 16)) && (!a.beta || aligned(a.beta, 16));
    // Four 16-byte pieces (eight single elements) per thread: few registers, so that some 40 warps per SM
    // keep ~80 KB in flight.  Rows longer than 1024 such threads hold take 8 (16) per thread, then the
    // kernel that reads the row again.  With few rows more threads share a row, for shorter chains.
    const int64_t pieces = vec ? a.N / V : a.N;
    int64_t per = vec ? 4 : 8;
    while (per > 1 && a.M * ((pieces + per - 1) / per) < int64_t(kNumSms) * 512 && pieces <= per / 2 * 512) per /= 2;
    if (pieces > per * kNormMaxThreads) per *= 2;
    if (pieces > per * kNormMaxThreads) {
        TPPO_CUDA_CHECK(launch_dense(norm_fwd_long_kernel<T, P>, dim3(unsigned(a.M)), dim3(kNormMaxThreads), 0, s, a));
        return TPPO_OK;
    }
    a.group = int32_t((pieces + per * 32 - 1) / (per * 32) * 32);
    const int groups = a.group == 32 ? 4 : 1;
    const unsigned blocks = unsigned((a.M + groups - 1) / groups);
    const auto go = [&](auto vecs, auto ch) -> int {
        TPPO_CUDA_CHECK(launch_dense(norm_fwd_kernel<T, P, decltype(vecs)::value, decltype(ch)::value>, dim3(blocks), dim3(a.group * groups), 0, s, a));
        return TPPO_OK;
    };
    if (vec) return with_pieces<1, 2, 4, 8>(int(per), [&](auto ch) { return go(std::integral_constant<int, V>(), ch); });
    return with_pieces<1, 2, 4, 8, 16>(int(per), [&](auto ch) { return go(std::integral_constant<int, 1>(), ch); });
}

constexpr int kNormMaxParts = 2 * kNumSms;

struct NormWs { float* partial; float* row_flag; size_t bytes; };
NormWs norm_carve(void* ws, int64_t M, int32_t N) {
    const size_t a = align_up(size_t(kNormMaxParts) * 2 * size_t(N) * 4, kWsAlign);
    const size_t b = align_up(size_t(M) * 4, kWsAlign);
    char* p = static_cast<char*>(ws);
    return {reinterpret_cast<float*>(p), reinterpret_cast<float*>(p + a), a + b};
}

constexpr size_t kRingBytes = 112 * 1024, kRingBytesAlone = 224 * 1024;

template <class T, class P>
int norm_bwd_typed(NormBwdArgs a, P* dgamma, P* dbeta, float* row_flag, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = a.N % V == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.dy, a.lddy, sizeof(T)) &&
                     (!a.dx || rows_aligned(a.dx, a.lddx, sizeof(T))) && (!a.gamma || aligned(a.gamma, 16));
    const int64_t pieces = vec ? a.N / V : a.N;
    const size_t stage = 2 * size_t(a.N) * sizeof(T);
    int parts = 0, rc = TPPO_OK;
    if (vec && a.M >= kNumSms && pieces >= 128 && stage * 2 <= kRingBytesAlone && pieces <= 512 * (32 / V)) {
        // two blocks per SM where their rings of at least three rows fit beside each other
        const bool pair = stage * 3 <= kRingBytes;
        const size_t budget = pair ? kRingBytes : kRingBytesAlone;
        int64_t stages = int64_t(budget / stage);
        if (stages > 8) stages = 8;
        a.stages = int32_t(stages);
        const int need = int((pieces + 319) / 320);
        const size_t smem = size_t(stages) * stage + 8 * 8;
        const int64_t most = kNumSms * (pair ? 2 : 1);
        parts = int(a.M < most ? a.M : most);
        const auto go = [&](auto ch) -> int {
            constexpr int CH = decltype(ch)::value;
            a.group = int32_t((pieces + CH * 32 - 1) / (CH * 32) * 32);
            auto kernel = norm_bwd_ring_kernel<T, P, V, CH>;
            TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)));
            TPPO_CUDA_CHECK(launch_dense(kernel, dim3(unsigned(parts)), dim3(a.group), smem, s, a));
            return TPPO_OK;
        };
        if constexpr (V == 8) rc = pieces > 2 * 512 ? go(std::integral_constant<int, 4>()) : with_pieces<1, 2>(need > 2 ? 2 : need, go);
        else rc = pieces > 4 * 512 ? go(std::integral_constant<int, 8>()) : with_pieces<1, 2, 4>(need > 4 ? 4 : need, go);
    } else if (pieces <= 512 * (vec ? 16 / V : 16)) {
        // the fewest columns per thread (16 at most) that keep a row within 256 threads, else 512
        static const int ladder[] = {1, 2, 4, 6, 8, 12, 16};
        int need = 0, group = 0;
        for (int k = 0; k < 14 && !need; ++k) {
            const int ch = ladder[k % 7];
            if (ch * (vec ? V : 1) > 16 || (vec && ch != 1 && ch != 2 && ch != 4)) continue;
            const int64_t g = (pieces + ch * 32 - 1) / (ch * 32) * 32;
            if (g <= (k < 7 ? 256 : 512)) { need = ch; group = int(g); }
        }
        a.group = group;
        const int groups = group >= 128 ? 1 : 256 / group;
        const int64_t rows = (a.M + groups - 1) / groups;
        const int64_t most = kNumSms * 2;
        parts = int(rows < most ? rows : most);
        const size_t smem = groups > 1 && a.partial ? size_t(a.N) * 8 : 0;
        const auto go = [&](auto vecs, auto ch) -> int {
            constexpr int VEC = decltype(vecs)::value, CH = decltype(ch)::value;
            // some sixteen elements of x and of dy in flight per thread and trip, at most four rows
            constexpr int ROWS = VEC * CH > 8 ? 1 : VEC * CH > 4 ? 2 : 4;
            TPPO_CUDA_CHECK(launch_dense(norm_bwd_kernel<T, P, VEC, CH, ROWS>, dim3(unsigned(parts)), dim3(a.group * groups), smem, s, a));
            return TPPO_OK;
        };
        if (vec) rc = with_pieces<1, 2, 4>(need, [&](auto ch) -> int {
            if constexpr (decltype(ch)::value * V > 16) return TPPO_ERR_UNSUPPORTED;
            else return go(std::integral_constant<int, V>(), ch);
        });
        else rc = with_pieces<1, 2, 4, 6, 8, 12, 16>(need, [&](auto ch) { return go(std::integral_constant<int, 1>(), ch); });
    } else {
        // the column sums read dy, which dx may overwrite: flags first, then the sums, then dx
        NormBwdArgs b = a;
        if (a.partial) {
            b.dx = nullptr;
            TPPO_CUDA_CHECK(launch_dense(norm_bwd_long_kernel<T, P>, dim3(unsigned(a.M)), dim3(kNormMaxThreads), 0, s, b, row_flag));
            parts = int(a.M < 64 ? a.M : 64);
            TPPO_CUDA_CHECK(launch_dense(norm_cols_kernel<T>, dim3(dim3((a.N + 255) / 256, parts)), dim3(256), 0, s, a, row_flag));
        }
        if (a.dx) {
            TPPO_CUDA_CHECK(launch_dense(norm_bwd_long_kernel<T, P>, dim3(unsigned(a.M)), dim3(kNormMaxThreads), 0, s, a, nullptr));
        }
    }
    if (rc != TPPO_OK || !a.partial) return rc;
    TPPO_CUDA_CHECK(launch_dense(norm_sum_kernel<P>, dim3(unsigned((2 * int64_t(a.N) + 31) / 32)), dim3(512), 0, s,
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
    const NormBwdArgs a{dy, x, gamma, mean, rstd, dx, params ? w.partial : nullptr, status, M, N, lddy, ldx, lddx, 0, 0};
    if (dtype == TPPO_BF16) {
        if (param_dtype == TPPO_F32)
            return norm_bwd_typed<bf16_bits, float>(a, static_cast<float*>(dgamma), static_cast<float*>(dbeta), w.row_flag, s);
        return norm_bwd_typed<bf16_bits, bf16_bits>(a, static_cast<bf16_bits*>(dgamma), static_cast<bf16_bits*>(dbeta), w.row_flag, s);
    }
    if (param_dtype == TPPO_F32)
        return norm_bwd_typed<float, float>(a, static_cast<float*>(dgamma), static_cast<float*>(dbeta), w.row_flag, s);
    return norm_bwd_typed<float, bf16_bits>(a, static_cast<bf16_bits*>(dgamma), static_cast<bf16_bits*>(dbeta), w.row_flag, s);
}
