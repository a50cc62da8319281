// Backward pass of the residual join; see residual_norm.cuh.
#include <type_traits>

#include "residual_norm.cuh"

namespace tppo {
namespace {

// The scalars of a row's backward pass, from its three sums: m2 = mean(a2 hh), m1 = mean(a1 zz), with hh = h r2 and zz = z r1.
//     d = dh + r2 (a2 - m2 hh) = dh + r2 a2 - (m2 r2^2) h,      dz = r1 (a1 - m1 zz) = r1 a1 - (m1 r1^2) z
// The right-hand forms save three operations per element, but their factors leave fp32 before the result does: at a mean square
// of 2^100 they kept no bit of gradients of 2^-50.  With 16 elements per thread or more and no gate per element, rows with
// scales from 2^-20 to 2^20, any that training meets, take them (gradients keep their precision down to 2^-86) and other rows
// the left-hand ones, at one branch per row ([16384, 5120] bf16 215 us, 5121 columns 312; without the branch 223 and 330).  With 8
// elements or a gate per element all rows take the left-hand forms: two forms cost such a kernel more registers than they
// save operations ([16384, 5120] bf16 gated 297 us, with the branch 323; [65536, 256] 52 and 56; [8192, 5120] fp32 167 and 168).
struct JoinRow { float r1, r2, m2, m1; bool good; };
__host__ __device__ constexpr bool join_two_forms(int e, bool gated) { return e >= 16 && !gated; }
__device__ __forceinline__ bool join_ordinary(float r) { return r >= 0x1p-20f && r <= 0x1p20f; }
// zs: r1 where the sums were taken with z as it is, 1 where with zz.
__device__ __forceinline__ JoinRow join_row(const JoinArgs& a, float r1, float r2, float zs, const float (&s)[3], bool reports) {
    const bool post = a.norms & TPPO_NORM_POST, pre = a.norms & TPPO_NORM_PRE;
    const float inv = 1.f / float(a.N);
    JoinRow w;
    w.r1 = post ? r1 : 1.f;
    w.r2 = pre ? r2 : 0.f;
    w.m2 = pre ? s[0] * inv * r2 : 0.f;
    w.m1 = post ? (s[1] - (w.m2 * r2) * (s[2] * r2)) * inv * zs : 0.f;
    const bool stats = !((post && r1 == 0.f) || (pre && r2 == 0.f));
    w.good = is_finite(s[0]) && is_finite(s[1]) && is_finite(w.m2) && is_finite(w.m1);
    if (!w.good && stats && reports && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
    w.good = w.good && stats;
    return w;
}

// Pairs of fp32 values, on which one instruction works at a time: at some 30 operations per element the backward pass of
// bf16 rows is otherwise bound by its instructions.
template <class T> struct JoinPairs { static constexpr int N = Join<T>::VEC / 2; };
template <class T>
__device__ __forceinline__ void join_piece(uint32_t at, uint64_t (&v)[JoinPairs<T>::N]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = ptx::lds128(at);
        v[0] = ptx::pack_f32x2(bf16_lo(w.x), bf16_hi(w.x));
        v[1] = ptx::pack_f32x2(bf16_lo(w.y), bf16_hi(w.y));
        v[2] = ptx::pack_f32x2(bf16_lo(w.z), bf16_hi(w.z));
        v[3] = ptx::pack_f32x2(bf16_lo(w.w), bf16_hi(w.w));
    } else {
        asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "r"(at));
    }
}
template <class T, class C>
__device__ __forceinline__ void join_store(const C& k, int c, T* row, const uint64_t (&v)[JoinPairs<T>::N]) {
    if (k.all(c)) {
        uint4 w;
        if constexpr (sizeof(T) == 2)
            w = make_uint4(ptx::pack_bf16x2_from_f32x2(v[0]), ptx::pack_bf16x2_from_f32x2(v[1]), ptx::pack_bf16x2_from_f32x2(v[2]),
                           ptx::pack_bf16x2_from_f32x2(v[3]));
        else
            w = make_uint4(uint32_t(v[0]), uint32_t(v[0] >> 32), uint32_t(v[1]), uint32_t(v[1] >> 32));
        *reinterpret_cast<uint4*>(row + k.col(c)) = w;
    } else {
#pragma unroll
        for (int i = 0; i < Join<T>::VEC; ++i) {
            float lo, hi;
            ptx::unpack_f32x2(v[i / 2], lo, hi);
            if (k.has(c, i)) store_f32(row + k.col(c) + i, i % 2 ? hi : lo);
        }
    }
}

template <class T, int E, bool PRE, bool GATED, bool SHIFT>
__global__ void __launch_bounds__(join_threads(E), 1) join_bwd_kernel(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef JoinThread<T, E, SHIFT, join_bwd_regs(E), kBwdIn> Thread;
    constexpr int VEC = Thread::VEC, CH = Thread::CH, P = VEC / 2;
    Thread th(a, smem);
    pdl_launch();
    pdl_wait();
    for (int s = 0; s < a.stages; ++s) th.fetch(a, th.row + s * th.step, th.stage_at(a, s));
    th.load_params(a, smem);
    __syncthreads();
    using ptx::fma_f32x2;
    using ptx::mul_f32x2;
    const bool add = a.in[kDh] != nullptr, post = a.norms & TPPO_NORM_POST;
    uint64_t sum_post[CH][P], sum_pre[CH][P];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < P; ++i) sum_post[c][i] = sum_pre[c][i] = 0;
    int turn = 0;
    uint32_t stage = th.stage_at(a, 0);
    float r1_next = post && th.row < a.M ? a.r_post[th.row] : 1.f, r2_next = PRE && th.row < a.M ? a.r_pre[th.row] : 0.f;
    for (int64_t r = th.row; r < a.M; r += th.step) {
        const float r1 = r1_next, r2 = r2_next;
        if (r + th.step < a.M) {                          // a row ahead, like the copies
            if (post) r1_next = a.r_post[r + th.step];
            if (PRE) r2_next = a.r_pre[r + th.step];
        }
        th.land(a, stage);
        auto row = [&](auto scaled) {
            constexpr bool SCALED = decltype(scaled)::value;
            const uint64_t r1_2 = ptx::pack_f32x2(r1, r1), r2_2 = ptx::pack_f32x2(r2, r2);
            uint64_t q[3] = {0, 0, 0};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!th.k.any(c)) continue;
                uint64_t w[P], d[P], g[P];
                join_piece<T>(th.at(a, stage, kZ, c), w);
                th.post(a, c, g);
#pragma unroll
                for (int i = 0; i < P; ++i) w[i] = mul_f32x2(SCALED ? mul_f32x2(w[i], r1_2) : w[i], g[i]);
                if (GATED) {
                    join_piece<T>(th.at(a, stage, kGate, c), g);
#pragma unroll
                    for (int i = 0; i < P; ++i) w[i] = mul_f32x2(w[i], g[i]);
                }
#pragma unroll
                for (int i = 0; i < P; ++i) d[i] = 0;
                if (add) join_piece<T>(th.at(a, stage, kDh, c), d);
                if (PRE) {
                    uint64_t n[P], h[P];
                    join_piece<T>(th.at(a, stage, kDn, c), n);
                    join_piece<T>(th.at(a, stage, kH, c), h);
                    th.pre(a, c, g);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        n[i] = mul_f32x2(n[i], g[i]);
                        q[0] = fma_f32x2(n[i], h[i], q[0]);
                        q[2] = fma_f32x2(h[i], w[i], q[2]);
                        d[i] = fma_f32x2(r2_2, n[i], d[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < P; ++i) q[1] = fma_f32x2(d[i], w[i], q[1]);
            }
            float s[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                float lo, hi;
                ptx::unpack_f32x2(q[i], lo, hi);
                s[i] = lo + hi;
            }
            th.sum(s);
            const JoinRow w = join_row(a, r1, r2, SCALED ? 1.f : r1, s, th.t == 0);
            T *dz = th.out(a, 0, r), *dres = th.out(a, 1, r), *dgate = th.out(a, 2, r);
            if (!w.good) {                                // the same for the whole group
                if (a.out[0]) th.store_zeros(dz);
                if (a.out[1]) th.store_zeros(dres);
                if (a.out[2]) th.store_zeros(dgate);
                return;
            }
            const float k1 = SCALED ? w.m1 : w.m1 * r1 * r1, k2 = SCALED ? w.m2 : w.m2 * r2 * r2;
            const uint64_t k1_2 = ptx::pack_f32x2(-k1, -k1), k2_2 = ptx::pack_f32x2(-k2, -k2), alpha_2 = ptx::pack_f32x2(a.alpha, a.alpha);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!th.k.any(c)) continue;
                uint64_t z[P], d[P], g[P], v[P];
#pragma unroll
                for (int i = 0; i < P; ++i) d[i] = 0;
                if (add) join_piece<T>(th.at(a, stage, kDh, c), d);
                if (PRE) {
                    uint64_t n[P], h[P];
                    join_piece<T>(th.at(a, stage, kDn, c), n);
                    join_piece<T>(th.at(a, stage, kH, c), h);
                    th.pre(a, c, g);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        if (SCALED) h[i] = mul_f32x2(h[i], r2_2);
                        else n[i] = mul_f32x2(n[i], r2_2);
                        sum_pre[c][i] = fma_f32x2(n[i], h[i], sum_pre[c][i]);
                        if (SCALED) d[i] = fma_f32x2(r2_2, fma_f32x2(k2_2, h[i], mul_f32x2(n[i], g[i])), d[i]);
                        else d[i] = fma_f32x2(k2_2, h[i], fma_f32x2(n[i], g[i], d[i]));
                    }
                }
                if (a.out[1]) {
#pragma unroll
                    for (int i = 0; i < P; ++i) v[i] = mul_f32x2(alpha_2, d[i]);
                    join_store<T>(th.k, c, dres, v);
                }
                join_piece<T>(th.at(a, stage, kZ, c), z);
                th.post(a, c, g);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    if (SCALED) z[i] = mul_f32x2(z[i], r1_2);
                    else d[i] = mul_f32x2(d[i], r1_2);
                }
                if (GATED) {
                    join_piece<T>(th.at(a, stage, kGate, c), v);
                    if (a.out[2]) {
                        uint64_t o[P];
#pragma unroll
                        for (int i = 0; i < P; ++i) o[i] = mul_f32x2(mul_f32x2(d[i], z[i]), g[i]);
                        join_store<T>(th.k, c, dgate, o);
                    }
#pragma unroll
                    for (int i = 0; i < P; ++i) d[i] = mul_f32x2(d[i], v[i]);
                }
#pragma unroll
                for (int i = 0; i < P; ++i) sum_post[c][i] = fma_f32x2(d[i], z[i], sum_post[c][i]);
                if (a.out[0]) {
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        v[i] = fma_f32x2(k1_2, z[i], mul_f32x2(d[i], g[i]));
                        if (SCALED) v[i] = mul_f32x2(r1_2, v[i]);
                    }
                    join_store<T>(th.k, c, dz, v);
                }
            }
        };
        if constexpr (join_two_forms(E, GATED)) {
            if ((!post || join_ordinary(r1)) && (!PRE || join_ordinary(r2))) row(std::false_type{});
            else row(std::true_type{});
        } else {
            row(std::true_type{});
        }
        th.fetch(a, r + a.stages * th.step, stage);
        if (++turn == a.stages) turn = 0;
        stage = th.stage_at(a, turn);
    }
    if (!a.partial) return;
    // the groups' sums meet in the ring's memory: group 0 adds the others' to its own, in order
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float* all = reinterpret_cast<float*>(smem + kJoinRedBytes);           // [group][2 * E][T]
    if (th.group > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float* to = all + ((th.group - 1) * 2 * E + c * VEC + 2 * i) * a.T + th.t;
                ptx::unpack_f32x2(sum_post[c][i], to[0], to[a.T]);
                ptx::unpack_f32x2(sum_pre[c][i], to[E * a.T], to[(E + 1) * a.T]);
            }
    }
    __syncthreads();
    if (th.group > 0) return;
    float* part = a.partial + int64_t(blockIdx.x) * 2 * a.N;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float v[4];
            ptx::unpack_f32x2(sum_post[c][i], v[0], v[1]);
            ptx::unpack_f32x2(sum_pre[c][i], v[2], v[3]);
            for (int g = 1; g < a.groups; ++g) {
                const float* from = all + ((g - 1) * 2 * E + c * VEC + 2 * i) * a.T + th.t;
                v[0] += from[0]; v[1] += from[a.T];
                v[2] += from[E * a.T]; v[3] += from[(E + 1) * a.T];
            }
#pragma unroll
            for (int l = 0; l < 2; ++l)
                if (th.k.has(c, 2 * i + l)) {
                    part[th.k.col(c) + 2 * i + l] = v[l];
                    part[int64_t(a.N) + th.k.col(c) + 2 * i + l] = v[2 + l];
                }
        }
}

// ---- any length and alignment --------------------------------------------------------------------------------
// Backward pass of such rows in two launches: the three sums of every row, then, with no thread depending on another,
// the gradients, a block walking down its strip of columns.  10 elements moved per element of a row instead of 6.
// VEC: columns per access, 16 bytes' worth where all rows start and end on 16-byte boundaries, else 1.
// Loads stand under no condition, so that they leave together: a matrix that is not there has z's address (and its values
// replaced), and the parameters have been made whole by a small launch in front.
struct JoinWide {
    const void* in[kBwdIn]; int64_t ld[kBwdIn];           // none is NULL
    uint32_t has;                                         // bit m: matrix m is there
    const float* post; const float* pre;                  // gate row * gamma_post, gamma_pre
};
template <class T, int VEC>
__device__ __forceinline__ void join_read(const JoinWide& a, int m, int64_t r, int c, float otherwise, float (&v)[VEC]) {
    load_vec<VEC>(static_cast<const T*>(a.in[m]) + r * a.ld[m] + c, v);
    if (!(a.has >> m & 1u)) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = otherwise;
    }
}
__global__ void __launch_bounds__(256) join_params_kernel(const void* gate_row, const void* gamma_post, const void* gamma_pre, int32_t p32, int32_t N,
                                                          float* post, float* pre) {
    pdl_launch();
    pdl_wait();
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (c >= N) return;
    post[c] = param(gate_row, c, p32) * param(gamma_post, c, p32);
    pre[c] = param(gamma_pre, c, p32);
}
template <class T, int VEC>
__global__ void __launch_bounds__(kJoinAnyThreads, 2) join_row_sums_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ JoinWide w) {
    __shared__ float red[3 * 32];
    pdl_launch();
    pdl_wait();
    for (int64_t r = blockIdx.x; r < a.M; r += gridDim.x) {
        const float r1 = a.r_post ? a.r_post[r] : 1.f, r2 = a.r_pre ? a.r_pre[r] : 0.f;
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll(VEC == 1 ? 4 : 1)
        for (int c = threadIdx.x * VEC; c < a.N; c += kJoinAnyThreads * VEC) {
            float z[VEC], g[VEC], d[VEC], n[VEC], h[VEC], gp[VEC], gn[VEC];
            join_read<T, VEC>(w, kZ, r, c, 0.f, z);
            join_read<T, VEC>(w, kGate, r, c, 1.f, g);
            join_read<T, VEC>(w, kDh, r, c, 0.f, d);
            join_read<T, VEC>(w, kDn, r, c, 0.f, n);
            join_read<T, VEC>(w, kH, r, c, 0.f, h);
            load_vec<VEC>(w.post + c, gp);
            load_vec<VEC>(w.pre + c, gn);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float x = z[i] * r1 * (g[i] * gp[i]), a2 = n[i] * gn[i];
                s[0] = fmaf(a2, h[i], s[0]);
                s[1] = fmaf(fmaf(r2, a2, d[i]), x, s[1]);
                s[2] = fmaf(h[i], x, s[2]);
            }
        }
        block_sums(s, red);
        if (threadIdx.x == 0) {
            const JoinRow q = join_row(a, r1, r2, 1.f, s, true);
            // zeros: a row to leave out
            a.rows[r] = q.good ? make_float4(q.r1, q.r2, q.m1, q.m2) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
}

// Threads of a strip: with fewer bytes of a row HBM's pages are opened for too little.
template <int VEC> __host__ __device__ constexpr int join_strip() { return VEC == 1 ? 512 : 128; }
template <class T, int VEC>
__global__ void __launch_bounds__(join_strip<VEC>(), VEC == 1 ? 2 : 4)
join_columns_kernel(const __grid_constant__ JoinArgs a, const __grid_constant__ JoinWide p) {
    pdl_launch();
    pdl_wait();
    const int64_t chunk = blockIdx.y, r0 = a.M * chunk / gridDim.y, r1 = a.M * (chunk + 1) / gridDim.y;
    const int64_t at = (int64_t(blockIdx.x) * join_strip<VEC>() + threadIdx.x) * VEC;
    if (at >= a.N) return;
    const int c = int(at);
    float g[VEC], gn[VEC], sum_post[VEC], sum_pre[VEC];
    load_vec<VEC>(p.post + c, g);
    load_vec<VEC>(p.pre + c, gn);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum_post[i] = sum_pre[i] = 0;
    // two rows at a time: four of single elements need more than the 64 registers of this occupancy (5000 x 12001 bf16 704 us
    // for the whole pass, with two 496)
#pragma unroll 2
    for (int64_t r = r0; r < r1; ++r) {
        const float4 w = __ldcg(a.rows + r);
        float z[VEC], gv[VEC], d[VEC], n[VEC], h[VEC], o[VEC];
        join_read<T, VEC>(p, kZ, r, c, 0.f, z);
        join_read<T, VEC>(p, kGate, r, c, 1.f, gv);
        join_read<T, VEC>(p, kDh, r, c, 0.f, d);
        join_read<T, VEC>(p, kDn, r, c, 0.f, n);
        join_read<T, VEC>(p, kH, r, c, 0.f, h);
        const bool good = w.x != 0.f;                     // r1 of a row with statistics is not 0
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            h[i] *= w.y;
            if (good) sum_pre[i] = fmaf(n[i], h[i], sum_pre[i]);
            d[i] = fmaf(w.y, fmaf(-w.w, h[i], n[i] * gn[i]), d[i]);
            o[i] = good ? a.alpha * d[i] : 0.f;
            z[i] *= w.x;
        }
        if (a.out[1]) store_vec<VEC>(static_cast<T*>(a.out[1]) + r * a.ldo[1] + c, o);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            o[i] = good ? d[i] * z[i] * g[i] : 0.f;
            d[i] *= gv[i];
            if (good) sum_post[i] = fmaf(d[i], z[i], sum_post[i]);
        }
        if (a.out[2]) store_vec<VEC>(static_cast<T*>(a.out[2]) + r * a.ldo[2] + c, o);
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = good ? w.x * fmaf(-w.z, z[i], d[i] * g[i]) : 0.f;
        if (a.out[0]) store_vec<VEC>(static_cast<T*>(a.out[0]) + r * a.ldo[0] + c, o);
    }
    if (a.partial) {
        float* part = a.partial + chunk * 2 * a.N;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            part[c + i] = sum_post[i];
            part[int64_t(a.N) + c + i] = sum_pre[i];
        }
    }
}

// Adds the blocks' partial rows up in a fixed order (eight strands of them) and finishes the gradients:
//     dgamma_post = gate row * S, dgate row = gamma_post * S, dgamma_pre = the second sum.
// A factor that is not finite leaves every row out, so that S is 0 and so is the gradient.
struct JoinSumArgs {
    const float* partial; int64_t rows; int32_t N;
    const void* gate_row; const void* gamma_post;
    void* dgate_row; void* dgamma_post; void* dgamma_pre; int32_t p32;
};
__device__ __forceinline__ float join_scaled(float sum, float factor) { return sum == 0.f || factor == 0.f ? 0.f : sum * factor; }
__global__ void __launch_bounds__(256) join_sum_kernel(const JoinSumArgs a) {
    __shared__ float red[8][32];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int64_t col = int64_t(blockIdx.x) * 32 + lane, all = int64_t(2) * a.N;
    float v = 0;
    if (col < all) {
#pragma unroll 8
        for (int64_t r = strand; r < a.rows; r += 8) v += __ldcg(a.partial + r * all + col);
    }
    red[strand][lane] = v;
    __syncthreads();
    if (strand != 0 || col >= all) return;
    for (int i = 1; i < 8; ++i) v += red[i][lane];
    if (col < a.N) {
        if (a.dgamma_post) put_param(a.dgamma_post, col, a.p32, join_scaled(v, param(a.gate_row, col, a.p32)));
        if (a.dgate_row) put_param(a.dgate_row, col, a.p32, join_scaled(v, param(a.gamma_post, col, a.p32)));
    } else if (a.dgamma_pre) {
        put_param(a.dgamma_pre, col - a.N, a.p32, v);
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
template <class T, int E, bool PRE>
int launch_bwd(const JoinArgs& a, const JoinPlan& p, cudaStream_t s) {
    auto kernel = a.in[kGate] ? (p.shift ? join_bwd_kernel<T, E, PRE, true, true> : join_bwd_kernel<T, E, PRE, true, false>)
                              : (p.shift ? join_bwd_kernel<T, E, PRE, false, true> : join_bwd_kernel<T, E, PRE, false, false>);
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kJoinSmem));
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(p.grid), dim3(a.T * a.groups), p.smem, s, a));
    return TPPO_OK;
}

int64_t join_chunks(int64_t M) { return M < kJoinAnyBlocks ? (M + 7) / 8 * 8 : kJoinAnyBlocks; }

template <class T, int VEC>
int run_bwd_any(JoinArgs& a, JoinSumArgs& sum, cudaStream_t s) {
    JoinWide w{};
    for (int i = 0; i < kBwdIn; ++i) {
        const bool has = a.in[i] != nullptr;
        w.in[i] = has ? a.in[i] : a.in[kZ];
        w.ld[i] = has ? a.ld[i] : a.ld[kZ];
        w.has |= has ? 1u << i : 0u;
    }
    w.post = a.params;
    w.pre = a.params + align_up(size_t(a.N), 64);
    TPPO_CUDA_CHECK(launch_dense(join_params_kernel, dim3(unsigned((int64_t(a.N) + 255) / 256)), dim3(256), 0, s, a.gate_row, a.gamma_post, a.gamma_pre,
                                 a.p32, a.N, a.params, a.params + align_up(size_t(a.N), 64)));
    TPPO_CUDA_CHECK(launch_dense(join_row_sums_kernel<T, VEC>, dim3(unsigned(a.M < 4 * kNumSms ? a.M : 4 * kNumSms)), dim3(kJoinAnyThreads), 0, s, a, w));
    // enough chunks of rows to fill the GPU some times over
    constexpr int kStrip = join_strip<VEC>();
    const int64_t strips = (int64_t(a.N) + kStrip * VEC - 1) / (kStrip * VEC), most = join_chunks(a.M);
    int64_t chunks = ((VEC == 1 ? 8 : 32) * kNumSms + strips - 1) / strips;
    if (chunks > (a.M + 7) / 8) chunks = (a.M + 7) / 8;
    if (chunks > most) chunks = most;
    sum.rows = chunks;
    TPPO_CUDA_CHECK(launch_dense(join_columns_kernel<T, VEC>, dim3(unsigned(strips), unsigned(chunks)), dim3(kStrip), 0, s, a, w));
    return TPPO_OK;
}

template <class T>
int run_bwd(JoinArgs& a, bool same, JoinSumArgs& sum, cudaStream_t s) {
    constexpr int vec = Join<T>::VEC;
    JoinPlan p;
    const int64_t width = join_width(a, p, vec);
    const bool whole = same && !p.shift;                  // every row is a number of 16-byte pieces
    if (same) {
        join_choose(a, p, {8, 16, 24}, vec, width, true);
    }
    sum.rows = p.grid;
    const bool pre = a.norms & TPPO_NORM_PRE;
    if (p.E == 8) return pre ? launch_bwd<T, 8, true>(a, p, s) : launch_bwd<T, 8, false>(a, p, s);
    if (p.E == 24) return pre ? launch_bwd<T, 24, true>(a, p, s) : launch_bwd<T, 24, false>(a, p, s);
    if (p.E == 16) return pre ? launch_bwd<T, 16, true>(a, p, s) : launch_bwd<T, 16, false>(a, p, s);
    return whole ? run_bwd_any<T, vec>(a, sum, s) : run_bwd_any<T, 1>(a, sum, s);
}

}  // namespace

// The rows' scalars in front, then the two rows of parameters, the partial column sums behind them.
static size_t join_rows_bytes(int64_t M) { return align_up(size_t(M > 0 ? M : 1) * sizeof(float4), kWsAlign); }
static size_t join_params_bytes(int32_t N) { return 2 * align_up(size_t(N), 64) * sizeof(float); }
size_t residual_norm_workspace_bytes(int64_t M, int32_t N) {
    if (N <= 0) return 0;
    return join_rows_bytes(M) + join_params_bytes(N) + align_up(size_t(M > 0 ? join_chunks(M) : 1) * 2 * size_t(N) * sizeof(float), kWsAlign);
}

}  // namespace tppo

TPPO_API int tppo_residual_norm_bwd(const void* dh, int64_t lddh, const void* dn, int64_t lddn, const void* z, int64_t ldz,
                                    const void* h, int64_t ldh, const void* gate, int64_t ldg, int32_t dtype, int64_t M, int32_t N,
                                    const void* gamma_post, const void* gamma_pre, int32_t param_dtype,
                                    const float* rstd_post, const float* rstd_pre, float alpha, int32_t norms,
                                    void* dz, int64_t lddz, void* dresidual, int64_t lddr, void* dgate, int64_t lddg,
                                    void* dgamma_post, void* dgamma_pre, int32_t* status, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    using namespace tppo;
    if (M < 0 || N < 1 || !type_ok(dtype) || !type_ok(param_dtype) || (norms & ~3) || !is_finite_host(alpha)) return TPPO_ERR_INVALID_ARG;
    const bool post = norms & TPPO_NORM_POST, pre = norms & TPPO_NORM_PRE;
    const bool full = gate && ldg != 0;
    if ((gamma_post && !post) || (gamma_pre && !pre) || (dgamma_post && !post) || (dgamma_pre && !pre) || (dgate && !gate))
        return TPPO_ERR_INVALID_ARG;
    if (M > 0 && (!z || (dn != nullptr) != pre || (h != nullptr) != pre || (rstd_post != nullptr) != post || (rstd_pre != nullptr) != pre))
        return TPPO_ERR_INVALID_ARG;
    if (ldz < N || (dh && lddh < N) || (pre && (lddn < N || ldh < N)) || (full && ldg < N) || (dz && lddz < N) || (dresidual && lddr < N) ||
        (dgate && full && lddg < N))
        return TPPO_ERR_INVALID_ARG;
    const size_t e = size_of(dtype), pe = size_of(param_dtype);
    if (!aligned(dh, e) || !aligned(dn, e) || !aligned(z, e) || !aligned(h, e) || !aligned(gate, full ? e : pe) || !aligned(dz, e) ||
        !aligned(dresidual, e) || !aligned(dgate, full ? e : pe) || !aligned(gamma_post, pe) || !aligned(gamma_pre, pe) ||
        !aligned(dgamma_post, pe) || !aligned(dgamma_pre, pe) || !aligned(rstd_post, 4) || !aligned(rstd_pre, 4) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || N > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    const bool sums = dgamma_post || dgamma_pre || (dgate && !full);
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < residual_norm_workspace_bytes(M, N)) return TPPO_ERR_WORKSPACE;
    JoinArgs a{};
    a.in[kZ] = z; a.ld[kZ] = ldz;
    if (pre) { a.in[kH] = h; a.ld[kH] = ldh; a.in[kDn] = dn; a.ld[kDn] = lddn; }
    if (dh) { a.in[kDh] = dh; a.ld[kDh] = lddh; }
    if (full) { a.in[kGate] = gate; a.ld[kGate] = ldg; }
    for (int i = 0; i < kBwdIn; ++i)
        if (a.in[i]) a.slot[i] = a.arrays++;
    a.gate_row = full ? nullptr : gate;
    a.gamma_post = gamma_post; a.gamma_pre = gamma_pre; a.p32 = param_dtype == TPPO_F32;
    a.out[0] = dz; a.out[1] = dresidual; a.out[2] = full ? dgate : nullptr;
    a.ldo[0] = lddz; a.ldo[1] = lddr; a.ldo[2] = lddg;
    a.r_post = const_cast<float*>(rstd_post); a.r_pre = const_cast<float*>(rstd_pre);
    a.rows = static_cast<float4*>(workspace);
    a.params = reinterpret_cast<float*>(static_cast<char*>(workspace) + join_rows_bytes(M));
    a.partial = sums ? reinterpret_cast<float*>(static_cast<char*>(workspace) + join_rows_bytes(M) + join_params_bytes(N)) : nullptr;
    a.status = status;
    a.M = M; a.N = N; a.alpha = alpha; a.norms = norms;
    a.shift_step = int32_t(ldz % 16);
    a.one_ld = 1;
    for (int i = 0; i < kBwdIn; ++i) a.one_ld &= !a.in[i] || a.ld[i] == ldz;
    for (int i = 0; i < 3; ++i) a.one_ld &= !a.out[i] || a.ldo[i] == ldz;
    bool same = true;
    for (int i = 0; i < kBwdIn; ++i) same = same && same_start(z, ldz, a.in[i], a.ld[i], e);
    for (int i = 0; i < 3; ++i) same = same && same_start(z, ldz, a.out[i], a.ldo[i], e);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    JoinSumArgs sum{a.partial, 0, N, a.gate_row, gamma_post, full ? nullptr : dgate, dgamma_post, dgamma_pre, a.p32};
    if (M > 0) {
        const int r = dtype == TPPO_F32 ? run_bwd<float>(a, same, sum, s) : run_bwd<bf16_bits>(a, same, sum, s);
        if (r != TPPO_OK) return r;
    }
    if (!sums) return TPPO_OK;
    TPPO_CUDA_CHECK(launch_dense(join_sum_kernel, dim3(unsigned((int64_t(2) * N + 31) / 32)), dim3(256), 0, s, sum));
    return TPPO_OK;
}
