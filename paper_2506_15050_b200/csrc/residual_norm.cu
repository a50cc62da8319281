// The residual join: a block's output normed, gated and added to the scaled residual stream, and the sum normed
// for the next block; forward and backward with the parameters' gradients.  With root-mean-square norms,
//     h = alpha * residual + gate * gamma_post * z * r1,   n = h * r2 * gamma_pre
//     d = dh + r2 * (a2 - h r2^2 mean(a2 h)),  a2 = dn * gamma_pre;   dresidual = alpha * d
//     a1 = d * gate * gamma_post,   dz = r1 * (a1 - z r1^2 mean(a1 z)),   dgate = d * z * r1 * gamma_post
//     dgamma_post = sum_rows d * gate * z * r1,   dgamma_pre = sum_rows dn * h * r2
// All arithmetic is fp32; each input is read once, each output rounded once.  4 elements move forward and 6
// backward per element of a row (one and two more with a gate per element), so HBM is the bound.
//
// One block per SM, cut into groups of warps that walk rows of their own.  Each thread brings its 16-byte
// pieces of the next rows into a ring of shared memory of its own with cp.async: what it copies only it reads,
// so the ring needs no barrier, and 100-200 KB per SM stay in flight whatever the arithmetic does.  gate *
// gamma_post and gamma_pre sit in shared memory as fp32 for the block's life.
//
// Forward needs two sums over the row, one behind the other.  Backward takes one: with w = gate gamma_post z,
//     sum(a1 z) = sum((dh + r2 a2) w) - r2^3 mean(a2 h) sum(h w),
// three sums that do not wait for one another, met at one barrier per row.  (The same expansion of sum(h^2) would
// lose all its digits where the block's output cancels the residual, so the forward pass does not use it.)
//
// Rows that do not start on 16-byte boundaries are read by the same aligned pieces, the first and last of which
// hold elements of neighbouring rows or of nothing (a piece with one element of the row in it is mapped), cleared
// when they have arrived, and stored element by element.  A block only takes rows that start at the same place of
// a piece, so that a thread's columns, parameters and column sums stay its own.
// Rows that do not fit, and matrices whose rows do not start at the same place of a piece, are read again for each sweep.
#include <initializer_list>

#include "dense_common.cuh"

namespace tppo {
namespace {

constexpr int kJoinSmem = 224 * 1024;
constexpr int kJoinAnyThreads = 512, kJoinAnyBlocks = kNumSms * 2;
constexpr int kJoinStages = 4;

enum { kZ = 0, kRes = 1, kGate = 2, kFwdIn = 3 };         // forward inputs
enum { kH = 1, kDn = 3, kDh = 4, kBwdIn = 5 };            // backward: z, h, gate, dn, dh

struct JoinArgs {
    const void* in[kBwdIn];                               // matrices, NULL where there is none
    int64_t ld[kBwdIn];
    int32_t slot[kBwdIn];                                 // place in a stage
    const void* gate_row; const void* gamma_post; const void* gamma_pre;      // NULL: 1
    int32_t p32;                                          // parameters are fp32
    void* out[3]; int64_t ldo[3];                         // h, n | dz, dresidual, dgate
    float* r_post; float* r_pre;                          // out | in; NULL in the backward pass: no such norm
    float* partial;                                       // column sums: [blocks][2][N]
    float4* rows;                                         // r1, r2, k1, k2 of every row, where two launches share the work
    int32_t* status;
    int64_t M; int32_t N; float alpha, eps; int32_t norms;
    int32_t T, groups, stages, arrays;                    // threads per group; groups per block; stages; matrices per stage
    int32_t shift_step;                                   // rows start (first row's + r * this) elements into a piece
};

template <class T> struct Join { static constexpr int VEC = 16 / sizeof(T); };

__device__ __forceinline__ float param(const void* p, int64_t i, bool f32) {
    return !p ? 1.f : f32 ? static_cast<const float*>(p)[i] : load_f32(static_cast<const bf16_bits*>(p) + i);
}
__device__ __forceinline__ void put_param(void* p, int64_t i, bool f32, float v) {
    if (f32) store_f32(static_cast<float*>(p) + i, v);
    else store_f32(static_cast<bf16_bits*>(p) + i, v);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most `stages - 1` of this thread's groups of copies are outstanding.
__device__ __forceinline__ void copy_wait(int stages) {
    switch (stages) {
        case 1: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
        case 2: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
        case 3: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
        default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    }
}

// A thread's pieces of a row: piece c covers columns col(c) .. col(c) + VEC - 1.  SHIFT: rows need not start on a
// 16-byte boundary, or end on one; pieces may then lie partly outside the row.
template <class T, bool SHIFT>
struct JoinColumns {
    static constexpr int VEC = Join<T>::VEC;
    int first, step, N;
    __device__ __forceinline__ int col(int c) const { return first + c * step; }
    uint32_t edges = 0;                                   // bit c: piece c lies partly outside
    __device__ __forceinline__ bool any(int c) const { return col(c) < N && (!SHIFT || col(c) + VEC > 0); }
    __device__ __forceinline__ bool all(int c) const { return !SHIFT || (edges >> c & 1u) == 0; }
    __device__ __forceinline__ bool has(int c, int i) const { return unsigned(col(c) + i) < unsigned(N); }
};

template <class T>
__device__ __forceinline__ void join_widen(uint4 w, float (&v)[Join<T>::VEC]) {
    if constexpr (sizeof(T) == 2) {
        v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
        v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z); v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
    } else {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    }
}
template <class T>
__device__ __forceinline__ void join_piece(uint32_t at, float (&v)[Join<T>::VEC]) { join_widen<T>(ptx::lds128(at), v); }
template <class T, class C>
__device__ __forceinline__ void join_store(const C& k, int c, T* row, const float (&v)[Join<T>::VEC]) {
    if (k.all(c)) {
        store_vec<Join<T>::VEC>(row + k.col(c), v);
    } else {
#pragma unroll
        for (int i = 0; i < Join<T>::VEC; ++i)
            if (k.has(c, i)) store_f32(row + k.col(c) + i, v[i]);
    }
}

// Sums over a group's warps in a fixed order.  `red`: two sets of V * 32 floats per group, used in turn, so that
// one barrier per sum suffices.
struct GroupSum {
    float* red; int warps, warp, bar, threads, turn;
    template <int V>
    __device__ __forceinline__ void operator()(float (&v)[V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = warp_sum(v[i]);
        if (warps == 1) return;
        float* r = red + turn * V * 32;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) r[i * 32 + warp] = v[i];
        }
        asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(threads) : "memory");
        float4 s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < warps; w += 4) {              // places of warps that the group does not have stay 0
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float4 p = *reinterpret_cast<const float4*>(r + i * 32 + w);
                s[i].x += p.x; s[i].y += p.y; s[i].z += p.z; s[i].w += p.w;
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (s[i].x + s[i].y) + (s[i].z + s[i].w);
    }
};
constexpr int kJoinRedBytes = 20 * 2 * 3 * 32 * 4;        // 20 groups

// What both passes set up: this thread's group, columns, ring and parameters.  REGS: the parameters of its columns are in
// registers, else in the block's shared memory.
template <class T, int E, bool SHIFT, bool REGS, int IN>
struct JoinThread {
    static constexpr int VEC = Join<T>::VEC, CH = E / VEC;
    int t, group, pieces;
    JoinColumns<T, SHIFT> k;
    uint32_t post_at, pre_at, ring;
    int64_t row, step;                                    // first row, rows between two of this group
    GroupSum sum;
    float post_reg[REGS ? CH : 1][VEC], pre_reg[REGS ? CH : 1][VEC];

    __device__ __forceinline__ JoinThread(const JoinArgs& a, uint8_t* smem) {
        group = int(threadIdx.x) / a.T;
        t = int(threadIdx.x) % a.T;
        pieces = a.T * CH;
        row = int64_t(blockIdx.x) + int64_t(group) * gridDim.x;
        step = int64_t(a.groups) * gridDim.x;
        int shift = 0;
        if (SHIFT) {
            const uintptr_t start = reinterpret_cast<uintptr_t>(a.in[kZ]) / sizeof(T);
            shift = int((start + uint64_t(row) * uint64_t(a.shift_step)) % VEC);
        }
        k.first = t * VEC - shift;
        k.step = a.T * VEC;
        k.N = a.N;
        if (SHIFT) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (k.any(c) && (k.col(c) < 0 || k.col(c) + VEC > a.N)) k.edges |= 1u << c;
        }
        float* red = reinterpret_cast<float*>(smem);
        for (int i = int(threadIdx.x); i < kJoinRedBytes / 4; i += int(blockDim.x)) red[i] = 0.f;
        sum = GroupSum{red + group * 2 * 3 * 32, a.T / 32, t / 32, a.groups == 1 ? 0 : group + 1, a.T, 0};
        post_at = ptx::smem_addr(smem) + kJoinRedBytes;
        pre_at = post_at + uint32_t(pieces) * VEC * 4;
        ring = (REGS ? post_at : pre_at + uint32_t(pieces) * VEC * 4) + uint32_t(group * a.stages * a.arrays) * uint32_t(pieces) * 16;
    }
    __device__ __forceinline__ uint32_t at(const JoinArgs& a, int stage, int m, int c) const {
        return ring + (uint32_t((stage * a.arrays + a.slot[m]) * CH + c) * uint32_t(a.T) + uint32_t(t)) * 16;
    }
    // Starts the copies of row r; always one group of copies, so that waits can count them.
    __device__ __forceinline__ void fetch(const JoinArgs& a, int64_t r, int stage) const {
        if (r < a.M) {
#pragma unroll
            for (int m = 0; m < IN; ++m) {
                if (!a.in[m]) continue;
                const T* p = static_cast<const T*>(a.in[m]) + r * a.ld[m];
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (k.any(c)) copy16(at(a, stage, m, c), p + k.col(c));
            }
        }
        copy_commit();
    }
    // Until the oldest row's copies have landed; what its edge pieces brought from outside the row becomes 0.
    __device__ __forceinline__ void land(const JoinArgs& a, int stage) const {
        copy_wait(a.stages);
        if constexpr (SHIFT) {
            if (k.edges == 0) return;
#pragma unroll 1
            for (int m = 0; m < IN; ++m) {
                if (!a.in[m]) continue;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    if (k.all(c)) continue;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        if (k.has(c, i)) continue;
                        if constexpr (sizeof(T) == 2) ptx::sts_u16(at(a, stage, m, c) + 2 * i, 0);
                        else asm volatile("st.shared.u32 [%0], %1;" ::"r"(at(a, stage, m, c) + 4 * i), "r"(0) : "memory");
                    }
                }
            }
        }
    }
    // gate row * gamma_post and gamma_pre; 0 outside the row.  Shared memory keeps them as planes of float4, so that
    // neighbouring threads read neighbouring 16 bytes.
    __device__ __forceinline__ void load_params(const JoinArgs& a, uint8_t* smem) {
        if constexpr (REGS) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int col = k.col(c) + i;
                    const bool in = k.has(c, i);
                    post_reg[c][i] = in ? param(a.gate_row, col, a.p32) * param(a.gamma_post, col, a.p32) : 0.f;
                    pre_reg[c][i] = in ? param(a.gamma_pre, col, a.p32) : 0.f;
                }
        } else {
            float* q = reinterpret_cast<float*>(smem + kJoinRedBytes);
            const int shift = t * VEC - k.first;
#pragma unroll 4
            for (int e = int(threadIdx.x); e < pieces * VEC; e += int(blockDim.x)) {
                const int col = e - shift, to = (e % VEC / 4 * pieces + e / VEC) * 4 + e % 4;
                const bool in = unsigned(col) < unsigned(a.N);
                q[to] = in ? param(a.gate_row, col, a.p32) * param(a.gamma_post, col, a.p32) : 0.f;
                q[to + pieces * VEC] = in ? param(a.gamma_pre, col, a.p32) : 0.f;
            }
        }
    }
    __device__ __forceinline__ void params(uint32_t base, const float (&reg)[REGS ? CH : 1][VEC], int c, int threads, float (&v)[VEC]) const {
        if constexpr (REGS) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = reg[c][i];
        } else {
#pragma unroll
            for (int j = 0; j < VEC / 4; ++j) {
                const uint4 w = ptx::lds128(base + (j * pieces + c * threads + t) * 16);
                v[4 * j] = __uint_as_float(w.x); v[4 * j + 1] = __uint_as_float(w.y);
                v[4 * j + 2] = __uint_as_float(w.z); v[4 * j + 3] = __uint_as_float(w.w);
            }
        }
    }
    __device__ __forceinline__ void params(uint32_t base, const float (&reg)[REGS ? CH : 1][VEC], int c, int threads, uint64_t (&v)[VEC / 2]) const {
        if constexpr (REGS) {
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) v[i] = ptx::pack_f32x2(reg[c][2 * i], reg[c][2 * i + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < VEC / 4; ++j)
                asm volatile("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(v[2 * j]), "=l"(v[2 * j + 1]) : "r"(base + (j * pieces + c * threads + t) * 16));
        }
    }
    template <class V> __device__ __forceinline__ void post(const JoinArgs& a, int c, V& v) const { params(post_at, post_reg, c, a.T, v); }
    template <class V> __device__ __forceinline__ void pre(const JoinArgs& a, int c, V& v) const { params(pre_at, pre_reg, c, a.T, v); }
    __device__ __forceinline__ void store_zeros(T* row) const {
        float zero[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) zero[i] = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (k.any(c)) join_store<T>(k, c, row, zero);
    }
};

// Elements per thread, with how many threads in a block they go, and where the parameters are.
__host__ __device__ constexpr int join_fwd_threads(int e) { return e == 32 ? 512 : 640; }
__host__ __device__ constexpr bool join_fwd_regs(int e) { return e <= 32; }
__host__ __device__ constexpr bool join_bwd_regs(int e) { return e <= 8; }

template <class T, int E, bool GATED, bool SHIFT>
__global__ void __launch_bounds__(join_fwd_threads(E), 1) join_fwd_kernel(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef JoinThread<T, E, SHIFT, join_fwd_regs(E), kFwdIn> Thread;
    constexpr int VEC = Thread::VEC, CH = Thread::CH;
    Thread th(a, smem);
    pdl_launch();
    pdl_wait();
    for (int s = 0; s < a.stages; ++s) th.fetch(a, th.row + s * th.step, s);
    th.load_params(a, smem);
    __syncthreads();
    const bool post = a.norms & TPPO_NORM_POST, pre = a.norms & TPPO_NORM_PRE;
    const float inv = 1.f / float(a.N);
    int stage = 0;
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
            r1 = rsqrtf(fmaf(s[0], inv, a.eps));
            good = is_finite(s[0]) && is_finite(r1);
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
        if (++stage == a.stages) stage = 0;
        s[0] = q[0] + q[1];
        th.sum(s);
        const float r2 = pre ? rsqrtf(fmaf(s[0], inv, a.eps)) : 1.f;
        good = good && is_finite(s[0]) && is_finite(r2);
        if (th.t == 0) {
            if (a.r_post) a.r_post[r] = good ? r1 : 0.f;
            if (a.r_pre) a.r_pre[r] = good ? r2 : 0.f;
            if (!good && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
        }
        T* ho = static_cast<T*>(a.out[0]) + r * a.ldo[0];
        T* no = static_cast<T*>(a.out[1]) + (pre ? r * a.ldo[1] : 0);
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

// The scalars of a row's backward pass, from its three sums.
struct JoinRow { float r1, r2, k2, k1; bool good; };
__device__ __forceinline__ JoinRow join_row(const JoinArgs& a, float r1, float r2, const float (&s)[3], bool reports) {
    const bool post = a.norms & TPPO_NORM_POST, pre = a.norms & TPPO_NORM_PRE;
    const float inv = 1.f / float(a.N);
    JoinRow w;
    w.r1 = post ? r1 : 1.f;
    w.r2 = pre ? r2 : 0.f;
    w.k2 = pre ? s[0] * inv * r2 * r2 * r2 : 0.f;                         // d = dh + r2 a2 - k2 h
    w.k1 = post ? (s[1] - w.k2 * s[2]) * inv * r1 * r1 * r1 : 0.f;        // dz = r1 a1 - k1 z
    const bool stats = !((post && r1 == 0.f) || (pre && r2 == 0.f));
    w.good = is_finite(s[0]) && is_finite(s[1]) && is_finite(s[2]) && is_finite(w.k2) && is_finite(w.k1);
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

// The fewer threads share a row, the less its sums and copies cost; the registers of 32 columns' gradients then leave room
// for 320 threads.
__host__ __device__ constexpr int join_bwd_threads(int e) { return e == 32 ? 320 : 640; }

template <class T, int E, bool PRE, bool GATED, bool SHIFT>
__global__ void __launch_bounds__(join_bwd_threads(E), 1) join_bwd_kernel(const __grid_constant__ JoinArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    typedef JoinThread<T, E, SHIFT, join_bwd_regs(E), kBwdIn> Thread;
    constexpr int VEC = Thread::VEC, CH = Thread::CH, P = VEC / 2;
    Thread th(a, smem);
    pdl_launch();
    pdl_wait();
    for (int s = 0; s < a.stages; ++s) th.fetch(a, th.row + s * th.step, s);
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
    int stage = 0;
    float r1_next = post && th.row < a.M ? a.r_post[th.row] : 1.f, r2_next = PRE && th.row < a.M ? a.r_pre[th.row] : 0.f;
    for (int64_t r = th.row; r < a.M; r += th.step) {
        const float r1 = r1_next, r2 = r2_next;
        if (r + th.step < a.M) {                          // a row ahead, like the copies
            if (post) r1_next = a.r_post[r + th.step];
            if (PRE) r2_next = a.r_pre[r + th.step];
        }
        th.land(a, stage);
        const uint64_t r2_2 = ptx::pack_f32x2(r2, r2);
        uint64_t q[3] = {0, 0, 0};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!th.k.any(c)) continue;
            uint64_t w[P], d[P], g[P];
            join_piece<T>(th.at(a, stage, kZ, c), w);
            th.post(a, c, g);
#pragma unroll
            for (int i = 0; i < P; ++i) w[i] = mul_f32x2(w[i], g[i]);
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
        const JoinRow w = join_row(a, r1, r2, s, th.t == 0);
        T* dz = static_cast<T*>(a.out[0]) + (a.out[0] ? r * a.ldo[0] : 0);
        T* dres = static_cast<T*>(a.out[1]) + (a.out[1] ? r * a.ldo[1] : 0);
        T* dgate = static_cast<T*>(a.out[2]) + (a.out[2] ? r * a.ldo[2] : 0);
        if (w.good) {
            const uint64_t r1_2 = ptx::pack_f32x2(w.r1, w.r1), k1_2 = ptx::pack_f32x2(-w.k1, -w.k1), k2_2 = ptx::pack_f32x2(-w.k2, -w.k2);
            const uint64_t alpha_2 = ptx::pack_f32x2(a.alpha, a.alpha);
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
                        n[i] = mul_f32x2(n[i], r2_2);
                        sum_pre[c][i] = fma_f32x2(n[i], h[i], sum_pre[c][i]);
                        d[i] = fma_f32x2(k2_2, h[i], fma_f32x2(n[i], g[i], d[i]));
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
                for (int i = 0; i < P; ++i) d[i] = mul_f32x2(d[i], r1_2);
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
                    for (int i = 0; i < P; ++i) v[i] = fma_f32x2(k1_2, z[i], mul_f32x2(d[i], g[i]));
                    join_store<T>(th.k, c, dz, v);
                }
            }
        } else {                                          // the same for the whole group
            if (a.out[0]) th.store_zeros(dz);
            if (a.out[1]) th.store_zeros(dres);
            if (a.out[2]) th.store_zeros(dgate);
        }
        th.fetch(a, r + a.stages * th.step, stage);
        if (++stage == a.stages) stage = 0;
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

// ---- any length and alignment: one block per row, swept once per sum -----------------------------------------
template <int V>
__device__ __forceinline__ void block_sums(float (&v)[V], float* red) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = warp_sum(v[i]);
    __syncthreads();                                      // the previous sums have been read
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) red[i * 32 + (threadIdx.x >> 5)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = 0;
        for (int w = 0; w < kJoinAnyThreads / 32; ++w) v[i] += red[i * 32 + w];
    }
}

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
            r1 = rsqrtf(fmaf(s[0], inv, a.eps));
            good = is_finite(s[0]) && is_finite(r1);
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
        const float r2 = pre ? rsqrtf(fmaf(s[0], inv, a.eps)) : 1.f;
        good = good && is_finite(s[0]) && is_finite(r2);
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

// Backward pass of such rows in two launches: the three sums of every row, then, with no thread depending on another,
// the gradients, a block walking down its strip of columns.  10 elements moved per element of a row instead of 6.
// VEC: columns per access, 16 bytes' worth where all rows start and end on 16-byte boundaries, else 1.
template <class T, int VEC>
__device__ __forceinline__ void join_read(const JoinArgs& a, int m, int64_t r, int c, float otherwise, float (&v)[VEC]) {
    if (a.in[m]) {
        load_vec<VEC>(static_cast<const T*>(a.in[m]) + r * a.ld[m] + c, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = otherwise;
    }
}
template <int VEC>
__device__ __forceinline__ void join_read_params(const void* p, int c, bool f32, float (&v)[VEC]) {
    const bool whole = VEC > 1 && reinterpret_cast<uintptr_t>(p) % 16 == 0;       // 1 where there is none
    if (p && whole && f32) {
        load_vec<VEC>(static_cast<const float*>(p) + c, v);
    } else if (p && whole) {
        load_vec<VEC>(static_cast<const bf16_bits*>(p) + c, v);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = param(p, c + i, f32);
    }
}
template <class T, int VEC>
__global__ void __launch_bounds__(kJoinAnyThreads) join_row_sums_kernel(const __grid_constant__ JoinArgs a) {
    __shared__ float red[3 * 32];
    pdl_launch();
    pdl_wait();
    const bool pre = a.norms & TPPO_NORM_PRE;
    for (int64_t r = blockIdx.x; r < a.M; r += gridDim.x) {
        const float r1 = a.r_post ? a.r_post[r] : 1.f, r2 = a.r_pre ? a.r_pre[r] : 0.f;
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll 2
        for (int c = threadIdx.x * VEC; c < a.N; c += kJoinAnyThreads * VEC) {
            float z[VEC], g[VEC], d[VEC], n[VEC], h[VEC];
            join_read<T, VEC>(a, kZ, r, c, 0.f, z);
            join_read<T, VEC>(a, kGate, r, c, 1.f, g);
            join_read<T, VEC>(a, kDh, r, c, 0.f, d);
            if (pre) {
                join_read<T, VEC>(a, kDn, r, c, 0.f, n);
                join_read<T, VEC>(a, kH, r, c, 0.f, h);
            }
            float gr[VEC], gp[VEC], gn[VEC];
            join_read_params<VEC>(a.gate_row, c, a.p32, gr);
            join_read_params<VEC>(a.gamma_post, c, a.p32, gp);
            join_read_params<VEC>(a.gamma_pre, c, a.p32, gn);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float w = z[i] * (g[i] * gr[i] * gp[i]);
                if (pre) {
                    const float a2 = n[i] * gn[i];
                    s[0] = fmaf(a2, h[i], s[0]);
                    s[2] = fmaf(h[i], w, s[2]);
                    d[i] = fmaf(r2, a2, d[i]);
                }
                s[1] = fmaf(d[i], w, s[1]);
            }
        }
        block_sums(s, red);
        if (threadIdx.x == 0) {
            const JoinRow w = join_row(a, r1, r2, s, true);
            // zeros: a row to leave out
            a.rows[r] = w.good ? make_float4(w.r1, w.r2, w.k1, w.k2) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
}

constexpr int kJoinStrip = 128;                           // threads of a strip
template <class T, int VEC>
__global__ void __launch_bounds__(kJoinStrip) join_columns_kernel(const __grid_constant__ JoinArgs a) {
    pdl_launch();
    pdl_wait();
    const bool pre = a.norms & TPPO_NORM_PRE;
    const int64_t chunk = blockIdx.y, r0 = a.M * chunk / gridDim.y, r1 = a.M * (chunk + 1) / gridDim.y;
    const int64_t at = (int64_t(blockIdx.x) * kJoinStrip + threadIdx.x) * VEC;
    if (at >= a.N) return;
    const int c = int(at);
    float g[VEC], gn[VEC], sum_post[VEC], sum_pre[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        g[i] = param(a.gate_row, c + i, a.p32) * param(a.gamma_post, c + i, a.p32);
        gn[i] = param(a.gamma_pre, c + i, a.p32);
        sum_post[i] = sum_pre[i] = 0;
    }
#pragma unroll 2
    for (int64_t r = r0; r < r1; ++r) {
        const float4 w = __ldcg(a.rows + r);
        float z[VEC], gv[VEC], d[VEC], n[VEC], h[VEC], o[VEC];
        join_read<T, VEC>(a, kZ, r, c, 0.f, z);
        join_read<T, VEC>(a, kGate, r, c, 1.f, gv);
        join_read<T, VEC>(a, kDh, r, c, 0.f, d);
        if (pre) {
            join_read<T, VEC>(a, kDn, r, c, 0.f, n);
            join_read<T, VEC>(a, kH, r, c, 0.f, h);
        }
        const bool good = w.x != 0.f;                     // r1 of a row with statistics is not 0
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            if (pre) {
                const float m = n[i] * w.y;
                if (good) sum_pre[i] = fmaf(m, h[i], sum_pre[i]);
                d[i] = fmaf(-w.w, h[i], fmaf(m, gn[i], d[i]));
            }
            o[i] = good ? a.alpha * d[i] : 0.f;
            d[i] *= w.x;
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
        for (int i = 0; i < VEC; ++i) o[i] = good ? fmaf(-w.z, z[i], d[i] * g[i]) : 0.f;
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
struct JoinSumArgs {
    const float* partial; int64_t rows; int32_t N;
    const void* gate_row; const void* gamma_post;
    void* dgate_row; void* dgamma_post; void* dgamma_pre; int32_t p32;
};
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
        if (a.dgamma_post) put_param(a.dgamma_post, col, a.p32, v * param(a.gate_row, col, a.p32));
        if (a.dgate_row) put_param(a.dgate_row, col, a.p32, v * param(a.gamma_post, col, a.p32));
    } else if (a.dgamma_pre) {
        put_param(a.dgamma_pre, col - a.N, a.p32, v);
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
struct JoinPlan { int E = 0, grid = 0; bool shift = false; size_t smem = 0; };    // E = 0: the kernels for any row

// Groups and stages of a ring kernel for `e` elements per thread; false where it does not fit.
bool join_fit(JoinArgs& a, JoinPlan& p, int e, int vec, int threads, bool regs, int64_t width, bool sums) {
    const int64_t T = (width + 32 * e - 1) / (32 * e) * 32;
    if (T > threads) return false;
    int groups = threads / int(T);
    if (T > 32 && groups > 15) groups = 15;               // hardware barriers
    if (a.M < int64_t(kNumSms) * groups) groups = int((a.M + kNumSms - 1) / kNumSms);
    const int64_t row = T * e / vec * 16;                 // bytes of a matrix' row in a stage
    const int64_t params = (regs ? 0 : T * e * 8) + kJoinRedBytes;
    const int64_t slots = (kJoinSmem - params) / (row * a.arrays);
    if (slots < 1) return false;
    if (groups > 1 && groups > slots / 2) groups = slots / 2 > 1 ? int(slots / 2) : 1;
    a.T = int(T);
    a.groups = groups;
    a.stages = int(slots / groups < kJoinStages ? slots / groups : kJoinStages);
    int64_t blocks = (a.M + groups - 1) / groups;
    if (blocks > kNumSms) blocks = kNumSms;
    // rows that start at changing places of a piece come in classes; a grid of a multiple of eight keeps a block in one
    if (a.shift_step % vec != 0) blocks = blocks <= 144 ? (blocks + 7) / 8 * 8 : 144;
    const int64_t ring = params + row * a.arrays * a.groups * a.stages;
    const int64_t meet = sums ? int64_t(groups - 1) * T * e * 8 + kJoinRedBytes : 0;
    p.E = e;
    p.grid = int(blocks);
    p.smem = size_t(ring > meet ? ring : meet);
    return true;
}
// Of the numbers of elements per thread in `kinds`, the one with the least estimated time per row: instructions of the
// row's warps -- so many per element, some 200 (forward) or 250 per warp for its share of sums, copies and addresses --
// times (1 / warps on the SM + 1 / 20), the time per instruction that was measured with 5, 10 and 20 of them.  At 5120
// columns of bf16 that is 40 elements forward (129 us for 16384 rows; 16: 148, 32: 149, 8: 206) and 16 backward (224;
// 32: 241, 8: 276), with a gate per element 16 (160; 40: 206) and 8 (299; 32: 438, 16: 476), of fp32 16 forward (8192
// rows: 109; 8: 128, 40: 153) and 8 backward (176; 16: 196, 32: 260).  Of equal ones the first.
void join_choose(JoinArgs& a, JoinPlan& p, std::initializer_list<int> kinds, int vec, int64_t width, bool bwd) {
    const JoinArgs given = a;
    const JoinPlan start = p;
    double least = 0;
    for (const int e : kinds) {
        JoinArgs b = given;
        JoinPlan q = start;
        if (!join_fit(b, q, e, vec, bwd ? join_bwd_threads(e) : join_fwd_threads(e), bwd ? join_bwd_regs(e) : join_fwd_regs(e), width, bwd) ||
            b.groups * b.stages < 2)
            continue;
        const int warps = b.T / 32, per = bwd ? (b.in[kGate] ? 36 : 30) : (b.in[kGate] ? 17 : 14) + (e == 32 ? 3 : 0);
        const int fixed = (bwd ? 250 : 200) - (warps == 1 ? 80 : 0);                // a warp by itself needs no barrier
        const double cost = warps * double(per * e + fixed) * (1.0 / (warps * b.groups) + 0.05);
        if (p.E == 0 || cost < least) {
            least = cost;
            a = b;
            p = q;
        }
    }
}
// The columns a row's pieces cover, and whether some lie partly outside it.
int64_t join_width(const JoinArgs& a, JoinPlan& p, int vec) {
    p.shift = a.shift_step % vec != 0 || reinterpret_cast<uintptr_t>(a.in[kZ]) % 16 != 0;
    const int64_t pieces = (int64_t(a.N) + (p.shift ? vec - 1 : 0) + vec - 1) / vec;
    p.shift = p.shift || a.N % vec != 0;
    return pieces * vec;
}

template <class T, int E>
int launch_fwd(const JoinArgs& a, const JoinPlan& p, cudaStream_t s) {
    auto kernel = a.in[kGate] ? (p.shift ? join_fwd_kernel<T, E, true, true> : join_fwd_kernel<T, E, true, false>)
                              : (p.shift ? join_fwd_kernel<T, E, false, true> : join_fwd_kernel<T, E, false, false>);
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kJoinSmem));
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(p.grid), dim3(a.T * a.groups), p.smem, s, a));
    return TPPO_OK;
}
template <class T, int E, bool PRE>
int launch_bwd(const JoinArgs& a, const JoinPlan& p, cudaStream_t s) {
    auto kernel = a.in[kGate] ? (p.shift ? join_bwd_kernel<T, E, PRE, true, true> : join_bwd_kernel<T, E, PRE, true, false>)
                              : (p.shift ? join_bwd_kernel<T, E, PRE, false, true> : join_bwd_kernel<T, E, PRE, false, false>);
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

int64_t join_chunks(int64_t M) { return M < kJoinAnyBlocks ? (M + 7) / 8 * 8 : kJoinAnyBlocks; }

template <class T, int VEC>
int run_bwd_any(JoinArgs& a, JoinSumArgs& sum, cudaStream_t s) {
    TPPO_CUDA_CHECK(launch_dense(join_row_sums_kernel<T, VEC>, dim3(unsigned(a.M < 4 * kNumSms ? a.M : 4 * kNumSms)), dim3(kJoinAnyThreads), 0, s, a));
    // enough chunks of rows to fill the GPU some times over
    const int64_t strips = (int64_t(a.N) + kJoinStrip * VEC - 1) / (kJoinStrip * VEC), most = join_chunks(a.M);
    int64_t chunks = (32 * kNumSms + strips - 1) / strips;
    if (chunks > (a.M + 7) / 8) chunks = (a.M + 7) / 8;
    if (chunks > most) chunks = most;
    sum.rows = chunks;
    TPPO_CUDA_CHECK(launch_dense(join_columns_kernel<T, VEC>, dim3(unsigned(strips), unsigned(chunks)), dim3(kJoinStrip), 0, s, a));
    return TPPO_OK;
}

template <class T>
int run_bwd(JoinArgs& a, bool same, JoinSumArgs& sum, cudaStream_t s) {
    constexpr int vec = Join<T>::VEC;
    JoinPlan p;
    const int64_t width = join_width(a, p, vec);
    const bool whole = same && !p.shift;                  // every row is a number of 16-byte pieces
    if (same) {
        join_choose(a, p, {8, 16, 32}, vec, width, true);
    }
    const bool pre = a.norms & TPPO_NORM_PRE;
    sum.rows = p.grid;
    switch (p.E) {
        case 8: return pre ? launch_bwd<T, 8, true>(a, p, s) : launch_bwd<T, 8, false>(a, p, s);
        case 16: return pre ? launch_bwd<T, 16, true>(a, p, s) : launch_bwd<T, 16, false>(a, p, s);
        case 32: return pre ? launch_bwd<T, 32, true>(a, p, s) : launch_bwd<T, 32, false>(a, p, s);
    }
    return whole ? run_bwd_any<T, vec>(a, sum, s) : run_bwd_any<T, 1>(a, sum, s);
}

bool type_ok(int32_t t) { return t == TPPO_BF16 || t == TPPO_F32; }
size_t size_of(int32_t t) { return t == TPPO_F32 ? 4 : 2; }

// Whether the rows of two matrices start at the same place of a 16-byte piece, row by row.
bool same_start(const void* p, int64_t ldp, const void* q, int64_t ldq, size_t e) {
    if (!p || !q) return true;
    return (reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(q)) % 16 == 0 && ((ldp - ldq) * int64_t(e)) % 16 == 0;
}

}  // namespace

// The rows' scalars in front, the partial column sums behind them.
static size_t join_rows_bytes(int64_t M) { return align_up(size_t(M > 0 ? M : 1) * sizeof(float4), kWsAlign); }
size_t residual_norm_workspace_bytes(int64_t M, int32_t N) {
    if (N <= 0) return 0;
    return join_rows_bytes(M) + align_up(size_t(M > 0 ? join_chunks(M) : 1) * 2 * size_t(N) * sizeof(float), kWsAlign);
}

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
    const bool same = same_start(z, ldz, residual, ldr, e) && same_start(z, ldz, a.in[kGate], ldg, e) && same_start(z, ldz, h, ldh, e) &&
                      same_start(z, ldz, n, ldn, e);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == TPPO_F32 ? run_fwd<float>(a, same, s) : run_fwd<bf16_bits>(a, same, s);
}

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
    a.partial = sums ? reinterpret_cast<float*>(static_cast<char*>(workspace) + join_rows_bytes(M)) : nullptr;
    a.status = status;
    a.M = M; a.N = N; a.alpha = alpha; a.norms = norms;
    a.shift_step = int32_t(ldz % 16);
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
