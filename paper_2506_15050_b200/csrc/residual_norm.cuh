// The residual join: a block's output normed, gated and added to the scaled residual stream, and the sum normed
// for the next block; forward and backward with the parameters' gradients.  With root-mean-square norms,
//     h = alpha * residual + gate * gamma_post * z * r1,   n = h * r2 * gamma_pre
//     d = dh + r2 * (a2 - hh mean(a2 hh)),  a2 = dn * gamma_pre,  hh = h * r2;   dresidual = alpha * d
//     a1 = d * gate * gamma_post,   dz = r1 * (a1 - zz mean(a1 zz)),  zz = z * r1;   dgate = d * zz * gamma_post
//     dgamma_post = sum_rows d * gate * zz,   dgamma_pre = sum_rows dn * hh
// All arithmetic is fp32; each input is read once, each output rounded once.  4 elements move forward and 6
// backward per element of a row (one and two more with a gate per element), so HBM is the bound.
//
// One block per SM, cut into groups of warps that walk rows of their own.  Each thread brings its 16-byte
// pieces of the next rows into a ring of shared memory of its own with cp.async: what it copies only it reads,
// so the ring needs no barrier, and 100-200 KB per SM stay in flight whatever the arithmetic does.  gate *
// gamma_post and gamma_pre stay in registers or shared memory as fp32 for the block's life.
//   [16384, 5120] bf16: forward 122-126 us (5.3-5.5 TB/s, 0.81-0.84 of the measured copy rate), backward 214-225 us (4.5-4.7
//   TB/s); without a gate and the norm in front, "add and norm": 127 and 210 us
//   [8192, 5120] fp32: forward 110-116 us (5.8-6.1 TB/s), backward 167 us (6.0 TB/s)
//
// Forward needs two sums over the row, one behind the other.  Backward takes one: with w = gate gamma_post zz,
//     sum(a1 zz) = sum((dh + r2 a2) w) - r2^2 mean(a2 hh) sum(h w),
// three sums that do not wait for one another, met at one barrier per row.  (The same expansion of sum(h^2) would
// lose all its digits where the block's output cancels the residual, so the forward pass does not use it.)
//
// Rows that do not start on 16-byte boundaries are read by the same aligned pieces, the first and last of which
// hold elements of neighbouring rows or of nothing (a piece with one element of the row in it is mapped), cleared
// when they have arrived, and stored element by element.  A block only takes rows that start at the same place of
// a piece, so that a thread's columns, parameters and column sums stay its own.
// Rows that do not fit, and matrices whose rows do not start at the same place of a piece, are read again for each sweep.
#pragma once

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
    float4* rows;                                         // r1, r2, m1, m2 of every row, where two launches share the work,
    float* params;                                        // and the parameters as they use them: two rows
    int32_t* status;
    int64_t M; int32_t N; float alpha, eps; int32_t norms;
    int32_t T, groups, stages, arrays;                    // threads per group; groups per block; stages; matrices per stage
    int32_t shift_step;                                   // rows start (first row's + r * this) elements into a piece
    int32_t one_ld;                                       // all matrices have the row stride of the first
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
    // This thread's part of a stage, and its place of piece c of matrix m in it.
    __device__ __forceinline__ uint32_t stage_at(const JoinArgs& a, int stage) const {
        return ring + uint32_t(t) * 16 + uint32_t(stage * a.arrays) * uint32_t(CH * a.T * 16);
    }
    __device__ __forceinline__ uint32_t at(const JoinArgs& a, uint32_t stage, int m, int c) const {
        return stage + uint32_t(a.slot[m] * CH + c) * uint32_t(a.T * 16);
    }
    // Starts the copies of row r; always one group of copies, so that waits can count them.
    __device__ __forceinline__ void fetch(const JoinArgs& a, int64_t r, uint32_t stage) const {
        if (r < a.M) {
            const int64_t common = r * a.ld[0] + k.first;
#pragma unroll
            for (int m = 0; m < IN; ++m) {
                if (!a.in[m]) continue;
                const T* p = static_cast<const T*>(a.in[m]) + (a.one_ld ? common : r * a.ld[m] + k.first);
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (k.any(c)) copy16(at(a, stage, m, c), p + c * k.step);
            }
        }
        copy_commit();
    }
    // Row r of an output.
    __device__ __forceinline__ T* out(const JoinArgs& a, int i, int64_t r) const {
        return a.out[i] ? static_cast<T*>(a.out[i]) + r * (a.one_ld ? a.ld[0] : a.ldo[i]) : nullptr;
    }
    // Until the oldest row's copies have landed; what its edge pieces brought from outside the row becomes 0.
    __device__ __forceinline__ void land(const JoinArgs& a, uint32_t stage) const {
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
__host__ __device__ constexpr int join_threads(int e) { return e == 32 ? 512 : e == 24 ? 480 : 640; }
__host__ __device__ constexpr bool join_fwd_regs(int e) { return e <= 32; }
__host__ __device__ constexpr bool join_bwd_regs(int e) { return e <= 8; }

// Sums over a block of kJoinAnyThreads, of the kernels for any length and alignment.
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

// 1 / sqrt(sum / N + eps) of a row's sum of squares, and whether it stands for the row.  A square below fp32's normal
// range is off by up to 2^-150, and so is the mean of many: from 2^-126 on that is a rounding, below it takes bits.
constexpr float kJoinLeastMean = 0x1p-126f;
__device__ __forceinline__ float join_rstd(float sum, float inv, float eps, bool& good) {
    const float mean = fmaf(sum, inv, eps);
    good = good && is_finite(sum) && mean >= kJoinLeastMean;
    return rsqrtf(mean);
}

// ---- host side --------------------------------------------------------------------------------------------------
struct JoinPlan { int E = 0, grid = 0; bool shift = false; size_t smem = 0; };    // E = 0: the kernels for any row

// Groups and stages of a ring kernel for `e` elements per thread; false where it does not fit.
inline bool join_fit(JoinArgs& a, JoinPlan& p, int e, int vec, int threads, bool regs, int64_t width, bool sums) {
    const int64_t T = (width + 32 * e - 1) / (32 * e) * 32;
    if (T > threads) return false;
    int groups = threads / int(T);
    if (T > 32 && groups > 15) groups = 15;               // hardware barriers
    if (a.M < int64_t(kNumSms) * groups) groups = int((a.M + kNumSms - 1) / kNumSms);
    const int64_t row = T * e / vec * 16;                 // bytes of a matrix' row in a stage
    const int64_t params = (regs ? 0 : T * e * 8) + kJoinRedBytes;
    const int64_t slots = (kJoinSmem - params) / (row * a.arrays);
    if (slots < 1) return false;
    if (groups > 1 && groups > slots / 2) groups = slots / 2 > 1 ? int(slots / 2) : slots > 1 ? 2 : 1;
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
// columns of bf16 that was 40 elements forward (129 us for 16384 rows; 16: 148, 32: 149, 8: 206) and 16 backward (224;
// 8: 276, 32 with half the threads 241), with a gate per element 16 (155-160; 40: 206) and 8 (296; 16 with one group 476), of
// fp32 16 forward (8192 rows: 109; 8: 128, 40: 153) and 8 backward (176; 16 with one group 196, with two of a single
// stage 6 % more than 8), and of 5121 bf16 columns 24 backward, two groups of a single stage (311; 16 in one group 406).  Of equal ones the first.
inline void join_choose(JoinArgs& a, JoinPlan& p, std::initializer_list<int> kinds, int vec, int64_t width, bool bwd) {
    const JoinArgs given = a;
    const JoinPlan start = p;
    double least = 0;
    for (const int e : kinds) {
        JoinArgs b = given;
        JoinPlan q = start;
        if (!join_fit(b, q, e, vec, join_threads(e), bwd ? join_bwd_regs(e) : join_fwd_regs(e), width, bwd))
            continue;
        const int warps = b.T / 32, per = bwd ? (b.in[kGate] ? 36 : 30) : (b.in[kGate] ? 17 : 14) + (e == 32 ? 3 : 0);
        const int fixed = (bwd ? 250 : 200) - (warps == 1 ? 80 : 0);                // a warp by itself needs no barrier
        double cost = warps * double(per * e + fixed) * (1.0 / (warps * b.groups) + 0.05);
        if (b.stages == 1) cost *= b.groups == 1 ? 2.5 : 1.35;        // nothing on its way while a row is worked on
        if (p.E == 0 || cost < least) {
            least = cost;
            a = b;
            p = q;
        }
    }
}
// The columns a row's pieces cover, and whether some lie partly outside it.
inline int64_t join_width(const JoinArgs& a, JoinPlan& p, int vec) {
    p.shift = a.shift_step % vec != 0 || reinterpret_cast<uintptr_t>(a.in[kZ]) % 16 != 0;
    const int64_t pieces = (int64_t(a.N) + (p.shift ? vec - 1 : 0) + vec - 1) / vec;
    p.shift = p.shift || a.N % vec != 0;
    return pieces * vec;
}

inline bool type_ok(int32_t t) { return t == TPPO_BF16 || t == TPPO_F32; }
inline size_t size_of(int32_t t) { return t == TPPO_F32 ? 4 : 2; }

// Whether the rows of two matrices start at the same place of a 16-byte piece, row by row.
inline bool same_start(const void* p, int64_t ldp, const void* q, int64_t ldq, size_t e) {
    if (!p || !q) return true;
    return (reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(q)) % 16 == 0 && ((ldp - ldq) * int64_t(e)) % 16 == 0;
}

}  // namespace
}  // namespace tppo
