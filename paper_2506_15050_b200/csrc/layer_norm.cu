// Layer norm over the rows of a matrix, forward and backward with the reduction of the weight's and
// the bias' gradients:
//     y  = (x - mean) * rstd * gamma + beta,      rstd = 1 / sqrt(mean((x - mean)^2) + eps)
//     dx = rstd * (a - mean(a) - h * mean(a * h)),   h = (x - mean) * rstd,  a = dy * gamma
//     dgamma = sum_rows dy * h,   dbeta = sum_rows dy
// All arithmetic is fp32; the inputs are read once and the outputs rounded once.
//
// Both passes have 2 resp. 3 elements to move per element, and fp32 rows are bound by that.  Of bf16 rows an
// element costs some 12 instructions forward and 25 backward, and what the SM has resident waits together:
// backward at 5120 columns one block of 640 threads, at one barrier per trip (61 % of the issue slots used,
// fixed latency first among the stalls).  Long rows are brought in by bulk (TMA) copies through a ring of
// shared memory, which keeps 100-200 KB per SM in flight while blocks go from row to row; short rows are
// loaded into the registers of one or a few warps.  The sums of gamma and beta stay in the registers of a
// block's threads for its whole walk over the rows; each block writes one partial row of them to the
// workspace and a second kernel adds those in a fixed order, so the gradients do not depend on scheduling.
// Rows too long for either way take kernels that read the row again from L2.
//   [16384, 5120] bf16: forward 62-64 us (5.3 TB/s, 0.81 of the measured copy rate), backward 109-112 us (4.5 TB/s)
//   [16384, 5120] fp32: forward 107 us (6.3 TB/s), backward 168 us (6.0 TB/s)
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
    int32_t stages;           // ring kernel
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

// ---- rows fed by bulk copies --------------------------------------------------------------------
// The arithmetic of these kernels runs on pairs of fp32 values in 64-bit registers: fewer instructions, though
// plain floats take the same time within 3 %.
typedef uint64_t f32x2;
__device__ __forceinline__ f32x2 twice(float v) { return ptx::pack_f32x2(v, v); }
__device__ __forceinline__ float pair_sum(f32x2 v) {
    float lo, hi;
    ptx::unpack_f32x2(v, lo, hi);
    return lo + hi;
}
// How a thread meets its columns.  RowVec: rows of 16-byte aligned 16-byte pieces.  RowAny: rows at any
// element, copied with the 16-byte granules they touch; a piece is two columns `group` apart, loaded and
// stored one element at a time.
template <class T> struct RowVec {
    typedef T Elem;
    static constexpr bool kAny = false;
    static constexpr int kVec = 16 / int(sizeof(T)), kPairs = kVec / 2;
    __device__ __forceinline__ static int col(int c, int group, int t) { return (c * group + t) * kVec; }
    // pairs of columns from `col` of the row whose first element is at shared address `row`
    __device__ __forceinline__ static void load(uint32_t row, int col, int, int, f32x2 (&v)[kPairs]) {
        widen(ptx::lds128(row + col * uint32_t(sizeof(T))), v);
    }
    __device__ __forceinline__ static void widen(const uint4& w, f32x2 (&v)[kPairs]) {
        if constexpr (kVec == 8) {
            v[0] = ptx::pack_f32x2(bf16_lo(w.x), bf16_hi(w.x));
            v[1] = ptx::pack_f32x2(bf16_lo(w.y), bf16_hi(w.y));
            v[2] = ptx::pack_f32x2(bf16_lo(w.z), bf16_hi(w.z));
            v[3] = ptx::pack_f32x2(bf16_lo(w.w), bf16_hi(w.w));
        } else {
            v[0] = ptx::pack_f32x2(__uint_as_float(w.x), __uint_as_float(w.y));
            v[1] = ptx::pack_f32x2(__uint_as_float(w.z), __uint_as_float(w.w));
        }
    }
    __device__ __forceinline__ static void store(T* row, int col, int, int, const f32x2 (&v)[kPairs]) {
        if constexpr (kVec == 8) {
            *reinterpret_cast<uint4*>(row + col) =
                make_uint4(ptx::pack_bf16x2_from_f32x2(v[0]), ptx::pack_bf16x2_from_f32x2(v[1]),
                           ptx::pack_bf16x2_from_f32x2(v[2]), ptx::pack_bf16x2_from_f32x2(v[3]));
        } else {
            float4 o;
            ptx::unpack_f32x2(v[0], o.x, o.y);
            ptx::unpack_f32x2(v[1], o.z, o.w);
            *reinterpret_cast<float4*>(row + col) = o;
        }
    }
    template <class P>
    __device__ __forceinline__ static void params(const P* p, int col, int, int, float otherwise, f32x2 (&v)[kPairs]) {
        float f[kVec];
        load_params<kVec>(p, col, otherwise, f);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = ptx::pack_f32x2(f[2 * i], f[2 * i + 1]);
    }
    // gamma as fp32 in shared memory
    __device__ __forceinline__ static void gamma(uint32_t gam, int col, int, int, f32x2 (&g)[kPairs]) {
#pragma unroll
        for (int i = 0; i < kPairs; i += 2) {
            const uint4 w = ptx::lds128(gam + (col + 2 * i) * 4);
            g[i] = ptx::pack_f32x2(__uint_as_float(w.x), __uint_as_float(w.y));
            g[i + 1] = ptx::pack_f32x2(__uint_as_float(w.z), __uint_as_float(w.w));
        }
    }
    // the pair (v, v) as far as its columns exist, else 0
    __device__ __forceinline__ static f32x2 where(int, int, int, float v) { return twice(v); }
    __device__ __forceinline__ static void put(float* row, int col, int, int, const f32x2 (&v)[kPairs]) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            float2 w;
            ptx::unpack_f32x2(v[i], w.x, w.y);
            *reinterpret_cast<float2*>(row + col + 2 * i) = w;
        }
    }
    __host__ __device__ static uint32_t pitch(int N) { return uint32_t(N) * sizeof(T); }
};
template <class T> struct RowAny {
    typedef T Elem;
    static constexpr bool kAny = true;
    static constexpr int kVec = 2, kPairs = 1;
    __device__ __forceinline__ static float element(uint32_t at) {
        if constexpr (sizeof(T) == 2) return __uint_as_float(uint32_t(ptx::lds_u16(at)) << 16);
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
        return v;
    }
    __device__ __forceinline__ static int col(int c, int group, int t) { return c * 2 * group + t; }
    __device__ __forceinline__ static void load(uint32_t row, int col, int group, int N, f32x2 (&v)[1]) {
        const float lo = element(row + col * uint32_t(sizeof(T)));
        v[0] = ptx::pack_f32x2(lo, col + group < N ? element(row + (col + group) * uint32_t(sizeof(T))) : 0.f);
    }
    __device__ __forceinline__ static void store(T* row, int col, int group, int N, const f32x2 (&v)[1]) {
        float lo, hi;
        ptx::unpack_f32x2(v[0], lo, hi);
        store_f32(row + col, lo);
        if (col + group < N) store_f32(row + col + group, hi);
    }
    template <class P>
    __device__ __forceinline__ static void params(const P* p, int col, int group, int N, float otherwise, f32x2 (&v)[1]) {
        v[0] = ptx::pack_f32x2(p ? load_f32(p + col) : otherwise, col + group < N ? (p ? load_f32(p + col + group) : otherwise) : 0.f);
    }
    __device__ __forceinline__ static void gamma(uint32_t gam, int col, int group, int N, f32x2 (&g)[1]) {
        float lo, hi = 0.f;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(lo) : "r"(gam + col * 4));
        if (col + group < N) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(hi) : "r"(gam + (col + group) * 4));
        g[0] = ptx::pack_f32x2(lo, hi);
    }
    __device__ __forceinline__ static f32x2 where(int col, int group, int N, float v) {
        return ptx::pack_f32x2(v, col + group < N ? v : 0.f);
    }
    __device__ __forceinline__ static void put(float* row, int col, int group, int N, const f32x2 (&v)[1]) {
        float lo, hi;
        ptx::unpack_f32x2(v[0], lo, hi);
        row[col] = lo;
        if (col + group < N) row[col + group] = hi;
    }
    __host__ __device__ static uint32_t pitch(int N) { return (uint32_t(N) * sizeof(T) + 15 + 15) / 16 * 16; }
};

// A matrix whose rows are copied to shared memory.
template <class Q> struct RowSource {
    const typename Q::Elem* p; int64_t ld, M; int32_t N;

    // shared address of row r's first element, given where its copy starts
    __device__ __forceinline__ uint32_t first(int64_t r, uint32_t at) const {
        return Q::kAny ? at + uint32_t(reinterpret_cast<uintptr_t>(p + r * ld) & 15) : at;
    }
    // Bytes of row r that a bulk copy brings, and where they start.  RowAny: whole granules, those
    // at the matrix' two ends only as far as they lie inside it.
    __device__ __forceinline__ uint32_t span(int64_t r, uintptr_t& lo) const {
        const uintptr_t begin = reinterpret_cast<uintptr_t>(p + r * ld), end = begin + uintptr_t(N) * sizeof(*p);
        lo = begin;
        if (!Q::kAny) return uint32_t(end - begin);
        lo = begin & ~uintptr_t(15);
        uintptr_t hi = (end + 15) & ~uintptr_t(15);
        if (r == 0 && lo < begin) lo += 16;
        if (r == M - 1 && hi > end) hi -= 16;
        return hi > lo ? uint32_t(hi - lo) : 0u;
    }
    // Called by one thread: the elements of row r that no bulk copy brings, then (after the barrier has
    // been told) the copy itself.
    __device__ __forceinline__ void edges(int64_t r, uint32_t at) const {
        if (!Q::kAny || (r != 0 && r != M - 1)) return;
        uintptr_t lo;
        const uint32_t bytes = span(r, lo);
        const uintptr_t begin = reinterpret_cast<uintptr_t>(p + r * ld), hi = lo + bytes;
        for (int c = 0; c < N; ++c) {
            const uintptr_t q = begin + uintptr_t(c) * sizeof(*p);
            if (bytes > 0 && q >= lo && q < hi) { c += int((hi - q) / sizeof(*p)) - 1; continue; }
            const uint32_t to = first(r, at) + uint32_t(c) * uint32_t(sizeof(*p));
            if constexpr (sizeof(*p) == 2) ptx::sts_u16(to, *reinterpret_cast<const uint16_t*>(q));
            else asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(*reinterpret_cast<const float*>(q)) : "memory");
        }
        // the stage's next row is written by a bulk copy of this thread: another proxy, ordered behind these stores
        ptx::fence_proxy_async_smem();
    }
    __device__ __forceinline__ void copy(int64_t r, uint32_t at, uint32_t bar) const {
        uintptr_t lo;
        const uint32_t bytes = span(r, lo);
        const uintptr_t begin = reinterpret_cast<uintptr_t>(p + r * ld) & ~uintptr_t(15);
        if (bytes > 0) ptx::bulk_load(at + uint32_t(lo - (Q::kAny ? begin : lo)), reinterpret_cast<const void*>(lo), bytes, bar);
    }
    __device__ __forceinline__ uint32_t bytes(int64_t r) const {
        uintptr_t lo;
        return span(r, lo);
    }
};

constexpr size_t kRingSmem = 220 * 1024;       // of all blocks on an SM together
// What the ring kernels may be launched with.  A function's limit is state of the device that all calls share:
// it is set to the same value every time, since another host thread may be about to launch with more than
// this call needs.
constexpr int kRingLimit = int(kRingSmem) + 128;
constexpr int kRingThreads = 512;
constexpr int kRingWarps = kRingThreads / 32;
// Sum of one float per warp, in warp order, read by every thread itself (entries past the block's warps
// are 0).
__device__ __forceinline__ float ring_sum(const float* red, int warps) {
    float s = 0.f;
    for (int w = 0; w < warps; w += 4) {
        const float4 v = *reinterpret_cast<const float4*>(red + w);
        s += (v.x + v.y) + (v.z + v.w);
    }
    return s;
}

// A wait that ran out is not repeated: the rows are then garbage, and flagged.  Where it was the issuing
// thread's, no further copy is issued, and before the block's memory goes away those in flight are awaited
// here, each within the limit again: one stage per `step` rows, from row `lost` on, which was the one waited
// for.  (`lost` is in shared memory and read behind the loop: a call or a register inside it costs up to 6 %.)
__device__ __forceinline__ void ring_drain(uint32_t full, int stages, int64_t lost, int64_t step, int64_t M) {
    const int64_t trip = (lost - int64_t(blockIdx.x)) / step;
    int stage = int(trip % stages);
    uint32_t phase = uint32_t(trip / stages) & 1u;
    for (int k = 0; k < stages && lost < M; ++k, lost += step) {
        if (!ptx::mbar_wait<false>(full + 8 * stage, phase)) return;
        if (++stage == stages) { stage = 0; phase ^= 1u; }
    }
}

// Forward: a block per row, rows brought in `stages` ahead; gamma and beta stay in registers.
template <class Q, class P, int CH>
__global__ void __launch_bounds__(kRingThreads) norm_fwd_ring_kernel(const NormFwdArgs a) {
    typedef typename Q::Elem T;
    constexpr int PAIRS = Q::kPairs;
    extern __shared__ __align__(128) uint8_t ring[];     // [stages] rows, then one barrier per stage
    __shared__ __align__(16) float red[2][kRingWarps];
    __shared__ int64_t lost;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, warps = blockDim.x >> 5;
    const uint32_t pitch = Q::pitch(a.N);
    const uint32_t base = ptx::smem_addr(ring), full = base + a.stages * pitch;
    const float inv_n = 1.f / float(a.N);
    const int64_t step = gridDim.x;
    const RowSource<Q> x{static_cast<const T*>(a.x), a.ldx, a.M, a.N};
    auto issue = [&](int64_t r, int s) {
        x.edges(r, base + s * pitch);
        ptx::mbar_arrive_expect_tx(full + 8 * s, x.bytes(r));
        x.copy(r, base + s * pitch, full + 8 * s);
    };
    if (t < 2 * kRingWarps) (&red[0][0])[t] = 0.f;
    if (t == 0) {
        lost = -1;
        for (int s = 0; s < a.stages; ++s) ptx::mbar_init(full + 8 * s, 1);
        ptx::fence_mbar_init_cluster();
    }
    pdl_launch();
    pdl_wait();
    if (t == 0)
        for (int s = 0; s < a.stages && blockIdx.x + s * step < a.M; ++s) issue(blockIdx.x + s * step, s);
    f32x2 g[CH][PAIRS], b[CH][PAIRS];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = Q::col(c, a.group, t);
        if (col < a.N) {
            Q::params(static_cast<const P*>(a.gamma), col, a.group, a.N, 1.f, g[c]);
            Q::params(static_cast<const P*>(a.beta), col, a.group, a.N, 0.f, b[c]);
        }
    }
    __syncthreads();
    int stage = 0;
    uint32_t phase = 0;
    bool timed_out = false;
    for (int64_t r = blockIdx.x; r < a.M; r += step) {
        if (!timed_out) timed_out = !ptx::mbar_wait<false>(full + 8 * stage, phase);
        if (timed_out && t == 0 && lost < 0) lost = r;
        f32x2 v[CH][PAIRS], s = 0;
        const uint32_t at = x.first(r, base + stage * pitch);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = Q::col(c, a.group, t);
            if (col < a.N) {
                Q::load(at, col, a.group, a.N, v[c]);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) s = ptx::add_f32x2(s, v[c][i]);
            }
        }
        float sum = warp_sum(pair_sum(s));
        if (lane == 0) red[0][warp] = sum;
        __syncthreads();                          // the sums are there, and the stage has been read
        if (t == 0 && !timed_out && r + a.stages * step < a.M) issue(r + a.stages * step, stage);
        if (++stage == a.stages) { stage = 0; phase ^= 1u; }
        // one step on the residual (Markstein's correction of a quotient): sum * (1 / N) alone may miss the value of a
        // row that holds nothing else
        const float total = ring_sum(red[0], warps), about = total * inv_n;
        const float mean = fmaf(fmaf(-about, float(a.N), total), inv_n, about);
        s = 0;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = Q::col(c, a.group, t);
            if (col < a.N) {
                const f32x2 minus = Q::where(col, a.group, a.N, -mean);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    v[c][i] = ptx::add_f32x2(v[c][i], minus);
                    s = ptx::fma_f32x2(v[c][i], v[c][i], s);
                }
            }
        }
        sum = warp_sum(pair_sum(s));
        if (lane == 0) red[1][warp] = sum;
        __syncthreads();
        const float var = ring_sum(red[1], warps) * inv_n;
        const float rstd = rsqrtf(var + a.eps);
        const bool good = is_finite(var) && is_finite(rstd);        // see norm_fwd_kernel
        if (t == 0) {
            if (a.mean) a.mean[r] = good ? mean : 0.f;
            if (a.rstd) a.rstd[r] = good ? rstd : 0.f;
            if (!good && a.status) atomicOr(a.status, TPPO_DEV_NONFINITE);
        }
        T* y = static_cast<T*>(a.y) + r * a.ldy;
        const f32x2 scale = twice(rstd);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = Q::col(c, a.group, t);
            if (col < a.N) {
                f32x2 o[PAIRS];
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) o[i] = 0;
                if (good) {
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) o[i] = ptx::fma_f32x2(ptx::mul_f32x2(v[c][i], scale), g[c][i], b[c][i]);
                }
                Q::store(y, col, a.group, a.N, o);
            }
        }
    }
    if (timed_out) {
        if (t == 0) ring_drain(full, a.stages, lost, step, a.M);
        if (a.status) atomicOr(a.status, TPPO_DEV_WAIT_TIMEOUT);
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

// Aligned rows, one phase: a block takes ROWS rows at a time out of a ring of shared memory that bulk
// copies fill `stages` such groups of rows ahead, one barrier for each group (one per row keeps the compiler
// from loading a row while it waits for the next: 72 us instead of 47 for 16384 x 2048); every thread keeps its columns of x - mean (and of dy, as loaded) from
// the sums to the results, and one barrier serves all rows of a trip.
template <class T, class P, int CH, int ROWS, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_bwd_rows_kernel(const NormBwdArgs a) {
    typedef RowVec<T> Q;
    constexpr int PAIRS = Q::kPairs, VALUES = 2 * ROWS;
    extern __shared__ __align__(128) uint8_t ring[];     // [stages][ROWS][x row, dy row], then one barrier per stage
    __shared__ float red[2][20][VALUES];
    __shared__ int64_t lost;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, warps = blockDim.x >> 5;
    const uint32_t row_bytes = uint32_t(a.N) * sizeof(T), stage_bytes = ROWS * 2 * row_bytes;
    const uint32_t base = ptx::smem_addr(ring), full = base + a.stages * stage_bytes;
    const float inv_n = 1.f / float(a.N);
    const int64_t step = gridDim.x;
    const P* gamma = static_cast<const P*>(a.gamma);
    // by the first warp: rows r0, r0 + step, .. into stage s, a lane per copy
    auto issue = [&](int64_t r0, int s) {
        if (r0 >= a.M) return;
        const uint32_t bar = full + 8 * s;
        const int64_t r = r0 + (lane >> 1) * step;
        const bool mine = lane < 2 * ROWS && r < a.M;
        const uint32_t copies = __popc(__ballot_sync(0xffffffffu, mine));
        if (lane == 0) ptx::mbar_arrive_expect_tx(bar, copies * row_bytes);
        __syncwarp();
        if (mine)
            ptx::bulk_load(base + s * stage_bytes + lane * row_bytes,
                           lane & 1 ? static_cast<const T*>(a.dy) + r * a.lddy : static_cast<const T*>(a.x) + r * a.ldx, row_bytes, bar);
    };
    if (t == 0) {
        lost = -1;
        for (int s = 0; s < a.stages; ++s) ptx::mbar_init(full + 8 * s, 1);
        ptx::fence_mbar_init_cluster();
    }
    pdl_launch();
    pdl_wait();
    if (warp == 0) {
        __syncwarp();
        for (int s = 0; s < a.stages; ++s) issue(blockIdx.x + s * ROWS * step, s);
    }
    f32x2 dg[CH][PAIRS], db[CH][PAIRS], g[CH][PAIRS];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = Q::col(c, a.group, t);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) dg[c][i] = db[c][i] = 0;
        if (col < a.N) Q::params(gamma, col, a.group, a.N, 1.f, g[c]);
    }
    __syncthreads();
    int stage = 0, flip = 0;
    uint32_t phase = 0;
    bool timed_out = false;
    float next_mean[ROWS], next_rstd[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int64_t r = blockIdx.x + k * step;
        next_mean[k] = r < a.M ? a.mean[r] : 0.f;
        next_rstd[k] = r < a.M ? a.rstd[r] : 0.f;
    }
    for (int64_t r0 = blockIdx.x; r0 < a.M; r0 += ROWS * step, flip ^= 1) {
        float mean[ROWS], rstd[ROWS], part[VALUES];
        uint4 raw[ROWS][CH];
        f32x2 e[ROWS][CH][PAIRS];                // x - mean
        if (!timed_out) timed_out = !ptx::mbar_wait_warp<false>(full + 8 * stage, phase);   // one answer per warp: the first issues
        const uint32_t here = base + stage * stage_bytes;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t r = r0 + k * step, ahead = r + ROWS * step;
            mean[k] = next_mean[k];
            rstd[k] = next_rstd[k];
            if (ahead < a.M) { next_mean[k] = a.mean[ahead]; next_rstd[k] = a.rstd[ahead]; }
            f32x2 s = 0, q = 0;                   // sum of a, sum of a e
            if (r < a.M) {
                const f32x2 minus = twice(-mean[k]);
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const int col = Q::col(c, a.group, t);
                    if (col < a.N) {
                        const uint32_t at = here + k * 2 * row_bytes + col * uint32_t(sizeof(T));
                        f32x2 d[PAIRS];
                        raw[k][c] = ptx::lds128(at + row_bytes);
                        Q::widen(ptx::lds128(at), e[k][c]);
                        Q::widen(raw[k][c], d);
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) {
                            const f32x2 av = ptx::mul_f32x2(d[i], g[c][i]);
                            e[k][c][i] = ptx::add_f32x2(e[k][c][i], minus);
                            s = ptx::add_f32x2(s, av);
                            q = ptx::fma_f32x2(av, e[k][c][i], q);
                        }
                    }
                }
            }
            part[2 * k] = pair_sum(s);
            part[2 * k + 1] = pair_sum(q) * rstd[k];
        }
        float total = warp_sum_many<VALUES>(part);            // of value lane % VALUES
        if (lane < VALUES) red[flip][warp][lane] = total;
        __syncthreads();                          // the partial sums are there, and the stage has been read
        if (warp == 0) {
            if (!timed_out) issue(r0 + int64_t(a.stages) * ROWS * step, stage);
            else if (t == 0 && lost < 0) lost = r0;
        }
        if (++stage == a.stages) { stage = 0; phase ^= 1u; }
        total = 0.f;
        for (int w = lane / VALUES; w < warps; w += 32 / VALUES) total += red[flip][w][lane % VALUES];
#pragma unroll
        for (int o = VALUES; o < 32; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t r = r0 + k * step;
            const float c1 = __shfl_sync(0xffffffffu, total, 2 * k) * inv_n;
            const float c2 = __shfl_sync(0xffffffffu, total, 2 * k + 1) * inv_n;
            if (r >= a.M) continue;
            const bool good = norm_row_good(c1, c2, rstd[k], t == 0, a.status);
            const f32x2 scale = twice(rstd[k]), u = twice(-rstd[k] * c1), v = twice(-rstd[k] * c2);
            T* dx = a.dx ? static_cast<T*>(a.dx) + r * a.lddx : nullptr;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = Q::col(c, a.group, t);
                if (col < a.N) {
                    f32x2 d[PAIRS];
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) d[i] = 0;
                    if (good) {
                        Q::widen(raw[k][c], d);
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) {
                            const f32x2 h = ptx::mul_f32x2(e[k][c][i], scale);
                            dg[c][i] = ptx::fma_f32x2(d[i], h, dg[c][i]);
                            db[c][i] = ptx::add_f32x2(db[c][i], d[i]);
                            d[i] = ptx::fma_f32x2(ptx::mul_f32x2(d[i], g[c][i]), scale, ptx::fma_f32x2(h, v, u));
                        }
                    }
                    if (dx) Q::store(dx, col, a.group, a.N, d);
                }
            }
        }
    }
    if (timed_out) {
        if (t == 0) ring_drain(full, a.stages, lost, ROWS * step, a.M);
        if (a.status) atomicOr(a.status, TPPO_DEV_WAIT_TIMEOUT);
    }
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.x) * 2 * a.N;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = Q::col(c, a.group, t);
        if (col < a.N) {
            Q::put(out, col, a.group, a.N, dg[c]);
            Q::put(out + a.N, col, a.group, a.N, db[c]);
        }
    }
}

// Rows that one phase does not hold in registers -- aligned ones of more than 8192 columns -- or that are not
// 16-byte aligned: a block takes two rows at a time out of a ring of shared memory that bulk copies fill
// `stages` rows ahead, in two phases:
//   sums    half of the block's warps on each row, lanes along it: sum a and sum a (x - mean)
//   finish  every thread its CH pieces of columns of both rows: column sums (in registers for the whole
//           walk) and dx
// Both phases read the row from shared memory.  Where the registers have the room, one phase with one barrier
// for several rows is faster (the table in norm_bwd_typed: 47 us against 106 for 16384 x 2048).
template <class Q, class P, int CH>
__global__ void __launch_bounds__(CH * Q::kVec > 16 ? 512 : 640) norm_bwd_ring_kernel(const NormBwdArgs a) {
    typedef typename Q::Elem T;
    constexpr int PAIRS = Q::kPairs;
    extern __shared__ __align__(128) uint8_t ring[];     // [stages][x row, dy row], one barrier per stage, gamma as fp32
    __shared__ float2 red[2][10];                        // [row][warp of its half]
    __shared__ float2 stat[2][2];                        // [trip parity][row] mean, rstd
    __shared__ int64_t lost;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, half = int(blockDim.x) >> 6;   // warps per row
    const uint32_t pitch = Q::pitch(a.N), stage_bytes = 2 * pitch;
    const uint32_t base = ptx::smem_addr(ring), full = base + a.stages * stage_bytes, gam = full + 8 * 16;
    const float inv_n = 1.f / float(a.N);
    const int64_t step = gridDim.x;
    const int rows = a.stages > 1 ? 2 : 1;               // per trip
    const RowSource<Q> sx{static_cast<const T*>(a.x), a.ldx, a.M, a.N}, sd{static_cast<const T*>(a.dy), a.lddy, a.M, a.N};
    auto issue = [&](int64_t r, int s) {
        const uint32_t bar = full + 8 * s, at = base + s * stage_bytes;
        sx.edges(r, at);
        sd.edges(r, at + pitch);
        ptx::mbar_arrive_expect_tx(bar, sx.bytes(r) + sd.bytes(r));
        sx.copy(r, at, bar);
        sd.copy(r, at + pitch, bar);
    };
    if (t == 0) {
        lost = -1;
        for (int s = 0; s < a.stages; ++s) ptx::mbar_init(full + 8 * s, 1);
        ptx::fence_mbar_init_cluster();
    }
    pdl_launch();
    pdl_wait();
    if (t == 0)
        for (int s = 0; s < a.stages && blockIdx.x + s * step < a.M; ++s) issue(blockIdx.x + s * step, s);
    for (int c = t; c < a.N; c += blockDim.x) {
        const float v = a.gamma ? load_f32(static_cast<const P*>(a.gamma) + c) : 1.f;
        asm volatile("st.shared.f32 [%0], %1;" ::"r"(gam + c * 4), "f"(v) : "memory");
    }
    auto load_stat = [&](int64_t r, int slot) {
        stat[slot][t] = r < a.M ? make_float2(a.mean[r], a.rstd[r]) : make_float2(0.f, 0.f);
    };
    if (t < rows) load_stat(blockIdx.x + t * step, 0);
    f32x2 dg[CH][PAIRS], db[CH][PAIRS];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) dg[c][i] = db[c][i] = 0;
    __syncthreads();
    int stage = 0, flip = 0;
    uint32_t phase = 0;
    bool timed_out = false;
    const int mine = warp >= half ? 1 : 0, part = warp - mine * half;
    for (int64_t r0 = blockIdx.x; r0 < a.M; r0 += rows * step, flip ^= 1) {
        const bool two = rows == 2 && r0 + step < a.M;        // the last trip may have one row
        const int stage1 = stage + 1 == a.stages ? 0 : stage + 1;
        const uint32_t phase1 = stage + 1 == a.stages ? phase ^ 1u : phase;
        if (t < rows) load_stat(r0 + (rows + t) * step, flip ^ 1);
        // sums
        if (part < half && (mine == 0 || two)) {
            const int st = mine ? stage1 : stage;
            if (!timed_out) timed_out = !ptx::mbar_wait<false>(full + 8 * st, mine ? phase1 : phase);
            const float2 ms = stat[flip][mine];
            const f32x2 minus = twice(-ms.x);
            const int64_t r = r0 + mine * step;
            const uint32_t ax = sx.first(r, base + st * stage_bytes), ad = sd.first(r, base + st * stage_bytes + pitch);
            f32x2 s = 0, q = 0;
            // the warps of a row stand side by side as the block's threads do for their columns
#pragma unroll 4
            for (int c = 0; Q::col(c, half * 32, part * 32 + lane) < a.N; ++c) {
                const int col = Q::col(c, half * 32, part * 32 + lane);
                f32x2 x[PAIRS], d[PAIRS], g[PAIRS];
                Q::load(ax, col, half * 32, a.N, x);
                Q::load(ad, col, half * 32, a.N, d);
                Q::gamma(gam, col, half * 32, a.N, g);
#pragma unroll
                for (int i = 0; i < PAIRS; ++i) {
                    const f32x2 av = ptx::mul_f32x2(d[i], g[i]);
                    s = ptx::add_f32x2(s, av);
                    q = ptx::fma_f32x2(av, ptx::add_f32x2(x[i], minus), q);
                }
            }
            float v[2] = {pair_sum(s), pair_sum(q) * ms.y};
            const float sum = warp_sum_many<2>(v);
            const float other = __shfl_sync(0xffffffffu, sum, 1);
            if (lane == 0) red[mine][part] = make_float2(sum, other);
        }
        __syncthreads();
        // finish
#pragma unroll 1
        for (int k = 0; k < (two ? 2 : 1); ++k) {
            const int st = k ? stage1 : stage;
            if (!timed_out) timed_out = !ptx::mbar_wait<false>(full + 8 * st, k ? phase1 : phase);   // done: the sums waited
            const float2 ms = stat[flip][k];
            float c1 = 0.f, c2 = 0.f;
            for (int w = 0; w < half; ++w) {
                c1 += red[k][w].x;
                c2 += red[k][w].y;
            }
            c1 *= inv_n;
            c2 *= inv_n;
            const bool good = norm_row_good(c1, c2, ms.y, t == 0, a.status);
            const f32x2 minus = twice(-ms.x), scale = twice(ms.y), u = twice(-ms.y * c1), v = twice(-ms.y * c2);
            T* dx = a.dx ? static_cast<T*>(a.dx) + (r0 + k * step) * a.lddx : nullptr;
            const int64_t r = r0 + k * step;
            const uint32_t ax = sx.first(r, base + st * stage_bytes), ad = sd.first(r, base + st * stage_bytes + pitch);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = Q::col(c, a.group, t);
                if (col < a.N) {
                    f32x2 x[PAIRS], d[PAIRS], g[PAIRS];
                    if (good) {
                        Q::load(ax, col, a.group, a.N, x);
                        Q::load(ad, col, a.group, a.N, d);
                        Q::gamma(gam, col, a.group, a.N, g);
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) {
                            const f32x2 h = ptx::mul_f32x2(ptx::add_f32x2(x[i], minus), scale);
                            dg[c][i] = ptx::fma_f32x2(d[i], h, dg[c][i]);
                            db[c][i] = ptx::add_f32x2(db[c][i], d[i]);
                            d[i] = ptx::fma_f32x2(ptx::mul_f32x2(d[i], g[i]), scale, ptx::fma_f32x2(h, v, u));
                        }
                        if (dx) Q::store(dx, col, a.group, a.N, d);
                    } else if (dx) {
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) d[i] = 0;
                        Q::store(dx, col, a.group, a.N, d);
                    }
                }
            }
        }
        __syncthreads();                          // both stages have been read, and `red`
        if (t == 0) {
            if (!timed_out) {
                if (r0 + a.stages * step < a.M) issue(r0 + a.stages * step, stage);
                if (rows == 2 && r0 + (a.stages + 1) * step < a.M) issue(r0 + (a.stages + 1) * step, stage1);
            } else if (lost < 0) {
                lost = r0;                        // or the row behind it: row r0 is there then
            }
        }
        if (rows == 1) {
            phase ^= 1u;
        } else {
            stage = stage1 + 1 == a.stages ? 0 : stage1 + 1;
            phase = stage1 + 1 == a.stages ? phase1 ^ 1u : phase1;
        }
    }
    if (timed_out) {
        if (t == 0) ring_drain(full, a.stages, lost, step, a.M);
        if (a.status) atomicOr(a.status, TPPO_DEV_WAIT_TIMEOUT);
    }
    if (!a.partial) return;
    float* out = a.partial + int64_t(blockIdx.x) * 2 * a.N;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = Q::col(c, a.group, t);
        if (col < a.N) {
            Q::put(out, col, a.group, a.N, dg[c]);
            Q::put(out + a.N, col, a.group, a.N, db[c]);
        }
    }
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

// dgamma / dbeta = the sum of `parts` partial rows, in ascending order within each of the 32 strands of
// a column (eight loads in flight) and then over the strands; fp64, rounded once.
template <class P>
__global__ void __launch_bounds__(1024) norm_sum_kernel(const float* partial, int32_t parts, int32_t N, P* dgamma,
                                                        P* dbeta) {
    __shared__ double s[32][33];
    pdl_launch();
    pdl_wait();
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int64_t j = int64_t(blockIdx.x) * 32 + lane;           // column of the [2N]-wide partial row
    double t = 0.0;
    if (j < 2 * int64_t(N)) {
        for (int p0 = strand; p0 < parts; p0 += 8 * 32) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p0 + 32 * k < parts ? partial[int64_t(p0 + 32 * k) * 2 * N + j] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += double(v[k]);
        }
    }
    s[strand][lane] = t;
    __syncthreads();
    if (strand == 0 && j < 2 * int64_t(N)) {
        t = 0.0;
#pragma unroll
        for (int k = 0; k < 32; ++k) t += s[k][lane];
        if (j < N) { if (dgamma) store_f32(dgamma + j, float(t)); }
        else if (dbeta) store_f32(dbeta + (j - N), float(t));
    }
}

// Most blocks, and so partial rows, of a backward pass: eight per SM of short rows, three of long ones.
constexpr int kNormColParts = 64;              // partial rows of norm_cols_kernel
constexpr int32_t kNormRingCols = 512 * 32;    // most columns of the kernels that walk over rows: threads times columns of each
int norm_max_parts(int32_t N) { return N <= 512 ? 8 * kNumSms : N <= 2048 ? 5 * kNumSms : 3 * kNumSms; }

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
    // Rows by bulk copies: 32 columns per thread -- what a row costs beside its elements (two sums over the
    // block, the ring) is some 150 instructions per thread -- and as many blocks per SM as their registers
    // allow, with rings of three rows or more.  Measured over 8192 rows, against rows loaded straight into
    // registers: bf16 4096 27 us / 30, 2048 21 / 14; fp32 8192 92 / 104, 6400 76 / 74; unaligned bf16 3001
    // 68 / 86, 2051 60 / 56, unaligned fp32 5121 126 / 185, 3001 70 / 67; with 1000 rows it loses up to 4096.
    const bool long_rows = vec ? a.N >= (V == 8 ? 4096 : 8192) : a.N >= (V == 8 ? 2560 : 4096);
    const bool use_ring = long_rows && a.M >= (a.N >= 10240 ? 4 * kNumSms : 2048);
    const int64_t threads = (int64_t(a.N) + 32 * 32 - 1) / (32 * 32) * 32;
    int64_t per_sm = threads <= kRingThreads ? kRingThreads / threads : 0;
    if (per_sm > 4) per_sm = 4;
    const size_t row = vec ? RowVec<T>::pitch(a.N) : RowAny<T>::pitch(a.N);
    const int64_t fit = per_sm > 0 ? int64_t(kRingSmem / per_sm / row) : 0;
    if (use_ring && fit >= 3) {
        a.stages = int32_t(fit < 8 ? fit : 8);
        a.group = int32_t(threads);
        const size_t smem = size_t(a.stages) * row + 8 * 8;
        auto kernel = vec ? norm_fwd_ring_kernel<RowVec<T>, P, 32 / V> : norm_fwd_ring_kernel<RowAny<T>, P, 16>;
        TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingLimit));
        TPPO_CUDA_CHECK(launch_dense(kernel, dim3(unsigned(kNumSms * per_sm)), dim3(a.group), smem, s, a));
        return TPPO_OK;
    }
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


struct NormWs { float* partial; float* row_flag; size_t bytes; };
NormWs norm_carve(void* ws, int64_t M, int32_t N) {
    // no more partial rows than rows; rows of more than 16384 columns are summed by norm_cols_kernel.  Fewer columns
    // may take more partial rows: the room is that of every N up to this one.
    size_t most = 0;
    for (int32_t n : {512, 2048, kNormRingCols, N}) {
        if (n > N) n = N;
        int64_t parts = n > kNormRingCols ? kNormColParts : norm_max_parts(n);
        if (parts > M) parts = M < 1 ? 1 : M;
        if (most < size_t(parts) * n) most = size_t(parts) * n;
    }
    const size_t a = align_up(most * 2 * 4, kWsAlign);
    const size_t b = align_up(size_t(M) * 4, kWsAlign);
    char* p = static_cast<char*>(ws);
    return {reinterpret_cast<float*>(p), reinterpret_cast<float*>(p + a), a + b};
}

template <class T, class P>
int norm_bwd_typed(NormBwdArgs a, P* dgamma, P* dbeta, float* row_flag, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = a.N % V == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.dy, a.lddy, sizeof(T)) &&
                     (!a.dx || rows_aligned(a.dx, a.lddx, sizeof(T))) && (!a.gamma || aligned(a.gamma, 16));
    const int64_t pieces = vec ? a.N / V : a.N;
    int parts = 0, rc = TPPO_OK;
    const auto threads_of = [&](int cols, int unit) { return (int64_t(a.N) + cols * unit - 1) / (cols * unit) * unit; };
    const size_t stage = 2 * size_t(vec ? RowVec<T>::pitch(a.N) : RowAny<T>::pitch(a.N)), params = size_t(a.N) * 4 + 8 * 16;
    // rows per trip of the one-phase kernel and threads per SM: what the registers hold
    const int64_t eight = threads_of(8, 32);
    const bool deep = eight > 640;              // 16 columns per thread
    const int per_trip = deep ? 1 : V == 8 && eight <= 512 ? 4 : 2;
    const int resident = deep || (V == 8 && eight <= 512) ? 512 : 640;
    const int64_t row_threads = deep ? threads_of(16, 32) : eight;
    const int cols = threads_of(16, 64) <= 640 ? 16 : 32;
    // Which kernel, as measured (us; registers / one phase / two phases):
    //   bf16, 16384 rows of 256: 15 / 16 / -, 512: 21 / 19 / 24, 2048: 90 / 47 / 106, 4096: 150 / 83 / 114, 5120: - / 109
    //   / 128 (187 with 16 columns per thread); 8192 rows of 6144: - / 90 / 116 (two rows per trip 105: it spills),
    //   8192: 153 / 100 / 128; 4096 rows of 384: 12 / 11 / -, 256: 11 / 11 / -;
    //   fp32, 16384 rows of 256: 15 / 21 / -, 384: 22 / 24 / -, 512: 44 / 27 / -; 8192 rows of 2048: 46 / 34 / 51, 5120:
    //   150 / 83 / 119, 6144: - / 99 / 124, 8192: 177 / 146 / 158;
    //   unaligned bf16, 8192 rows of 263: 43 / - / 33, 1283: 71 / - / 45, 5121: 499 / - / 148 (1000 rows of 1283: 16 / - / 17);
    //   unaligned fp32, 8192 rows of 515: 29 / - / 31, 1777: 56 / - / 89, 3001: 106 / - / 88
    const bool one = vec && a.M >= kNumSms && a.N >= 512 && row_threads <= resident &&
                     2 * per_trip * stage + 8 * 16 <= kRingSmem;
    const bool two = !one && a.M >= kNumSms && threads_of(cols, 64) <= (cols == 16 ? 640 : 512) && stage + params <= kRingSmem &&
                     (vec ? a.N > 2048 : a.N >= 2048 || (V == 8 && a.M >= 2048));
    if (one) {
        a.group = int32_t(row_threads);
        int64_t per_sm = resident / a.group;
        if (per_sm > norm_max_parts(a.N) / kNumSms) per_sm = norm_max_parts(a.N) / kNumSms;
        while (per_sm > 1 && kRingSmem / per_sm < 2 * per_trip * stage + 8 * 16) --per_sm;
        const int64_t fit = int64_t((kRingSmem / per_sm - 8 * 16) / (per_trip * stage));
        a.stages = int32_t(fit < 16 ? fit : 16);
        const size_t smem = size_t(a.stages) * per_trip * stage + 8 * 16;
        // a block makes a whole trip at least, where that leaves one per SM: partial rows cost too (1000 x 1024 10 -> 8 us)
        const int64_t most = kNumSms * per_sm, trips = a.M / per_trip;
        parts = int(trips > most ? most : trips > kNumSms ? trips : kNumSms);
        auto kernel = norm_bwd_rows_kernel<T, P, 8 / V, 2, 640>;
        if constexpr (V == 8) {
            if (eight <= 512) kernel = norm_bwd_rows_kernel<T, P, 1, 4, 512>;
        }
        if (deep) kernel = norm_bwd_rows_kernel<T, P, 16 / V, 1, 512>;
        TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingLimit));
        TPPO_CUDA_CHECK(launch_dense(kernel, dim3(unsigned(parts)), dim3(a.group), smem, s, a));
    } else if (two) {
        a.group = int32_t(threads_of(cols, 64));
        int64_t per_sm = 640 / a.group;
        if (per_sm > norm_max_parts(a.N) / kNumSms) per_sm = norm_max_parts(a.N) / kNumSms;
        while (per_sm > 1 && kRingSmem / per_sm < 4 * stage + params) --per_sm;
        const int64_t fit = int64_t((kRingSmem / per_sm - params) / stage);
        a.stages = int32_t(fit < 16 ? fit : 16);
        const size_t smem = size_t(a.stages) * stage + params;
        const int64_t most = kNumSms * per_sm;
        parts = int(a.M < most ? a.M : most);
        auto kernel = vec ? (cols == 16 ? norm_bwd_ring_kernel<RowVec<T>, P, 16 / V> : norm_bwd_ring_kernel<RowVec<T>, P, 32 / V>)
                          : (cols == 16 ? norm_bwd_ring_kernel<RowAny<T>, P, 8> : norm_bwd_ring_kernel<RowAny<T>, P, 16>);
        TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingLimit));
        TPPO_CUDA_CHECK(launch_dense(kernel, dim3(unsigned(parts)), dim3(a.group), smem, s, a));
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
            parts = int(a.M < kNormColParts ? a.M : kNormColParts);
            TPPO_CUDA_CHECK(launch_dense(norm_cols_kernel<T>, dim3(dim3((a.N + 255) / 256, parts)), dim3(256), 0, s, a, row_flag));
        }
        if (a.dx) {
            TPPO_CUDA_CHECK(launch_dense(norm_bwd_long_kernel<T, P>, dim3(unsigned(a.M)), dim3(kNormMaxThreads), 0, s, a, nullptr));
        }
    }
    if (rc != TPPO_OK || !a.partial) return rc;
    TPPO_CUDA_CHECK(launch_dense(norm_sum_kernel<P>, dim3(unsigned((2 * int64_t(a.N) + 31) / 32)), dim3(1024), 0, s,
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
    if (M < 0 || N < 1 || ldx < N || ldy < N || !(eps >= 0.f) || !is_finite_host(eps))
        return TPPO_ERR_INVALID_ARG;
    if (!type_known(dtype) || ((gamma || beta) && !type_known(param_dtype))) return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || N > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    if (M == 0) return TPPO_OK;
    if (!x || !y) return TPPO_ERR_INVALID_ARG;
    const size_t es = type_size(dtype), ps = type_size(param_dtype);
    if (!aligned(x, es) || !aligned(y, es) || !aligned(gamma, ps) || !aligned(beta, ps) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(status, 4))
        return TPPO_ERR_INVALID_ARG;
    const NormFwdArgs a{x, gamma, beta, y, mean, rstd, status, M, N, ldx, ldy, eps, 0, 0};
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
    if (M < 0 || N < 1 || lddy < N || ldx < N || (dx && lddx < N)) return TPPO_ERR_INVALID_ARG;
    if (!type_known(dtype) || ((gamma || params) && !type_known(param_dtype))) return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || N > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
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
