// The global norm of many gradients, and clipping by it:
//     sum_sq = sum_i |g_i|^2,   coef = min(1, max_norm / sqrt(sum_sq)),   out_i = coef * g_i
// Both calls stream: the norm reads every element once, clipping reads it once more and writes it once, so
// HBM bounds them (or L2, for gradients that fit there): 600 million bf16 elements are read in 184 us (6.5 TB/s) and
// scaled into other buffers in 362 (6.6 TB/s).  The list of tensors travels in the kernel's
// parameters -- no copy to the device, nothing to keep in step with it, and a captured graph carries it along.
// Work is cut into chunks of 8192 elements of one tensor; units of 256 threads take them in turn, so that a
// unit searches its first tensor once and then only steps on.  Clipping walks backwards: what the norm read last is
// what L2 still holds.
//
// A thread squares 32 elements of a chunk in fp32 (four chains of eight, then two joins: up to ten roundings) and adds their
// sum to a 64-bit total: sum_sq is within 10 * 2^-24 of itself and the norm within 5 * 2^-24, some 1.5e-7 of sum_sq where all
// elements are alike and every thread errs the same way.  Where that sum could have lost more -- it is not finite, or below
// 2^-100 -- the 32 squares are taken again in 64 bits, so the bound holds over the whole range of fp32, and the result is
// infinite only for an element that is not finite.  (A run of zeros is below 2^-100 too: 600 million of them take 232 us.)
// Partial sums are added in a fixed order.  Short lists take one cluster of eight blocks, which meet in its
// shared memory: one launch instead of two.
#include <memory>
#include <new>

#include "dense_common.cuh"

namespace tppo {
namespace {

constexpr int kGradUnit = 256;                  // threads that walk a range of chunks
constexpr int kGradPieces = 4;                  // 8-element pieces of a chunk per thread
constexpr int kGradChunk = kGradUnit * kGradPieces * 8;
constexpr int kGradGrid = kNumSms * 4;
constexpr int kClipInPlaceGrid = kNumSms * 64;
constexpr int kGradCluster = 8, kGradClusterThreads = 1024;
constexpr int kGradClusterChunks = 4 * kGradCluster * kGradClusterThreads / kGradUnit;
constexpr int kGradFew = 64, kGradMany = 1024;  // tensors per launch: 29 bytes each of the 32764 for parameters

enum : uint8_t { kSrcF32 = 1, kDstF32 = 2, kAligned = 4 };      // and the length of the head << 4

template <int CAP>
struct GradList {
    const void* src[CAP];
    void* dst[CAP];
    int64_t n[CAP];
    int32_t first[CAP + 1];                     // first chunk of each tensor
    int32_t count, in_place;                    // in_place: every tensor is its own output
    uint8_t kind[CAP];
};

// A chunk of a tensor: elements [at, at + len) in pieces of eight, aligned for 16-byte accesses with kAligned;
// the first chunk of an aligned tensor also has the `head` elements in front of its first boundary.
struct GradChunk {
    int64_t at;
    int32_t len, head;
};
template <int CAP>
__device__ __forceinline__ GradChunk grad_chunk(const GradList<CAP>& l, int t, int c) {
    const int head = l.kind[t] >> 4, in = c - l.first[t];
    GradChunk k;
    k.at = head + int64_t(in) * kGradChunk;
    const int64_t left = l.n[t] - k.at;
    k.len = int32_t(left < kGradChunk ? left : kGradChunk);
    k.head = in == 0 ? head : 0;
    return k;
}
// The tensor that chunk c belongs to.
template <int CAP>
__device__ __forceinline__ int grad_find(const GradList<CAP>& l, int c) {
    int lo = 0, hi = l.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (l.first[mid] <= c) lo = mid; else hi = mid;
    }
    return lo;
}

// This thread's elements of a chunk: pieces of eight 256 pieces apart, or single elements 256 apart where
// 16-byte accesses are not possible.  What lies beyond the chunk is 0.
template <class T>
__device__ __forceinline__ void grad_load(const T* p, int len, bool vec, int tid, float (&v)[kGradPieces][8]) {
    if (vec && len == kGradChunk) {
#pragma unroll
        for (int i = 0; i < kGradPieces; ++i) load_vec<8>(p + (tid + i * kGradUnit) * 8, v[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < kGradPieces; ++i) {
        const int at = (tid + i * kGradUnit) * 8;
        if (vec && at + 8 <= len) {
            load_vec<8>(p + at, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = vec ? at + j : tid + (i * 8 + j) * kGradUnit;
                v[i][j] = e < len ? load_f32(p + e) : 0.f;
            }
        }
    }
}
// Eight elements as loaded, widened and scaled by f0 * f1.
template <class S> struct GradPiece;
template <> struct GradPiece<bf16_bits> {
    uint4 w;
    __device__ __forceinline__ void load(const bf16_bits* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void scaled(float f0, float f1, float (&v)[8]) const {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = bf16_lo(u[j]) * f0 * f1;
            v[2 * j + 1] = bf16_hi(u[j]) * f0 * f1;
        }
    }
};
template <> struct GradPiece<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = __ldcs(reinterpret_cast<const float4*>(p));
        b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void scaled(float f0, float f1, float (&v)[8]) const {
        v[0] = a.x * f0 * f1; v[1] = a.y * f0 * f1; v[2] = a.z * f0 * f1; v[3] = a.w * f0 * f1;
        v[4] = b.x * f0 * f1; v[5] = b.y * f0 * f1; v[6] = b.z * f0 * f1; v[7] = b.w * f0 * f1;
    }
};
template <class S, class D>
__device__ __forceinline__ void grad_scale_piece(const GradPiece<S>& w, D* q, bool zero, float f0, float f1) {
    float v[8];
    w.scaled(f0, f1, v);
    if (zero) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
    }
    store_vec<8>(q, v);
}
// A chunk scaled by f0 * f1; with f1 = 0 it becomes 0 whatever it holds.  Whole chunks, which nearly all of a large list
// are, have 64 bytes per thread on their way; the others go a piece at a time.
template <class S, class D>
__device__ __forceinline__ void grad_scale(const S* p, D* q, int len, bool vec, int tid, float f0, float f1) {
    const bool zero = f1 == 0.f;
    if (vec && len == kGradChunk) {
        constexpr int kBatch = kGradPieces * 2 / int(sizeof(S));
        GradPiece<S> w[kBatch];
#pragma unroll
        for (int first = 0; first < kGradPieces; first += kBatch) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) w[i].load(p + (tid + (first + i) * kGradUnit) * 8);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) grad_scale_piece(w[i], q + (tid + (first + i) * kGradUnit) * 8, zero, f0, f1);
        }
    } else if (vec) {
#pragma unroll 1
        for (int at = tid * 8; at + 8 <= len; at += kGradUnit * 8) {
            GradPiece<S> w;
            w.load(p + at);
            grad_scale_piece(w, q + at, zero, f0, f1);
        }
        const int e = (len & ~7) + tid;                   // what is left of the last piece
        if (e < len) store_f32(q + e, zero ? 0.f : load_f32(p + e) * f0 * f1);
    } else {
#pragma unroll 4
        for (int e = tid; e < len; e += kGradUnit) store_f32(q + e, zero ? 0.f : load_f32(p + e) * f0 * f1);
    }
}
__device__ __forceinline__ float grad_element(const void* p, int64_t e, bool f32) {
    return f32 ? load_f32(static_cast<const float*>(p) + e) : load_f32(static_cast<const bf16_bits*>(p) + e);
}
__device__ __forceinline__ void grad_put(void* p, int64_t e, bool f32, float v) {
    if (f32) store_f32(static_cast<float*>(p) + e, v);
    else store_f32(static_cast<bf16_bits*>(p) + e, v);
}

// Sum over the block in a fixed order; the result is thread 0's.
__device__ __forceinline__ double block_sum(double v, double* red) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) v = warp_sum(threadIdx.x < blockDim.x >> 5 ? red[threadIdx.x] : 0.0);
    return v;
}

__device__ __forceinline__ void grad_result(double total, double* sum_sq, float* norm, int32_t* status) {
    const bool good = total - total == 0.0;
    if (!good) total = __longlong_as_double(0x7ff0000000000000ll);
    *sum_sq = total;
    if (norm) *norm = float(sqrt(total));
    if (!good && status) atomicOr(status, TPPO_DEV_NONFINITE);
}

template <int CAP, bool CLUSTER>
__global__ void __launch_bounds__(CLUSTER ? kGradClusterThreads : kGradUnit, CLUSTER ? 1 : 4)
grad_norm_kernel(const __grid_constant__ GradList<CAP> l, double* partial, double* sum_sq, float* norm, int32_t* status) {
    __shared__ double red[32], parts[kGradCluster];
    if constexpr (CLUSTER) ptx::cluster_arrive();         // the wait is in front of the first store into another block
    pdl_launch();
    pdl_wait();
    const int per = int(blockDim.x) / kGradUnit, unit = int(blockIdx.x) * per + int(threadIdx.x) / kGradUnit;
    const int units = int(gridDim.x) * per, tid = int(threadIdx.x) % kGradUnit, chunks = l.first[l.count];
    int t = unit < chunks ? grad_find(l, unit) : 0;
    double sum = 0;
    for (int c = unit; c < chunks; c += units) {
        while (c >= l.first[t + 1]) ++t;
        const GradChunk k = grad_chunk(l, t, c);
        const bool f32 = l.kind[t] & kSrcF32, vec = l.kind[t] & kAligned;
        float v[kGradPieces][8], s[4] = {0.f, 0.f, 0.f, 0.f};
        if (f32) grad_load(static_cast<const float*>(l.src[t]) + k.at, k.len, vec, tid, v);
        else grad_load(static_cast<const bf16_bits*>(l.src[t]) + k.at, k.len, vec, tid, v);
#pragma unroll
        for (int i = 0; i < kGradPieces; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j & 3] = fmaf(v[i][j], v[i][j], s[j & 3]);
        const float run = (s[0] + s[1]) + (s[2] + s[3]);
        if (run >= 0x1p-100f && run <= kFltMax) {
            sum += double(run);
        } else {
#pragma unroll
            for (int i = 0; i < kGradPieces; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = fma(double(v[i][j]), double(v[i][j]), sum);
        }
        if (tid < k.head) {
            const double e = grad_element(l.src[t], tid, f32);
            sum = fma(e, e, sum);
        }
    }
    sum = block_sum(sum, red);
    if constexpr (CLUSTER) {
        ptx::cluster_wait();                              // every block of the cluster runs: its shared memory may be written
        if (threadIdx.x == 0) {
            const uint32_t at = ptx::map_to_cta(ptx::smem_addr(parts + ptx::cluster_ctarank()), 0);
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(sum) : "memory");
        }
        ptx::cluster_sync_all();
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            double total = 0;
            for (int i = 0; i < kGradCluster; ++i) total += parts[i];
            grad_result(total, sum_sq, norm, status);
        }
    } else if (threadIdx.x == 0) {
        partial[blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(1024) grad_sum_kernel(const double* partial, int64_t n, double* sum_sq, float* norm, int32_t* status) {
    __shared__ double red[32];
    pdl_launch();
    pdl_wait();
    double v = 0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) v += __ldcg(partial + i);
    v = block_sum(v, red);
    if (threadIdx.x == 0) grad_result(v, sum_sq, norm, status);
}

template <int CAP>
__global__ void __launch_bounds__(kGradUnit, 8)
grad_clip_kernel(const __grid_constant__ GradList<CAP> l, const double* sum_sq, double max_norm, float* coef, int32_t* status) {
    __shared__ float factor[2];
    pdl_launch();
    pdl_wait();
    if (threadIdx.x == 0) {
        const double total = *sum_sq;
        const bool good = total >= 0 && total - total == 0.0;       // a NaN fails both
        const double norm = sqrt(total);
        const double c = !good ? 0.0 : norm <= max_norm ? 1.0 : max_norm / norm;
        // far below 1 it is applied in two steps, so that a subnormal factor costs no precision
        factor[0] = c < 0x1p-96 ? 0x1p-96f : 1.f;
        factor[1] = float(c < 0x1p-96 ? c * 0x1p96 : c);
        if (blockIdx.x == 0) {
            if (coef) *coef = float(c);
            if (!good && status) atomicOr(status, TPPO_DEV_NONFINITE);
        }
    }
    __syncthreads();
    const float f0 = factor[0], f1 = factor[1];
    const bool stays = f0 == 1.f && f1 == 1.f;
    if (stays && l.in_place) return;
    const int units = int(gridDim.x), unit = int(blockIdx.x), tid = int(threadIdx.x), chunks = l.first[l.count];
    int t = unit < chunks ? grad_find(l, chunks - 1 - unit) : 0;
    for (int c = chunks - 1 - unit; c >= 0; c -= units) {
        while (c < l.first[t]) --t;
        const bool f32 = l.kind[t] & kSrcF32, to_f32 = l.kind[t] & kDstF32, vec = l.kind[t] & kAligned;
        if (stays && l.src[t] == l.dst[t] && f32 == to_f32) continue;
        const GradChunk k = grad_chunk(l, t, c);
        const float* s32 = static_cast<const float*>(l.src[t]) + k.at;
        const bf16_bits* s16 = static_cast<const bf16_bits*>(l.src[t]) + k.at;
        float* d32 = static_cast<float*>(l.dst[t]) + k.at;
        bf16_bits* d16 = static_cast<bf16_bits*>(l.dst[t]) + k.at;
        if (f32 && to_f32) grad_scale(s32, d32, k.len, vec, tid, f0, f1);
        else if (f32) grad_scale(s32, d16, k.len, vec, tid, f0, f1);
        else if (to_f32) grad_scale(s16, d32, k.len, vec, tid, f0, f1);
        else grad_scale(s16, d16, k.len, vec, tid, f0, f1);
        if (tid < k.head) grad_put(l.dst[t], tid, to_f32, f1 == 0.f ? 0.f : grad_element(l.src[t], tid, f32) * f0 * f1);
    }
}

int64_t esize(int32_t dtype) { return dtype == TPPO_F32 ? 4 : 2; }

bool tensor_ok(const tppo_tensor& t) {
    return (t.dtype == TPPO_BF16 || t.dtype == TPPO_F32) && t.n >= 0 && (t.n == 0 || t.data) && aligned(t.data, size_t(esize(t.dtype)));
}

// Elements in front of the first one that starts on a 16-byte boundary.
int head_of(const void* p, int32_t dtype) {
    const int64_t e = esize(dtype);
    return int((16 - reinterpret_cast<uintptr_t>(p) % 16) % 16 / e);
}

// Whether `count` tensors are well formed and their chunks fit 32 bits.
int check(const tppo_tensor* a, const tppo_tensor* out, int32_t count) {
    if (count < 0 || (count > 0 && !a)) return TPPO_ERR_INVALID_ARG;
    int64_t chunks = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (!tensor_ok(a[i]) || (out && (!tensor_ok(out[i]) || out[i].n != a[i].n))) return TPPO_ERR_INVALID_ARG;
        if (a[i].n > int64_t(1) << 42) return TPPO_ERR_UNSUPPORTED;
        chunks += a[i].n / kGradChunk + 1;
        if (chunks > 0x7fffffff) return TPPO_ERR_UNSUPPORTED;
    }
    return TPPO_OK;
}

// Marks in `skip` the tensors of a list that are in place and the same as an earlier one: blocks write in no order, so that each
// is to be scaled once.  An output at the address of another entry's gradient or output is refused.  `table`: room for 2^bits
// places, more than `count`: the entries in place by their address.  1000 tensors in place take 1 to 2 us of host time;
// sorting all spans, to refuse every overlap, took 20 to 50.
int clip_places(const tppo_tensor* a, const tppo_tensor* out, int32_t count, int bits, int32_t* table, uint8_t* skip) {
    const uint64_t mask = (uint64_t(1) << bits) - 1;
    for (uint64_t i = 0; i <= mask; ++i) table[i] = -1;
    // the place of the entry whose output is at p, or the free one where it would be
    auto place = [&](const void* p) -> int32_t& {
        uint64_t h = (reinterpret_cast<uint64_t>(p) * 0x9e3779b97f4a7c15ull) >> (64 - bits);
        while (table[h] >= 0 && a[table[h]].data != p) h = (h + 1) & mask;
        return table[h];
    };
    auto in_place = [&](int32_t i) { return !out || out[i].data == a[i].data; };
    for (int32_t i = 0; i < count; ++i) {
        skip[i] = 0;
        if (a[i].n == 0 || !in_place(i)) continue;
        int32_t& at = place(a[i].data);
        if (at < 0) {
            at = i;
        } else {
            if (a[at].n != a[i].n || a[at].dtype != a[i].dtype) return TPPO_ERR_INVALID_ARG;
            skip[i] = 1;
        }
    }
    for (int32_t i = 0; i < count; ++i)
        if (a[i].n != 0 && !in_place(i) && (place(a[i].data) >= 0 || place(out[i].data) >= 0)) return TPPO_ERR_INVALID_ARG;
    return TPPO_OK;
}
// Which tensors of a list clipping leaves out; NULL without memory of its own where none is in place.
struct ClipPlaces {
    int32_t few_table[4 * kGradFew];
    uint8_t few_skip[kGradFew];
    std::unique_ptr<int32_t[]> table;
    std::unique_ptr<uint8_t[]> many_skip;
    const uint8_t* skip = nullptr;

    int find(const tppo_tensor* a, const tppo_tensor* out, int32_t count) {
        bool any = false;
        for (int32_t i = 0; i < count; ++i) {
            if (a[i].n == 0 || (out && out[i].data != a[i].data)) continue;
            if (out && out[i].dtype != a[i].dtype) return TPPO_ERR_INVALID_ARG;      // its gradient in another type
            any = true;
        }
        if (!any) return TPPO_OK;
        int bits = 1;
        while ((int64_t(1) << bits) < 2 * int64_t(count)) ++bits;
        int32_t* t = few_table;
        uint8_t* k = few_skip;
        if (count > kGradFew) {
            table.reset(new (std::nothrow) int32_t[size_t(1) << bits]);
            many_skip.reset(new (std::nothrow) uint8_t[size_t(count)]);
            t = table.get();
            k = many_skip.get();
            if (!t || !k) return TPPO_ERR_UNSUPPORTED;
        }
        skip = k;
        return clip_places(a, out, count, bits, t, k);
    }
};

// `skip`: NULL, or which tensors to leave out.
template <int CAP>
void fill(GradList<CAP>& l, const tppo_tensor* a, const tppo_tensor* out, int32_t count, const uint8_t* skip) {
    int64_t chunks = 0;
    l.count = 0;
    l.in_place = 1;
    for (int32_t i = 0; i < count; ++i) {
        if (a[i].n == 0 || (skip && skip[i])) continue;
        const tppo_tensor& o = out ? out[i] : a[i];
        // eight elements of either tensor start on a boundary once the first `head` are gone: the bf16 one decides
        int head = head_of(a[i].data, a[i].dtype);
        if (o.dtype == TPPO_BF16 && a[i].dtype != TPPO_BF16) head = head_of(o.data, o.dtype);
        const bool vec = aligned(static_cast<char*>(a[i].data) + head * esize(a[i].dtype), 16) &&
                         aligned(static_cast<char*>(o.data) + head * esize(o.dtype), 16);
        if (!vec) head = 0;
        if (head > a[i].n) head = int(a[i].n);
        const int k = l.count++;
        l.src[k] = a[i].data;
        l.dst[k] = o.data;
        if (o.data != a[i].data || o.dtype != a[i].dtype) l.in_place = 0;
        l.n[k] = a[i].n;
        l.first[k] = int32_t(chunks);
        l.kind[k] = uint8_t((a[i].dtype == TPPO_F32 ? kSrcF32 : 0) | (o.dtype == TPPO_F32 ? kDstF32 : 0) | (vec ? kAligned : 0) | head << 4);
        const int64_t body = a[i].n - head;
        chunks += body > 0 ? (body + kGradChunk - 1) / kGradChunk : 1;
    }
    l.first[l.count] = int32_t(chunks);
}

template <int CAP>
int norm_part(const tppo_tensor* a, int32_t count, bool only, double* partial, int64_t& parts, double* sum_sq, float* norm, int32_t* status, cudaStream_t s) {
    GradList<CAP> l;
    fill(l, a, nullptr, count, nullptr);
    const int chunks = l.first[l.count];
    if (only && chunks <= kGradClusterChunks) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(kGradCluster);
        cfg.blockDim = dim3(kGradClusterThreads);
        cfg.stream = s;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kGradCluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        TPPO_CUDA_CHECK(cudaLaunchKernelEx(&cfg, grad_norm_kernel<CAP, true>, l, partial, sum_sq, norm, status));
        return TPPO_OK;
    }
    const int grid = chunks < kGradGrid ? chunks : kGradGrid;
    if (grid == 0) return TPPO_OK;
    TPPO_CUDA_CHECK(launch_dense(grad_norm_kernel<CAP, false>, dim3(grid), dim3(kGradUnit), 0, s, l, partial + parts, sum_sq, norm, status));
    parts += grid;
    return TPPO_OK;
}

template <int CAP>
int clip_part(const tppo_tensor* a, const tppo_tensor* out, const uint8_t* skip, int32_t count, const double* sum_sq, double max_norm, float* coef, int32_t* status, cudaStream_t s) {
    GradList<CAP> l;
    fill(l, a, out, count, skip);
    const int chunks = l.first[l.count];
    // A block per chunk, in the order of their addresses: 600 million bf16 elements in 362 us, the copy rate.  Blocks that
    // take several drift apart, and HBM's pages suffer: 408 with 64 per SM, 490 with the 8 that fit.  In place there may
    // be nothing to do, and 73 thousand blocks that find that out take 78 us, 64 per SM 15; over the limit the smaller grid
    // costs 380 us where other buffers take 353.
    const int most = l.in_place ? kClipInPlaceGrid : 0x7fffffff, grid = chunks < 1 ? 1 : chunks < most ? chunks : most;
    TPPO_CUDA_CHECK(launch_dense(grad_clip_kernel<CAP>, dim3(grid), dim3(kGradUnit), 0, s, l, sum_sq, max_norm, coef, status));
    return TPPO_OK;
}

}  // namespace

size_t grad_norm_workspace_bytes(int64_t count) {
    if (count > 0x7fffffff) return 0;
    return align_up(size_t((count + kGradMany - 1) / kGradMany + 1) * kGradGrid * sizeof(double), kWsAlign);
}

}  // namespace tppo

TPPO_API int tppo_grad_norm(const tppo_tensor* grads, int32_t count, double* sum_sq, float* norm, int32_t* status,
                            void* workspace, size_t workspace_bytes, void* stream) {
    using namespace tppo;
    const int bad = check(grads, nullptr, count);
    if (bad != TPPO_OK) return bad;
    if (!sum_sq || !aligned(sum_sq, 8) || !aligned(norm, 4) || !aligned(status, 4)) return TPPO_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, kWsAlign) || workspace_bytes < grad_norm_workspace_bytes(count)) return TPPO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    double* partial = static_cast<double*>(workspace);
    int64_t parts = 0;
    if (count <= kGradMany) {
        const int r = count <= kGradFew ? norm_part<kGradFew>(grads, count, true, partial, parts, sum_sq, norm, status, s)
                                        : norm_part<kGradMany>(grads, count, true, partial, parts, sum_sq, norm, status, s);
        if (r != TPPO_OK || parts == 0) return r;
    } else {
        for (int32_t i = 0; i < count; i += kGradMany) {
            const int r = norm_part<kGradMany>(grads + i, count - i < kGradMany ? count - i : kGradMany, false, partial, parts, sum_sq, norm, status, s);
            if (r != TPPO_OK) return r;
        }
    }
    TPPO_CUDA_CHECK(launch_dense(grad_sum_kernel, dim3(1), dim3(1024), 0, s, partial, parts, sum_sq, norm, status));
    return TPPO_OK;
}

TPPO_API int tppo_grad_clip(const tppo_tensor* grads, int32_t count, const double* sum_sq, double max_norm,
                            const tppo_tensor* out, float* coef, int32_t* status, void* stream) {
    using namespace tppo;
    const int bad = check(grads, out, count);
    if (bad != TPPO_OK) return bad;
    if (!sum_sq || !aligned(sum_sq, 8) || !aligned(coef, 4) || !aligned(status, 4) || !(max_norm >= 0) || max_norm - max_norm != 0)
        return TPPO_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    ClipPlaces places;
    const int twice = places.find(grads, out, count);
    if (twice != TPPO_OK) return twice;
    const uint8_t* skip = places.skip;
    if (count <= kGradFew) return clip_part<kGradFew>(grads, out, skip, count, sum_sq, max_norm, coef, status, s);
    for (int32_t i = 0; i < count; i += kGradMany) {
        const int r = clip_part<kGradMany>(grads + i, out ? out + i : nullptr, skip ? skip + i : nullptr, count - i < kGradMany ? count - i : kGradMany,
                                           sum_sq, max_norm, i == 0 ? coef : nullptr, i == 0 ? status : nullptr, s);
        if (r != TPPO_OK) return r;
    }
    return TPPO_OK;
}
