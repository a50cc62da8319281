// Helpers shared by the dense operators (layer norm, linear, orthogonalised update): typed element
// access, row geometry checks and the launch of a programmatic dependent.
#pragma once

#include "common.cuh"
#include "ptx.cuh"

namespace tppo {

typedef uint16_t bf16_bits;           // storage of one bf16 element

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const bf16_bits* p) { return __uint_as_float(uint32_t(*p) << 16); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(bf16_bits* p, float v) { *p = bf16_bits(pack_bf16x2(v, 0.f) & 0xffffu); }

// VEC elements at p, which is aligned to min(16, VEC * sizeof(T)) bytes, widened to fp32.
template <int VEC>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[VEC]) {
    if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4) {
            const float4 w = *reinterpret_cast<const float4*>(p + i);
            v[i] = w.x; v[i + 1] = w.y; v[i + 2] = w.z; v[i + 3] = w.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = p[i];
    }
}
template <int VEC>
__device__ __forceinline__ void load_vec(const bf16_bits* p, float (&v)[VEC]) {
    if constexpr (VEC % 8 == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 8) {
            const uint4 w = *reinterpret_cast<const uint4*>(p + i);
            v[i] = bf16_lo(w.x); v[i + 1] = bf16_hi(w.x); v[i + 2] = bf16_lo(w.y); v[i + 3] = bf16_hi(w.y);
            v[i + 4] = bf16_lo(w.z); v[i + 5] = bf16_hi(w.z); v[i + 6] = bf16_lo(w.w); v[i + 7] = bf16_hi(w.w);
        }
    } else if constexpr (VEC == 4) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x); v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = load_f32(p + i);
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[VEC]) {
    if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 4)
            *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) p[i] = v[i];
    }
}
template <int VEC>
__device__ __forceinline__ void store_vec(bf16_bits* p, const float (&v)[VEC]) {
    if constexpr (VEC % 8 == 0) {
#pragma unroll
        for (int i = 0; i < VEC; i += 8)
            *reinterpret_cast<uint4*>(p + i) =
                make_uint4(pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]),
                           pack_bf16x2(v[i + 4], v[i + 5]), pack_bf16x2(v[i + 6], v[i + 7]));
    } else if constexpr (VEC == 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) store_f32(p + i, v[i]);
    }
}

// The largest finite value of an element type.
__device__ __forceinline__ float top_of(const float*) { return kFltMax; }
__device__ __forceinline__ float top_of(const bf16_bits*) { return kBf16Max; }
__device__ __forceinline__ bool is_finite(float v) { return fabsf(v) <= kFltMax; }

inline bool is_finite_host(float v) { return v - v == 0.f; }
// Whether every row of a matrix starts on a 16-byte boundary.
inline bool rows_aligned(const void* p, int64_t ld, size_t esize) { return aligned(p, 16) && (ld * int64_t(esize)) % 16 == 0; }

// Rows and columns beyond this would take tile and column arithmetic past 32 bits.
constexpr int64_t kDenseMaxSize = int64_t(1) << 30;

// The two halves of a programmatic dependent launch: the primary lets its dependent start, the
// dependent waits for the primary's memory.
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// How a launch stands to the ones before and after it on the stream: bits.
//   kChain   (none) needs what its predecessor wrote: waits for it before touching global memory.  What
//            follows may start at any time and waits likewise.
//   kLead    lets what follows start only when every block of this launch has seen its predecessor's end
//            -- so that the follower may run beside it.
//   kBeside  follows a kLead, or a kBeside behind one, and needs nothing that these write: everything
//            before them was complete, and performed for the whole lead's grid, when it was let start.  It
//            begins with no wait, which is what the documentation ties visibility to, so it takes none on trust:
//            a gpu-scope fence (and one towards the copy engine's proxy) stands before its first load, and what
//            a call rewrites in its workspace each time is read at L2 (tensor copies, __ldcg), where the
//            lead's wait has it.  It waits for its predecessor before it ends, so that its own end covers
//            theirs for whatever comes next.
//   kTail    what follows starts when this launch has ended.  A product's CTA that waits on an SM holds nearly all
//            of its shared memory, which a kernel that streams through L1 then lacks (16384 x 5120: dz 109
//            us instead of 116, 20 us of a whole backward pass).
// A dependent starts when every block of its primary has asked for it, so all of those are resident by then
// and none can be kept from an SM by a dependent that waits.
enum : int32_t { kChain = 0, kLead = 1, kBeside = 2, kTail = 4 };
typedef int32_t Link;
__device__ __forceinline__ void link_begin(Link link) {
    if (!(link & (kLead | kTail))) pdl_launch();
    if (link & kBeside) asm volatile("fence.acq_rel.gpu;\n\tfence.proxy.async.global;" ::: "memory");
    else pdl_wait();
    if (link & kLead) pdl_launch();
}
__device__ __forceinline__ void link_end(Link link) {
    if (link & kBeside) pdl_wait();
}
// The links of launches that do not depend on one another, in the order of their launch; `last`: what the
// last of them adds.
struct LinkGroup {
    int left, total;
    Link last;
    explicit LinkGroup(int launches, Link last_adds = kChain) : left(launches), total(launches), last(last_adds) {}
    Link next() {
        const Link l = left < total ? kBeside : total > 1 ? kLead : kChain;
        return --left == 0 ? l | last : l;
    }
};
// kTail for a kernel that streams `elements` before a product, from some 10 us of it on: a shorter one gains
// more from having the product's start behind it.
inline Link stream_link(int64_t elements) { return elements > (int64_t(1) << 23) ? kTail : kChain; }

// Launches `kernel` on `s` as a programmatic dependent of whatever precedes it there: its blocks may
// start while that still runs, so every kernel launched this way calls pdl_wait() before it touches
// global memory, or link_begin() then and link_end() at its end.
template <class... Params, class... Args>
cudaError_t launch_dense(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const Args&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

}  // namespace tppo
