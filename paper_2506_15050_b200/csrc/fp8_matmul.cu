// Products of 8-bit matrices with a scale per block of 128 elements of the contraction:
//     y[m, n] = sum_b sa(b, m) sb(b, n) P_b[m, n],   P_b[m, n] = sum_{k in block b} a[m, k] b[n, k]
// P_b comes from tcgen05.mma (kind::f8f6f4, e4m3, fp32 accumulators); it has to leave tensor memory for every
// block, since the scales differ from block to block: eight warps read it (tcgen05.ld), scale it and add it to the
// output tile, which they hold in registers in fp32, while the tensor cores fill the other accumulator.
//
//   fp8_gemm_kernel   many output tiles: persistent CTAs, 128 x 256 tiles.  A block of the contraction is 512 clocks of
//                     the tensor cores; scaling it costs a warp 128 columns: with one scale for all of them
//                     (square blocks of b) one packed fma per two values, with a scale per column one packed
//                     multiplication more.
//   fp8_split_kernel  few output tiles (one to some hundred tokens): the output is taken TRANSPOSED, the 128 accumulator
//                     rows running along n and the BN columns along m, and the contraction is split over the CTAs of
//                     a cluster, whose partial sums meet in distributed shared memory in a fixed order.
//
// Roles of a CTA's warps: 0 TMA loads, 1 tcgen05.mma, 2-9 scaling and output.  Scales travel through a ring of their
// own: an operand stage is free as soon as the tensor cores have read it, its scales only when the eight warps have.
// Every wait is bounded; one that runs out raises TPPO_DEV_WAIT_TIMEOUT, outputs are then incomplete, the copies in
// flight land and tensor memory is released.
#include "dense_common.cuh"
#include "umma.cuh"

namespace tppo {

bool make_u8_tensor_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_rows);
bool make_f32_tensor_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_cols);

namespace {

constexpr int kF8TileM = 128, kF8Block = 128;             // accumulator rows; elements that share a scale = bytes of a swizzled row
constexpr int kF8Threads = 320, kF8Warps = 8;
constexpr uint32_t kF8ABytes = kF8TileM * kF8Block;

// Instruction descriptor (fields as in umma::instr_desc_bf16): fp32 accumulators, both operands e4m3 (0), K-major.
__host__ __device__ constexpr uint32_t f8_instr_desc(int n) {
    return (1u << 4) | (uint32_t(n >> 3) << 17) | (uint32_t(kF8TileM >> 4) << 24);
}
// One 128 x N x 32 step, issued by one thread.
__device__ __forceinline__ void mma_f8(uint32_t tmem_d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void f8_tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ uint64_t f8_pair(uint32_t lo, uint32_t hi) { return uint64_t(lo) | uint64_t(hi) << 32; }

// The operand ring and the ring of scales.
//   AROWS / BROWS: that operand has a scale per row, which the ring carries (128 / BN of them per block), each
//   operand's on a 128-byte boundary, as tensor copies ask
template <int BN> __host__ __device__ constexpr uint32_t f8_slot() { return kF8TileM * 4 + (BN * 4 < 128 ? 128 : BN * 4); }
template <int BN, int STAGES, int SLOTS, bool AROWS, bool BROWS>
struct F8Ring {
    static constexpr uint32_t kStage = kF8ABytes + BN * kF8Block;
    static constexpr uint32_t kSlot = f8_slot<BN>(), kScaleBytes = (AROWS ? kF8TileM * 4 : 0) + (BROWS ? BN * 4 : 0);
    static_assert(AROWS || BROWS, "one of the operands has a scale per row");
    uint32_t base, scales, full, empty, sfull, sempty;
    int stage = 0, slot = 0;
    uint32_t phase = 0, sphase = 0;

    __device__ __forceinline__ void next() {
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    __device__ __forceinline__ void next_slot() {
        if (++slot == SLOTS) { slot = 0; sphase ^= 1u; }
    }
    // Loads blocks [k0, k1) of the tile whose first A and B rows are am and bn.
    __device__ __forceinline__ bool load(const CUtensorMap* ma, const CUtensorMap* mb, const CUtensorMap* msa, const CUtensorMap* msb,
                                         int am, int bn, int k0, int k1) {
        for (int kb = k0; kb < k1; ++kb) {
            if (!ptx::mbar_wait<false>(empty + 8 * stage, phase ^ 1u)) return false;
            const uint32_t fb = full + 8 * stage, sa = base + stage * kStage;
            ptx::mbar_arrive_expect_tx(fb, kStage);
            umma::tma_load_2d(sa, ma, fb, kb * kF8Block, am);
            umma::tma_load_2d(sa + kF8ABytes, mb, fb, kb * kF8Block, bn);
            next();
            if (!ptx::mbar_wait<false>(sempty + 8 * slot, sphase ^ 1u)) return false;
            const uint32_t sb = sfull + 8 * slot, s = scales + slot * kSlot;
            ptx::mbar_arrive_expect_tx(sb, kScaleBytes);
            if (AROWS) umma::tma_load_2d(s, msa, sb, am, kb);
            if (BROWS) umma::tma_load_2d(s + kF8TileM * 4, msb, sb, bn, kb);
            next_slot();
        }
        return true;
    }
    // After a wait ran out: let the copies already issued land before the CTA's memory goes away.
    __device__ __forceinline__ void drain() {
        for (int s = 0; s < STAGES; ++s)
            if (!ptx::mbar_wait<false>(full + 8 * s, s < stage ? phase : phase ^ 1u)) return;
        for (int s = 0; s < SLOTS; ++s)
            if (!ptx::mbar_wait<false>(sfull + 8 * s, s < slot ? sphase : sphase ^ 1u)) return;
    }
    // One block into accumulator d.
    __device__ __forceinline__ bool multiply(uint32_t d) {
        if (!ptx::mbar_wait<false>(full + 8 * stage, phase)) return false;
        umma::fence_after_thread_sync();
        const uint32_t sa = base + stage * kStage;
        const uint64_t ad = umma::smem_desc(sa, 16, 1024), bd = umma::smem_desc(sa + kF8ABytes, 16, 1024);
#pragma unroll
        for (int j = 0; j < kF8Block / 32; ++j)
            mma_f8(d, umma::smem_desc_advance(ad, j * 32), umma::smem_desc_advance(bd, j * 32), f8_instr_desc(BN), j != 0 ? 1u : 0u);
        umma::mma_commit(empty + 8 * stage);
        next();
        return true;
    }
};

// A scale of square blocks: [row blocks, contraction blocks].
struct F8Square { const float* p; int64_t ld; };

// acc (COLS columns of this thread's accumulator row, as pairs) += f * column scales * the finished block at `taddr`.
// `scales`: shared-memory address of the columns' scales, or 0: none.
template <int COLS, bool BROWS>
__device__ __forceinline__ void f8_scale(uint32_t taddr, float f, uint32_t scales, uint64_t (&acc)[COLS / 2]) {
    constexpr int kChunk = COLS < 32 ? 8 : 32;
    const uint64_t ff = ptx::pack_f32x2(f, f);
#pragma unroll
    for (int c = 0; c < COLS; c += kChunk) {
        uint32_t v[kChunk];
        if constexpr (kChunk == 32) umma::tmem_ld32(taddr + c, v);
        else f8_tmem_ld8(taddr + c, v);
        umma::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < kChunk; i += 4) {
            uint64_t lo = f8_pair(v[i], v[i + 1]), hi = f8_pair(v[i + 2], v[i + 3]);
            if (BROWS) {
                const uint4 s = ptx::lds128(scales + (c + i) * 4);
                lo = ptx::mul_f32x2(lo, f8_pair(s.x, s.y));
                hi = ptx::mul_f32x2(hi, f8_pair(s.z, s.w));
            }
            acc[(c + i) / 2] = ptx::fma_f32x2(lo, ff, acc[(c + i) / 2]);
            acc[(c + i) / 2 + 1] = ptx::fma_f32x2(hi, ff, acc[(c + i) / 2 + 1]);
        }
    }
}

struct F8Out {
    void* y; int64_t ldy, M; int32_t N; int32_t* status;
    int32_t aligned;          // rows of y start on 16-byte boundaries
};
// A finished element; 0 and a flag where it is not finite or leaves its type.
template <class T>
__device__ __forceinline__ float f8_finish(float v, bool& bad) {
    const bool good = fabsf(v) <= top_of(static_cast<const T*>(nullptr));
    bad |= !good;
    return good ? v : 0.f;
}

// ---- many tiles -------------------------------------------------------------------------------------------------
constexpr int kF8BN = 256, kF8Stages = 4, kF8Slots = 8;
constexpr uint32_t kF8Staging = 2048;                     // per warp: 32 rows of 64 bytes
constexpr size_t kF8Smem = size_t(kF8Stages) * (kF8ABytes + kF8BN * kF8Block) + kF8Slots * f8_slot<kF8BN>() + kF8Warps * kF8Staging +
                           1024 /* alignment */ + 512 /* barriers */;

struct F8Shape { int32_t m_tiles, n_tiles, blocks, total, group_m; };

__device__ __forceinline__ void f8_tile(const F8Shape& g, int t, int& mt, int& nt) {
    const int per = g.group_m * g.n_tiles, gi = t / per, first = gi * g.group_m;
    const int gm = min(g.group_m, g.m_tiles - first), in = t - gi * per;
    mt = first + in % gm;
    nt = in / gm;
}

// A warp's 32 rows by 128 columns of the output, turned through shared memory 64 bytes of each row at a time so that
// four lanes store 64 consecutive bytes.
template <class T>
__device__ __forceinline__ void f8_store(const F8Out& o, int64_t m0, int n0, const uint64_t (&acc)[64], uint32_t sw) {
    constexpr int kCols = 64 / int(sizeof(T)), kPer = 16 / int(sizeof(T));
    const int lane = threadIdx.x & 31;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < 128; c += kCols) {
        const int n = n0 + c;
        if (m0 >= o.M || n >= o.N) break;
        float f[kCols];
#pragma unroll
        for (int i = 0; i < kCols; i += 2) {
            ptx::unpack_f32x2(acc[(c + i) / 2], f[i], f[i + 1]);
            if (m0 + lane < o.M) {                        // rows and columns beyond the matrix are sums of zeros
                f[i] = f8_finish<T>(f[i], bad);
                f[i + 1] = f8_finish<T>(f[i + 1], bad);
            }
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 w;
            if constexpr (sizeof(T) == 2)
                w = make_uint4(pack_bf16x2(f[8 * j], f[8 * j + 1]), pack_bf16x2(f[8 * j + 2], f[8 * j + 3]),
                               pack_bf16x2(f[8 * j + 4], f[8 * j + 5]), pack_bf16x2(f[8 * j + 6], f[8 * j + 7]));
            else
                w = make_uint4(__float_as_uint(f[4 * j]), __float_as_uint(f[4 * j + 1]), __float_as_uint(f[4 * j + 2]), __float_as_uint(f[4 * j + 3]));
            ptx::sts128(sw + lane * 64 + ((j ^ ((lane >> 1) & 3)) << 4), w);
        }
        __syncwarp();
        if (o.aligned) {
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int r = it * 8 + (lane >> 2), j = lane & 3, col = n + j * kPer;
                const uint4 w = ptx::lds128(sw + r * 64 + ((j ^ ((r >> 1) & 3)) << 4));
                if (m0 + r >= o.M || col >= o.N) continue;
                T* p = static_cast<T*>(o.y) + (m0 + r) * o.ldy + col;
                if (col + kPer <= o.N) {
                    *reinterpret_cast<uint4*>(p) = w;
                } else {
                    const uint32_t part[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        if (col + i >= o.N) break;
                        if constexpr (sizeof(T) == 2) p[i] = T(part[i / 2] >> (i % 2 * 16));
                        else p[i] = __uint_as_float(part[i]);
                    }
                }
            }
        } else {
            // a warp stores 32 consecutive bf16, or two rows of 16 consecutive fp32
            constexpr int kRows = 32 / kCols;
            for (int r0 = 0; r0 < 32; r0 += kRows) {
                const int r = r0 + lane / kCols, col = lane % kCols, j = col / kPer;
                const uint32_t at = sw + r * 64 + ((j ^ ((r >> 1) & 3)) << 4) + (col % kPer) * int(sizeof(T));
                if (m0 + r >= o.M || n + col >= o.N) continue;
                T* p = static_cast<T*>(o.y) + (m0 + r) * o.ldy + n + col;
                if constexpr (sizeof(T) == 2) {
                    *p = ptx::lds_u16(at);
                } else {
                    float v;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
                    *p = v;
                }
            }
        }
    }
    if (bad && o.status) atomicOr(o.status, TPPO_DEV_NONFINITE);
}

template <class T, bool BROWS>
__global__ void __launch_bounds__(kF8Threads, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_sa,
                const __grid_constant__ CUtensorMap map_sb, const F8Square square, const F8Shape g, const F8Out out) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    typedef F8Ring<kF8BN, kF8Stages, kF8Slots, true, BROWS> Ring;
    const uint32_t scales = base + kF8Stages * Ring::kStage, staging = scales + kF8Slots * f8_slot<kF8BN>();
    const uint32_t bars = staging + kF8Warps * kF8Staging;
    const uint32_t full = bars, empty = full + 8 * kF8Stages, sfull = empty + 8 * kF8Stages, sempty = sfull + 8 * kF8Slots;
    const uint32_t acc_full = sempty + 8 * kF8Slots, acc_empty = acc_full + 16, slot = acc_empty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kF8Stages; ++s) {
            ptx::mbar_init(full + 8 * s, 1);
            ptx::mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < kF8Slots; ++s) {
            ptx::mbar_init(sfull + 8 * s, 1);
            ptx::mbar_init(sempty + 8 * s, kF8Warps);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(acc_full + 8 * a, 1);
            ptx::mbar_init(acc_empty + 8 * a, kF8Warps);
        }
        ptx::fence_mbar_init_cluster();
        umma::prefetch_tensormap(&map_a);
        umma::prefetch_tensormap(&map_b);
        umma::prefetch_tensormap(&map_sa);
        if (BROWS) umma::prefetch_tensormap(&map_sb);
    }
    if (warp == 1) {
        umma::tmem_alloc(slot, 512);
        umma::tmem_relinquish();
    }
    umma::fence_before_thread_sync();
    __syncthreads();
    umma::fence_after_thread_sync();
    const uint32_t tmem = *reinterpret_cast<uint32_t*>(smem_raw + (slot - raw));
    pdl_launch();                        // only now, with the tensor memory in hand: a dependent CTA on this SM allocates too
    pdl_wait();

    bool timed_out = false;
    if (warp == 0) {
        if (lane == 0) {
            Ring ring{base, scales, full, empty, sfull, sempty};
            for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
                int mt, nt;
                f8_tile(g, t, mt, nt);
                timed_out = !ring.load(&map_a, &map_b, &map_sa, &map_sb, mt * kF8TileM, nt * kF8BN, 0, g.blocks);
            }
            if (timed_out) ring.drain();
        }
    } else if (warp == 1) {
        if (lane == 0) {
            Ring ring{base, scales, full, empty, sfull, sempty};
            uint32_t n = 0;              // blocks so far: they take the two accumulators in turn
            for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
                for (int kb = 0; kb < g.blocks; ++kb, ++n) {
                    const uint32_t acc = n & 1;
                    if (!ptx::mbar_wait<false>(acc_empty + 8 * acc, ((n >> 1) & 1) ^ 1u)) { timed_out = true; break; }
                    umma::fence_after_thread_sync();
                    if (!ring.multiply(tmem + acc * kF8BN)) { timed_out = true; break; }
                    umma::mma_commit(acc_full + 8 * acc);
                }
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lanes = uint32_t(q * 32) << 16, sw = staging + (warp - 2) * kF8Staging;
        uint32_t n = 0, sslot = 0, sphase = 0;
        for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
            int mt, nt;
            f8_tile(g, t, mt, nt);
            const int n0 = nt * kF8BN + half * 128;
            const float* sq = nullptr;
            if (!BROWS) sq = square.p + int64_t(n0 < out.N ? n0 / 128 : 0) * square.ld;
            float sb = BROWS ? 1.f : __ldg(sq);
            uint64_t acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0;
            for (int kb = 0; kb < g.blocks; ++kb, ++n) {
                const float sb_next = !BROWS && kb + 1 < g.blocks ? __ldg(sq + kb + 1) : 1.f;
                if (!ptx::mbar_wait_warp<false>(sfull + 8 * sslot, sphase)) { timed_out = true; break; }
                const uint32_t s = scales + sslot * Ring::kSlot;
                float sa;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(sa) : "r"(s + (q * 32 + lane) * 4));
                if (!ptx::mbar_wait_warp<false>(acc_full + 8 * (n & 1), (n >> 1) & 1)) { timed_out = true; break; }
                umma::fence_after_thread_sync();
                f8_scale<128, BROWS>(tmem + lanes + (n & 1) * kF8BN + half * 128, sa * sb, s + kF8TileM * 4 + half * 512, acc);
                umma::fence_before_thread_sync();
                __syncwarp();
                if (lane == 0) {
                    ptx::mbar_arrive(acc_empty + 8 * (n & 1));
                    ptx::mbar_arrive(sempty + 8 * sslot);
                }
                if (++sslot == kF8Slots) { sslot = 0; sphase ^= 1u; }
                sb = sb_next;
            }
            if (!timed_out) f8_store<T>(out, int64_t(mt) * kF8TileM + q * 32, n0, acc, sw);
        }
    }
    if (timed_out && out.status) atomicOr(out.status, TPPO_DEV_WAIT_TIMEOUT);
    umma::fence_before_thread_sync();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        umma::tmem_dealloc(tmem, 512);
    }
}

// ---- few tiles --------------------------------------------------------------------------------------------------
// Accumulator rows: output columns n; accumulator columns: output rows m.  Each of the cluster's CTAs owns ceil(BN /
// CTAs) accumulator columns: every CTA stores its partial sums into the owner's shared memory, and after one cluster
// barrier the owner adds them in rank order.  Up to 64 columns the sums have memory of their own and two CTAs share an
// SM; 128 columns lay them over the operand ring, which needs one more barrier.
template <int BN> __host__ __device__ constexpr bool f8_overlay() { return BN >= 128; }
template <int BN> __host__ __device__ constexpr int f8_stages() { return BN <= 16 ? 5 : BN <= 32 ? 4 : BN <= 64 ? 3 : 6; }
constexpr int kF8SplitSlots = 4;
template <int BN> __host__ __device__ constexpr uint32_t f8_ring() { return uint32_t(f8_stages<BN>()) * (kF8ABytes + BN * kF8Block); }
template <int BN> __host__ __device__ constexpr uint32_t f8_body() { return f8_ring<BN>() + (f8_overlay<BN>() ? 0u : (BN + 8) * 128 * 4); }
template <int BN> __host__ __device__ constexpr size_t f8_split_smem() {
    return f8_body<BN>() + kF8SplitSlots * f8_slot<BN>() + 1024 /* alignment */ + 256 /* barriers */;
}

struct F8SplitShape { int32_t col_tiles, blocks; };

template <class T, int BN, bool AROWS>
__global__ void __launch_bounds__(kF8Threads, BN <= 64 ? 2 : 1)
fp8_split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_sa,
                 const __grid_constant__ CUtensorMap map_sb, const F8Square square, const F8SplitShape g, const F8Out out) {
    constexpr int STAGES = f8_stages<BN>(), kEpiThreads = kF8Threads - 64, kHalf = BN / 2;
    constexpr uint32_t kCols = 2 * BN < 32 ? 32 : 2 * BN;             // two accumulators
    extern __shared__ uint8_t smem_raw[];
    // dynamic shared memory starts at the same address in every CTA of a kernel, so `sums` is common to the cluster
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    typedef F8Ring<BN, STAGES, kF8SplitSlots, AROWS, true> Ring;
    const uint32_t sums = base + (f8_overlay<BN>() ? 0u : f8_ring<BN>()), scales = base + f8_body<BN>();
    const uint32_t bars = scales + kF8SplitSlots * f8_slot<BN>();
    const uint32_t full = bars, empty = full + 8 * STAGES, sfull = empty + 8 * STAGES, sempty = sfull + 8 * kF8SplitSlots;
    const uint32_t acc_full = sempty + 8 * kF8SplitSlots, acc_empty = acc_full + 16, slot = acc_empty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = int(ptx::cluster_ctarank());
    int splits;
    asm volatile("mov.u32 %0, %cluster_nctarank;" : "=r"(splits));
    const int tile = int(blockIdx.x) / splits;
    const int rt = tile / g.col_tiles, ct = tile % g.col_tiles;
    const int k0 = int(int64_t(g.blocks) * rank / splits), k1 = int(int64_t(g.blocks) * (rank + 1) / splits);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            ptx::mbar_init(full + 8 * s, 1);
            ptx::mbar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < kF8SplitSlots; ++s) {
            ptx::mbar_init(sfull + 8 * s, 1);
            ptx::mbar_init(sempty + 8 * s, kF8Warps);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(acc_full + 8 * a, 1);
            ptx::mbar_init(acc_empty + 8 * a, kF8Warps);
        }
        ptx::fence_mbar_init_cluster();
        umma::prefetch_tensormap(&map_a);
        umma::prefetch_tensormap(&map_b);
        if (AROWS) umma::prefetch_tensormap(&map_sa);
        umma::prefetch_tensormap(&map_sb);
    }
    if (warp == 1) {
        umma::tmem_alloc(slot, kCols);
        umma::tmem_relinquish();
    }
    umma::fence_before_thread_sync();
    __syncthreads();
    ptx::cluster_sync_all();                 // every CTA of the cluster runs: its shared memory may be written
    umma::fence_after_thread_sync();
    const uint32_t tmem = *reinterpret_cast<uint32_t*>(smem_raw + (slot - raw));
    pdl_launch();
    pdl_wait();

    bool timed_out = false;
    uint64_t acc[kHalf / 2];
#pragma unroll
    for (int i = 0; i < kHalf / 2; ++i) acc[i] = 0;
    const int q = warp & 3, half = (warp - 2) >> 2;
    if (warp == 0) {
        if (lane == 0) {
            Ring ring{base, scales, full, empty, sfull, sempty};
            timed_out = !ring.load(&map_a, &map_b, &map_sa, &map_sb, rt * kF8TileM, ct * BN, k0, k1);
            if (timed_out) ring.drain();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            Ring ring{base, scales, full, empty, sfull, sempty};
            for (uint32_t n = 0; n < uint32_t(k1 - k0); ++n) {
                if (!ptx::mbar_wait<false>(acc_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1u)) { timed_out = true; break; }
                umma::fence_after_thread_sync();
                if (!ring.multiply(tmem + (n & 1) * BN)) { timed_out = true; break; }
                umma::mma_commit(acc_full + 8 * (n & 1));
            }
        }
        __syncwarp();
    } else {
        const uint32_t lanes = uint32_t(q * 32) << 16;
        const float* sq = AROWS ? nullptr : square.p + int64_t(rt) * square.ld;
        uint32_t sslot = 0, sphase = 0;
        float sa_next = AROWS || k0 >= k1 ? 1.f : __ldg(sq + k0);
        for (int kb = k0; kb < k1; ++kb) {
            const uint32_t n = uint32_t(kb - k0);
            float sa = sa_next;
            if (!AROWS && kb + 1 < k1) sa_next = __ldg(sq + kb + 1);
            if (!ptx::mbar_wait_warp<false>(sfull + 8 * sslot, sphase)) { timed_out = true; break; }
            const uint32_t s = scales + sslot * Ring::kSlot;
            if (AROWS) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(sa) : "r"(s + (q * 32 + lane) * 4));
            if (!ptx::mbar_wait_warp<false>(acc_full + 8 * (n & 1), (n >> 1) & 1)) { timed_out = true; break; }
            umma::fence_after_thread_sync();
            f8_scale<kHalf, true>(tmem + lanes + (n & 1) * BN + half * kHalf, sa, s + kF8TileM * 4 + half * kHalf * 4, acc);
            umma::fence_before_thread_sync();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive(acc_empty + 8 * (n & 1));
                ptx::mbar_arrive(sempty + 8 * sslot);
            }
            if (++sslot == kF8SplitSlots) { sslot = 0; sphase ^= 1u; }
        }
    }
    if (f8_overlay<BN>()) ptx::cluster_sync_all();       // every ring of the cluster has been consumed
    const int own = (BN + splits - 1) / splits, c0 = rank * own;
    if (warp >= 2 && !timed_out) {
        const int r = q * 32 + lane;
        int owner = half * kHalf / own, in = half * kHalf - owner * own;
#pragma unroll
        for (int i = 0; i < kHalf; ++i) {
            // [source rank][owned column][128 rows] at the owner
            float lo, hi;
            ptx::unpack_f32x2(acc[i / 2], lo, hi);
            const uint32_t at = ptx::map_to_cta(sums + ((rank * own + in) * 128 + r) * 4, uint32_t(owner));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(i & 1 ? hi : lo) : "memory");
            if (++in == own) { in = 0; ++owner; }
        }
    }
    umma::fence_before_thread_sync();
    ptx::cluster_sync_all();                 // all partial sums have arrived; nobody writes here any more
    umma::fence_after_thread_sync();
    if (warp >= 2) {
        const int units = max(0, min(own, BN - c0)) * 16;
        bool bad = false;
#pragma unroll 1
        for (int u = int(threadIdx.x) - 64; u < units; u += kEpiThreads) {
            const int64_t m = int64_t(ct) * BN + c0 + u / 16;
            const int n = rt * kF8TileM + (u % 16) * 8;
            if (m >= out.M || n >= out.N) continue;
            float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            uint32_t p = sums + ((u / 16) * 128 + (u % 16) * 8) * 4;
            for (int s = 0; s < splits; ++s, p += uint32_t(own) * 512) {
                const uint4 a = ptx::lds128(p), b = ptx::lds128(p + 16);
                w[0] += __uint_as_float(a.x); w[1] += __uint_as_float(a.y);
                w[2] += __uint_as_float(a.z); w[3] += __uint_as_float(a.w);
                w[4] += __uint_as_float(b.x); w[5] += __uint_as_float(b.y);
                w[6] += __uint_as_float(b.z); w[7] += __uint_as_float(b.w);
            }
            T* y = static_cast<T*>(out.y) + m * out.ldy + n;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = f8_finish<T>(w[i], bad);
            if (out.aligned && n + 8 <= out.N) {
                store_vec<8>(y, w);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (n + i < out.N) store_f32(y + i, w[i]);
            }
        }
        if (bad && out.status) atomicOr(out.status, TPPO_DEV_NONFINITE);
    } else if (warp == 1) {
        umma::tmem_dealloc(tmem, kCols);     // all tensor-memory loads are behind the barrier
    }
    if (timed_out && out.status) atomicOr(out.status, TPPO_DEV_WAIT_TIMEOUT);
}

// ---- host side --------------------------------------------------------------------------------------------------
struct F8Operand { const void* p; int64_t rows, ld; const float* scale; int64_t lds; bool by_rows; };

// How a product is cut: bn 0 = the persistent kernel, else the split kernel's columns (output rows) per tile and the
// CTAs that share a tile's contraction: the least estimated time in SM clocks.  A block of 128 bytes moves as many
// operand bytes as a step of the 16-bit products, whose fitted constants serve here.
struct F8Cut { int bn, splits; };
F8Cut f8_cut(int64_t m, int64_t n, int64_t blocks) {
    // CTAs that fit on the GPU at once in clusters of s, at two and at one per SM (the driver's count)
    static const int64_t pair[9] = {0, 296, 296, 279, 284, 280, 270, 259, 264};
    static const int64_t alone[9] = {0, 148, 148, 135, 132, 130, 132, 105, 120};
    const int64_t rows = (n + 127) / 128, big = (m + 127) / 128 * ((n + 255) / 256);
    F8Cut best{0, 1};
    int64_t least = 5000 + (big + kNumSms - 1) / kNumSms * blocks * 600 + 4000;
    for (int bn = 16; bn <= 128; bn *= 2) {
        const int64_t tiles = rows * ((m + bn - 1) / bn);
        const int64_t stages = bn <= 16 ? 5 : bn <= 32 ? 4 : bn <= 64 ? 3 : 6;
        for (int s = 1; s <= 8 && (s == 1 || blocks >= 2 * s); ++s) {
            const int64_t slots = bn <= 64 ? pair[s] : alone[s];
            const int64_t waves = (tiles * s + slots - 1) / slots, steps = (blocks + s - 1) / s;
            const int64_t both = bn <= 64 && tiles * s > kNumSms ? 2 : 1;         // CTAs that share an SM
            int64_t step = 2500 / (stages * both);
            if (step < 2 * (128 + bn)) step = 2 * (128 + bn);
            const int64_t cost = waves * (2500 * (1 + both) + steps * both * step + ((bn + s - 1) / s * 62 + bn * 28) * (1 + both) / 2);
            if (cost < least) { least = cost; best = {bn, s}; }
        }
        if (bn >= m) break;                  // one tile holds all output rows already
    }
    return best;
}

template <class T, bool BROWS>
int f8_gemm(const F8Operand& a, const F8Operand& b, int64_t K, int64_t blocks, const F8Out& out, cudaStream_t s) {
    CUtensorMap ma, mb, msa, msb{};
    if (!make_u8_tensor_map(&ma, a.p, a.rows, K, a.ld, kF8TileM) || !make_u8_tensor_map(&mb, b.p, b.rows, K, b.ld, kF8BN) ||
        !make_f32_tensor_map(&msa, a.scale, blocks, a.rows, a.lds, kF8TileM) ||
        (BROWS && !make_f32_tensor_map(&msb, b.scale, blocks, b.rows, b.lds, kF8BN)))
        return TPPO_ERR_CUDA;
    F8Shape g;
    g.m_tiles = int32_t((a.rows + kF8TileM - 1) / kF8TileM);
    g.n_tiles = int32_t((b.rows + kF8BN - 1) / kF8BN);
    g.blocks = int32_t(blocks);
    g.group_m = 16;
    const int64_t total = int64_t(g.m_tiles) * g.n_tiles;
    if (total > 0x7fffffff - kNumSms) return TPPO_ERR_UNSUPPORTED;
    g.total = int32_t(total);
    auto kernel = fp8_gemm_kernel<T, BROWS>;
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kF8Smem)));
    const int grid = g.total < kNumSms ? g.total : kNumSms;
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(grid), dim3(kF8Threads), kF8Smem, s, ma, mb, msa, msb, F8Square{b.scale, b.lds}, g, out));
    return TPPO_OK;
}

template <class T, int BN, bool AROWS>
int f8_split(const F8Operand& a, const F8Operand& b, int64_t K, int64_t blocks, int splits, const F8Out& out, cudaStream_t s) {
    CUtensorMap ma, mb, msa{}, msb;
    if (!make_u8_tensor_map(&ma, a.p, a.rows, K, a.ld, kF8TileM) || !make_u8_tensor_map(&mb, b.p, b.rows, K, b.ld, BN) ||
        (AROWS && !make_f32_tensor_map(&msa, a.scale, blocks, a.rows, a.lds, kF8TileM)) ||
        !make_f32_tensor_map(&msb, b.scale, blocks, b.rows, b.lds, BN))
        return TPPO_ERR_CUDA;
    F8SplitShape g;
    const int64_t row_tiles = (a.rows + kF8TileM - 1) / kF8TileM, col_tiles = (b.rows + BN - 1) / BN;
    if (row_tiles * col_tiles * splits > 0x7fffffff) return TPPO_ERR_UNSUPPORTED;
    g.col_tiles = int32_t(col_tiles);
    g.blocks = int32_t(blocks);
    auto kernel = fp8_split_kernel<T, BN, AROWS>;
    constexpr size_t smem = f8_split_smem<BN>();
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)));
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(row_tiles * col_tiles * splits));
    cfg.blockDim = dim3(kF8Threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(splits);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    TPPO_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, ma, mb, msa, msb, F8Square{a.scale, a.lds}, g, out));
    return TPPO_OK;
}

template <class T, bool BROWS>
int f8_product(const F8Operand& a, const F8Operand& b, int64_t K, const F8Out& out, cudaStream_t s) {
    const int64_t blocks = (K + kF8Block - 1) / kF8Block;
    const F8Cut c = f8_cut(a.rows, b.rows, blocks);
    switch (c.bn) {                          // the split kernel's rows are the output's columns
        case 16: return f8_split<T, 16, BROWS>(b, a, K, blocks, c.splits, out, s);
        case 32: return f8_split<T, 32, BROWS>(b, a, K, blocks, c.splits, out, s);
        case 64: return f8_split<T, 64, BROWS>(b, a, K, blocks, c.splits, out, s);
        case 128: return f8_split<T, 128, BROWS>(b, a, K, blocks, c.splits, out, s);
        default: return f8_gemm<T, BROWS>(a, b, K, blocks, out, s);
    }
}

int64_t whole(int64_t ld, int64_t unit) { return (ld + unit - 1) / unit * unit; }

}  // namespace
}  // namespace tppo

TPPO_API int tppo_fp8_matmul(const void* a, int64_t lda, const float* a_scale, int64_t ldas, const void* b, int64_t ldb,
                             const float* b_scale, int64_t ldbs, int32_t b_block, int64_t M, int64_t N, int64_t K, void* y, int32_t y_dtype,
                             int64_t ldy, int32_t* status, void* stream) {
    using namespace tppo;
    if (M < 0 || N < 0 || K < 0 || (y_dtype != TPPO_BF16 && y_dtype != TPPO_F32) || (b_block != TPPO_FP8_ROWS && b_block != TPPO_FP8_SQUARE))
        return TPPO_ERR_INVALID_ARG;
    if (M > kDenseMaxSize || N > kDenseMaxSize || K > kDenseMaxSize) return TPPO_ERR_UNSUPPORTED;
    const size_t e = y_dtype == TPPO_F32 ? 4 : 2;
    if (!aligned(status, 4) || !aligned(y, e)) return TPPO_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return TPPO_OK;
    if (!y || ldy < N) return TPPO_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (K == 0) {
        TPPO_CUDA_CHECK(cudaMemset2DAsync(y, size_t(ldy) * e, 0, size_t(N) * e, size_t(M), s));
        return TPPO_OK;
    }
    const int64_t kb = (K + kF8Block - 1) / kF8Block;
    const bool rows = b_block == TPPO_FP8_ROWS;
    if (!a || !a_scale || !b || !b_scale || !aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 16) || !aligned(b_scale, rows ? 16 : 4))
        return TPPO_ERR_INVALID_ARG;
    // a matrix of one row needs no stride
    if (lda < K || ldb < K || (M > 1 && lda % 16) || (N > 1 && ldb % 16) || ldas < M || (kb > 1 && ldas % 4) || ldbs < (rows ? N : kb) ||
        (rows && kb > 1 && ldbs % 4))
        return TPPO_ERR_INVALID_ARG;
    const F8Operand oa{a, M, whole(lda, 16), a_scale, whole(ldas, 4), true};
    const F8Operand ob{b, N, whole(ldb, 16), b_scale, rows ? whole(ldbs, 4) : ldbs, rows};
    const F8Out out{y, ldy, M, int32_t(N), status, rows_aligned(y, ldy, e)};
    if (y_dtype == TPPO_F32) return rows ? f8_product<float, true>(oa, ob, K, out, s) : f8_product<float, false>(oa, ob, K, out, s);
    return rows ? f8_product<bf16_bits, true>(oa, ob, K, out, s) : f8_product<bf16_bits, false>(oa, ob, K, out, s);
}
