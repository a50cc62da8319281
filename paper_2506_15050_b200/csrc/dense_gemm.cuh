// The two tensor-core products behind the dense operators: D = A * B over 16-bit operands (bf16, or
// fp16 with F16) with fp32 accumulation in tensor memory, and a caller-supplied epilogue that gets
// finished fp32 values eight at a time along the contiguous dimension of its outputs.
//
//   dense_gemm_kernel   many output tiles: persistent CTAs, 128 x 256 tiles, two accumulators so
//                       that the epilogue of a tile overlaps the main loop of the next.  Output
//                       rows are accumulator rows.  With SYM only the tiles that touch the lower
//                       triangle of a symmetric product are computed, and the epilogue writes each
//                       element to its mirrored place too.  16384 x 5120 x 5120: 600 us, 1430 TFLOP/s.
//   dense_split_kernel  few output tiles (one to some hundred tokens, small matrices): the output is
//                       taken TRANSPOSED -- the 128 accumulator rows run along the contiguous output
//                       dimension, the BN columns along its rows, so that one token costs a 16-wide
//                       instruction instead of a 128-high tile -- and the contraction is split over the
//                       CTAs of a cluster, whose partial sums meet in distributed shared memory: no
//                       workspace, no second launch, a fixed order of addition.
//
// Roles of a CTA's warps: 0 TMA loads, 1 tcgen05.mma, 2-9 epilogue.  Every wait is bounded; one that
// runs out raises TPPO_DEV_WAIT_TIMEOUT, outputs are then incomplete, and tensor memory is released.
#pragma once

#include "dense_common.cuh"
#include "umma.cuh"
#include "umma_gemm.cuh"      // make_bf16_tensor_map

namespace tppo {

constexpr int kDenseTileM = 128;
constexpr int kDenseTileK = 64;                       // one 128-byte swizzled row of 16-bit elements
constexpr int kDenseThreads = 320;
constexpr int kDenseEpiWarps = 8;
constexpr uint32_t kDenseABytes = kDenseTileM * kDenseTileK * 2;      // 16 KB
constexpr uint32_t kDenseBox64 = 64 * kDenseTileK * 2;                // 64 x 64 box of an MN-major operand
constexpr uint32_t kDenseStageEpi = 32 * 32 * 4;                      // one warp's 32 x 32 fp32 chunk

// Instruction descriptor (see umma::instr_desc_bf16) for either 16-bit format.
template <bool F16>
__host__ __device__ constexpr uint32_t dense_instr_desc(int n, int a_mn, int b_mn) {
    const uint32_t d = umma::instr_desc_bf16(kDenseTileM, n, a_mn, b_mn);
    return F16 ? d & ~((7u << 7) | (7u << 10)) : d;
}

// 8 consecutive fp32 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr) : "memory");
}
// The operand ring both kernels share: producer and MMA issuer for one output tile.
template <int AMAJ, int BMAJ, bool F16, int BN, int STAGES>
struct DenseRing {
    static constexpr uint32_t kBBytes = BN * kDenseTileK * 2;
    static constexpr uint32_t kStage = kDenseABytes + kBBytes;
    uint32_t base, full, empty;
    int stage = 0;
    uint32_t phase = 0;

    __device__ __forceinline__ void next() {
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    // Loads k steps [k0, k1) of the tile whose first A and B indices are am and bn.
    __device__ __forceinline__ bool load(const CUtensorMap* ma, const CUtensorMap* mb, int am, int bn, int k0, int k1) {
        for (int ks = k0; ks < k1; ++ks) {
            if (!ptx::mbar_wait<false>(empty + 8 * stage, phase ^ 1u)) return false;
            const uint32_t fb = full + 8 * stage, sa = base + stage * kStage, sb = sa + kDenseABytes;
            ptx::mbar_arrive_expect_tx(fb, kStage);
            const int k = ks * kDenseTileK;
            if (AMAJ == 0) {
                umma::tma_load_2d(sa, ma, fb, k, am);
            } else {
#pragma unroll
                for (int q = 0; q < kDenseTileM / 64; ++q) umma::tma_load_2d(sa + q * kDenseBox64, ma, fb, am + 64 * q, k);
            }
            if (BMAJ == 0) {
                umma::tma_load_2d(sb, mb, fb, k, bn);
            } else {
#pragma unroll
                for (int q = 0; q < BN / 64; ++q) umma::tma_load_2d(sb + q * kDenseBox64, mb, fb, bn + 64 * q, k);
            }
            next();
        }
        return true;
    }
    // After a wait ran out: let the copies already issued land before the CTA's memory goes away.
    __device__ __forceinline__ void drain() {
        for (int s = 0; s < STAGES; ++s) {
            const uint32_t issued = s < stage ? phase : phase ^ 1u;       // parity of the stage's last load
            if (!ptx::mbar_wait<false>(full + 8 * s, issued)) return;
        }
    }
    __device__ __forceinline__ bool multiply(uint32_t d, int steps) {
        constexpr uint32_t idesc = dense_instr_desc<F16>(BN, AMAJ, BMAJ);
        constexpr uint32_t a_kstep = AMAJ ? 16 * 128 : 32, b_kstep = BMAJ ? 16 * 128 : 32;
        for (int ks = 0; ks < steps; ++ks) {
            if (!ptx::mbar_wait<false>(full + 8 * stage, phase)) return false;
            umma::fence_after_thread_sync();
            const uint32_t sa = base + stage * kStage, sb = sa + kDenseABytes;
            const uint64_t ad = umma::smem_desc(sa, AMAJ ? kDenseBox64 : 16, 1024);
            const uint64_t bd = umma::smem_desc(sb, BMAJ ? kDenseBox64 : 16, 1024);
#pragma unroll
            for (int j = 0; j < kDenseTileK / 16; ++j)
                umma::mma_bf16(d, umma::smem_desc_advance(ad, j * a_kstep), umma::smem_desc_advance(bd, j * b_kstep), idesc,
                               (ks | j) != 0 ? 1u : 0u);
            umma::mma_commit(empty + 8 * stage);
            next();
        }
        return true;
    }
};

// ---- many tiles ---------------------------------------------------------------------------------
constexpr int kDenseBN = 256;
constexpr int kDenseStages = 4;
constexpr size_t kDenseSmem = size_t(kDenseStages) * (kDenseABytes + kDenseBN * 128) + kDenseEpiWarps * kDenseStageEpi +
                              1024 /* alignment */ + 128 /* barriers */;

struct DenseShape {
    int32_t m_tiles, n_tiles, k_steps, total;
    int32_t group_m;          // m-tiles per raster group: tiles of a group run next to each other in time
    Link link;
};

template <bool SYM>
__device__ __forceinline__ void dense_tile(const DenseShape& g, int t, int& mt, int& nt) {
    if (SYM) {      // rows 2p and 2p+1 of tiles hold p+1 tiles each, p(p+1) tiles lie in front of them
        int p = int((sqrtf(4.f * float(t) + 1.f) - 1.f) * 0.5f);
        while (p * (p + 1) > t) --p;
        while ((p + 1) * (p + 2) <= t) ++p;
        const int in = t - p * (p + 1);
        mt = 2 * p + (in > p);
        nt = in > p ? in - p - 1 : in;
    } else {
        const int per = g.group_m * g.n_tiles, gi = t / per, first = gi * g.group_m;
        const int gm = min(g.group_m, g.m_tiles - first), in = t - gi * per;
        mt = first + in % gm;
        nt = in / gm;
    }
}

// Epi: bool outside(row, col) const -- nothing at or beyond (row, col) belongs to the matrix
//      void load(row, col, Loads&) const -- starts reading what the elements (row, col .. col+7) need
//      void operator()(row, col, float (&v)[8], const Loads&) const -- finishes them
// and for the persistent kernel, whose lanes go down their eight columns eight rows at a time: Cursor, what
// stays the same on the way; open(Cursor&, row, col); fetch(cursor, trip, Loads&) as load; finish<true>(
// cursor, trip, v, loads) as operator().
// kRows: whether there are bool by_rows() const (uniform), finish<false> -- all but the stores of the
// main output, whose values stay in v -- and put(row, col, float), which stores one.
// Rows and columns may lie outside the matrix.

// Where 16-byte piece `piece` of row `row` of a warp's 32 x 32 chunk sits: XORed with a swizzle of the row,
// so that rows written by lane, pieces of rows and pieces of columns are all read and written without a
// bank conflict.
__device__ __forceinline__ uint32_t dense_piece(int row, int piece) {
    return uint32_t(row * 128 + ((piece ^ (row & 7) ^ ((row >> 3) << 1)) << 4));
}
// One warp's share of a finished tile: 32 accumulator rows (output rows m0 ..) by 128 columns (output
// columns n_first ..) at tensor-memory address `taddr`, 32 x 32 at a time.  `sw`: its 4 KB of shared memory.
template <bool SYM, class Epi>
__device__ __forceinline__ void dense_epilogue(const Epi& epi, int64_t m0, int n_first, uint32_t taddr, uint32_t sw) {
    const int lane = threadIdx.x & 31;
    // rows of the output that take no 16-byte stores: the finished values go back to shared memory, and a
    // warp stores 32 consecutive elements at a time
    bool by_rows = false;
    if constexpr (Epi::kRows) by_rows = epi.by_rows();
#pragma unroll 1
    for (int c = 0; c < kDenseBN / 2; c += 32) {
        const int n0 = n_first + c;
        if (SYM && n0 > m0) break;            // above the diagonal: another chunk's mirror image
        if (epi.outside(m0, n0)) break;
        // a lane finishes eight elements of four rows, eight apart -- and, below the diagonal of a symmetric
        // product, of their mirror images.  What the epilogue reads is fetched while the accumulator is
        // fetched and turned.
        constexpr int kPasses = SYM ? 2 : 1;
        const bool mirrored = SYM && n0 < m0;
        typename Epi::Cursor cursor[kPasses];
        typename Epi::Loads ahead[kPasses][4];
        epi.open(cursor[0], m0 + (lane >> 2), n0 + (lane & 3) * 8);
#pragma unroll
        for (int it = 0; it < 4; ++it) epi.fetch(cursor[0], it, ahead[0][it]);
        if constexpr (SYM) {
            if (mirrored) {
                epi.open(cursor[1], int64_t(n0) + (lane >> 2), int(m0) + (lane & 3) * 8);
#pragma unroll
                for (int it = 0; it < 4; ++it) epi.fetch(cursor[1], it, ahead[1][it]);
            }
        }
        uint32_t v[32];
        umma::tmem_ld32(taddr + c, v);
        umma::tmem_ld_wait();
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            ptx::sts128(sw + dense_piece(lane, j), make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
        __syncwarp();
        // one copy of a long epilogue's code: unrolled it does not fit the instruction cache (134 us instead
        // of 116 for 16384 x 5120 outputs of a 128-long contraction); the short ones of the symmetric
        // products gain from four (2304 x 2304 update 500 -> 455 us)
#pragma unroll(SYM ? 4 : 1)
        for (int it = 0; it < 4; ++it) {
            const typename Epi::Loads mine = ahead[0][0];
#pragma unroll
            for (int i = 0; i < 3; ++i) ahead[0][i] = ahead[0][i + 1];
            const int r = it * 8 + (lane >> 2), j = (lane & 3) * 2;
            const uint4 lo = ptx::lds128(sw + dense_piece(r, j)), hi = ptx::lds128(sw + dense_piece(r, j + 1));
            float w[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                          __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
            if constexpr (Epi::kRows) {
                if (by_rows) {
                    epi.template finish<false>(cursor[0], it, w, mine);
                    ptx::sts128(sw + dense_piece(r, j), make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]),
                                                                   __float_as_uint(w[2]), __float_as_uint(w[3])));
                    ptx::sts128(sw + dense_piece(r, j + 1), make_uint4(__float_as_uint(w[4]), __float_as_uint(w[5]),
                                                                       __float_as_uint(w[6]), __float_as_uint(w[7])));
                    continue;
                }
            }
            epi.template finish<true>(cursor[0], it, w, mine);
        }
        if constexpr (Epi::kRows) {
            if (by_rows) {
                __syncwarp();
#pragma unroll 8
                for (int r = 0; r < 32; ++r) {
                    float f;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(sw + dense_piece(r, lane >> 2) + (lane & 3) * 4));
                    epi.put(m0 + r, n0 + lane, f);
                }
            }
        }
        if constexpr (SYM) {
            if (mirrored) {
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int col = it * 8 + (lane >> 2), r0 = (lane & 3) * 8;
                    float w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w[i])
                                     : "r"(sw + dense_piece(r0 + i, col >> 2) + (col & 3) * 4));
                    epi.template finish<true>(cursor[1], it, w, ahead[1][it]);
                }
            }
        }
    }
}

template <int AMAJ, int BMAJ, bool F16, bool SYM, class Epi>
__global__ void __launch_bounds__(kDenseThreads, 1)
dense_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const DenseShape g,
                  const Epi epi, int32_t* status) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    typedef DenseRing<AMAJ, BMAJ, F16, kDenseBN, kDenseStages> Ring;
    const uint32_t stage_epi = base + kDenseStages * Ring::kStage;
    const uint32_t bars = stage_epi + kDenseEpiWarps * kDenseStageEpi;
    const uint32_t full = bars, empty = bars + 8 * kDenseStages;
    const uint32_t acc_full = bars + 16 * kDenseStages, acc_empty = acc_full + 16, slot = acc_empty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kDenseStages; ++s) {
            ptx::mbar_init(full + 8 * s, 1);
            ptx::mbar_init(empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(acc_full + 8 * a, 1);
            ptx::mbar_init(acc_empty + 8 * a, kDenseEpiWarps);
        }
        ptx::fence_mbar_init_cluster();
        umma::prefetch_tensormap(&map_a);
        umma::prefetch_tensormap(&map_b);
    }
    if (warp == 1) {
        umma::tmem_alloc(slot, 512);
        umma::tmem_relinquish();
    }
    umma::fence_before_thread_sync();
    __syncthreads();
    umma::fence_after_thread_sync();
    const uint32_t tmem = *reinterpret_cast<uint32_t*>(smem_raw + (slot - raw));
    // only now, with the tensor memory in hand: a dependent CTA on this SM allocates too
    link_begin(g.link);

    bool timed_out = false;
    if (warp == 0) {
        if (lane == 0) {
            Ring ring{base, full, empty};
            for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
                int mt, nt;
                dense_tile<SYM>(g, t, mt, nt);
                timed_out = !ring.load(&map_a, &map_b, mt * kDenseTileM, nt * kDenseBN, 0, g.k_steps);
            }
            if (timed_out) ring.drain();
        }
    } else if (warp == 1) {
        if (lane == 0) {
            Ring ring{base, full, empty};
            int local = 0;
            for (int t = blockIdx.x; t < g.total; t += gridDim.x, ++local) {
                const int acc = local & 1;
                if (!ptx::mbar_wait<false>(acc_empty + 8 * acc, ((local >> 1) & 1) ^ 1u)) { timed_out = true; break; }
                umma::fence_after_thread_sync();
                if (!ring.multiply(tmem + acc * kDenseBN, g.k_steps)) { timed_out = true; break; }
                umma::mma_commit(acc_full + 8 * acc);
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t sw = stage_epi + (warp - 2) * kDenseStageEpi;
        int local = 0;
        for (int t = blockIdx.x; t < g.total; t += gridDim.x, ++local) {
            int mt, nt;
            dense_tile<SYM>(g, t, mt, nt);
            const int acc = local & 1;
            if (!ptx::mbar_wait_warp<false>(acc_full + 8 * acc, (local >> 1) & 1)) { timed_out = true; break; }
            umma::fence_after_thread_sync();
            dense_epilogue<SYM>(epi, int64_t(mt) * kDenseTileM + q * 32, nt * kDenseBN + half * (kDenseBN / 2),
                                tmem + acc * kDenseBN + (uint32_t(q * 32) << 16) + half * (kDenseBN / 2), sw);
            umma::fence_before_thread_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * acc);
        }
    }
    if (timed_out && status) atomicOr(status, TPPO_DEV_WAIT_TIMEOUT);
    umma::fence_before_thread_sync();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        umma::tmem_dealloc(tmem, 512);
    }
    link_end(g.link);
}

// ---- few tiles ----------------------------------------------------------------------------------
// Accumulator rows: output columns (contiguous); accumulator columns: output rows.  A is therefore
// the operand indexed by the output column, B the one indexed by the output row.
//
// Each of the cluster's CTAs owns ceil(BN / CTAs) accumulator columns: every CTA stores its partial sums
// straight from tensor memory into the owner's shared memory, and after one cluster barrier the owner
// adds them in rank order and runs the epilogue.  (Letting the owner fetch them instead costs a second
// barrier and a remote round trip: 11-13 us instead of 8-9 per launch of a chain of small products.)
// Up to 64 columns the sums have memory of their own and two CTAs share an SM; wider tiles lay them over
// the operand ring, which needs one more barrier (every CTA has consumed its ring) but leaves 192 KB to
// the ring: at some 2000 clocks of loaded L2 latency the operand rate is the bytes in flight, and a
// 128-column tile with 128 KB was bound by them.
template <int BN> __host__ __device__ constexpr bool dense_split_overlay() { return BN >= 128; }
template <int BN> __host__ __device__ constexpr int dense_split_stages() {
    return BN <= 16 ? 5 : BN <= 32 ? 4 : BN <= 64 ? 3 : BN <= 128 ? 6 : 4;
}
template <int BN> __host__ __device__ constexpr uint32_t dense_split_ring() {
    return uint32_t(dense_split_stages<BN>()) * (kDenseABytes + BN * 128);
}
template <int BN> __host__ __device__ constexpr uint32_t dense_split_body() {
    return dense_split_ring<BN>() + (dense_split_overlay<BN>() ? 0u : (BN + 8) * 128 * 4);
}
template <int BN> __host__ __device__ constexpr size_t dense_split_smem() {
    return dense_split_body<BN>() + 1024 /* alignment */ + 128 /* barriers */;
}

struct DenseSplitShape {
    int32_t col_tiles;        // tiles along the output rows (BN each)
    int32_t k_steps;
    Link link;
};

template <int AMAJ, int BMAJ, bool F16, int BN, class Epi>
__global__ void __launch_bounds__(kDenseThreads)
dense_split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const DenseSplitShape g, const Epi epi, int32_t* status) {
    constexpr int STAGES = dense_split_stages<BN>(), kEpiThreads = kDenseThreads - 64;
    constexpr uint32_t kCols = BN < 32 ? 32 : BN;
    extern __shared__ uint8_t smem_raw[];
    // dynamic shared memory starts at the same address in every CTA of a kernel, so `sums` is common to
    // the cluster
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    typedef DenseRing<AMAJ, BMAJ, F16, BN, STAGES> Ring;
    const uint32_t sums = base + (dense_split_overlay<BN>() ? 0u : dense_split_ring<BN>()), bars = base + dense_split_body<BN>();
    const uint32_t full = bars, empty = bars + 8 * STAGES, acc_full = bars + 16 * STAGES, slot = acc_full + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = int(ptx::cluster_ctarank());
    int splits;
    asm volatile("mov.u32 %0, %cluster_nctarank;" : "=r"(splits));
    const int tile = int(blockIdx.x) / splits;
    const int rt = tile / g.col_tiles, ct = tile % g.col_tiles;
    const int k0 = int(int64_t(g.k_steps) * rank / splits), k1 = int(int64_t(g.k_steps) * (rank + 1) / splits);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            ptx::mbar_init(full + 8 * s, 1);
            ptx::mbar_init(empty + 8 * s, 1);
        }
        ptx::mbar_init(acc_full, 1);
        ptx::fence_mbar_init_cluster();
        umma::prefetch_tensormap(&map_a);
        umma::prefetch_tensormap(&map_b);
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
    link_begin(g.link);

    // this CTA's columns and, per thread, (output row, eight output columns) units; what the epilogue
    // reads is fetched kAhead units ahead, for the first ones while the product runs
    const int own = (BN + splits - 1) / splits, c0 = rank * own;
    const int units = max(0, min(own, BN - c0)) * 16;
    const int64_t row0 = int64_t(ct) * BN + c0;
    const int col0 = rt * kDenseTileM, u0 = int(threadIdx.x) - 64;
    constexpr int kAhead = BN >= 64 ? 4 : BN / 16;
    typename Epi::Loads ahead[kAhead];
    if (warp >= 2) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int u = u0 + i * kEpiThreads;
            if (u < units) epi.load(row0 + u / 16, col0 + (u % 16) * 8, ahead[i]);
        }
    }

    bool timed_out = false;
    if (warp == 0) {
        if (lane == 0) {
            Ring ring{base, full, empty};
            timed_out = !ring.load(&map_a, &map_b, rt * kDenseTileM, ct * BN, k0, k1);
            if (timed_out) ring.drain();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            Ring ring{base, full, empty};
            timed_out = !ring.multiply(tmem, k1 - k0);
            if (!timed_out) umma::mma_commit(acc_full);
        }
        __syncwarp();
    } else {
        timed_out = !ptx::mbar_wait_warp<false>(acc_full, 0);
    }
    if (dense_split_overlay<BN>()) ptx::cluster_sync_all();      // every ring of the cluster has been consumed
    if (warp >= 2 && !timed_out) {
        const int q = warp & 3, half = (warp - 2) >> 2, r = q * 32 + lane;
        constexpr int kChunk = BN >= 64 ? 32 : 8;
        umma::fence_after_thread_sync();
#pragma unroll 1
        for (int c = half * (BN / 2); c < (half + 1) * (BN / 2); c += kChunk) {
            uint32_t v[kChunk];
            if constexpr (kChunk == 32) umma::tmem_ld32(tmem + (uint32_t(q * 32) << 16) + c, v);
            else tmem_ld8(tmem + (uint32_t(q * 32) << 16) + c, v);
            umma::tmem_ld_wait();
            int owner = c / own, in = c - owner * own;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                // [source rank][owned column][128 rows] at the owner
                const uint32_t at = ptx::map_to_cta(sums + ((rank * own + in) * 128 + r) * 4, uint32_t(owner));
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v[i]) : "memory");
                if (++in == own) { in = 0; ++owner; }
            }
        }
    }
    umma::fence_before_thread_sync();
    ptx::cluster_sync_all();                 // all partial sums have arrived; nobody writes here any more
    umma::fence_after_thread_sync();
    if (warp >= 2) {
        // not unrolled: the code runs a few times per launch, and fetching it costs more than running it
        // (0.7 us per copy)
#pragma unroll 1
        for (int u = u0; u < units; u += kEpiThreads) {
            const int64_t m = row0 + u / 16;
            const int n = col0 + (u % 16) * 8;
            const typename Epi::Loads mine = ahead[0];
#pragma unroll
            for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
            const int v = u + kAhead * kEpiThreads;
            if (v < units) epi.load(row0 + v / 16, col0 + (v % 16) * 8, ahead[kAhead - 1]);
            if (epi.outside(m, n)) continue;
            float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            uint32_t p = sums + ((u / 16) * 128 + (u % 16) * 8) * 4;
            for (int s = 0; s < splits; ++s, p += uint32_t(own) * 512) {
                const uint4 a = ptx::lds128(p), b = ptx::lds128(p + 16);
                w[0] += __uint_as_float(a.x); w[1] += __uint_as_float(a.y);
                w[2] += __uint_as_float(a.z); w[3] += __uint_as_float(a.w);
                w[4] += __uint_as_float(b.x); w[5] += __uint_as_float(b.y);
                w[6] += __uint_as_float(b.z); w[7] += __uint_as_float(b.w);
            }
            epi(m, n, w, mine);
        }
    } else if (warp == 1) {
        umma::tmem_dealloc(tmem, kCols);     // all tensor-memory loads are behind the barrier
    }
    if (timed_out && status) atomicOr(status, TPPO_DEV_WAIT_TIMEOUT);
    link_end(g.link);
}

// ---- host side ------------------------------------------------------------------------------------
// One operand: a row-major 16-bit matrix [rows, cols] with row stride ld, 16-byte aligned rows.
struct DenseOperand { const void* p; int64_t rows, cols, ld; };

// D[m, n] = sum_k A(m, k) B(k, n).  AMAJ 0: a is [m, k]; 1: a is [k, m].  BMAJ 0: b is [n, k]; 1: b is [k, n].
template <int AMAJ, int BMAJ, bool F16, bool SYM, class Epi>
int dense_gemm(const DenseOperand& a, const DenseOperand& b, int64_t m, int64_t n, int64_t k, const Epi& epi,
               int32_t* status, cudaStream_t s, Link link) {
    CUtensorMap ma, mb;
    if (!make_bf16_tensor_map(&ma, a.p, a.rows, a.cols, a.ld, AMAJ ? 64 : kDenseTileM) ||
        !make_bf16_tensor_map(&mb, b.p, b.rows, b.cols, b.ld, BMAJ ? 64 : kDenseBN))
        return TPPO_ERR_CUDA;
    DenseShape g;
    g.m_tiles = int32_t((m + kDenseTileM - 1) / kDenseTileM);
    g.n_tiles = int32_t((n + kDenseBN - 1) / kDenseBN);
    g.k_steps = int32_t((k + kDenseTileK - 1) / kDenseTileK);
    g.group_m = 16;
    g.link = link;
    const int32_t pairs = g.m_tiles / 2;
    const int64_t total = SYM ? int64_t(pairs) * (pairs + 1) + (g.m_tiles % 2 ? pairs + 1 : 0) : int64_t(g.m_tiles) * g.n_tiles;
    if (total > 0x7fffffff) return TPPO_ERR_UNSUPPORTED;
    g.total = int32_t(total);
    auto kernel = dense_gemm_kernel<AMAJ, BMAJ, F16, SYM, Epi>;
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kDenseSmem)));
    const int grid = g.total < kNumSms ? g.total : kNumSms;
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(grid), dim3(kDenseThreads), kDenseSmem, s, ma, mb, g, epi, status));
    return TPPO_OK;
}

// The same product through dense_split_kernel with the roles of the operands exchanged: the caller
// passes the operand of the output's columns first.  AMAJ 0: a is [n, k]; 1: a is [k, n].
// BMAJ 0: b is [m, k]; 1: b is [k, m].
template <int AMAJ, int BMAJ, bool F16, int BN, class Epi>
int dense_split(const DenseOperand& a, const DenseOperand& b, int64_t m, int64_t n, int64_t k, int splits, const Epi& epi,
                int32_t* status, cudaStream_t s, Link link) {
    CUtensorMap ma, mb;
    if (!make_bf16_tensor_map(&ma, a.p, a.rows, a.cols, a.ld, AMAJ ? 64 : kDenseTileM) ||
        !make_bf16_tensor_map(&mb, b.p, b.rows, b.cols, b.ld, BMAJ ? 64 : BN))
        return TPPO_ERR_CUDA;
    DenseSplitShape g;
    const int64_t row_tiles = (n + kDenseTileM - 1) / kDenseTileM, col_tiles = (m + BN - 1) / BN;
    g.col_tiles = int32_t(col_tiles);
    g.k_steps = int32_t((k + kDenseTileK - 1) / kDenseTileK);
    g.link = link;
    if (row_tiles * col_tiles * splits > 0x7fffffff) return TPPO_ERR_UNSUPPORTED;
    auto kernel = dense_split_kernel<AMAJ, BMAJ, F16, BN, Epi>;
    constexpr size_t smem = dense_split_smem<BN>();
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)));
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(row_tiles * col_tiles * splits));
    cfg.blockDim = dim3(kDenseThreads);
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
    TPPO_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, ma, mb, g, epi, status));
    return TPPO_OK;
}

// How a product is cut: bn 0 = the persistent kernel, else the split kernel's accumulator columns (output
// rows) per tile and the CTAs that share a tile's contraction.  The choice is the least estimated time
// in SM clocks; the constants were fitted to measured launches (16 sizes from 256^3 to 2048 x 5120 x 5120,
// every cut of each; the choice is within a few percent of the best of them but for two at 12 %):
//   start and end of a CTA 5000, of two on one SM 7500; a k step is bound by its operand bytes at 64 per
//   clock or by 2500 clocks of latency over the stages in flight on the SM; sending a column of partial
//   sums 28, finishing one 62; a 128 x 256 tile of the persistent kernel 650 per step and 11500 for the
//   last epilogue, which nothing overlaps.
struct DenseCut { int bn, splits; };
inline DenseCut dense_cut(int64_t m, int64_t n, int64_t k, int64_t big_tiles, int least_bn) {
    // CTAs that fit on the GPU at once in clusters of s, at two and at one per SM (the driver's count)
    static const int64_t pair[9] = {0, 296, 296, 279, 284, 280, 270, 259, 264};
    static const int64_t alone[9] = {0, 148, 148, 135, 132, 130, 132, 105, 120};
    const int64_t rows = (n + 127) / 128, ks = (k + 63) / 64;
    DenseCut best{0, 1};
    int64_t least = 5000 + (big_tiles + kNumSms - 1) / kNumSms * ks * 650 + 11500;
    for (int bn = least_bn; bn <= 256; bn *= 2) {
        const int64_t tiles = rows * ((m + bn - 1) / bn);
        const int64_t stages = bn <= 16 ? 5 : bn <= 32 ? 4 : bn <= 64 ? 3 : bn <= 128 ? 6 : 4;
        for (int s = 1; s <= 8 && (s == 1 || ks >= 2 * s); ++s) {
            const int64_t slots = bn <= 64 ? pair[s] : alone[s];
            const int64_t waves = (tiles * s + slots - 1) / slots, steps = (ks + s - 1) / s;
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

// D[m, n].  P: the operand indexed by m (PMAJ 0: [m, k], 1: [k, m]), Q: the one indexed by n (QMAJ 0:
// [n, k], 1: [k, n]).  SYM: D is symmetric (m = n); the persistent kernel then computes half of it.
template <int PMAJ, int QMAJ, bool F16, bool SYM, class Epi>
int dense_product(const DenseOperand& P, const DenseOperand& Q, int64_t m, int64_t n, int64_t k, const Epi& epi,
                  int32_t* status, cudaStream_t s, Link link = kChain) {
    const int64_t mt = (m + 127) / 128, nt = (n + 255) / 256;
    const int64_t tiles = SYM ? mt / 2 * (mt / 2 + 1) + (mt % 2 ? mt / 2 + 1 : 0) : mt * nt;
    // one operand box of 64 outer indices is the least an MN-major operand can be loaded in
    constexpr int B16 = PMAJ ? 64 : 16, B32 = PMAJ ? 64 : 32;
    const DenseCut c = dense_cut(m, n, k, tiles, B16);
    if (c.bn == 0) return dense_gemm<PMAJ, QMAJ, F16, SYM>(P, Q, m, n, k, epi, status, s, link);
    if (c.bn == 16) return dense_split<QMAJ, PMAJ, F16, B16>(Q, P, m, n, k, c.splits, epi, status, s, link);
    if (c.bn == 32) return dense_split<QMAJ, PMAJ, F16, B32>(Q, P, m, n, k, c.splits, epi, status, s, link);
    if (c.bn == 64) return dense_split<QMAJ, PMAJ, F16, 64>(Q, P, m, n, k, c.splits, epi, status, s, link);
    if (c.bn == 128) return dense_split<QMAJ, PMAJ, F16, 128>(Q, P, m, n, k, c.splits, epi, status, s, link);
    return dense_split<QMAJ, PMAJ, F16, 256>(Q, P, m, n, k, c.splits, epi, status, s, link);
}

}  // namespace tppo
