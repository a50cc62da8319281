// Products of 8-bit matrices with a power-of-two scale per block of 128 elements of the contraction:
//     y[m, n] = sum_b sa(b, m) sb(b, n) sum_{k in block b} a[m, k] b[n, k]
// The tensor cores apply the scales: tcgen05.mma kind::mxf8f6f4 takes, beside its 8-bit operands, an 8-bit exponent per
// operand row and 32 elements, here the same one for the four steps of a block.  Sums therefore stay in tensor memory
// over the whole contraction, in fp32.  (With kind::f8f6f4 every block's sums have to be read, scaled and added in
// registers: 255 instructions per warp and block, and a round trip between two kinds of warps per 512 clocks of
// products: 16384 x 5120 x 5120 took 517 us, with a scale per column of the output 755-800.)
//
// The exponents have to lie in tensor memory: that of operand row r in lane r % 32 of column r / 32, in each of the four
// quarters of 32 lanes; the instruction names the byte of that 32-bit cell which it uses.  Four warps write them there
// from registers (tcgen05.st), four blocks of the contraction at a time, one per byte.  A scale that is not a power of
// two becomes the exponent's NaN, and its outputs 0 with TPPO_DEV_NONFINITE.
//
// The tensor cores drop what lies below the accumulator's last bit at every step of 32: 1.2e-6 of the result (by norms, normal
// inputs) over a contraction of 16384, 3.9e-6 over 40000.  For bf16 outputs it does not show; for fp32 ones the output warps
// take the sums over eight blocks at a time and add them up in registers, on narrower tiles whose sums the registers hold
// (5120 x 5120 of a contraction of 16384: 443 us; with sixteen blocks 414, in one go 374).  What is left is 7e-8 at 4096,
// 1.0e-7 at 16384 and 1.3e-7 at 40000: the S = K / 1024 additions in registers round once each, which grows with the root
// of S.  With the contraction split over CTAs 1.4e-7 at 131072 and 2.5e-7 at a million.
//
//   fp8_gemm_kernel   many output tiles: persistent CTAs, 128 x 240 tiles (208 for fp32): two accumulators, so that the output of
//                     a tile overlaps the products of the next, and two sets of exponents.
//   fp8_split_kernel  few output tiles (one to some hundred tokens): the output is taken TRANSPOSED, the 128 accumulator
//                     rows running along n and the BN columns along m, and the contraction is split over the CTAs of
//                     a cluster, whose partial sums meet in distributed shared memory in a fixed order.
// Every wait is bounded; one that runs out raises TPPO_DEV_WAIT_TIMEOUT, outputs are then incomplete, the copies in
// flight land and tensor memory is released.
#include "dense_common.cuh"
#include "umma.cuh"

namespace tppo {

bool make_u8_tensor_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_rows);

namespace {

constexpr int kF8TileM = 128, kF8Block = 128;             // accumulator rows; elements that share a scale = bytes of a swizzled row
constexpr int kF8Group = 4;                               // blocks whose exponents share a 32-bit cell
constexpr uint32_t kF8ABytes = kF8TileM * kF8Block;

// Instruction descriptor of the block-scaled kind: both operands e4m3 (0) and K-major, N >> 3 in [17,23), exponent-only
// scales in bit 23, M >> 4 in [24,29), the byte of the scale cells in [4,6) for B and [29,31) for A.
__device__ __forceinline__ uint32_t f8_instr_desc(int n, int byte) {
    return (uint32_t(byte) << 4) | (uint32_t(n >> 3) << 17) | (1u << 23) | (uint32_t(kF8TileM >> 4) << 24) | (uint32_t(byte) << 29);
}
// One 128 x N x 32 step, issued by one thread; sfa, sfb: tensor-memory addresses of the operands' scales.
__device__ __forceinline__ void mma_f8(uint32_t tmem_d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                       uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(tmem_d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void f8_tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void f8_tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void f8_tmem_st4(uint32_t taddr, const uint32_t* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void f8_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A barrier of four warps that tells each whether all of them came with `ok`.
__device__ __forceinline__ bool f8_meet(bool ok) {
    uint32_t all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, 1, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(all) : "r"(ok ? 1u : 0u) : "memory");
    return all != 0;
}

// The scales of an operand: of (row, block) at p[block * by_block + (row >> shift) * by_row].
struct F8Scales {
    const float* p;
    int64_t by_block, by_row;
    int32_t shift, rows;
};
// The exponent byte of a scale.
__device__ __forceinline__ uint32_t f8_exponent(float s) {
    const uint32_t b = __float_as_uint(s), e = b >> 23;
    return (b & 0x807fffffu) != 0 || e == 0 || e == 255 ? 0xffu : e;
}
// The rings of a CTA: operand stages in shared memory, and two sets of exponents in tensor memory (columns `sf`, A's
// four followed by B's), each for a group of blocks.
template <int BN, int STAGES>
struct F8Ring {
    static constexpr uint32_t kStage = kF8ABytes + BN * kF8Block;
    static constexpr int kBCols = BN <= 128 ? 4 : 8, kSet = 4 + kBCols;
    static constexpr uint32_t kCells = 2 * kSet * 32 * 4;
    uint32_t base, full, empty, sfull, sempty, sf;
    int stage = 0;
    uint32_t phase = 0, set = 0, sphase = 0;

    __device__ __forceinline__ void next() {
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
    __device__ __forceinline__ void next_set() {
        set ^= 1u;
        if (set == 0) sphase ^= 1u;
    }
    // Loads blocks [k0, k1) of the tile whose first A and B rows are am and bn.
    __device__ __forceinline__ bool load(const CUtensorMap* ma, const CUtensorMap* mb, int am, int bn, int k0, int k1) {
        for (int kb = k0; kb < k1; ++kb) {
            if (!ptx::mbar_wait<false>(empty + 8 * stage, phase ^ 1u)) return false;
            const uint32_t fb = full + 8 * stage, sa = base + stage * kStage;
            ptx::mbar_arrive_expect_tx(fb, kStage);
            umma::tma_load_2d(sa, ma, fb, kb * kF8Block, am);
            umma::tma_load_2d(sa + kF8ABytes, mb, fb, kb * kF8Block, bn);
            next();
        }
        return true;
    }
    // After a wait ran out: let the copies already issued land before the CTA's memory goes away.
    __device__ __forceinline__ void drain() {
        for (int s = 0; s < STAGES; ++s)
            if (!ptx::mbar_wait<false>(full + 8 * s, s < stage ? phase : phase ^ 1u)) return;
    }
    // The exponents of blocks [k0, k1), by four warps.  Each reads the scales of a quarter of the columns, three groups
    // ahead -- under the operands' traffic a load takes some 2000 clocks -- and makes their cells; through shared
    // memory (`cells`: two sets of [kSet][32] words) every warp gets all of them and writes them to the quarter of the lanes
    // that it can reach.  `w`: the warp's number among the four, `quarter`: the address of its lanes.  A warp whose wait ran
    // out still comes to the next meeting, from which all four leave.
    __device__ __forceinline__ bool scales(const F8Scales& a, const F8Scales& b, uint32_t cells, int w, uint32_t quarter, int am, int bn,
                                           int k0, int k1) {
        constexpr int kMine = kSet / 4, kAhead = 3;
        const int lane = threadIdx.x & 31;
        const float* p[kMine];
        int64_t by_block[kMine];
        bool in[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int c = w * kMine + i;
            const bool of_a = c < 4;
            const F8Scales& s = of_a ? a : b;
            const int row = of_a ? am + 32 * c + lane : bn + 32 * (c - 4) + lane;
            in[i] = row < s.rows;            // rows beyond the operand, blocks beyond the contraction: 2^0; their products are 0
            by_block[i] = s.by_block;
            p[i] = s.p + int64_t(row >> s.shift) * s.by_row + k0 * s.by_block;
        }
        float v[kAhead][kMine][kF8Group];
        int next = k0;                       // the first block not yet read
        auto read = [&](float (&to)[kMine][kF8Group]) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
#pragma unroll
                for (int j = 0; j < kF8Group; ++j) to[i][j] = in[i] && next + j < k1 ? p[i][j * by_block[i]] : 1.f;
                p[i] += kF8Group * by_block[i];
            }
            next += kF8Group;
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(v[i]);
        bool ok = true;
        for (int kb = k0; kb < k1; kb += kF8Group) {
            const uint32_t mine = cells + (set * kSet + w * kMine) * 128 + lane * 4;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const uint32_t cell = f8_exponent(v[0][i][0]) | f8_exponent(v[0][i][1]) << 8 | f8_exponent(v[0][i][2]) << 16 |
                                      f8_exponent(v[0][i][3]) << 24;
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(mine + i * 128), "r"(cell) : "memory");
            }
            if (!f8_meet(ok)) return false;
            uint32_t all[kSet];
#pragma unroll
            for (int c = 0; c < kSet; ++c)
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(all[c]) : "r"(cells + (set * kSet + c) * 128 + lane * 4));
            ok = ptx::mbar_wait_warp<false>(sempty + 8 * set, sphase ^ 1u);
            if (!ok) continue;
            umma::fence_after_thread_sync();
#pragma unroll
            for (int c = 0; c < kSet; c += 4) f8_tmem_st4(sf + quarter + set * kSet + c, all + c);
            f8_tmem_st_wait();
            umma::fence_before_thread_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(sfull + 8 * set);
            next_set();
#pragma unroll
            for (int i = 0; i + 1 < kAhead; ++i)
#pragma unroll
                for (int j = 0; j < kMine; ++j)
#pragma unroll
                    for (int l = 0; l < kF8Group; ++l) v[i][j][l] = v[i + 1][j][l];
            read(v[kAhead - 1]);
        }
        return f8_meet(ok);
    }
    // The products of blocks [k0, k1) into accumulator d.
    __device__ __forceinline__ bool multiply(uint32_t d, int k0, int k1) {
        for (int kb = k0; kb < k1; ++kb) {
            const int byte = (kb - k0) % kF8Group;
            if (byte == 0 && !ptx::mbar_wait<false>(sfull + 8 * set, sphase)) return false;
            if (!ptx::mbar_wait<false>(full + 8 * stage, phase)) return false;
            umma::fence_after_thread_sync();
            const uint32_t sa = base + stage * kStage, sfa = sf + set * kSet, idesc = f8_instr_desc(BN, byte);
            const uint64_t ad = umma::smem_desc(sa, 16, 1024), bd = umma::smem_desc(sa + kF8ABytes, 16, 1024);
#pragma unroll
            for (int j = 0; j < kF8Block / 32; ++j)
                mma_f8(d, umma::smem_desc_advance(ad, j * 32), umma::smem_desc_advance(bd, j * 32), idesc, sfa, sfa + 4,
                       kb != k0 || j != 0 ? 1u : 0u);
            umma::mma_commit(empty + 8 * stage);
            next();
            if (byte == kF8Group - 1 || kb + 1 == k1) {
                umma::mma_commit(sempty + 8 * set);
                next_set();
            }
        }
        return true;
    }
};

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
template <class T> __host__ __device__ constexpr int f8_bn() { return sizeof(T) == 4 ? 208 : 240; }
template <class T> __host__ __device__ constexpr int f8_segment() { return sizeof(T) == 4 ? 8 : 1 << 30; }       // blocks summed by the tensor cores
constexpr int kF8Stages = 4;
constexpr int kF8GemmThreads = 448;                       // warps 0-3 exponents, 4-11 output, 12 TMA loads, 13 tcgen05.mma
constexpr int kF8OutWarps = 8;
constexpr uint32_t kF8Staging = 4096;                     // per output warp: 32 rows of 128 bytes
template <class T> __host__ __device__ constexpr size_t f8_smem() {
    return size_t(kF8Stages) * (kF8ABytes + f8_bn<T>() * kF8Block) + kF8OutWarps * kF8Staging + F8Ring<f8_bn<T>(), kF8Stages>::kCells +
           1024 /* alignment */ + 128 /* barriers */;
}

struct F8Shape { int32_t m_tiles, n_tiles, blocks, total, group_m; };

__device__ __forceinline__ void f8_tile(const F8Shape& g, int t, int& mt, int& nt) {
    const int per = g.group_m * g.n_tiles, gi = t / per, first = gi * g.group_m;
    const int gm = min(g.group_m, g.m_tiles - first), in = t - gi * per;
    mt = first + in % gm;
    nt = in / gm;
}

// Where 16-byte piece j of row r of a warp's 32 x 128-byte staging sits.
__device__ __forceinline__ uint32_t f8_piece(int r, int j) { return uint32_t(r * 128 + ((j ^ (r & 7)) << 4)); }

// Sums of a thread's accumulator row over the segments of the contraction: acc += columns [0, COLS) at `taddr`.
template <int COLS>
__device__ __forceinline__ void f8_add(uint32_t taddr, float (&acc)[COLS]) {
    constexpr int kChunk = COLS % 16 == 0 ? 16 : 8;
#pragma unroll
    for (int c = 0; c < COLS; c += kChunk) {
        uint32_t v[kChunk];
        if constexpr (kChunk == 16) f8_tmem_ld16(taddr + c, v);
        else f8_tmem_ld8(taddr + c, v);
        umma::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < kChunk; ++i) acc[c + i] += __uint_as_float(v[i]);
    }
}

// A warp's 32 rows from m0 of output columns [n0, n1): turned through shared memory 128 bytes of each row at a time, so
// that eight lanes store 128 consecutive bytes.  fetch(c, f): this lane's columns n0 + c .. n0 + c + 31.
template <class T, bool UNROLL, int SPAN, class Fetch>
__device__ __forceinline__ void f8_store(const F8Out& o, int64_t m0, int n0, int n1, uint32_t sw, const Fetch& fetch) {
    constexpr int kCols = 128 / int(sizeof(T)), kPer = 16 / int(sizeof(T));
    const int lane = threadIdx.x & 31;
    bool bad = false;
    if (m0 >= o.M) return;
#pragma unroll(UNROLL ? (SPAN + kCols - 1) / kCols : 1)
    for (int c0 = 0; c0 < SPAN; c0 += kCols) {
        const int n = n0 + c0;
        if (n >= n1) break;
        __syncwarp();                        // the last chunk has been read
#pragma unroll
        for (int part = 0; part < kCols / 32; ++part) {
            float f[32];
            fetch(c0 + part * 32, f);
#pragma unroll
            for (int i = 0; i < 32; ++i) {   // what lies beyond the tile is another one's
                bool off = false;
                f[i] = f8_finish<T>(f[i], off);
                bad |= off && n + part * 32 + i < n1 && m0 + lane < o.M;
            }
#pragma unroll
            for (int j = 0; j < 32 / kPer; ++j) {
                uint4 w;
                if constexpr (sizeof(T) == 2)
                    w = make_uint4(pack_bf16x2(f[8 * j], f[8 * j + 1]), pack_bf16x2(f[8 * j + 2], f[8 * j + 3]),
                                   pack_bf16x2(f[8 * j + 4], f[8 * j + 5]), pack_bf16x2(f[8 * j + 6], f[8 * j + 7]));
                else
                    w = make_uint4(__float_as_uint(f[4 * j]), __float_as_uint(f[4 * j + 1]), __float_as_uint(f[4 * j + 2]), __float_as_uint(f[4 * j + 3]));
                ptx::sts128(sw + f8_piece(lane, part * (32 / kPer) + j), w);
            }
        }
        __syncwarp();
        if (o.aligned) {
#pragma unroll
            for (int it = 0; it < 8; ++it) {
                const int r = it * 4 + (lane >> 3), j = lane & 7, col = n + j * kPer;
                if (m0 + r >= o.M || col >= n1) continue;
                const uint4 w = ptx::lds128(sw + f8_piece(r, j));
                T* p = static_cast<T*>(o.y) + (m0 + r) * o.ldy + col;
                if (col + kPer <= n1) {
                    *reinterpret_cast<uint4*>(p) = w;
                } else {
                    const uint32_t part[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        if (col + i >= n1) break;
                        if constexpr (sizeof(T) == 2) p[i] = T(part[i / 2] >> (i % 2 * 16));
                        else p[i] = __uint_as_float(part[i]);
                    }
                }
            }
        } else {
#pragma unroll 4
            for (int i = lane; i < 32 * kCols; i += 32) {                 // 32 consecutive elements at a time
                const int r = i / kCols, c = i % kCols;
                const uint32_t at = sw + f8_piece(r, c / kPer) + (c % kPer) * int(sizeof(T));
                if (m0 + r >= o.M || n + c >= n1) continue;
                T* p = static_cast<T*>(o.y) + (m0 + r) * o.ldy + n + c;
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

template <class T>
__global__ void __launch_bounds__(kF8GemmThreads, 1)
fp8_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const F8Scales sa, const F8Scales sb,
                const F8Shape g, const F8Out out) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    constexpr int kF8BN = f8_bn<T>(), kSegment = f8_segment<T>();
    typedef F8Ring<kF8BN, kF8Stages> Ring;
    static_assert(2 * kF8BN + 2 * Ring::kSet <= 512, "two accumulators and two sets of exponents fit tensor memory");
    const uint32_t staging = base + kF8Stages * Ring::kStage, cells = staging + kF8OutWarps * kF8Staging;
    const uint32_t bars = cells + Ring::kCells;
    const uint32_t full = bars, empty = full + 8 * kF8Stages, sfull = empty + 8 * kF8Stages, sempty = sfull + 16;
    const uint32_t acc_full = sempty + 16, acc_empty = acc_full + 16, slot = acc_empty + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kF8Stages; ++s) {
            ptx::mbar_init(full + 8 * s, 1);
            ptx::mbar_init(empty + 8 * s, 1);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(sfull + 8 * a, 4);
            ptx::mbar_init(sempty + 8 * a, 1);
            ptx::mbar_init(acc_full + 8 * a, 1);
            ptx::mbar_init(acc_empty + 8 * a, kF8OutWarps);
        }
        ptx::fence_mbar_init_cluster();
        umma::prefetch_tensormap(&map_a);
        umma::prefetch_tensormap(&map_b);
    }
    if (warp == 13) {
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
    Ring ring{base, full, empty, sfull, sempty, tmem + 2 * kF8BN};
    if (warp < 4) {
        for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
            int mt, nt;
            f8_tile(g, t, mt, nt);
            timed_out = !ring.scales(sa, sb, cells, warp, uint32_t(warp * 32) << 16, mt * kF8TileM, nt * kF8BN, 0, g.blocks);
        }
    } else if (warp < 12) {
        // two groups of four warps share the columns: 128 and the rest, or halves where the sums are in registers
        constexpr int kSpan = kSegment < (1 << 30) ? kF8BN / 2 : 128;
        const int q = warp & 3, half = (warp - 4) >> 2;
        const uint32_t sw = staging + (warp - 4) * kF8Staging, at = tmem + (uint32_t(q * 32) << 16) + half * kSpan;
        uint32_t n = 0;                      // accumulators so far
        for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
            int mt, nt;
            f8_tile(g, t, mt, nt);
            const int first = nt * kF8BN, n0 = first + half * kSpan;
            const int n1 = min(out.N, half == 0 ? first + kSpan : first + kF8BN);
            const int64_t m0 = int64_t(mt) * kF8TileM + q * 32;
            auto done = [&] {
                umma::fence_before_thread_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * (n & 1));
                ++n;
            };
            if constexpr (kSegment < (1 << 30)) {
                float acc[kSpan];
#pragma unroll
                for (int i = 0; i < kSpan; ++i) acc[i] = 0.f;
                for (int kb = 0; kb < g.blocks; kb += kSegment) {
                    if (!ptx::mbar_wait_warp<false>(acc_full + 8 * (n & 1), (n >> 1) & 1)) { timed_out = true; break; }
                    umma::fence_after_thread_sync();
                    f8_add(at + (n & 1) * kF8BN, acc);
                    done();
                }
                if (!timed_out)
                    f8_store<T, true, kSpan>(out, m0, n0, n1, sw, [&](int c, float (&f)[32]) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) f[i] = c + i < kSpan ? acc[c + i < kSpan ? c + i : 0] : 0.f;
                    });
            } else {
                if (!ptx::mbar_wait_warp<false>(acc_full + 8 * (n & 1), (n >> 1) & 1)) { timed_out = true; break; }
                umma::fence_after_thread_sync();
                f8_store<T, false, kSpan>(out, m0, n0, n1, sw, [&](int c, float (&f)[32]) {
                    uint32_t v[32];
                    umma::tmem_ld32(at + (n & 1) * kF8BN + c, v);
                    umma::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
                });
                done();
            }
        }
    } else if (warp == 12) {
        if (lane == 0) {
            for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
                int mt, nt;
                f8_tile(g, t, mt, nt);
                timed_out = !ring.load(&map_a, &map_b, mt * kF8TileM, nt * kF8BN, 0, g.blocks);
            }
            if (timed_out) ring.drain();
        }
    } else if (lane == 0) {
        uint32_t n = 0;
        for (int t = blockIdx.x; t < g.total && !timed_out; t += gridDim.x) {
            for (int kb = 0; kb < g.blocks; ++n) {
                const int next = g.blocks - kb > kSegment ? kb + kSegment : g.blocks;
                const uint32_t acc = n & 1;
                if (!ptx::mbar_wait<false>(acc_empty + 8 * acc, ((n >> 1) & 1) ^ 1u)) { timed_out = true; break; }
                umma::fence_after_thread_sync();
                if (!ring.multiply(tmem + acc * kF8BN, kb, next)) { timed_out = true; break; }
                umma::mma_commit(acc_full + 8 * acc);
                kb = next;
            }
        }
    }
    if (timed_out && out.status) atomicOr(out.status, TPPO_DEV_WAIT_TIMEOUT);
    umma::fence_before_thread_sync();
    __syncthreads();
    if (warp == 13) {
        __syncwarp();
        umma::tmem_dealloc(tmem, 512);
    }
}

// ---- few tiles --------------------------------------------------------------------------------------------------
// Accumulator rows: output columns n; accumulator columns: output rows m.  Each of the cluster's CTAs owns ceil(BN /
// CTAs) accumulator columns: every CTA stores its partial sums into the owner's shared memory, and after one cluster
// barrier the owner adds them in rank order.  Up to 64 columns the sums have memory of their own and two CTAs share an
// SM; 128 columns lay them over the operand ring, which needs one more barrier.
// Warps: 0 TMA loads, 1 tcgen05.mma, 2-9 output, 10-13 exponents.
constexpr int kF8SplitThreads = 448;
template <int BN> __host__ __device__ constexpr bool f8_overlay() { return BN >= 128; }
template <int BN> __host__ __device__ constexpr int f8_stages() { return BN <= 16 ? 5 : BN <= 32 ? 4 : BN <= 64 ? 3 : 6; }
template <int BN> __host__ __device__ constexpr uint32_t f8_ring() { return uint32_t(f8_stages<BN>()) * (kF8ABytes + BN * kF8Block); }
template <int BN> __host__ __device__ constexpr uint32_t f8_body() { return f8_ring<BN>() + (f8_overlay<BN>() ? 0u : (BN + 8) * 128 * 4); }
template <int BN> __host__ __device__ constexpr size_t f8_split_smem() { return f8_body<BN>() + F8Ring<BN, f8_stages<BN>()>::kCells + 1024 /* alignment */ + 192 /* barriers */; }

struct F8SplitShape { int32_t col_tiles, blocks; };

template <class T, int BN>
__global__ void __launch_bounds__(kF8SplitThreads, BN <= 64 ? 2 : 1)
fp8_split_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const F8Scales sa, const F8Scales sb,
                 const F8SplitShape g, const F8Out out) {
    constexpr int STAGES = f8_stages<BN>(), kEpiThreads = kF8OutWarps * 32, kHalf = BN / 2;
    typedef F8Ring<BN, STAGES> Ring;
    constexpr int kSegment = f8_segment<T>(), kAccs = kSegment < (1 << 30) ? 2 : 1;
    constexpr uint32_t kUsed = kAccs * BN + 2 * Ring::kSet, kCols = kUsed <= 32 ? 32 : kUsed <= 64 ? 64 : kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
    extern __shared__ uint8_t smem_raw[];
    // dynamic shared memory starts at the same address in every CTA of a kernel, so `sums` is common to the cluster
    const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
    const uint32_t sums = base + (f8_overlay<BN>() ? 0u : f8_ring<BN>()), cells = base + f8_body<BN>();
    const uint32_t bars = cells + Ring::kCells, full = bars, empty = full + 8 * STAGES, sfull = empty + 8 * STAGES, sempty = sfull + 16, acc_full = sempty + 16;
    const uint32_t acc_empty = acc_full + 16, slot = acc_empty + 16;
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
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(sfull + 8 * a, 4);
            ptx::mbar_init(sempty + 8 * a, 1);
            ptx::mbar_init(acc_full + 8 * a, 1);
            ptx::mbar_init(acc_empty + 8 * a, 8);
        }
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
    pdl_launch();
    pdl_wait();

    bool timed_out = false;
    Ring ring{base, full, empty, sfull, sempty, tmem + kAccs * BN};
    const int q = warp & 3, half = (warp - 2) >> 2;
    float acc[kAccs == 2 ? kHalf : 1];       // sums over the segments of the contraction
#pragma unroll
    for (int i = 0; i < (kAccs == 2 ? kHalf : 1); ++i) acc[i] = 0.f;
    if (warp == 0) {
        if (lane == 0) {
            timed_out = !ring.load(&map_a, &map_b, rt * kF8TileM, ct * BN, k0, k1);
            if (timed_out) ring.drain();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t n = 0;
            for (int kb = k0; kb < k1 && !timed_out; ++n) {
                const int next = k1 - kb > kSegment ? kb + kSegment : k1;
                timed_out = !ptx::mbar_wait<false>(acc_empty + 8 * (n & 1), ((n >> 1) & 1) ^ 1u);
                umma::fence_after_thread_sync();
                if (!timed_out) timed_out = !ring.multiply(tmem + (n & 1) * BN, kb, next);
                if (!timed_out) umma::mma_commit(acc_full + 8 * (n & 1));
                kb = next;
            }
        }
        __syncwarp();
    } else if (warp < 10) {
        uint32_t n = 0;
        if constexpr (kAccs == 2) {
            for (int kb = k0; kb < k1 && !timed_out; kb += kSegment, ++n) {
                timed_out = !ptx::mbar_wait_warp<false>(acc_full + 8 * (n & 1), (n >> 1) & 1);
                if (timed_out) break;
                umma::fence_after_thread_sync();
                f8_add(tmem + (uint32_t(q * 32) << 16) + (n & 1) * BN + half * kHalf, acc);
                umma::fence_before_thread_sync();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * (n & 1));
            }
        } else {
            timed_out = !ptx::mbar_wait_warp<false>(acc_full, 0);
        }
    } else {
        timed_out = !ring.scales(sa, sb, cells, warp - 10, uint32_t(q * 32) << 16, rt * kF8TileM, ct * BN, k0, k1);
    }
    if (f8_overlay<BN>()) ptx::cluster_sync_all();       // every ring of the cluster has been consumed
    const int own = (BN + splits - 1) / splits, c0 = rank * own;
    if (warp >= 2 && warp < 10 && !timed_out) {
        const int r = q * 32 + lane;
        int owner = half * kHalf / own, in = half * kHalf - owner * own;
        auto send = [&](uint32_t v) {        // [source rank][owned column][128 rows] at the owner
            const uint32_t at = ptx::map_to_cta(sums + ((rank * own + in) * 128 + r) * 4, uint32_t(owner));
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
            if (++in == own) { in = 0; ++owner; }
        };
        if constexpr (kAccs == 2) {
#pragma unroll
            for (int i = 0; i < kHalf; ++i) send(__float_as_uint(acc[i]));
        } else {
            constexpr int kChunk = BN >= 64 ? 32 : 8;
            umma::fence_after_thread_sync();
#pragma unroll 1
            for (int c = half * kHalf; c < (half + 1) * kHalf; c += kChunk) {
                uint32_t v[kChunk];
                if constexpr (kChunk == 32) umma::tmem_ld32(tmem + (uint32_t(q * 32) << 16) + c, v);
                else f8_tmem_ld8(tmem + (uint32_t(q * 32) << 16) + c, v);
                umma::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < kChunk; ++i) send(v[i]);
            }
        }
    }
    umma::fence_before_thread_sync();
    ptx::cluster_sync_all();                 // all partial sums have arrived; nobody writes here any more
    umma::fence_after_thread_sync();
    if (warp >= 2 && warp < 10) {
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
            for (int i = 0; i < 8; ++i) {
                bool off = false;
                w[i] = f8_finish<T>(w[i], off);
                bad |= off && n + i < out.N;
            }
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
struct F8Operand { const void* p; int64_t rows, ld; F8Scales s; };

// How a product is cut: bn 0 = the persistent kernel, else the split kernel's columns (output rows) per tile and the
// CTAs that share a tile's contraction: the least estimated time in SM clocks.  A block of 128 bytes moves as many
// operand bytes as a step of the 16-bit products, whose fitted constants serve here; the persistent kernel takes some
// 600 per block and 6000 at the ends, 18000 where its last output rows leave one element at a time.  Of 20 sizes from
// 1 x 1024 x 1024 to 2048 x 5120 x 5120, timed with every cut, the choice is the best or within 5 % of it but for 515 x
// 777 x 1001 (8.7 us; 7.2 with 32 columns and two CTAs).
struct F8Cut { int bn, splits; };
F8Cut f8_cut(int64_t m, int64_t n, int64_t blocks, int big_n, bool whole_rows) {
    // CTAs that fit on the GPU at once in clusters of s, at two and at one per SM (the driver's count)
    static const int64_t pair[9] = {0, 296, 296, 279, 284, 280, 270, 259, 264};
    static const int64_t alone[9] = {0, 148, 148, 135, 132, 130, 132, 105, 120};
    const int64_t rows = (n + 127) / 128, big = (m + 127) / 128 * ((n + big_n - 1) / big_n);
    F8Cut best{0, 1};
    int64_t least = 5000 + (big + kNumSms - 1) / kNumSms * blocks * (big_n * 5 / 2) + (whole_rows ? 6000 : 18000);
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

template <class T>
int f8_gemm(const F8Operand& a, const F8Operand& b, int64_t K, int64_t blocks, const F8Out& out, cudaStream_t s) {
    CUtensorMap ma, mb;
    if (!make_u8_tensor_map(&ma, a.p, a.rows, K, a.ld, kF8TileM) || !make_u8_tensor_map(&mb, b.p, b.rows, K, b.ld, f8_bn<T>())) return TPPO_ERR_CUDA;
    F8Shape g;
    g.m_tiles = int32_t((a.rows + kF8TileM - 1) / kF8TileM);
    g.n_tiles = int32_t((b.rows + f8_bn<T>() - 1) / f8_bn<T>());
    g.blocks = int32_t(blocks);
    g.group_m = 16;
    const int64_t total = int64_t(g.m_tiles) * g.n_tiles;
    if (total > 0x7fffffff - kNumSms) return TPPO_ERR_UNSUPPORTED;
    g.total = int32_t(total);
    auto kernel = fp8_gemm_kernel<T>;
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(f8_smem<T>())));
    const int grid = g.total < kNumSms ? g.total : kNumSms;
    TPPO_CUDA_CHECK(launch_dense(kernel, dim3(grid), dim3(kF8GemmThreads), f8_smem<T>(), s, ma, mb, a.s, b.s, g, out));
    return TPPO_OK;
}

template <class T, int BN>
int f8_split(const F8Operand& a, const F8Operand& b, int64_t K, int64_t blocks, int splits, const F8Out& out, cudaStream_t s) {
    CUtensorMap ma, mb;
    if (!make_u8_tensor_map(&ma, a.p, a.rows, K, a.ld, kF8TileM) || !make_u8_tensor_map(&mb, b.p, b.rows, K, b.ld, BN)) return TPPO_ERR_CUDA;
    F8SplitShape g;
    const int64_t row_tiles = (a.rows + kF8TileM - 1) / kF8TileM, col_tiles = (b.rows + BN - 1) / BN;
    if (row_tiles * col_tiles * splits > 0x7fffffff) return TPPO_ERR_UNSUPPORTED;
    g.col_tiles = int32_t(col_tiles);
    g.blocks = int32_t(blocks);
    auto kernel = fp8_split_kernel<T, BN>;
    constexpr size_t smem = f8_split_smem<BN>();
    TPPO_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)));
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(row_tiles * col_tiles * splits));
    cfg.blockDim = dim3(kF8SplitThreads);
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
    TPPO_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, ma, mb, a.s, b.s, g, out));
    return TPPO_OK;
}

template <class T>
int f8_product(const F8Operand& a, const F8Operand& b, int64_t K, const F8Out& out, cudaStream_t s) {
    const int64_t blocks = (K + kF8Block - 1) / kF8Block;
    const F8Cut c = f8_cut(a.rows, b.rows, blocks, f8_bn<T>(), out.aligned != 0);
    switch (c.bn) {                          // the split kernel's rows are the output's columns
        case 16: return f8_split<T, 16>(b, a, K, blocks, c.splits, out, s);
        case 32: return f8_split<T, 32>(b, a, K, blocks, c.splits, out, s);
        case 64: return f8_split<T, 64>(b, a, K, blocks, c.splits, out, s);
        case 128: return f8_split<T, 128>(b, a, K, blocks, c.splits, out, s);
        default: return f8_gemm<T>(a, b, K, blocks, out, s);
    }
}

F8Scales scales_of(const float* p, int64_t ld, int64_t rows, bool by_rows) {
    return by_rows ? F8Scales{p, ld, 1, 0, int32_t(rows)} : F8Scales{p, 1, ld, 7, int32_t(rows)};
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
    if (!a || !a_scale || !b || !b_scale || !aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4))
        return TPPO_ERR_INVALID_ARG;
    // a matrix of one row needs no stride
    if (lda < K || ldb < K || (M > 1 && lda % 16) || (N > 1 && ldb % 16) || ldas < M || ldbs < (rows ? N : kb))
        return TPPO_ERR_INVALID_ARG;
    const F8Operand oa{a, M, whole(lda, 16), scales_of(a_scale, ldas, M, true)};
    const F8Operand ob{b, N, whole(ldb, 16), scales_of(b_scale, ldbs, N, rows)};
    const F8Out out{y, ldy, M, int32_t(N), status, rows_aligned(y, ldy, e)};
    return y_dtype == TPPO_F32 ? f8_product<float>(oa, ob, K, out, s) : f8_product<bf16_bits>(oa, ob, K, out, s);
}

TPPO_API int32_t tppo_test_fp8_cut(int64_t M, int64_t N, int64_t K, int32_t y_dtype, int32_t aligned_rows) {
    using namespace tppo;
    if (M < 1 || N < 1 || K < 1 || M > kDenseMaxSize || N > kDenseMaxSize || K > kDenseMaxSize) return -1;
    const F8Cut c = f8_cut(M, N, (K + kF8Block - 1) / kF8Block, y_dtype == TPPO_F32 ? f8_bn<float>() : f8_bn<bf16_bits>(), aligned_rows != 0);
    return c.bn * 16 + c.splits;
}
