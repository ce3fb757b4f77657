// The contraction kernel of the floating-point head: D = A B^T on the tcgen05 tensor
// cores with 16-bit operands, 32-bit sums and an epilogue of the caller's.
//
// D[m][n] = sum_k A[m][k] B[n][k].  Each operand is a tensor map of rank 3 over planes of a
// matrix, stored either along K (inner dimension k) or along M / N (inner dimension m or n).
// An operand may be split into a high and a low half (HA, HB = 2 planes a matrix); then
// D = high high + high low + low high, each half loaded once.  The planes of a batch's
// matrices follow one another.  Everything past a matrix's end reads as zero (the maps'
// bounds).
//
// One persistent CTA an SM: warp 0 loads tiles of 64 along K by TMA into a ring of
// shared-memory stages, warp 1 issues the MMAs, warps 4..11 drain the sums from TMEM
// through the epilogue (two warps a TMEM lane quadrant, half the columns each), while
// the MMAs of the next tile fill the other of two accumulators.  CG = 2 pairs two CTAs
// of a cluster on one 256-row tile: each loads its own 128 rows of A and half the
// columns of B, and the MMAs that one thread of the pair issues read both halves.  That
// halves the bytes of B an SM has to load for the same products: loads are what bounds both
// forms (about 53 bytes a clock into an SM, see hg_pick(); a pair's block of 64 along K then
// takes 0.35 us, its MMAs 0.25 at 2.07 GHz).  Measured (2 M N K operations over time): 8192 x
// 64000 x 2048 1.81 PFLOP/s and 16384 x 2048 x 8192 1.83 where the clock holds, 1.6 to 1.75
// under the power limit; the library's bf16 product makes 1.90 and 1.71.
//
// KS > 1 gives a tile's K to a cluster of KS (2, 4 or 8) lone CTAs, where there are few tiles:
// their sums meet in distributed shared memory, a slice of the columns for each CTA (of eight, for
// the first four), are added in the CTAs' order, and taken through the epilogue there.
//
// Every wait is bounded; on expiry the kernel raises TIMEOUT, drains its own copies and
// MMAs in flight (bounded as well), frees TMEM and returns.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstdint>

#include "prof.cuh"
#include "tc_ptx.cuh"

namespace nitro {
namespace {

constexpr int kHgThreads = 384;
constexpr int kHgEpiWarp0 = 4, kHgEpiWarps = 8;
constexpr int kHgBK = 64;                // K elements a stage: rows of 128 bytes
constexpr uint64_t kDrainNs = 50000000ull;

struct HgArgs {
    int M, N;                  // valid rows and columns of D
    int tiles_m, tiles_n, splits, batch, total;
    int kb_total, kb_per_split;   // K blocks of a pass, of a split
    int planes_a, planes_b;    // planes that a matrix of the batch has
    int upper;                 // symmetric D: only tiles that reach the diagonal or lie right of it
    int band;                  // row tiles that are walked together
    int fold;                  // K in two halves, an accumulator each (Epi::kFold only)
    int stage;                 // bytes that a CTA's stage gets
    uint32_t* status;
};

struct HgTile {
    int m, n, split, batch, kb0, kb1;
};

template <int TM, int BN>
__device__ __forceinline__ HgTile hg_decode(const HgArgs& g, int idx) {
    HgTile t;
    const int per = g.total / (g.splits * g.batch);
    const int outer = idx / per;
    idx -= outer * per;
    t.split = outer % g.splits;
    t.batch = outer / g.splits;
    if (g.upper) {
        int m = 0;
        for (; m < g.tiles_m; ++m) {
            const int row = g.tiles_n - m * TM / BN;
            if (idx < row) break;
            idx -= row;
        }
        t.m = m;
        t.n = m * TM / BN + idx;
    } else {
        const int in_band = g.band * g.tiles_n;
        const int b = idx / in_band;
        const int rows = min(g.band, g.tiles_m - b * g.band);
        const int r = idx - b * in_band;
        t.n = r / rows;
        t.m = b * g.band + r - t.n * rows;
    }
    t.kb0 = t.split * g.kb_per_split;
    t.kb1 = min(g.kb_total, t.kb0 + g.kb_per_split);
    return t;
}

template <int CG, int BN, int HA, int HB>
struct HgCfg {
    static constexpr int A_BYTES = 128 * 128;
    static constexpr int B_ROWS = BN / CG;
    static constexpr int B_BYTES = B_ROWS * 128;
    static constexpr int STAGE = HA * A_BYTES + HB * B_BYTES;
    static constexpr int S = 212992 / STAGE < 8 ? 212992 / STAGE : 8;      // 2 to 8
    static constexpr int SMEM = S * STAGE + kHgEpiWarps * 2048 + 1024 + 256;
    static constexpr int TCOLS = 2 * BN;
};

// instruction descriptor of kind::f16 with f32 sums: both operands bf16 or both f16
__host__ __device__ constexpr uint32_t hg_idesc(bool f16, int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | (a_mn ? (1u << 15) : 0u) | (b_mn ? (1u << 16) : 0u) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <int CG>
__device__ __forceinline__ void hg_tma(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2) {
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
            : "memory");
    else
        tma_load_3d(dst, m, bar, c0, c1, c2);
}
template <int CG>
__device__ __forceinline__ void hg_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 2)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        umma_bf16(d, a, b, idesc, accumulate);
}
// arrives at `bar` (of both CTAs of a pair) once the MMAs issued so far are done
template <int CG>
__device__ __forceinline__ void hg_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
    else
        umma_commit(bar);
}
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
// gives up after limit_ns without raising anything
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
    const uint64_t t0 = global_ns();
    while (!mbar_try_wait(bar, parity) && global_ns() - t0 < limit_ns) {
    }
}

// TMEM columns: taken (their address goes to shared memory) and given back by one warp, of
// both CTAs where they work as a pair
template <int CG>
__device__ __forceinline__ void hg_tmem_alloc(uint32_t slot, uint32_t cols) {
    if constexpr (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void hg_tmem_free(uint32_t tmem, uint32_t cols) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}

// TMEM gives a thread a row.  Global memory wants a warp's accesses in few lines: 32 rows of 16
// bytes each are 32 lines an instruction, and cost the epilogues of 128 x 128 tiles 6 us.
// So rows go through 2 KB of the warp's own: 32 rows x 64 bytes, as four 16-byte chunks of the
// thread's row (mine) or spread over the lanes so that eight rows' 64 bytes are one
// instruction (line(i): row 8 i + lane / 4, chunk lane % 4).
struct HgStage {
    uint4* at;
    int lane;
    __device__ __forceinline__ uint4& slot(int row, int j) const { return at[row * 4 + (j ^ ((row >> 1) & 3))]; }
    __device__ __forceinline__ void to_lines(uint4* v) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) slot(lane, j) = v[j];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = slot(8 * i + (lane >> 2), lane & 3);
        __syncwarp();
    }
    __device__ __forceinline__ void to_mine(uint4* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) slot(8 * i + (lane >> 2), lane & 3) = v[i];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = slot(lane, j);
        __syncwarp();
    }
    // rows of unaligned matrices go out value by value, a row an instruction (or two of fp32): put, then value(row, j)
    __device__ __forceinline__ void put(const uint4* v) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) slot(lane, j) = v[j];
        __syncwarp();
    }
    template <typename T>
    __device__ __forceinline__ T value(int row, int j) const {
        constexpr int E = 16 / (int)sizeof(T);
        return reinterpret_cast<const T*>(&slot(row, j / E))[j % E];
    }
    __device__ __forceinline__ int line_row(int i) const { return 8 * i + (lane >> 2); }
    __device__ __forceinline__ int line_chunk() const { return lane & 3; }
};

// A thread's part of a tile: its row, the first row of its warp, its columns (width of them)
// and which part of the tile's columns that is.
struct HgPart {
    int row, row0, rows, col0, width, slot;      // rows: below which rows are valid
    HgStage stage;
};

// 32 rows x 32 16-bit values, a thread's row in w[16], to rows row0.. of a matrix at
// column col; valid rows, columns below `cols` (vec: rows 16-byte aligned).  All lanes.
__device__ __forceinline__ void hg_store16(const HgPart& p, const uint32_t* w, uint16_t* base, int64_t ld, int col, int cols,
                                           bool vec) {
    uint4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    if (!vec) {
        // (eight values a lane at the lines' places are eight stores to 32 sectors each: the gradient of 6008 x 2337 took 76 us, now 33)
        p.stage.put(v);
        const int rows = min(32, p.rows - p.row0);
        if ((((uintptr_t)base | (uintptr_t)(ld * 2) | (uintptr_t)(col * 2)) & 3) == 0) {      // two values a lane, two rows an instruction
            const int j = 2 * (p.stage.lane & 15), c = col + j;
            uint16_t* dst = base + (int64_t)(p.row0 + (p.stage.lane >> 4)) * ld + c;
#pragma unroll 4
            for (int r = p.stage.lane >> 4; r < rows; r += 2, dst += 2 * ld) {
                const uint32_t w = p.stage.value<uint32_t>(r, j >> 1);
                if (c + 2 <= cols) *reinterpret_cast<uint32_t*>(dst) = w;
                else if (c < cols) *dst = (uint16_t)w;
            }
            __syncwarp();
            return;
        }
        const int c = col + p.stage.lane;
        uint16_t* dst = base + (int64_t)p.row0 * ld + c;
#pragma unroll 4
        for (int r = 0; r < rows; ++r, dst += ld)
            if (c < cols) *dst = p.stage.value<uint16_t>(r, p.stage.lane);
        __syncwarp();
        return;
    }
    p.stage.to_lines(v);
    const int c = col + 8 * p.stage.line_chunk(), row = p.row0 + p.stage.line_row(0);
    uint16_t* dst = base + (int64_t)row * ld + c;
    if (p.row0 + 32 <= p.rows && col + 32 <= cols) {       // nearly all
#pragma unroll
        for (int i = 0; i < 4; ++i, dst += 8 * ld) *reinterpret_cast<uint4*>(dst) = v[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i, dst += 8 * ld) {
        if (row + 8 * i >= p.rows || c >= cols) continue;
        if (c + 8 <= cols) {
            *reinterpret_cast<uint4*>(dst) = v[i];
        } else {
            const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < cols) dst[j] = (uint16_t)(u[j >> 1] >> (16 * (j & 1)));
        }
    }
}

// Whether an epilogue takes two planes of B in turns of 16 rows: columns 32 i .. 32 i + 15 of D are then rows
// 16 i .. 16 i + 15 of the first plane, and the 16 columns after them the same rows of the second.
template <class Epi>
constexpr bool hg_pairs = false;

// Epi: struct Args, and per tile and thread
//   Epi(args, g, tile, part)
//   void fetch(c)           starts loading what cols(c) needs (called for c = 0; cols(c)
//                           calls it for the next)
//   void cols(c, v)         v[0..32): columns col0 + c .. col0 + c + 31 of the thread's row; all
//                           lanes call it, rows and columns past the end among them
//   void done()
//   kTail                   whether tail(args, g, shared word) follows, called by every thread once the CTA's
//                           tiles are done
//   kFold                   whether K may go to the two accumulators by halves, to be added here
template <class Epi, int CG, int BN, bool AMN, bool BMN, bool F16, int HA, int HB, int KS>
__global__ void __launch_bounds__(kHgThreads, 1)
    k_head_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const HgArgs g,
                const __grid_constant__ typename Epi::Args ea) {
    using C = HgCfg<CG, BN, HA, HB>;
    constexpr int S = C::S, TM = 128 * CG;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S * C::STAGE + kHgEpiWarps * 2048);
    // bars: full [S], empty [S], tmem full [2], tmem empty [2], drain
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * S + 5);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars);
    const auto full_bar = [&](int s) { return bar0 + 8u * s; };
    const auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
    const auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * S + b); };
    const auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * S + 2 + b); };
    const uint32_t drain_bar = bar0 + 8u * (2 * S + 4);
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    static_assert(KS == 1 || (CG == 1 && BN == 128), "a tile's K is shared out among lone CTAs");
    // a cluster that shares a tile's K: its CTAs are the tile's splits
    const int part = KS > 1 ? (int)cluster_rank() : 0;
    int unit = (int)blockIdx.x / (KS > 1 ? KS : CG);
    if constexpr (KS > 1) {
        const int tiles = g.total / (KS * g.batch);
        unit += (unit / tiles * (KS - 1) + part) * tiles;
    }
    const int units = KS > 1 ? g.total : (int)gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull_bar(b), 1);
            mbar_init(tempty_bar(b), CG * kHgEpiWarps);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) hg_tmem_alloc<CG>(smem_u32(tmem_slot), C::TCOLS);
    if (warp == 0 && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmA)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmB)) : "memory");
    }
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();   // the peer's barriers are set up
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            // ---------------- TMA producer: this CTA's rows of A and its share of B's
            int st = 0, loaded = 0;
            uint32_t ph = 1;
            const uint32_t s0 = smem_u32(smem);
            for (int tile = unit; tile < g.total; tile += units) {
                const HgTile T = hg_decode<TM, BN>(g, tile);
                const int m0 = T.m * TM + rank * 128, n0 = T.n * BN + rank * C::B_ROWS;
                for (int kb = T.kb0; kb < T.kb1; ++kb) {
                    if (!mbar_wait(empty_bar(st), ph, abort_flag, g.status)) goto producer_out;
                    const uint32_t a_dst = s0 + st * C::STAGE, b_dst = a_dst + HA * C::A_BYTES;
                    uint32_t fb = full_bar(st);
                    if (CG == 1 || rank == 0) mbar_expect_tx(fb, CG * g.stage);
                    if constexpr (CG == 2) fb = remote_smem(fb, 0);
#pragma unroll
                    for (int h = 0; h < HA; ++h) {
                        const uint32_t dst = a_dst + h * C::A_BYTES;
                        const int z = T.batch * g.planes_a + h;
                        if constexpr (AMN) {
#pragma unroll
                            for (int j = 0; j < 2; ++j) hg_tma<CG>(dst + j * 8192, &tmA, fb, m0 + 64 * j, kb * kHgBK, z);
                        } else {
                            hg_tma<CG>(dst, &tmA, fb, kb * kHgBK, m0, z);
                        }
                    }
#pragma unroll
                    for (int h = 0; h < HB; ++h) {
                        const uint32_t dst = b_dst + h * C::B_BYTES;
                        const int z = T.batch * g.planes_b + h;
                        if constexpr (BMN) {
#pragma unroll
                            for (int j = 0; j < C::B_ROWS / 64; ++j)
                                hg_tma<CG>(dst + j * 8192, &tmB, fb, n0 + 64 * j, kb * kHgBK, z);
                        } else if constexpr (hg_pairs<Epi>) {
#pragma unroll
                            for (int j = 0; j < C::B_ROWS / 32; ++j)
                                hg_tma<CG>(dst + j * 4096, &tmB, fb, kb * kHgBK, n0 / 2 + 16 * j, 0);
                        } else {
                            hg_tma<CG>(dst, &tmB, fb, kb * kHgBK, n0, z);
                        }
                    }
                    ++loaded;
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
            }
        producer_out:
            // a wait gave up: the copies in flight land before shared memory is given back
            if (*abort_flag) {
                for (int k = max(0, loaded - S); k < loaded; ++k)
                    mbar_drain(full_bar(k % S), (uint32_t)(k / S) & 1u, kDrainNs);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            // ---------------- MMA issuer
            constexpr uint32_t idesc = hg_idesc(F16, TM, BN, AMN, BMN);
            const uint32_t s0 = smem_u32(smem);
            const uint64_t da0 = AMN ? desc_sw128_mn(s0, 8192) : desc_sw128(s0);
            const uint64_t db0 = BMN ? desc_sw128_mn(s0 + HA * C::A_BYTES, 8192) : desc_sw128(s0 + HA * C::A_BYTES);
            // a step of 16 along K: 32 bytes of a row, or 16 rows of 128 bytes
            constexpr uint64_t kStepA = AMN ? 2048 >> 4 : 32 >> 4, kStepB = BMN ? 2048 >> 4 : 32 >> 4;
            int st = 0, it = 0;
            uint32_t ph = 0;
            for (int tile = unit; tile < g.total; tile += units, ++it) {
                const HgTile T = hg_decode<TM, BN>(g, tile);
                const bool fold = Epi::kFold && g.fold;
                int buf = fold ? 0 : it & 1, first = T.kb0;
                const int half_k = fold ? (T.kb0 + T.kb1 + 1) / 2 : T.kb1;
                const uint32_t free_ph = ((uint32_t)(fold ? it : it >> 1) & 1u) ^ 1u;
                if (!mbar_wait(tempty_bar(buf), free_ph, abort_flag, g.status)) break;
                tc_fence_after();
                uint32_t d = tmem + (uint32_t)(buf * BN);
                bool ok = true;
                for (int kb = T.kb0; kb < T.kb1; ++kb) {
                    if (Epi::kFold && kb == half_k) {
                        hg_commit<CG>(tfull_bar(0));
                        buf = 1;
                        first = kb;
                        d = tmem + (uint32_t)BN;
                        if (!(ok = mbar_wait(tempty_bar(1), free_ph, abort_flag, g.status))) break;
                        tc_fence_after();
                    }
                    if (!(ok = mbar_wait(full_bar(st), ph, abort_flag, g.status))) break;
                    tc_fence_after();
                    const uint64_t so = (uint64_t)((uint32_t)(st * C::STAGE) >> 4);
#pragma unroll
                    for (int h = 0; h < HA + HB - 1; ++h) {
                        // high high, high low, low high
                        const uint64_t da = da0 + so + (h >= HB ? C::A_BYTES >> 4 : 0);
                        const uint64_t db = db0 + so + (h > 0 && h < HB ? C::B_BYTES >> 4 : 0);
#pragma unroll
                        for (int k = 0; k < kHgBK / 16; ++k)
                            hg_mma<CG>(d, da + k * kStepA, db + k * kStepB, idesc, kb > first || (h | k) != 0 ? 1u : 0u);
                    }
                    hg_commit<CG>(empty_bar(st));
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
                if (!ok) break;
                hg_commit<CG>(tfull_bar(buf));
            }
            if (*abort_flag) {   // MMAs in flight end before TMEM is freed
                hg_commit<CG>(drain_bar);
                mbar_drain(drain_bar, 0, kDrainNs);
            }
            pdl_trigger();
        }
    } else if (warp >= kHgEpiWarp0) {
        // ---------------- epilogue
        const int q = warp & 3, half = (warp - kHgEpiWarp0) >> 2;
        int it = 0;
        bool alive = true;
        for (int tile = unit; tile < g.total && alive; tile += units, ++it) {
            const HgTile T = hg_decode<TM, BN>(g, tile);
            const int buf = it & 1;
            const int row0 = T.m * TM + rank * 128 + q * 32;
            const HgStage hs{reinterpret_cast<uint4*>(smem + S * C::STAGE) + (warp - kHgEpiWarp0) * 128, lane};
            // The first tile's columns are gone through once before its sums are there, with no valid
            // row: the epilogue's instructions are then cached.  A launch runs each for the first time,
            // and 32 columns took 2.5 to 3.8 us, mostly waiting for them.  For the same reason the
            // columns are a rolled loop.
#pragma unroll 1
            for (int dry = it == 0; dry >= 0; --dry) {
                asm volatile("" : "+r"(dry));
                if constexpr (KS > 1) {
                    constexpr int W = KS > 4 ? 32 : BN / KS;         // columns of a CTA's slice
                    float4* stage = reinterpret_cast<float4*>(smem); // [KS][W / 4][128], where the operands were
                    const HgPart hp{row0 + lane, row0, dry ? 0 : g.M, T.n * BN + part * W + 32 * half, 32, (part * W >> 5) + half, hs};
                    HgTile whole = T;            // what arrives at the epilogue is the sum of all splits
                    whole.split = 0;
                    Epi epi(ea, g, whole, hp);
                    const bool mine = part < BN / W && 32 * half < W;
                    bool ok = true;
                    float v[32] = {};
                    if (!dry) {
                        if (mine) epi.fetch(0);
                        ok = mbar_wait(tfull_bar(buf), 0, abort_flag, g.status);
                        ok = __all_sync(0xffffffffu, ok);
                        tc_fence_after();
                        cluster_barrier();       // every CTA's MMAs have read their operands
                        const uint32_t src = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(half * (BN / 2));
#pragma unroll 1
                        for (int c = 0; c < BN / 2; c += 32) {
                            uint32_t w[32];
                            __syncwarp();
                            tmem_ld32_nowait(src + c, w);
                            tmem_wait_ld<32>(w);
                            const int col = half * (BN / 2) + c;
                            const uint32_t to =
                                remote_smem(smem_u32(stage + (part * (W / 4) + (col % W) / 4) * 128 + q * 32 + lane), col / W);
#pragma unroll
                            for (int j = 0; j < 8; ++j) st_remote4(to + j * 2048, w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                        }
                        cluster_barrier();
                        if (mine) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                float4 s = stage[(8 * half + j) * 128 + q * 32 + lane];
#pragma unroll
                                for (int k = 1; k < KS; ++k) {
                                    const float4 o = stage[(k * (W / 4) + 8 * half + j) * 128 + q * 32 + lane];
                                    s.x += o.x, s.y += o.y, s.z += o.z, s.w += o.w;
                                }
                                v[4 * j] = s.x, v[4 * j + 1] = s.y, v[4 * j + 2] = s.z, v[4 * j + 3] = s.w;
                            }
                        }
                    }
                    if (mine && ok) {
                        epi.cols(0, v);
                        if (!dry) epi.done();
                    }
                } else {
                    const HgPart hp{row0 + lane, row0, dry ? 0 : g.M, T.n * BN + half * (BN / 2), BN / 2, half, hs};
                    Epi epi(ea, g, T, hp);
                    const bool fold = Epi::kFold && g.fold;
                    const int use = fold ? 0 : buf;
                    if (!dry) {
                        epi.fetch(0);
                        const uint32_t full_ph = (uint32_t)(fold ? it : it >> 1) & 1u;
                        bool ok = mbar_wait(tfull_bar(use), full_ph, abort_flag, g.status);
                        if (fold) ok = ok && mbar_wait(tfull_bar(1), full_ph, abort_flag, g.status);
                        if (!(alive = __all_sync(0xffffffffu, ok))) break;
                        tc_fence_after();
                    }
                    const uint32_t src = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(use * BN + half * (BN / 2));
                    const int end = dry ? 32 : BN / 2;
#pragma unroll 1
                    for (int c = 0; c < end; c += 32) {
                        uint32_t v[32];
                        __syncwarp();
                        tmem_ld32_nowait(src + c, v);
                        tmem_wait_ld<32>(v);
                        if constexpr (Epi::kFold) {
                            if (fold) {
                                uint32_t w[32];
                                tmem_ld32_nowait(src + BN + c, w);
                                tmem_wait_ld<32>(w);
#pragma unroll
                                for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(w[j]));
                            }
                        }
                        if (!dry && c + 32 == BN / 2) {
                            // the sums are in registers: the accumulator may be filled again
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) {
                                for (int b = use; b <= (fold ? 1 : use); ++b) {
                                    if constexpr (CG == 2) mbar_arrive_remote(remote_smem(tempty_bar(b), 0));
                                    else mbar_arrive(tempty_bar(b));
                                }
                            }
                        }
                        epi.cols(c, reinterpret_cast<float*>(v));
                    }
                    if (!dry) epi.done();
                }
            }
        }
    }
    if constexpr (KS > 1) {
        if (warp < kHgEpiWarp0) {    // the two of the epilogue's exchange
            __syncwarp();
            cluster_barrier();
            cluster_barrier();
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (Epi::kTail) Epi::tail(ea, g, reinterpret_cast<int*>(tmem_slot + 2));
    if constexpr (CG == 2 || KS > 1) cluster_barrier();   // no copy, MMA or arrival of the pair is outstanding
    if (warp == 2) {
        tc_fence_after();
        hg_tmem_free<CG>(tmem, C::TCOLS);
    }
}

// ------------------------------------------------------------------ host side
// An operand: planes of a matrix with `outer` rows of `inner` 16-bit elements, ld apart.
struct HgOperand {
    const void* base;
    int64_t inner, outer, ld, planes, plane;   // plane: elements from one plane to the next
};

inline bool hg_map(CUtensorMap* m, const HgOperand& o, bool f16, int box_outer, int box_planes = 1) {
    auto fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dim[3] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer, (cuuint64_t)o.planes};
    cuuint64_t stride[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(o.planes > 1 ? o.plane : o.ld * o.outer) * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_outer, (cuuint32_t)box_planes}, step[3] = {1, 1, 1};
    return fn(m, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.base),
              dim, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct HgProblem {
    int64_t M, N, K;
    int batch = 1, planes_a = 1, planes_b = 1;
    bool upper = false, fold = false;
    // few rows of A: a tile's stage gets these (a multiple of 8) and no rows past them, whose sums nobody takes.  128: all
    int rows_a = 128;
    int eights = 0;            // clusters of eight that the caller takes at most (hg_eights()); 0: seven eighths of the SMs' worth
    uint32_t* status = nullptr;
    int prof = 0;
    double ops = 0, bytes = 0;
};

// Splits of K that have work when `want` are asked for.
inline int hg_splits(int64_t K, int want) {
    const int kb = (int)((K + kHgBK - 1) / kHgBK);
    const int per = (kb + want - 1) / want;
    return (kb + per - 1) / per;
}

// How a product runs: CTAs that work on a tile (1 or 2), its columns, and splits of K.
struct HgPick {
    int cg, bn, splits;        // splits: slices of the caller's
    int ks = 1;                // CTAs of a cluster that share a tile's K
};

inline int64_t hg_tiles(const HgProblem& p, int cg, int bn) {
    const int tm = 128 * cg;
    const int64_t rows = (p.M + tm - 1) / tm, cols = (p.N + bn - 1) / bn;
    if (!p.upper) return rows * cols * p.batch;
    int64_t n = 0;
    for (int64_t m = 0; m < rows; ++m) n += cols - m * tm / bn;
    return n * p.batch;
}

// The cheapest in clocks of its busiest SM: rounds of tiles times a tile's K blocks, each of
// which takes as long as its MMAs (2 BN clocks a product of halves) or its loads, about 53
// bytes a clock into an SM's shared memory (a pair's 256 x 256: 32 KB in 600 clocks against
// 512 of MMAs; its 256 x 128: 24 KB in 550 against 256; measured on 8192 x 2048 x 16384).
// Splits into the caller's slices (at most max_splits) or over a cluster pay for their joining.
inline HgPick hg_pick(const HgProblem& p, int ha = 1, int hb = 1, int max_splits = 1) {
    const int sms = sm_count();
    static const struct { int cg, bn; } kForms[] = {{2, 256}, {2, 128}, {1, 256}, {1, 128}};
    HgPick best{2, 256, 1};
    int64_t least = INT64_MAX;
    const int64_t kb = (p.K + kHgBK - 1) / kHgBK;
    for (const auto& f : kForms) {
        const int64_t tiles = hg_tiles(p, f.cg, f.bn), units = sms / f.cg;
        const int64_t mma = 2 * f.bn * (ha + hb - 1), load = (ha * (f.cg == 1 ? p.rows_a : 128) * 128 + hb * (f.bn / f.cg) * 128) / 53 + 30;
        const int64_t clocks = std::max(mma, load);
        const auto cost = [&](int s) {
            // and a tile's way through TMEM, most of it beside the next tile's MMAs; a pair's barriers
            return (tiles * s + units - 1) / units * ((kb + s - 1) / s * clocks + 6 * f.bn) + (f.cg == 2 ? 2500 : 0);
        };
        const auto take = [&](int64_t c, HgPick t) {
            if (c < least) {
                least = c;
                best = t;
            }
        };
        for (int s = 1; s <= max_splits && s <= kb; ++s)
            if (hg_splits(p.K, s) == s)
                take(cost(s) + (s > 1 ? 4000 + (int64_t)s * p.M * p.N * p.batch * 8 / 3500 : 0), {f.cg, f.bn, s});
        for (int s = 2; f.cg == 1 && f.bn == 128 && s <= 8 && (s < 8 || (p.eights ? tiles <= p.eights : 8 * tiles <= sms / 8 * 7)); s *= 2)
            if (hg_splits(p.K, s) == s) take(cost(s) + 6000 + (s == 8 ? 1000 : 0), {1, 128, 1, s});
    }
    return best;
}

template <class Epi, int CG, int BN, bool AMN, bool BMN, bool F16, int HA, int HB, int KS = 1>
cudaError_t hg_launch_as(int splits, const HgProblem& p, const HgOperand& a, const HgOperand& b, const typename Epi::Args& ea,
                         cudaStream_t s) {
    using C = HgCfg<CG, BN, HA, HB>;
    CUtensorMap ma, mb;
    static_assert(!hg_pairs<Epi> || (!BMN && HB == 1), "pairs of planes go along K");
    const int rows_a = CG == 1 && !AMN && p.M <= p.rows_a ? p.rows_a : 128;
    if (!hg_map(&ma, a, F16, AMN ? 64 : rows_a)) return cudaErrorInvalidValue;
    if (!(hg_pairs<Epi> ? hg_map(&mb, b, F16, 16, 2) : hg_map(&mb, b, F16, BMN ? 64 : C::B_ROWS))) return cudaErrorInvalidValue;
    HgArgs g{};
    g.M = (int)p.M;
    g.N = (int)p.N;
    g.tiles_m = (int)((p.M + 128 * CG - 1) / (128 * CG));
    g.tiles_n = (int)((p.N + BN - 1) / BN);
    g.batch = p.batch;
    g.kb_total = (int)((p.K + kHgBK - 1) / kHgBK);
    g.kb_per_split = (g.kb_total + splits - 1) / splits;
    g.splits = (g.kb_total + g.kb_per_split - 1) / g.kb_per_split;
    g.total = (int)hg_tiles(p, CG, BN) * g.splits;
    g.planes_a = p.planes_a;
    g.planes_b = p.planes_b;
    g.upper = p.upper ? 1 : 0;
    g.fold = p.fold && KS == 1 && g.kb_per_split > 1 ? 1 : 0;
    // row tiles whose A stays in L2 while B goes past them once: 40 MB (8192 x 64000 x 2048 in
    // bands of 2048 rows read B, 262 MB, four times: a step 5.55 ms, with these 5.48, under the power limit)
    g.band = (int)std::min<int64_t>(64, std::max<int64_t>(4, ((int64_t)40 << 20) / ((int64_t)128 * CG * HA * 2 * p.K)));
    g.stage = HA * rows_a * 128 + HB * C::B_BYTES;
    g.status = p.status;
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    const int sms = sm_count(&dev);
    const auto kernel = k_head_gemm<Epi, CG, BN, AMN, BMN, F16, HA, HB, KS>;
    const cudaError_t e = once_per_device(ready, dev, [kernel] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    });
    if (e != cudaSuccess) return e;
    const int grid = std::min(g.total, sms / CG) * CG;
    ProfScope ps(p.prof, s, p.ops, p.bytes);
    if constexpr (KS > 1) return launch_cluster(kernel, dim3(g.total), kHgThreads, KS, s, C::SMEM, ma, mb, g, ea);
    else if constexpr (CG == 2) return launch_cluster(kernel, dim3(grid), kHgThreads, 2, s, C::SMEM, ma, mb, g, ea);
    else return launch_k(kernel, dim3(grid), dim3(kHgThreads), C::SMEM, s, ma, mb, g, ea);
}

// Clusters of eight CTAs, one an SM, that surely run at once: half the SMs' worth.  (152 SMs do not hold 16 of them, as their
// parts hold whole clusters only: 64 x 2048 x 1024 took 16.6 us with 16 and 7.4 in clusters of four.  15 run at once, but 10 to 15 tiles
// gain by them along 8192 features only, 15.6 to 13.5 us with 64 rows, and lose along 4096, 10.7 to 11.1, and 2048, 8.2 to 9.7.)
inline int hg_eights() { return std::max(1, sm_count() / 16); }

// D = A B^T through Epi; AMN / BMN: the operand's inner dimension is M / N, else K; HA, HB:
// halves of the operands.
template <class Epi, bool AMN, bool BMN, bool F16, int HA = 1, int HB = 1>
cudaError_t hg_launch(const HgPick& t, const HgProblem& p, const HgOperand& a, const HgOperand& b,
                      const typename Epi::Args& ea, cudaStream_t s) {
    // (a K too short for the cluster goes to lone CTAs)
    if (t.ks == 2 && hg_splits(p.K, 2) == 2) return hg_launch_as<Epi, 1, 128, AMN, BMN, F16, HA, HB, 2>(2, p, a, b, ea, s);
    if (t.ks == 4 && hg_splits(p.K, 4) == 4) return hg_launch_as<Epi, 1, 128, AMN, BMN, F16, HA, HB, 4>(4, p, a, b, ea, s);
    if (t.ks == 8 && hg_splits(p.K, 8) == 8) return hg_launch_as<Epi, 1, 128, AMN, BMN, F16, HA, HB, 8>(8, p, a, b, ea, s);
    if (t.cg == 2 && t.bn == 256) return hg_launch_as<Epi, 2, 256, AMN, BMN, F16, HA, HB>(t.splits, p, a, b, ea, s);
    if (t.cg == 2) return hg_launch_as<Epi, 2, 128, AMN, BMN, F16, HA, HB>(t.splits, p, a, b, ea, s);
    if (t.bn == 256) return hg_launch_as<Epi, 1, 256, AMN, BMN, F16, HA, HB>(t.splits, p, a, b, ea, s);
    return hg_launch_as<Epi, 1, 128, AMN, BMN, F16, HA, HB>(t.splits, p, a, b, ea, s);
}

}  // namespace
}  // namespace nitro
