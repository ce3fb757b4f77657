// Microscaled 4-bit floating point (OCP MX: e2m1 values, a power of two per 32 of them):
// quantisation, its inverse, and the product y = Q(x) W^T with 4-bit weights.
//
// A block's scale is 2^(floor(log2 max|v|) - 2), kept as that exponent + 127; a value
// goes to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times the scale, ties to the even
// code, 6 at most.  All of it is exact in 32 bits, so there is one right result.
//
// Layout.  Codes: [rows][blocks][16] bytes, value 2i of a block in the low half of byte i.
// Scales: tiles of 128 rows x 4 blocks, 512 bytes each, ordered [row tile][block tile];
// row r, block j of a tile at (r % 32) 16 + (r / 32) 4 + j.  That is the order in which
// the tensor cores take scales from TMEM, so a tile goes from global memory to shared
// memory by one bulk copy and on to TMEM by one tcgen05.cp.
//
// The product runs on tcgen05.mma kind::mxf4 (products and scales exact, 32-bit sums).
#include <new>
#include <vector>

#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "prof.cuh"
#include "tc_ptx.cuh"

using namespace nitro;

namespace nitro {
namespace {

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t blocks_of(int64_t cols) { return (cols + 31) / 32; }
int64_t code_bytes(int64_t rows, int64_t cols) { return rows * blocks_of(cols) * 16; }
int64_t scale_bytes(int64_t rows, int64_t cols) { return round_up(rows, 128) * round_up(blocks_of(cols), 4); }

// place of the scale of (row, block j); tiles: tiles along the blocks
__device__ __forceinline__ int64_t scale_at(int64_t row, int j, int tiles) {
    return ((row >> 7) * tiles + (j >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (j & 3);
}

template <typename T>
__device__ __forceinline__ float to_float(T v) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)v << 16);
    else return v;
}

// two values -> two e2m1 codes in a byte, b in the high half; nearest, ties to even, at most 6
__device__ __forceinline__ uint32_t e2m1x2(float a, float b) {
    uint32_t r;
    asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n cvt.u32.u8 %0, t;\n}\n" : "=r"(r) : "f"(a), "f"(b));
    return r;
}

// Four threads a block, eight values each.  The grid covers the scales' padding too.
template <typename T>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T* x, int64_t ldx, int rows, int cols, uint8_t* q, uint8_t* sc,
                                                      int blocks, int64_t rows_pad, int vec) {
    pdl_wait();
    const int tiles = (blocks + 3) / 4;
    const int64_t per_row = (int64_t)tiles * 16, n = rows_pad * per_row;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int part = (int)(i - row * per_row), blk = part >> 2, c = part * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        if (row < rows && c < cols) {
            const T* src = x + row * ldx + c;
            if (vec && c + 8 <= cols) {
                if constexpr (sizeof(T) == 2) {
                    const uint4 w = *reinterpret_cast<const uint4*>(src);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[2 * j] = __uint_as_float(u[j] << 16);
                        v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
                    }
                } else {
                    const float4 a = reinterpret_cast<const float4*>(src)[0], b = reinterpret_cast<const float4*>(src)[1];
                    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < cols) v[j] = to_float(src[j]);
            }
        }
        // magnitudes as integers keep their order, and a NaN is the largest
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // exponent + 127 of the scale: that of the largest less 2, at least 0; 255: not finite
        const uint32_t e = top >> 23;
        const uint32_t s = e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
        // 2^(127 - s): 254 - s as an exponent field (s = 254 cannot be)
        const float inv = __uint_as_float((254u - min(s, 253u)) << 23);
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= e2m1x2(v[2 * j] * inv, v[2 * j + 1] * inv) << (8 * j);
        if (row < rows && blk < blocks) *reinterpret_cast<uint32_t*>(q + (row * blocks + blk) * 16 + (part & 3) * 4) = w;
        if ((part & 3) == 0) sc[scale_at(row, blk, tiles)] = row < rows && blk < blocks ? (uint8_t)s : 0;
    }
}

__device__ __forceinline__ float e2m1_value(uint32_t code) {
    // magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6: twice that in half a byte each
    const float m = 0.5f * (float)((0xc8643210u >> (4 * (code & 7))) & 15u);
    return code & 8 ? -m : m;
}
__device__ __forceinline__ float e8m0_value(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_dequantize(const uint8_t* q, const uint8_t* sc, int rows, int cols, int blocks,
                                                        T* out, int64_t ldo, float* scales, int vec) {
    pdl_wait();
    const int tiles = (blocks + 3) / 4;
    const int64_t per_row = (int64_t)blocks * 4, n = rows * per_row;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per_row;
        const int part = (int)(i - row * per_row), blk = part >> 2, c = part * 8;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(q + i * 4);
        const float s = e8m0_value(sc[scale_at(row, blk, tiles)]);
        if (scales && (part & 3) == 0) scales[row * blocks + blk] = s;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = e2m1_value((w >> (4 * j)) & 15u) * s;
        T* dst = out + row * ldo + c;
        if constexpr (sizeof(T) == 2) {
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
                u[j] = *reinterpret_cast<const uint32_t*>(&p);
            }
            if (vec && c + 8 <= cols) *reinterpret_cast<uint4*>(dst) = make_uint4(u[0], u[1], u[2], u[3]);
            else
                for (int j = 0; j < 8; ++j)
                    if (c + j < cols) dst[j] = (uint16_t)(u[j >> 1] >> (16 * (j & 1)));
        } else {
            if (vec && c + 8 <= cols) {
                reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else
                for (int j = 0; j < 8; ++j)
                    if (c + j < cols) dst[j] = v[j];
        }
    }
}

// ------------------------------------------------------------------ product
// D[p][q] = sum_k P[p][k] Q[q][k], 128 rows of P (TMEM lanes) x BN rows of Q (columns) a
// tile.  SWAP: P is W and Q the features, for few samples: a tile then has 128 weights'
// rows and as few columns as there are samples, and the weights stream past once.
constexpr int kMxThreads = 384, kMxEpiWarp0 = 4, kMxEpiWarps = 8;

struct MxArgs {
    int P, Q;                // valid rows
    int tiles_p, tiles_q, splits, total, band;
    int k64;                 // steps of 64 along K
    int stages, stages_per_split;
    const uint8_t *sp, *sq;  // scales
    int tiles_k;             // scale tiles along K
    void* y;                 // output, or slices of 32-bit partial sums
    int64_t ldy, slice;
    int out;                 // 0 bf16, 1 fp32
    int vec;                 // rows of y are 16-byte aligned
    uint32_t* status;
};

template <int BN>
struct MxCfg {
    static constexpr int P_BYTES = 128 * 128, Q_BYTES = BN * 128;
    static constexpr int STAGE = P_BYTES + Q_BYTES + 2048;    // and 1 KB of scales each
    static constexpr int S = BN >= 128 ? 6 : 8;
    static constexpr int SMEM = S * STAGE + 1024 + 256;
    static constexpr int SF = 2 * BN;                          // TMEM columns of the scales: 2 x 16
    static constexpr int TCOLS = 2 * BN + 32 <= 128 ? 128 : 2 * BN + 32 <= 256 ? 256 : 512;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
// 32 rows of 16 bytes (a scale tile) -> four TMEM columns, the same for every lane quadrant
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t saddr) {
    const uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
}
// kind::mxf4, e2m1 operands, e8m0 scales of 32; half: which two of a scale word's four bytes
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                         uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
__host__ __device__ constexpr uint32_t mx_idesc(int n, int half) {
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (8u << 24) |
           ((uint32_t)(2 * half) << 29);
}

struct MxTile {
    int p, q, split, s0, s1;
};
__device__ __forceinline__ MxTile mx_decode(const MxArgs& g, int idx) {
    MxTile t;
    const int per = g.tiles_p * g.tiles_q;
    t.split = idx / per;
    idx -= t.split * per;
    const int in_band = g.band * g.tiles_q, b = idx / in_band, rows = min(g.band, g.tiles_p - b * g.band), r = idx - b * in_band;
    t.q = r / rows;
    t.p = b * g.band + r - t.q * rows;
    t.s0 = t.split * g.stages_per_split;
    t.s1 = min(g.stages, t.s0 + g.stages_per_split);
    return t;
}

template <int BN, bool SWAP>
__global__ void __launch_bounds__(kMxThreads, 1)
    k_mx4_gemm(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ, const MxArgs g) {
    using C = MxCfg<BN>;
    constexpr int S = C::S;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    // stages of operands (1024-byte aligned), then the scales
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S * C::STAGE);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * S + 5);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars), s0 = smem_u32(smem), sf0 = s0 + S * (C::P_BYTES + C::Q_BYTES);
    const auto full_bar = [&](int s) { return bar0 + 8u * s; };
    const auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
    const auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * S + b); };
    const auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * S + 2 + b); };
    const uint32_t drain_bar = bar0 + 8u * (2 * S + 4);
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull_bar(b), 1);
            mbar_init(tempty_bar(b), kMxEpiWarps);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                     "r"(C::TCOLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            int st = 0, loaded = 0;
            uint32_t ph = 1;
            for (int tile = blockIdx.x; tile < g.total; tile += gridDim.x) {
                const MxTile T = mx_decode(g, tile);
                const uint8_t* sp = g.sp + (int64_t)T.p * g.tiles_k * 512;
                const uint8_t* sq = g.sq + (int64_t)(T.q * BN / 128) * g.tiles_k * 512;
                for (int k = T.s0; k < T.s1; ++k) {
                    if (!mbar_wait(empty_bar(st), ph, abort_flag, g.status)) goto producer_out;
                    const uint32_t dp = s0 + st * (C::P_BYTES + C::Q_BYTES), dq = dp + C::P_BYTES, ds = sf0 + st * 2048;
                    const uint32_t fb = full_bar(st);
                    const uint32_t sb = (uint32_t)min(2, g.tiles_k - 2 * k) * 512u;
                    mbar_expect_tx(fb, C::P_BYTES + C::Q_BYTES + 2 * sb);
                    tma_load_2d(dp, &tmP, fb, k * 128, T.p * 128);
                    tma_load_2d(dq, &tmQ, fb, k * 128, T.q * BN);
                    bulk_load(ds, sp + (int64_t)k * 1024, sb, fb);
                    bulk_load(ds + 1024, sq + (int64_t)k * 1024, sb, fb);
                    ++loaded;
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
            }
        producer_out:
            if (*abort_flag) {
                const uint64_t t0 = global_ns();
                for (int k = max(0, loaded - S); k < loaded; ++k)
                    while (!mbar_try_wait(full_bar(k % S), (uint32_t)(k / S) & 1u) && global_ns() - t0 < 50000000ull) {
                    }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint64_t dp0 = desc_sw128(s0), dq0 = desc_sw128(s0 + C::P_BYTES);
            int st = 0, it = 0, n = 0;
            uint32_t ph = 0;
            for (int tile = blockIdx.x; tile < g.total; tile += gridDim.x, ++it) {
                const MxTile T = mx_decode(g, tile);
                const int buf = it & 1;
                if (!mbar_wait(tempty_bar(buf), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, g.status)) break;
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * BN);
                bool ok = true;
                for (int k = T.s0; k < T.s1; ++k, ++n) {
                    if (!(ok = mbar_wait(full_bar(st), ph, abort_flag, g.status))) break;
                    tc_fence_after();
                    const int steps = min(4, g.k64 - 4 * k);
                    const uint32_t sf = tmem + C::SF + 16u * (n & 1), ds = sf0 + st * 2048;
                    copy_scales(sf, ds);
                    copy_scales(sf + 8, ds + 1024);
                    if (steps > 2) {
                        copy_scales(sf + 4, ds + 512);
                        copy_scales(sf + 12, ds + 1536);
                    }
                    const uint64_t so = (uint64_t)((uint32_t)(st * (C::P_BYTES + C::Q_BYTES)) >> 4);
                    // where the columns' tile starts inside a scale tile of 128 rows: 32 rows a TMEM column
                    const uint32_t q32 = BN < 128 ? (uint32_t)((T.q * BN) & 127) >> 5 : 0u;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps)
                            mma_mxf4(d, dp0 + so + 2 * j, dq0 + so + 2 * j, mx_idesc(BN, j & 1), sf + 4u * (j >> 1),
                                     sf + 8 + 4u * (j >> 1) + q32, (k > T.s0 || j > 0) ? 1u : 0u);
                    umma_commit(empty_bar(st));
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
                if (!ok) break;
                umma_commit(tfull_bar(buf));
            }
            if (*abort_flag) {
                umma_commit(drain_bar);
                const uint64_t t0 = global_ns();
                while (!mbar_try_wait(drain_bar, 0) && global_ns() - t0 < 50000000ull) {
                }
            }
            pdl_trigger();
        }
    } else if (warp >= kMxEpiWarp0) {
        const int q = warp & 3, half = (warp - kMxEpiWarp0) >> 2;
        int it = 0;
        for (int tile = blockIdx.x; tile < g.total; tile += gridDim.x, ++it) {
            const MxTile T = mx_decode(g, tile);
            const int buf = it & 1;
            const bool ok = mbar_wait(tfull_bar(buf), (uint32_t)(it >> 1) & 1u, abort_flag, g.status);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const int row = T.p * 128 + q * 32 + lane, col0 = T.q * BN + half * (BN / 2);
            const uint32_t src = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * BN + half * (BN / 2));
            float* yf = static_cast<float*>(g.y) + T.split * g.slice;
            uint16_t* yb = static_cast<uint16_t*>(g.y);
#pragma unroll
            for (int c = 0; c < BN / 2; c += 16) {
                uint32_t v[16];
                tmem_ld16_nowait(src + c, v);
                tmem_wait_ld<16>(v);
                if (c + 16 == BN / 2) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty_bar(buf));
                }
                const int n = g.Q - (col0 + c);
                if (row >= g.P || n <= 0) continue;
                const float* f = reinterpret_cast<const float*>(v);
                if constexpr (SWAP) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (j >= n) continue;
                        const int64_t at = (int64_t)(col0 + c + j) * g.ldy + row;
                        if (g.out) yf[at] = f[j];
                        else yb[at] = __bfloat16_as_ushort(__float2bfloat16_rn(f[j]));
                    }
                } else {
                    const int64_t at = (int64_t)row * g.ldy + col0 + c;
                    if (g.out) {
                        if (g.vec && n >= 16) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                reinterpret_cast<float4*>(yf + at)[j] = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                if (j < n) yf[at + j] = f[j];
                        }
                    } else {
                        uint32_t w[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
                            w[j] = *reinterpret_cast<const uint32_t*>(&p);
                        }
                        if (g.vec && n >= 16) {
                            reinterpret_cast<uint4*>(yb + at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                            reinterpret_cast<uint4*>(yb + at)[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                if (j < n) yb[at + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
                        }
                    }
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::TCOLS) : "memory");
    }
}

// y from the slices of its 32-bit partial sums, in their order.
__global__ void __launch_bounds__(256) k_mx4_join(const float* part, int slices, int64_t slice, int64_t ldp, int rows, int cols,
                                                  void* y, int64_t ldy, int out) {
    pdl_wait();
    const int64_t n = (int64_t)rows * cols;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols, c = i - r * cols;
        float v = 0.0f;
        for (int k = 0; k < slices; ++k) v += part[k * slice + r * ldp + c];
        if (out) static_cast<float*>(y)[r * ldy + c] = v;
        else static_cast<uint16_t*>(y)[r * ldy + c] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
    }
}

// ------------------------------------------------------------------ host side
bool mx_map(CUtensorMap* m, const uint8_t* codes, int64_t rows, int64_t pitch, int box_rows) {
    auto fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dim[2] = {(cuuint64_t)pitch, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)pitch};
    cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(codes), dim, stride, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool SWAP>
cudaError_t mx_launch(const uint8_t* p, int64_t np, const uint8_t* q, int64_t nq, int64_t pitch, MxArgs g, double ops,
                      double bytes, cudaStream_t s) {
    using C = MxCfg<BN>;
    CUtensorMap mp, mq;
    if (!mx_map(&mp, p, np, pitch, 128) || !mx_map(&mq, q, nq, pitch, BN)) return cudaErrorInvalidValue;
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    const int sms = sm_count(&dev);
    const cudaError_t e = once_per_device(ready, dev, [] {
        return cudaFuncSetAttribute(k_mx4_gemm<BN, SWAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    });
    if (e != cudaSuccess) return e;
    ProfScope ps(K_MX4_LINEAR, s, ops, bytes);
    return launch_k(k_mx4_gemm<BN, SWAP>, dim3(std::min(g.total, sms)), dim3(kMxThreads), C::SMEM, s, mp, mq, g);
}

template <typename T>
cudaError_t quantize(const T* x, int64_t ldx, int rows, int cols, uint8_t* q, uint8_t* sc, cudaStream_t s) {
    const int blocks = (int)blocks_of(cols);
    const int64_t pad = round_up(rows, 128), n = pad * ((blocks + 3) / 4) * 16;
    const int grid = (int)std::min<int64_t>((n + 255) / 256, (int64_t)sm_count() * 16);
    const int vec = ((uintptr_t)x & 15) == 0 && ldx * (int64_t)sizeof(T) % 16 == 0;
    ProfScope ps(K_MX4_QUANTIZE, s, 0.0, (double)rows * cols * (sizeof(T) + 17.0 / 32.0));
    return launch_k(k_mx4_quantize<T>, dim3(grid), dim3(256), 0, s, x, ldx, rows, cols, q, sc, blocks, pad, vec);
}

bool mx4_shape(int rows, int cols) { return rows >= 0 && cols >= 1 && rows <= (1 << 24) && cols <= (1 << 24); }

bool mx4_source(const void* x, int type, int64_t ldx, int rows, int cols) {
    if ((type != NITRO_BF16 && type != NITRO_F32) || ldx < cols) return false;
    return rows == 0 || (x && ((uintptr_t)x & (type == NITRO_F32 ? 3 : 1)) == 0);
}

constexpr int64_t kPartFloats = (int64_t)8 << 20;     // slices of partial sums: at most 32 MB

}  // namespace
}  // namespace nitro

struct nitro_mx4 {
    int max_rows = 0, in = 0, out = 0;
    uint8_t *xq = nullptr, *xs = nullptr;
    float* part = nullptr;
    uint32_t* status = nullptr;
    std::vector<void*> allocs;
};

#define TRY(expr)                                         \
    do {                                                  \
        if ((expr) != cudaSuccess) return NITRO_ERR_CUDA; \
    } while (0)

extern "C" {

nitro_status nitro_mx4_bytes(int rows, int cols, size_t* codes, size_t* scales) {
    if (!codes || !scales || !mx4_shape(rows, cols)) return NITRO_ERR_ARG;
    *codes = (size_t)code_bytes(rows, cols);
    *scales = (size_t)scale_bytes(rows, cols);
    return NITRO_OK;
}

nitro_status nitro_mx4_quantize(const void* x, int type, int64_t ldx, int rows, int cols, uint8_t* codes, uint8_t* scales,
                                void* stream) {
    if (!mx4_shape(rows, cols) || !mx4_source(x, type, ldx, rows, cols)) return NITRO_ERR_ARG;
    if (rows == 0) return NITRO_OK;
    if (!codes || !scales || ((uintptr_t)codes & 15) || ((uintptr_t)scales & 15)) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (type == NITRO_BF16) TRY(quantize((const uint16_t*)x, ldx, rows, cols, codes, scales, s));
    else TRY(quantize((const float*)x, ldx, rows, cols, codes, scales, s));
    return NITRO_OK;
}

nitro_status nitro_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int cols, void* out, int type,
                                  int64_t ldo, float* scale_values, void* stream) {
    if (!mx4_shape(rows, cols) || !mx4_source(out, type, ldo, rows, cols)) return NITRO_ERR_ARG;
    if (rows == 0) return NITRO_OK;
    if (!codes || !scales || ((uintptr_t)codes & 15) || ((uintptr_t)scales & 15) || ((uintptr_t)scale_values & 3))
        return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int blocks = (int)blocks_of(cols);
    const int64_t n = (int64_t)rows * blocks * 4;
    const int grid = (int)std::min<int64_t>((n + 255) / 256, (int64_t)sm_count() * 16);
    const int size = type == NITRO_BF16 ? 2 : 4;
    const int vec = ((uintptr_t)out & 15) == 0 && ldo * size % 16 == 0;
    ProfScope ps(K_MX4_DEQUANTIZE, s, 0.0, (double)rows * cols * (size + 17.0 / 32.0));
    if (type == NITRO_BF16)
        TRY(launch_k(k_mx4_dequantize<uint16_t>, dim3(grid), dim3(256), 0, s, codes, scales, rows, cols, blocks,
                     (uint16_t*)out, ldo, scale_values, vec));
    else
        TRY(launch_k(k_mx4_dequantize<float>, dim3(grid), dim3(256), 0, s, codes, scales, rows, cols, blocks, (float*)out, ldo,
                     scale_values, vec));
    return NITRO_OK;
}

nitro_status nitro_mx4_create(int max_rows, int in, int out_features, nitro_mx4** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (max_rows < 1 || max_rows > (1 << 20) || in < 1 || in > (1 << 20) || out_features < 1 || out_features > (1 << 24) ||
        (int64_t)max_rows * in > ((int64_t)1 << 36))
        return NITRO_ERR_ARG;
    nitro_mx4* h = new (std::nothrow) nitro_mx4();
    if (!h) return NITRO_ERR_CUDA;
    h->max_rows = max_rows;
    h->in = in;
    h->out = out_features;
    const auto alloc = [h](auto** p, int64_t bytes) {
        void* q = nullptr;
        if (cudaMalloc(&q, (size_t)bytes) != cudaSuccess) return false;
        h->allocs.push_back(q);
        *p = static_cast<std::remove_reference_t<decltype(*p)>>(q);
        return true;
    };
    const bool ok = alloc(&h->xq, code_bytes(max_rows, in)) && alloc(&h->xs, scale_bytes(max_rows, in)) &&
                    alloc(&h->part, kPartFloats * 4) && alloc(&h->status, 4) && cudaMemset(h->status, 0, 4) == cudaSuccess;
    if (!ok) {
        nitro_mx4_destroy(h);
        return NITRO_ERR_CUDA;
    }
    *out = h;
    return NITRO_OK;
}

nitro_status nitro_mx4_linear(nitro_mx4* h, const void* x, int x_type, int64_t ldx, int rows, const uint8_t* w_codes,
                              const uint8_t* w_scales, void* y, int y_type, int64_t ldy, void* stream) {
    if (!h || rows < 0 || rows > h->max_rows || !mx4_source(x, x_type, ldx, rows, h->in) ||
        !mx4_source(y, y_type, ldy, rows, h->out))
        return NITRO_ERR_ARG;
    if (rows == 0) return NITRO_OK;
    if (!w_codes || !w_scales || ((uintptr_t)w_codes & 15) || ((uintptr_t)w_scales & 15)) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (x_type == NITRO_BF16) TRY(quantize((const uint16_t*)x, ldx, rows, h->in, h->xq, h->xs, s));
    else TRY(quantize((const float*)x, ldx, rows, h->in, h->xq, h->xs, s));
    const int64_t pitch = blocks_of(h->in) * 16;
    const bool swap = rows <= 64;
    const int bn = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    const int sms = sm_count();
    MxArgs g{};
    g.P = swap ? h->out : rows;
    g.Q = swap ? rows : h->out;
    g.tiles_p = (g.P + 127) / 128;
    g.tiles_q = (g.Q + bn - 1) / bn;
    g.band = 16;
    g.k64 = (h->in + 63) / 64;
    g.stages = (g.k64 + 3) / 4;
    g.tiles_k = (int)((blocks_of(h->in) + 3) / 4);
    g.sp = swap ? w_scales : h->xs;
    g.sq = swap ? h->xs : w_scales;
    g.status = h->status;
    // K is shared out where that shortens the longest CTA's work
    const int64_t tiles = (int64_t)g.tiles_p * g.tiles_q;
    const int64_t ldp = round_up(h->out, 4);
    int best = 1;
    int64_t cost = (tiles + sms - 1) / sms * g.stages;
    for (int k = 2; k <= 16 && k <= g.stages && k * rows * ldp <= kPartFloats; ++k) {
        const int per = (g.stages + k - 1) / k, real = (g.stages + per - 1) / per;
        const int64_t c = (tiles * real + sms - 1) / sms * per + 3;    // and joining them: about three stages
        if (c < cost) {
            cost = c;
            best = real;
        }
    }
    g.stages_per_split = (g.stages + best - 1) / best;
    g.splits = (g.stages + g.stages_per_split - 1) / g.stages_per_split;
    g.total = (int)(tiles * g.splits);
    g.y = g.splits > 1 ? h->part : y;
    g.ldy = g.splits > 1 ? ldp : ldy;
    g.slice = rows * ldp;
    g.out = g.splits > 1 || y_type == NITRO_F32;
    g.vec = g.splits > 1 || (((uintptr_t)y & 15) == 0 && ldy * (y_type == NITRO_F32 ? 4 : 2) % 16 == 0);
    const double ops = 2.0 * rows * h->in * h->out;
    const double bytes = (double)code_bytes(h->out, h->in) * 17 / 16 + code_bytes(rows, h->in) + 2.0 * rows * h->out;
    const uint8_t *p = swap ? w_codes : h->xq, *q = swap ? h->xq : w_codes;
    if (bn == 32) TRY((mx_launch<32, true>(p, g.P, q, g.Q, pitch, g, ops, bytes, s)));
    else if (bn == 64) TRY((mx_launch<64, true>(p, g.P, q, g.Q, pitch, g, ops, bytes, s)));
    else TRY((mx_launch<128, false>(p, g.P, q, g.Q, pitch, g, ops, bytes, s)));
    if (g.splits > 1) {
        const int64_t n = (int64_t)rows * h->out;
        ProfScope ps(K_MX4_LINEAR, s, 0.0, (4.0 * g.splits + 2.0) * n);
        TRY(launch_k(k_mx4_join, dim3((unsigned)std::min<int64_t>((n + 255) / 256, sms * 8)), dim3(256), 0, s,
                     (const float*)h->part, g.splits, g.slice, ldp, rows, h->out, y, ldy, (int)(y_type == NITRO_F32)));
    }
    return NITRO_OK;
}

nitro_status nitro_mx4_status(nitro_mx4* h, int clear) {
    if (!h) return NITRO_ERR_ARG;
    uint32_t bits = 0;
    if (cudaDeviceSynchronize() != cudaSuccess ||
        cudaMemcpy(&bits, h->status, 4, cudaMemcpyDeviceToHost) != cudaSuccess ||
        (clear && cudaMemset(h->status, 0, 4) != cudaSuccess))
        return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_mx4_destroy(nitro_mx4* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    for (void* p : h->allocs) cudaFree(p);
    delete h;
}

}  // extern "C"
