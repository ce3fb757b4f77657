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
// the tensor cores take scales from TMEM, so a tile is one run of bytes in global and shared
// memory and goes on to TMEM by one tcgen05.cp.
//
// The product runs on tcgen05.mma kind::mxf4 (products and scales exact, 32-bit sums).
#include <new>

#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "head_gemm.cuh"

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

// eight values -> eight e2m1 codes, v[0] lowest; nearest, ties to even, at most 6
__device__ __forceinline__ uint32_t e2m1x8(const float* v) {
    uint32_t r;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}\n"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// 32 bytes in one access (both 32-byte aligned)
__device__ __forceinline__ void load32(const void* p, uint4* a, uint4* b) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a->x), "=r"(a->y), "=r"(a->z), "=r"(a->w), "=r"(b->x), "=r"(b->y), "=r"(b->z), "=r"(b->w)
                 : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
// what rows at p, ld values apart, are aligned to: 32, 16 or fewer bytes (2, 1, 0)
int row_vec(const void* p, int64_t ld, int size) {
    const uintptr_t low = (uintptr_t)p | (uintptr_t)(ld * size);
    return (low & 31) == 0 ? 2 : (low & 15) == 0 ? 1 : 0;
}

// eight values as loaded
template <typename T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
    // the largest magnitude's bits (magnitudes as integers keep their order, and a NaN is the largest)
    __device__ __forceinline__ uint32_t top() const {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
        if constexpr (sizeof(T) == 2) {
            const uint32_t m = __vmaxu2(__vmaxu2(u[0] & 0x7fff7fffu, u[1] & 0x7fff7fffu),
                                        __vmaxu2(u[2] & 0x7fff7fffu, u[3] & 0x7fff7fffu));
            return max(m << 16, m & 0xffff0000u);
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, u[j] & 0x7fffffffu);
            return m;
        }
    }
    // times 2^k, the float `f`: exact where it matters (below the smallest normal it is 0 as a code)
    __device__ __forceinline__ uint32_t codes(float f) const {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
        float v[8];
        if constexpr (sizeof(T) == 2) {
            const __nv_bfloat162 k = __float2bfloat162_rn(f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&u[j]), k);
                const uint32_t b = *reinterpret_cast<const uint32_t*>(&p);
                v[2 * j] = __uint_as_float(b << 16);
                v[2 * j + 1] = __uint_as_float(b & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(u[j]) * f;
        }
        return e2m1x8(v);
    }
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* src, int n, bool vec) {
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = make_uint4(0, 0, 0, 0);
    if (vec && n >= 8) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) r.w[j] = reinterpret_cast<const uint4*>(src)[j];
    } else if (n > 0) {
        uint32_t* u = reinterpret_cast<uint32_t*>(r.w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= n) continue;
            if constexpr (sizeof(T) == 2) u[j >> 1] |= (uint32_t)src[j] << (16 * (j & 1));
            else u[j] = __float_as_uint(src[j]);
        }
    }
    return r;
}
// sixteen, vec: see row_vec
template <typename T>
__device__ __forceinline__ void load16(Raw8<T>* r, const T* src, int n, int vec) {
    if (vec == 2 && n >= 16) {
        if constexpr (sizeof(T) == 2) {
            load32(src, &r[0].w[0], &r[1].w[0]);
        } else {
            load32(src, &r[0].w[0], &r[0].w[1]);
            load32(src + 8, &r[1].w[0], &r[1].w[1]);
        }
        return;
    }
    r[0] = load8(src, n, vec != 0);
    r[1] = load8(src + 8, n - 8, vec != 0);
}
// Rows at odd addresses.  A lane's sixteen values by sixteen accesses of its own would be 32 sectors
// each; here half a warp takes sixteen values together, two lanes' an instruction, and they change
// hands in shared memory (`box`: a warp's 32 x 16 values).  All lanes call; `n` of a lane's values
// are in its row, none if not above 0.  16384 x 4097 in bf16: to 4 bits 73 -> 67 us, back 401 -> 62.
template <typename T>
__device__ __forceinline__ void lanes_load16(T* box, int lane, const T* src, int n, Raw8<T>* r) {
    T v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int of = 2 * i + (lane >> 4);
        const T* at = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(src), of));
        v[i] = (lane & 15) < __shfl_sync(0xffffffffu, n, of) ? at[lane & 15] : (T)0;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) box[(2 * i + (lane >> 4)) * 16 + (lane & 15)] = v[i];
    __syncwarp();
    const uint4* mine = reinterpret_cast<const uint4*>(box + lane * 16);
#pragma unroll
    for (int j = 0; j < (int)sizeof(T); ++j) r[j / (sizeof(T) / 2)].w[j % (sizeof(T) / 2)] = mine[j];
    __syncwarp();
}
template <typename T>
__device__ __forceinline__ void lanes_store16(T* box, int lane, T* dst, int n, const uint4* v) {
    uint4* mine = reinterpret_cast<uint4*>(box + lane * 16);
#pragma unroll
    for (int j = 0; j < (int)sizeof(T); ++j) mine[j] = v[j];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int of = 2 * i + (lane >> 4);
        T* at = reinterpret_cast<T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), of));
        if ((lane & 15) < __shfl_sync(0xffffffffu, n, of)) at[lane & 15] = box[of * 16 + (lane & 15)];
    }
    __syncwarp();
}
// a block's scale as stored, from its largest magnitude's bits: that exponent less 2, at
// least 0; 255: not finite
__device__ __forceinline__ uint32_t scale_code(uint32_t top) {
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}
// 2^(127 - s), what a block's values are multiplied by: 254 - s as an exponent (s = 254 cannot be)
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __uint_as_float((254u - min(s, 253u)) << 23); }

// Two threads a block, sixteen values each, two such loads in flight.  The grid covers the
// scales' padding too.  Bound by memory and, nearly, by the instructions (9 a value): 16384 x
// 4096 in bf16 28.7 us, 5.9 TB/s; with 16-byte loads, one multiplication and one integer
// maximum a value and a division an item 58 us.
template <typename T>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T* x, int64_t ldx, int rows, int cols, uint8_t* q, uint8_t* sc,
                                                      int blocks, int64_t rows_pad, int vec) {
    __shared__ __align__(16) T box[8][512];
    pdl_wait();
    const int tiles = (blocks + 3) / 4, per = tiles * 8;
    const int64_t n = rows_pad * per, step = (int64_t)gridDim.x * 256;
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, step, per);
    for (int64_t base = blockIdx.x * (int64_t)256; base < n; base += 2 * step) {
        Raw8<T> raw[2][2];
        int64_t row[2];
        int part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            row[u] = at.row;
            part[u] = at.part;
            const int c = at.part * 16;
            const T* src = x + at.row * ldx + c;
            const int left = at.row < rows ? cols - c : 0;
            if (vec) load16(raw[u], src, left, vec);
            else lanes_load16(box[threadIdx.x >> 5], threadIdx.x & 31, src, left, raw[u]);
            at.next();
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t top = max(raw[u][0].top(), raw[u][1].top());
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const uint32_t s = scale_code(top);
            const float inv = scale_inverse(s);
            const uint2 w = make_uint2(raw[u][0].codes(inv), raw[u][1].codes(inv));
            const int blk = part[u] >> 1;
            const bool in = row[u] < rows && blk < blocks;
            if (in) *reinterpret_cast<uint2*>(q + (row[u] * blocks + blk) * 16 + (part[u] & 1) * 8) = w;
            if ((part[u] & 1) == 0 && row[u] < rows_pad) sc[scale_at(row[u], blk, tiles)] = in ? (uint8_t)s : 0;
        }
    }
}

// a scale as a value
__device__ __forceinline__ float e8m0_value(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}
// Codes 4h to 4h + 3 of a word as two words of two bf16 each: the halves of the magnitudes 0,
// 1/2, 1, 3/2, 2, 3, 4, 6 (0000 3f00 3f80 3fc0 4000 4040 4080 40c0) looked up byte by byte, four
// codes a look-up, and the codes' sign bits.
__device__ __forceinline__ void e2m1_bf16x4(uint32_t w, int h, uint32_t* out) {
    const uint32_t sel = (w >> (16 * h)) & 0x7777u;
    const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, sel), lo = __byte_perm(0xc0800000u, 0xc0804000u, sel);
    // bytes 1 and 3: the one that has a code's sign on top
    const uint32_t up = w << 4;
    out[0] = __byte_perm(lo, hi, 0x5140) | (__byte_perm(up, w, h ? 0x6020 : 0x4000) & 0x80008000u);
    out[1] = __byte_perm(lo, hi, 0x7362) | (__byte_perm(up, w, h ? 0x7030 : 0x5010) & 0x80008000u);
}

// Sixteen values a thread, two loads in flight.  Bound by memory: 16384 x 4096 to bf16 31 us,
// 5.7 TB/s (36.5 with 16-byte stores, which fill half a sector each).
template <typename T>
__global__ void __launch_bounds__(256) k_mx4_dequantize(const uint8_t* q, const uint8_t* sc, int rows, int cols, int blocks,
                                                        T* out, int64_t ldo, float* scales, int vec) {
    __shared__ __align__(16) T box[8][512];
    pdl_wait();
    const int tiles = (blocks + 3) / 4, per = blocks * 2;
    const int64_t step = (int64_t)gridDim.x * 256;
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, step, per);
    const uint2* src = reinterpret_cast<const uint2*>(q) + blockIdx.x * (int64_t)256 + threadIdx.x;
    while (__any_sync(0xffffffffu, at.row < rows)) {
        uint2 w[2] = {};
        uint32_t s[2] = {};
        int64_t row[2];
        int part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u, src += step) {
            row[u] = at.row;
            part[u] = at.part;
            if (at.row < rows) {
                w[u] = *src;
                s[u] = sc[scale_at(at.row, at.part >> 1, tiles)];
            }
            at.next();
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool in = row[u] < rows;
            if (vec && !in) continue;
            const int c = part[u] * 16;
            const float f = e8m0_value(s[u]);
            if (in && scales && (part[u] & 1) == 0) scales[row[u] * blocks + (part[u] >> 1)] = f;
            T* dst = out + row[u] * ldo + c;
            __align__(16) uint32_t v[8];      // two values each, as bf16
            e2m1_bf16x4(w[u].x, 0, v);
            e2m1_bf16x4(w[u].x, 1, v + 2);
            e2m1_bf16x4(w[u].y, 0, v + 4);
            e2m1_bf16x4(w[u].y, 1, v + 6);
            if constexpr (sizeof(T) == 2) {
                const __nv_bfloat162 k = __float2bfloat162_rn(f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&v[j]), k);
                    v[j] = *reinterpret_cast<const uint32_t*>(&p);
                }
                if (!vec) {
                    lanes_store16(box[threadIdx.x >> 5], threadIdx.x & 31, dst, in ? cols - c : 0, reinterpret_cast<const uint4*>(v));
                } else if (vec == 2 && c + 16 <= cols) {
                    store32(dst, v);
                } else if (c + 16 <= cols) {
                    reinterpret_cast<uint4*>(dst)[0] = make_uint4(v[0], v[1], v[2], v[3]);
                    reinterpret_cast<uint4*>(dst)[1] = make_uint4(v[4], v[5], v[6], v[7]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < cols) dst[j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
                }
            } else {
                __align__(16) float o[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16) * f;
                if (!vec) {
                    lanes_store16(box[threadIdx.x >> 5], threadIdx.x & 31, dst, in ? cols - c : 0, reinterpret_cast<const uint4*>(o));
                } else if (vec == 2 && c + 16 <= cols) {
                    store32(dst, reinterpret_cast<const uint32_t*>(o));
                    store32(dst + 8, reinterpret_cast<const uint32_t*>(o) + 8);
                } else if (c + 16 <= cols) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        reinterpret_cast<float4*>(dst)[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < cols) dst[j] = o[j];
                }
            }
        }
    }
}

// ------------------------------------------------------------------ product
// D[p][q] = sum_k P[p][k] Q[q][k], 128 CG rows of P (TMEM lanes) x BN rows of Q (columns) a
// tile, 256 elements of K (128 bytes) a stage.  SWAP: P is W and Q the features, for few
// samples: a tile then has 128 of W's rows and as few columns as there are samples, and the
// weights stream past once.  CG = 2 pairs two CTAs on 256 x 256 (see head_gemm.cuh): at the
// 4-bit rate the MMAs of a stage take a third of the time of its loads, so what counts is
// products a byte loaded.  FX (bf16 or fp32, for SWAP): Q's codes and scales are not loaded but made by
// the epilogue warps from the features themselves, stage by stage, which saves the launch
// that would quantise them; every CTA does so for its own, so it is for few rows.  A pair's accumulator and scales fill TMEM, so its drain waits for
// the next tile's MMAs, but not for its loads.
//
// Scales go from shared memory to TMEM by tcgen05.cp, 34 ns a tile of 512 bytes, which hold the
// thread that issues them; with six of them before a stage's four MMAs (45 ns each) in one thread a
// stage took 0.5 us (8192^3: 243 us).  So a thread of its own issues them, up to four stages ahead.
// Measured: 8192^3 204 us, 5.4 PFLOP/s, 0.41 us a stage of 35 KB a CTA, bound by its loads; one
// row x 4096 x 10000 10 us, of which 79 CTAs' sixteen stages are 6.  (Scales put into TMEM by
// warps, tcgen05.st: 405 us.)
constexpr int kMxThreads = 384, kMxEpiWarp0 = 4, kMxEpiWarps = 8;
constexpr int kMxScaleBufs = 4;      // stages whose scales are in TMEM

struct MxArgs {
    int P, Q;                // valid rows
    int tiles_p, tiles_q, splits, total, band;
    int k64;                 // steps of 64 along K
    int stages, stages_per_split;
    void* y;                 // output, or slices of 32-bit partial sums
    int64_t ldy, slice;
    int out;                 // 0 bf16, 1 fp32
    int vec;                 // rows of y are 16-byte aligned
    uint32_t* status;
    const void* x;           // FX: the features [Q][in]
    int64_t ldx;
    int in, vec_x;
};
struct MxMaps {
    CUtensorMap p, q, sp, sq;      // codes, scale tiles
};

struct NoFx {};

template <int CG, int BN>
struct MxCfg {
    static constexpr int P_BYTES = 128 * 128, Q_ROWS = BN / CG, Q_BYTES = Q_ROWS * 128;
    static constexpr int QT = BN > 128 ? 2 : 1;               // scale tiles of 128 rows a tile's columns take
    static constexpr int SF_BYTES = 1024 + QT * 1024;
    static constexpr int STAGE = P_BYTES + Q_BYTES + SF_BYTES;
    static constexpr int S = BN >= 128 ? 6 : 8;
    static constexpr int SMEM = S * STAGE + kMxEpiWarps * 2048 + 256;
    static constexpr int NBUF = CG == 2 ? 1 : 2;               // accumulators
    static constexpr int SF = NBUF * BN, SF_COLS = 8 + 8 * QT; // TMEM columns of a stage's scales
    static constexpr int SF_END = SF + kMxScaleBufs * SF_COLS;
    static constexpr int TCOLS = SF_END <= 128 ? 128 : SF_END <= 256 ? 256 : 512;
    static_assert(SF_END <= 512, "TMEM");
};

template <int CG>
__device__ __forceinline__ void mx_tma(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1)
            : "memory");
    else
        tma_load_2d(dst, m, bar, c0, c1);
}
// 32 rows of 16 bytes (a scale tile) -> four TMEM columns, the same for every lane quadrant
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint32_t saddr) {
    const uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
    if constexpr (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                         uint32_t accumulate) {
    if constexpr (CG == 2)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
            : "memory");
}
// kind::mxf4, e2m1 operands, e8m0 scales of 32; half: which two of a scale word's four bytes
__host__ __device__ constexpr uint32_t mx_idesc(int m, int n, int half) {
    return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) |
           ((uint32_t)(m >> 4) << 24) | ((uint32_t)(2 * half) << 29);
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

template <int CG, int BN, bool SWAP, typename FX>
__global__ void __launch_bounds__(kMxThreads, 1) k_mx4_gemm(const __grid_constant__ MxMaps maps, const MxArgs g) {
    using C = MxCfg<CG, BN>;
    constexpr int S = C::S;
    constexpr bool kFx = !std::is_same_v<FX, NoFx>;
    static_assert(!kFx || (SWAP && BN == 32), "features in the kernel: for few rows");
    extern __shared__ __align__(1024) uint8_t smem[];
    // stages of operands (1024-byte aligned), the scales, the warps' own 2 KB
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S * C::STAGE + kMxEpiWarps * 2048);
    // barriers: full [S], empty [S], tmem full [2], empty [2], drain [2], scales in [4] and out of use [4]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * S + 6 + 2 * kMxScaleBufs);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t bar0 = smem_u32(bars), s0 = smem_u32(smem), sf0 = s0 + S * (C::P_BYTES + C::Q_BYTES);
    const auto full_bar = [&](int s) { return bar0 + 8u * s; };
    const auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
    const auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * S + b); };
    const auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * S + 2 + b); };
    const auto drain_bar = [&](int i) { return bar0 + 8u * (2 * S + 4 + i); };
    const auto sin_bar = [&](int b) { return bar0 + 8u * (2 * S + 6 + b); };
    const auto sout_bar = [&](int b) { return bar0 + 8u * (2 * S + 6 + kMxScaleBufs + b); };
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    const int unit = (int)blockIdx.x / CG, units = (int)gridDim.x / CG;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full_bar(s), kFx ? 2 : 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull_bar(b), 1);
            mbar_init(tempty_bar(b), CG * kMxEpiWarps);
        }
        for (int b = 0; b < kMxScaleBufs; ++b) {
            mbar_init(sin_bar(b), 1);
            mbar_init(sout_bar(b), 1);
        }
        mbar_init(drain_bar(0), 1);
        mbar_init(drain_bar(1), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) hg_tmem_alloc<CG>(smem_u32(tmem_slot), C::TCOLS);
    if constexpr (kFx) {     // rows past the last one stay zero
        for (int i = threadIdx.x; i < S * C::STAGE / 16; i += kMxThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0 && lane < 4)
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.p + lane)) : "memory");
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            int st = 0, loaded = 0;
            uint32_t ph = 1;
            for (int tile = unit; tile < g.total; tile += units) {
                const MxTile T = mx_decode(g, tile);
                const int p0 = T.p * 128 * CG + rank * 128, q0 = T.q * BN;
                for (int k = T.s0; k < T.s1; ++k) {
                    if (!mbar_wait(empty_bar(st), ph, abort_flag, g.status)) goto producer_out;
                    const uint32_t dp = s0 + st * (C::P_BYTES + C::Q_BYTES), dq = dp + C::P_BYTES, ds = sf0 + st * C::SF_BYTES;
                    uint32_t fb = full_bar(st);
                    if (CG == 1 || rank == 0) mbar_expect_tx(fb, kFx ? C::P_BYTES + 1024 : CG * C::STAGE);
                    if constexpr (CG == 2) fb = remote_smem(fb, 0);
                    mx_tma<CG>(dp, &maps.p, fb, k * 128, p0);
                    mx_tma<CG>(ds, &maps.sp, fb, k * 256, p0 / 128);
                    if constexpr (!kFx) {
                        mx_tma<CG>(dq, &maps.q, fb, k * 128, q0 + rank * C::Q_ROWS);
                        // both CTAs of a pair hold the scales of all columns
                        mx_tma<CG>(ds + 1024, &maps.sq, fb, k * 256, q0 / 128);
                    }
                    ++loaded;
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
            }
        producer_out:
            if (*abort_flag) {
                for (int k = max(0, loaded - S); k < loaded; ++k)
                    mbar_drain(full_bar(k % S), (uint32_t)(k / S) & 1u, kDrainNs);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint64_t dp0 = desc_sw128(s0), dq0 = desc_sw128(s0 + C::P_BYTES);
            int st = 0, it = 0, n = 0;
            uint32_t ph = 0;
            for (int tile = unit; tile < g.total; tile += units, ++it) {
                const MxTile T = mx_decode(g, tile);
                const int buf = it % C::NBUF;
                if (!mbar_wait(tempty_bar(buf), ((uint32_t)(it / C::NBUF) & 1u) ^ 1u, abort_flag, g.status)) break;
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * BN);
                bool ok = true;
                for (int k = T.s0; k < T.s1; ++k, ++n) {
                    const int sbuf = n % kMxScaleBufs;
                    ok = mbar_wait(full_bar(st), ph, abort_flag, g.status) &&
                         mbar_wait(sin_bar(sbuf), (uint32_t)(n / kMxScaleBufs) & 1u, abort_flag, g.status);
                    if (!ok) break;
                    tc_fence_after();
                    const int steps = min(4, g.k64 - 4 * k);
                    const uint32_t sp = tmem + C::SF + C::SF_COLS * sbuf, sq = sp + 8;
                    const uint64_t so = (uint64_t)((uint32_t)(st * (C::P_BYTES + C::Q_BYTES)) >> 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < steps)
                            mma_mxf4<CG>(d, dp0 + so + 2 * j, dq0 + so + 2 * j, mx_idesc(128 * CG, BN, j & 1), sp + 4u * (j >> 1),
                                         sq + 4u * C::QT * (j >> 1), (k > T.s0 || j > 0) ? 1u : 0u);
                    hg_commit<CG>(empty_bar(st));
                    hg_commit<CG>(sout_bar(sbuf));
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
                if (!ok) break;
                hg_commit<CG>(tfull_bar(buf));
            }
            if (*abort_flag) {
                hg_commit<CG>(drain_bar(0));
                mbar_drain(drain_bar(0), 0, kDrainNs);
            }
            pdl_trigger();
        }
    } else if (warp == 3) {
        if (lane == 0 && rank == 0) {
            // ---------------- scales to TMEM, ahead of the MMAs
            int st = 0, n = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int tile = unit; tile < g.total && ok; tile += units) {
                const MxTile T = mx_decode(g, tile);
                for (int k = T.s0; k < T.s1; ++k, ++n) {
                    const int sbuf = n % kMxScaleBufs;
                    ok = mbar_wait(full_bar(st), ph, abort_flag, g.status) &&
                         mbar_wait(sout_bar(sbuf), ((uint32_t)(n / kMxScaleBufs) & 1u) ^ 1u, abort_flag, g.status);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sp = tmem + C::SF + C::SF_COLS * sbuf, sq = sp + 8, ds = sf0 + st * C::SF_BYTES;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        copy_scales<CG>(sp + 4 * j, ds + 512 * j);
#pragma unroll
                        for (int r = 0; r < C::QT; ++r) copy_scales<CG>(sq + 4 * (C::QT * j + r), ds + 1024 + 1024 * r + 512 * j);
                    }
                    hg_commit<CG>(sin_bar(sbuf));
                    if (++st == S) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
            }
            if (*abort_flag) {
                hg_commit<CG>(drain_bar(1));
                mbar_drain(drain_bar(1), 0, kDrainNs);
            }
        }
    } else if (warp >= kMxEpiWarp0) {
        const int q = warp & 3, half = (warp - kMxEpiWarp0) >> 2;
        const HgStage hs{reinterpret_cast<uint4*>(smem + S * C::STAGE) + (warp - kMxEpiWarp0) * 128, lane};
        int it = 0, made = 0;       // made: stages of the tiles before
        for (int tile = unit; tile < g.total; tile += units, ++it) {
            const MxTile T = mx_decode(g, tile);
            const int buf = it % C::NBUF;
            if constexpr (kFx) {
                // Every eighth stage is this warp's, so that the loads' latencies overlap (all
                // warps on each stage took 16.5 us where two launches take 14.4): sixteen values a
                // thread, two threads a block, two rows at a time, four of those in flight.
                const int part = lane & 15, r0 = lane >> 4, blk = part >> 1;
                const FX* x = static_cast<const FX*>(g.x);
                bool ok = true;
                for (int k = T.s0 + warp - kMxEpiWarp0; k < T.s1 && ok; k += kMxEpiWarps) {
                    const int n = made + k - T.s0, st = n % S, c = k * 256 + part * 16;
                    uint8_t* dq = smem + st * (C::P_BYTES + C::Q_BYTES) + C::P_BYTES;
                    uint8_t* ds = smem + S * (C::P_BYTES + C::Q_BYTES) + st * C::SF_BYTES + 1024;
                    for (int rb = 0; rb < g.Q; rb += 8) {
                        Raw8<FX> raw[4][2];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = rb + 2 * u + r0, left = r < g.Q ? g.in - c : 0;
                            const FX* src = x + r * g.ldx + c;
                            load16(raw[u], src, left, g.vec_x);
                        }
                        if (rb == 0) {
                            ok = mbar_wait(empty_bar(st), ((uint32_t)(n / S) & 1u) ^ 1u, abort_flag, g.status);
                            if (!(ok = __all_sync(0xffffffffu, ok))) break;
                        }
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = rb + 2 * u + r0;
                            uint32_t top = max(raw[u][0].top(), raw[u][1].top());
                            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                            const uint32_t s = scale_code(top);
                            const float inv = scale_inverse(s);
                            const uint2 w = make_uint2(raw[u][0].codes(inv), raw[u][1].codes(inv));
                            if (r >= g.Q) continue;
                            *reinterpret_cast<uint2*>(dq + r * 128 + ((blk ^ (r & 7)) << 4) + (part & 1) * 8) = w;
                            if ((part & 1) == 0) ds[(blk >> 2) * 512 + r * 16 + (blk & 3)] = (uint8_t)s;
                        }
                        __syncwarp();
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0 && ok) mbar_arrive(full_bar(st));
                }
                if (!ok) break;
                made += T.s1 - T.s0;
            }
            const bool ok = mbar_wait(tfull_bar(buf), (uint32_t)(it / C::NBUF) & 1u, abort_flag, g.status);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const int row0 = T.p * 128 * CG + rank * 128 + q * 32, row = row0 + lane, col0 = T.q * BN + half * (BN / 2);
            const uint32_t src = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * BN + half * (BN / 2));
            float* yf = static_cast<float*>(g.y) + T.split * g.slice;
            uint16_t* yb = static_cast<uint16_t*>(g.y);
            const auto release = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 2) mbar_arrive_remote(remote_smem(tempty_bar(buf), 0));
                    else mbar_arrive(tempty_bar(buf));
                }
            };
            if constexpr (SWAP) {
#pragma unroll 1
                for (int c = 0; c < BN / 2; c += 16) {
                    uint32_t v[16];
                    __syncwarp();
                    tmem_ld16_nowait(src + c, v);
                    tmem_wait_ld<16>(v);
                    if (c + 16 == BN / 2) release();
                    const int n = g.Q - (col0 + c);
                    if (row >= g.P || n <= 0) continue;
                    const float* f = reinterpret_cast<const float*>(v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        if (j >= n) continue;
                        const int64_t at = (int64_t)(col0 + c + j) * g.ldy + row;
                        if (g.out) yf[at] = f[j];
                        else yb[at] = __bfloat16_as_ushort(__float2bfloat16_rn(f[j]));
                    }
                }
            } else {
                // all columns in bf16 leave TMEM before the first is stored, so that the next tile's
                // MMAs wait no longer than for that
                constexpr int N = BN / 64;
                const HgPart hp{row, row0, g.P, col0, BN / 2, half, hs};
                if (!g.out) {
                    uint32_t w[N][16];
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        uint32_t v[32];
                        __syncwarp();
                        tmem_ld32_nowait(src + 32 * c, v);
                        tmem_wait_ld<32>(v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const __nv_bfloat162 p = __floats2bfloat162_rn(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
                            w[c][j] = *reinterpret_cast<const uint32_t*>(&p);
                        }
                    }
                    release();
#pragma unroll
                    for (int c = 0; c < N; ++c)
                        if (col0 + 32 * c < g.Q) hg_store16(hp, w[c], yb, g.ldy, col0 + 32 * c, g.Q, g.vec != 0);
                } else {
#pragma unroll 1
                    for (int c = 0; c < BN / 2; c += 32) {
                        uint4 v[8];
                        __syncwarp();
                        tmem_ld32_nowait(src + c, reinterpret_cast<uint32_t*>(v));
                        tmem_wait_ld<32>(reinterpret_cast<uint32_t*>(v));
                        if (c + 32 == BN / 2) release();
                        if (!g.vec) {      // see hg_store16()
                            const int rows = min(32, g.P - row0);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int cc = col0 + c + 16 * h + (lane & 15);
                                hs.put(v + 4 * h);
                                float* dst = yf + (int64_t)(row0 + (lane >> 4)) * g.ldy + cc;
#pragma unroll 4
                                for (int r = lane >> 4; r < rows; r += 2, dst += 2 * g.ldy)
                                    if (cc < g.Q) *dst = hs.value<float>(r, lane & 15);
                                __syncwarp();
                            }
                            continue;
                        }
                        hs.to_lines(v);
                        hs.to_lines(v + 4);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int r = row0 + hs.line_row(k & 3), cc = col0 + c + 16 * (k >> 2) + 4 * hs.line_chunk();
                            if (r >= g.P || cc >= g.Q) continue;
                            float* dst = yf + (int64_t)r * g.ldy + cc;
                            if (cc + 4 <= g.Q) {
                                *reinterpret_cast<uint4*>(dst) = v[k];
                            } else {
                                const uint32_t u[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (cc + j < g.Q) dst[j] = __uint_as_float(u[j]);
                            }
                        }
                    }
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_barrier();
    if (warp == 2) {
        tc_fence_after();
        hg_tmem_free<CG>(tmem, C::TCOLS);
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
// scale tiles as rows of words, two tiles along K a box; those past the end read as zero
bool mx_scale_map(CUtensorMap* m, const uint8_t* scales, int64_t rows, int64_t tiles_k, int box_tiles) {
    auto fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dim[2] = {(cuuint64_t)tiles_k * 128, (cuuint64_t)((rows + 127) / 128)}, stride[1] = {(cuuint64_t)tiles_k * 512};
    cuuint32_t box[2] = {256, (cuuint32_t)box_tiles}, step[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t*>(scales), dim, stride, box, step,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct MxOperand {
    const uint8_t *codes, *scales;
    int64_t rows;
};

template <int CG, int BN, bool SWAP, typename FX = NoFx>
cudaError_t mx_launch(const MxOperand& p, const MxOperand& q, int in, MxArgs g, double ops, double bytes, cudaStream_t s) {
    using C = MxCfg<CG, BN>;
    MxMaps m;
    const int64_t pitch = blocks_of(in) * 16, tiles_k = (blocks_of(in) + 3) / 4;
    if (!mx_map(&m.p, p.codes, p.rows, pitch, 128) || !mx_scale_map(&m.sp, p.scales, p.rows, tiles_k, 1)) return cudaErrorInvalidValue;
    if (std::is_same_v<FX, NoFx>) {
        if (!mx_map(&m.q, q.codes, q.rows, pitch, C::Q_ROWS) || !mx_scale_map(&m.sq, q.scales, q.rows, tiles_k, C::QT))
            return cudaErrorInvalidValue;
    } else {
        m.q = m.p;      // not read
        m.sq = m.sp;
    }
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    const int sms = sm_count(&dev);
    const cudaError_t e = once_per_device(ready, dev, [] {
        return cudaFuncSetAttribute(k_mx4_gemm<CG, BN, SWAP, FX>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    });
    if (e != cudaSuccess) return e;
    const int grid = std::min(g.total, sms / CG) * CG;
    ProfScope ps(K_MX4_LINEAR, s, ops, bytes);
    if constexpr (CG == 2) return launch_cluster(k_mx4_gemm<CG, BN, SWAP, FX>, dim3(grid), kMxThreads, 2, s, C::SMEM, m, g);
    else return launch_k(k_mx4_gemm<CG, BN, SWAP, FX>, dim3(grid), dim3(kMxThreads), C::SMEM, s, m, g);
}


template <typename T>
cudaError_t quantize(const T* x, int64_t ldx, int rows, int cols, uint8_t* q, uint8_t* sc, cudaStream_t s) {
    const int blocks = (int)blocks_of(cols);
    const int64_t pad = round_up(rows, 128), n = pad * ((blocks + 3) / 4) * 8;
    static std::atomic<int> resident{0};
    const int grid = one_wave(k_mx4_quantize<T>, resident, n);
    const int vec = row_vec(x, ldx, (int)sizeof(T));
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
    StatusWord status;
    DeviceAllocs allocs;
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
    const int64_t n = (int64_t)rows * blocks * 2;
    static std::atomic<int> resident[2];
    const int grid = type == NITRO_BF16 ? one_wave(k_mx4_dequantize<uint16_t>, resident[0], n)
                                        : one_wave(k_mx4_dequantize<float>, resident[1], n);
    const int size = type == NITRO_BF16 ? 2 : 4;
    const int vec = row_vec(out, ldo, size);
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
    const bool ok = h->allocs.take(&h->xq, code_bytes(max_rows, in)) && h->allocs.take(&h->xs, scale_bytes(max_rows, in)) &&
                    h->allocs.take(&h->part, kPartFloats) && h->status.take();
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
    // up to this many rows the product's CTAs quantise them themselves
    const bool inside = rows <= 32;
    if (!inside) {
        if (x_type == NITRO_BF16) TRY(quantize((const uint16_t*)x, ldx, rows, h->in, h->xq, h->xs, s));
        else TRY(quantize((const float*)x, ldx, rows, h->in, h->xq, h->xs, s));
    }
    // Few samples: W's rows along the lanes.  Else pairs, or 128 x 128 tiles where those finish
    // earlier: a stage takes a lone CTA and a pair the same time (32 KB into an SM).
    const bool swap = rows <= 64;
    const int sms = sm_count();
    MxArgs g{};
    g.P = swap ? h->out : rows;
    g.Q = swap ? rows : h->out;
    g.band = 8;
    g.k64 = (h->in + 63) / 64;
    g.stages = (g.k64 + 3) / 4;
    g.status = h->status.at;
    const int64_t ldp = round_up(h->out, 4);
    int cg = 1, bn = 0, splits = 1;
    int64_t cost = INT64_MAX;
    const auto consider = [&](int c, int n) {
        // K is shared out where that shortens the longest CTA's work
        const int64_t tiles = (int64_t)((g.P + 128 * c - 1) / (128 * c)) * ((g.Q + n - 1) / n), units = sms / c;
        for (int k = 1; k <= 16 && k <= g.stages && (k == 1 || k * rows * ldp <= kPartFloats); ++k) {
            const int per = (g.stages + k - 1) / k;
            if ((g.stages + per - 1) / per != k) continue;
            // in stages: two for a tile's ends, eight to join splits (by four 300 x 4096 x 4096 took a split and
            // 19.7 us, now 14.8, and 500 x 2048 x 2048 15.8, now 11.3; by twelve 16 x 4096 x 4096 loses one
            // that is worth having, 9.1 against 11.5)
            const int64_t t = (tiles * k + units - 1) / units * (per + 2) + (k > 1 ? 8 : 0);
            if (t < cost) {
                cost = t;
                cg = c;
                bn = n;
                splits = k;
            }
        }
    };
    if (swap) {
        consider(1, inside ? 32 : 64);
    } else {
        consider(2, 256);
        consider(1, 128);
    }
    g.tiles_p = (g.P + 128 * cg - 1) / (128 * cg);
    g.tiles_q = (g.Q + bn - 1) / bn;
    g.stages_per_split = (g.stages + splits - 1) / splits;
    g.splits = splits;
    g.total = g.tiles_p * g.tiles_q * splits;
    g.y = splits > 1 ? h->part : y;
    g.ldy = splits > 1 ? ldp : ldy;
    g.slice = rows * ldp;
    g.out = splits > 1 || y_type == NITRO_F32;
    g.vec = splits > 1 || (((uintptr_t)y & 15) == 0 && ldy * (y_type == NITRO_F32 ? 4 : 2) % 16 == 0);
    const double ops = 2.0 * rows * h->in * h->out;
    const double bytes = (double)code_bytes(h->out, h->in) * 17 / 16 + code_bytes(rows, h->in) + 2.0 * rows * h->out;
    const MxOperand x_op{h->xq, h->xs, rows}, w_op{w_codes, w_scales, h->out};
    g.x = x;
    g.ldx = ldx;
    g.in = h->in;
    g.vec_x = row_vec(x, ldx, x_type == NITRO_F32 ? 4 : 2);
    if (inside && x_type == NITRO_BF16) TRY((mx_launch<1, 32, true, uint16_t>(w_op, x_op, h->in, g, ops, bytes, s)));
    else if (inside) TRY((mx_launch<1, 32, true, float>(w_op, x_op, h->in, g, ops, bytes, s)));
    else if (bn == 64) TRY((mx_launch<1, 64, true>(w_op, x_op, h->in, g, ops, bytes, s)));
    else if (cg == 1) TRY((mx_launch<1, 128, false>(x_op, w_op, h->in, g, ops, bytes, s)));
    else TRY((mx_launch<2, 256, false>(x_op, w_op, h->in, g, ops, bytes, s)));
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
    if (!h->status.read(clear != 0, &bits)) return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_mx4_destroy(nitro_mx4* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    h->allocs.free();
    h->status.free();
    delete h;
}

}  // extern "C"
