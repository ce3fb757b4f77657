// What the head's operators share beside the contraction: products into 32-bit slices or bf16 matrices, rows of
// a product on the CUDA cores, and exponentials and packing.
#pragma once

#include "head_gemm.cuh"

namespace nitro {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// 2^t of an exponential's argument, below 2^-126 zero: one instruction, where exp2f has four (a logit's
// part of an epilogue then is half as long)
__device__ __forceinline__ float ex2(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}

__device__ __forceinline__ void pack_bf16_32(const float* v, uint32_t* w) {
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
}

// ------------------------------------------------------------------ epilogues
// 32-bit sums into slice `split` of c, or added to what it holds.
struct EpiAcc {
    static constexpr bool kFold = false, kTail = false;
    struct Args {
        float* c;
        int64_t ldc, slice;   // ldc a multiple of 32
        int add;
    };
    const Args& a;
    const HgArgs& g;
    const HgPart& p;
    float* base;
    float4 old[8];         // lines of two 16-column halves
    __device__ __forceinline__ EpiAcc(const Args& a_, const HgArgs& g_, const HgTile& t, const HgPart& p_) : a(a_), g(g_), p(p_) {
        base = a.c + t.split * a.slice + p.col0;
    }
    __device__ __forceinline__ float4* line(int c, int k) const {
        const int row = p.row0 + p.stage.line_row(k & 3);
        if (row >= p.rows || p.col0 + c >= a.ldc) return nullptr;
        return reinterpret_cast<float4*>(base + (int64_t)row * a.ldc + c + 16 * (k >> 2) + 4 * p.stage.line_chunk());
    }
    __device__ __forceinline__ void fetch(int c) {
        if (!a.add) return;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (const float4* q = line(c, k)) old[k] = *q;
    }
    __device__ __forceinline__ void cols(int c, float* v) {
        uint4* w = reinterpret_cast<uint4*>(v);
        p.stage.to_lines(w);
        p.stage.to_lines(w + 4);
        float4* f = reinterpret_cast<float4*>(v);
        if (a.add) {
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k].x += old[k].x, f[k].y += old[k].y, f[k].z += old[k].z, f[k].w += old[k].w;
        }
        if (c + 32 < p.width) fetch(c + 32);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (float4* q = line(c, k)) *q = f[k];
    }
    __device__ __forceinline__ void done() {}
};

struct EpiBf16 {
    static constexpr bool kFold = false, kTail = false;
    struct Args {
        uint16_t* c;
        int64_t ldc;
        int vec;              // rows are 16-byte aligned
        const float* factor;  // of the row, or of all rows; null: all
        int one;
        float all = 1.0f;
    };
    const Args& a;
    const HgArgs& g;
    const HgPart& p;
    float f = 0.0f;
    __device__ __forceinline__ EpiBf16(const Args& a_, const HgArgs& g_, const HgTile&, const HgPart& p_) : a(a_), g(g_), p(p_) {
        if (p.row < p.rows) f = a.factor ? a.factor[a.one ? 0 : p.row] : a.all;
    }
    __device__ __forceinline__ void fetch(int) {}
    __device__ __forceinline__ void cols(int c, float* v) {
        if (p.col0 + c >= g.N) return;
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= f;
        uint32_t w[16];
        pack_bf16_32(v, w);
        hg_store16(p, w, a.c, a.ldc, p.col0 + c, g.N, a.vec != 0);
    }
    __device__ __forceinline__ void done() {}
};

// ------------------------------------------------------------------ few rows
// Eight elements of a row of a piece of 256: VEC takes eight in a row, 16 bytes (8 of int8), else every 32nd
template <typename T, bool VEC, bool WHOLE>
__device__ __forceinline__ void few_load(const T* row, int piece, int lane, int features, float* v) {
    if constexpr (VEC && WHOLE) {
        const T* at = row + piece + 8 * lane;
        if constexpr (sizeof(T) == 2) {
            const uint4 u = __ldg(reinterpret_cast<const uint4*>(at));
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
        } else {
            const uint2 u = __ldg(reinterpret_cast<const uint2*>(at));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)((j < 4 ? u.x : u.y) >> (8 * (j & 3)));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = piece + (VEC ? 8 * lane + j : 32 * j + lane);
            v[j] = 0.0f;
            if (WHOLE || col < features) {
                if constexpr (sizeof(T) == 2) v[j] = __uint_as_float((uint32_t)__ldg(row + col) << 16);
                else v[j] = (float)__ldg(row + col);
            }
        }
    }
}

template <typename T, int R, int C, bool VEC, bool WHOLE>
__device__ __forceinline__ void few_step(const T* const* x, const uint16_t* const* w, int piece, int lane, int features,
                                         float (*acc)[C]) {
    float wv[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) few_load<uint16_t, VEC, WHOLE>(w[c], piece, lane, features, wv[c]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float xv[8];
        few_load<T, VEC, WHOLE>(x[r], piece, lane, features, xv);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[r][c] = fmaf(xv[j], wv[c][j], acc[r][c]);
    }
}

// v[0..N) summed over the warp's lanes; a lane gets the sum number lane / (32 / N)
template <int N>
__device__ __forceinline__ float few_sum(float* v, int lane) {
    int bit = 16;
#pragma unroll
    for (int h = N / 2; h > 0; h >>= 1, bit >>= 1) {
        const bool up = lane & bit;
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
        }
    }
    for (; bit > 0; bit >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], bit);
    return v[0];
}

// ------------------------------------------------------------------ rows
// A matrix in bf16 from the slices of its 32-bit sums (EpiAcc), four columns a thread; factor: of the row, null: all.
__global__ void __launch_bounds__(256) k_head_slices(const float* c, int64_t ldc, int64_t slice, int slices, int cols,
                                                 const float* factor, float all, uint16_t* dx, int64_t lddx, int vec) {
    pdl_wait();
    const int64_t row = blockIdx.x;
    const float f = factor ? factor[row] : all;
    for (int j = (blockIdx.y * 256 + threadIdx.x) * 4; j < cols; j += gridDim.y * 1024) {
        float4 v = *reinterpret_cast<const float4*>(c + row * ldc + j);      // ldc holds the padding
        for (int k = 1; k < slices; ++k) {
            const float4 o = *reinterpret_cast<const float4*>(c + k * slice + row * ldc + j);
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        const uint32_t w[2] = {pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f)};
        uint16_t* dst = dx + row * lddx + j;
        if (vec && j + 4 <= cols) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
        else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < cols) dst[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
        }
    }
}

// A weight gradient of zeros (of an empty batch) into rows ld apart.
__global__ void __launch_bounds__(256) k_head_zero(uint16_t* dw, int64_t ld, int64_t rows, int cols) {
    pdl_wait();
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, (int64_t)gridDim.x * 256, cols);
    for (; at.row < rows; at.next()) dw[at.row * ld + at.part] = 0;
}

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

inline bool tma_rows(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

}  // namespace
}  // namespace nitro

#define TRY(expr)                                         \
    do {                                                  \
        if ((expr) != cudaSuccess) return NITRO_ERR_CUDA; \
    } while (0)
