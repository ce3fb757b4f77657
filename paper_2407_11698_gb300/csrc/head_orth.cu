// An update made orthogonal by Newton-Schulz steps: X0 = M / (|M|_F + 1e-7), then
//   A = X X^T,   X <- a X + (b A + c A^2) X
// (A = X^T X and X <- a X + X (b A + c A^2) where M has more rows than columns), which
// moves every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// The products run on k_head_gemm (head_gemm.cuh) in fp16 with 32-bit sums.  X, A and
// B = b A + c A^2 are kept times powers of two that put the largest value each can take
// below fp16's largest.  A value is two fp16 halves, v = high + low (22 bits and more),
// and a product of two such tensors is three, high high + high low + low high: a step
// multiplies what rounding adds outside M's own directions by a = 3.4 each, so an error
// of the first step is 3.4^4 = 140 times larger at the end, and with 11 bits a gradient
// of low rank (one batch's) comes out some per cent off.  Late steps need no low halves
// (orth_halves()).
//
// A and B are symmetric: only tiles that reach the diagonal or lie right of it are
// computed, and stored twice.
#include <cfloat>
#include <cmath>
#include <new>
#include <vector>

#include "head_gemm.cuh"

using namespace nitro;

namespace nitro {
namespace {

constexpr float kNormEps = 1e-7f;
constexpr int kNormCtas = 1024;     // partial sums of squares a matrix, at most

// v -> its high and low half
__device__ __forceinline__ void split_half(float v, __half* hi, __half* lo) {
    *hi = __float2half_rn(v);
    *lo = __float2half_rn(v - __half2float(*hi));
}
__device__ __forceinline__ uint32_t pack_half(__half a, __half b) {
    return (uint32_t)__half_as_ushort(a) | (uint32_t)__half_as_ushort(b) << 16;
}
// 32 floats as high (and low, if lo) halves at an 64-byte aligned place
__device__ __forceinline__ void store_halves(uint16_t* hi, uint16_t* lo, const float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            __half h0, h1, l0, l1;
            split_half(v[8 * j + 2 * k], &h0, &l0);
            split_half(v[8 * j + 2 * k + 1], &h1, &l1);
            h[k] = pack_half(h0, h1);
            l[k] = pack_half(l0, l1);
        }
        reinterpret_cast<uint4*>(hi)[j] = make_uint4(h[0], h[1], h[2], h[3]);
        if (lo) reinterpret_cast<uint4*>(lo)[j] = make_uint4(l[0], l[1], l[2], l[3]);
    }
}
// adds f times the 32 values held at hi (+ lo)
__device__ __forceinline__ void add_halves(const uint16_t* hi, const uint16_t* lo, float f, float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint4 h = reinterpret_cast<const uint4*>(hi)[j];
        const uint4 l = lo ? reinterpret_cast<const uint4*>(lo)[j] : make_uint4(0, 0, 0, 0);
        const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hw[k]));
            const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&lw[k]));
            v[8 * j + 2 * k] = fmaf(f, a.x + b.x, v[8 * j + 2 * k]);
            v[8 * j + 2 * k + 1] = fmaf(f, a.y + b.y, v[8 * j + 2 * k + 1]);
        }
    }
}

// Planes of a tensor of the batch: high at base + 2 b plane, low one plane further.
struct Planes {
    uint16_t* base;
    int64_t ld, plane;      // ld a multiple of 64
};

// The symmetric products.  A = f sum; B = f sum + g A with A's planes in `add`.  Elements
// right of the diagonal are stored at (row, col) and (col, row), the others left to them.
struct EpiSym {
    struct Args {
        Planes out, add;     // add.base may be null
        float f, fa;
        int low, low_add;    // whether out gets, and add has, low halves
        const float* scale;  // of the matrix's planes, or null (1): A takes its square
    };
    const Args& a;
    const HgArgs& g;
    int row, col0;
    uint16_t *hi, *lo;
    const uint16_t* add = nullptr;
    float f;
    __device__ __forceinline__ EpiSym(const Args& a_, const HgArgs& g_, const HgTile& t, int row_, int col0_, int)
        : a(a_), g(g_), row(row_), col0(col0_) {
        hi = a.out.base + 2 * t.batch * a.out.plane;
        lo = a.low ? hi + a.out.plane : nullptr;
        f = a.f;
        if (a.scale) f *= a.scale[t.batch] * a.scale[t.batch];
        if (a.add.base) add = a.add.base + 2 * t.batch * a.add.plane + (int64_t)row * a.add.ld;
    }
    __device__ __forceinline__ void cols(int c, float* v) {
        const int col = col0 + c;
        if (row >= g.M || col >= g.N || col + 31 < row) return;
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= f;
        if (add) add_halves(add + col, a.low_add ? add + a.add.plane + col : nullptr, a.fa, v);
        if (col > row) {
            // the padding of a row may be written
            uint16_t* h = hi + (int64_t)row * a.out.ld + col;
            store_halves(h, lo ? lo + (h - hi) : nullptr, v);
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const int cj = col + j;
            if (cj < row || cj >= g.N) continue;
            __half h, l;
            split_half(v[j], &h, &l);
            hi[(int64_t)cj * a.out.ld + row] = __half_as_ushort(h);
            if (lo) lo[(int64_t)cj * a.out.ld + row] = __half_as_ushort(l);
            if (col <= row) {
                hi[(int64_t)row * a.out.ld + cj] = __half_as_ushort(h);
                if (lo) lo[(int64_t)row * a.out.ld + cj] = __half_as_ushort(l);
            }
        }
    }
    __device__ __forceinline__ void done() {}
};

// X <- a X + f sum, as planes for the next step or, at the last one, in bf16.
struct EpiUpdate {
    struct Args {
        Planes x, out;
        float f, fx;         // times the sum, times X's planes
        int low_x, low;
        uint16_t* last;      // or null
        int64_t ld_last, stride_last;
        int vec;
        const float* scale;  // of the matrix's planes, or null: 1
    };
    const Args& a;
    const HgArgs& g;
    int row, col0, batch;
    float f, fx;
    __device__ __forceinline__ EpiUpdate(const Args& a_, const HgArgs& g_, const HgTile& t, int row_, int col0_, int)
        : a(a_), g(g_), row(row_), col0(col0_), batch(t.batch) {
        const float k = a.scale ? a.scale[batch] : 1.0f;
        f = a.f * k;
        fx = a.fx * k;
    }
    __device__ __forceinline__ void cols(int c, float* v) {
        const int col = col0 + c;
        if (row >= g.M || col >= g.N) return;
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= f;
        const uint16_t* x = a.x.base + 2 * batch * a.x.plane + (int64_t)row * a.x.ld + col;
        add_halves(x, a.low_x ? x + a.x.plane : nullptr, fx, v);
        if (!a.last) {
            uint16_t* o = a.out.base + 2 * batch * a.out.plane + (int64_t)row * a.out.ld + col;
            store_halves(o, a.low ? o + a.out.plane : nullptr, v);
            return;
        }
        uint16_t* o = a.last + batch * a.stride_last + (int64_t)row * a.ld_last + col;
        const int n = g.N - col;
        if (a.vec && n >= 32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(v[8 * j + 2 * k], v[8 * j + 2 * k + 1]);
                    w[k] = *reinterpret_cast<const uint32_t*>(&p);
                }
                reinterpret_cast<uint4*>(o)[j] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < n) o[j] = __bfloat16_as_ushort(__float2bfloat16_rn(v[j]));
        }
    }
    __device__ __forceinline__ void done() {}
};

// ------------------------------------------------------------------ norm and first planes
template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)v << 16);
    else if constexpr (sizeof(T) == 8) return (float)v * 0x1p-32f;   // squares of int64 gradients stay inside fp32
    else return v;
}
// 16 bytes of a row: E values, those past n zero
template <typename T>
struct Vec16 {
    static constexpr int E = 16 / (int)sizeof(T);
    union {
        uint4 w;
        T v[E];
    };
    __device__ __forceinline__ void load(const T* src, int n, bool vec) {
        if (vec && n >= E) {
            w = *reinterpret_cast<const uint4*>(src);
        } else {
            w = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j < n) v[j] = src[j];
        }
    }
};
constexpr int kOrthInFlight = 4;    // loads of a thread in flight

// Sum of squares of a matrix, a partial of each CTA (blockIdx.y: the matrix).
template <typename T>
__global__ void __launch_bounds__(256) k_orth_norm(const T* m, int64_t ld, int64_t stride, int rows, int cols, float* part,
                                                   int vec) {
    constexpr int E = Vec16<T>::E;
    __shared__ float sh[8];
    pdl_wait();
    const T* src = m + blockIdx.y * stride;
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, (int64_t)gridDim.x * 256, (cols + E - 1) / E);
    float s[kOrthInFlight] = {};
    while (at.row < rows) {
        Vec16<T> r[kOrthInFlight];
#pragma unroll
        for (int u = 0; u < kOrthInFlight; ++u) {
            r[u].load(src + at.row * ld + at.part * E, at.row < rows ? cols - at.part * E : 0, vec != 0);
            at.next();
        }
#pragma unroll
        for (int u = 0; u < kOrthInFlight; ++u)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float v = as_float(r[u].v[j]);
                s[u] = fmaf(v, v, s[u]);
            }
    }
    float t = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) t += sh[w];
        part[blockIdx.y * kNormCtas + blockIdx.x] = t;
    }
}

// X0 as planes (padding columns zero).  The planes hold M times the power of two that puts
// 1 / (|M| + eps) times mul between mul / 2 and mul; what is left of the factor, in (1/2, 1], goes
// to scale and is multiplied in by the first step's products.  So bf16 values keep their
// bits: their low halves are zero, and the first step leaves them out.
template <typename T>
__global__ void __launch_bounds__(256) k_orth_pack(const T* m, int64_t ld, int64_t stride, int rows, int cols,
                                                   const float* part, int parts, float mul, Planes out, int low, int vec, float* scale) {
    constexpr int E = Vec16<T>::E;
    __shared__ float sh[8];
    pdl_wait();
    float s = 0.0f;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[blockIdx.y * kNormCtas + i];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0f;
    for (int w = 0; w < 8; ++w) s += sh[w];
    // int64 values were taken times 2^-32, so is the 1e-7
    const float eps = sizeof(T) == 8 ? kNormEps * 0x1p-32f : kNormEps;
    const float full = 1.0f / (sqrtf(s) + eps);
    int e;
    const float left = frexpf(full, &e);      // in [1/2, 1); a norm that is not finite leaves 0 or NaN
    const float f = isfinite(full) && full > 0.0f ? ldexpf(mul, e) : mul * full;
    if (blockIdx.x == 0 && threadIdx.x == 0) scale[blockIdx.y] = isfinite(full) && full > 0.0f ? left : 1.0f;
    const T* src = m + blockIdx.y * stride;
    uint16_t* hi = out.base + 2 * blockIdx.y * out.plane;
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, (int64_t)gridDim.x * 256, (int)(out.ld / E));
    while (at.row < rows) {
        Vec16<T> r[kOrthInFlight];
        int64_t to[kOrthInFlight];
#pragma unroll
        for (int u = 0; u < kOrthInFlight; ++u) {
            to[u] = at.row < rows ? at.row * out.ld + at.part * E : -1;
            r[u].load(src + at.row * ld + at.part * E, at.row < rows ? cols - at.part * E : 0, vec != 0);
            at.next();
        }
#pragma unroll
        for (int u = 0; u < kOrthInFlight; ++u) {
            if (to[u] < 0) continue;
            uint32_t h[E / 2], l[E / 2];
#pragma unroll
            for (int j = 0; j < E / 2; ++j) {
                __half h0, h1, l0, l1;
                split_half(as_float(r[u].v[2 * j]) * f, &h0, &l0);
                split_half(as_float(r[u].v[2 * j + 1]) * f, &h1, &l1);
                h[j] = pack_half(h0, h1);
                l[j] = pack_half(l0, l1);
            }
            const auto put = [](uint16_t* p, const uint32_t* w) {
                if constexpr (E == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
                else if constexpr (E == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t*>(p) = w[0];
            };
            put(hi + to[u], h);
            if (low) put(hi + out.plane + to[u], l);
        }
    }
}

// steps = 0: M / (|M| + eps) itself.
__global__ void __launch_bounds__(256) k_orth_copy(Planes x, float mul, int low, const float* scale, int rows, int cols,
                                                   uint16_t* out, int64_t ld, int64_t stride) {
    pdl_wait();
    mul *= scale[blockIdx.y];
    const uint16_t* hi = x.base + 2 * blockIdx.y * x.plane;
    const int64_t n = (int64_t)rows * cols;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / cols, c = i - r * cols;
        const uint16_t* p = hi + r * x.ld + c;
        const float v = (__half2float(__ushort_as_half(p[0])) + (low ? __half2float(__ushort_as_half(p[x.plane])) : 0.0f)) * mul;
        out[blockIdx.y * stride + r * ld + c] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
    }
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

}  // namespace
}  // namespace nitro

struct nitro_orth {
    int max_count = 0, rows = 0, cols = 0, small = 0;   // small = min(rows, cols)
    Planes x[2], a, b;
    float* part = nullptr;
    float* scale = nullptr;    // [max_count], see k_orth_pack
    uint32_t* status = nullptr;
    std::vector<void*> allocs;
};

namespace {

template <typename T>
bool oalloc(nitro_orth* h, T** p, int64_t count) {
    void* q = nullptr;
    if (cudaMalloc(&q, (size_t)count * sizeof(T)) != cudaSuccess) return false;
    h->allocs.push_back(q);
    *p = static_cast<T*>(q);
    return true;
}

#define TRY(expr)                                         \
    do {                                                  \
        if ((expr) != cudaSuccess) return NITRO_ERR_CUDA; \
    } while (0)

// The power of two that puts `top` between 2^14 and 2^15.
float half_scale(double top) { return (float)std::ldexp(1.0, 15 - (int)std::ceil(std::log2(std::max(top, 1e-6)))); }

// The largest singular value that can occur before each step (from 1), and the largest
// |b s^2 + c s^4|; false where they leave the range that fp16 planes hold.
bool orth_range(const float* k, int steps, double* top, double* top_b) {
    double hi = 1.0, all = 1.0, bmax = 0.0;
    for (int i = 0; i < steps; ++i) {
        double next = 0.0;
        for (int j = 0; j <= 4096; ++j) {
            const double s = hi * j / 4096, s2 = s * s, p = k[1] * s2 + (double)k[2] * s2 * s2;
            next = std::max(next, std::fabs(s * (k[0] + p)));
            bmax = std::max(bmax, std::fabs(p));
        }
        if (i + 1 < steps) all = std::max(all, next);
        hi = next;
        if (!(hi <= 8.0) || !(bmax <= 1024.0)) return false;
    }
    // rounding moves a value past its bound a little
    *top = 1.01 * all;
    *top_b = 1.01 * bmax + 1e-3;
    return true;
}

// Whether step i of `steps` works with both halves.
bool orth_halves(int i, int steps) { return steps - i > 2; }

template <typename T>
nitro_status orth_first(nitro_orth* h, const T* m, int64_t ld, int64_t stride, int count, float mul, bool low, cudaStream_t s) {
    const int64_t n = (int64_t)h->rows * h->cols;
    constexpr int E = Vec16<T>::E;
    const int vec = ((uintptr_t)m & 15) == 0 && ld % E == 0 && (count == 1 || stride % E == 0);
    const int most = 8 * sm_count() / count + 1;
    const int parts = (int)std::min<int64_t>(std::min(kNormCtas, most), (n / E + 255) / 256 + 1);
    {
        ProfScope ps(K_ORTH_PACK, s, 0.0, (double)sizeof(T) * n * count);
        TRY(launch_k(k_orth_norm<T>, dim3(parts, count), dim3(256), 0, s, m, ld, stride, h->rows, h->cols, h->part, vec));
    }
    const int64_t items = h->rows * (h->x[0].ld / E);
    const int grid = (int)std::min<int64_t>((items + 255) / 256, most);
    ProfScope ps(K_ORTH_PACK, s, 0.0, (double)(sizeof(T) + (low ? 4 : 2)) * n * count);
    TRY(launch_k(k_orth_pack<T>, dim3(grid, count), dim3(256), 0, s, m, ld, stride, h->rows, h->cols, (const float*)h->part,
                 parts, mul, h->x[0], low ? 1 : 0, vec, h->scale));
    return NITRO_OK;
}

HgOperand operand(const Planes& p, int64_t inner, int64_t outer, int count) {
    return {p.base, inner, outer, p.ld, 2 * (int64_t)count, p.plane};
}

}  // namespace

extern "C" {

nitro_status nitro_orth_create(int max_count, int rows, int cols, nitro_orth** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (max_count < 1 || rows < 1 || cols < 1 || max_count > 4096 || rows > (1 << 18) || cols > (1 << 18) ||
        std::min(rows, cols) > (1 << 15) || (int64_t)max_count * rows * cols > ((int64_t)1 << 33))
        return NITRO_ERR_ARG;
    nitro_orth* h = new (std::nothrow) nitro_orth();
    if (!h) return NITRO_ERR_CUDA;
    h->max_count = max_count;
    h->rows = rows;
    h->cols = cols;
    h->small = std::min(rows, cols);
    for (Planes* p : {&h->x[0], &h->x[1]}) *p = {nullptr, round_up(cols, 64), rows * round_up(cols, 64)};
    for (Planes* p : {&h->a, &h->b}) *p = {nullptr, round_up(h->small, 64), h->small * round_up(h->small, 64)};
    bool ok = oalloc(h, &h->part, (int64_t)max_count * kNormCtas) && oalloc(h, &h->scale, max_count) && oalloc(h, &h->status, 1) &&
              cudaMemset(h->status, 0, 4) == cudaSuccess;
    for (Planes* p : {&h->x[0], &h->x[1], &h->a, &h->b}) ok = ok && oalloc(h, &p->base, 2 * max_count * p->plane);
    if (!ok) {
        nitro_orth_destroy(h);
        return NITRO_ERR_CUDA;
    }
    *out = h;
    return NITRO_OK;
}

nitro_status nitro_orth_run(nitro_orth* h, const void* m, int m_type, int64_t ldm, int64_t stride_m, int count, int steps,
                            const float* coef, uint16_t* out, int64_t ldo, int64_t stride_o, void* stream) {
    if (!h || count < 0 || count > h->max_count || steps < 0 || steps > 100 || ldm < h->cols || ldo < h->cols ||
        (m_type != NITRO_BF16 && m_type != NITRO_F32 && m_type != NITRO_I64))
        return NITRO_ERR_ARG;
    if (count > 1 && (stride_m < (h->rows - 1) * ldm + h->cols || stride_o < (h->rows - 1) * ldo + h->cols)) return NITRO_ERR_ARG;
    static const float kDefault[3] = {3.4445f, -4.7750f, 2.0315f};
    const float* k = coef ? coef : kDefault;
    double top, top_b;
    if (!orth_range(k, steps, &top, &top_b)) return NITRO_ERR_ARG;
    if (count == 0) return NITRO_OK;
    const uintptr_t size = m_type == NITRO_BF16 ? 2 : m_type == NITRO_F32 ? 4 : 8;
    if (!m || !out || ((uintptr_t)m & (size - 1)) || ((uintptr_t)out & 1)) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool tall = h->rows > h->cols;
    const int n = h->small;
    const int64_t big = std::max(h->rows, h->cols);
    const float sx = half_scale(top), sa = half_scale(top * top), sb = half_scale(top_b);
    const bool low0 = m_type != NITRO_BF16 && (steps == 0 || orth_halves(0, steps));
    nitro_status st;
    if (m_type == NITRO_BF16) st = orth_first(h, (const uint16_t*)m, ldm, stride_m, count, sx, low0, s);
    else if (m_type == NITRO_F32) st = orth_first(h, (const float*)m, ldm, stride_m, count, sx, low0, s);
    else st = orth_first(h, (const int64_t*)m, ldm, stride_m, count, sx, low0, s);
    if (st != NITRO_OK) return st;
    if (steps == 0) {
        const int grid = (int)std::min<int64_t>(((int64_t)h->rows * h->cols + 255) / 256, 8 * sm_count());
        ProfScope ps(K_ORTH_PACK, s, 0.0, 6.0 * count * h->rows * h->cols);
        TRY(launch_k(k_orth_copy, dim3(grid, count), dim3(256), 0, s, h->x[0], 1.0f / sx, (int)low0, (const float*)h->scale, h->rows, h->cols, out, ldo, stride_o));
        return NITRO_OK;
    }
    bool low_x = low0;
    for (int i = 0; i < steps; ++i) {
        const Planes& x = h->x[i & 1];
        const bool low = orth_halves(i, steps), low_next = i + 1 < steps && orth_halves(i + 1, steps);
        HgProblem p;
        p.batch = count;
        p.planes_a = p.planes_b = 2;
        p.status = h->status;
        const HgOperand ox = operand(x, h->cols, h->rows, count), oa = operand(h->a, n, n, count), ob = operand(h->b, n, n, count);
        // A.  A bf16 matrix is held exactly by the first step's high halves.
        p.M = p.N = n;
        p.K = big;
        p.upper = true;
        p.products = low_x ? 3 : 1;
        p.prof = K_ORTH_GRAM;
        p.ops = (double)count * n * n * big;
        const float* g0 = i == 0 ? h->scale : nullptr;
        const EpiSym::Args ga{h->a, {nullptr, 0, 0}, sa / (sx * sx), 0.0f, low, 0, g0};
        if (tall && low_x) TRY((hg_launch<EpiSym, true, true, true, 2, 2>(hg_pick(p), p, ox, ox, ga, s)));
        else if (tall) TRY((hg_launch<EpiSym, true, true, true>(hg_pick(p), p, ox, ox, ga, s)));
        else if (low_x) TRY((hg_launch<EpiSym, false, false, true, 2, 2>(hg_pick(p), p, ox, ox, ga, s)));
        else TRY((hg_launch<EpiSym, false, false, true>(hg_pick(p), p, ox, ox, ga, s)));
        // B = b A + c A^2
        p.K = n;
        p.products = low ? 3 : 1;
        p.prof = K_ORTH_SQUARE;
        p.ops = (double)count * n * n * n;
        const EpiSym::Args gb{h->b, h->a, k[2] * sb / (sa * sa), k[1] * sb / sa, low, low, nullptr};
        if (low) TRY((hg_launch<EpiSym, false, false, true, 2, 2>(hg_pick(p), p, oa, oa, gb, s)));
        else TRY((hg_launch<EpiSym, false, false, true>(hg_pick(p), p, oa, oa, gb, s)));
        // X
        p.M = h->rows;
        p.N = h->cols;
        p.upper = false;
        p.products = 1 + low + (low && low_x);
        p.prof = K_ORTH_UPDATE;
        p.ops = 2.0 * count * n * n * big;
        const bool last = i + 1 == steps;
        const float so = last ? 1.0f : sx;
        const EpiUpdate::Args gu{x, h->x[(i + 1) & 1], so / (sb * sx), k[0] * so / sx, low_x, low_next, last ? out : nullptr,
                                 ldo, stride_o, ((uintptr_t)out & 15) == 0 && ldo % 8 == 0 && (count == 1 || stride_o % 8 == 0), g0};
        const HgPick t = hg_pick(p);
        if (tall && low && low_x) TRY((hg_launch<EpiUpdate, false, false, true, 2, 2>(t, p, ox, ob, gu, s)));
        else if (tall && low) TRY((hg_launch<EpiUpdate, false, false, true, 1, 2>(t, p, ox, ob, gu, s)));
        else if (tall) TRY((hg_launch<EpiUpdate, false, false, true>(t, p, ox, ob, gu, s)));
        else if (low && low_x) TRY((hg_launch<EpiUpdate, false, true, true, 2, 2>(t, p, ob, ox, gu, s)));
        else if (low) TRY((hg_launch<EpiUpdate, false, true, true, 2, 1>(t, p, ob, ox, gu, s)));
        else TRY((hg_launch<EpiUpdate, false, true, true>(t, p, ob, ox, gu, s)));
        low_x = low_next;
    }
    return NITRO_OK;
}

nitro_status nitro_orth_status(nitro_orth* h, int clear) {
    if (!h) return NITRO_ERR_ARG;
    uint32_t bits = 0;
    if (cudaDeviceSynchronize() != cudaSuccess ||
        cudaMemcpy(&bits, h->status, 4, cudaMemcpyDeviceToHost) != cudaSuccess ||
        (clear && cudaMemset(h->status, 0, 4) != cudaSuccess))
        return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_orth_destroy(nitro_orth* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    for (void* p : h->allocs) cudaFree(p);
    delete h;
}

}  // extern "C"
