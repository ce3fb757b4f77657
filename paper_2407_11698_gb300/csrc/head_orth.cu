// An update made orthogonal by Newton-Schulz steps: X0 = M / (|M|_F + 1e-7), then
//   A = X X^T,   B = a I + b A + c A^2,   X <- B X
// (A = X^T X and X <- X B where M has more rows than columns), which
// moves every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// The products run on k_head_gemm (head_gemm.cuh) in fp16 with 32-bit sums.  X, A and
// B are kept times powers of two that put the largest value each can take
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

#include "head_gemm.cuh"

using namespace nitro;

namespace nitro {
namespace {

constexpr float kNormEps = 1e-7f;
constexpr int kNormCtas = 1024;     // partial sums of squares a matrix, at most

__device__ __forceinline__ float2 halves2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// two values -> a word of their high and a word of their low halves.  Pairs, since the
// conversion of two floats to a pair is one instruction at a higher rate than that of one.
__device__ __forceinline__ void split_pair(float a, float b, uint32_t* hi, uint32_t* lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 back = __half22float2(h);
    const __half2 l = __floats2half2_rn(a - back.x, b - back.y);
    *hi = *reinterpret_cast<const uint32_t*>(&h);
    *lo = *reinterpret_cast<const uint32_t*>(&l);
}
// 32 x 32 values of a warp held as halves, loaded ahead of their use (lines, see HgStage)
struct Halves32 {
    uint4 h[4], l[4];
    // valid rows of a matrix at column col; lo may be null
    __device__ __forceinline__ void load(const HgPart& p, const uint16_t* hi, const uint16_t* lo, int64_t ld, int col) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = p.row0 + p.stage.line_row(i);
            const int64_t at = (int64_t)row * ld + col + 8 * p.stage.line_chunk();
            h[i] = l[i] = make_uint4(0, 0, 0, 0);
            if (row >= p.rows) continue;
            h[i] = *reinterpret_cast<const uint4*>(hi + at);
            if (lo) l[i] = *reinterpret_cast<const uint4*>(lo + at);
        }
    }
    // v = g v + f times the thread's row
    __device__ __forceinline__ void join(const HgPart& p, bool low, float g, float f, float* v) {
        p.stage.to_mine(h);
        if (low) p.stage.to_mine(l);
        const uint32_t *hw = reinterpret_cast<const uint32_t*>(h), *lw = reinterpret_cast<const uint32_t*>(l);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float2 a = halves2(hw[j]), b = halves2(lw[j]);
            v[2 * j] = fmaf(f, a.x + b.x, v[2 * j] * g);
            v[2 * j + 1] = fmaf(f, a.y + b.y, v[2 * j + 1] * g);
        }
    }
};

// Planes of a tensor of the batch: high at base + 2 b plane, low one plane further.
struct Planes {
    uint16_t* base;
    int64_t ld, plane;      // ld a multiple of 64
};

// The symmetric products.  A = f sum; B = f sum + fa A + diag I with A's planes in `add`.  Blocks of
// 32 x 32 right of the diagonal are stored at (row, col) and (col, row).
struct EpiSym {
    static constexpr bool kFold = false, kTail = false;
    struct Args {
        Planes out, add;     // add.base may be null
        float f, fa, diag;   // diag: added on the diagonal
        int low, low_add;    // whether out gets, and add has, low halves
        const float* scale;  // of the matrix's planes, or null (1): A takes its square
    };
    const Args& a;
    const HgArgs& g;
    const HgPart& p;
    uint16_t *hi, *lo;
    const uint16_t* add = nullptr;
    float f;
    Halves32 old;
    __device__ __forceinline__ EpiSym(const Args& a_, const HgArgs& g_, const HgTile& t, const HgPart& p_) : a(a_), g(g_), p(p_) {
        hi = a.out.base + 2 * t.batch * a.out.plane;
        lo = a.low ? hi + a.out.plane : nullptr;
        f = a.f;
        if (a.scale) f *= a.scale[t.batch] * a.scale[t.batch];
        if (a.add.base) add = a.add.base + 2 * t.batch * a.add.plane;
    }
    // no column of the warp's rows is right of the diagonal
    __device__ __forceinline__ bool skip(int col) const { return col >= g.N || col + 31 < p.row0; }
    __device__ __forceinline__ void fetch(int c) {
        const int col = p.col0 + c;
        if (add && !skip(col)) old.load(p, add, a.low_add ? add + a.add.plane : nullptr, a.add.ld, col);
    }
    __device__ __forceinline__ void cols(int c, float* v) {
        const int col = p.col0 + c, row = p.row;
        const bool none = skip(col);
        if (!none) {
            if (add) old.join(p, a.low_add != 0, f, a.fa, v);
            else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= f;
            }
        }
        if (c + 32 < p.width) fetch(c + 32);
        if (none) return;
        if (col == p.row0) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += j == p.stage.lane ? a.diag : 0.0f;
        }
        uint32_t h[16], l[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) split_pair(v[2 * j], v[2 * j + 1], &h[j], &l[j]);
        hg_store16(p, h, hi, a.out.ld, col, (int)a.out.ld, true);     // paddings may be written
        if (lo) hg_store16(p, l, lo, a.out.ld, col, (int)a.out.ld, true);
        // a block on the diagonal (both start at multiples of 32) holds both of its halves
        if (col == p.row0) return;
        // and as columns, two rows a store: lanes 2i and 2i + 1 swap, one takes the even
        // columns, the other the odd
        const int odd = p.stage.lane & 1;
        const int64_t to = (int64_t)(col + odd) * a.out.ld + (row - odd);
        const auto mirror = [&](uint16_t* plane, const uint32_t* w) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t other = __shfl_xor_sync(0xffffffffu, w[j], 1);
                const uint32_t pair = odd ? __byte_perm(other, w[j], 0x7632) : __byte_perm(w[j], other, 0x5410);
                if (row - odd < p.rows && col + 2 * j + odd < g.N)
                    *reinterpret_cast<uint32_t*>(plane + to + 2 * j * a.out.ld) = pair;
            }
        };
        mirror(hi, h);
        if (lo) mirror(lo, l);
    }
    __device__ __forceinline__ void done() {}
};

// X <- f sum, as planes for the next step or, at the last one, in bf16.
struct EpiUpdate {
    static constexpr bool kFold = false, kTail = false;
    struct Args {
        Planes out;
        float f;
        int low;
        uint16_t* last;      // or null
        int64_t ld_last, stride_last;
        int vec;
        const float* scale;  // of the matrix's planes, or null: 1
    };
    const Args& a;
    const HgArgs& g;
    const HgPart& p;
    int batch;
    float f;
    __device__ __forceinline__ EpiUpdate(const Args& a_, const HgArgs& g_, const HgTile& t, const HgPart& p_)
        : a(a_), g(g_), p(p_), batch(t.batch) {
        f = a.scale ? a.f * a.scale[batch] : a.f;
    }
    __device__ __forceinline__ void fetch(int) {}
    __device__ __forceinline__ void cols(int c, float* v) {
        const int col = p.col0 + c;
        if (col >= g.N) return;
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= f;
        uint32_t h[16], l[16];
        if (!a.last) {
#pragma unroll
            for (int j = 0; j < 16; ++j) split_pair(v[2 * j], v[2 * j + 1], &h[j], &l[j]);
            uint16_t* o = a.out.base + 2 * batch * a.out.plane;      // a row's padding may be written
            hg_store16(p, h, o, a.out.ld, col, (int)a.out.ld, true);
            if (a.low) hg_store16(p, l, o + a.out.plane, a.out.ld, col, (int)a.out.ld, true);
            return;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const __nv_bfloat162 w = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            h[j] = *reinterpret_cast<const uint32_t*>(&w);
        }
        hg_store16(p, h, a.last + batch * a.stride_last, a.ld_last, col, g.N, a.vec != 0);
    }
    __device__ __forceinline__ void done() {}
};

// ------------------------------------------------------------------ norm and first planes
template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 2) {
        return __uint_as_float((uint32_t)v << 16);
    } else if constexpr (sizeof(T) == 8) {
        // times 2^-32: squares of int64 gradients stay inside fp32.  By pieces of 16 bits, since the
        // conversion instruction is slow (the norm of eight 256 x 2304: 15 us): 2^23 + piece is a
        // float with the piece for its low bits; the top piece is taken as 2^15 more than it is.
        const uint32_t lo = (uint32_t)v, hi = (uint32_t)((uint64_t)v >> 32) ^ 0x80000000u;
        const auto piece = [](uint32_t w, uint32_t sel) { return __uint_as_float(__byte_perm(w, 0x4B000000u, sel)); };
        float f = fmaf(piece(hi, 0x7632) - (8388608.0f + 32768.0f), 65536.0f, piece(hi, 0x7610) - 8388608.0f);
        f = fmaf(piece(lo, 0x7632) - 8388608.0f, 0x1p-16f, f);
        return fmaf(piece(lo, 0x7610) - 8388608.0f, 0x1p-32f, f);
    } else {
        return v;
    }
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

// Squares of fp32 and bf16 values from 1.8e19 on do not fit 32 bits.  Where their sum is not finite, that of
// the values times 2^-96 is taken: 2^33 squares of the largest then sum up to 2^97, and where a sum has passed 2^128 the
// values that count are above 2^47.  (The sum of values that are not finite stays so; int64 values
// are scaled anyway.)
constexpr float kFar = 0x1p-96f;
constexpr int kFarBits = 96;
__device__ __forceinline__ bool is_far(float s) { return !(s <= FLT_MAX); }

// 1 / (norm + eps) as left 2^e, left in [1/2, 1), from the sum of squares s (far: of the values times kFar); false
// where that is not finite or zero: left is then 1 and *whole the factor itself.
template <typename T>
__device__ __forceinline__ bool norm_inverse(float s, bool far, float* left, int* e, float* whole) {
    // int64 values were taken times 2^-32, so is the 1e-7; beside far values it is nothing
    const float eps = far ? 0.0f : sizeof(T) == 8 ? kNormEps * 0x1p-32f : kNormEps;
    const float full = 1.0f / (sqrtf(s) + eps);
    *left = frexpf(full, e);
    *e -= far ? kFarBits : 0;
    *whole = full;
    if (isfinite(full) && full > 0.0f) return true;
    *left = 1.0f;
    return false;
}

// Sum of squares of a matrix, a partial of each CTA (blockIdx.y: the matrix): x that of the values, y of them
// times kFar, for which a CTA whose sum is not finite goes through its values again.
template <typename T>
__global__ void __launch_bounds__(256) k_orth_norm(const T* m, int64_t ld, int64_t stride, int rows, int cols, float2* part,
                                                   int vec) {
    constexpr int E = Vec16<T>::E;
    __shared__ float sh[2][8];
    pdl_wait();
    const T* src = m + blockIdx.y * stride;
    // the CTA's sum of the squares of values times f, in every thread
    const auto sum = [&](float f, float* warps) {
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
                    const float v = as_float(r[u].v[j]) * f;
                    s[u] = fmaf(v, v, s[u]);
                }
        }
        float t = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
        if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = t;
        __syncthreads();
        t = warps[0];
        for (int w = 1; w < 8; ++w) t += warps[w];
        return t;
    };
    float2 t;
    t.x = sum(1.0f, sh[0]);
    t.y = t.x * kFar * kFar;
    if (sizeof(T) < 8 && is_far(t.x)) t.y = sum(kFar, sh[1]);
    if (threadIdx.x == 0) part[blockIdx.y * kNormCtas + blockIdx.x] = t;
}

// X0 as planes (padding columns zero).  The planes hold M times the power of two that puts
// 1 / (|M| + eps) times mul between mul / 2 and mul; what is left of the factor, in (1/2, 1], goes
// to scale and is multiplied in by the first step's products.  So bf16 values keep their
// bits: their low halves are zero, and the first step leaves them out.
template <typename T>
__global__ void __launch_bounds__(256) k_orth_pack(const T* m, int64_t ld, int64_t stride, int rows, int cols,
                                                   const float2* part, int parts, float mul, Planes out, int low, int vec, float* scale) {
    constexpr int E = Vec16<T>::E;
    __shared__ float2 sh[8];
    pdl_wait();
    float2 s = make_float2(0.0f, 0.0f);
    for (int i = threadIdx.x; i < parts; i += 256) {
        const float2 o = part[blockIdx.y * kNormCtas + i];
        s.x += o.x, s.y += o.y;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s.x += __shfl_xor_sync(0xffffffffu, s.x, d), s.y += __shfl_xor_sync(0xffffffffu, s.y, d);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    s = make_float2(0.0f, 0.0f);
    for (int w = 0; w < 8; ++w) s.x += sh[w].x, s.y += sh[w].y;
    const bool far = sizeof(T) < 8 && is_far(s.x);
    int e;
    float left, full;
    const float f = norm_inverse<T>(far ? s.y : s.x, far, &left, &e, &full) ? ldexpf(mul, e) : mul * full;
    if (blockIdx.x == 0 && threadIdx.x == 0) scale[blockIdx.y] = left;
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
            for (int j = 0; j < E / 2; ++j)
                split_pair(as_float(r[u].v[2 * j]) * f, as_float(r[u].v[2 * j + 1]) * f, &h[j], &l[j]);
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

// ------------------------------------------------------------------ small matrices
// All steps in one launch for matrices whose shorter side m is at most 128: a cluster of
// C CTAs holds X (m x n, the transpose of a tall matrix) in shared memory, n / C columns each,
// as the 64-column blocks of 128-byte rows that the MMAs read along K (A = X X^T) and
// across it (B X) alike.  Every CTA has all of A and B.  A step is three batches of MMAs,
// each followed by its sums' way through the registers into the next one's operands; for
// C > 1 the parts of A meet by column slices in distributed shared memory, are added in the
// CTAs' order, and go back to all.  Bound by the latency of that chain: 50 x 100 takes 29 us,
// 1.9 a batch (the same by k_head_gemm, 17 launches, 107), 128 x 256 50, and with the
// exchange 128 x 1024 95.
// A wait that gives up latches TIMEOUT; the CTA then goes through the rest without waiting, so
// that the cluster's barriers and stores stay matched.
constexpr int kOsThreads = 512;      // four warps a TMEM lane quadrant, a quarter of the columns each

struct OsArgs {
    const void* m;
    int64_t ld, stride;
    uint16_t* out;
    int64_t ld_out, stride_out;
    int rows, cols;          // of M
    int tall;
    int mp;                  // m rounded up to 32
    int nb;                  // blocks of 64 columns a CTA holds
    int steps;
    int exact_first;         // X0's low halves are zero
    int vec, vec_out;        // rows of M and of the result are 16-byte aligned
    float mul, fa, fs, fsa, diag, fu, fu_last;
    uint32_t* status;
};

// byte offset of 16-byte chunk j of row r in a block of 128-byte rows (128-byte swizzle)
__device__ __forceinline__ uint32_t sw_chunk(int r, int j) { return (uint32_t)(r * 128 + ((j ^ (r & 7)) << 4)); }

template <typename T, int C>
__global__ void __launch_bounds__(kOsThreads, 1) k_orth_small(const OsArgs a) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int sb = (a.mp + 63) / 64;                     // blocks of A and B
    uint8_t* xh = smem;                                  // [nb] blocks of 16 KB, then their low halves
    uint8_t* xl = xh + a.nb * 16384;
    uint8_t* sh = xl + a.nb * 16384;                     // A, then B
    uint8_t* sl = sh + sb * 16384;
    uint8_t* tail = sl + sb * 16384;
    uint64_t* bar = reinterpret_cast<uint64_t*>(tail);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float2* parts = reinterpret_cast<float2*>(tail + 64);  // [16] warps, then [8] CTAs
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = C > 1 ? (int)cluster_rank() : 0;
    const int64_t mat = blockIdx.x / C;
    const int m = a.tall ? a.cols : a.rows, n = a.tall ? a.rows : a.cols;
    const int c0 = rank * a.nb * 64;                     // this CTA's first column of X
    const int nc = max(0, min(a.nb * 64, n - c0));
    const uint32_t bar_a = smem_u32(bar);
    if (tid == 0) {
        mbar_init(bar_a, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) hg_tmem_alloc<1>(smem_u32(tmem_slot), 512);
    for (int i = tid; i < a.nb * 2048; i += kOsThreads) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    // ---------------- norm and first planes
    // 16 bytes of M at a time; until the norm is known, the bits of a value (fp32) wait in its
    // places in the two planes
    constexpr int E = Vec16<T>::E;
    const T* src = static_cast<const T*>(a.m) + mat * a.stride + (a.tall ? c0 * a.ld : c0);
    const int len = a.tall ? m : nc, lines = a.tall ? nc : m;      // of this CTA's slice as it lies in memory
    float s = 0.0f, sf = 0.0f;       // sums of squares, of the values and of them times kFar
    if (len > 0) {
        RowWalk at(tid, kOsThreads, (len + E - 1) / E);
        while (at.row < lines) {
            constexpr int U = 4;
            Vec16<T> v[U];
            int line[U], pos[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                line[u] = at.row < lines ? (int)at.row : -1;
                pos[u] = at.part * E;
                v[u].load(src + at.row * a.ld + at.part * E, at.row < lines ? len - at.part * E : 0, a.vec != 0);
                at.next();
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (line[u] < 0) continue;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    if (pos[u] + j >= len) continue;
                    const float f = as_float(v[u].v[j]);
                    s = fmaf(f, f, s);
                    if (sizeof(T) < 8) sf = fmaf(f * kFar, f * kFar, sf);
                    const int r = a.tall ? pos[u] + j : line[u], c = a.tall ? line[u] : pos[u] + j;
                    const uint32_t o = (uint32_t)(c >> 6) * 16384 + sw_chunk(r, (c & 63) >> 3) + (c & 7) * 2;
                    *reinterpret_cast<uint16_t*>(xh + o) = (uint16_t)(__float_as_uint(f) >> 16);
                    *reinterpret_cast<uint16_t*>(xl + o) = (uint16_t)__float_as_uint(f);
                }
            }
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, d);
        if (sizeof(T) < 8) sf += __shfl_xor_sync(0xffffffffu, sf, d);
    }
    if (lane == 0) parts[warp] = make_float2(s, sf);
    __syncthreads();
    s = sf = 0.0f;
    for (int w = 0; w < 16; ++w) s += parts[w].x, sf += parts[w].y;
    if constexpr (C > 1) {
        cluster_barrier();       // every CTA of the cluster runs
        if (tid < C) {
            const uint32_t to = remote_smem(smem_u32(parts + 16 + rank), (uint32_t)tid);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(s), "f"(sf) : "memory");
        }
        cluster_barrier();
        s = sf = 0.0f;
        for (int r = 0; r < C; ++r) s += parts[16 + r].x, sf += parts[16 + r].y;
    }
    const bool far = sizeof(T) < 8 && is_far(s);
    int e;
    float left, full;            // see k_orth_pack
    const float f0 = norm_inverse<T>(far ? sf : s, far, &left, &e, &full) ? ldexpf(a.mul, e) : a.mul * full;
    for (int i = tid; i < a.nb * 1024; i += kOsThreads) {
        const uint4 hv = reinterpret_cast<const uint4*>(xh)[i], lv = reinterpret_cast<const uint4*>(xl)[i];
        const uint32_t hr[4] = {hv.x, hv.y, hv.z, hv.w}, lr[4] = {lv.x, lv.y, lv.z, lv.w};
        uint32_t hw[4], lw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            split_pair(__uint_as_float(__byte_perm(lr[j], hr[j], 0x5410)) * f0, __uint_as_float(__byte_perm(lr[j], hr[j], 0x7632)) * f0,
                       &hw[j], &lw[j]);
        reinterpret_cast<uint4*>(xh)[i] = make_uint4(hw[0], hw[1], hw[2], hw[3]);
        reinterpret_cast<uint4*>(xl)[i] = make_uint4(lw[0], lw[1], lw[2], lw[3]);
    }

    // ---------------- steps
    const int q = warp & 3, half = warp >> 2, row = q * 32 + lane;
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const uint32_t d_a = tmem, d_s = tmem + 128, d_u = tmem + 256;
    uint32_t phase = 0;
    bool dead = false;
    // operands are in shared memory: the MMAs of a batch, and their end
    const auto batch = [&](auto issue) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncthreads();
        if (tid == 0 && !*abort_flag) {
            tc_fence_after();
            issue();
            umma_commit(bar_a);
        }
        __syncwarp();
        dead = dead || !mbar_wait(bar_a, phase, abort_flag, a.status);
        dead = __any_sync(0xffffffffu, dead);
        phase ^= 1u;
        tc_fence_after();
    };
    // high high, high low and low high products of two operands whose low halves lie lo_a and lo_b bytes on
    const auto products = [&](uint32_t d, uint64_t da, uint64_t db, uint32_t lo_a, uint32_t lo_b, bool with_lo_a, bool with_lo_b,
                              uint32_t idesc, int ks, auto step_a, auto step_b) {
        uint32_t acc = 0;
        for (int h = 0; h < 3; ++h) {
            if ((h == 1 && !with_lo_b) || (h == 2 && !with_lo_a)) continue;
            const uint64_t pa = da + (h == 2 ? lo_a >> 4 : 0), pb = db + (h == 1 ? lo_b >> 4 : 0);
            for (int k = 0; k < ks; ++k) {
                umma_bf16(d, pa + step_a(k), pb + step_b(k), idesc, acc);
                acc = 1;
            }
        }
    };
    const auto along = [](int k) { return (uint64_t)((k >> 2) * (16384 >> 4) + (k & 3) * (32 >> 4)); };
    const auto across = [](int k) { return (uint64_t)(k * (2048 >> 4)); };
    const uint32_t id_s = hg_idesc(true, 128, a.mp, false, false), id_u = hg_idesc(true, 128, a.nb * 64, false, true);
    const int ks_x = max(1, (nc + 15) / 16);
    const uint32_t xh_a = smem_u32(xh), sh_a = smem_u32(sh);
    const uint32_t x_lo = (uint32_t)a.nb * 16384, s_lo = (uint32_t)sb * 16384;
    const int s0 = half * (a.mp / 4), s1 = s0 + a.mp / 4;        // this thread's columns of A and B,
    const int u0 = half * (a.nb * 16), u1 = u0 + a.nb * 16;      // and of X
    // body(column, eight sums) over a thread's columns, 32 of them loaded together
    const auto columns = [&](uint32_t d, int from, int to, auto body) {
        for (int c = from; c < to; c += 32) {
            uint32_t v[4][8];
            __syncwarp();
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + 8 * u < to) tmem_ld8_nowait(d + lanes + c + 8 * u, v[u]);
            tmem_wait_ld<8>(v[0]);
            reg_touch8(v[1]);
            reg_touch8(v[2]);
            reg_touch8(v[3]);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c + 8 * u < to) body(c + 8 * u, v[u]);
        }
    };

    for (int i = 0; i < a.steps; ++i) {
        const bool low = a.steps - i > 2, low_next = a.steps - i > 3, low_x = low && !(i == 0 && a.exact_first);
        const float k0 = i == 0 ? left : 1.0f;
        // A = X X^T
        batch([&] { products(d_a, desc_sw128(xh_a), desc_sw128(xh_a), x_lo, x_lo, low_x, low_x, id_s, ks_x, along, along); });
        const float fa = a.fa * k0 * k0;
        if constexpr (C == 1) {
            columns(d_a, s0, s1, [&](int c, const uint32_t* v) {
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    split_pair(__uint_as_float(v[2 * j]) * fa, __uint_as_float(v[2 * j + 1]) * fa, &hw[j], &lw[j]);
                const uint32_t o = (uint32_t)(c >> 6) * 16384 + sw_chunk(row, (c & 63) >> 3);
                *reinterpret_cast<uint4*>(sh + o) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
                if (low) *reinterpret_cast<uint4*>(sl + o) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
            });
        } else {
            // slices of cw columns: [source][four columns][row] where A and B lie, free until then
            const int cw = a.mp / C, quads = cw / 4;
            const uint32_t stage = smem_u32(sh);
            cluster_barrier();               // no CTA's MMAs read its B any more
            columns(d_a, s0, s1, [&](int c, const uint32_t* v) {
                if (row >= a.mp) return;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = c + 4 * j, to = col / cw;
                    st_remote4(remote_smem(stage + (uint32_t)(((rank * quads + (col - to * cw) / 4) * 128 + row) * 16), (uint32_t)to), v[4 * j],
                               v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
            });
            cluster_barrier();
            constexpr int U = 8 / C;         // 128 rows x 32 / C quads of columns at most
            float4 mine[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int idx = tid + u * kOsThreads, r = idx & 127, qd = idx >> 7;
                mine[u] = make_float4(0, 0, 0, 0);
                if (qd >= quads || r >= a.mp) continue;
                for (int k = 0; k < C; ++k) {
                    const float4 o = reinterpret_cast<const float4*>(sh)[(k * quads + qd) * 128 + r];
                    mine[u].x += o.x, mine[u].y += o.y, mine[u].z += o.z, mine[u].w += o.w;
                }
            }
            cluster_barrier();               // every slice is read
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int idx = tid + u * kOsThreads, r = idx & 127, qd = idx >> 7, col = rank * cw + qd * 4;
                if (qd >= quads || r >= a.mp) continue;
                uint32_t hw[2], lw[2];
                split_pair(mine[u].x * fa, mine[u].y * fa, &hw[0], &lw[0]);
                split_pair(mine[u].z * fa, mine[u].w * fa, &hw[1], &lw[1]);
                const uint32_t o = (uint32_t)(col >> 6) * 16384 + sw_chunk(r, (col & 63) >> 3) + (col & 7) * 2;
#pragma unroll
                for (int k = 0; k < C; ++k) {
                    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(remote_smem(sh_a + o, (uint32_t)k)),
                                 "r"(hw[0]), "r"(hw[1])
                                 : "memory");
                    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(remote_smem(sh_a + s_lo + o, (uint32_t)k)),
                                 "r"(lw[0]), "r"(lw[1])
                                 : "memory");
                }
            }
            asm volatile("fence.proxy.async;" ::: "memory");
            cluster_barrier();
        }
        // B = a I + b A + c A^2
        batch([&] { products(d_s, desc_sw128(sh_a), desc_sw128(sh_a), s_lo, s_lo, low, low, id_s, a.mp / 16, along, along); });
        columns(d_s, s0, s1, [&](int c, const uint32_t* v) {
            const uint32_t o = (uint32_t)(c >> 6) * 16384 + sw_chunk(row, (c & 63) >> 3);
            const uint4 hv = *reinterpret_cast<const uint4*>(sh + o);
            const uint4 lv = low ? *reinterpret_cast<const uint4*>(sl + o) : make_uint4(0, 0, 0, 0);
            const uint32_t hr[4] = {hv.x, hv.y, hv.z, hv.w}, lr[4] = {lv.x, lv.y, lv.z, lv.w};
            uint32_t hw[4], lw[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = halves2(hr[j]), y = halves2(lr[j]);
                const int at = row - c - 2 * j;
                split_pair(fmaf(a.fsa, x.x + y.x, __uint_as_float(v[2 * j]) * a.fs) + (at == 0 ? a.diag : 0.0f),
                           fmaf(a.fsa, x.y + y.y, __uint_as_float(v[2 * j + 1]) * a.fs) + (at == 1 ? a.diag : 0.0f), &hw[j], &lw[j]);
            }
            *reinterpret_cast<uint4*>(sh + o) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
            if (low) *reinterpret_cast<uint4*>(sl + o) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
        });
        // X = B X
        batch([&] {
            products(d_u, desc_sw128(sh_a), desc_sw128_mn(xh_a, 16384), s_lo, x_lo, low, low_x, id_u, a.mp / 16, along, across);
        });
        const bool last = i + 1 == a.steps;
        const float fu = (last ? a.fu_last : a.fu) * k0;
        columns(d_u, u0, u1, [&](int c, const uint32_t* v) {
            if (row >= m || c >= nc) return;
            const uint32_t o = (uint32_t)(c >> 6) * 16384 + sw_chunk(row, (c & 63) >> 3);
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(v[j]) * fu;
            if (!last) {
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) split_pair(f[2 * j], f[2 * j + 1], &hw[j], &lw[j]);
                *reinterpret_cast<uint4*>(xh + o) = make_uint4(hw[0], hw[1], hw[2], hw[3]);
                if (low_next) *reinterpret_cast<uint4*>(xl + o) = make_uint4(lw[0], lw[1], lw[2], lw[3]);
                return;
            }
            uint32_t w[4];      // the result, where X's high halves were
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
                w[j] = *reinterpret_cast<const uint32_t*>(&p);
            }
            *reinterpret_cast<uint4*>(xh + o) = make_uint4(w[0], w[1], w[2], w[3]);
        });
    }
    // ---------------- result: lanes along the rows of memory
    __syncthreads();
    uint16_t* dst = a.out + mat * a.stride_out + (a.tall ? c0 * a.ld_out : c0);
    const auto at_x = [&](int r, int c) { return (uint32_t)(c >> 6) * 16384 + sw_chunk(r, (c & 63) >> 3) + (c & 7) * 2; };
    if (len > 0 && !a.tall && a.vec_out) {
        const int per = (nc + 7) / 8;
        RowWalk at(tid, kOsThreads, per);
        for (; at.row < m; at.next()) {
            const int r = (int)at.row, c = at.part * 8;
            const uint4 w = *reinterpret_cast<const uint4*>(xh + at_x(r, c));
            uint16_t* p = dst + r * a.ld_out + c;
            if (c + 8 <= nc) {
                *reinterpret_cast<uint4*>(p) = w;
            } else {
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < nc) p[j] = (uint16_t)(u[j >> 1] >> (16 * (j & 1)));
            }
        }
    } else if (len > 0) {
        RowWalk at(tid, kOsThreads, len);
        for (; at.row < lines; at.next()) {
            const int r = a.tall ? at.part : (int)at.row, c = a.tall ? (int)at.row : at.part;
            dst[at.row * a.ld_out + at.part] = *reinterpret_cast<const uint16_t*>(xh + at_x(r, c));
        }
    }
    if (dead && tid == 0) {      // MMAs in flight end before TMEM is freed
        umma_commit(bar_a);
        mbar_drain(bar_a, phase, kDrainNs);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if constexpr (C > 1) cluster_barrier();
    if (warp == 0) {
        tc_fence_after();
        hg_tmem_free<1>(tmem, 512);
    }
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

}  // namespace
}  // namespace nitro

struct nitro_orth {
    int max_count = 0, rows = 0, cols = 0, small = 0;   // small = min(rows, cols)
    Planes x[2], a, b;
    float2* part = nullptr;    // [max_count][kNormCtas], see k_orth_norm
    float* scale = nullptr;    // [max_count], see k_orth_pack
    StatusWord status;
    DeviceAllocs allocs;
};

namespace {

#define TRY(expr)                                         \
    do {                                                  \
        if ((expr) != cudaSuccess) return NITRO_ERR_CUDA; \
    } while (0)

// The power of two that puts `top` between 2^14 and 2^15.
float half_scale(double top) { return (float)std::ldexp(1.0, 15 - (int)std::ceil(std::log2(std::max(top, 1e-6)))); }

// The largest singular value that can occur before each step (from 1), and the largest
// |a + b s^2 + c s^4|; false where they leave the range that fp16 planes hold.
bool orth_range(const float* k, int steps, double* top, double* top_b) {
    double hi = 1.0, all = 1.0, bmax = 0.0;
    const double a = k[0], b = k[1], c = k[2];
    const auto p = [=](double s2) { return a + b * s2 + c * s2 * s2; };
    if (!(std::fabs(a) < 1e6 && std::fabs(b) < 1e6 && std::fabs(c) < 1e6)) return false;
    for (int i = 0; i < steps; ++i) {
        // s (a + b s^2 + c s^4) and a + b s^2 + c s^4 on [0, hi]: at its ends and where they turn
        const double end = hi * hi, disc = 9 * b * b - 20 * a * c;
        double at[5] = {end, -1, -1, -1, 0};
        if (c != 0) at[3] = -b / (2 * c);
        if (c != 0 && disc >= 0) {
            at[1] = (-3 * b + std::sqrt(disc)) / (10 * c);
            at[2] = (-3 * b - std::sqrt(disc)) / (10 * c);
        } else if (c == 0 && b != 0) {
            at[1] = -a / (3 * b);
        }
        double next = 0.0;
        for (const double s2 : at) {
            if (!(s2 >= 0 && s2 <= end)) continue;
            next = std::max(next, std::sqrt(s2) * std::fabs(p(s2)));
            bmax = std::max(bmax, std::fabs(p(s2)));
        }
        if (i + 1 < steps) all = std::max(all, next);
        hi = next;
        if (!(hi <= 8.0) || !(bmax <= 1024.0)) return false;
    }
    // rounding moves a value past its bound a little
    *top = 1.01 * all;
    *top_b = 1.01 * bmax;
    return true;
}

// Whether step i of `steps` works with both halves.
bool orth_halves(int i, int steps) { return steps - i > 2; }

template <typename T>
nitro_status orth_first(nitro_orth* h, const T* m, int64_t ld, int64_t stride, int count, float mul, bool low, cudaStream_t s) {
    const int64_t n = (int64_t)h->rows * h->cols;
    constexpr int E = Vec16<T>::E;
    const int vec = ((uintptr_t)m & 15) == 0 && ld % E == 0 && (count == 1 || stride % E == 0);
    static std::atomic<int> resident[2];
    const int64_t items = h->rows * (h->x[0].ld / E);
    // one wave for all matrices together
    const auto share = [count](int grid) { return std::max(1, grid / count); };
    const int parts = std::min(kNormCtas, share(one_wave(k_orth_norm<T>, resident[0], (items + 3) / 4 * count)));
    {
        ProfScope ps(K_ORTH_PACK, s, 0.0, (double)sizeof(T) * n * count);
        TRY(launch_k(k_orth_norm<T>, dim3(parts, count), dim3(256), 0, s, m, ld, stride, h->rows, h->cols, h->part, vec));
    }
    const int grid = share(one_wave(k_orth_pack<T>, resident[1], (items + 3) / 4 * count));
    ProfScope ps(K_ORTH_PACK, s, 0.0, (double)(sizeof(T) + (low ? 4 : 2)) * n * count);
    TRY(launch_k(k_orth_pack<T>, dim3(grid, count), dim3(256), 0, s, m, ld, stride, h->rows, h->cols, (const float2*)h->part,
                 parts, mul, h->x[0], low ? 1 : 0, vec, h->scale));
    return NITRO_OK;
}

// The one-launch form: its cluster size, or 0 where it does not apply.  Up to 256 columns a
// CTA (128 KB of halves).  The exchange grows with the square of the shorter side: by eight
// CTAs a side above 64 is as slow as by launches (128 x 2048 133 us, 128 x 2500 by launches 127;
// 64 x 2048 64 us).
int small_cluster(const nitro_orth* h) {
    if (h->small > 128) return 0;
    const int big = std::max(h->rows, h->cols);
    for (int c = 1; c <= 8; c *= 2)
        if (big <= 256 * c) return c == 8 && h->small > 64 ? 0 : c;
    return 0;
}

template <typename T, int C>
cudaError_t small_launch(const OsArgs& a, int count, cudaStream_t s) {
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    sm_count(&dev);
    const int sb = (a.mp + 63) / 64;
    const size_t smem = (size_t)(2 * a.nb + 2 * sb) * 16384 + 1024 + 256;
    const cudaError_t e = once_per_device(ready, dev, [] {
        return cudaFuncSetAttribute(k_orth_small<T, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, 12 * 16384 + 1280);
    });
    if (e != cudaSuccess) return e;
    if constexpr (C > 1) return launch_cluster(k_orth_small<T, C>, dim3((unsigned)count * C), kOsThreads, C, s, smem, a);
    else return launch_k(k_orth_small<T, C>, dim3((unsigned)count), dim3(kOsThreads), smem, s, a);
}

template <typename T>
cudaError_t small_run(int c, OsArgs a, int count, cudaStream_t s) {
    const int m = std::min(a.rows, a.cols), n = std::max(a.rows, a.cols);
    a.mp = (int)round_up(m, 32);
    a.nb = (n + 64 * c - 1) / (64 * c);
    switch (c) {
        case 1: return small_launch<T, 1>(a, count, s);
        case 2: return small_launch<T, 2>(a, count, s);
        case 4: return small_launch<T, 4>(a, count, s);
        default: return small_launch<T, 8>(a, count, s);
    }
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
    bool ok = h->allocs.take(&h->part, (int64_t)max_count * kNormCtas) && h->allocs.take(&h->scale, max_count) && h->status.take();
    for (Planes* p : {&h->x[0], &h->x[1], &h->a, &h->b}) ok = ok && h->allocs.take(&p->base, 2 * max_count * p->plane);
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
    if (const int c = steps > 0 ? small_cluster(h) : 0) {
        const OsArgs a{m, ldm, stride_m, out, ldo, stride_o, h->rows, h->cols, tall, 0, 0, steps, m_type == NITRO_BF16,
                       ((uintptr_t)m & 15) == 0 && ldm * size % 16 == 0 && stride_m * size % 16 == 0,
                       ((uintptr_t)out & 15) == 0 && ldo % 8 == 0 && stride_o % 8 == 0, sx,
                       sa / (sx * sx), k[2] * sb / (sa * sa), k[1] * sb / sa, k[0] * sb, 1.0f / sb,
                       1.0f / (sb * sx), h->status.at};
        ProfScope ps(K_ORTH_SMALL, s, (double)count * steps * n * n * (3.0 * big + n), (double)count * n * big * (size + 2));
        TRY(m_type == NITRO_BF16 ? small_run<uint16_t>(c, a, count, s)
            : m_type == NITRO_F32 ? small_run<float>(c, a, count, s) : small_run<int64_t>(c, a, count, s));
        return NITRO_OK;
    }
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
        p.status = h->status.at;
        const HgOperand ox = operand(x, h->cols, h->rows, count), oa = operand(h->a, n, n, count), ob = operand(h->b, n, n, count);
        // A.  A bf16 matrix is held exactly by the first step's high halves.
        p.M = p.N = n;
        p.K = big;
        p.upper = true;
        const HgPick tg = low_x ? hg_pick(p, 2, 2) : hg_pick(p);
        p.prof = K_ORTH_GRAM;
        p.ops = (double)count * n * n * big;
        const float* g0 = i == 0 ? h->scale : nullptr;
        const EpiSym::Args ga{h->a, {nullptr, 0, 0}, sa / (sx * sx), 0.0f, 0.0f, low, 0, g0};
        if (tall && low_x) TRY((hg_launch<EpiSym, true, true, true, 2, 2>(tg, p, ox, ox, ga, s)));
        else if (tall) TRY((hg_launch<EpiSym, true, true, true>(tg, p, ox, ox, ga, s)));
        else if (low_x) TRY((hg_launch<EpiSym, false, false, true, 2, 2>(tg, p, ox, ox, ga, s)));
        else TRY((hg_launch<EpiSym, false, false, true>(tg, p, ox, ox, ga, s)));
        // B = a I + b A + c A^2
        p.K = n;
        p.prof = K_ORTH_SQUARE;
        p.ops = (double)count * n * n * n;
        const EpiSym::Args gb{h->b, h->a, k[2] * sb / (sa * sa), k[1] * sb / sa, k[0] * sb, low, low, nullptr};
        if (low) TRY((hg_launch<EpiSym, false, false, true, 2, 2>(hg_pick(p, 2, 2), p, oa, oa, gb, s)));
        else TRY((hg_launch<EpiSym, false, false, true>(hg_pick(p), p, oa, oa, gb, s)));
        // X
        p.M = h->rows;
        p.N = h->cols;
        p.upper = false;
        p.prof = K_ORTH_UPDATE;
        p.ops = 2.0 * count * n * n * big;
        const bool last = i + 1 == steps;
        const float so = last ? 1.0f : sx;
        const EpiUpdate::Args gu{h->x[(i + 1) & 1], so / (sb * sx), low_next, last ? out : nullptr, ldo, stride_o,
                                 ((uintptr_t)out & 15) == 0 && ldo % 8 == 0 && (count == 1 || stride_o % 8 == 0), g0};
        const int hb = 1 + low, hx = 1 + (low && low_x);
        const HgPick t = tall ? hg_pick(p, hx, hb) : hg_pick(p, hb, hx);
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
    if (!h->status.read(clear != 0, &bits)) return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_orth_destroy(nitro_orth* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    h->allocs.free();
    h->status.free();
    delete h;
}

}  // extern "C"
