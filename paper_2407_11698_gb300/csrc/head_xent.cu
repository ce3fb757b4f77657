// Softmax cross entropy of a linear head over many classes: z = scale x W^T,
// loss_i = log sum_j exp z_ij - z_i,label, and its gradients
//   G_ij = softmax(z_i)_j - [j = label_i],   dx_i = gout_i scale (G W)_i,
//   dW = scale sum_i gout_i G_i^T x_i.
//
// The logits are never kept.  The forward's products leave, for every row and tile, the
// maximum and the sum of exponentials of the tile's columns, and a second kernel joins
// them.  The backward takes the products again, writes G in bf16 from the row's log-sum, the label's
// entry from the row's other ones (EpiProb), and takes the two products with it.  Where G would pass 4 GB it goes by
// pieces of the classes, over which dx sums in 32 bits.  The products are those of k_head_gemm
// (head_gemm.cuh), 2 rows features classes operations each: one in the forward, three in the
// backward, of which one is the logits' second time, a fifth to a quarter of a step.  (Two calls share nothing but
// lse.  One call for both could keep exponentials of the distance to a tile's maximum, 2 bytes a
// logit in fp16, instead; 32-bit logits would be 4, and 16-bit ones are off by 2^-9 of their size, far too
// much under an exponential.)
//
// A forward of a few rows, a server's, runs on the CUDA cores (k_xent_few).
//
// Where dx has fewer tiles than SMs its sum is split along the classes into 32-bit slices of
// a small workspace, or shared out in a cluster (head_gemm.cuh), as the logits' is.
#include <new>

#include "head_gemm.cuh"

using namespace nitro;

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
struct RowOut {
    const int32_t* labels;
    float* loss;
    float* lse;
    uint32_t* status;
    int classes;
    float k2;              // scale log2 e
};
// zt: the label's product.  The loss is small where the label's logit is the largest, so it is not taken from
// lse, whose rounding (2.4e-7 at 7) would be all of it, but from the logit's distance to the maximum.
__device__ __forceinline__ void write_row(const RowOut& o, int64_t row, float m2, float sum, float zt) {
    const float l2 = log2f(sum), lse = (m2 + l2) * kLn2;
    const int lab = o.labels[row];
    const bool live = lab >= 0 && lab < o.classes;
    if (!live && lab != -1) atomicOr(o.status, ST_BAD_LABEL);
    o.lse[row] = lse;
    o.loss[row] = live ? (l2 - fmaf(zt, o.k2, -m2)) * kLn2 : 0.0f;
}

// (max, sum of 2^(t - max)) pairs into one.  A NaN among the logits is in a sum, not in a maximum.
struct MaxSum {
    float m = -INFINITY, s = 0.0f;
    __device__ __forceinline__ void join(float om, float os) {
        const float t = fmaxf(m, om), base = t == -INFINITY ? 0.0f : t;
        s = s * exp2f(m - base) + os * exp2f(om - base);
        m = t;
    }
};

// Every thread of every CTA, its parts and label logits written: the last CTA to come here joins the
// rows' parts [parts][rows].  ticket: zero before and after; word: the CTA's own, in shared memory.
template <int THREADS>
__device__ __forceinline__ void join_as_last(const float2* part, int parts, int rows, const float* zt, uint32_t* ticket,
                                             const RowOut& out, int* word) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) *word = atomicAdd(ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!*word) return;
    __threadfence();
    if (threadIdx.x == 0) *ticket = 0;
    // 8 or 32 lanes a row, so that the rows' loads are under way together
    const int width = rows >= THREADS / 8 ? 8 : 32, sub = threadIdx.x & (width - 1);
    for (int r0 = 0; r0 < rows; r0 += THREADS / width) {
        const int row = r0 + threadIdx.x / width;
        MaxSum v;
        if (row < rows) {
#pragma unroll 4
            for (int i = sub; i < parts; i += width) {
                const float2 p = __ldcg(part + (int64_t)i * rows + row);
                v.join(p.x, p.y);
            }
        }
        for (int d = width >> 1; d > 0; d >>= 1)
            v.join(__shfl_xor_sync(0xffffffffu, v.m, d), __shfl_xor_sync(0xffffffffu, v.s, d));
        if (sub == 0 && row < rows) {
            const int lab = out.labels[row];
            write_row(out, row, v.m, v.s, lab >= 0 && lab < out.classes ? __ldcg(zt + row) : 0.0f);
        }
    }
}

// Row statistics of a tile in base 2: (max, sum of 2^(t - max)), t = z log2 e, and the
// label's product.  A thread holds one row, so nothing is exchanged.
struct EpiStats {
    static constexpr bool kFold = true, kTail = true;
    struct Args {
        const int32_t* labels;
        float k2;             // scale log2 e
        float2* part;         // [per tiles_n][rows]
        int per;              // parts that a tile's columns are taken in
        float* zt;            // [rows]
        uint32_t* ticket;     // zero before and after
        int parts;            // few parts of few rows: the last CTA joins them, else 0
        RowOut out;
    };
    const Args& a;
    const HgArgs& g;
    int row, col0, slot, lab;
    float mx = -INFINITY, sum = 0.0f;
    __device__ __forceinline__ EpiStats(const Args& a_, const HgArgs& g_, const HgTile& t, const HgPart& p)
        : a(a_), g(g_), row(p.row), col0(p.col0) {
        slot = a.per * t.n + p.slot;
        lab = row < p.rows ? a.labels[row] : -1;
    }
    __device__ __forceinline__ void fetch(int) {}
    __device__ __forceinline__ void cols(int c, float* v) {
        const int n = g.N - (col0 + c);
        if (n <= 0) return;
        float top[8];
        if (n < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j < n ? v[j] : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) top[j] = fmaxf(fmaxf(v[j], v[j + 8]), fmaxf(v[j + 16], v[j + 24]));
#pragma unroll
        for (int j = 0; j < 4; ++j) top[j] = fmaxf(top[j], top[j + 4]);
        const float m = fmaxf(mx, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.k2);
        const float base = m == -INFINITY ? 0.0f : m;
        float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            s0 += ex2(fmaf(v[j], a.k2, -base));
            s1 += ex2(fmaf(v[j + 1], a.k2, -base));
            s2 += ex2(fmaf(v[j + 2], a.k2, -base));
            s3 += ex2(fmaf(v[j + 3], a.k2, -base));
        }
        // A term is 1 at most but for the rounding of its maximum, which moves it by a factor of up to 2 below 2^24; a
        // sum above 64 is that of masked classes (2^31 and more, where the factor is past the range)
        const float s = (s0 + s1) + (s2 + s3);
        sum = sum * exp2f(mx - base) + (s > 64.0f ? 1.0f : s);
        mx = m;
        const int at = lab - (col0 + c);
        if (at >= 0 && at < 32 && at < n) {
            float z = 0.0f;
#pragma unroll
            for (int j = 0; j < 32; ++j) z = j == at ? v[j] : z;
            a.zt[row] = z;
        }
    }
    __device__ __forceinline__ void done() {
        if (row < g.M) a.part[(int64_t)slot * g.M + row] = make_float2(mx, sum);
    }
    // the last CTA joins the parts
    static __device__ __forceinline__ void tail(const Args& a, const HgArgs& g, int* word) {
        if (a.parts) join_as_last<kHgThreads>(a.part, a.parts, g.M, a.zt, a.ticket, a.out, word);
    }
};

// softmax - onehot of a piece, rounded once to bf16, the type that the products with it
// take.  The row's factor gout scale is left to their ends (dx) and to x (dw): multiplied
// in here, the -1 at the label, exact in bf16 and most of a row's weight, would be rounded
// as well, alike in every row.  Rows that are left out give zeros.
//
// The label's entry is minus the sum of the row's other entries.  As the label's exponential less one it would
// be off by the rounding of lse, 2^-24 |lse| and more, which is all of it and many times its size in a
// confident row (loss 1e-6 at lse 20).  So a tile leaves the sum of its columns, the label's apart, and
// k_xent_label writes the entry (part), or it is there already (rest).
struct EpiProb {
    static constexpr bool kFold = true, kTail = false;
    struct Args {
        const int32_t* labels;
        const float* lse;
        float k2;
        int classes, v0;      // all classes, and the piece's first
        uint16_t* G;          // [rows][ldg], ldg a multiple of 64, or null: the sums alone
        int64_t ldg, low;     // low: from G to what its rounding left over, 0: not kept
        float* part;          // [per tiles_n][rows] sums, or null
        int per;              // parts that a tile's columns are taken in
        const float* rest;    // [rows] the sums over all classes, where part is null
    };
    const Args& a;
    const HgArgs& g;
    const HgPart& p;
    int lab = -1, slot;
    float l2 = 0.0f, entry = 0.0f, sum = 0.0f;
    bool live = false;
    __device__ __forceinline__ EpiProb(const Args& a_, const HgArgs& g_, const HgTile& t, const HgPart& p_)
        : a(a_), g(g_), p(p_), slot(a_.per * t.n + p_.slot) {
        if (p.row < p.rows) {
            lab = a.labels[p.row];
            live = lab >= 0 && lab < a.classes;
            lab -= a.v0;
            l2 = a.lse[p.row] * kLog2e;
            if (a.rest) entry = -a.rest[p.row];
        }
    }
    __device__ __forceinline__ void fetch(int) {}
    __device__ __forceinline__ void cols(int c, float* v) {
        const int col = p.col0 + c, n = g.N - col;
        if (n <= 0) return;
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = ex2(fmaf(v[j], a.k2, -l2));
        if (n < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j < n ? v[j] : 0.0f;
        }
        const int at = lab - col;
        if (live && at >= 0 && at < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = j == at ? entry : v[j];
        }
        if (a.part) {
            float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
            for (int j = 0; j < 32; j += 4) s0 += v[j], s1 += v[j + 1], s2 += v[j + 2], s3 += v[j + 3];
            sum += (s0 + s1) + (s2 + s3);
            if (!a.G) return;
        }
        uint32_t w[16];
        const auto pack = [&] {
            pack_bf16_32(v, w);
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = live ? w[j] : 0u;
        };
        pack();
        hg_store16(p, w, a.G, a.ldg, col, (int)a.ldg, true);   // a row's padding may be written
        if (a.low) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] -= __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
            pack();
            hg_store16(p, w, a.G + a.low, a.ldg, col, (int)a.ldg, true);
        }
    }
    __device__ __forceinline__ void done() {
        if (a.part && p.row < p.rows) a.part[(int64_t)slot * g.M + p.row] = sum;
    }
};

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
        const float* factor;  // of the row, or of all rows
        int one;
    };
    const Args& a;
    const HgArgs& g;
    const HgPart& p;
    float f = 0.0f;
    __device__ __forceinline__ EpiBf16(const Args& a_, const HgArgs& g_, const HgTile&, const HgPart& p_) : a(a_), g(g_), p(p_) {
        if (p.row < p.rows) f = a.factor[a.one ? 0 : p.row];
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
// The forward of up to kFewRows rows on the CUDA cores: W's bytes bound it, and a sum that is
// rounded at every step is nearer than the tensor cores', which cut off: with one to four rows
// a confident row's small loss is all there is to be off from (4096 features, 1000 classes:
// up to 2.9e-6 of the loss on the tensor cores, 3e-7 here).  One launch, no copies and no tensor maps:
// 4 x 512 x 10000 6.8 us (9.6 on the tensor cores; W's 10 MB from L2), 4 x 4096 x 64000 111 us (W at 4.7 TB/s).
//
// A warp takes C classes (over ks warps of a CTA by pieces of 256 features, where there are few), R
// rows at a time in registers; x comes from L1 after the first class.  Its sums are
// exchanged so that each lane ends with one (row, class), whose statistics it keeps.
struct FewArgs {
    int64_t ldx, ldw;
    int rows, features, ks;
    float2* part;          // [CTAs][rows]
    float* zt;
    uint32_t* ticket;
    RowOut out;
};

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

template <typename T, int R, int C, bool VEC>
__global__ void __launch_bounds__(256, 2) k_xent_few(const T* x, const uint16_t* w, const FewArgs a) {
    constexpr int N = R * C, kLanes = 32 / N;     // lanes that hold the same sum
    __shared__ float sums[2][8][N];
    __shared__ float2 rows_sh[8][R];
    __shared__ int last;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = warp % a.ks, per = 8 / a.ks;
    const int groups = (a.out.classes + C - 1) / C, row = lane / kLanes / C;
    const bool mine = sub == 0 && lane % kLanes == 0 && row < a.rows;
    const int lab = mine ? a.out.labels[row] : -1;
    const T* xr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xr[r] = x + min(r, a.rows - 1) * a.ldx;
    MaxSum st;
    int turn = 0;
    for (int g0 = blockIdx.x * per; g0 < groups; g0 += gridDim.x * per, turn ^= 1) {
        const int first = (g0 + warp / a.ks) * C;
        float acc[R][C];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i / C][i % C] = 0.0f;
        if (first < a.out.classes) {
            const uint16_t* wr[C];
#pragma unroll
            for (int c = 0; c < C; ++c) wr[c] = w + min(first + c, a.out.classes - 1) * a.ldw;
            int piece = sub * 256;
#pragma unroll 2
            for (; piece + 256 <= a.features; piece += a.ks * 256)
                few_step<T, R, C, VEC, true>(xr, wr, piece, lane, a.features, acc);
            if (piece < a.features) few_step<T, R, C, VEC, false>(xr, wr, piece, lane, a.features, acc);
        }
        float z = few_sum<N>(&acc[0][0], lane);
        if (a.ks > 1) {
            if (lane % kLanes == 0) sums[turn][warp][lane / kLanes] = z;
            __syncthreads();       // the other turn's sums are read by now
            if (mine) {
                z = sums[turn][warp][lane / kLanes];
                for (int k = 1; k < a.ks; ++k) z += sums[turn][warp + k][lane / kLanes];
            }
        }
        const int cls = first + lane / kLanes % C;
        if (mine && cls < a.out.classes) {
            const float t = z * a.out.k2;
            // what t's rounding left over: see write_row().  A masked class may have a t that is not finite, or
            // one of 2^31 and more, whose rounding alone is past an exponential's range.
            const float rest = exp2f(fmaf(z, a.out.k2, -t));
            if (t != -INFINITY) st.join(t, rest > 2.0f ? 1.0f : rest);
            if (cls == lab) a.zt[row] = z;
        }
    }
    // over the lanes of a row, the warps, and then the CTAs
#pragma unroll
    for (int d = 1; d < kLanes * C; d <<= 1)
        st.join(__shfl_xor_sync(0xffffffffu, st.m, d), __shfl_xor_sync(0xffffffffu, st.s, d));
    if (lane % (kLanes * C) == 0) rows_sh[warp][row] = make_float2(st.m, st.s);
    __syncthreads();
    if (threadIdx.x < a.rows) {
        MaxSum v;
        for (int i = 0; i < 8; ++i) v.join(rows_sh[i][threadIdx.x].x, rows_sh[i][threadIdx.x].y);
        a.part[(int64_t)blockIdx.x * a.rows + threadIdx.x] = make_float2(v.m, v.s);
    }
    join_as_last<256>(a.part, gridDim.x, a.rows, a.zt, a.ticket, a.out, &last);
}

// ------------------------------------------------------------------ row kernels
// Joins a row's tiles: 32 rows a CTA, the tiles over its warps.
__global__ void __launch_bounds__(256) k_xent_join(const float2* part, int parts, int rows, const float* zt, const RowOut o) {
    __shared__ float2 sh[8][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
    MaxSum v;
    if (row < rows)
        for (int i = w; i < parts; i += 8) {
            const float2 p = part[(int64_t)i * rows + row];
            v.join(p.x, p.y);
        }
    sh[w][lane] = make_float2(v.m, v.s);
    __syncthreads();
    if (w == 0 && row < rows) {
        for (int i = 1; i < 8; ++i) v.join(sh[i][lane].x, sh[i][lane].y);
        const int lab = o.labels[row];
        write_row(o, row, v.m, v.s, lab >= 0 && lab < o.classes ? zt[row] : 0.0f);
    }
}

// The label's entry of G from the sums of its row's other entries, or those sums alone (rest): 32 rows a
// CTA, the parts over its warps.
__global__ void __launch_bounds__(256) k_xent_label(const float* part, int parts, int rows, const int32_t* labels, int classes,
                                                    uint16_t* G, int64_t ldg, int64_t low, float* rest) {
    __shared__ float sh[8][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (row < rows)
        for (int i = w; i < parts; i += 8) v += part[(int64_t)i * rows + row];
    sh[w][lane] = v;
    __syncthreads();
    if (w != 0 || row >= rows) return;
    for (int i = 1; i < 8; ++i) v += sh[i][lane];
    if (rest) {
        rest[row] = v;
        return;
    }
    const int lab = labels[row];
    if (lab < 0 || lab >= classes) return;
    const __nv_bfloat16 h = __float2bfloat16_rn(-v);
    uint16_t* at = G + row * ldg + lab;
    *at = __bfloat16_as_ushort(h);
    if (low) at[low] = __bfloat16_as_ushort(__float2bfloat16_rn(-v - __bfloat162float(h)));
}

// dx in bf16 from the slices of its 32-bit sums, four columns a thread.
__global__ void __launch_bounds__(256) k_xent_dx(const float* c, int64_t ldc, int64_t slice, int slices, int features,
                                                 const float* factor, uint16_t* dx, int64_t lddx, int vec) {
    pdl_wait();
    const int64_t row = blockIdx.x;
    const float f = factor[row];
    for (int j = (blockIdx.y * 256 + threadIdx.x) * 4; j < features; j += gridDim.y * 1024) {
        float4 v = *reinterpret_cast<const float4*>(c + row * ldc + j);      // ldc holds the padding
        for (int k = 1; k < slices; ++k) {
            const float4 o = *reinterpret_cast<const float4*>(c + k * slice + row * ldc + j);
            v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
        }
        const uint32_t w[2] = {pack_bf16(v.x * f, v.y * f), pack_bf16(v.z * f, v.w * f)};
        uint16_t* dst = dx + row * lddx + j;
        if (vec && j + 4 <= features) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
        else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < features) dst[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
        }
    }
}

// A weight gradient of zeros (of an empty batch) into rows ld apart.
__global__ void __launch_bounds__(256) k_xent_zero(uint16_t* dw, int64_t ld, int64_t rows, int cols) {
    pdl_wait();
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, (int64_t)gridDim.x * 256, cols);
    for (; at.row < rows; at.next()) dw[at.row * ld + at.part] = 0;
}

// What the backward takes of x and gout: rows that are left out become zeros, so that an
// infinity or NaN in them meets no weight gradient (0 times it is NaN); the others
// x gout_i / ref, ref = the largest |gout| of the rows with a label, so that no factor is above 1 whatever the
// gradients' range (a quotient by a smaller one can pass bf16), and under a mean, where all
// are alike, x stays what it is.  factor[0] = scale ref, factor[1 + i] = scale gout_i.
struct PackGrad {
    const int32_t* labels;     // or null: a plain copy
    const float* gout;         // or null: 1
    float* factor;
    float scale;
    int classes;
    const float* tops;         // the largest |gout| of parts of the rows, or null: the rows are gone through
    int n_tops;
    // |gout| of a row, 0 where it is left out
    __device__ __forceinline__ float size(int64_t row) const {
        const int lab = labels[row];
        return lab >= 0 && lab < classes ? fabsf(gout[row]) : 0.0f;
    }
};

// The largest of the threads' values (none negative; a NaN counts for nothing), in every thread of 256.
__device__ __forceinline__ float block_max(float v) {
    __shared__ float sh[8];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) v = fmaxf(v, sh[w]);
    return v;
}

// The largest |gout| of a CTA's rows, for batches of more rows than every CTA of k_xent_pack should go through.
__global__ void __launch_bounds__(256) k_xent_top(const PackGrad pg, int rows, float* tops) {
    pdl_wait();
    float v = 0.0f;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < rows; i += gridDim.x * 256) v = fmaxf(v, pg.size(i));
    v = block_max(v);
    if (threadIdx.x == 0) tops[blockIdx.x] = v;
}

// Rows of x as bf16 with a stride of ldp (a multiple of 8; padding zero): int8 activations
// are exact in bf16.
// plain (may be null): the rows as they are, as well.
template <typename T>
__global__ void __launch_bounds__(256) k_xent_pack(const T* x, int64_t ldx, int rows, int cols, uint16_t* out, int64_t ldp,
                                                   const PackGrad pg, uint16_t* plain) {
    pdl_wait();
    float ref = 1.0f;
    if (pg.labels && pg.gout) {
        float v = 0.0f;
        if (pg.tops)
            for (int i = threadIdx.x; i < pg.n_tops; i += 256) v = fmaxf(v, pg.tops[i]);
        else
            for (int i = threadIdx.x; i < rows; i += 256) v = fmaxf(v, pg.size(i));
        ref = block_max(v);
    }
    if (pg.labels && blockIdx.x == 0 && threadIdx.x == 0) pg.factor[0] = pg.scale * ref;
    const int per = (int)(ldp / 8);
    const int64_t words = (int64_t)rows * per, step = (int64_t)gridDim.x * 256;
    const bool vec = sizeof(T) == 2 ? (((uintptr_t)x | (uintptr_t)(ldx * 2)) & 15) == 0
                                    : (((uintptr_t)x | (uintptr_t)ldx) & 7) == 0;
    RowWalk at(blockIdx.x * (int64_t)256 + threadIdx.x, step, per);
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < words; i += step, at.next()) {
        const int64_t row = at.row;
        const int c = at.part * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        bool live = true;
        float f = 1.0f;
        if (pg.labels) {
            const int lab = pg.labels[row];
            live = lab >= 0 && lab < pg.classes;
            const float go = live ? (pg.gout ? pg.gout[row] : 1.0f) : 0.0f;
            f = go == ref ? 1.0f : go == -ref ? -1.0f : go / ref;      // (an infinity among them, too)
            live = live && go != 0.0f;
            if (c == 0) pg.factor[1 + row] = pg.scale * go;
        }
        if (live || plain) {
            const T* src = x + row * ldx + c;
            uint32_t* w = reinterpret_cast<uint32_t*>(&v);
            if constexpr (sizeof(T) == 2) {
                if (vec && c + 8 <= cols) v = *reinterpret_cast<const uint4*>(src);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < cols) w[j >> 1] |= (uint32_t)src[j] << (16 * (j & 1));
                }
            } else {
                uint32_t b[2] = {0x80808080u, 0x80808080u};   // bytes hold x + 128
                if (vec && c + 8 <= cols) {
                    const uint2 r = *reinterpret_cast<const uint2*>(src);
                    b[0] ^= r.x;
                    b[1] ^= r.y;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (c + j < cols) b[j >> 2] ^= (uint32_t)(uint8_t)src[j] << (8 * (j & 3));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = bf16x2(b[j >> 1], 2 * (j & 1));
            }
            if (plain) reinterpret_cast<uint4*>(plain)[i] = v;
            if (!live) v = make_uint4(0, 0, 0, 0);
            else if (f != 1.0f) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = pack_bf16(__uint_as_float(w[j] << 16) * f, __uint_as_float(w[j] & 0xffff0000u) * f);
            }
        }
        reinterpret_cast<uint4*>(out)[i] = v;
    }
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Up to this many rows G is kept as two bf16 halves: the rounding of one entry, up to 2^-8 of
// it, can be most of a lone row's error, and averages out over more.
constexpr int kRowsWithLow = 32;

// The tensor cores drop the bits that a sum's 32 do not hold, so its error grows with the
// additions.  The loss of some hundred rows is off, of its size, in one sum by 3.6e-7 with 1024 features, 5.4e-7 with 1536,
// 7.2e-7 with 2000, 9.1e-7 with 2560, 1.25e-6 with 3500 and 1.46e-6 with 4096; in two halves, added with
// rounding, by half of that.  Halves from here on keep it below 7.5e-7 up to 4096 features; at 8192 x 4096 x
// 32000 they take 3 per cent more time.
constexpr int kFoldFeatures = 2048;

// Parts of all rows that the forward's last CTA still joins by itself; more go to a launch of
// their own (4 rows x 512 x 10000, taken here: 11.1 us with that launch and 9.9 without; 64 x 4096 x 1000,
// 2048 parts: 12.9 and 14.8).
constexpr int64_t kPartsInOne = 1024;

// The forward takes up to kFewRows rows to k_xent_few, from five on only where the head is small or
// TMA cannot take W.  us, k_xent_few and the tensor cores: 4 rows x 512 x 10000 6.8 and 9.6, x 4096
// x 64000 111 and 127; 8 rows x 4096 x 1000 8.2 and 12.2, x 512 x 10000 8.9 and 10.2, but x 1000 x 20011
// 20.7 and 16.4 to 19; the same with W's rows at odd addresses 23.8 and 32.2.
constexpr int kFewRows = 8;
constexpr int64_t kFewProducts = (int64_t)8 << 20;
constexpr int kFewCtas = 512;      // at most

// Rows that every CTA of k_xent_pack goes through for the largest |gout|; more are gone through once, by a launch
// of up to kTopCtas.  A backward for dw of 512 features and 64 classes, us, gone through by every CTA and by a launch:
// 1000 rows 18.9 and 19.3, 2000 20.3 and 20.3, 4000 22.3 and 21.9, 8192 26.6 and 25.3, 65536 131 and 96.
constexpr int kRowsInPack = 2048;
constexpr int kTopCtas = 64;

// G: at most 4 GB.  Beyond that the classes go in pieces, whose rows' sums have to be known before the first
// piece's products: the logits are then taken a third time, and dx's 32-bit sums are read and written
// again by every piece.
constexpr int64_t kGElems = (int64_t)1 << 31;
constexpr int64_t kAccFloats = (int64_t)16 << 20;   // slices beyond one: at most 64 MB together

}  // namespace
}  // namespace nitro

struct nitro_xent {
    int max_rows = 0, features = 0, classes = 0;
    int64_t ldp = 0, g_elems = 0, acc_floats = 0;
    uint16_t* xp = nullptr;     // [max_rows][ldp] bf16 copy of x where TMA cannot take its rows
    uint16_t* xg = nullptr;     // and as dw's product takes it, see PackGrad
    uint16_t* wp = nullptr;     // [classes][ldp] copy of W where its rows are not aligned for TMA
    uint16_t* G = nullptr;
    float* acc = nullptr;
    float2* part = nullptr;
    float* zt = nullptr;        // [max_rows] the forward's label logits, the backward's sums (EpiProb::Args::rest)
    float* factor = nullptr;    // [1 + max_rows], see PackGrad, and [kTopCtas]
    uint32_t* ticket = nullptr; // of the forward's CTAs
    bool clean = false;         // the ticket, see clear_once
    StatusWord status;
    DeviceAllocs allocs;
};

namespace {

#define TRY(expr)                                         \
    do {                                                  \
        if ((expr) != cudaSuccess) return NITRO_ERR_CUDA; \
    } while (0)

bool tma_rows(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

cudaError_t pack_rows(const void* x, int type, int64_t ldx, int rows, int cols, uint16_t* out, int64_t ldp,
                      const PackGrad& pg, cudaStream_t s, uint16_t* plain = nullptr) {
    static std::atomic<int> resident[2];
    const int64_t words = rows * (ldp / 8);
    const int grid = type == NITRO_I8 ? one_wave(k_xent_pack<int8_t>, resident[0], words) : one_wave(k_xent_pack<uint16_t>, resident[1], words);
    ProfScope ps(K_XENT_PACK, s, 0.0, (double)rows * cols * (type == NITRO_I8 ? 3 : 4));
    if (type == NITRO_I8)
        return launch_k(k_xent_pack<int8_t>, dim3(grid), dim3(256), 0, s, (const int8_t*)x, ldx, rows, cols, out, ldp, pg,
                        plain);
    return launch_k(k_xent_pack<uint16_t>, dim3(grid), dim3(256), 0, s, (const uint16_t*)x, ldx, rows, cols, out, ldp, pg,
                    plain);
}

bool copies(const void* x, int type, int64_t ldx) { return type == NITRO_I8 || !tma_rows(x, ldx); }

// W as an operand along K; a copy where TMA cannot take its rows.
cudaError_t w_operand(nitro_xent* h, const uint16_t* w, int64_t ldw, cudaStream_t s, HgOperand* ow) {
    const bool copy = copies(w, NITRO_BF16, ldw);
    *ow = {copy ? h->wp : w, h->features, h->classes, copy ? h->ldp : ldw, 1, 0};
    return copy ? pack_rows(w, NITRO_BF16, ldw, h->classes, h->features, h->wp, h->ldp, PackGrad{}, s) : cudaSuccess;
}

bool xent_args(const nitro_xent* h, const void* x, int x_type, int64_t ldx, const void* w, int64_t ldw,
               const int32_t* labels, int rows, float scale) {
    if (!h || rows < 0 || rows > h->max_rows || (x_type != NITRO_BF16 && x_type != NITRO_I8)) return false;
    if (ldx < h->features || ldw < h->features || !(scale > 0.0f) || scale > 1e30f) return false;
    if (rows > 0 && (!x || !w || !labels)) return false;
    return ((uintptr_t)w & 1) == 0 && (x_type == NITRO_I8 || ((uintptr_t)x & 1) == 0);
}

HgProblem logits_problem(const nitro_xent* h, int rows, int64_t classes) {
    HgProblem p{rows, classes, h->features};
    p.status = h->status.at;
    p.prof = K_XENT_LOGITS;
    p.ops = 2.0 * rows * classes * h->features;
    return p;
}

template <typename T, int R, int C>
cudaError_t few_as(bool vec, const void* x, const uint16_t* w, const FewArgs& a, int grid, cudaStream_t s) {
    return vec ? launch_k(k_xent_few<T, R, C, true>, dim3(grid), dim3(256), 0, s, (const T*)x, w, a)
               : launch_k(k_xent_few<T, R, C, false>, dim3(grid), dim3(256), 0, s, (const T*)x, w, a);
}
template <typename T>
cudaError_t few_rows(bool vec, int c, const void* x, const uint16_t* w, const FewArgs& a, int grid, cudaStream_t s) {
    if (c == 4) return a.rows <= 1 ? few_as<T, 1, 4>(vec, x, w, a, grid, s) : a.rows <= 4 ? few_as<T, 4, 4>(vec, x, w, a, grid, s) : few_as<T, 8, 4>(vec, x, w, a, grid, s);
    return a.rows <= 1 ? few_as<T, 1, 1>(vec, x, w, a, grid, s) : a.rows <= 4 ? few_as<T, 4, 1>(vec, x, w, a, grid, s) : few_as<T, 8, 1>(vec, x, w, a, grid, s);
}

cudaError_t forward_few(nitro_xent* h, const void* x, int x_type, int64_t ldx, const uint16_t* w, int64_t ldw, int rows,
                        const RowOut& ro, cudaStream_t s) {
    // two CTAs an SM; four classes a warp where that leaves no warp idle, else one, and its features
    // over as many warps as are free
    const int ctas = std::min(2 * sm_count(), kFewCtas), warps = 8 * ctas, pieces = (h->features + 255) / 256;
    const int c = (int64_t)((h->classes + 3) / 4) * std::min(8, pieces) >= warps / 2 ? 4 : 1;
    const int groups = (h->classes + c - 1) / c;
    int ks = 1;
    while (ks < 8 && 2 * ks <= pieces && (int64_t)groups * 2 * ks <= warps) ks *= 2;
    const FewArgs a{ldx, ldw, rows, h->features, ks, h->part, h->zt, h->ticket, ro};
    const int grid = std::min(ctas, (groups + 8 / ks - 1) / (8 / ks));
    const bool i8 = x_type == NITRO_I8;
    const bool vec = tma_rows(w, ldw) && (i8 ? ((uintptr_t)x & 7) == 0 && ldx % 8 == 0 : tma_rows(x, ldx));
    ProfScope ps(K_XENT_LOGITS, s, 2.0 * rows * h->classes * h->features, 2.0 * h->classes * h->features);
    return i8 ? few_rows<int8_t>(vec, c, x, w, a, grid, s) : few_rows<uint16_t>(vec, c, x, w, a, grid, s);
}

}  // namespace

extern "C" {

nitro_status nitro_xent_create(int max_rows, int features, int classes, nitro_xent** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (max_rows < 1 || features < 1 || classes < 1 || max_rows > (1 << 20) || features > (1 << 17) ||
        classes > (1 << 24) || (int64_t)max_rows * features > ((int64_t)1 << 34) ||
        (int64_t)classes * features > ((int64_t)1 << 36))
        return NITRO_ERR_ARG;
    nitro_xent* h = new (std::nothrow) nitro_xent();
    if (!h) return NITRO_ERR_CUDA;
    h->max_rows = max_rows;
    h->features = features;
    h->classes = classes;
    h->ldp = round_up(features, 8);
    h->g_elems = std::min(kGElems, std::max(max_rows, 2 * std::min(max_rows, kRowsWithLow)) * round_up(classes, 64));
    h->acc_floats = std::max(max_rows * round_up(features, 32), kAccFloats);
    const int64_t parts = 4 * ((classes + 127) / 128);
    // (the ticket is cleared by the first forward)
    const bool ok = h->allocs.take(&h->xp, max_rows * h->ldp) && h->allocs.take(&h->xg, max_rows * h->ldp) &&
                    h->allocs.take(&h->wp, classes * h->ldp) && h->allocs.take(&h->G, h->g_elems) &&
                    h->allocs.take(&h->acc, h->acc_floats) &&
                    h->allocs.take(&h->part, std::max<int64_t>(parts * max_rows, kFewCtas * kFewRows)) &&
                    h->allocs.take(&h->zt, max_rows) && h->allocs.take(&h->factor, max_rows + 1 + kTopCtas) &&
                    h->allocs.take(&h->ticket, 1) && h->status.take();
    if (!ok) {
        nitro_xent_destroy(h);
        return NITRO_ERR_CUDA;
    }
    *out = h;
    return NITRO_OK;
}

nitro_status nitro_xent_forward(nitro_xent* h, const void* x, int x_type, int64_t ldx, const uint16_t* w, int64_t ldw,
                                const int32_t* labels, int rows, float scale, float* loss, float* lse, void* stream) {
    if (!xent_args(h, x, x_type, ldx, w, ldw, labels, rows, scale)) return NITRO_ERR_ARG;
    if (rows == 0) return NITRO_OK;
    if (!loss || !lse) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    TRY(clear_once(h->clean, h->ticket, 4, s));
    const RowOut ro{labels, loss, lse, h->status.at, h->classes, scale * kLog2e};
    if (rows <= kFewRows && (rows <= 4 || (int64_t)h->classes * h->features <= kFewProducts || copies(w, NITRO_BF16, ldw))) {
        TRY(forward_few(h, x, x_type, ldx, w, ldw, rows, ro, s));
        return NITRO_OK;
    }
    HgOperand ox{x, h->features, rows, ldx, 1, 0}, ow;
    if (copies(x, x_type, ldx)) {
        TRY(pack_rows(x, x_type, ldx, rows, h->features, h->xp, h->ldp, PackGrad{}, s));
        ox = {h->xp, h->features, rows, h->ldp, 1, 0};
    }
    TRY(w_operand(h, w, ldw, s, &ow));
    HgProblem p = logits_problem(h, rows, h->classes);
    p.fold = h->features > kFoldFeatures;
    const HgPick t = hg_pick(p);
    const int per = t.ks > 1 ? 4 : 2, parts = per * ((h->classes + t.bn - 1) / t.bn);
    const bool few = (int64_t)parts * rows <= kPartsInOne;
    const EpiStats::Args ea{labels, scale * kLog2e, h->part, per, h->zt, h->ticket, few ? parts : 0, ro};
    TRY((hg_launch<EpiStats, false, false, false>(t, p, ox, ow, ea, s)));
    if (few) return NITRO_OK;
    ProfScope ps(K_XENT_ROWS, s, 0.0, 8.0 * parts * rows);
    TRY(launch_k(k_xent_join, dim3((rows + 31) / 32), dim3(256), 0, s, (const float2*)h->part, parts, rows,
                 (const float*)h->zt, ro));
    return NITRO_OK;
}

nitro_status nitro_xent_backward(nitro_xent* h, const void* x, int x_type, int64_t ldx, const uint16_t* w, int64_t ldw,
                                 const int32_t* labels, int rows, float scale, const float* lse, const float* gout,
                                 uint16_t* dx, int64_t lddx, uint16_t* dw, int64_t lddw, void* stream) {
    if (!xent_args(h, x, x_type, ldx, w, ldw, labels, rows, scale)) return NITRO_ERR_ARG;
    if ((dx && (lddx < h->features || ((uintptr_t)dx & 1))) || (dw && (lddw < h->features || ((uintptr_t)dw & 1))))
        return NITRO_ERR_ARG;
    if (rows > 0 && !lse) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int F = h->features, V = h->classes;
    if (rows == 0) {   // an empty batch has a weight gradient of zero
        if (dw && lddw == F) {
            TRY(cudaMemsetAsync(dw, 0, sizeof(uint16_t) * (size_t)V * F, s));
        } else if (dw) {
            static std::atomic<int> resident{0};
            ProfScope ps(K_XENT_DW, s, 0.0, 2.0 * V * F);
            TRY(launch_k(k_xent_zero, dim3(one_wave(k_xent_zero, resident, (int64_t)V * F)), dim3(256), 0, s, dw, lddw, (int64_t)V, F));
        }
        return NITRO_OK;
    }
    if (!dx && !dw) return NITRO_OK;
    HgOperand ox{x, F, rows, ldx, 1, 0}, ow;
    const bool copy = copies(x, x_type, ldx);
    if (copy) ox = {h->xp, F, rows, h->ldp, 1, 0};
    PackGrad pg{labels, gout, h->factor, scale, V, nullptr, 0};
    if (gout && rows > kRowsInPack) {
        float* tops = h->factor + 1 + h->max_rows;
        pg.n_tops = std::min(kTopCtas, (rows + 255) / 256);
        ProfScope ps(K_XENT_PACK, s, 0.0, 8.0 * rows);
        TRY(launch_k(k_xent_top, dim3(pg.n_tops), dim3(256), 0, s, pg, rows, tops));
        pg.tops = tops;
    }
    TRY(pack_rows(x, x_type, ldx, rows, F, h->xg, h->ldp, pg, s, copy ? h->xp : nullptr));
    TRY(w_operand(h, w, ldw, s, &ow));
    const HgOperand og{h->xg, F, rows, h->ldp, 1, 0};
    const int halves = rows <= kRowsWithLow ? 2 : 1;
    int64_t piece = std::min<int64_t>(round_up(V, 64), h->g_elems / halves / rows / 64 * 64);
    // the logits of n classes through EpiProb, and what follows from its sums
    float* sums = reinterpret_cast<float*>(h->part);
    const auto softmax = [&](const HgOperand& wp, int64_t n, EpiProb::Args ep) -> nitro_status {
        HgProblem p = logits_problem(h, rows, n);
        p.fold = F > kFoldFeatures;         // as in the forward
        const HgPick t = hg_pick(p);
        ep.per = t.ks > 1 ? 4 : 2;
        TRY((hg_launch<EpiProb, false, false, false>(t, p, ox, wp, ep, s)));
        if (!ep.part) return NITRO_OK;
        const int parts = ep.per * (int)((n + t.bn - 1) / t.bn);
        ProfScope ps(K_XENT_ROWS, s, 0.0, 4.0 * parts * rows);
        TRY(launch_k(k_xent_label, dim3((rows + 31) / 32), dim3(256), 0, s, (const float*)sums, parts, rows, labels, V, ep.G, ep.ldg,
                     ep.low, ep.G ? nullptr : h->zt));
        return NITRO_OK;
    };
    EpiProb::Args ep{labels, lse, scale * kLog2e, V, 0, nullptr, 0, 0, sums, 0, nullptr};
    if (piece < V) {
        piece = piece / 256 * 256;
        if (const nitro_status st = softmax(ow, V, ep)) return st;
        ep.part = nullptr;
        ep.rest = h->zt;
    }
    // dx: in slices along the classes where its tiles leave SMs idle
    const int64_t ldc = round_up(F, 32);
    const HgProblem pd{rows, F, std::min<int64_t>(piece, V)};
    const HgPick td = hg_pick(pd, halves, 1, (int)std::max<int64_t>(1, std::min<int64_t>(16, h->acc_floats / (rows * ldc))));
    const bool direct = piece >= V && td.splits == 1;
    for (int64_t v0 = 0; v0 < V; v0 += piece) {
        const int64_t n = std::min<int64_t>(piece, V - v0);
        HgOperand wp = ow;
        wp.base = static_cast<const uint16_t*>(ow.base) + v0 * ow.ld;
        wp.outer = n;
        ep.v0 = (int)v0;
        ep.G = h->G;
        ep.ldg = round_up(n, 64);
        ep.low = halves == 2 ? rows * ep.ldg : 0;
        if (const nitro_status st = softmax(wp, n, ep)) return st;
        const HgOperand G{h->G, n, rows, ep.ldg, halves, rows * ep.ldg};
        if (dx) {
            HgProblem p{rows, F, n};
            p.planes_a = halves;
            p.status = h->status.at;
            p.prof = K_XENT_DX;
            p.ops = 2.0 * rows * n * F;
            if (direct) {
                const EpiBf16::Args eb{dx, lddx, tma_rows(dx, lddx), h->factor + 1, 0};
                if (halves == 2) TRY((hg_launch<EpiBf16, false, true, false, 2, 1>(td, p, G, wp, eb, s)));
                else TRY((hg_launch<EpiBf16, false, true, false>(td, p, G, wp, eb, s)));
            } else {
                // a shorter last piece has as many slices or fewer: it adds to the first ones
                const HgPick t{td.cg, td.bn, hg_splits(n, td.splits), td.ks};
                const EpiAcc::Args ea{h->acc, ldc, rows * ldc, v0 > 0};
                if (halves == 2) TRY((hg_launch<EpiAcc, false, true, false, 2, 1>(t, p, G, wp, ea, s)));
                else TRY((hg_launch<EpiAcc, false, true, false>(t, p, G, wp, ea, s)));
            }
        }
        if (dw) {
            HgProblem p{n, F, rows};
            p.planes_a = halves;
            p.status = h->status.at;
            p.prof = K_XENT_DW;
            p.ops = 2.0 * rows * n * F;
            const EpiBf16::Args eb{dw + v0 * lddw, lddw, tma_rows(dw, lddw), h->factor, 1};
            if (halves == 2) TRY((hg_launch<EpiBf16, true, true, false, 2, 1>(hg_pick(p, 2), p, G, og, eb, s)));
            else TRY((hg_launch<EpiBf16, true, true, false>(hg_pick(p), p, G, og, eb, s)));
        }
    }
    if (dx && !direct) {
        ProfScope ps(K_XENT_ROWS, s, 0.0, (4.0 * td.splits + 2.0) * rows * F);
        TRY(launch_k(k_xent_dx, dim3(rows, (unsigned)std::min(8, (F + 1023) / 1024)), dim3(256), 0, s, (const float*)h->acc,
                     ldc, rows * ldc, td.splits, F, (const float*)h->factor + 1, dx, lddx,
                     (int)(((uintptr_t)dx & 7) == 0 && lddx % 4 == 0)));
    }
    return NITRO_OK;
}

nitro_status nitro_xent_status(nitro_xent* h, int clear) {
    if (!h) return NITRO_ERR_ARG;
    uint32_t bits = 0;
    if (!h->status.read(clear != 0, &bits)) return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : bits & ST_BAD_LABEL ? NITRO_ERR_ARG : NITRO_OK;
}

void nitro_xent_destroy(nitro_xent* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    h->allocs.free();
    h->status.free();
    delete h;
}

}  // extern "C"
