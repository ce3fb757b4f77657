// A gated feed-forward block: z = scale x W^T, W's first `hidden` rows the gate's, out = act(a) b with
// z = [a b], and its gradients
//   D = [dout b act'(a), dout act(a)],   dx = scale D W,   dW = scale D^T x.
//
// The forward is one product (head_gemm.cuh) whose tiles hold gate and up columns in turns of 16, so that the
// epilogue has both of a unit in one thread: z goes through memory only as what the backward keeps of it, 32 bits a
// value (8 rows hidden bytes each way, beside 12 rows hidden features operations; 16 bits would
// put a rounding of 2^-9 under both gradients, and taking the products again costs a third of a step).
// The backward writes D in bf16, which both products with it take.  4 rows hidden features operations forward and
// 8 backward: 8192 x 2048 x 8192 1.09 to 1.17 ms at the power limit, forward 332 to 348 us (1.66 to 1.58 PFLOP/s), D 143 (6.6 TB/s), dx 324
// to 340, dW 299 to 307 (1.7 and 1.84).  Few rows run on the CUDA cores, where W's bytes bound them (k_glu_few).
#include <new>

#include "head_act.cuh"

using namespace nitro;

namespace nitro {
namespace {

// Where saved has z: of whole blocks of 16 units a line of 128 bytes for each row, gates first, row after row and block after
// block, so that lines are aligned whatever `hidden` is; then the units that are left, gates and ups of a row together.
struct Saved {
    float* base;
    int64_t rows;
    int hidden;
    __device__ __forceinline__ int blocks() const { return hidden >> 4; }
    __device__ __forceinline__ float* line(int block, int64_t row) const { return base + (block * rows + row) * 32; }
    // z of a unit past the whole blocks, its gate; *up: from there to its up
    __device__ __forceinline__ float* rest(int unit, int64_t row, int* up) const {
        *up = hidden & 15;
        return base + blocks() * rows * 32 + row * 2 * *up + (unit & 15);
    }
    __device__ __forceinline__ float* at(int unit, int64_t row, int* up) const {
        if (unit >> 4 == blocks()) return rest(unit, row, up);
        *up = 16;
        return line(unit >> 4, row) + (unit & 15);
    }
};

// out and saved of a tile: columns come in turns of 16 gates and the 16 ups of the same units.
struct EpiGlu {
    static constexpr bool kFold = true, kTail = false;
    struct Args {
        uint16_t* out;
        int64_t ldo;
        Saved saved;          // base null: not kept
        int vec;              // out's rows are 16-byte aligned
        int hidden, act;
        float scale;
    };
    const Args& a;
    const HgPart& p;
    uint32_t kept[8];         // 16 units' outputs, until the next 16 fill their line of 64 bytes
    __device__ __forceinline__ EpiGlu(const Args& a_, const HgArgs&, const HgTile&, const HgPart& p_) : a(a_), p(p_) {}
    __device__ __forceinline__ void fetch(int) {}
    __device__ __forceinline__ void save(const float* v, int unit) const {
        if (unit + 16 > a.hidden) {           // the units past the whole blocks
            int up;
            float* dst = a.saved.rest(unit, p.row, &up);
            if (p.row < p.rows)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (unit + j < a.hidden) dst[j] = v[j], dst[up + j] = v[16 + j];
            return;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint4 w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float* f = v + 16 * half + 4 * j;
                w[j] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            }
            p.stage.to_lines(w);
            const int row = p.row0 + p.stage.line_row(0);
            uint4* dst = reinterpret_cast<uint4*>(a.saved.line(unit >> 4, row) + 16 * half + 4 * p.stage.line_chunk());
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (row + 8 * i < p.rows) dst[8 * i * 8] = w[i];
        }
    }
    __device__ __forceinline__ void cols(int c, float* v) {
        const int unit = (p.col0 + c) >> 1;
        if (unit < a.hidden) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= a.scale;
            if (a.saved.base) save(v, unit);
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float2 r = mul2(act_value<decltype(act)::value>(make_float2(v[j], v[j + 1])), make_float2(v[16 + j], v[17 + j]));
                    v[j] = r.x, v[j + 1] = r.y;
                }
            });
        }
        uint32_t w[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[8 + j] = pack_bf16(v[2 * j], v[2 * j + 1]);
        if (p.width == 32) {     // a cluster's slice: the thread's row alone
            if (p.row >= p.rows || unit >= a.hidden) return;
            uint16_t* dst = a.out + p.row * a.ldo + unit;
            if (a.vec && unit + 16 <= a.hidden) {
                reinterpret_cast<uint4*>(dst)[0] = make_uint4(w[8], w[9], w[10], w[11]);
                reinterpret_cast<uint4*>(dst)[1] = make_uint4(w[12], w[13], w[14], w[15]);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (unit + j < a.hidden) dst[j] = (uint16_t)(w[8 + (j >> 1)] >> (16 * (j & 1)));
            }
        } else if (c & 32) {
            if (unit - 16 >= a.hidden) return;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = kept[j];
            hg_store16(p, w, a.out, a.ldo, unit - 16, a.hidden, a.vec != 0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) kept[j] = w[8 + j];
        }
    }
    __device__ __forceinline__ void done() {}
};
template <>
constexpr bool hg_pairs<EpiGlu> = true;

// ------------------------------------------------------------------ few rows
// A warp takes C units, so 2 C rows of W (over ks warps of a CTA by pieces of 256 features, where there are few), and R
// rows of x at a time; its sums are exchanged so that each lane ends with one (row, unit, half).  W's bytes bound a lone row:
// 4096 x 4096 12.5 us, 5.4 TB/s (6.2 us from the second level cache).
struct FewGluArgs {
    int64_t ldx, ldw, ldo;
    int rows, features, hidden, ks, act;
    uint16_t* out;
    Saved saved;           // base null: not kept
    float scale;
};

template <typename T, int R, int C, bool VEC>
__global__ void __launch_bounds__(256, 2) k_glu_few(const T* x, const uint16_t* w, const FewGluArgs a) {
    constexpr int N = 2 * R * C, kLanes = 32 / N;     // lanes that hold the same sum
    __shared__ float sums[2][8][N];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = warp % a.ks, per = 8 / a.ks;
    const int groups = (a.hidden + C - 1) / C;
    int turn = 0;
    for (int g0 = blockIdx.x * per; g0 < groups; g0 += gridDim.x * per) {
        const int first = (g0 + warp / a.ks) * C;
        for (int r0 = 0; r0 < a.rows; r0 += R, turn ^= 1) {       // (W's rows are in the first level cache from the second time on)
            float acc[R][2 * C];
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i / (2 * C)][i % (2 * C)] = 0.0f;
            if (first < a.hidden) {
                const T* xr[R];
#pragma unroll
                for (int r = 0; r < R; ++r) xr[r] = x + min(r0 + r, a.rows - 1) * a.ldx;
                const uint16_t* wr[2 * C];
#pragma unroll
                for (int c = 0; c < 2 * C; ++c)
                    wr[c] = w + (min(first + c % C, a.hidden - 1) + (int64_t)(c / C) * a.hidden) * a.ldw;
                int piece = sub * 256;
                for (; piece + 256 <= a.features; piece += a.ks * 256)
                    few_step<T, R, 2 * C, VEC, true>(xr, wr, piece, lane, a.features, acc);
                if (piece < a.features) few_step<T, R, 2 * C, VEC, false>(xr, wr, piece, lane, a.features, acc);
            }
            float z = few_sum<N>(&acc[0][0], lane);
            if (a.ks > 1) {
                if (lane % kLanes == 0) sums[turn][warp][lane / kLanes] = z;
                __syncthreads();       // the other turn's sums are read by now
                if (sub == 0) {
                    z = sums[turn][warp][lane / kLanes];
                    for (int k = 1; k < a.ks; ++k) z += sums[turn][warp + k][lane / kLanes];
                }
            }
            z *= a.scale;
            const float up = __shfl_down_sync(0xffffffffu, z, C * kLanes);
            const int i = lane / kLanes, row = r0 + i / (2 * C), unit = first + i % C;
            if (sub == 0 && lane % kLanes == 0 && row < a.rows && unit < a.hidden) {
                const bool gate = i % (2 * C) < C;
                if (a.saved.base) {
                    int to_up;
                    float* dst = a.saved.at(unit, row, &to_up);
                    dst[gate ? 0 : to_up] = z;
                }
                if (gate) {
                    float v = 0.0f;
                    with_act(a.act, [&](auto act) { v = act_value<decltype(act)::value>(z); });
                    a.out[row * a.ldo + unit] = __bfloat16_as_ushort(__float2bfloat16_rn(v * up));
                }
            }
        }
    }
}

// ------------------------------------------------------------------ elementwise
// Rows as bf16 with a stride of ldp (a multiple of 8): int8 activations are exact in bf16.
struct PackJob {
    const void* x;
    int64_t ldx, rows, ldp;
    uint16_t* out;
    int cols, i8;
    int ctas;              // 0: nothing to do
};
template <typename T>
__device__ __forceinline__ void pack_rows(const PackJob& j, int cta) {
    const T* x = static_cast<const T*>(j.x);
    const int per = (int)(j.ldp / 8);
    const int64_t words = j.rows * per, step = (int64_t)j.ctas * 256, first = cta * (int64_t)256 + threadIdx.x;
    const bool vec = (((uintptr_t)x | (uintptr_t)(j.ldx * sizeof(T))) & (8 * sizeof(T) - 1)) == 0;
    RowWalk at(first, step, per);
    for (int64_t i = first; i < words; i += step, at.next()) {
        const int c = at.part * 8;
        const T* src = x + at.row * j.ldx + c;
        uint32_t w[4] = {0, 0, 0, 0};
        if constexpr (sizeof(T) == 2) {
            if (vec && c + 8 <= j.cols) {
                *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(src);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < j.cols) w[k >> 1] |= (uint32_t)src[k] << (16 * (k & 1));
            }
        } else {
            uint32_t b[2] = {0x80808080u, 0x80808080u};   // bytes hold x + 128
            if (vec && c + 8 <= j.cols) {
                const uint2 r = *reinterpret_cast<const uint2*>(src);
                b[0] ^= r.x;
                b[1] ^= r.y;
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < j.cols) b[k >> 2] ^= (uint32_t)(uint8_t)src[k] << (8 * (k & 3));
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = bf16x2(b[k >> 1], 2 * (k & 1));
        }
        reinterpret_cast<uint4*>(j.out)[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// D [rows][ldd] from saved and dout, and what its rounding left over `low` elements on (0: not kept): four units a
// thread, past the whole blocks one.
struct GradJob {
    Saved saved;
    const uint16_t* dout;
    int64_t lddout, rows, ldd, low;
    uint16_t* D;
    int hidden, act;
    int align;             // units that dout's rows and D's second half start at multiples of: 4, 2 or 1
    int ctas;
};
// N values of 16 bits at an address that is a multiple of `align` of them
template <int N>
__device__ __forceinline__ void store16(uint16_t* dst, const uint32_t* w, int align) {
    if (N == 4 && align >= 4) {
        *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    } else if (N == 4 && align == 2) {
        reinterpret_cast<uint32_t*>(dst)[0] = w[0];
        reinterpret_cast<uint32_t*>(dst)[1] = w[1];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) dst[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}
template <int N>
__device__ __forceinline__ void grad_units(const GradJob& job, int64_t row, int unit, const float* gate, int up) {
    constexpr int P = (N + 1) / 2;
    float2 a[P], b[P], g[P];
    const uint16_t* d = job.dout + row * job.lddout + unit;
    if constexpr (N == 4) {
        const float4 z = *reinterpret_cast<const float4*>(gate), y = *reinterpret_cast<const float4*>(gate + up);
        a[0] = make_float2(z.x, z.y), a[1] = make_float2(z.z, z.w);
        b[0] = make_float2(y.x, y.y), b[1] = make_float2(y.z, y.w);
        uint32_t w[2];
        if (job.align == 4) {
            *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(d);
        } else if (job.align == 2) {
            w[0] = reinterpret_cast<const uint32_t*>(d)[0];
            w[1] = reinterpret_cast<const uint32_t*>(d)[1];
        } else {
            w[0] = d[0] | (uint32_t)d[1] << 16;
            w[1] = d[2] | (uint32_t)d[3] << 16;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) g[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    } else {
        a[0] = make_float2(gate[0], 0.0f), b[0] = make_float2(gate[up], 0.0f), g[0] = make_float2(__uint_as_float((uint32_t)d[0] << 16), 0.0f);
    }
    with_act(job.act, [&](auto k) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float2 v;
            const float2 slope = act_slope<decltype(k)::value>(a[j], &v);
            a[j] = mul2(mul2(g[j], b[j]), slope);
            b[j] = mul2(g[j], v);
        }
    });
    uint16_t* dst = job.D + row * job.ldd + unit;
    for (int half = 0;; ++half) {
        uint32_t wa[P], wb[P];
#pragma unroll
        for (int j = 0; j < P; ++j) wa[j] = pack_bf16(a[j].x, a[j].y), wb[j] = pack_bf16(b[j].x, b[j].y);
        store16<N>(dst, wa, 4);
        store16<N>(dst + job.hidden, wb, job.align);
        if (job.low == 0 || half == 1) break;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            a[j] = sub2(a[j], make_float2(__uint_as_float(wa[j] << 16), __uint_as_float(wa[j] & 0xffff0000u)));
            b[j] = sub2(b[j], make_float2(__uint_as_float(wb[j] << 16), __uint_as_float(wb[j] & 0xffff0000u)));
        }
        dst += job.low;
    }
}
// units of a row that a thread takes, as items
__host__ __device__ __forceinline__ int grad_items(int hidden) { return hidden / 16 * 4 + hidden % 16; }
__device__ __forceinline__ void grad_rows(const GradJob& job, int cta) {
    const int per = grad_items(job.hidden), quads = job.saved.blocks() * 4;
    const int64_t items = job.rows * per, step = (int64_t)job.ctas * 256, first = cta * (int64_t)256 + threadIdx.x;
    RowWalk at(first, step, per);
    for (int64_t i = first; i < items; i += step, at.next()) {
        if (at.part < quads) {
            grad_units<4>(job, at.row, 4 * at.part, job.saved.line(at.part >> 2, at.row) + 4 * (at.part & 3), 16);
        } else {
            int up;
            const int unit = job.saved.blocks() * 16 + at.part - quads;
            const float* gate = job.saved.rest(unit, at.row, &up);
            grad_units<1>(job, at.row, unit, gate, up);
        }
    }
}

// All that goes before the products, each job on CTAs of its own: a launch costs as much as a small job.
__global__ void __launch_bounds__(256) k_glu_prep(const PackJob x, const PackJob w, const GradJob g) {
    pdl_wait();
    int cta = blockIdx.x;
    if (cta < g.ctas) {
        grad_rows(g, cta);
        return;
    }
    cta -= g.ctas;
    const PackJob& j = cta < x.ctas ? x : w;
    if (cta >= x.ctas) cta -= x.ctas;
    if (j.i8) pack_rows<int8_t>(j, cta);
    else pack_rows<uint16_t>(j, cta);
}

// Up to this many rows D is kept as two bf16 halves: the rounding of one entry, up to 2^-8 of
// it, can be most of a lone row's error, and averages out over more.
constexpr int kRowsWithLow = 32;
// Sums in two accumulators, added with rounding, from here on: the tensor cores cut off what 32 bits do not hold.
constexpr int kFoldFeatures = 2048;
constexpr int64_t kAccFloats = (int64_t)16 << 20;   // slices of dx: at most 64 MB together

}  // namespace
}  // namespace nitro

struct nitro_glu {
    int max_rows = 0, features = 0, hidden = 0;
    int64_t ldp = 0, ldd = 0, acc_floats = 0;
    uint16_t* xp = nullptr;     // [max_rows][ldp] bf16 copy of x where TMA cannot take its rows
    uint16_t* wp = nullptr;     // [2 hidden][ldp] copy of W likewise
    uint16_t* D = nullptr;
    float* acc = nullptr;
    StatusWord status;
    DeviceAllocs allocs;
};

namespace {

bool copies(const void* x, int type, int64_t ldx) { return type == NITRO_I8 || !tma_rows(x, ldx); }

// x and W as operands along K, copies where TMA cannot take their rows, and D's job, if there is one (g.rows > 0).
cudaError_t prepare(nitro_glu* h, const void* x, int x_type, int64_t ldx, const uint16_t* w, int64_t ldw, int rows, GradJob g,
                    cudaStream_t s, HgOperand* ox, HgOperand* ow) {
    PackJob jx{}, jw{};
    double bytes = 14.0 * g.rows * g.hidden;
    *ox = {x, h->features, rows, ldx, 1, 0};
    if (copies(x, x_type, ldx)) {
        jx = {x, ldx, rows, h->ldp, h->xp, h->features, x_type == NITRO_I8, 1};
        *ox = {h->xp, h->features, rows, h->ldp, 1, 0};
        bytes += (double)rows * h->features * (jx.i8 ? 3 : 4);
    }
    const int64_t rows_w = 2 * (int64_t)h->hidden;
    *ow = {w, h->features, rows_w, ldw, 1, 0};
    if (copies(w, NITRO_BF16, ldw)) {
        jw = {w, ldw, rows_w, h->ldp, h->wp, h->features, 0, 1};
        *ow = {h->wp, h->features, rows_w, h->ldp, 1, 0};
        bytes += 4.0 * rows_w * h->features;
    }
    const int64_t items[3] = {g.rows * grad_items(g.hidden), jx.ctas ? rows * (h->ldp / 8) : 0, jw.ctas ? rows_w * (h->ldp / 8) : 0};
    const int64_t all = items[0] + items[1] + items[2];
    if (all == 0) return cudaSuccess;
    // one wave of CTAs, shared out by their threads' work
    static std::atomic<int> resident{0};
    const int64_t wave = one_wave(k_glu_prep, resident, INT32_MAX);
    const auto share = [&](int64_t n) { return n ? (int)std::max<int64_t>(1, std::min<int64_t>((n + 255) / 256, wave * n / all)) : 0; };
    g.ctas = share(items[0]);
    jx.ctas = share(items[1]);
    jw.ctas = share(items[2]);
    ProfScope ps(K_GLU_PREP, s, 0.0, bytes);
    return launch_k(k_glu_prep, dim3(g.ctas + jx.ctas + jw.ctas), dim3(256), 0, s, jx, jw, g);
}

// Whether a forward goes to the CUDA cores: four rows always, up to 16 where W is small or TMA cannot take its rows.  us,
// k_glu_few and the tensor cores, features x hidden: 3 rows, 4096 x 4096 12.6 and 15; 5 to 8 rows 1000 x 1501 5.1 and 8.6, 2000 x
// 3000 12.4 and 13.2, 4096 x 4096 20 and 15.3, with odd rows 28 and 43; 9 to 16 rows 1000 x 1501 8.6 and 8.7, 4096 x 300 5.7 and 9.9, but 512 x
// 4096 7.2 and 6.0; with odd rows 1000 x 1501 9.7 and 12.7, 2000 x 3000 28 and 20.
bool few_rows_pay(const nitro_glu* h, int rows, bool copy) {
    const int64_t w = 2 * (int64_t)h->hidden * h->features, m = 1 << 20;
    return rows <= 4 || (rows <= 8 && (copy || w <= 8 * m)) || (rows <= 16 && w <= (copy ? 6 : 3) * m);
}

int rows_in_stage(int rows) { return rows < 128 ? (rows + 7) / 8 * 8 : 128; }

bool glu_args(const nitro_glu* h, const void* x, int x_type, int64_t ldx, const void* w, int64_t ldw, int rows, float scale,
              int act) {
    if (!h || rows < 0 || rows > h->max_rows || (x_type != NITRO_BF16 && x_type != NITRO_I8) || !act_known(act)) return false;
    if (ldx < h->features || ldw < h->features || !(scale > 0.0f) || scale > 1e30f) return false;
    if (rows > 0 && (!x || !w)) return false;
    return ((uintptr_t)w & 1) == 0 && (x_type == NITRO_I8 || ((uintptr_t)x & 1) == 0);
}

template <typename T, int R, int C>
cudaError_t few_as(bool vec, const void* x, const uint16_t* w, const FewGluArgs& a, int grid, cudaStream_t s) {
    return vec ? launch_k(k_glu_few<T, R, C, true>, dim3(grid), dim3(256), 0, s, (const T*)x, w, a)
               : launch_k(k_glu_few<T, R, C, false>, dim3(grid), dim3(256), 0, s, (const T*)x, w, a);
}
template <typename T>
cudaError_t few_rows(bool vec, int c, const void* x, const uint16_t* w, const FewGluArgs& a, int grid, cudaStream_t s) {
    if (a.rows > 4) return few_as<T, 8, 2>(vec, x, w, a, grid, s);
    if (c == 4) return a.rows <= 1 ? few_as<T, 1, 4>(vec, x, w, a, grid, s) : few_as<T, 4, 4>(vec, x, w, a, grid, s);
    return a.rows <= 1 ? few_as<T, 1, 1>(vec, x, w, a, grid, s) : few_as<T, 4, 1>(vec, x, w, a, grid, s);
}

cudaError_t forward_few(const nitro_glu* h, const void* x, int x_type, const uint16_t* w, FewGluArgs a, cudaStream_t s) {
    // two CTAs an SM; four units a warp (two of more than four rows) where that leaves no warp idle, else one; a warp's
    // features over as many warps as are free
    const int ctas = 2 * sm_count(), warps = 8 * ctas, pieces = (h->features + 255) / 256;
    const int c = a.rows > 4 ? 2 : (int64_t)((h->hidden + 3) / 4) * std::min(8, pieces) >= warps / 2 ? 4 : 1;
    const int groups = (h->hidden + c - 1) / c;
    a.ks = 1;
    while (a.ks < 8 && 2 * a.ks <= pieces && (int64_t)groups * 2 * a.ks <= warps) a.ks *= 2;
    const int per = 8 / a.ks, grid = std::min(ctas, (groups + per - 1) / per);
    const bool i8 = x_type == NITRO_I8;
    const bool vec = tma_rows(w, a.ldw) && (i8 ? ((uintptr_t)x & 7) == 0 && a.ldx % 8 == 0 : tma_rows(x, a.ldx));
    ProfScope ps(K_GLU_FWD, s, 4.0 * a.rows * h->hidden * h->features, 4.0 * h->hidden * h->features);
    return i8 ? few_rows<int8_t>(vec, c, x, w, a, grid, s) : few_rows<uint16_t>(vec, c, x, w, a, grid, s);
}

}  // namespace

extern "C" {

nitro_status nitro_glu_create(int max_rows, int features, int hidden, nitro_glu** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (max_rows < 1 || features < 1 || hidden < 1 || max_rows > (1 << 20) || features > (1 << 17) || hidden > (1 << 20) ||
        (int64_t)max_rows * std::max(features, hidden) > ((int64_t)1 << 34) || (int64_t)hidden * features > ((int64_t)1 << 34))
        return NITRO_ERR_ARG;
    nitro_glu* h = new (std::nothrow) nitro_glu();
    if (!h) return NITRO_ERR_CUDA;
    h->max_rows = max_rows;
    h->features = features;
    h->hidden = hidden;
    h->ldp = round_up(features, 8);
    h->ldd = round_up(2 * (int64_t)hidden, 8);
    h->acc_floats = std::min(16 * max_rows * round_up(features, 32), kAccFloats);
    const bool ok = h->allocs.take(&h->xp, max_rows * h->ldp) && h->allocs.take(&h->wp, 2 * hidden * h->ldp) &&
                    h->allocs.take(&h->D, std::max(max_rows, 2 * std::min(max_rows, kRowsWithLow)) * h->ldd) &&
                    h->allocs.take(&h->acc, h->acc_floats) && h->status.take();
    if (!ok) {
        nitro_glu_destroy(h);
        return NITRO_ERR_CUDA;
    }
    *out = h;
    return NITRO_OK;
}

nitro_status nitro_glu_forward(nitro_glu* h, const void* x, int x_type, int64_t ldx, const uint16_t* w, int64_t ldw, int rows,
                               float scale, int act, uint16_t* out, int64_t ldo, float* saved, void* stream) {
    if (!glu_args(h, x, x_type, ldx, w, ldw, rows, scale, act) || ldo < h->hidden) return NITRO_ERR_ARG;
    if (((uintptr_t)out & 1) || ((uintptr_t)saved & 15)) return NITRO_ERR_ARG;
    if (rows == 0) return NITRO_OK;
    if (!out) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (few_rows_pay(h, rows, copies(w, NITRO_BF16, ldw))) {
        TRY(forward_few(h, x, x_type, w, FewGluArgs{ldx, ldw, ldo, rows, h->features, h->hidden, 1, act, out, Saved{saved, rows, h->hidden}, scale}, s));
        return NITRO_OK;
    }
    HgOperand ox, ow;
    TRY(prepare(h, x, x_type, ldx, w, ldw, rows, GradJob{}, s, &ox, &ow));
    ow = {ow.base, ow.inner, h->hidden, ow.ld, 2, h->hidden * ow.ld};
    HgProblem p{rows, 2 * round_up(h->hidden, 16), h->features};
    p.status = h->status.at;
    p.prof = K_GLU_FWD;
    p.ops = 4.0 * rows * h->hidden * h->features;
    p.fold = h->features > kFoldFeatures;
    p.rows_a = rows_in_stage(rows);
    p.eights = hg_eights();
    const EpiGlu::Args ea{out, ldo, Saved{saved, rows, h->hidden}, tma_rows(out, ldo), h->hidden, act, scale};
    TRY((hg_launch<EpiGlu, false, false, false>(hg_pick(p), p, ox, ow, ea, s)));
    return NITRO_OK;
}

nitro_status nitro_glu_backward(nitro_glu* h, const void* x, int x_type, int64_t ldx, const uint16_t* w, int64_t ldw, int rows,
                                float scale, int act, const float* saved, const uint16_t* dout, int64_t lddout, uint16_t* dx,
                                int64_t lddx, uint16_t* dw, int64_t lddw, void* stream) {
    if (!glu_args(h, x, x_type, ldx, w, ldw, rows, scale, act) || lddout < h->hidden) return NITRO_ERR_ARG;
    if ((dx && (lddx < h->features || ((uintptr_t)dx & 1))) || (dw && (lddw < h->features || ((uintptr_t)dw & 1))))
        return NITRO_ERR_ARG;
    if (rows > 0 && (!saved || !dout || ((uintptr_t)saved & 15) || ((uintptr_t)dout & 1))) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int F = h->features;
    const int64_t H2 = 2 * (int64_t)h->hidden;
    if (rows == 0) {   // an empty batch has a weight gradient of zero
        if (dw && lddw == F) {
            TRY(cudaMemsetAsync(dw, 0, sizeof(uint16_t) * (size_t)(H2 * F), s));
        } else if (dw) {
            static std::atomic<int> resident{0};
            ProfScope ps(K_GLU_DW, s, 0.0, 2.0 * H2 * F);
            TRY(launch_k(k_head_zero, dim3(one_wave(k_head_zero, resident, H2 * F)), dim3(256), 0, s, dw, lddw, H2, F));
        }
        return NITRO_OK;
    }
    if (!dx && !dw) return NITRO_OK;
    const int halves = rows <= kRowsWithLow ? 2 : 1;
    const int64_t plane = rows * h->ldd;
    const uintptr_t starts = (uintptr_t)dout | (uintptr_t)(lddout * 2) | (uintptr_t)h->hidden * 2;
    const int align = starts % 8 == 0 ? 4 : starts % 4 == 0 ? 2 : 1;
    const GradJob g{Saved{const_cast<float*>(saved), rows, h->hidden}, dout, lddout, rows, h->ldd, halves == 2 ? plane : 0, h->D, h->hidden, act, align, 0};
    HgOperand ox, ow;
    TRY(prepare(h, x, x_type, ldx, w, ldw, rows, g, s, &ox, &ow));
    const HgOperand D{h->D, H2, rows, h->ldd, halves, plane};
    if (dx) {
        HgProblem p{rows, F, H2};
        p.planes_a = halves;
        p.status = h->status.at;
        p.prof = K_GLU_DX;
        p.ops = 4.0 * rows * h->hidden * F;
        p.rows_a = rows_in_stage(rows);
        p.eights = hg_eights();
        // in slices along the hidden units where its tiles leave SMs idle
        const int64_t ldc = round_up(F, 32);
        const HgPick t = hg_pick(p, halves, 1, (int)std::max<int64_t>(1, std::min<int64_t>(16, h->acc_floats / (rows * ldc))));
        if (t.splits == 1) {
            const EpiBf16::Args eb{dx, lddx, tma_rows(dx, lddx), nullptr, 0, scale};
            if (halves == 2) TRY((hg_launch<EpiBf16, false, true, false, 2, 1>(t, p, D, ow, eb, s)));
            else TRY((hg_launch<EpiBf16, false, true, false>(t, p, D, ow, eb, s)));
        } else {
            const EpiAcc::Args ea{h->acc, ldc, rows * ldc, 0};
            if (halves == 2) TRY((hg_launch<EpiAcc, false, true, false, 2, 1>(t, p, D, ow, ea, s)));
            else TRY((hg_launch<EpiAcc, false, true, false>(t, p, D, ow, ea, s)));
            ProfScope ps(K_GLU_DX, s, 0.0, (4.0 * t.splits + 2.0) * rows * F);
            TRY(launch_k(k_head_slices, dim3(rows, (unsigned)std::min(8, (F + 1023) / 1024)), dim3(256), 0, s, (const float*)h->acc, ldc,
                         rows * ldc, t.splits, F, (const float*)nullptr, scale, dx, lddx,
                         (int)(((uintptr_t)dx & 7) == 0 && lddx % 4 == 0)));
        }
    }
    if (dw) {
        HgProblem p{H2, F, rows};
        p.planes_a = halves;
        p.status = h->status.at;
        p.prof = K_GLU_DW;
        p.ops = 4.0 * rows * h->hidden * F;
        p.eights = hg_eights();
        const EpiBf16::Args eb{dw, lddw, tma_rows(dw, lddw), nullptr, 0, scale};
        if (halves == 2) TRY((hg_launch<EpiBf16, true, true, false, 2, 1>(hg_pick(p, 2), p, D, ox, eb, s)));
        else TRY((hg_launch<EpiBf16, true, true, false>(hg_pick(p), p, D, ox, eb, s)));
    }
    return NITRO_OK;
}

nitro_status nitro_glu_status(nitro_glu* h, int clear) {
    if (!h) return NITRO_ERR_ARG;
    uint32_t bits = 0;
    if (!h->status.read(clear != 0, &bits)) return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_glu_destroy(nitro_glu* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    h->allocs.free();
    h->status.free();
    delete h;
}

}  // extern "C"
