// Group norm with an activation on channels-last maps x [samples][pixels][channels]: per sample and group of
// neighbouring channels mean m and variance v over N = pixels channels / groups values, r = 1 / sqrt(v + eps),
//   h = (x - m) r,  u = gamma h + beta,  y = act(u);
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du h,  t = gamma du,
//   dx = r (t - sum_g t / N - h sum_g (t h) / N).
//
// A thread keeps V neighbouring channels and goes along the pixels.  Where a cluster's shared memory holds a slab of a sample, a
// direction is one launch and one pass over memory (k_gn_one, k_gn_one_back): 128 x 4096 x 256 bf16 with silu 112 us forward,
// 4.8 TB/s, and 244 backward, 3.3, where a pass for the sums and one for the result took 1092 together.  17 and 29 instructions a
// value bound them, a third to a half of those the joining of sums, and 24 and 16 warps an SM.  Larger slabs take the
// two passes, over batches of samples that stay in L2 in between; the last CTA of a sample joins its chunks' sums.
//
// A thread's sums are of distances to its first value, and parts are joined as (count, mean, sum of squared distances) with
// means taken from the group's first value, so a mean far from zero costs the variance no digits.
#include <new>

#include "head_act.cuh"

using namespace nitro;

namespace nitro {
namespace {

constexpr int kGnThreads = 256;
constexpr int kGnBatch = 1024;                 // samples of a launch, at most
constexpr int kGnCtas = 608;                   // CTAs of a launch of two passes, unless there are more samples: four an SM
constexpr int64_t kGnBatchBytes = (int64_t)100 << 20;
constexpr int kGnChannels = 8192;

// V values of a row as fp32 pairs (of one value: itself and 0); rows are aligned to V values
template <typename T, int V>
struct Vals {
    static constexpr int N = (V + 1) / 2;
    static __device__ __forceinline__ void load(const T* p, float2* v) {
        if constexpr (V == 1) {
            v[0].y = 0.0f;
            if constexpr (sizeof(T) == 1) v[0].x = (float)(*reinterpret_cast<const int8_t*>(p));
            else if constexpr (sizeof(T) == 2) v[0].x = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
            else v[0].x = *reinterpret_cast<const float*>(p);
        } else {
            constexpr int W = V * (int)sizeof(T) / 4;      // words
            uint32_t w[W];
            if constexpr (W % 4 == 0) {
#pragma unroll
                for (int i = 0; i < W / 4; ++i) *reinterpret_cast<uint4*>(w + 4 * i) = reinterpret_cast<const uint4*>(p)[i];
            } else if constexpr (W == 2) {
                *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
            } else {
                w[0] = *reinterpret_cast<const uint32_t*>(p);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if constexpr (sizeof(T) == 1) {        // 2^23 + (v + 128) as a float has v + 128 in its low byte
                    const uint32_t b = w[j >> 1] ^ 0x80808080u;
                    v[j] = add2(make_float2(__uint_as_float(__byte_perm(b, 0x4B000000u, 0x7540 + 2 * (j & 1))),
                                            __uint_as_float(__byte_perm(b, 0x4B000000u, 0x7541 + 2 * (j & 1)))),
                                pair(-8388736.0f));
                } else if constexpr (sizeof(T) == 2) {
                    v[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
                } else {
                    v[j] = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
                }
            }
        }
    }
    static __device__ __forceinline__ void store(T* p, const float2* v) {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p) = __bfloat16_as_ushort(__float2bfloat16_rn(v[0].x));
            else *reinterpret_cast<float*>(p) = v[0].x;
        } else {
            constexpr int W = V * (int)sizeof(T) / 4;
            uint32_t w[W];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if constexpr (sizeof(T) == 2) w[j] = pack_bf16(v[j].x, v[j].y);
                else w[2 * j] = __float_as_uint(v[j].x), w[2 * j + 1] = __float_as_uint(v[j].y);
            }
            if constexpr (W % 4 == 0) {
#pragma unroll
                for (int i = 0; i < W / 4; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
            } else {
                *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
            }
        }
    }
};
// A channel's group and its place there; per: channels of a group
struct GnGroup {
    int g, r, per;
    // f(j, group) for V channels from there on; alike: they are of one group
    template <int V, class F>
    __device__ __forceinline__ void each(bool alike, F&& f) const {
        int gj = g, rj = r;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            f(j, gj);
            if (!alike && ++rj == per) rj = 0, ++gj;
        }
    }
};
__device__ __forceinline__ float& at2(float2* v, int j) { return j & 1 ? v[j >> 1].y : v[j >> 1].x; }

// A thread's channels: statistics of their groups, gamma and beta
template <int V>
struct GnChannels {
    static constexpr int N = (V + 1) / 2;
    alignas(16) float2 gamma[N + (N & 1)], beta[N + (N & 1)];
    float2 m[N], r[N];
    static __device__ __forceinline__ void param(const float* p, float none, int c, float2* v) {
        if (p && V > 1 && ((uintptr_t)p & 15) == 0) {
#pragma unroll
            for (int j = 0; j < N; j += 2) *reinterpret_cast<float4*>(v + j) = *reinterpret_cast<const float4*>(p + c + 2 * j);
        } else {
#pragma unroll
            for (int j = 0; j < 2 * N; ++j) at2(v, j) = p && j < V ? p[c + j] : none;
        }
    }
    __device__ __forceinline__ void params(int c, const float* g, const float* b) {
        param(g, 1.0f, c, gamma);
        param(b, 0.0f, c, beta);
    }
    // statistics of a sample's groups
    __device__ __forceinline__ void stats(const GnGroup& at, bool alike, const float* mean, const float* rstd) {
        if (alike) {
            const float a = mean[at.g], b = rstd[at.g];
#pragma unroll
            for (int j = 0; j < N; ++j) m[j] = pair(a), r[j] = pair(b);
            return;
        }
        m[N - 1].y = r[N - 1].y = 0.0f;
        at.each<V>(false, [&](int j, int g) {
            at2(m, j) = mean[g];
            at2(r, j) = rstd[g];
        });
    }
    // act(gamma r (x - m) + beta), r times gamma in r
    template <int ACT>
    __device__ __forceinline__ void apply(float2* x) const {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = act_value<ACT>(fma2(sub2(x[j], m[j]), r[j], beta[j]));
    }
    // x to h, dy to du
    template <int ACT>
    __device__ __forceinline__ void slopes(float2* x, float2* dy) const {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float2 value;
            x[j] = mul2(sub2(x[j], m[j]), r[j]);
            dy[j] = mul2(dy[j], act_slope<ACT>(fma2(gamma[j], x[j], beta[j]), &value));
        }
    }
    // dx = r (gamma du - u - h v) of group means u and v, as (gamma r) du - (x - m) r^2 v - r u: to gamma, r and beta
    __device__ __forceinline__ void to_dx(const float2* u, const float2* v) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            gamma[j] = mul2(gamma[j], r[j]);
            beta[j] = mul2(mul2(r[j], u[j]), pair(-1.0f));
            r[j] = mul2(mul2(r[j], mul2(r[j], v[j])), pair(-1.0f));
        }
    }
    __device__ __forceinline__ void dx(float2* x, const float2* du) const {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = fma2(du[j], gamma[j], fma2(sub2(x[j], m[j]), r[j], beta[j]));
    }
};

// (count, mean, sum of squared distances) joined with another's
struct Moments {
    float n = 0.0f, m = 0.0f, q = 0.0f;
    __device__ __forceinline__ void add(float on, float om, float oq) {
        const float t = n + on, w = t > 0.0f ? on * rcp(t) : 0.0f, diff = om - m;
        q += oq + diff * diff * (n * w);
        m = fmaf(diff, w, m);
        n = t;
    }
    // with those of the lanes at distances first .. last (powers of two)
    __device__ __forceinline__ void join(int first, int last) {
        for (int d = first; d <= last; d <<= 1)
            add(__shfl_xor_sync(0xffffffffu, n, d), __shfl_xor_sync(0xffffffffu, m, d), __shfl_xor_sync(0xffffffffu, q, d));
    }
};

// Sums of a thread's values in V channels, from its first ones on
template <int V>
struct Sums {
    static constexpr int N = (V + 1) / 2;
    float2 k[N], sum[N], sq[N];
    __device__ __forceinline__ Sums() {
#pragma unroll
        for (int j = 0; j < N; ++j) k[j] = sum[j] = sq[j] = pair(0.0f);
    }
    // a run's sums to these: long ones go by runs, as squares far below a sum's last place are lost
    // more often than they are rounded up
    __device__ __forceinline__ void take(Sums& run) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            sum[j] = add2(sum[j], run.sum[j]);
            sq[j] = add2(sq[j], run.sq[j]);
            run.sum[j] = run.sq[j] = pair(0.0f);
        }
    }
    __device__ __forceinline__ void add(const float2* v) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float2 d = sub2(v[j], k[j]);
            sum[j] = add2(sum[j], d);
            sq[j] = fma2(d, d, sq[j]);
        }
    }
    // to means, from origin(group) on, in sum and squared distances in sq, of n values
    template <class F>
    __device__ __forceinline__ void finish(float n, const GnGroup& at, bool alike, F&& origin) {
        const float one = n > 0.0f ? rcp(n) : 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float2 m = mul2(sum[j], pair(one));
            sq[j] = fma2(mul2(m, pair(-1.0f)), sum[j], sq[j]);
            sq[j] = make_float2(sq[j].x < 0.0f ? 0.0f : sq[j].x, sq[j].y < 0.0f ? 0.0f : sq[j].y);     // (a NaN stays)
            sum[j] = m;
        }
        const float first = origin(at.g);
        at.each<V>(alike, [&](int j, int g) { at2(sum, j) = n > 0.0f ? at2(sum, j) + (at2(k, j) - (alike ? first : origin(g))) : 0.0f; });
    }
};

// A vector's place in shared memory: planes of 16 bytes a thread (or less, the vector itself)
template <typename T, int V>
struct Slots {
    static constexpr int BYTES = V * (int)sizeof(T), PLANE = BYTES < 16 ? BYTES : 16, PLANES = BYTES / PLANE;
    static constexpr int STEP = kGnThreads * BYTES;          // from a thread's vector to its next
    static __device__ __forceinline__ uint8_t* first(uint8_t* base) { return base + (int)threadIdx.x * PLANE; }
    // Place: whose places the vector takes, its own or those of wider values that replace it later
    template <class Place = Slots>
    static __device__ __forceinline__ void fetch(uint8_t* to, const T* src) {
        if constexpr (PLANE < 4) {
            *reinterpret_cast<T*>(to) = *src;
        } else {
#pragma unroll
            for (int i = 0; i < PLANES; ++i) {
                const uint32_t dst = smem_u32(to + i * kGnThreads * Place::PLANE);
                const char* s = reinterpret_cast<const char*>(src) + i * PLANE;
                if constexpr (PLANE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(s) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(s), "n"(PLANE) : "memory");
            }
        }
    }
    template <class Place = Slots>
    static __device__ __forceinline__ void get(const uint8_t* from, float2* v) {
#pragma unroll
        for (int i = 0; i < PLANES; ++i)
            Vals<T, V / PLANES>::load(reinterpret_cast<const T*>(from + i * kGnThreads * Place::PLANE), v + i * (V / PLANES / 2));
    }
    static __device__ __forceinline__ void put(uint8_t* to, const float2* v) {
#pragma unroll
        for (int i = 0; i < PLANES; ++i)
            Vals<T, V / PLANES>::store(reinterpret_cast<T*>(to + i * kGnThreads * PLANE), v + i * (V / PLANES / 2));
    }
};
__device__ __forceinline__ void copies_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// ------------------------------------------------------------------ two passes
// fetch(i, s) for i = 0 .. n - 1 starts the copies of a thread's step i to its place s of a ring, use(i, s) works on them.
constexpr int kRingGroups = 3, kRingGroup = 2, kRing = kRingGroups * kRingGroup;
template <class Fetch, class Use>
__device__ __forceinline__ void through_ring(int n, Fetch&& fetch, Use&& use) {
    const auto group = [&](int i, int s) {
#pragma unroll
        for (int k = 0; k < kRingGroup; ++k)
            if (i + k < n) fetch(i + k, s + k);
        copies_group();
    };
#pragma unroll
    for (int g = 0; g < kRingGroups; ++g) group(g * kRingGroup, g * kRingGroup);
    for (int i = 0, s = 0; i < n; i += kRingGroup) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kRingGroups - 1) : "memory");
#pragma unroll
        for (int k = 0; k < kRingGroup; ++k)
            if (i + k < n) use(i + k, s + k);
        group(i + kRing, s);
        s = s + kRingGroup == kRing ? 0 : s + kRingGroup;
    }
}

// CTAs of a backward pass that an SM holds by their registers
constexpr int gn_resident(int v) { return v == 8 ? 2 : 4; }

// What is common to the four passes.
struct GnShape {
    int pixels, channels, groups, per;   // per: channels of a group
    int chunk, chunks;                   // pixels of a CTA, CTAs of a sample
    int vecs, slabs, rows;               // vectors of a pixel that a CTA takes at once, how often, pixels at once
    int act;
    const float* gamma;                  // or null
    const float* beta;                   // or null
};

// A thread's place: vector `vec` of a slab, pixel `row` of those that a CTA takes at once
struct GnPlace {
    int row, vec;
    bool live;
    __device__ __forceinline__ GnPlace(const GnShape& s) {
        row = (int)threadIdx.x / s.vecs;
        vec = (int)threadIdx.x - row * s.vecs;
        live = row < s.rows;
    }
    // first channel in slab i, or -1
    template <int V>
    __device__ __forceinline__ int channel(const GnShape& s, int i) const {
        const int c = (i * s.vecs + vec) * V;
        return live && c < s.channels ? c : -1;
    }
    // pixels of np that the thread takes
    __device__ __forceinline__ int steps(const GnShape& s, int np) const { return row < np ? (np - row + s.rows - 1) / s.rows : 0; }
    __device__ __forceinline__ GnGroup group(const GnShape& s, int c) const {
        const int g = c / s.per;
        return {g, c - g * s.per, s.per};
    }
};

// Every thread of a sample's CTAs, their parts written: true in the last to come here.
__device__ __forceinline__ bool gn_last(uint32_t* ticket, int chunks, int* word) {
    if (chunks == 1) {
        __syncthreads();
        return true;
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t n = atomicAdd(ticket, 1u);
        if (n == (uint32_t)chunks - 1) *ticket = 0;
        *word = n == (uint32_t)chunks - 1;
    }
    __syncthreads();
    __threadfence();
    return *word;
}

// mean and rstd of a sample's groups.  Dynamic shared memory: the ring, two values a channel.
template <typename X, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_stats(const X* x, int64_t ldx, int64_t sx, const GnShape s, float eps, float2* parts,
                                                         uint32_t* ticket, float* mean, float* rstd) {
    using SX = Slots<X, V>;
    extern __shared__ __align__(16) uint8_t data[];
    float* chan = reinterpret_cast<float*>(data + kRing * SX::STEP);      // [channels] means, [channels] squared distances
    __shared__ float red[2][kGnThreads * V];          // [rows][slab's channels]
    __shared__ int word;
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    const int width = s.vecs * V;
    x += sample * sx;
    const auto origin = [&](int g) {         // what a group's means are taken from
        float2 k;
        Vals<X, 1>::load(x + g * s.per, &k);
        return k.x;
    };
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c >= 0) {
            Sums<V> t, run;
            const X* src = x + (int64_t)(p0 + at.row) * ldx + c;
            if (at.row < np) Vals<X, V>::load(src, t.k);
#pragma unroll
            for (int j = 0; j < t.N; ++j) run.k[j] = t.k[j];
            const int64_t step = s.rows * ldx;
            const int n = at.steps(s, np);
            uint8_t* slot = SX::first(data);
            through_ring(
                n, [&](int i, int k) { SX::fetch(slot + k * SX::STEP, src + i * step); },
                [&](int i, int k) {
                    float2 v[Sums<V>::N];
                    SX::get(slot + k * SX::STEP, v);
                    run.add(v);
                    if ((i & 31) == 31) t.take(run);
                });
            t.take(run);
            t.finish((float)n, at.group(s, c), s.per % V == 0, origin);      // 0 for rows past the chunk
#pragma unroll
            for (int j = 0; j < V; ++j) {
                red[0][at.row * width + at.vec * V + j] = at2(t.sum, j);
                red[1][at.row * width + at.vec * V + j] = at2(t.sq, j);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < width; i += blockDim.x) {
            const int ch = slab * width + i;
            if (ch >= s.channels) break;
            Moments a;
            for (int r = 0; r < min(s.rows, np); ++r)
                a.add((float)((np - r + s.rows - 1) / s.rows), red[0][r * width + i], red[1][r * width + i]);
            chan[ch] = a.m;
            chan[s.channels + ch] = a.q;
        }
        __syncthreads();
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    parts += (int64_t)sample * s.chunks * s.groups;
    for (int g = warp; g < s.groups; g += warps) {
        Moments a;
        for (int c = lane; c < s.per; c += 32) a.add((float)np, chan[g * s.per + c], chan[s.channels + g * s.per + c]);
        a.join(1, 16);
        if (lane == 0) parts[(int64_t)blockIdx.x * s.groups + g] = make_float2(a.m, a.q);
    }
    if (!gn_last(ticket + sample, s.chunks, &word)) return;
    for (int g = warp; g < s.groups; g += warps) {
        Moments a;
#pragma unroll 4
        for (int i = lane; i < s.chunks; i += 32) {
            const float2 v = __ldcg(parts + (int64_t)i * s.groups + g);
            a.add((float)(min(s.chunk, s.pixels - i * s.chunk)) * (float)s.per, v.x, v.y);
        }
        a.join(1, 16);
        if (lane == 0) {
            mean[(int64_t)sample * s.groups + g] = origin(g) + a.m;
            rstd[(int64_t)sample * s.groups + g] = 1.0f / sqrtf(a.q / a.n + eps);
        }
    }
}

template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_apply(const X* x, int64_t ldx, int64_t sx, const GnShape s, const float* mean,
                                                         const float* rstd, Y* y, int64_t ldy, int64_t sy) {
    using SX = Slots<X, V>;
    extern __shared__ __align__(16) uint8_t data[];
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c < 0) continue;
        GnChannels<V> ch;
        ch.params(c, s.gamma, s.beta);
        ch.stats(at.group(s, c), s.per % V == 0, mean + (int64_t)sample * s.groups, rstd + (int64_t)sample * s.groups);
#pragma unroll
        for (int j = 0; j < ch.N; ++j) ch.r[j] = mul2(ch.r[j], ch.gamma[j]);
        const X* src = x + sample * sx + (int64_t)(p0 + at.row) * ldx + c;
        Y* dst = y + sample * sy + (int64_t)(p0 + at.row) * ldy + c;
        const int64_t xs = s.rows * ldx, ys = s.rows * ldy;
        with_act(s.act, [&](auto act) {
            uint8_t* slot = SX::first(data);
            through_ring(
                at.steps(s, np), [&](int i, int k) { SX::fetch(slot + k * SX::STEP, src + i * xs); },
                [&](int i, int k) {
                    float2 v[ch.N];
                    SX::get(slot + k * SX::STEP, v);
                    ch.template apply<decltype(act)::value>(v);
                    Vals<Y, V>::store(dst + i * ys, v);
                });
        });
    }
}

// Sums over a chunk: of du and du h for each channel (part_c [sample][chunk][2][channels]), and over a sample's
// groups of gamma du and gamma du h, divided by their count (means [sample][groups]).
template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads, gn_resident(V)) k_gn_sums(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                           const GnShape s, const float* mean, const float* rstd, float* part_c,
                                                           float2* parts, uint32_t* ticket, float2* means) {
    using SX = Slots<X, V>;
    using SY = Slots<Y, V>;
    extern __shared__ __align__(16) uint8_t data[];
    uint8_t *xslot = SX::first(data), *gslot = SY::first(data + kRing * SX::STEP);
    __shared__ float red[2][kGnThreads * V];
    __shared__ int word;
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    const int width = s.vecs * V;
    float* out = part_c + ((int64_t)sample * s.chunks + blockIdx.x) * 2 * s.channels;
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c >= 0) {
            GnChannels<V> ch;
            ch.params(c, s.gamma, s.beta);
            ch.stats(at.group(s, c), s.per % V == 0, mean + (int64_t)sample * s.groups, rstd + (int64_t)sample * s.groups);
            float2 a[ch.N], b[ch.N];
#pragma unroll
            for (int j = 0; j < ch.N; ++j) a[j] = b[j] = pair(0.0f);
            const X* src = x + sample * sx + (int64_t)(p0 + at.row) * ldx + c;
            const Y* grad = dy + sample * sdy + (int64_t)(p0 + at.row) * lddy + c;
            const int64_t xs = s.rows * ldx, gs = s.rows * lddy;
            with_act(s.act, [&](auto act) {
                through_ring(
                    at.steps(s, np),
                    [&](int i, int k) {
                        SX::fetch(xslot + k * SX::STEP, src + i * xs);
                        SY::fetch(gslot + k * SY::STEP, grad + i * gs);
                    },
                    [&](int, int k) {
                        float2 v[ch.N], g[ch.N];
                        SX::get(xslot + k * SX::STEP, v);
                        SY::get(gslot + k * SY::STEP, g);
                        ch.template slopes<decltype(act)::value>(v, g);
#pragma unroll
                        for (int j = 0; j < ch.N; ++j) {
                            a[j] = add2(a[j], g[j]);
                            b[j] = fma2(g[j], v[j], b[j]);
                        }
                    });
            });
#pragma unroll
            for (int j = 0; j < V; ++j) {
                red[0][at.row * width + at.vec * V + j] = at2(a, j);
                red[1][at.row * width + at.vec * V + j] = at2(b, j);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * width; i += blockDim.x) {
            const int half = i >= width, k = i - half * width, chn = slab * width + k;
            if (chn >= s.channels) continue;
            float v = 0.0f;
            for (int r = 0; r < s.rows; ++r) v += red[half][r * width + k];
            out[half * s.channels + chn] = v;
        }
        __syncthreads();
    }
    if (!means) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    parts += (int64_t)sample * s.chunks * s.groups;
    for (int g = warp; g < s.groups; g += warps) {
        float a = 0.0f, b = 0.0f;
        for (int i = lane; i < s.per; i += 32) {
            const int c = g * s.per + i;
            const float k = s.gamma ? s.gamma[c] : 1.0f;
            a = fmaf(k, out[c], a);
            b = fmaf(k, out[s.channels + c], b);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d), b += __shfl_xor_sync(0xffffffffu, b, d);
        if (lane == 0) parts[(int64_t)blockIdx.x * s.groups + g] = make_float2(a, b);
    }
    if (!gn_last(ticket + sample, s.chunks, &word)) return;
    const float count = (float)s.pixels * (float)s.per;
    for (int g = warp; g < s.groups; g += warps) {
        float a = 0.0f, b = 0.0f;
#pragma unroll 4
        for (int i = lane; i < s.chunks; i += 32) {
            const float2 v = __ldcg(parts + (int64_t)i * s.groups + g);
            a += v.x;
            b += v.y;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d), b += __shfl_xor_sync(0xffffffffu, b, d);
        if (lane == 0) means[(int64_t)sample * s.groups + g] = make_float2(a / count, b / count);
    }
}

template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads, gn_resident(V)) k_gn_dx(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                         const GnShape s, const float* mean, const float* rstd, const float2* means,
                                                         Y* dx, int64_t lddx, int64_t sdx) {
    using SX = Slots<X, V>;
    using SY = Slots<Y, V>;
    extern __shared__ __align__(16) uint8_t data[];
    uint8_t *xslot = SX::first(data), *gslot = SY::first(data + kRing * SX::STEP);
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c < 0) continue;
        GnChannels<V> ch, to;
        ch.params(c, s.gamma, s.beta);
        ch.stats(at.group(s, c), s.per % V == 0, mean + (int64_t)sample * s.groups, rstd + (int64_t)sample * s.groups);
        to = ch;
        {
            float2 u[ch.N], v[ch.N];
            u[ch.N - 1].y = v[ch.N - 1].y = 0.0f;
            at.group(s, c).template each<V>(s.per % V == 0, [&](int j, int g) {
                const float2 t = means[(int64_t)sample * s.groups + g];
                at2(u, j) = t.x;
                at2(v, j) = t.y;
            });
            to.to_dx(u, v);
        }
        const X* src = x + sample * sx + (int64_t)(p0 + at.row) * ldx + c;
        const Y* grad = dy + sample * sdy + (int64_t)(p0 + at.row) * lddy + c;
        Y* dst = dx + sample * sdx + (int64_t)(p0 + at.row) * lddx + c;
        const int64_t xs = s.rows * ldx, gs = s.rows * lddy, ds = s.rows * lddx;
        with_act(s.act, [&](auto act) {
            through_ring(
                at.steps(s, np),
                [&](int i, int k) {
                    SX::fetch(xslot + k * SX::STEP, src + i * xs);
                    SY::fetch(gslot + k * SY::STEP, grad + i * gs);
                },
                [&](int i, int k) {
                    float2 v[ch.N], h[ch.N], g[ch.N];
                    SX::get(xslot + k * SX::STEP, v);
                    SY::get(gslot + k * SY::STEP, g);
#pragma unroll
                    for (int j = 0; j < ch.N; ++j) h[j] = v[j];
                    ch.template slopes<decltype(act)::value>(h, g);
                    to.dx(v, g);
                    Vals<Y, V>::store(dst + i * ds, v);
                });
        });
    }
}

// ------------------------------------------------------------------ one pass
// Both directions in one launch with one pass over memory, where a cluster's shared memory holds a slab of a sample: whole
// groups, `width` channels at all pixels, shared out over ks CTAs by pixels.  A thread copies its own vectors to
// shared memory and alone reads them there, so nothing waits for them but itself; channels' sums meet in the
// warp's lanes, over the CTA's warps, and over the cluster's shared memory.
//
// Lanes: 2^k >= width / V to a pixel (those past the width idle), so the lanes of a channel are found by shuffles.
constexpr int kGnWarps = kGnThreads / 32;
struct GnOne {
    int pixels, channels, groups, per;
    int width, gs, slabs, ks;            // channels and groups of a slab, slabs of a sample, CTAs of a cluster
    int vecs, lane_log;                  // vectors of a slab's pixel, and the lanes' logarithm
    int chunk, steps;                    // pixels of a CTA, of which a thread takes every (256 / lanes)th
    int alike, entries;                  // vectors are of one group each; a group's vectors, or its channels where they are not
    FloorDiv32 by_per;
    int act;
    const float* gamma;                  // or null
    const float* beta;                   // or null
};

// A thread's copies go in up to kGnStages groups, so that the first are taken while the others are under way
constexpr int kGnStages = 4;
__device__ __forceinline__ void copies_landed(int stage) {
    if (stage == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (stage == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stage == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// p of the cluster's `ks` CTAs, all loads under way together
__device__ __forceinline__ void ld_remote(const float* p, int ks, float* v) {
    const uint32_t at = smem_u32(p);
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (r < ks) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(remote_smem(at, r)) : "memory");
}
// (nothing is handed over: peers learn that their shared memory has been read)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }

// A thread's part of a slab.  Grid: (slabs ks, samples)
struct GnPart {
    int sample, rank, c, g0, row, rows;           // first channel (-1: idle lane), the slab's first group, first pixel of the chunk's, step
    int count, stage;                             // pixels that the thread takes, of a stage
    int64_t p0;
    GnGroup group;                                // of the first channel
    __device__ __forceinline__ GnPart(const GnOne& s, int v) {
        const int slab = blockIdx.x / (unsigned)s.ks, vec = threadIdx.x & ((1 << s.lane_log) - 1);
        rank = blockIdx.x - slab * s.ks;
        sample = blockIdx.y;
        row = threadIdx.x >> s.lane_log;
        rows = kGnThreads >> s.lane_log;
        const int first = slab * s.width + min(vec, s.vecs - 1) * v, g = s.by_per.udiv(first);
        group = {g, first - g * s.per, s.per};
        c = vec < s.vecs ? first : -1;
        g0 = slab * s.gs;
        p0 = (int64_t)rank * s.chunk;
        const int np = min(s.chunk, s.pixels - rank * s.chunk);
        count = c >= 0 && row < np ? (np - row + rows - 1) >> (8 - s.lane_log) : 0;
        stage = (s.steps + kGnStages - 1) / kGnStages;
    }
};
static_assert(kGnThreads == 256, "rows are 256 / lanes");

template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads, 3) k_gn_one(const X* x, int64_t ldx, int64_t sx, const GnOne s, float eps, float* mean,
                                                          float* rstd, Y* y, int64_t ldy, int64_t sy) {
    using SX = Slots<X, V>;
    constexpr int N = (V + 1) / 2;
    extern __shared__ __align__(16) uint8_t data[];
    const int gs = s.gs, lanes = 1 << s.lane_log;
    float* warp_m = reinterpret_cast<float*>(data + (s.steps * SX::STEP + 15) / 16 * 16);      // [warps][entries] means, from the group's origin
    float* warp_q = warp_m + kGnWarps * s.width;                                               // and squared distances
    float* group = warp_q + kGnWarps * s.width;                                                // [3][groups of the slab]: counts, means, distances
    float* stat = group + 3 * gs;                                                              // [2][groups]: origin, then mean; rstd
    __shared__ float warp_n[kGnWarps];
    pdl_wait();
    const GnPart at(s, V);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    x += at.sample * sx;
    uint8_t* slot = SX::first(data);
    {
        const X* src = x + (at.p0 + at.row) * ldx + at.c;
        const int64_t step = at.rows * ldx;
        uint8_t* to = slot;
        for (int k = 0, i = 0; k < kGnStages; ++k) {
            const int end = min(at.count, (k + 1) * at.stage);
#pragma unroll 4
            for (; i < end; ++i, src += step, to += SX::STEP) SX::fetch(to, src);
            copies_group();
        }
    }
    const auto origin = [&](int g) {         // what a group's means are taken from
        float2 k;
        Vals<X, 1>::load(x + g * s.per, &k);
        return k.x;
    };
    // (read before the first y is written, which may be x itself)
    for (int g = threadIdx.x; g < gs; g += kGnThreads) stat[g] = origin(at.g0 + g);
    GnChannels<V> ch;
    if (at.c >= 0) ch.params(at.c, s.gamma, s.beta);
    Sums<V> t;
    {
        const uint8_t* from = slot;
        for (int k = 0, i = 0; k < kGnStages; ++k) {
            copies_landed(k);
            if (k == 0 && at.count > 0) SX::get(slot, t.k);
            const int end = min(at.count, (k + 1) * at.stage);
#pragma unroll 4
            for (; i < end; ++i, from += SX::STEP) {
                float2 v[N];
                SX::get(from, v);
                t.add(v);
            }
        }
    }
    __syncthreads();                         // the origins are there
    float n = (float)at.count;
    t.finish(n, at.group, s.alike, [&](int g) { return stat[g - at.g0]; });
    // A vector of one group goes on as one entry, others channel by channel
    if (s.alike) {
        float2 m = t.sum[0];
#pragma unroll
        for (int j = 1; j < N; ++j) m = add2(m, t.sum[j]);
        Moments a;
        a.n = n * V;
        a.m = V == 1 ? m.x : (m.x + m.y) * (1.0f / V);
        float2 q = pair(0.0f);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float2 d = sub2(t.sum[j], pair(a.m));
            q = add2(q, fma2(mul2(d, d), pair(n), t.sq[j]));
        }
        a.q = V == 1 ? t.sq[0].x : q.x + q.y;
        if (n == 0.0f) a = Moments();
        a.join(lanes, 16);
        if (lane < s.vecs) {
            warp_m[warp * s.width + lane] = a.m;
            warp_q[warp * s.width + lane] = a.q;
            if (lane == 0) warp_n[warp] = a.n;
        }
    } else {
        float cn = n;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            Moments a;
            a.n = n, a.m = at2(t.sum, j), a.q = at2(t.sq, j);
            a.join(lanes, 16);
            if (lane < s.vecs) {
                warp_m[warp * s.width + lane * V + j] = a.m;
                warp_q[warp * s.width + lane * V + j] = a.q;
            }
            cn = a.n;
        }
        if (lane == 0) warp_n[warp] = cn;
    }
    __syncthreads();
    // a group's entries: those of a warp to a lane of eight
    for (int g0 = 0; g0 < gs; g0 += kGnThreads / kGnWarps) {
        const int g = g0 + threadIdx.x / kGnWarps, w = threadIdx.x % kGnWarps, per = s.entries;
        Moments a;
        if (g < gs)
            for (int i = 0; i < per; ++i) a.add(warp_n[w], warp_m[w * s.width + g * per + i], warp_q[w * s.width + g * per + i]);
        a.join(1, kGnWarps / 2);
        if (g < gs && w == 0) group[g] = a.n, group[gs + g] = a.m, group[2 * gs + g] = a.q;
    }
    if (s.ks > 1) cluster_barrier();
    else __syncthreads();
    for (int g = threadIdx.x; g < gs; g += kGnThreads) {
        Moments a;
        if (s.ks == 1) a.n = group[g], a.m = group[gs + g], a.q = group[2 * gs + g];
        else {
            float rn[8], rm[8], rq[8];
            ld_remote(group + g, s.ks, rn);
            ld_remote(group + gs + g, s.ks, rm);
            ld_remote(group + 2 * gs + g, s.ks, rq);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < s.ks) a.add(rn[r], rm[r], rq[r]);
        }
        const float mu = stat[g] + a.m, rs = 1.0f / sqrtf(a.q / a.n + eps);
        stat[g] = mu;
        stat[gs + g] = rs;
        if (at.rank == 0 && mean) {
            mean[(int64_t)at.sample * s.groups + at.g0 + g] = mu;
            rstd[(int64_t)at.sample * s.groups + at.g0 + g] = rs;
        }
    }
    if (s.ks > 1) cluster_arrive();          // this CTA has read its peers' shared memory
    __syncthreads();
    if (at.count > 0) {
        ch.stats(at.group, s.alike, stat - at.g0, stat + gs - at.g0);
#pragma unroll
        for (int j = 0; j < N; ++j) ch.r[j] = mul2(ch.r[j], ch.gamma[j]);
        Y* dst = y + at.sample * sy + (at.p0 + at.row) * ldy + at.c;
        const int64_t step = at.rows * ldy;
        const uint8_t* from = slot;
        with_act(s.act, [&](auto act) {
#pragma unroll 4
            for (int i = 0; i < at.count; ++i, from += SX::STEP, dst += step) {
                float2 v[N];
                SX::get(from, v);
                ch.template apply<decltype(act)::value>(v);
                Vals<Y, V>::store(dst, v);
            }
        });
    }
    if (s.ks > 1) cluster_wait();            // and they this one's
}

// The gradients: du replaces dy in shared memory, in 32 bits, so that the slopes are taken once.  sums: of du and
// du h for each sample and channel [sample][2][channels], or null.  dx may be null.
template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads, 2) k_gn_one_back(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                               const GnOne s, const float* mean, const float* rstd, float* sums, Y* dx,
                                                               int64_t lddx, int64_t sdx) {
    using SX = Slots<X, V>;
    using SY = Slots<Y, V>;
    using SD = Slots<float, V>;
    constexpr int N = (V + 1) / 2;
    extern __shared__ __align__(16) uint8_t data[];
    const int xb = (s.steps * SX::STEP + 15) / 16 * 16, gs = s.gs;
    uint8_t* grads = data + xb;
    float* warp_s = reinterpret_cast<float*>(grads + s.steps * SD::STEP);      // [2][warps][width]
    float* chan = warp_s + 2 * kGnWarps * s.width;                             // [2][width]
    float* means = chan + 2 * s.width;                                         // [2][groups]
    float* gamma = means + 2 * gs;                                             // [width]
    pdl_wait();
    const GnPart at(s, V);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *xslot = SX::first(data), *gslot = SD::first(grads);
    {
        const X* src = x + at.sample * sx + (at.p0 + at.row) * ldx + at.c;
        const Y* grad = dy + at.sample * sdy + (at.p0 + at.row) * lddy + at.c;
        const int64_t xs = at.rows * ldx, ys = at.rows * lddy;
        uint8_t *tx = xslot, *tg = gslot;
        for (int k = 0, i = 0; k < kGnStages; ++k) {
            const int end = min(at.count, (k + 1) * at.stage);
#pragma unroll 2
            for (; i < end; ++i, src += xs, grad += ys, tx += SX::STEP, tg += SD::STEP) {
                SX::fetch(tx, src);
                SY::template fetch<SD>(tg, grad);
            }
            copies_group();
        }
    }
    const int c0 = at.g0 * s.per;
    for (int i = threadIdx.x; i < s.width; i += kGnThreads) gamma[i] = s.gamma ? s.gamma[c0 + i] : 1.0f;
    GnChannels<V> ch;
    float2 a[N], b[N];
#pragma unroll
    for (int j = 0; j < N; ++j) a[j] = b[j] = pair(0.0f);
    if (at.c >= 0) {
        ch.params(at.c, s.gamma, s.beta);
        ch.stats(at.group, s.alike, mean + (int64_t)at.sample * s.groups, rstd + (int64_t)at.sample * s.groups);
    }
    with_act(s.act, [&](auto act) {
        const uint8_t* tx = xslot;
        uint8_t* tg = gslot;
        for (int k = 0, i = 0; k < kGnStages; ++k) {
            copies_landed(k);
            const int end = min(at.count, (k + 1) * at.stage);
#pragma unroll 2
            for (; i < end; ++i, tx += SX::STEP, tg += SD::STEP) {
                float2 v[N], du[N];
                SX::get(tx, v);
                SY::template get<SD>(tg, du);
                ch.template slopes<decltype(act)::value>(v, du);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    a[j] = add2(a[j], du[j]);
                    b[j] = fma2(du[j], v[j], b[j]);
                }
                SD::put(tg, du);
            }
        }
    });
    for (int d = 1 << s.lane_log; d < 32; d <<= 1) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            a[j] = add2(a[j], make_float2(__shfl_xor_sync(0xffffffffu, a[j].x, d), V > 1 ? __shfl_xor_sync(0xffffffffu, a[j].y, d) : 0.0f));
            b[j] = add2(b[j], make_float2(__shfl_xor_sync(0xffffffffu, b[j].x, d), V > 1 ? __shfl_xor_sync(0xffffffffu, b[j].y, d) : 0.0f));
        }
    }
    if (lane < s.vecs) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            warp_s[warp * s.width + lane * V + j] = at2(a, j);
            warp_s[(kGnWarps + warp) * s.width + lane * V + j] = at2(b, j);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * s.width; i += kGnThreads) {
        const int half = i >= s.width, c = i - half * s.width;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kGnWarps; ++w) v += warp_s[(half * kGnWarps + w) * s.width + c];
        chan[i] = v;
    }
    if (s.ks > 1) {
        cluster_barrier();
        // all ranks' sums, in their order, to where the warps' were
        for (int i = threadIdx.x; i < 2 * s.width; i += kGnThreads) {
            float v = 0.0f, o[8];
            ld_remote(chan + i, s.ks, o);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < s.ks) v += o[r];
            warp_s[i] = v;
        }
        cluster_arrive();          // this CTA has read its peers' shared memory
    }
    __syncthreads();
    const float* total = s.ks > 1 ? warp_s : chan;
    if (sums && at.rank == 0)
        for (int i = threadIdx.x; i < 2 * s.width; i += kGnThreads) {
            const int half = i >= s.width;
            sums[((int64_t)at.sample * 2 + half) * s.channels + c0 + i - half * s.width] = total[i];
        }
    if (dx) {
        const float one = 1.0f / ((float)s.pixels * (float)s.per);
        for (int g0 = 0; g0 < gs; g0 += kGnThreads / 8) {        // eight lanes a group
            const int g = g0 + threadIdx.x / 8;
            float u = 0.0f, v = 0.0f;
            if (g < gs)
                for (int i = threadIdx.x % 8; i < s.per; i += 8) {
                    const int c = g * s.per + i;
                    u = fmaf(gamma[c], total[c], u);
                    v = fmaf(gamma[c], total[s.width + c], v);
                }
#pragma unroll
            for (int d = 4; d > 0; d >>= 1) u += __shfl_xor_sync(0xffffffffu, u, d), v += __shfl_xor_sync(0xffffffffu, v, d);
            if (g < gs && threadIdx.x % 8 == 0) means[g] = u * one, means[gs + g] = v * one;
        }
        __syncthreads();
        if (at.count > 0) {
            a[N - 1].y = b[N - 1].y = 0.0f;
            at.group.template each<V>(s.alike, [&](int j, int g) {
                at2(a, j) = means[g - at.g0];
                at2(b, j) = means[gs + g - at.g0];
            });
            ch.to_dx(a, b);
            Y* dst = dx + at.sample * sdx + (at.p0 + at.row) * lddx + at.c;
            const int64_t step = at.rows * lddx;
            const uint8_t *tx = xslot, *tg = gslot;
#pragma unroll 4
            for (int i = 0; i < at.count; ++i, tx += SX::STEP, tg += SD::STEP, dst += step) {
                float2 v[N], du[N];
                SX::get(tx, v);
                SD::get(tg, du);
                ch.dx(v, du);
                Vals<Y, V>::store(dst, v);
            }
        }
    }
    if (s.ks > 1) cluster_wait();            // and they this one's
}

// dgamma and dbeta from the chunks' sums [rows][2][channels]: 32 channels a CTA, the rows over its warps.
__global__ void __launch_bounds__(1024) k_gn_params(const float* part, int rows, int channels, float* dgamma, float* dbeta, int add) {
    __shared__ float sh[32][33];
    pdl_wait();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, half = blockIdx.y;
    float v = 0.0f;
    if (c < channels) {
#pragma unroll 8
        for (int i = w; i < rows; i += 32) v += part[((int64_t)i * 2 + half) * channels + c];
    }
    sh[w][lane] = v;
    __syncthreads();
    v = sh[lane][w];          // a warp a channel
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    const int ch = blockIdx.x * 32 + w;
    float* out = half ? dgamma : dbeta;
    if (lane == 0 && ch < channels && out) out[ch] = add ? out[ch] + v : v;
}

}  // namespace
}  // namespace nitro

struct nitro_gnorm {
    int max_samples = 0, max_pixels = 0, channels = 0, groups = 0;
    int batch = 0;                   // samples of a launch, at most
    float* part_c = nullptr;         // [chunks of a batch][2][channels]
    float2* part = nullptr;          // [chunks of a batch][groups]
    float2* means = nullptr;         // [batch][groups]
    float* mean = nullptr;           // [batch][groups], where the caller wants none
    float* rstd = nullptr;
    uint32_t* ticket = nullptr;      // [batch]
    bool clean = false;              // the tickets, see clear_once
    StatusWord status;
    DeviceAllocs allocs;
};

namespace {

int type_size(int type) { return type == NITRO_I8 ? 1 : type == NITRO_BF16 ? 2 : type == NITRO_F32 ? 4 : 0; }

// A map as the calls get it: null where the call has none.
struct Map {
    const void* p;
    int type;
    int64_t ld, stride;
    bool fits(int samples, int pixels, int channels) const {
        return ld >= channels && (samples <= 1 || stride >= (int64_t)pixels * ld) && (uintptr_t)p % type_size(type) == 0 &&
               ld < ((int64_t)1 << 40) && stride < ((int64_t)1 << 50);
    }
    // rows start at multiples of v values
    bool aligned(int v, int samples) const {
        const int64_t b = (int64_t)v * type_size(type), a = b < 16 ? b : 16;
        return !p || ((uintptr_t)p % a == 0 && ld * type_size(type) % a == 0 && (samples <= 1 || stride * type_size(type) % a == 0));
    }
};

// resident: CTAs an SM holds
GnShape shape(const nitro_gnorm* h, int pixels, int samples, int v, int resident, int act, const float* gamma, const float* beta) {
    GnShape s{};
    s.pixels = pixels;
    s.channels = h->channels;
    s.groups = h->groups;
    s.per = h->channels / h->groups;
    const int vecs = (h->channels + v - 1) / v;
    s.slabs = (vecs + kGnThreads - 1) / kGnThreads;
    s.vecs = (vecs + s.slabs - 1) / s.slabs;
    s.rows = kGnThreads / s.vecs;
    // one wave of CTAs in all, of eight steps at least
    const int wave = std::min(kGnCtas, resident * sm_count());
    const int want = std::max(1, std::min(wave / samples, (pixels + 8 * s.rows - 1) / (8 * s.rows)));
    s.chunk = (pixels + want - 1) / want;
    s.chunks = (pixels + s.chunk - 1) / s.chunk;
    s.act = act;
    s.gamma = gamma;
    s.beta = beta;
    return s;
}

int pick_v(const nitro_gnorm* h, int samples, std::initializer_list<Map> maps) {
    for (int v : {8, 4}) {
        bool ok = h->channels % v == 0;
        for (const Map& m : maps) ok = ok && m.aligned(v, samples);
        if (ok) return v;
    }
    return 1;
}

// f(value of the type, ...) for the types' numbers
template <class F>
cudaError_t with_x(int type, F&& f) {
    if (type == NITRO_I8) return f((int8_t)0);
    if (type == NITRO_BF16) return f((uint16_t)0);
    return f(0.0f);
}
template <class F>
cudaError_t with_y(int type, F&& f) {
    if (type == NITRO_BF16) return f((uint16_t)0);
    return f(0.0f);
}
template <class F>
cudaError_t with_v(int v, F&& f) {
    if (v == 8) return f(std::integral_constant<int, 8>{});
    if (v == 4) return f(std::integral_constant<int, 4>{});
    return f(std::integral_constant<int, 1>{});
}

bool gn_args(const nitro_gnorm* h, const Map& x, int samples, int pixels, int act) {
    return h && samples >= 0 && samples <= h->max_samples && pixels >= 1 && pixels <= h->max_pixels && act_known(act) &&
           (x.type == NITRO_I8 || x.type == NITRO_BF16 || x.type == NITRO_F32) && (samples == 0 || x.p) &&
           x.fits(samples, pixels, h->channels);
}
// fp32 arrays (null: none)
bool floats(std::initializer_list<const void*> ps) {
    uintptr_t bits = 0;
    for (const void* p : ps) bits |= (uintptr_t)p;
    return bits % sizeof(float) == 0;
}
bool y_type_known(int t) { return t == NITRO_BF16 || t == NITRO_F32; }
template <typename T>
const T* sample_at(const Map& m, int64_t i) {
    return static_cast<const T*>(m.p) + i * m.stride;
}

// samples of a batch: what both passes read stays in L2 in between
int batch_size(const nitro_gnorm* h, int pixels, int bytes_a_value) {
    const int64_t n = kGnBatchBytes / ((int64_t)pixels * h->channels * bytes_a_value);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, h->batch));
}

// How a call runs in one pass, or ks = 0: x_bytes, dy_bytes: of a value in shared memory; ctas: that an SM should hold.
// The narrowest slab of whole groups whose rows are lines of 64 bytes of x, or of 32 where there are few CTAs; the least CTAs that hold it; and more
// of them while SMs are idle.
GnOne one_pass(const nitro_gnorm* h, int samples, int pixels, int v, int x_size, int value_bytes, int ctas, int act, const float* gamma,
               const float* beta, int* smem) {
    GnOne s{};
    s.pixels = pixels;
    s.channels = h->channels;
    s.groups = h->groups;
    s.per = h->channels / h->groups;
    s.by_per = FloorDiv32::make(s.per);
    s.act = act;
    s.gamma = gamma;
    s.beta = beta;
    const int sms = sm_count();
    const auto fit = [&](int m, int ks, int budget) {      // m groups a slab
        s.width = m * s.per;
        s.gs = m;
        s.slabs = h->groups / m;
        s.ks = ks;
        s.vecs = s.width / v;
        s.alike = s.per % v == 0;
        s.entries = s.alike ? s.per / v : s.per;
        for (s.lane_log = 0; 1 << s.lane_log < s.vecs;) ++s.lane_log;
        const int rows = kGnThreads >> s.lane_log;
        s.chunk = (pixels + ks - 1) / ks;
        s.steps = (s.chunk + rows - 1) / rows;
        const int64_t bytes = (int64_t)s.steps * kGnThreads * v * value_bytes + 32 + 4 * (2 * kGnWarps + 3) * (int64_t)s.width + 20 * m;
        *smem = (int)bytes;
        return bytes <= budget;
    };
    const auto slab_ok = [&](int m) { return h->groups % m == 0 && m * s.per % v == 0 && m * s.per / v <= 32; };
    // groups of a slab whose rows have `line` bytes, else as many as there may be
    const auto slab = [&](int line) {
        int best = 0;
        for (int m = 1; m <= h->groups && m * s.per <= 32 * v; ++m) {
            if (!slab_ok(m)) continue;
            best = m;
            if (m * s.per * x_size >= line) break;
        }
        return best;
    };
    if (slab(64) == 0) return GnOne{};
    const int widest = (int64_t)samples * (h->groups / slab(64)) >= sms ? 64 : 32;
    const int share = 226 * 1024 / ctas - 1024;
    for (int budget : {share, 110 * 1024, 224 * 1024})
        for (int line = widest; line >= 16; line /= 2)
            for (int ks = 1; ks <= 8; ks *= 2) {
                if (!fit(slab(line), ks, budget)) continue;
                const int least = ks;
                while (ks < 8 && (int64_t)samples * s.slabs * ks * 2 <= 2 * sms && s.steps > 2 * (ks / least)) ks *= 2;
                if (ks > least) fit(slab(line), ks, budget);
                return s;
            }
    return GnOne{};
}

template <typename K>
cudaError_t one_ready(K* kernel, std::atomic<uint64_t>& ready, int smem = 226 * 1024) {
    int dev = 0;
    sm_count(&dev);
    return once_per_device(ready, dev, [kernel, smem] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
}

}  // namespace

extern "C" {

nitro_status nitro_gnorm_create(int max_samples, int max_pixels, int channels, int groups, nitro_gnorm** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (max_samples < 1 || max_pixels < 1 || channels < 1 || groups < 1 || max_samples > 65535 || max_pixels > (1 << 30) || channels > kGnChannels ||
        channels % groups != 0 || (int64_t)max_pixels * channels > ((int64_t)1 << 38) / max_samples)
        return NITRO_ERR_ARG;
    nitro_gnorm* h = new (std::nothrow) nitro_gnorm();
    if (!h) return NITRO_ERR_CUDA;
    h->max_samples = max_samples;
    h->max_pixels = max_pixels;
    h->channels = channels;
    h->groups = groups;
    h->batch = std::min(max_samples, kGnBatch);
    const int64_t parts = std::max(kGnCtas, kGnBatch), stats = (int64_t)h->batch * groups;
    // (the tickets are cleared by the first call)
    const bool ok = h->allocs.take(&h->part_c, parts * 2 * channels) && h->allocs.take(&h->part, parts * groups) &&
                    h->allocs.take(&h->means, stats) && h->allocs.take(&h->mean, stats) && h->allocs.take(&h->rstd, stats) &&
                    h->allocs.take(&h->ticket, h->batch) && h->status.take();
    if (!ok) {
        nitro_gnorm_destroy(h);
        return NITRO_ERR_CUDA;
    }
    *out = h;
    return NITRO_OK;
}

nitro_status nitro_gnorm_forward(nitro_gnorm* h, const void* x, int x_type, int64_t ldx, int64_t stride_x, int samples, int pixels,
                                 const float* gamma, const float* beta, float eps, int act, void* y, int y_type, int64_t ldy,
                                 int64_t stride_y, float* mean, float* rstd, void* stream) {
    const Map mx{x, x_type, ldx, stride_x}, my{y, y_type, ldy, stride_y};
    if (!gn_args(h, mx, samples, pixels, act) || !y_type_known(y_type) || !my.fits(samples, pixels, h->channels)) return NITRO_ERR_ARG;
    if (!(eps > 0.0f) || eps > 3e38f || !mean != !rstd || !floats({gamma, beta, mean, rstd})) return NITRO_ERR_ARG;
    if (samples == 0) return NITRO_OK;
    if (!y) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    TRY(clear_once(h->clean, h->ticket, sizeof(uint32_t) * h->batch, s));
    const int v = pick_v(h, samples, {mx, my}), C = h->channels;
    int smem = 0;
    const GnOne one = one_pass(h, samples, pixels, v, type_size(x_type), type_size(x_type), 3, act, gamma, beta, &smem);
    if (one.ks) {
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v(v, [&](auto vt) {
                    constexpr int V = decltype(vt)::value;
                    static std::atomic<uint64_t> ready{0};
                    const cudaError_t e = one_ready(k_gn_one<X, Y, V>, ready);
                    if (e != cudaSuccess) return e;
                    ProfScope ps(K_GNORM_FWD, s, 0.0, (double)samples * pixels * C * (sizeof(X) + sizeof(Y)));
                    return launch_cluster(k_gn_one<X, Y, V>, dim3(one.slabs * one.ks, samples), kGnThreads, one.ks, s, smem,
                                          (const X*)x, ldx, stride_x, one, eps, mean, rstd, (Y*)y, ldy, stride_y);
                });
            });
        }));
        return NITRO_OK;
    }
    const int batch = batch_size(h, pixels, type_size(x_type));
    for (int s0 = 0; s0 < samples; s0 += batch) {
        const int n = std::min(batch, samples - s0);
        const GnShape sh = shape(h, pixels, n, v, 4, act, gamma, beta);
        float* m = mean ? mean + (int64_t)s0 * h->groups : h->mean;
        float* r = rstd ? rstd + (int64_t)s0 * h->groups : h->rstd;
        const double values = (double)n * pixels * C;
        const dim3 grid(sh.chunks, n), block((sh.rows * sh.vecs + 31) / 32 * 32);
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_v(v, [&](auto vt) {
                constexpr int V = decltype(vt)::value;
                static std::atomic<uint64_t> ready{0};
                const cudaError_t e = one_ready(k_gn_stats<X, V>, ready, kRing * Slots<X, V>::STEP + 8 * kGnChannels);
                if (e != cudaSuccess) return e;
                ProfScope ps(K_GNORM_FWD, s, 0.0, values * sizeof(X));
                return launch_k(k_gn_stats<X, V>, grid, block, kRing * Slots<X, V>::STEP + 8 * C, s, sample_at<X>(mx, s0), ldx, stride_x, sh, eps, h->part,
                                h->ticket, m, r);
            });
        }));
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v(v, [&](auto vt) {
                    constexpr int V = decltype(vt)::value;
                    constexpr int kSmem = kRing * Slots<X, V>::STEP;
                    static std::atomic<uint64_t> ready{0};
                    const cudaError_t e = one_ready(k_gn_apply<X, Y, V>, ready, kSmem);
                    if (e != cudaSuccess) return e;
                    ProfScope ps(K_GNORM_FWD, s, 0.0, values * (sizeof(X) + sizeof(Y)));
                    return launch_k(k_gn_apply<X, Y, V>, grid, block, kSmem, s, sample_at<X>(mx, s0), ldx, stride_x, sh, (const float*)m,
                                    (const float*)r, const_cast<Y*>(sample_at<Y>(my, s0)), ldy, stride_y);
                });
            });
        }));
    }
    return NITRO_OK;
}

nitro_status nitro_gnorm_backward(nitro_gnorm* h, const void* x, int x_type, int64_t ldx, int64_t stride_x, int samples, int pixels,
                                  const float* gamma, const float* beta, const float* mean, const float* rstd, int act,
                                  const void* dy, int y_type, int64_t lddy, int64_t stride_dy, void* dx, int64_t lddx,
                                  int64_t stride_dx, float* dgamma, float* dbeta, void* stream) {
    const Map mx{x, x_type, ldx, stride_x}, mdy{dy, y_type, lddy, stride_dy}, mdx{dx, y_type, lddx, stride_dx};
    if (!gn_args(h, mx, samples, pixels, act) || !y_type_known(y_type) || !mdy.fits(samples, pixels, h->channels) ||
        (dx && !mdx.fits(samples, pixels, h->channels)))
        return NITRO_ERR_ARG;
    if ((samples > 0 && (!dy || !mean || !rstd)) || !floats({gamma, beta, mean, rstd, dgamma, dbeta})) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int C = h->channels;
    if (samples == 0) {   // an empty batch has gradients of zero
        for (float* p : {dgamma, dbeta})
            if (p) TRY(cudaMemsetAsync(p, 0, sizeof(float) * C, s));
        return NITRO_OK;
    }
    if (!dx && !dgamma && !dbeta) return NITRO_OK;
    TRY(clear_once(h->clean, h->ticket, sizeof(uint32_t) * h->batch, s));
    const int v = pick_v(h, samples, {mx, mdy, mdx});
    int smem = 0;
    const GnOne one = one_pass(h, samples, pixels, v, type_size(x_type), type_size(x_type) + 4, 2, act, gamma, beta, &smem);
    if (one.ks) {
        // the sums of at most a batch's samples are kept at a time
        const int most = dgamma || dbeta ? std::max(kGnCtas, kGnBatch) : samples;
        for (int s0 = 0; s0 < samples; s0 += most) {
            const int n = std::min(most, samples - s0);
            TRY(with_x(x_type, [&](auto xt) {
                using X = decltype(xt);
                return with_y(y_type, [&](auto yt) {
                    using Y = decltype(yt);
                    return with_v(v, [&](auto vt) {
                        constexpr int V = decltype(vt)::value;
                        static std::atomic<uint64_t> ready{0};
                        const cudaError_t e = one_ready(k_gn_one_back<X, Y, V>, ready);
                        if (e != cudaSuccess) return e;
                        ProfScope ps(K_GNORM_BWD, s, 0.0, (double)n * pixels * C * (sizeof(X) + (dx ? 2 : 1) * sizeof(Y)));
                        return launch_cluster(k_gn_one_back<X, Y, V>, dim3(one.slabs * one.ks, n), kGnThreads, one.ks, s, smem,
                                              sample_at<X>(mx, s0), ldx, stride_x, sample_at<Y>(mdy, s0), lddy, stride_dy, one,
                                              mean + (int64_t)s0 * h->groups, rstd + (int64_t)s0 * h->groups,
                                              dgamma || dbeta ? h->part_c : nullptr, dx ? const_cast<Y*>(sample_at<Y>(mdx, s0)) : nullptr, lddx, stride_dx);
                    });
                });
            }));
            if (dgamma || dbeta) {
                ProfScope ps(K_GNORM_PARAMS, s, 0.0, 8.0 * n * C);
                TRY(launch_k(k_gn_params, dim3((C + 31) / 32, 2), dim3(1024), 0, s, (const float*)h->part_c, n, C, dgamma, dbeta, (int)(s0 > 0)));
            }
        }
        return NITRO_OK;
    }
    const int batch = batch_size(h, pixels, type_size(x_type) + type_size(y_type));
    for (int s0 = 0; s0 < samples; s0 += batch) {
        const int n = std::min(batch, samples - s0);
        const GnShape sh = shape(h, pixels, n, v, gn_resident(v), act, gamma, beta);
        const float *m = mean + (int64_t)s0 * h->groups, *r = rstd + (int64_t)s0 * h->groups;
        const double values = (double)n * pixels * C;
        const dim3 grid(sh.chunks, n), block((sh.rows * sh.vecs + 31) / 32 * 32);
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v(v, [&](auto vt) {
                    constexpr int V = decltype(vt)::value;
                    constexpr int kSmem = kRing * (Slots<X, V>::STEP + Slots<Y, V>::STEP);
                    static std::atomic<uint64_t> ready{0};
                    const cudaError_t e = one_ready(k_gn_sums<X, Y, V>, ready, kSmem);
                    if (e != cudaSuccess) return e;
                    ProfScope ps(K_GNORM_BWD, s, 0.0, values * (sizeof(X) + sizeof(Y)));
                    return launch_k(k_gn_sums<X, Y, V>, grid, block, kSmem, s, sample_at<X>(mx, s0), ldx, stride_x, sample_at<Y>(mdy, s0),
                                    lddy, stride_dy, sh, m, r, h->part_c, h->part, h->ticket, dx ? h->means : nullptr);
                });
            });
        }));
        if (dx)
            TRY(with_x(x_type, [&](auto xt) {
                using X = decltype(xt);
                return with_y(y_type, [&](auto yt) {
                    using Y = decltype(yt);
                    return with_v(v, [&](auto vt) {
                        constexpr int V = decltype(vt)::value;
                        constexpr int kSmem = kRing * (Slots<X, V>::STEP + Slots<Y, V>::STEP);
                        static std::atomic<uint64_t> ready{0};
                        const cudaError_t e = one_ready(k_gn_dx<X, Y, V>, ready, kSmem);
                        if (e != cudaSuccess) return e;
                        ProfScope ps(K_GNORM_BWD, s, 0.0, values * (sizeof(X) + 2 * sizeof(Y)));
                        return launch_k(k_gn_dx<X, Y, V>, grid, block, kSmem, s, sample_at<X>(mx, s0), ldx, stride_x,
                                        sample_at<Y>(mdy, s0), lddy, stride_dy, sh, m, r, (const float2*)h->means,
                                        const_cast<Y*>(sample_at<Y>(mdx, s0)), lddx, stride_dx);
                    });
                });
            }));
        if (dgamma || dbeta) {
            ProfScope ps(K_GNORM_PARAMS, s, 0.0, 8.0 * n * sh.chunks * C);
            TRY(launch_k(k_gn_params, dim3((C + 31) / 32, 2), dim3(1024), 0, s, (const float*)h->part_c, n * sh.chunks, C, dgamma, dbeta,
                         (int)(s0 > 0)));
        }
    }
    return NITRO_OK;
}

nitro_status nitro_gnorm_status(nitro_gnorm* h, int clear) {
    if (!h) return NITRO_ERR_ARG;
    uint32_t bits = 0;
    if (!h->status.read(clear != 0, &bits)) return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_gnorm_destroy(nitro_gnorm* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    h->allocs.free();
    h->status.free();
    delete h;
}

}  // extern "C"
