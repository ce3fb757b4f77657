// Group norm with an activation on channels-last maps x [samples][pixels][channels]: per sample and group of
// neighbouring channels mean m and variance v over N = pixels channels / groups values, r = 1 / sqrt(v + eps),
//   h = (x - m) r,  u = gamma h + beta,  y = act(u);
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du h,  t = gamma du,
//   dx = r (t - sum_g t / N - h sum_g (t h) / N).
//
// A thread keeps V neighbouring channels and goes along the pixels.  Where a cluster's shared memory holds a slab of a sample, a
// direction is one launch and one pass over memory (k_gn_one, k_gn_one_back): 128 x 4096 x 256 bf16 with silu 106 us forward,
// 5.0 TB/s, and 225 backward, 3.6, where a pass for the sums and one for the result took 1092 together.  Their instructions a
// value bound them, a third to a half of those the joining of sums, and 24 and 16 warps an SM.  Larger slabs take the
// two passes, over batches of samples that stay in L2 in between; the last CTA of a sample joins its chunks' sums.
//
// A thread's sums are of distances to its first value, and parts are joined as (count, mean, sum of squared distances) with
// means taken from the group's first value, so a mean far from zero costs the variance no digits.
#include <new>

#include "head_gnorm.cuh"

using namespace nitro;

namespace nitro {
namespace {

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

// Sums of many values go in runs, of a thread's and of the threads', which are then added up: equal values are all rounded the same way in
// one sum (2^28 equal dy in one channel: dbeta 1.9e-5 off).
constexpr int kValueRun = 32, kRowRun = 16;

// CTAs of a backward pass that an SM holds by their registers
constexpr int gn_resident(int v) { return v == 8 ? 2 : 4; }

// What is common to the four passes.
struct GnShape {
    int pixels, channels, groups, per;   // per: channels of a group
    int chunk, chunks;                   // pixels of a CTA, CTAs of a sample
    int vecs, slabs, rows;               // vectors of a pixel that a CTA takes at once, how often, pixels at once
    int act;
    int whole;                           // what is written starts at multiples of a vector
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
template <typename X, int V, bool W>
__global__ void __launch_bounds__(kGnThreads) k_gn_stats(const X* x, int64_t ldx, int64_t sx, const GnShape s, float eps, float2* parts,
                                                         uint32_t* ticket, float* mean, float* rstd) {
    using SX = Slots<X, V, W>;
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
            if (at.row < np) {
                if constexpr (W) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float2 one;
                        Vals<X, 1>::load(src + j, &one);
                        at2(t.k, j) = one.x;
                    }
                } else {
                    Vals<X, V>::load(src, t.k);
                }
            }
#pragma unroll
            for (int j = 0; j < t.N; ++j) run.k[j] = t.k[j];
            const int64_t step = s.rows * ldx;
            const int n = at.steps(s, np);
            uint8_t* slot = SX::first(data);
            through_ring(
                n, [&](int i, int k) { SX::fetch(slot + k * SX::STEP, src + i * step); },
                [&](int i, int k) {
                    float2 v[Sums<V>::N];
                    SX::get(slot + k * SX::STEP, v, low_bits(src + i * step));
                    run.add(v);
                    if (i % kValueRun == kValueRun - 1) t.take(run);
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
            for (int r = 0; r < min(s.rows, np);) {
                Moments run;
                for (const int to = min(min(s.rows, np), r + kRowRun); r < to; ++r)
                    run.add((float)((np - r + s.rows - 1) / s.rows), red[0][r * width + i], red[1][r * width + i]);
                a.add(run.n, run.m, run.q);
            }
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

template <typename X, typename Y, int V, bool W>
__global__ void __launch_bounds__(kGnThreads) k_gn_apply(const X* x, int64_t ldx, int64_t sx, const GnShape s, const float* mean,
                                                         const float* rstd, Y* y, int64_t ldy, int64_t sy) {
    using SX = Slots<X, V, W>;
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
                    SX::get(slot + k * SX::STEP, v, low_bits(src + i * xs));
                    ch.template apply<decltype(act)::value>(v);
                    store_row<Y, V, W>(dst + i * ys, v, s.whole);
                });
        });
    }
}

// Sums over a chunk: of du and du h for each channel (part_c [sample][chunk][2][channels]), and over a sample's
// groups of gamma du and gamma du h, divided by their count (means [sample][groups]).
template <typename X, typename Y, int V, bool W>
__global__ void __launch_bounds__(kGnThreads, gn_resident(V)) k_gn_sums(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                           const GnShape s, const float* mean, const float* rstd, float* part_c,
                                                           float2* parts, uint32_t* ticket, float2* means) {
    using SX = Slots<X, V, W>;
    using SY = Slots<Y, V, W>;
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
            // (runs are added up where the sums are wanted in the end, which takes no registers)
            float *suma = red[0] + at.row * width + at.vec * V, *sumb = red[1] + at.row * width + at.vec * V;
#pragma unroll
            for (int j = 0; j < V; ++j) suma[j] = sumb[j] = 0.0f;
            const auto end_run = [&] {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    suma[j] += at2(a, j);
                    sumb[j] += at2(b, j);
                    at2(a, j) = at2(b, j) = 0.0f;
                }
            };
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
                    [&](int i, int k) {
                        float2 v[ch.N], g[ch.N];
                        SX::get(xslot + k * SX::STEP, v, low_bits(src + i * xs));
                        SY::get(gslot + k * SY::STEP, g, low_bits(grad + i * gs));
                        ch.template slopes<decltype(act)::value>(v, g);
#pragma unroll
                        for (int j = 0; j < ch.N; ++j) {
                            a[j] = add2(a[j], g[j]);
                            b[j] = fma2(g[j], v[j], b[j]);
                        }
                        if (i % kValueRun == kValueRun - 1) end_run();
                    });
            });
            end_run();
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * width; i += blockDim.x) {
            const int half = i >= width, k = i - half * width, chn = slab * width + k;
            if (chn >= s.channels) continue;
            float v = 0.0f;
            for (int r = 0; r < s.rows;) {
                float run = 0.0f;
                for (const int to = min(s.rows, r + kRowRun); r < to; ++r) run += red[half][r * width + k];
                v += run;
            }
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

template <typename X, typename Y, int V, bool W>
__global__ void __launch_bounds__(kGnThreads, gn_resident(V)) k_gn_dx(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                         const GnShape s, const float* mean, const float* rstd, const float2* means,
                                                         Y* dx, int64_t lddx, int64_t sdx) {
    using SX = Slots<X, V, W>;
    using SY = Slots<Y, V, W>;
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
                    SX::get(xslot + k * SX::STEP, v, low_bits(src + i * xs));
                    SY::get(gslot + k * SY::STEP, g, low_bits(grad + i * gs));
#pragma unroll
                    for (int j = 0; j < ch.N; ++j) h[j] = v[j];
                    ch.template slopes<decltype(act)::value>(h, g);
                    to.dx(v, g);
                    store_row<Y, V, W>(dst + i * ds, v, s.whole);
                });
        });
    }
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

// in: what is read, out: what is written; whole: whether that starts at multiples of a vector.  Rows that start anywhere are
// copied by words, in vectors of eight values, of four where some are fp32 (lanes' words are nearer to each other): 64 x 1024 x 256, rows
// 259 apart, forward and backward 62 us with int8 x, 80 with bf16, 118 with fp32 (the other width 66, 77, 144; two samples of
// 100000 x 96: 86, 94, 174 against 105, 112, 181), where single values take 150, 150 and 134, and aligned rows 52, 52 and
// 114.  Aligned vectors of four come before words of eight: rows 260 apart 57, 74 and 113 us against 60, 79 and 113.
Width pick_v(const nitro_gnorm* h, int samples, std::initializer_list<Map> in, std::initializer_list<Map> out, int* whole) {
    const auto aligned = [&](std::initializer_list<Map> maps, int v) {
        for (const Map& m : maps)
            if (!m.aligned(v, samples)) return false;
        return true;
    };
    *whole = 1;
    const int C = h->channels;
    for (int v : {8, 4})
        if (C % v == 0 && aligned(in, v) && aligned(out, v)) return {v, false};
    if (C % 4 != 0) return {1, false};
    bool wide = false;
    for (const auto& maps : {in, out})
        for (const Map& m : maps) wide = wide || m.type == NITRO_F32;
    const int v = wide || C % 8 != 0 ? 4 : 8;
    *whole = aligned(out, v);
    return {v, true};
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
// samples of a batch: what both passes read stays in L2 in between
int batch_size(const nitro_gnorm* h, int pixels, int bytes_a_value) {
    const int64_t n = kGnBatchBytes / ((int64_t)pixels * h->channels * bytes_a_value);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, h->batch));
}

// bytes of a vector of x in shared memory
int slot_bytes(int x_type, Width w) {
    const int size = w.v * type_size(x_type);
    return size + (w.words && type_size(x_type) < 4 ? 4 : 0);
}

// How a call runs in one pass, or ks = 0: slot: bytes of a vector in shared memory; ctas: that an SM should hold.
// The narrowest slab of whole groups whose rows are lines of 64 bytes of x, or of 32 where there are few CTAs; the least CTAs that hold it; and more
// of them while SMs are idle.
GnOne one_pass(const nitro_gnorm* h, int samples, int pixels, int v, int x_size, int slot, int ctas, int act, const float* gamma,
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
        const int64_t bytes = (int64_t)s.steps * kGnThreads * slot + 32 + 4 * (2 * kGnWarps + 3) * (int64_t)s.width + 20 * m;
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
    int whole = 0;
    const Width w = pick_v(h, samples, {mx}, {my}, &whole);
    const int v = w.v, C = h->channels;
    int smem = 0;
    GnOne one = one_pass(h, samples, pixels, v, type_size(x_type), slot_bytes(x_type, w), 3, act, gamma, beta, &smem);
    one.whole = whole;
    if (one.ks) {
        TRY(gn_one_forward(one, samples, smem, x, x_type, ldx, stride_x, eps, mean, rstd, y, y_type, ldy, stride_y, w, s));
        return NITRO_OK;
    }
    const int batch = batch_size(h, pixels, type_size(x_type));
    for (int s0 = 0; s0 < samples; s0 += batch) {
        const int n = std::min(batch, samples - s0);
        GnShape sh = shape(h, pixels, n, v, 4, act, gamma, beta);
        sh.whole = whole;
        float* m = mean ? mean + (int64_t)s0 * h->groups : h->mean;
        float* r = rstd ? rstd + (int64_t)s0 * h->groups : h->rstd;
        const double values = (double)n * pixels * C;
        const dim3 grid(sh.chunks, n), block((sh.rows * sh.vecs + 31) / 32 * 32);
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_v<sizeof(X) == 4>(w, [&](auto vt, auto wt) {
                constexpr int V = decltype(vt)::value;
                constexpr bool W = decltype(wt)::value;
                static std::atomic<uint64_t> ready{0};
                const cudaError_t e = one_ready(k_gn_stats<X, V, W>, ready, kRing * Slots<X, V, W>::STEP + 8 * kGnChannels);
                if (e != cudaSuccess) return e;
                ProfScope ps(K_GNORM_FWD, s, 0.0, values * sizeof(X));
                return launch_k(k_gn_stats<X, V, W>, grid, block, kRing * Slots<X, V, W>::STEP + 8 * C, s, sample_at<X>(mx, s0), ldx, stride_x, sh, eps, h->part,
                                h->ticket, m, r);
            });
        }));
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v<sizeof(X) == 4 || sizeof(Y) == 4>(w, [&](auto vt, auto wt) {
                    constexpr int V = decltype(vt)::value;
                    constexpr bool W = decltype(wt)::value;
                    constexpr int kSmem = kRing * Slots<X, V, W>::STEP;
                    static std::atomic<uint64_t> ready{0};
                    const cudaError_t e = one_ready(k_gn_apply<X, Y, V, W>, ready, kSmem);
                    if (e != cudaSuccess) return e;
                    ProfScope ps(K_GNORM_FWD, s, 0.0, values * (sizeof(X) + sizeof(Y)));
                    return launch_k(k_gn_apply<X, Y, V, W>, grid, block, kSmem, s, sample_at<X>(mx, s0), ldx, stride_x, sh, (const float*)m,
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
    int whole = 0;
    const Width w = pick_v(h, samples, {mx, mdy}, {mdx}, &whole);
    const int v = w.v;
    int smem = 0;
    GnOne one = one_pass(h, samples, pixels, v, type_size(x_type), slot_bytes(x_type, w) + 4 * v, 2, act, gamma, beta, &smem);
    one.whole = whole;
    if (one.ks) {
        // the sums of at most a batch's samples are kept at a time
        const int most = dgamma || dbeta ? std::max(kGnCtas, kGnBatch) : samples;
        for (int s0 = 0; s0 < samples; s0 += most) {
            const int n = std::min(most, samples - s0);
            TRY(gn_one_backward(one, n, smem, sample_at(mx, s0), x_type, ldx, stride_x, mean + (int64_t)s0 * h->groups,
                                rstd + (int64_t)s0 * h->groups, sample_at(mdy, s0), y_type, lddy, stride_dy, dgamma || dbeta ? h->part_c : nullptr,
                                dx ? const_cast<void*>(sample_at(mdx, s0)) : nullptr, lddx, stride_dx, w, s));
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
        GnShape sh = shape(h, pixels, n, v, gn_resident(v), act, gamma, beta);
        sh.whole = whole;
        const float *m = mean + (int64_t)s0 * h->groups, *r = rstd + (int64_t)s0 * h->groups;
        const double values = (double)n * pixels * C;
        const dim3 grid(sh.chunks, n), block((sh.rows * sh.vecs + 31) / 32 * 32);
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v<sizeof(X) == 4 || sizeof(Y) == 4>(w, [&](auto vt, auto wt) {
                    constexpr int V = decltype(vt)::value;
                    constexpr bool W = decltype(wt)::value;
                    constexpr int kSmem = kRing * (Slots<X, V, W>::STEP + Slots<Y, V, W>::STEP);
                    static std::atomic<uint64_t> ready{0};
                    const cudaError_t e = one_ready(k_gn_sums<X, Y, V, W>, ready, kSmem);
                    if (e != cudaSuccess) return e;
                    ProfScope ps(K_GNORM_BWD, s, 0.0, values * (sizeof(X) + sizeof(Y)));
                    return launch_k(k_gn_sums<X, Y, V, W>, grid, block, kSmem, s, sample_at<X>(mx, s0), ldx, stride_x, sample_at<Y>(mdy, s0),
                                    lddy, stride_dy, sh, m, r, h->part_c, h->part, h->ticket, dx ? h->means : nullptr);
                });
            });
        }));
        if (dx)
            TRY(with_x(x_type, [&](auto xt) {
                using X = decltype(xt);
                return with_y(y_type, [&](auto yt) {
                    using Y = decltype(yt);
                    return with_v<sizeof(X) == 4 || sizeof(Y) == 4>(w, [&](auto vt, auto wt) {
                        constexpr int V = decltype(vt)::value;
                        constexpr bool W = decltype(wt)::value;
                        constexpr int kSmem = kRing * (Slots<X, V, W>::STEP + Slots<Y, V, W>::STEP);
                        static std::atomic<uint64_t> ready{0};
                        const cudaError_t e = one_ready(k_gn_dx<X, Y, V, W>, ready, kSmem);
                        if (e != cudaSuccess) return e;
                        ProfScope ps(K_GNORM_BWD, s, 0.0, values * (sizeof(X) + 2 * sizeof(Y)));
                        return launch_k(k_gn_dx<X, Y, V, W>, grid, block, kSmem, s, sample_at<X>(mx, s0), ldx, stride_x,
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
