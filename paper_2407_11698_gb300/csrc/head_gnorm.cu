// Group norm with an activation on channels-last maps x [samples][pixels][channels]: per sample and group of
// neighbouring channels mean m and variance v over N = pixels channels / groups values, r = 1 / sqrt(v + eps),
//   h = (x - m) r,  u = gamma h + beta,  y = act(u);
//   du = dy act'(u),  dbeta = sum du,  dgamma = sum du h,  t = gamma du,
//   dx = r (t - sum_g t / N - h sum_g (t h) / N).
//
// A thread keeps V neighbouring channels and goes along the pixels; a CTA takes a chunk of a sample's pixels.  Each
// direction is a pass for the sums and one for the result, over batches of samples that stay in L2 in between.  The last CTA
// of a sample joins its chunks' sums.  A thread's sums are of distances to its first value, and parts are joined as
// (count, mean, sum of squared distances) with means taken from the group's first value, so a mean far from zero costs the
// variance no digits.
#include <new>

#include "head_act.cuh"

using namespace nitro;

namespace nitro {
namespace {

constexpr int kGnThreads = 256;
constexpr int kGnBatch = 1024;                 // samples of a launch, at most
constexpr int kGnCtas = 1216;                  // CTAs of a launch, unless there are more samples (eight an SM)
constexpr int64_t kGnBatchBytes = (int64_t)64 << 20;
constexpr int kGnChannels = 8192;

// V values of a row as fp32; rows are aligned to V values
template <typename T, int V>
struct Vals {
    static constexpr int W = V * (int)sizeof(T) / 4;      // words
    static __device__ __forceinline__ void load(const T* p, float* v) {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 1) v[0] = (float)(*reinterpret_cast<const int8_t*>(p));
            else if constexpr (sizeof(T) == 2) v[0] = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
            else v[0] = *reinterpret_cast<const float*>(p);
        } else {
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
            for (int j = 0; j < V; ++j) {
                if constexpr (sizeof(T) == 1)          // 2^23 + (v + 128) as a float has v + 128 in its low byte
                    v[j] = __uint_as_float(__byte_perm(w[j >> 2] ^ 0x80808080u, 0x4B000000u, 0x7540 + (j & 3))) - 8388736.0f;
                else if constexpr (sizeof(T) == 2) v[j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
                else v[j] = __uint_as_float(w[j]);
            }
        }
    }
    static __device__ __forceinline__ void store(T* p, const float* v) {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p) = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
            else *reinterpret_cast<float*>(p) = v[0];
        } else {
            uint32_t w[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if constexpr (sizeof(T) == 2) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
                else w[i] = __float_as_uint(v[i]);
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
};

// A warp's (count, mean, squared distances) triples into one: count-weighted.  cnt may be zero.
__device__ __forceinline__ void gn_join(float& n, float& mean, float& m2) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float on = __shfl_xor_sync(0xffffffffu, n, d), om = __shfl_xor_sync(0xffffffffu, mean, d),
                    o2 = __shfl_xor_sync(0xffffffffu, m2, d);
        const float t = n + on, w = t > 0.0f ? on / t : 0.0f, diff = om - mean;
        m2 += o2 + diff * diff * n * w;
        mean = fmaf(diff, w, mean);
        n = t;
    }
}
__device__ __forceinline__ void gn_add(float& n, float& mean, float& m2, float on, float om, float o2) {
    const float t = n + on, w = t > 0.0f ? on / t : 0.0f, diff = om - mean;
    m2 += o2 + diff * diff * n * w;
    mean = fmaf(diff, w, mean);
    n = t;
}

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

// mean and rstd of a sample's groups.  Dynamic shared memory: two values a channel.
template <typename X, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_stats(const X* x, int64_t ldx, int64_t sx, const GnShape s, float eps, float2* part,
                                                         uint32_t* ticket, float* mean, float* rstd) {
    extern __shared__ float chan[];                   // [channels] means, [channels] squared distances
    __shared__ float red[2][kGnThreads * V];          // [rows][slab's channels]
    __shared__ int word;
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    const int width = s.vecs * V;
    x += sample * sx;
    const auto origin = [&](int g) {         // what a group's means are taken from
        float k;
        Vals<X, 1>::load(x + g * s.per, &k);
        return k;
    };
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c >= 0) {
            float k[V], sum[V], sq[V];
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] = sq[j] = k[j] = 0.0f;
            const X* src = x + (int64_t)(p0 + at.row) * ldx + c;
            if (at.row < np) Vals<X, V>::load(src, k);
            const int64_t step = s.rows * ldx;
#pragma unroll 4
            for (int p = at.row; p < np; p += s.rows, src += step) {
                float v[V];
                Vals<X, V>::load(src, v);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float d = v[j] - k[j];
                    sum[j] += d;
                    sq[j] = fmaf(d, d, sq[j]);
                }
            }
            const float n = (float)((np - at.row + s.rows - 1) / s.rows);       // 0 for rows past the chunk
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float m = at.row < np ? sum[j] / n : 0.0f;
                red[0][at.row * width + at.vec * V + j] = (k[j] - origin((c + j) / s.per)) + m;
                red[1][at.row * width + at.vec * V + j] = fmaxf(fmaf(-m, sum[j], sq[j]), 0.0f);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < width; i += blockDim.x) {
            const int ch = slab * width + i;
            if (ch >= s.channels) break;
            float n = 0.0f, m = 0.0f, m2 = 0.0f;
            for (int r = 0; r < min(s.rows, np); ++r)
                gn_add(n, m, m2, (float)((np - r + s.rows - 1) / s.rows), red[0][r * width + i], red[1][r * width + i]);
            chan[ch] = m;
            chan[s.channels + ch] = m2;
        }
        __syncthreads();
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    part += (int64_t)sample * s.chunks * s.groups;
    for (int g = warp; g < s.groups; g += warps) {
        float n = 0.0f, m = 0.0f, m2 = 0.0f;
        for (int c = lane; c < s.per; c += 32) gn_add(n, m, m2, (float)np, chan[g * s.per + c], chan[s.channels + g * s.per + c]);
        gn_join(n, m, m2);
        if (lane == 0) part[(int64_t)blockIdx.x * s.groups + g] = make_float2(m, m2);
    }
    if (!gn_last(ticket + sample, s.chunks, &word)) return;
    for (int g = warp; g < s.groups; g += warps) {
        float n = 0.0f, m = 0.0f, m2 = 0.0f;
        for (int i = lane; i < s.chunks; i += 32) {
            const float2 v = __ldcg(part + (int64_t)i * s.groups + g);
            gn_add(n, m, m2, (float)(min(s.chunk, s.pixels - i * s.chunk)) * (float)s.per, v.x, v.y);
        }
        gn_join(n, m, m2);
        if (lane == 0) {
            mean[(int64_t)sample * s.groups + g] = origin(g) + m;
            rstd[(int64_t)sample * s.groups + g] = 1.0f / sqrtf(m2 / n + eps);
        }
    }
}

// A thread's channels: statistics of their groups, gamma and beta
template <int V>
struct GnChannels {
    float m[V], r[V], gamma[V], beta[V];
    __device__ __forceinline__ void load(const GnShape& s, int c, const float* mean, const float* rstd) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int g = (c + j) / s.per;
            m[j] = mean[g];
            r[j] = rstd[g];
            gamma[j] = s.gamma ? s.gamma[c + j] : 1.0f;
            beta[j] = s.beta ? s.beta[c + j] : 0.0f;
        }
    }
};

template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_apply(const X* x, int64_t ldx, int64_t sx, const GnShape s, const float* mean,
                                                         const float* rstd, Y* y, int64_t ldy, int64_t sy) {
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c < 0) continue;
        GnChannels<V> ch;
        ch.load(s, c, mean + (int64_t)sample * s.groups, rstd + (int64_t)sample * s.groups);
#pragma unroll
        for (int j = 0; j < V; ++j) ch.r[j] *= ch.gamma[j];
        const X* src = x + sample * sx + (int64_t)(p0 + at.row) * ldx + c;
        Y* dst = y + sample * sy + (int64_t)(p0 + at.row) * ldy + c;
        with_act(s.act, [&](auto act) {
#pragma unroll 4
            for (int p = at.row; p < np; p += s.rows, src += s.rows * ldx, dst += s.rows * ldy) {
                float v[V];
                Vals<X, V>::load(src, v);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = act_value<decltype(act)::value>(fmaf(v[j] - ch.m[j], ch.r[j], ch.beta[j]));
                Vals<Y, V>::store(dst, v);
            }
        });
    }
}

// du and h of V values
template <int ACT, int V>
__device__ __forceinline__ void gn_slopes(const GnChannels<V>& ch, float* x, float* dy) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
        x[j] = (x[j] - ch.m[j]) * ch.r[j];
        dy[j] *= act_slope<ACT>(fmaf(ch.gamma[j], x[j], ch.beta[j])).y;
    }
}

// Sums over a chunk: of du and du h for each channel (part_c [sample][chunk][2][channels]), and over a sample's
// groups of gamma du and gamma du h, divided by their count (means [sample][groups]).
template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_sums(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                        const GnShape s, const float* mean, const float* rstd, float* part_c,
                                                        float2* part, uint32_t* ticket, float2* means) {
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
            ch.load(s, c, mean + (int64_t)sample * s.groups, rstd + (int64_t)sample * s.groups);
            float a[V], b[V];
#pragma unroll
            for (int j = 0; j < V; ++j) a[j] = b[j] = 0.0f;
            const X* src = x + sample * sx + (int64_t)(p0 + at.row) * ldx + c;
            const Y* grad = dy + sample * sdy + (int64_t)(p0 + at.row) * lddy + c;
            with_act(s.act, [&](auto act) {
#pragma unroll 2
                for (int p = at.row; p < np; p += s.rows, src += s.rows * ldx, grad += s.rows * lddy) {
                    float v[V], g[V];
                    Vals<X, V>::load(src, v);
                    Vals<Y, V>::load(grad, g);
                    gn_slopes<decltype(act)::value, V>(ch, v, g);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        a[j] += g[j];
                        b[j] = fmaf(g[j], v[j], b[j]);
                    }
                }
            });
#pragma unroll
            for (int j = 0; j < V; ++j) {
                red[0][at.row * width + at.vec * V + j] = a[j];
                red[1][at.row * width + at.vec * V + j] = b[j];
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
    part += (int64_t)sample * s.chunks * s.groups;
    __threadfence_block();
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
        if (lane == 0) part[(int64_t)blockIdx.x * s.groups + g] = make_float2(a, b);
    }
    if (!gn_last(ticket + sample, s.chunks, &word)) return;
    const float count = (float)s.pixels * (float)s.per;
    for (int g = warp; g < s.groups; g += warps) {
        float a = 0.0f, b = 0.0f;
        for (int i = lane; i < s.chunks; i += 32) {
            const float2 v = __ldcg(part + (int64_t)i * s.groups + g);
            a += v.x;
            b += v.y;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d), b += __shfl_xor_sync(0xffffffffu, b, d);
        if (lane == 0) means[(int64_t)sample * s.groups + g] = make_float2(a / count, b / count);
    }
}

template <typename X, typename Y, int V>
__global__ void __launch_bounds__(kGnThreads) k_gn_dx(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                      const GnShape s, const float* mean, const float* rstd, const float2* means,
                                                      Y* dx, int64_t lddx, int64_t sdx) {
    pdl_wait();
    const int sample = blockIdx.y, p0 = blockIdx.x * s.chunk, p1 = min(s.pixels, p0 + s.chunk), np = p1 - p0;
    const GnPlace at(s);
    for (int slab = 0; slab < s.slabs; ++slab) {
        const int c = at.channel<V>(s, slab);
        if (c < 0) continue;
        GnChannels<V> ch;
        ch.load(s, c, mean + (int64_t)sample * s.groups, rstd + (int64_t)sample * s.groups);
        float2 t[V];
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = means[(int64_t)sample * s.groups + (c + j) / s.per];
        const X* src = x + sample * sx + (int64_t)(p0 + at.row) * ldx + c;
        const Y* grad = dy + sample * sdy + (int64_t)(p0 + at.row) * lddy + c;
        Y* dst = dx + sample * sdx + (int64_t)(p0 + at.row) * lddx + c;
        with_act(s.act, [&](auto act) {
#pragma unroll 2
            for (int p = at.row; p < np; p += s.rows, src += s.rows * ldx, grad += s.rows * lddy, dst += s.rows * lddx) {
                float v[V], g[V];
                Vals<X, V>::load(src, v);
                Vals<Y, V>::load(grad, g);
                gn_slopes<decltype(act)::value, V>(ch, v, g);
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = ch.r[j] * fmaf(-v[j], t[j].y, fmaf(ch.gamma[j], g[j], -t[j].x));
                Vals<Y, V>::store(dst, v);
            }
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

GnShape shape(const nitro_gnorm* h, int pixels, int samples, int v, int act, const float* gamma, const float* beta) {
    GnShape s{};
    s.pixels = pixels;
    s.channels = h->channels;
    s.groups = h->groups;
    s.per = h->channels / h->groups;
    const int vecs = (h->channels + v - 1) / v;
    s.slabs = (vecs + kGnThreads - 1) / kGnThreads;
    s.vecs = (vecs + s.slabs - 1) / s.slabs;
    s.rows = kGnThreads / s.vecs;
    // eight CTAs an SM in all, of eight steps at least
    const int want = std::max(1, std::min(kGnCtas / samples, (pixels + 8 * s.rows - 1) / (8 * s.rows)));
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
bool y_type_known(int t) { return t == NITRO_BF16 || t == NITRO_F32; }
template <typename T>
const T* sample_at(const Map& m, int64_t i) {
    return static_cast<const T*>(m.p) + i * m.stride;
}

// samples of a batch: what two passes touch stays in L2
int batch_size(const nitro_gnorm* h, int pixels, int bytes_a_value) {
    const int64_t n = kGnBatchBytes / ((int64_t)pixels * h->channels * bytes_a_value);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, h->batch));
}

}  // namespace

extern "C" {

nitro_status nitro_gnorm_create(int max_samples, int max_pixels, int channels, int groups, nitro_gnorm** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (max_samples < 1 || max_pixels < 1 || channels < 1 || groups < 1 || max_samples > 65535 || channels > kGnChannels ||
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
    if (!(eps > 0.0f) || eps > 3e38f || !mean != !rstd) return NITRO_ERR_ARG;
    if (samples == 0) return NITRO_OK;
    if (!y) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    TRY(clear_once(h->clean, h->ticket, sizeof(uint32_t) * h->batch, s));
    const int v = pick_v(h, samples, {mx, my}), C = h->channels;
    const int batch = batch_size(h, pixels, type_size(x_type) + type_size(y_type));
    for (int s0 = 0; s0 < samples; s0 += batch) {
        const int n = std::min(batch, samples - s0);
        const GnShape sh = shape(h, pixels, n, v, act, gamma, beta);
        float* m = mean ? mean + (int64_t)s0 * h->groups : h->mean;
        float* r = rstd ? rstd + (int64_t)s0 * h->groups : h->rstd;
        const double values = (double)n * pixels * C;
        const dim3 grid(sh.chunks, n), block((sh.rows * sh.vecs + 31) / 32 * 32);
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_v(v, [&](auto vt) {
                constexpr int V = decltype(vt)::value;
                static std::atomic<uint64_t> ready{0};
                int dev = 0;
                sm_count(&dev);
                const cudaError_t e = once_per_device(ready, dev, [] {
                    return cudaFuncSetAttribute(k_gn_stats<X, V>, cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * kGnChannels);
                });
                if (e != cudaSuccess) return e;
                ProfScope ps(K_GNORM_FWD, s, 0.0, values * sizeof(X));
                return launch_k(k_gn_stats<X, V>, grid, block, 8 * C, s, sample_at<X>(mx, s0), ldx, stride_x, sh, eps, h->part,
                                h->ticket, m, r);
            });
        }));
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v(v, [&](auto vt) {
                    constexpr int V = decltype(vt)::value;
                    ProfScope ps(K_GNORM_FWD, s, 0.0, values * (sizeof(X) + sizeof(Y)));
                    return launch_k(k_gn_apply<X, Y, V>, grid, block, 0, s, sample_at<X>(mx, s0), ldx, stride_x, sh, (const float*)m,
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
    if (samples > 0 && (!dy || !mean || !rstd)) return NITRO_ERR_ARG;
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
    const int batch = batch_size(h, pixels, type_size(x_type) + (dx ? 2 : 1) * type_size(y_type));
    for (int s0 = 0; s0 < samples; s0 += batch) {
        const int n = std::min(batch, samples - s0);
        const GnShape sh = shape(h, pixels, n, v, act, gamma, beta);
        const float *m = mean + (int64_t)s0 * h->groups, *r = rstd + (int64_t)s0 * h->groups;
        const double values = (double)n * pixels * C;
        const dim3 grid(sh.chunks, n), block((sh.rows * sh.vecs + 31) / 32 * 32);
        TRY(with_x(x_type, [&](auto xt) {
            using X = decltype(xt);
            return with_y(y_type, [&](auto yt) {
                using Y = decltype(yt);
                return with_v(v, [&](auto vt) {
                    constexpr int V = decltype(vt)::value;
                    ProfScope ps(K_GNORM_BWD, s, 0.0, values * (sizeof(X) + sizeof(Y)));
                    return launch_k(k_gn_sums<X, Y, V>, grid, block, 0, s, sample_at<X>(mx, s0), ldx, stride_x, sample_at<Y>(mdy, s0),
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
                        ProfScope ps(K_GNORM_BWD, s, 0.0, values * (sizeof(X) + 2 * sizeof(Y)));
                        return launch_k(k_gn_dx<X, Y, V>, grid, block, 0, s, sample_at<X>(mx, s0), ldx, stride_x,
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
