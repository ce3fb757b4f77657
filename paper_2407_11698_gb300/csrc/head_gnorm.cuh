// Group norm's parts: what its kernels share, and how its one-pass launches are reached.
#pragma once

#include <initializer_list>

#include "head_act.cuh"

namespace nitro {

// A call that goes in one pass: a slab of a sample is shared out over ks CTAs of a cluster by pixels
struct GnOne {
    int pixels, channels, groups, per;
    int width, gs, slabs, ks;            // channels and groups of a slab, slabs of a sample, CTAs of a cluster
    int vecs, lane_log;                  // vectors of a slab's pixel, and the lanes' logarithm
    int chunk, steps;                    // pixels of a CTA, of which a thread takes every (256 / lanes)th
    int whole;                           // what is written starts at multiples of a vector
    int alike, entries;                  // vectors are of one group each; a group's vectors, or its channels where they are not
    FloorDiv32 by_per;
    int act;
    const float* gamma;                  // or null
    const float* beta;                   // or null
};

// How wide vectors are, and whether they start at any value (Slots)
struct Width {
    int v;
    bool words;
};

namespace {

constexpr int kGnThreads = 256;
constexpr int kGnBatch = 1024;                 // samples of a launch, at most
constexpr int kGnCtas = 608;                   // CTAs of a launch of two passes, unless there are more samples: four an SM
constexpr int64_t kGnBatchBytes = (int64_t)100 << 20;
constexpr int kGnChannels = 8192;

// V values of a row as fp32 pairs (of one value: itself and 0); rows are aligned to V values
template <typename T, int V>
struct Vals {
    [[maybe_unused]] static constexpr int N = (V + 1) / 2;
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
            unpack(w, v);
        }
    }
    static __device__ __forceinline__ void unpack(const uint32_t* w, float2* v) {
        if constexpr (V > 1) {
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

// A vector's place in shared memory: planes of 16 bytes a thread (or less, the vector itself).  WORDS: vectors that start at any
// value; the 32-bit words that they reach into are copied (each holds a byte of the vector, so it is memory
// that is there), in planes of words, and shifted when they are read
template <typename T, int V, bool WORDS>
struct Slots {
    static constexpr int SIZE = V * (int)sizeof(T);
    static constexpr int BYTES = WORDS ? (SIZE + 3) / 4 * 4 + (sizeof(T) < 4 ? 4 : 0) : SIZE;
    static constexpr int PLANE = WORDS ? 4 : BYTES < 16 ? BYTES : 16, PLANES = BYTES / PLANE;
    static constexpr int STEP = kGnThreads * BYTES;          // from a thread's vector to its next
    static __device__ __forceinline__ uint8_t* first(uint8_t* base) { return base + (int)threadIdx.x * PLANE; }
    // Place: whose places the vector takes, its own or those of wider values that replace it later
    template <class Place>
    static __device__ __forceinline__ int plane(int i) {
        const int byte = i * PLANE;
        return byte / Place::PLANE * kGnThreads * Place::PLANE + byte % Place::PLANE;
    }
    template <class Place = Slots>
    static __device__ __forceinline__ void fetch(uint8_t* to, const T* src) {
        if constexpr (WORDS) {
            const uintptr_t at = (uintptr_t)src & ~(uintptr_t)3;
            const int end = (int)((uintptr_t)src & 3) + SIZE;
#pragma unroll
            for (int i = 0; i < PLANES; ++i)
                if (4 * i < end)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to + plane<Place>(i))), "l"(at + 4 * i) : "memory");
        } else if constexpr (PLANE < 4) {
            *reinterpret_cast<T*>(to) = *src;
        } else {
#pragma unroll
            for (int i = 0; i < PLANES; ++i) {
                const uint32_t dst = smem_u32(to + plane<Place>(i));
                const char* s = reinterpret_cast<const char*>(src) + i * PLANE;
                if constexpr (PLANE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(s) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(s), "n"(PLANE) : "memory");
            }
        }
    }
    // src: the vector's address, or its low bits
    template <class Place = Slots>
    static __device__ __forceinline__ void get(const uint8_t* from, float2* v, uint32_t src) {
        if constexpr (WORDS) {
            uint32_t w[PLANES + 1];
#pragma unroll
            for (int i = 0; i < PLANES; ++i) w[i] = *reinterpret_cast<const uint32_t*>(from + plane<Place>(i));
            if constexpr (sizeof(T) < 4) {
#pragma unroll
                for (int i = 0; i < SIZE / 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (src & 3));
            }
            Vals<T, V>::unpack(w, v);
        } else {
#pragma unroll
            for (int i = 0; i < PLANES; ++i)
                Vals<T, V / PLANES>::load(reinterpret_cast<const T*>(from + plane<Place>(i)), v + i * (V / PLANES / 2));
        }
    }
    static __device__ __forceinline__ void put(uint8_t* to, const float2* v) {
        static_assert(!WORDS, "values of the kernels' own are aligned");
#pragma unroll
        for (int i = 0; i < PLANES; ++i)
            Vals<T, V / PLANES>::store(reinterpret_cast<T*>(to + i * kGnThreads * PLANE), v + i * (V / PLANES / 2));
    }
};
__device__ __forceinline__ uint32_t low_bits(const void* p) { return (uint32_t)(uintptr_t)p; }

// V values of a row; whole: rows are aligned to V values
template <typename T, int V, bool WORDS>
__device__ __forceinline__ void store_row(T* p, const float2* v, bool whole) {
    if constexpr (WORDS) {
        if (!whole) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float2 x = make_float2(j & 1 ? v[j >> 1].y : v[j >> 1].x, 0.0f);
                Vals<T, 1>::store(p + j, &x);
            }
            return;
        }
    }
    Vals<T, V>::store(p, v);
}
__device__ __forceinline__ void copies_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// ------------------------------------------------------------------ one pass
// Both directions in one launch with one pass over memory, where a cluster's shared memory holds a slab of a sample: whole
// groups, `width` channels at all pixels, shared out over ks CTAs by pixels.  A thread copies its own vectors to
// shared memory and alone reads them there, so nothing waits for them but itself; channels' sums meet in the
// warp's lanes, over the CTA's warps, and over the cluster's shared memory.
//
// Lanes: 2^k >= width / V to a pixel (those past the width idle), so the lanes of a channel are found by shuffles.
constexpr int kGnWarps = kGnThreads / 32;

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

// ------------------------------------------------------------------ host side
inline int type_size(int type) { return type == NITRO_I8 ? 1 : type == NITRO_BF16 ? 2 : type == NITRO_F32 ? 4 : 0; }

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

inline const void* sample_at(const Map& m, int64_t i) { return static_cast<const char*>(m.p) + i * m.stride * type_size(m.type); }
template <typename T>
const T* sample_at(const Map& m, int64_t i) {
    return static_cast<const T*>(m.p) + i * m.stride;
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
// f(width, words); WIDE: for fp32 values, which take no words of eight
template <bool WIDE, class F>
cudaError_t with_v(Width w, F&& f) {
    if (w.words) {
        if constexpr (!WIDE)
            if (w.v == 8) return f(std::integral_constant<int, 8>{}, std::true_type{});
        return f(std::integral_constant<int, 4>{}, std::true_type{});
    }
    if (w.v == 8) return f(std::integral_constant<int, 8>{}, std::false_type{});
    if (w.v == 4) return f(std::integral_constant<int, 4>{}, std::false_type{});
    return f(std::integral_constant<int, 1>{}, std::false_type{});
}
template <typename K>
cudaError_t one_ready(K* kernel, std::atomic<uint64_t>& ready, int smem = 226 * 1024) {
    int dev = 0;
    sm_count(&dev);
    return once_per_device(ready, dev, [kernel, smem] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem); });
}

// and whether vectors are of one group each (single values always are)
template <bool WIDE, class F>
cudaError_t with_alike(Width w, bool alike, F&& f) {
    return with_v<WIDE>(w, [&](auto v, auto words) {
        if constexpr (decltype(v)::value == 1) return f(v, words, std::true_type{});
        else return alike ? f(v, words, std::true_type{}) : f(v, words, std::false_type{});
    });
}

}  // namespace

// The one-pass launches.  mean, rstd: null where nobody wants them.  sums: [samples][2][channels] or null
cudaError_t gn_one_forward(const GnOne& one, int samples, int smem, const void* x, int x_type, int64_t ldx, int64_t stride_x, float eps, float* mean,
                           float* rstd, void* y, int y_type, int64_t ldy, int64_t stride_y, Width v, cudaStream_t s);
cudaError_t gn_one_backward(const GnOne& one, int samples, int smem, const void* x, int x_type, int64_t ldx, int64_t stride_x, const float* mean,
                            const float* rstd, const void* dy, int y_type, int64_t lddy, int64_t stride_dy, float* sums, void* dx, int64_t lddx,
                            int64_t stride_dx, Width v, cudaStream_t s);
}  // namespace nitro
