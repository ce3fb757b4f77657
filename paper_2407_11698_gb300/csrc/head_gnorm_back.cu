// Group norm backward, one pass: see head_gnorm.cuh and head_gnorm.cu.
#include "head_gnorm.cuh"

using namespace nitro;

namespace nitro {
namespace {

// The gradients: du replaces dy in shared memory, in 32 bits, so that the slopes are taken once.  sums: of du and
// du h for each sample and channel [sample][2][channels], or null.  dx may be null.
template <typename X, typename Y, int V, bool W, bool ALIKE>
__global__ void __launch_bounds__(kGnThreads, 2) k_gn_one_back(const X* x, int64_t ldx, int64_t sx, const Y* dy, int64_t lddy, int64_t sdy,
                                                               const GnOne s, const float* mean, const float* rstd, float* sums, Y* dx,
                                                               int64_t lddx, int64_t sdx) {
    using SX = Slots<X, V, W>;
    using SY = Slots<Y, V, W>;
    using SD = Slots<float, V, false>;
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
    const uint32_t xlow0 = low_bits(x + at.sample * sx + (at.p0 + at.row) * ldx + at.c), xlow_step = (uint32_t)(at.rows * ldx * (int64_t)sizeof(X));
    const uint32_t glow0 = low_bits(dy + at.sample * sdy + (at.p0 + at.row) * lddy + at.c), glow_step = (uint32_t)(at.rows * lddy * (int64_t)sizeof(Y));
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
        ch.stats(at.group, ALIKE, mean + (int64_t)at.sample * s.groups, rstd + (int64_t)at.sample * s.groups);
    }
    with_act(s.act, [&](auto act) {
        const uint8_t* tx = xslot;
        uint8_t* tg = gslot;
        uint32_t xlow = xlow0, glow = glow0;
        for (int k = 0, i = 0; k < kGnStages; ++k) {
            copies_landed(k);
            const int end = min(at.count, (k + 1) * at.stage);
#pragma unroll 2
            for (; i < end; ++i, tx += SX::STEP, tg += SD::STEP, xlow += xlow_step, glow += glow_step) {
                float2 v[N], du[N];
                SX::get(tx, v, xlow);
                SY::template get<SD>(tg, du, glow);
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
            at.group.template each<V>(ALIKE, [&](int j, int g) {
                at2(a, j) = means[g - at.g0];
                at2(b, j) = means[gs + g - at.g0];
            });
            ch.to_dx(a, b);
            Y* dst = dx + at.sample * sdx + (at.p0 + at.row) * lddx + at.c;
            const int64_t step = at.rows * lddx;
            const uint8_t *tx = xslot, *tg = gslot;
            uint32_t xlow = xlow0;
#pragma unroll 4
            for (int i = 0; i < at.count; ++i, tx += SX::STEP, tg += SD::STEP, dst += step, xlow += xlow_step) {
                float2 v[N], du[N];
                SX::get(tx, v, xlow);
                SD::get(tg, du, 0);
                ch.dx(v, du);
                store_row<Y, V, W>(dst, v, s.whole);
            }
        }
    }
    if (s.ks > 1) cluster_wait();            // and they this one's
}

}  // namespace

cudaError_t gn_one_backward(const GnOne& one, int samples, int smem, const void* x, int x_type, int64_t ldx, int64_t stride_x, const float* mean,
                            const float* rstd, const void* dy, int y_type, int64_t lddy, int64_t stride_dy, float* sums, void* dx, int64_t lddx,
                            int64_t stride_dx, Width v, cudaStream_t s) {
    return with_x(x_type, [&](auto xt) {
        using X = decltype(xt);
        return with_y(y_type, [&](auto yt) {
            using Y = decltype(yt);
            return with_alike<sizeof(X) == 4 || sizeof(Y) == 4>(v, one.alike, [&](auto vt, auto wt, auto alike) {
                constexpr int V = decltype(vt)::value;
                constexpr bool W = decltype(wt)::value;
                constexpr bool A = decltype(alike)::value;
                static std::atomic<uint64_t> ready{0};
                const cudaError_t e = one_ready(k_gn_one_back<X, Y, V, W, A>, ready);
                if (e != cudaSuccess) return e;
                ProfScope ps(K_GNORM_BWD, s, 0.0, (double)samples * one.pixels * one.channels * (sizeof(X) + (dx ? 2 : 1) * sizeof(Y)));
                return launch_cluster(k_gn_one_back<X, Y, V, W, A>, dim3(one.slabs * one.ks, samples), kGnThreads, one.ks, s, smem, (const X*)x, ldx,
                                      stride_x, (const Y*)dy, lddy, stride_dy, one, mean, rstd, sums, (Y*)dx, lddx, stride_dx);
            });
        });
    });
}

}  // namespace nitro
