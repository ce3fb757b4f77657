// Group norm forward, one pass: see head_gnorm.cuh and head_gnorm.cu.
#include "head_gnorm.cuh"

using namespace nitro;

namespace nitro {
namespace {

template <typename X, typename Y, int V, bool W, bool ALIKE>
__global__ void __launch_bounds__(kGnThreads, 3) k_gn_one(const X* x, int64_t ldx, int64_t sx, const GnOne s, float eps, float* mean,
                                                          float* rstd, Y* y, int64_t ldy, int64_t sy) {
    using SX = Slots<X, V, W>;
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
    const uint32_t low0 = low_bits(x + (at.p0 + at.row) * ldx + at.c), low_step = (uint32_t)(at.rows * ldx * (int64_t)sizeof(X));
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
        uint32_t low = low0;
        for (int k = 0, i = 0; k < kGnStages; ++k) {
            copies_landed(k);
            if (k == 0 && at.count > 0) SX::get(slot, t.k, low0);
            const int end = min(at.count, (k + 1) * at.stage);
#pragma unroll 4
            for (; i < end; ++i, from += SX::STEP, low += low_step) {
                float2 v[N];
                SX::get(from, v, low);
                t.add(v);
            }
        }
    }
    __syncthreads();                         // the origins are there
    float n = (float)at.count;
    t.finish(n, at.group, ALIKE, [&](int g) { return stat[g - at.g0]; });
    // A vector of one group goes on as one entry, others channel by channel
    if (ALIKE) {
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
        ch.stats(at.group, ALIKE, stat - at.g0, stat + gs - at.g0);
#pragma unroll
        for (int j = 0; j < N; ++j) ch.r[j] = mul2(ch.r[j], ch.gamma[j]);
        Y* dst = y + at.sample * sy + (at.p0 + at.row) * ldy + at.c;
        const int64_t step = at.rows * ldy;
        const uint8_t* from = slot;
        uint32_t low = low0;
        with_act(s.act, [&](auto act) {
#pragma unroll 4
            for (int i = 0; i < at.count; ++i, from += SX::STEP, dst += step, low += low_step) {
                float2 v[N];
                SX::get(from, v, low);
                ch.template apply<decltype(act)::value>(v);
                store_row<Y, V, W>(dst, v, s.whole);
            }
        });
    }
    if (s.ks > 1) cluster_wait();            // and they this one's
}

}  // namespace

cudaError_t gn_one_forward(const GnOne& one, int samples, int smem, const void* x, int x_type, int64_t ldx, int64_t stride_x, float eps, float* mean,
                           float* rstd, void* y, int y_type, int64_t ldy, int64_t stride_y, Width v, cudaStream_t s) {
    return with_x(x_type, [&](auto xt) {
        using X = decltype(xt);
        return with_y(y_type, [&](auto yt) {
            using Y = decltype(yt);
            return with_alike<sizeof(X) == 4 || sizeof(Y) == 4>(v, one.alike, [&](auto vt, auto wt, auto alike) {
                constexpr int V = decltype(vt)::value;
                constexpr bool W = decltype(wt)::value;
                constexpr bool A = decltype(alike)::value;
                static std::atomic<uint64_t> ready{0};
                const cudaError_t e = one_ready(k_gn_one<X, Y, V, W, A>, ready);
                if (e != cudaSuccess) return e;
                ProfScope ps(K_GNORM_FWD, s, 0.0, (double)samples * one.pixels * one.channels * (sizeof(X) + sizeof(Y)));
                return launch_cluster(k_gn_one<X, Y, V, W, A>, dim3(one.slabs * one.ks, samples), kGnThreads, one.ks, s, smem, (const X*)x, ldx,
                                      stride_x, one, eps, mean, rstd, (Y*)y, ldy, stride_y);
            });
        });
    });
}

}  // namespace nitro
