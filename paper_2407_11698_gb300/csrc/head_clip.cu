// The norm over many gradients, sqrt(sum x^2) over all values of all matrices, and the gradients scaled by
// min(1, max_norm / norm).
//
// At creation the matrices are cut into pieces of about equal size, kept in a table on the device; CTA i takes pieces i,
// i + CTAs, ...  A first pass leaves each CTA's sums, the last CTA adds them in 64 bits in the CTAs' order, and a second pass
// scales.  Squares are summed three times, of x, of x 2^-80 and of x 2^90: the first passes fp32 from |x| = 2^64 on and
// loses values below 2^-75, and where its sum shows that, one of the others stands for it.
#include <new>

#include <cmath>
#include <vector>

#include "head_act.cuh"

using namespace nitro;

namespace nitro {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipCtas = 8;                       // an SM
constexpr int64_t kMostPieces = (int64_t)1 << 22;

// Rows of one matrix (of lone rows: a run of one).  vec: both sides' rows start at multiples of 16 bytes
struct Piece {
    const void* in;
    void* out;             // or null
    int64_t rows, cols, ld_in, ld_out;
    int type, vec;
};

struct Squares {
    float mid = 0.0f, big = 0.0f, small = 0.0f;
    __device__ __forceinline__ void add(float x) {
        mid = fmaf(x, x, mid);
        const float b = x * 0x1p-80f, s = x * 0x1p90f;
        big = fmaf(b, b, big);
        small = fmaf(s, s, small);
    }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

template <typename T>
struct Of;
template <>
struct Of<uint16_t> {
    static __device__ __forceinline__ float get(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t put(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
};
template <>
struct Of<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Of<int64_t> {
    static __device__ __forceinline__ float get(int64_t v) { return (float)v; }
    static __device__ __forceinline__ int64_t put(float v) { return (int64_t)v; }
};

// f(values, valid ones, address in `out` of the first) for the vectors of a piece, or its values one by one
template <typename T, class F>
__device__ __forceinline__ void each(const Piece& p, F&& f) {
    constexpr int V = 16 / (int)sizeof(T);
    const T* in = static_cast<const T*>(p.in);
    T* out = static_cast<T*>(p.out);
    if (p.vec) {
        const int64_t per = (p.cols + V - 1) / V, items = p.rows * per;
        RowWalk at(threadIdx.x, kClipThreads, (int)per);
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < items; i += kClipThreads, at.next()) {
            const int64_t c = (int64_t)at.part * V;
            const T* src = in + at.row * p.ld_in + c;
            T* dst = out + at.row * p.ld_out + c;
            T v[V];
            if (c + V <= p.cols) {
                *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(src);
                f(v, dst, std::integral_constant<int, V>{});
            } else {
                for (int j = 0; j < p.cols - c; ++j) {
                    v[0] = src[j];
                    f(v, dst + j, std::integral_constant<int, 1>{});
                }
            }
        }
        return;
    }
    const int64_t items = p.rows * p.cols;
    RowWalk at(threadIdx.x, kClipThreads, (int)p.cols);
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < items; i += kClipThreads, at.next()) {
        T v[1] = {in[at.row * p.ld_in + at.part]};
        f(v, out + at.row * p.ld_out + at.part, std::integral_constant<int, 1>{});
    }
}

struct ClipArgs {
    const Piece* pieces;
    int n;
    double* sums;          // [CTAs][3]
    uint32_t* ticket;      // zero before and after
    float* factor;
    float* norm;
    float limit;           // 0: the norm alone
};

__global__ void __launch_bounds__(kClipThreads) k_clip_norm(const ClipArgs a) {
    __shared__ double sh[3][kClipThreads / 32];
    __shared__ int last;
    pdl_wait();
    Squares q;
    for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
        const Piece p = a.pieces[i];
        const auto sum = [&](auto* v, auto*, auto n) {
#pragma unroll
            for (int j = 0; j < decltype(n)::value; ++j) q.add(Of<std::remove_reference_t<decltype(v[0])>>::get(v[j]));
        };
        if (p.type == NITRO_BF16) each<uint16_t>(p, sum);
        else if (p.type == NITRO_F32) each<float>(p, sum);
        else each<int64_t>(p, sum);
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const double s[3] = {warp_sum(q.mid), warp_sum(q.big), warp_sum(q.small)};
    if (lane == 0)
        for (int k = 0; k < 3; ++k) sh[k][warp] = s[k];
    __syncthreads();
    if (threadIdx.x < 3) {
        double v = 0.0;
        for (int w = 0; w < kClipThreads / 32; ++w) v += sh[threadIdx.x][w];
        a.sums[blockIdx.x * 3 + threadIdx.x] = v;
        __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        if (last) *a.ticket = 0;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (warp < 3) {
        double v = 0.0;
        for (int i = lane; i < gridDim.x; i += 32) v += __ldcg(a.sums + i * 3 + warp);
        v = warp_sum(v);
        if (lane == 0) sh[warp][0] = v;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    const double mid = sh[0][0], big = sh[1][0], small = sh[2][0];
    double norm = sqrt(mid);
    if (!(mid <= 3e38)) norm = sqrt(big) * 0x1p80;
    else if (mid < 0x1p-60) norm = sqrt(small) * 0x1p-90;
    *a.norm = (float)norm;
    *a.factor = norm > (double)a.limit && norm <= 1e300 ? (float)((double)a.limit / norm) : 1.0f;
}

__global__ void __launch_bounds__(kClipThreads) k_clip_scale(const ClipArgs a) {
    pdl_wait();
    const float f = *a.factor;
    for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
        const Piece p = a.pieces[i];
        if (!p.out || (f == 1.0f && p.out == p.in)) continue;
        const auto scale = [&](auto* v, auto* dst, auto n) {
            constexpr int V = decltype(n)::value;
            using T = std::remove_reference_t<decltype(v[0])>;
            T w[V];
#pragma unroll
            for (int j = 0; j < V; ++j) w[j] = f == 1.0f ? v[j] : Of<T>::put(Of<T>::get(v[j]) * f);
            if constexpr (V * sizeof(T) == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<uint4*>(w);
            else *dst = w[0];
        };
        if (p.type == NITRO_BF16) each<uint16_t>(p, scale);
        else each<float>(p, scale);
    }
}

int value_size(int type) { return type == NITRO_BF16 ? 2 : type == NITRO_F32 ? 4 : type == NITRO_I64 ? 8 : 0; }

// The bytes between a matrix's first and last value, and its rows within them
struct Range {
    uintptr_t at, end;
    int64_t pitch, width;      // bytes from row to row (0: a run without gaps), bytes of a row
};
Range range(const void* p, int64_t rows, int64_t cols, int64_t ld, int size) {
    const bool run = rows <= 1 || ld == cols;
    const uintptr_t at = (uintptr_t)p;
    return {at, at + (uintptr_t)(((rows - 1) * ld + cols) * size), run ? 0 : ld * size, cols * size};
}
bool overlap(const Range& a, const Range& b) {
    if (a.end <= b.at || b.end <= a.at) return false;
    if (a.pitch == 0 || a.pitch != b.pitch) return true;
    // columns of one wider buffer
    const int64_t d = (int64_t)((b.at > a.at ? b.at - a.at : a.at - b.at) % (uintptr_t)a.pitch);
    const int64_t first = b.at > a.at ? a.width : b.width, second = b.at > a.at ? b.width : a.width;
    return d < first || d + second > a.pitch;
}

}  // namespace
}  // namespace nitro

struct nitro_clip {
    int n = 0, ctas = 0;
    bool writes = false;
    double bytes = 0.0;
    Piece* pieces = nullptr;
    double* sums = nullptr;
    float* factor = nullptr;
    uint32_t* ticket = nullptr;
    bool clean = false;              // the ticket, see clear_once
    StatusWord status;
    DeviceAllocs allocs;
};

namespace {

// The pieces of all matrices into `to` (null: counted).  target: bytes of a piece
int64_t cut(const nitro_clip_matrix* list, int count, int64_t target, Piece* to) {
    int64_t n = 0;
    for (int i = 0; i < count; ++i) {
        nitro_clip_matrix m = list[i];
        if (m.rows == 0 || m.cols == 0) continue;
        const int size = value_size(m.type);
        if (m.rows == 1 || (m.ld_in == m.cols && (!m.out || m.ld_out == m.cols))) {
            m.cols *= m.rows;
            m.rows = 1;
        }
        const bool aligned = ((uintptr_t)m.in | (uintptr_t)m.out) % 16 == 0 &&
                             (m.rows == 1 || (m.ld_in * size % 16 == 0 && (!m.out || m.ld_out * size % 16 == 0)));
        const int64_t per = std::max<int64_t>(16, target / size / 16 * 16);      // values: a multiple of 16 bytes
        const int64_t wide = std::min(m.cols, per), tall = std::max<int64_t>(1, per / m.cols);
        for (int64_t r = 0; r < m.rows; r += tall)
            for (int64_t c = 0; c < m.cols; c += wide, ++n) {
                if (!to) continue;
                const char* in = static_cast<const char*>(m.in) + (r * m.ld_in + c) * size;
                char* out = m.out ? static_cast<char*>(m.out) + (r * m.ld_out + c) * size : nullptr;
                to[n] = {in, out, std::min(tall, m.rows - r), std::min(wide, m.cols - c), m.ld_in, m.ld_out, m.type, aligned};
            }
    }
    return n;
}

bool clip_list_ok(const nitro_clip_matrix* list, int count, double* bytes) {
    int64_t values = 0;
    for (int i = 0; i < count; ++i) {
        const nitro_clip_matrix& m = list[i];
        const int size = value_size(m.type);
        const int64_t most = (int64_t)1 << 40;
        if (size == 0 || m.rows < 0 || m.cols < 0 || m.rows > most || m.cols > most || m.ld_in > most || m.ld_out > most) return false;
        if (m.rows == 0 || m.cols == 0) continue;
        if (m.rows > most / m.cols || (values += m.rows * m.cols) > most) return false;
        if (!m.in || (uintptr_t)m.in % size || (uintptr_t)m.out % size || (m.out && m.type == NITRO_I64)) return false;
        if (m.rows > 1 && (m.ld_in < m.cols || (m.out && m.ld_out < m.cols))) return false;
        *bytes += (double)m.rows * m.cols * size;
    }
    return true;
}

// Whether every out is an `in` of its own or touches no other matrix.
bool outs_apart(const nitro_clip_matrix* list, int count) {
    struct Entry {
        Range r;
        int matrix;
        bool out;
    };
    std::vector<Entry> all;
    bool any = false;
    for (int i = 0; i < count; ++i) any = any || list[i].out;
    for (int i = 0; any && i < count; ++i) {
        const nitro_clip_matrix& m = list[i];
        if (m.rows == 0 || m.cols == 0) continue;
        const int size = value_size(m.type);
        all.push_back({range(m.in, m.rows, m.cols, m.ld_in, size), i, false});
        if (m.out) all.push_back({range(m.out, m.rows, m.cols, m.ld_out, size), i, true});
    }
    std::sort(all.begin(), all.end(), [](const Entry& a, const Entry& b) { return a.r.at < b.r.at; });
    std::vector<int> open;      // entries that reach past the current one's start
    for (int k = 0; k < (int)all.size(); ++k) {
        const Entry& e = all[k];
        int kept = 0;
        for (const int o : open) {
            const Entry& f = all[o];
            if (f.r.end <= e.r.at) continue;
            open[kept++] = o;
            if (!e.out && !f.out) continue;
            const nitro_clip_matrix& m = list[e.matrix];
            const bool itself = e.matrix == f.matrix && m.in == m.out && (m.rows == 1 || m.ld_in == m.ld_out);
            if (!itself && overlap(e.r, f.r)) return false;
        }
        open.resize(kept);
        open.push_back(k);
    }
    return true;
}

nitro_status clip_create(const nitro_clip_matrix* list, int count, nitro_clip** out) {
    double bytes = 0.0;
    if (!clip_list_ok(list, count, &bytes) || !outs_apart(list, count)) return NITRO_ERR_ARG;
    // Four pieces a CTA, so that none waits long for the last, of 4 to 64 KB
    const int most = kClipCtas * sm_count();
    int64_t target = std::min<int64_t>(65536, std::max<int64_t>(4096, (int64_t)(bytes / (4.0 * most))));
    int64_t n = cut(list, count, target, nullptr);
    while (n > kMostPieces && target < ((int64_t)1 << 30)) n = cut(list, count, target *= 4, nullptr);
    if (n > ((int64_t)1 << 30)) return NITRO_ERR_ARG;
    std::vector<Piece> host((size_t)n);
    cut(list, count, target, host.data());
    nitro_clip* h = new (std::nothrow) nitro_clip();
    if (!h) return NITRO_ERR_CUDA;
    h->n = (int)n;
    h->ctas = (int)std::max<int64_t>(1, std::min<int64_t>(n, most));
    h->bytes = bytes;
    for (int i = 0; i < count; ++i) h->writes = h->writes || (list[i].out && list[i].rows > 0 && list[i].cols > 0);
    const bool ok = h->allocs.take(&h->pieces, std::max<int64_t>(n, 1)) && h->allocs.take(&h->sums, 3 * h->ctas) &&
                    h->allocs.take(&h->factor, 1) && h->allocs.take(&h->ticket, 1) && h->status.take();
    // (on a stream of its own: the default one may be busy, or part of a capture)
    cudaStream_t s = nullptr;
    bool copied = ok && cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking) == cudaSuccess;
    if (copied) {
        copied = (n == 0 || cudaMemcpyAsync(h->pieces, host.data(), sizeof(Piece) * (size_t)n, cudaMemcpyHostToDevice, s) == cudaSuccess) &&
                 cudaStreamSynchronize(s) == cudaSuccess;
        cudaStreamDestroy(s);
    }
    if (!copied) {
        nitro_clip_destroy(h);
        return NITRO_ERR_CUDA;
    }
    *out = h;
    return NITRO_OK;
}

}  // namespace

extern "C" {

nitro_status nitro_clip_create(const nitro_clip_matrix* list, int count, nitro_clip** out) {
    if (!out) return NITRO_ERR_ARG;
    *out = nullptr;
    if (count < 0 || count > (1 << 20) || (count > 0 && !list)) return NITRO_ERR_ARG;
    try {
        return clip_create(list, count, out);
    } catch (...) {      // host memory
        return NITRO_ERR_CUDA;
    }
}

nitro_status nitro_clip_run(nitro_clip* h, float max_norm, float* norm, void* stream) {
    if (!h || !norm || (uintptr_t)norm % 4 || !(max_norm >= 0.0f) || (max_norm > 0.0f && !h->writes)) return NITRO_ERR_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    TRY(clear_once(h->clean, h->ticket, sizeof(uint32_t), s));
    const ClipArgs a{h->pieces, h->n, h->sums, h->ticket, h->factor, norm, max_norm};
    {
        ProfScope ps(K_CLIP, s, 0.0, h->bytes);
        TRY(launch_k(k_clip_norm, dim3(h->ctas), dim3(kClipThreads), 0, s, a));
    }
    if (max_norm > 0.0f) {
        ProfScope ps(K_CLIP, s, 0.0, 2.0 * h->bytes);
        TRY(launch_k(k_clip_scale, dim3(h->ctas), dim3(kClipThreads), 0, s, a));
    }
    return NITRO_OK;
}

nitro_status nitro_clip_status(nitro_clip* h, int clear) {
    if (!h) return NITRO_ERR_ARG;
    uint32_t bits = 0;
    if (!h->status.read(clear != 0, &bits)) return NITRO_ERR_CUDA;
    return bits & ST_TIMEOUT ? NITRO_ERR_TIMEOUT : NITRO_OK;
}

void nitro_clip_destroy(nitro_clip* h) {
    if (!h) return;
    cudaDeviceSynchronize();
    h->allocs.free();
    h->status.free();
    delete h;
}

}  // extern "C"
