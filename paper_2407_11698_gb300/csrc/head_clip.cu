// The norm over many gradients, sqrt(sum x^2) over all values of all matrices, and the gradients scaled by
// min(1, max_norm / norm).
//
// At creation the matrices are cut into pieces, kept in a table on the device, so that each warp of one CTA an SM has about
// the same bytes.  One cooperative launch: the warps sum their pieces' squares, every CTA waits for
// all CTAs' sums and adds them in the same order, and the warps scale their pieces, last ones first (the second level cache
// holds them).  A warp's first 13 KB stay in shared memory in between, so that up to 31 MB of
// gradients are read once; where there are more, 7 KB, and the others come through a ring of places there.
// 48 tensors, 2.6 GB: 1290 us, 6.0 TB/s over the values' two ways in and one out (the first 448 us, with SMs up to a sixth apart);
// 300 tensors, 29 MB: 25 us, of which 9 are loads, 3 sums, 3 notes and 6 stores; six tensors, 1 MB: 8.3.
// Squares are summed three times, of x, of x 2^-100 and of x 2^90: the first passes fp32 from |x| = 2^64 on and
// loses values below 2^-75, and where its sum shows that, one of the others stands for it.  Of 2^40 values the largest have a sum of 2^96
// in the second, and where the first passes 2^126 those that count are above 2^43, their squares in the second above 2^-114.
#include <new>

#include <cmath>
#include <cstring>
#include <vector>

#include "head_act.cuh"

using namespace nitro;

namespace nitro {
namespace {

constexpr int kClipThreads = 512, kClipWarps = kClipThreads / 32;
constexpr int kClipPlaces = 27;                                   // vectors of a lane in shared memory
constexpr int kClipGroups = 3, kClipGroup = 4;                    // of those the ones under way, in groups, where not all are to stay
constexpr int kClipRing = kClipGroups * kClipGroup;
constexpr int kClipSmem = kClipPlaces * kClipThreads * 16;
constexpr int kClipNotes = 5;                                     // that a lane looks at together
constexpr int64_t kMostPieces = (int64_t)1 << 26;

// How a piece's values are reached: one by one; as vectors, where rows start at multiples of 16 bytes on both sides; or,
// where they do not and the gaps between them are small, as all vectors from its first to its last value, of which
// the gaps and what lies beside the piece in its first and last vector count for nothing (those 16 bytes hold a value of
// the piece, so they are memory that is there).
enum : int { kSingles = 0, kRows = 1, kSpan = 2 };

// Rows of one matrix (of lone rows: a run of one)
struct Piece {
    const void* in;
    void* out;             // or null
    int64_t ld_in, ld_out;
    int rows, cols;
    int type, how;
};

// What a warp does: its first piece, how many it has, and where the others are
struct alignas(16) Work {
    Piece first;
    int n, rest;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll 1
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// A sum of 32-bit numbers with what its roundings leave over.  (64-bit additions would be as good, but one takes a warp
// some hundred clocks here: the three sums over warps, CTAs and the grid took 2.5 us longer.)
struct Exact {
    float hi = 0.0f, lo = 0.0f;
    __device__ __forceinline__ void add(float h, float l) {
        const float s = hi + h, b = s - hi;
        lo += l + ((hi - (s - b)) + (h - b));
        hi = s;
    }
    __device__ __forceinline__ void over_warp() {
#pragma unroll 1
        for (int d = 16; d > 0; d >>= 1) add(__shfl_xor_sync(0xffffffffu, hi, d), __shfl_xor_sync(0xffffffffu, lo, d));
    }
    // (what an infinite sum leaves over is a NaN)
    __device__ __forceinline__ float value() const { return hi <= 3e38f ? hi + lo : hi; }
};

// Sums of squares.  A lane's run takes kRun pairs at most before it goes to sums that keep what their roundings leave over: many squares are
// far below a long run's last place and are lost more often than they are rounded up, and equal ones are all rounded
// the same way (1500 equal values in one run: a norm 1.2e-5 off).
constexpr int kRun = 16;
constexpr float kBig = 0x1p-100f, kSmall = 0x1p90f;       // what values are scaled by in the other two sums
static_assert(kClipGroup * 8 / 2 <= kRun, "a run of vectors is a group");
struct Squares {
    float2 run = {0.0f, 0.0f}, run_big = {0.0f, 0.0f}, run_small = {0.0f, 0.0f};
    Exact mid, big, small;
    __device__ __forceinline__ void add(float2 x) {
        run = fma2(x, x, run);
        const float2 b = mul2(x, pair(kBig)), s = mul2(x, pair(kSmall));
        run_big = fma2(b, b, run_big);
        run_small = fma2(s, s, run_small);
    }
    __device__ __forceinline__ void end_run() {
        mid.add(run.x + run.y, 0.0f);
        big.add(run_big.x + run_big.y, 0.0f);
        small.add(run_small.x + run_small.y, 0.0f);
        run = run_big = run_small = pair(0.0f);
    }
};

// A type's 16 bytes as pairs of fp32 and back, and one value
template <typename T>
struct Of;
template <>
struct Of<uint16_t> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void get(const uint4& u, float2* v) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 put(const float2* v) {
        return make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
    }
    static __device__ __forceinline__ float get(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t put(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
};
template <>
struct Of<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void get(const uint4& u, float2* v) {
        v[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        v[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ uint4 put(const float2* v) {
        return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
    }
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Of<int64_t> {
    static constexpr int V = 2;
    static __device__ __forceinline__ void get(const uint4& u, float2* v) {
        v[0] = make_float2((float)(int64_t)(u.x | (uint64_t)u.y << 32), (float)(int64_t)(u.z | (uint64_t)u.w << 32));
    }
    static __device__ __forceinline__ float get(int64_t v) { return (float)v; }
};

// A piece's work: vectors, `items` of them, in rows of `per` where they are rows', and single values, the rows' ends or
// all of them.
template <typename T_, bool SPAN>
struct Parts {
    using T = T_;
    static constexpr bool kSpan = SPAN;
    static constexpr int V = Of<T>::V;
    int per, tail;               // whole vectors of a row, and values after them
    int items, singles;          // (a piece has at most 2^30 bytes)
    int before;                  // values in the first vector that are not the piece's
    __device__ __forceinline__ explicit Parts(const Piece& p) {
        before = 0;
        if constexpr (SPAN) {
            before = (int)((uintptr_t)p.in & 15) / (int)sizeof(T);
            per = tail = singles = 0;
            items = (before + (p.rows - 1) * (int)p.ld_in + p.cols + V - 1) / V;
        } else {
            per = p.how == kRows ? p.cols / V : 0;
            tail = p.cols - per * V;
            items = p.rows * per;
            singles = p.rows * tail;
        }
    }
    // steps that a warp takes for the vectors
    __device__ __forceinline__ int steps() const { return (items + 31) / 32; }
    // the addresses of vector i in `in` and, of rows, in `out`
    __device__ __forceinline__ const uint4* in(const Piece& p, int i) const {
        if constexpr (SPAN) return reinterpret_cast<const uint4*>((uintptr_t)p.in & ~(uintptr_t)15) + i;
        int row = 0;
        if (p.rows > 1) row = (uint32_t)i / (uint32_t)per;
        return reinterpret_cast<const uint4*>(static_cast<const T*>(p.in) + row * p.ld_in) + (i - row * per);
    }
    __device__ __forceinline__ uint4* out(const Piece& p, int i) const {
        int row = 0;
        if (p.rows > 1) row = (uint32_t)i / (uint32_t)per;
        return reinterpret_cast<uint4*>(static_cast<T*>(p.out) + row * p.ld_out) + (i - row * per);
    }
};
// f(address in `in`, address in `out`) for the lane's single values; end() after every kRun, and after the last
template <class Q, class F, class End>
__device__ __forceinline__ void singles(const Piece& p, const Q& q, int lane, F&& f, End&& end) {
    using T = typename Q::T;
    if (q.tail == 0) return;
    RowWalk at(lane, 32, q.tail);
    for (int i = lane; i < q.singles;) {
        const int to = min(q.singles, i + 32 * kRun);
#pragma unroll 4
        for (; i < to; i += 32, at.next()) {
            const int c = q.per * Of<T>::V + at.part;
            f(static_cast<const T*>(p.in) + at.row * p.ld_in + c, static_cast<T*>(p.out) + at.row * p.ld_out + c);
        }
        end();
    }
}

__device__ __forceinline__ void copy16(uint4* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

// Starts the copies of a piece's vectors while of `keep` places some are left; `kept`: the lane's first place.
// Steps of the piece.
template <class Q>
__device__ __forceinline__ int keep_piece(const Piece& p, int lane, uint4* kept, int keep, int slot) {
    const Q q(p);
    const int steps = q.steps(), n = min(steps, keep - slot);
#pragma unroll 4
    for (int k = 0; k < n; ++k)
        if (k * 32 + lane < q.items) copy16(kept + (slot + k) * 32, q.in(p, k * 32 + lane));
    return steps;
}

// f(step, the lane's place of its vector), by all lanes, for the steps from `from` on, last ones first, through a ring of
// places; end() after every few
template <class Q, class F, class End>
__device__ __forceinline__ void stream_piece(const Piece& p, const Q& q, int lane, uint4* ring, int from, F&& f, End&& end) {
    const auto fetch = [&](int last, uint4* to) {       // steps last, last - 1, ...
#pragma unroll
        for (int j = 0; j < kClipGroup; ++j) {
            const int step = last - j, i = step * 32 + lane;
            if (step >= from && i < q.items) copy16(to + j * 32, q.in(p, i));
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int k = q.steps() - 1;
#pragma unroll
    for (int g = 0; g < kClipGroups; ++g) fetch(k - g * kClipGroup, ring + g * kClipGroup * 32);
    for (int g = 0; k >= from; k -= kClipGroup) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kClipGroups - 1) : "memory");
        uint4* at = ring + g * kClipGroup * 32;
#pragma unroll
        for (int j = 0; j < kClipGroup; ++j)
            if (k - j >= from) f(k - j, at + j * 32);
        end();
        fetch(k - kClipRing, at);
        if (++g == kClipGroups) g = 0;
    }
}

// Vector i of a piece
template <class Q>
__device__ __forceinline__ void sum_vector(const Piece& p, const Q& q, int i, const uint4& u, Squares& sum) {
    constexpr int V = Q::V;
    if (i >= q.items) return;
    float2 v[V / 2];
    Of<typename Q::T>::get(u, v);
    if constexpr (Q::kSpan) {
        // values of the gaps, of the row's and beside the piece
        const int e = i * V - q.before, ld = (int)p.ld_in, end = (p.rows - 1) * ld + p.cols;
        int c = e < 0 ? e : (int)((uint32_t)e % (uint32_t)ld);
        if (e < 0 || e + V > end || c + V > p.cols) {
#pragma unroll
            for (int j = 0; j < V; ++j, ++c) {
                if (c >= ld) c = 0;
                float& x = j & 1 ? v[j >> 1].y : v[j >> 1].x;
                x = c >= 0 && c < p.cols && e + j < end ? x : 0.0f;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V / 2; ++j) sum.add(v[j]);
}

// Squares of what is not kept of a piece
template <class Q>
__device__ __forceinline__ int sum_piece(const Piece& p, int lane, uint4* ring, int keep, int slot, Squares& sum) {
    const Q q(p);
    const int steps = q.steps(), from = max(0, keep - slot);
    if (steps > from)
        stream_piece(p, q, lane, ring, from, [&](int step, uint4* at) { sum_vector(p, q, step * 32 + lane, *at, sum); },
                        [&] { sum.end_run(); });
    using T = typename Q::T;
    singles(p, q, lane, [&](const T* in, T*) { sum.add(make_float2(Of<T>::get(*in), 0.0f)); }, [&] { sum.end_run(); });
    return steps;
}

// and of what is
template <class Q>
__device__ __forceinline__ int sum_kept(const Piece& p, int lane, const uint4* kept, int keep, int slot, Squares& sum) {
    const Q q(p);
    const int steps = q.steps(), n = min(steps, keep - slot);
    for (int k = 0; k < n; k += kClipGroup) {
#pragma unroll
        for (int j = 0; j < kClipGroup; ++j)
            if (k + j < n) sum_vector(p, q, (k + j) * 32 + lane, kept[(slot + k + j) * 32], sum);
        sum.end_run();
    }
    return steps;
}

// What values are scaled by.  A factor below 2^-100, which 32 bits hold with few digits or not at all, is f kTinyStep^2: values that
// are not 0 once it has scaled them lose nothing in x kTinyStep, and (x kTinyStep) f passes neither end of the range.
constexpr float kTinyStep = 0x1p-76f;
struct Factor {
    float f;
    int tiny;
    __device__ __forceinline__ bool one() const { return f == 1.0f && !tiny; }
    __device__ __forceinline__ float times(float x) const { return tiny ? x * kTinyStep * f * kTinyStep : x * f; }
};

template <typename T>
__device__ __forceinline__ uint4 scaled(uint4 u, const Factor& f) {
    if (f.one()) return u;
    float2 v[Of<T>::V / 2];
    Of<T>::get(u, v);
    if (f.tiny) {
#pragma unroll
        for (int j = 0; j < Of<T>::V / 2; ++j) v[j] = mul2(mul2(mul2(v[j], pair(kTinyStep)), pair(f.f)), pair(kTinyStep));
    } else {
#pragma unroll
        for (int j = 0; j < Of<T>::V / 2; ++j) v[j] = mul2(v[j], pair(f.f));
    }
    return Of<T>::put(v);
}

// A step of a span: its 32 vectors, scaled, lie one after another at the lanes' places, and go out a value a lane, in
// their order.
template <class Q>
__device__ __forceinline__ void store_span(const Piece& p, const Q& q, int lane, int step, uint4* at, const Factor& f) {
    using T = typename Q::T;
    constexpr int E = 32 * Q::V;
    if (step * 32 + lane < q.items) *at = scaled<T>(*at, f);
    __syncwarp();
    const T* from = reinterpret_cast<const T*>(at - lane) + lane;
    const int ld = (int)p.ld_in, end = (p.rows - 1) * ld + p.cols;
    int e = step * E - q.before + lane;
    int row = e > 0 ? (uint32_t)e / (uint32_t)ld : 0, c = e - row * ld;
    T* to = static_cast<T*>(p.out) + row * p.ld_out + c;
#pragma unroll
    for (int k = 0; k < E; k += 32) {
        if (c >= 0 && c < p.cols && e < end) *to = from[k];
        e += 32, c += 32, to += 32;
        while (c >= ld) c -= ld, to += p.ld_out - ld;
    }
    __syncwarp();
}

// A piece scaled, its last vectors first; `slot` as above
template <class Q>
__device__ __forceinline__ void scale_piece(const Piece& p, int lane, uint4* kept, uint4* ring, int keep, int slot, const Factor& f) {
    const Q q(p);
    using T = typename Q::T;
    singles(p, q, lane, [&](const T* in, T* out) { *out = f.one() ? *in : Of<T>::put(f.times(Of<T>::get(*in))); }, [] {});
    const int steps = q.steps(), left = min(steps, max(0, keep - slot));         // steps that are kept
    if constexpr (Q::kSpan) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
        if (steps > left)
            stream_piece(p, q, lane, ring, left, [&](int step, uint4* at) { store_span(p, q, lane, step, at, f); }, [] {});
        for (int k = 0; k < left; ++k) store_span(p, q, lane, k, kept + (slot + k) * 32, f);
    } else {
        const auto one = [&](int step, const uint4* at) {
            const int i = step * 32 + lane;
            if (i < q.items) *q.out(p, i) = scaled<T>(*at, f);
        };
        if (steps > left) stream_piece(p, q, lane, ring, left, one, [] {});
#pragma unroll 4
        for (int k = 0; k < left; ++k) one(k, kept + (slot + k) * 32);
    }
}

// f(the piece's kind of Parts)
template <class Q>
struct Kind {
    using type = Q;
};
template <class F>
__device__ __forceinline__ int with_kind(const Piece& p, F&& f) {
    const bool span = p.how == kSpan;
    if (p.type == NITRO_BF16) return span ? f(Kind<Parts<uint16_t, true>>()) : f(Kind<Parts<uint16_t, false>>());
    if (p.type == NITRO_F32) return span ? f(Kind<Parts<float, true>>()) : f(Kind<Parts<float, false>>());
    return span ? f(Kind<Parts<int64_t, true>>()) : f(Kind<Parts<int64_t, false>>());
}

// What a CTA hands to the others: two numbers and the turn that they belong to, as one access of 16 bytes
struct alignas(16) Note {
    float a, b;
    uint64_t turn;
};
__device__ __forceinline__ void put_note(Note* to, float a, float b, uint64_t turn) {
    const uint64_t bits = __float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
    asm volatile("{\n .reg .b128 t;\n mov.b128 t, {%1, %2};\n st.relaxed.gpu.global.b128 [%0], t;\n}" ::"l"(to), "l"(bits), "l"(turn) : "memory");
}
__device__ __forceinline__ Note get_note(const Note* from) {
    uint64_t bits, turn;
    asm volatile("{\n .reg .b128 t;\n ld.relaxed.gpu.global.b128 t, [%2];\n mov.b128 {%0, %1}, t;\n}" : "=l"(bits), "=l"(turn) : "l"(from) : "memory");
    return {__uint_as_float((uint32_t)bits), __uint_as_float((uint32_t)(bits >> 32)), turn};
}
// f(note) for every 32nd CTA's note, once it is of this turn; gives up after a while (in_time false)
template <class F>
__device__ __forceinline__ void take_notes(const Note* notes, uint64_t turn, int lane, uint64_t& t0, bool& in_time, F&& f) {
    for (int i0 = lane; i0 < gridDim.x && in_time; i0 += 32 * kClipNotes) {
        Note n[kClipNotes];
        for (uint32_t k = 1;; ++k) {
            bool here = true;
#pragma unroll
            for (int j = 0; j < kClipNotes; ++j)
                if (i0 + 32 * j < gridDim.x) n[j] = get_note(notes + i0 + 32 * j);
#pragma unroll
            for (int j = 0; j < kClipNotes; ++j)
                if (i0 + 32 * j < gridDim.x) here = here && n[j].turn == turn;
            if (here) break;
            if ((k & 63) == 0) {           // (a read of the timer takes longer than most waits)
                const uint64_t now = global_ns();
                if (t0 == 0) t0 = now;
                if (now - t0 > kWaitNs) {
                    in_time = false;
                    break;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kClipNotes; ++j)
            if (i0 + 32 * j < gridDim.x) f(n[j]);
    }
}
// Sums of plain squares that are right
constexpr float kLeastMid = 0x1p-60f;
__device__ __forceinline__ bool in_range(float mid) { return mid >= kLeastMid && mid <= 1e38f; }

struct ClipArgs {
    const Work* work;      // [warps]
    const Piece* pieces;
    Note* notes;           // [2][CTAs]: the plain squares' sum, and the others'
    uint64_t* turn;        // how often the handle has run
    float* norm;
    float limit;           // 0: the norm alone
    int keep;              // vectors of a lane that stay in shared memory: all places, where they hold all of them
    uint32_t* status;
};

__global__ void __launch_bounds__(kClipThreads) k_clip(const ClipArgs a) {
    extern __shared__ uint4 stash[];      // [warps][places][32]
    __shared__ float4 sh[kClipWarps];
    __shared__ Factor factor;
    __shared__ int ok;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int keep = a.keep;
    uint4 *kept = stash + warp * kClipPlaces * 32 + lane, *ring = kept + (kClipPlaces - kClipRing) * 32;
    const Work work = a.work[blockIdx.x * kClipWarps + warp];
    const auto piece = [&](int i) { return i == 0 ? work.first : a.pieces[work.rest + i - 1]; };
    const uint64_t turn = *a.turn + 1;
    int slot = 0;
    for (int i = 0; i < work.n && slot < keep; ++i) {
        const Piece p = piece(i);
        slot += with_kind(p, [&](auto t) { return keep_piece<typename decltype(t)::type>(p, lane, kept, keep, slot); });
    }
    Squares q;
    slot = 0;
    for (int i = 0; i < work.n; ++i) {
        const Piece p = piece(i);
        slot += with_kind(p, [&](auto t) { return sum_piece<typename decltype(t)::type>(p, lane, ring, keep, slot, q); });
    }
    const int end = slot;
    asm volatile("cp.async.wait_all;" ::: "memory");
    slot = 0;
    for (int i = 0; i < work.n && slot < keep; ++i) {
        const Piece p = piece(i);
        slot += with_kind(p, [&](auto t) { return sum_kept<typename decltype(t)::type>(p, lane, kept, keep, slot, q); });
    }
    {
        Exact mid = q.mid;
        mid.over_warp();
        const float big = warp_sum(q.big.value()), small = warp_sum(q.small.value());
        if (lane == 0) sh[warp] = make_float4(mid.hi, mid.lo, big, small);
    }
    if (threadIdx.x == 0) ok = 1;
    __syncthreads();
    if (warp == 0) {
        const float4 mine = lane < kClipWarps ? sh[lane] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        Exact mid;
        mid.add(mine.x, mine.y);
        mid.over_warp();
        float big = warp_sum(mine.z), small = warp_sum(mine.w);
        if (gridDim.x > 1) {
            // Every CTA takes all CTAs' notes of this turn (of the norm alone: the first one).
            Note* own = a.notes + blockIdx.x;
            if (lane == 0) put_note(own, mid.hi, mid.lo, turn);
            if (lane == 1) put_note(own + gridDim.x, big, small, turn);
            if (a.limit == 0.0f && blockIdx.x != 0) return;
            uint64_t t0 = 0;
            bool in_time = true;
            mid = Exact();
            take_notes(a.notes, turn, lane, t0, in_time, [&](const Note& n) { mid.add(n.a, n.b); });
            mid.over_warp();
            if (!in_range(mid.hi)) {
                big = small = 0.0f;
                take_notes(a.notes + gridDim.x, turn, lane, t0, in_time, [&](const Note& n) { big += n.a, small += n.b; });
                big = warp_sum(big), small = warp_sum(small);
            }
            if (!__all_sync(0xffffffffu, in_time) && lane == 0) {
                atomicOr(a.status, ST_TIMEOUT);
                ok = 0;
            }
        }
        if (lane == 0) {
            // root + rest of the sum in the range that holds it, and the norm over that: 1 / unit.  The factor is limit unit / norm,
            // where the products are powers of two of `limit` without loss; step: 2^76 sqrt(unit), a tiny one's other part
            float root, rest = 0.0f, unit = 1.0f, step = 1.0f / kTinyStep;
            const bool large = !in_range(mid.hi) && !(mid.hi < kLeastMid);
            if (in_range(mid.hi)) {
                root = sqrtf(mid.hi);
                rest = (fmaf(-root, root, mid.hi) + mid.lo) * (0.5f / root);
            } else if (mid.hi < kLeastMid) {
                root = sqrtf(small);
                unit = kSmall;
                step = 0x1p121f;
            } else {
                root = sqrtf(big);
                unit = kBig;
                step = 0x1p26f;
            }
            const float norm = root + rest;
            if (blockIdx.x == 0) {
                *a.norm = norm / unit;
                *a.turn = turn;              // every CTA has read it: its notes are there
            }
            Factor f{1.0f, 0};
            if (norm > a.limit * unit && norm <= 3e38f) {
                f.tiny = a.limit * unit < norm * 0x1p-100f;
                // (limit kBig may lose digits: of large norms that is the last product)
                const float limit = f.tiny ? a.limit * step * step : large ? a.limit : a.limit * unit;
                f.f = limit / norm;
                f.f += (fmaf(-f.f, root, limit) - f.f * rest) / norm;
                if (large && !f.tiny) f.f *= unit;
            }
            factor = f;
        }
    }
    if (a.limit == 0.0f) return;
    __syncthreads();
    if (!ok) return;
    const Factor f = factor;
    slot = end;
    for (int i = work.n - 1; i >= 0; --i) {
        const Piece p = piece(i);
        with_kind(p, [&](auto t) {
            using Q = typename decltype(t)::type;
            slot -= Q(p).steps();
            if constexpr (sizeof(typename Q::T) < 8)
                if (p.out && !(f.one() && p.out == p.in)) scale_piece<Q>(p, lane, kept, ring, keep, slot, f);
            return 0;
        });
    }
}

int value_size(int type) { return type == NITRO_BF16 ? 2 : type == NITRO_F32 ? 4 : type == NITRO_I64 ? 8 : 0; }

// The bytes between a matrix's first and last value, and its rows within them
struct Range {
    uintptr_t at, end;
    int64_t pitch, width;      // bytes from row to row (0: a run without gaps), bytes of a row, or of the run
};
Range range(const void* p, int64_t rows, int64_t cols, int64_t ld, int size) {
    const bool run = rows <= 1 || ld == cols;
    const uintptr_t at = (uintptr_t)p;
    const int64_t bytes = ((rows - 1) * ld + cols) * size;
    return {at, at + (uintptr_t)bytes, run ? 0 : ld * size, run ? bytes : cols * size};
}
bool overlap(const Range& a, const Range& b) {
    if (a.end <= b.at || b.end <= a.at) return false;
    const int64_t pitch = std::max(a.pitch, b.pitch);
    if (pitch == 0 || (a.pitch != b.pitch && a.pitch != 0 && b.pitch != 0)) return true;
    // columns of one wider buffer, or of it and of one of its rows
    const int64_t d = (int64_t)((b.at > a.at ? b.at - a.at : a.at - b.at) % (uintptr_t)pitch);
    const int64_t first = b.at > a.at ? a.width : b.width, second = b.at > a.at ? b.width : a.width;
    return d < first || d + second > pitch;
}

}  // namespace
}  // namespace nitro

struct nitro_clip {
    int ctas = 0, keep = 0;
    bool writes = true;              // an out, or there are no values
    double bytes = 0.0;
    Note* notes = nullptr;           // [2][CTAs], and the turn; then work and pieces
    Work* work = nullptr;
    Piece* pieces = nullptr;
    // What all of them hold before the first run, page-locked, and whether they do.  The first run copies it, on its own stream:
    // a copy at creation would wait behind what the default stream has queued.  A captured run holds the copy too
    // and does not count as the first (see clear_once).
    uint8_t* start = nullptr;
    int64_t start_bytes = 0;
    bool started = false;
    StatusWord status;
    DeviceAllocs allocs;
};

namespace {

// Bytes that a piece costs beside its own: its description, and a step that it does not fill
constexpr int64_t kPieceCost = 512;
constexpr int64_t kLine = 512;       // a warp's vectors
constexpr int64_t kSpanGap = 64;     // bytes between rows that are read over

// A matrix as its pieces are made of it: without gaps it is one row
struct Whole {
    int64_t rows, cols, ld_in, ld_out;
    int size, how;
    int64_t pitch;           // bytes that a row costs
    explicit Whole(const nitro_clip_matrix& m) : rows(m.rows), cols(m.cols), ld_in(m.ld_in), ld_out(m.ld_out), size(value_size(m.type)) {
        if (rows == 1 || (ld_in == cols && (!m.out || ld_out == cols))) {
            cols *= rows;
            rows = 1;
        }
        const bool aligned = ((uintptr_t)m.in | (uintptr_t)m.out) % 16 == 0 &&
                             (rows == 1 || (ld_in * size % 16 == 0 && (!m.out || ld_out * size % 16 == 0)));
        const bool span = rows == 1 || ((ld_in - cols) * size <= kSpanGap && ld_in < (1 << 28));
        how = aligned ? kRows : span ? kSpan : kSingles;
        pitch = (rows > 1 && how == kSpan ? ld_in : cols) * size;
    }
    int64_t cost() const { return rows > 0 && cols > 0 ? kPieceCost + rows * pitch : 0; }
};

// All matrices as pieces, one warp's after another's: `share` of their cost to each.  to, first: null to count
// last: the cost that was left for the last warp
int64_t cut(const nitro_clip_matrix* list, int count, int64_t share, Piece* to, int* first, int warps, int64_t* last) {
    int64_t n = 0, used = 0;
    int w = 0;
    if (first) first[0] = 0;
    const auto next_warp = [&] {
        used = 0;
        ++w;
        if (first && w <= warps) first[w] = (int)n;
    };
    for (int i = 0; i < count; ++i) {
        const Whole m(list[i]);
        if (m.rows == 0 || m.cols == 0) continue;
        for (int64_t r = 0, c = 0; r < m.rows;) {
            // rows that are still the warp's; of rows longer than its share, whole lines; the last warp takes all that is left
            const int64_t most = std::min<int64_t>(w + 1 < warps ? std::max(share - used - kPieceCost, kLine) : (int64_t)1 << 30, (int64_t)1 << 30);
            int64_t rows = 1, cols = m.cols - c;
            if (c == 0 && m.pitch <= std::max(most, 4 * kLine)) rows = std::min(m.rows - r, std::max<int64_t>(1, most / m.pitch));
            else cols = std::min(cols, most / kLine * kLine / m.size);
            if (to) {
                const char* in = static_cast<const char*>(list[i].in) + (r * m.ld_in + c) * m.size;
                char* out = list[i].out ? static_cast<char*>(list[i].out) + (r * m.ld_out + c) * m.size : nullptr;
                to[n] = {in, out, rows > 1 ? m.ld_in : cols, rows > 1 ? m.ld_out : cols, (int)rows, (int)cols, list[i].type, m.how};
            }
            ++n;
            used += kPieceCost + (rows > 1 ? rows * m.pitch : cols * m.size);
            c += cols;
            if (c == m.cols) c = 0, r += rows;
            if (used + kPieceCost + kLine > share && w + 1 < warps) next_warp();
        }
    }
    *last = w + 1 == warps ? used : 0;
    while (w < warps) next_warp();
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

static_assert(sizeof(Note) % alignof(Work) == 0 && sizeof(Work) % alignof(Piece) == 0, "they follow one another");

cudaError_t start_once(nitro_clip* h, cudaStream_t s) {
    if (h->started) return cudaSuccess;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &capture);
    if (e == cudaSuccess) e = cudaMemcpyAsync(h->notes, h->start, (size_t)h->start_bytes, cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess && capture == cudaStreamCaptureStatusNone) h->started = true;
    return e;
}

nitro_status clip_create(const nitro_clip_matrix* list, int count, nitro_clip** out) {
    double bytes = 0.0;
    if (!clip_list_ok(list, count, &bytes) || !outs_apart(list, count)) return NITRO_ERR_ARG;
    // an SM's worth of threads takes 16 KB at once: fewer CTAs where there is less, and a cheaper barrier
    int64_t cost = 0;
    for (int i = 0; i < count; ++i) cost += Whole(list[i]).cost();
    const int ctas = (int)std::max<int64_t>(1, std::min<int64_t>(sm_count(), (cost + 16383) / 16384)), warps = ctas * kClipWarps;
    // (matrices that end inside a share, and rows, leave the others more than the mean)
    int64_t share = std::max<int64_t>((cost + warps - 1) / warps + kLine, 2 * kPieceCost), last = 0, n = 0;
    for (int tries = 0; tries < 64; ++tries, share += share / 64 + 64) {
        n = cut(list, count, share, nullptr, nullptr, warps, &last);
        if (last <= share) break;
    }
    if (n > kMostPieces) return NITRO_ERR_ARG;
    std::vector<Piece> host((size_t)n);
    std::vector<int> first((size_t)warps + 1);
    cut(list, count, share, host.data(), first.data(), warps, &last);
    std::vector<Work> work((size_t)warps);
    for (int w = 0; w < warps; ++w) {
        work[w].n = first[w + 1] - first[w];
        work[w].rest = first[w] + 1;
        work[w].first = work[w].n ? host[first[w]] : Piece{};
    }
    nitro_clip* h = new (std::nothrow) nitro_clip();
    if (!h) return NITRO_ERR_CUDA;
    h->ctas = ctas;
    int64_t most_steps = 0;
    for (int w = 0; w < warps; ++w) {
        int64_t steps = 0;
        for (int i = first[w]; i < first[w + 1]; ++i) {
            const Piece& p = host[i];
            const int64_t size = value_size(p.type), row = p.cols * size / 16, span = ((p.rows - 1) * p.ld_in + p.cols) * size / 16 + 2;
            if (p.how != kSingles) steps += ((p.how == kRows ? p.rows * row : span) + 31) / 32;
        }
        most_steps = std::max(most_steps, steps);
    }
    h->keep = most_steps <= kClipPlaces ? kClipPlaces : kClipPlaces - kClipRing;
    h->bytes = bytes;
    for (int i = 0; i < count; ++i) h->writes = h->writes && (list[i].rows == 0 || list[i].cols == 0);
    for (int i = 0; i < count; ++i) h->writes = h->writes || (list[i].out && list[i].rows > 0 && list[i].cols > 0);
    const int64_t notes = sizeof(Note) * (2 * ctas + 1), works = sizeof(Work) * work.size(), all = notes + works + sizeof(Piece) * n;
    uint8_t* block = nullptr;
    void* start = nullptr;
    if (!h->allocs.take(&block, all) || !h->status.take() || !allocated(cudaMallocHost(&start, (size_t)all))) {
        nitro_clip_destroy(h);
        return NITRO_ERR_CUDA;
    }
    h->start = static_cast<uint8_t*>(start);
    h->start_bytes = all;
    memset(h->start, 0, (size_t)notes);
    memcpy(h->start + notes, work.data(), (size_t)works);
    if (n) memcpy(h->start + notes + works, host.data(), sizeof(Piece) * (size_t)n);
    h->notes = reinterpret_cast<Note*>(block);
    h->work = reinterpret_cast<Work*>(block + notes);
    h->pieces = reinterpret_cast<Piece*>(block + notes + works);
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
    TRY(start_once(h, s));
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    sm_count(&dev);
    TRY(once_per_device(ready, dev, [] { return cudaFuncSetAttribute(k_clip, cudaFuncAttributeMaxDynamicSharedMemorySize, kClipSmem); }));
    const ClipArgs a{h->work, h->pieces, h->notes, &h->notes[2 * h->ctas].turn, norm, max_norm, h->keep, h->status.at};
    ProfScope ps(K_CLIP, s, 0.0, (max_norm > 0.0f ? 2.0 : 1.0) * h->bytes);
    // (its CTAs wait for one another)
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(h->ctas);
    cfg.blockDim = dim3(kClipThreads);
    cfg.dynamicSmemBytes = kClipSmem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    TRY(cudaLaunchKernelEx(&cfg, k_clip, a));
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
    if (h->start) cudaFreeHost(h->start);
    delete h;
}

}  // extern "C"
