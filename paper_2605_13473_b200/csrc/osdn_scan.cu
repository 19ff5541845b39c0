// Gated linear recurrence h_t = a_t h_{t-1} + b_t, a_t = exp(g_t), channel by channel: forward, backward, decode step.
#include <cstddef>

#include "osdn_rows.cuh"

namespace osdn {
namespace {

constexpr int TILE = 128;   // tokens between two states that the forward keeps for the backward

// exp(g) for g <= 0 in a form that keeps its distance from one.  Range reduction by powers of two (Cody and Waite:
// g = n ln 2 + r with ln 2 in two floats), expm1(r) by its Taylor series to r^7 (|r| <= 0.347: remainder below 2e-8 of r).
//   n = 0:  sign bit set, a = 1 + v, v = expm1(g), accurate relative to itself;
//   else:   sign bit clear, a = v.
// Stored as a rounded factor instead, a gate of -3e-4 keeps 1 - a to 1e-4 only, and the product of thousands of them
// drifts.  Factors below 2^-126 are zero.
struct Decay {
    float v;
    __device__ __forceinline__ static Decay of(float g)
    {
        g = g < -100.f ? -100.f : g;   // -inf too; a NaN stays one
        const float t = fmaf(g, 1.44269504f, 12582912.f);   // 1.5 * 2^23: the sum's low bits are round(g / ln 2)
        const float n = t - 12582912.f;
        float r = fmaf(n, -0.693147182f, g);
        r = fmaf(n, 1.90465421e-9f, r);                      // float(ln 2) - ln 2
        float q = fmaf(r, 1.f / 5040, 1.f / 720);
        q = fmaf(r, q, 1.f / 120);
        q = fmaf(r, q, 1.f / 24);
        q = fmaf(r, q, 1.f / 6);
        q = fmaf(r, q, 0.5f);
        const float p = fmaf(r * r, q, r);
        const float scale = __int_as_float((__float_as_int(t) << 23) + 0x3f800000);   // 2^n
        const float whole = n < -126.f ? 0.f : fmaf(p, scale, scale);
        return {n == 0.f && g <= 0.f ? -fabsf(p) : whole};
    }
    __device__ __forceinline__ bool near_one() const { return __float_as_int(v) < 0; }
    __device__ __forceinline__ float complement() const { return near_one() ? -v : 1.f - v; }
    __device__ __forceinline__ float times(float y) const { return fmaf(v, y, near_one() ? y : 0.f); }
    __device__ __forceinline__ float step(float h, float b) const { return fmaf(v, h, near_one() ? h + b : b); }   // a h + b
};

struct ScanArgs {
    const void *x, *dout;
    const float *gate, *init, *dfin;
    void *out, *dx;
    float *fin, *dgate, *dinit;
    float* saved;    // [tiles, C] (dense: [S, tiles, C]) state in front of every TILE-th row
    const int* cu;   // packed rows; else sequence s of a flat batch begins at row s T
    int S, T;        // sequences; rows of a dense sequence, or all packed rows
    int C, rows;     // rows of a walk: a dense sequence's, or the whole flat batch's
    int tiles, span; // tiles of a walk; CTAs that share it
    __device__ __forceinline__ int begin(int s) const { return cu ? cu[s] : s * T; }
};

// How a CTA covers a tile of TILE rows: groups of LANES threads side by side over LANES * VEC channels, each group TPG rows.
template <typename T_, int VEC_, int LANES_, int THREADS_> struct Cover {
    using T = T_;
    static constexpr int VEC = VEC_, LANES = LANES_, THREADS = THREADS_, WARPS = THREADS / 32, PER_WARP = 32 / LANES;
    static constexpr int CB = LANES * VEC, TPG = TILE * LANES / THREADS;
    static constexpr bool STAGED = VEC == 4;   // the next tile is on its way in shared memory while this one is computed
};
constexpr int MAX_SPAN = 16;

// VEC elements as they come from memory
template <typename T, int VEC> struct Raw;
template <> struct Raw<float, 4> {
    float4 v;
    __device__ __forceinline__ float get(int k) const { return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w; }
};
template <> struct Raw<__nv_bfloat16, 4> {
    uint2 v;
    __device__ __forceinline__ float get(int k) const
    {
        const uint32_t w = k < 2 ? v.x : v.y;
        return __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <typename T> struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ float get(int) const { return ldf(&v); }
};

template <int BYTES> __device__ __forceinline__ void copy_async(void* smem, const void* src, bool real)
{
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(smem);
    const int n = real ? BYTES : 0;   // the rest is filled with zeros
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(src), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(to), "l"(src), "r"(n), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Rows of one tensor, fetched tile by tile: each thread reads back what it copied itself.
template <typename E, int VEC, int N, int THREADS, bool STAGED> struct Fetch {
    Raw<E, VEC> r[N];
    __device__ __forceinline__ static void ask(char* stage, const E* p, size_t pitch, int live)
    {
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                copy_async<VEC * (int)sizeof(E)>(stage + (size_t)(i * THREADS + threadIdx.x) * VEC * sizeof(E),
                                                 i < live ? p + i * pitch : p, i < live);
        }
    }
    __device__ __forceinline__ void take(const char* stage, const E* p, size_t pitch, int live)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (STAGED) {
                r[i] = *reinterpret_cast<const Raw<E, VEC>*>(stage + (size_t)(i * THREADS + threadIdx.x) * VEC * sizeof(E));
            } else {
                r[i] = Raw<E, VEC>{};
                if (i < live) r[i] = *reinterpret_cast<const Raw<E, VEC>*>(p + i * pitch);
            }
        }
    }
};

// Where sequences begin and end among a group's rows t .. t+n-1 (bit i: row t + i); s: the sequence of row t.
struct Marks {
    unsigned first = 0, last = 0;
    int s = 0;
    __device__ __forceinline__ void find(const ScanArgs& a, int t, int n, int limit)
    {
        first = last = 0;
        if (t >= limit) return;
        n = min(n, limit - t);
        s = a.cu ? seq_of({a.cu, a.S, a.rows}, t) : t / a.T;
        for (int q = s, at = a.begin(q) == t ? t : -1;;) {
            if (at >= 0) first |= 1u << (at - t);
            const int end = max(a.begin(q + 1), max(at, t) + 1);
            if (end > t + n) break;
            last |= 1u << (end - 1 - t);
            if (end >= t + n) break;
            q = next(a, q, end);
            at = end;
        }
    }
    // the sequence that row t belongs to, the one before it being of sequence q
    __device__ __forceinline__ static int next(const ScanArgs& a, int q, int t)
    {
        ++q;
        while (q + 1 < a.S && a.begin(q + 1) <= t) ++q;
        return min(q, a.S - 1);
    }
};

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <int VEC> __device__ __forceinline__ void store_remote(float* mine, uint32_t rank, const float (&x)[VEC])
{
    uint32_t to;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    if constexpr (VEC == 4)
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]) : "memory");
    else
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(x[0]) : "memory");
}

// A stretch of rows maps the state in front of it to a h + b: the sum of its log gates, and b.
template <int VEC> struct Affine {
    float g[VEC], b[VEC];
};

__device__ __forceinline__ int div_up_dev(int a, int b) { return (a + b - 1) / b; }
// The sequence in front of q that is not empty (one there is: q does not begin the rows).
__device__ __forceinline__ int previous(const ScanArgs& a, int q)
{
    const int t = a.begin(q);
    --q;
    while (q > 0 && a.begin(q) >= t) --q;
    return max(q, 0);
}

// What the warps of a CTA (and the CTAs of a walk) tell one another: factor and b of their stretch; two sets, used in turn.
template <typename V> struct Exchange {
    float v[2][V::WARPS][V::CB], b[2][V::WARPS][V::CB], g[2][V::WARPS][V::CB];
    float cv[2][MAX_SPAN][V::CB], cb[2][MAX_SPAN][V::CB];
    // shared memory that a walk of `span` CTAs needs of it: a single one has no use for the last two
    static size_t bytes(int span) { return span > 1 ? sizeof(Exchange) : offsetof(Exchange, cv); }
};
template <typename V> struct Inner {   // the same for maps that stay inside a CTA
    float v[2][V::WARPS][V::CB], b[2][V::WARPS][V::CB];
};

// Within a warp, in the order of time (REVERSE: against it): `m` becomes the map of the stretches in front of this thread's own,
// and the warp's whole map goes to the exchange.
template <typename V, bool REVERSE, bool TOTALS, typename X>
__device__ __forceinline__ void meet_warp(Affine<V::VEC>& m, X& ex, int set)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, place = lane / V::LANES, c = (lane % V::LANES) * V::VEC;
#pragma unroll
    for (int d = 1; d < V::PER_WARP; d <<= 1) {
        const bool in = REVERSE ? place + d < V::PER_WARP : place >= d;
#pragma unroll
        for (int k = 0; k < V::VEC; ++k) {
            const float g = REVERSE ? __shfl_down_sync(~0u, m.g[k], d * V::LANES) : __shfl_up_sync(~0u, m.g[k], d * V::LANES);
            const float b = REVERSE ? __shfl_down_sync(~0u, m.b[k], d * V::LANES) : __shfl_up_sync(~0u, m.b[k], d * V::LANES);
            if (in) {
                m.b[k] = Decay::of(m.g[k]).step(b, m.b[k]);
                m.g[k] += g;
            }
        }
    }
    if (place == (REVERSE ? 0 : V::PER_WARP - 1)) {
        float v[V::VEC];
#pragma unroll
        for (int k = 0; k < V::VEC; ++k) v[k] = Decay::of(m.g[k]).v;
        store_vec<V::VEC>(&ex.v[set][warp][c], v);
        store_vec<V::VEC>(&ex.b[set][warp][c], m.b);
        if constexpr (TOTALS) store_vec<V::VEC>(&ex.g[set][warp][c], m.g);
    }
#pragma unroll
    for (int k = 0; k < V::VEC; ++k) {
        if constexpr (V::PER_WARP > 1) {
            const float g = REVERSE ? __shfl_down_sync(~0u, m.g[k], V::LANES) : __shfl_up_sync(~0u, m.g[k], V::LANES);
            const float b = REVERSE ? __shfl_down_sync(~0u, m.b[k], V::LANES) : __shfl_up_sync(~0u, m.b[k], V::LANES);
            const bool in = REVERSE ? place + 1 < V::PER_WARP : place > 0;
            m.g[k] = in ? g : 0.f;
            m.b[k] = in ? b : 0.f;
        } else {
            m.g[k] = 0.f;
            m.b[k] = 0.f;
        }
    }
}

template <int VEC> __device__ __forceinline__ void advance(float (&h)[VEC], const float* v, const float* b)
{
    float x[VEC], y[VEC];
    load_vec<VEC>(v, x);
    load_vec<VEC>(b, y);
#pragma unroll
    for (int k = 0; k < VEC; ++k) h[k] = Decay{x[k]}.step(h[k], y[k]);
}

// The CTA's whole map to every CTA of the walk (warp w to ranks w, w + WARPS, ..), behind a barrier that follows meet_warp.
template <typename V, bool REVERSE> __device__ __forceinline__ void tell_walk(Exchange<V>& ex, int set, uint32_t rank, int span)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane * V::VEC;
    if (lane >= V::LANES || warp >= span) return;
    float g[V::VEC] = {}, b[V::VEC] = {}, v[V::VEC];
    for (int j = 0; j < V::WARPS; ++j) {
        const int w = REVERSE ? V::WARPS - 1 - j : j;
        float x[V::VEC];
        load_vec<V::VEC>(&ex.g[set][w][c], x);
        advance<V::VEC>(b, &ex.v[set][w][c], &ex.b[set][w][c]);
#pragma unroll
        for (int k = 0; k < V::VEC; ++k) g[k] += x[k];
    }
#pragma unroll
    for (int k = 0; k < V::VEC; ++k) v[k] = Decay::of(g[k]).v;
    for (int r = warp; r < span; r += V::WARPS) {
        store_remote<V::VEC>(&ex.cv[set][rank][c], r, v);
        store_remote<V::VEC>(&ex.cb[set][rank][c], r, b);
    }
}

// The walk's state `base` through this tile row of CTAs; `mine`: in front of this CTA, then of this warp.
template <typename V, bool REVERSE>
__device__ __forceinline__ void fold(float (&base)[V::VEC], float (&mine)[V::VEC], float (&front)[V::VEC], const Exchange<V>& ex,
                                     int set, uint32_t rank, int span)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = (lane % V::LANES) * V::VEC;
    if (span > 1) {
        for (int r = 0; r < span; ++r) {
            if (r == (int)rank)
#pragma unroll
                for (int k = 0; k < V::VEC; ++k) mine[k] = base[k];
            advance<V::VEC>(base, &ex.cv[set][r][c], &ex.cb[set][r][c]);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V::VEC; ++k) mine[k] = base[k];
    }
#pragma unroll
    for (int k = 0; k < V::VEC; ++k) front[k] = mine[k];
    for (int j = 0; j < V::WARPS; ++j) {
        const int w = REVERSE ? V::WARPS - 1 - j : j;
        if (w == warp) {
#pragma unroll
            for (int k = 0; k < V::VEC; ++k) mine[k] = front[k];
            if (span > 1) break;
        }
        advance<V::VEC>(front, &ex.v[set][w][c], &ex.b[set][w][c]);
    }
    if (span == 1) {
#pragma unroll
        for (int k = 0; k < V::VEC; ++k) base[k] = front[k];
    }
}

// A state of an empty sequence (or its gradient) passes through; `place` of `places` thread groups of the walk.
template <int VEC>
__device__ __forceinline__ void pass_empty(const ScanArgs& a, const float* from, float* to, int place, int places, int c)
{
    for (int s = place; s < a.S; s += places) {
        if (a.cu[s + 1] > a.cu[s]) continue;
        float v[VEC] = {};
        if (from) load_vec<VEC>(from + (size_t)s * a.C + c, v);
        store_vec<VEC>(to + (size_t)s * a.C + c, v);
    }
}

// One walk = one dense sequence, or a whole flat batch with resets where sequences begin, over CB channels.  The walk's CTAs
// (span of them, one cluster) take a row of tiles at a time, each TILE rows: every thread maps its TPG rows to (sum of gates,
// b), the maps are combined over warp, CTA and cluster, and the rows are walked a second time from registers with the state
// in front of them.  out == nullptr: only the states are kept.
template <typename V, bool COMP, bool FLAT>
__global__ void __launch_bounds__(V::THREADS, 512 / V::THREADS) scan_fwd_kernel(ScanArgs a)
{
    using T = typename V::T;
    extern __shared__ __align__(16) char shared[];
    Exchange<V>& ex = *reinterpret_cast<Exchange<V>*>(shared + V::STAGED * TILE * V::CB * (4 + sizeof(T)));
    char* const stage = shared;
    pdl_wait();
    constexpr int VEC = V::VEC, TPG = V::TPG;
    const int lane = threadIdx.x & 31, group = threadIdx.x / V::LANES;
    const uint32_t rank = a.span > 1 ? cluster_rank() : 0;
    const int nblk = div_up_dev(a.C, V::CB);
    const int walk = blockIdx.x / a.span, s = walk / nblk;
    const int c = (walk % nblk) * V::CB + (lane % V::LANES) * VEC;
    const bool inside = c < a.C;
    const int limit = FLAT ? (a.cu ? min(max(a.cu[a.S], 0), a.rows) : a.rows) : a.rows;
    const size_t row0 = FLAT ? 0 : (size_t)s * a.rows;
    const T* x = static_cast<const T*>(a.x) + row0 * a.C + c;
    const float* gate = a.gate + row0 * a.C + c;
    T* out = static_cast<T*>(a.out) + row0 * a.C + c;
    float* saved = a.saved ? a.saved + (FLAT ? 0 : (size_t)s * a.tiles * a.C) + c : nullptr;
    if (FLAT && a.cu && a.fin && inside)
        pass_empty<VEC>(a, a.init, a.fin, rank * (V::THREADS / V::LANES) + group, a.span * (V::THREADS / V::LANES), c);
    float base[VEC] = {};
    if (!FLAT && a.init && inside) load_vec<VEC>(a.init + (size_t)s * a.C + c, base);
    char* gstage = stage;
    char* xstage = stage + V::THREADS * TPG * VEC * 4;
    const int steps = div_up_dev(a.tiles, a.span);
    using FetchG = Fetch<float, VEC, TPG, V::THREADS, V::STAGED>;
    using FetchX = Fetch<T, VEC, TPG, V::THREADS, V::STAGED>;
    auto row_of = [&](int step) { return (step * a.span + (int)rank) * TILE + group * TPG; };
    auto live_of = [&](int t) { return inside ? min(max(limit - t, 0), TPG) : 0; };
    auto ask = [&](int step) {
        const int t = row_of(step), live = live_of(t);
        const size_t at = live ? (size_t)t * a.C : 0;
        FetchG::ask(gstage, inside ? gate + at : a.gate, a.C, live);
        FetchX::ask(xstage, inside ? x + at : static_cast<const T*>(a.x), a.C, live);
    };
    if (V::STAGED) ask(0);
    if (a.span > 1) cluster_meet();   // every CTA of the walk runs before another one writes to its shared memory
    for (int step = 0; step < steps; ++step) {
        const int t = row_of(step), live = live_of(t), set = step & 1;
        const size_t at = (size_t)t * a.C;
        Marks marks;
        if (FLAT) marks.find(a, t, TPG, limit);
        FetchG fg;
        FetchX fx;
        if (V::STAGED) copies_wait();
        fg.take(gstage, gate + at, a.C, live);
        fx.take(xstage, x + at, a.C, live);
        Decay d[TPG][VEC];
        Affine<VEC> m = {};
        int q = marks.s;
#pragma unroll
        for (int i = 0; i < TPG; ++i) {
            if (FLAT && (marks.first >> i & 1)) {
                if (i) q = Marks::next(a, q, t + i);
                float h[VEC] = {};
                if (a.init && inside) load_vec<VEC>(a.init + (size_t)q * a.C + c, h);
#pragma unroll
                for (int k = 0; k < VEC; ++k) { m.b[k] = h[k]; m.g[k] = -INFINITY; }
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float g = fg.r[i].get(k);
                d[i][k] = Decay::of(g);
                const float y = fx.r[i].get(k);
                m.g[k] += g;
                m.b[k] = d[i][k].step(m.b[k], COMP ? d[i][k].complement() * y : y);
            }
        }
        meet_warp<V, false, true>(m, ex, set);
        __syncthreads();
        if (V::STAGED && step + 1 < steps) ask(step + 1);
        if (a.span > 1) {
            tell_walk<V, false>(ex, set, rank, a.span);
            cluster_meet();
        }
        float h[VEC], front[VEC];
        float mine[VEC];
        fold<V, false>(base, mine, front, ex, set, rank, a.span);
#pragma unroll
        for (int k = 0; k < VEC; ++k) h[k] = Decay::of(m.g[k]).step(mine[k], m.b[k]);
        if (saved && group == 0 && inside && t < a.tiles * TILE) store_vec<VEC>(saved + (size_t)(t / TILE) * a.C, h);
        q = marks.s;
#pragma unroll
        for (int i = 0; i < TPG; ++i) {
            if (i >= live) break;
            if (FLAT && (marks.first >> i & 1)) {
                if (i) q = Marks::next(a, q, t + i);
#pragma unroll
                for (int k = 0; k < VEC; ++k) h[k] = 0.f;
                if (a.init) load_vec<VEC>(a.init + (size_t)q * a.C + c, h);
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float y = fx.r[i].get(k);
                h[k] = d[i][k].step(h[k], COMP ? d[i][k].complement() * y : y);
            }
            if (a.out) store_vec<VEC>(out + at + (size_t)i * a.C, h);
            if (FLAT && a.fin && (marks.last >> i & 1)) store_vec<VEC>(a.fin + (size_t)q * a.C + c, h);
        }
    }
    if (!FLAT && a.fin && inside && rank == 0 && group == 0) store_vec<VEC>(a.fin + (size_t)s * a.C + c, base);
}

// The same walk from the end: e = a (dout + e), the state's gradient as the row before sees it.  Each tile walks its states
// forward again from the one that the forward kept, so that the gates' gradients take fp32 states:
//   dgate_t = (h_{t-1} [- x_t]) e_t,   dx_t = dh_t or (1 - a_t) dh_t,   dh_t = dout_t + e_{t+1}.
template <typename V, bool COMP, bool FLAT>
__global__ void __launch_bounds__(V::THREADS, 512 / V::THREADS) scan_bwd_kernel(ScanArgs a)
{
    using T = typename V::T;
    extern __shared__ __align__(16) char shared[];
    Inner<V>& inner = *reinterpret_cast<Inner<V>*>(shared);
    char* const stage = shared + sizeof(Inner<V>);
    Exchange<V>& ex = *reinterpret_cast<Exchange<V>*>(stage + V::STAGED * TILE * V::CB * (4 + 2 * sizeof(T)));
    pdl_wait();
    constexpr int VEC = V::VEC, TPG = V::TPG;
    const int lane = threadIdx.x & 31, group = threadIdx.x / V::LANES;
    const uint32_t rank = a.span > 1 ? cluster_rank() : 0;
    const int nblk = div_up_dev(a.C, V::CB);
    const int walk = blockIdx.x / a.span, s = walk / nblk;
    const int c = (walk % nblk) * V::CB + (lane % V::LANES) * VEC;
    const bool inside = c < a.C;
    const int limit = FLAT ? (a.cu ? min(max(a.cu[a.S], 0), a.rows) : a.rows) : a.rows;
    const size_t row0 = FLAT ? 0 : (size_t)s * a.rows;
    const T* x = static_cast<const T*>(a.x) + row0 * a.C + c;
    const T* dout = static_cast<const T*>(a.dout) + row0 * a.C + c;
    const float* gate = a.gate + row0 * a.C + c;
    T* dx = static_cast<T*>(a.dx) + row0 * a.C + c;
    float* dgate = a.dgate + row0 * a.C + c;
    const float* saved = a.saved + (FLAT ? 0 : (size_t)s * a.tiles * a.C) + c;
    if (FLAT && a.cu && a.dinit && inside)
        pass_empty<VEC>(a, a.dfin, a.dinit, rank * (V::THREADS / V::LANES) + group, a.span * (V::THREADS / V::LANES), c);
    float base[VEC] = {};
    if (!FLAT && a.dfin && inside) load_vec<VEC>(a.dfin + (size_t)s * a.C + c, base);
    char* gstage = stage;
    char* xstage = gstage + V::THREADS * TPG * VEC * 4;
    char* ystage = xstage + V::THREADS * TPG * VEC * sizeof(T);
    const int steps = div_up_dev(a.tiles, a.span);
    using FetchG = Fetch<float, VEC, TPG, V::THREADS, V::STAGED>;
    using FetchX = Fetch<T, VEC, TPG, V::THREADS, V::STAGED>;
    auto row_of = [&](int step) { return (a.tiles - 1 - step * a.span - (int)rank) * TILE + group * TPG; };   // < 0: none
    auto live_of = [&](int t) { return inside && t >= 0 ? min(max(limit - t, 0), TPG) : 0; };
    auto ask = [&](int step) {
        const int t = row_of(step), live = live_of(t);
        const size_t at = live ? (size_t)t * a.C : 0;
        FetchG::ask(gstage, inside ? gate + at : a.gate, a.C, live);
        FetchX::ask(xstage, inside ? x + at : static_cast<const T*>(a.x), a.C, live);
        FetchX::ask(ystage, inside ? dout + at : static_cast<const T*>(a.dout), a.C, live);
    };
    if (V::STAGED) ask(0);
    if (a.span > 1) cluster_meet();   // every CTA of the walk runs before another one writes to its shared memory
    for (int step = 0; step < steps; ++step) {
        const int t = row_of(step), live = live_of(t), set = step & 1;
        const size_t at = t >= 0 ? (size_t)t * a.C : 0;
        Marks marks;
        if (FLAT && t >= 0) marks.find(a, t, TPG, limit);
        FetchG fg;
        FetchX fx, fy;
        float h[VEC] = {};
        if (live) load_vec<VEC>(saved + (size_t)(t / TILE) * a.C, h);
        if (V::STAGED) copies_wait();
        fg.take(gstage, gate + at, a.C, live);
        fx.take(xstage, x + at, a.C, live);
        fy.take(ystage, dout + at, a.C, live);
        Decay d[TPG][VEC];
        Affine<VEC> m = {}, r = {};
        int q = marks.s;
#pragma unroll
        for (int i = 0; i < TPG; ++i) {
            if (FLAT && (marks.first >> i & 1)) {
                if (i) q = Marks::next(a, q, t + i);
                float f[VEC] = {};
                if (a.init && inside) load_vec<VEC>(a.init + (size_t)q * a.C + c, f);
#pragma unroll
                for (int k = 0; k < VEC; ++k) { m.b[k] = f[k]; m.g[k] = -INFINITY; }
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float g = fg.r[i].get(k);
                d[i][k] = Decay::of(g);
                const float y = fx.r[i].get(k);
                m.g[k] += g;
                r.g[k] += g;
                m.b[k] = d[i][k].step(m.b[k], COMP ? d[i][k].complement() * y : y);
            }
        }
        // against time: the sequence of the last row first
        int qlast = q;
        if (FLAT && marks.last) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) r.g[k] = -INFINITY;
        }
        q = qlast;
#pragma unroll
        for (int i = TPG - 1; i >= 0; --i) {
            if (FLAT && (marks.last >> i & 1)) {
                float f[VEC] = {};
                if (a.dfin && inside) load_vec<VEC>(a.dfin + (size_t)q * a.C + c, f);
#pragma unroll
                for (int k = 0; k < VEC; ++k) r.b[k] = f[k];
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) r.b[k] = d[i][k].times(fy.r[i].get(k) + r.b[k]);
            if (FLAT && i && (marks.first >> i & 1)) q = previous(a, q);
        }
        meet_warp<V, false, false>(m, inner, set);
        meet_warp<V, true, true>(r, ex, set);
        __syncthreads();
        if (V::STAGED && step + 1 < steps) ask(step + 1);
        if (a.span > 1) {
            tell_walk<V, true>(ex, set, rank, a.span);
            cluster_meet();
        }
        float e[VEC], front[VEC];
        fold<V, true>(base, e, front, ex, set, rank, a.span);
#pragma unroll
        for (int k = 0; k < VEC; ++k) e[k] = Decay::of(r.g[k]).step(e[k], r.b[k]);
        for (int w = 0; w < (int)(threadIdx.x >> 5); ++w)
            advance<VEC>(h, &inner.v[set][w][(lane % V::LANES) * VEC], &inner.b[set][w][(lane % V::LANES) * VEC]);
        float before[TPG][VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) h[k] = Decay::of(m.g[k]).step(h[k], m.b[k]);
        q = marks.s;
#pragma unroll
        for (int i = 0; i < TPG; ++i) {
            if (FLAT && (marks.first >> i & 1)) {
                if (i) q = Marks::next(a, q, t + i);
#pragma unroll
                for (int k = 0; k < VEC; ++k) h[k] = 0.f;
                if (a.init && inside) load_vec<VEC>(a.init + (size_t)q * a.C + c, h);
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float y = fx.r[i].get(k);
                before[i][k] = h[k];
                h[k] = d[i][k].step(h[k], COMP ? d[i][k].complement() * y : y);
            }
        }
        q = qlast;
#pragma unroll
        for (int i = TPG - 1; i >= 0; --i) {
            if (i < live) {
                if (FLAT && (marks.last >> i & 1)) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) e[k] = 0.f;
                    if (a.dfin) load_vec<VEC>(a.dfin + (size_t)q * a.C + c, e);
                }
                float px[VEC], pg[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const float dh = fy.r[i].get(k) + e[k];
                    e[k] = d[i][k].times(dh);
                    px[k] = COMP ? d[i][k].complement() * dh : dh;
                    pg[k] = (COMP ? before[i][k] - fx.r[i].get(k) : before[i][k]) * e[k];
                }
                store_vec<VEC>(dx + at + (size_t)i * a.C, px);
                store_vec<VEC>(dgate + at + (size_t)i * a.C, pg);
                if (FLAT && (marks.first >> i & 1)) {
                    if (a.dinit) store_vec<VEC>(a.dinit + (size_t)q * a.C + c, e);
                    if (i) q = previous(a, q);
                }
            }
        }
    }
    if (!FLAT && a.dinit && inside && rank == 0 && group == 0) store_vec<VEC>(a.dinit + (size_t)s * a.C + c, base);
}

// One thread per N channels of a sequence; the cached state is read and written once.
template <typename T, int N, bool COMP>
__global__ void __launch_bounds__(128) scan_step_kernel(const T* x, const float* gate, float* state, T* out, int B, int L, int C)
{
    pdl_wait();
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const int n = C / N;
    if (i >= (long long)B * n) return;
    const size_t b = i / n, c = (size_t)(i % n) * N;
    float h[N];
    load_vec<N>(state + b * C + c, h);
    for (int t = 0; t < L; ++t) {
        const size_t at = (b * L + t) * C + c;
        float g[N], y[N];
        load_vec<N>(gate + at, g);
        load_vec<N>(x + at, y);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const Decay d = Decay::of(g[j]);
            h[j] = d.step(h[j], COMP ? d.complement() * y[j] : y[j]);
        }
        store_vec<N>(out + at, h);
    }
    store_vec<N>(state + b * C + c, h);
}

// Sequences shorter than a tile are walked as one flat batch.
bool is_flat(const osdn_scan_params& p) { return p.nseq > 0 || (p.B > 1 && p.T < TILE); }

ScanArgs make_args(const osdn_scan_params& p)
{
    ScanArgs a{};
    a.cu = p.nseq > 0 ? p.cu_seqlens : nullptr;
    a.S = p.nseq > 0 ? p.nseq : p.B;
    a.T = p.T;
    a.C = p.C;
    a.rows = p.nseq > 0 || !is_flat(p) ? p.T : p.B * p.T;
    a.tiles = div_up(a.rows, TILE);
    return a;
}

template <typename V> bool launch_walks(void (*kernel)(ScanArgs), ScanArgs a, bool flat, int row_bytes, size_t inner, cudaStream_t st)
{
    const long long walks = (long long)(flat ? 1 : a.S) * div_up(a.C, V::CB);
    a.span = 1;
    while (a.span < MAX_SPAN && a.span < a.tiles && walks * a.span < 148 * 2) a.span *= 2;
    const size_t smem = inner + (V::STAGED ? (size_t)TILE * V::CB * row_bytes : 0) + Exchange<V>::bytes(a.span);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
    if (a.span > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return false;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(walks * a.span));
    cfg.blockDim = dim3(V::THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.span;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.span > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess;
}

template <typename T, bool COMP> bool launch_forward(const ScanArgs& a, bool flat, cudaStream_t st)
{
    auto go = [&](auto cover) {
        using V = decltype(cover);
        return launch_walks<V>(flat ? scan_fwd_kernel<V, COMP, true> : scan_fwd_kernel<V, COMP, false>, a, flat, 4 + sizeof(T), 0, st);
    };
    return a.C % 4 == 0 ? go(Cover<T, 4, 16, 256>{}) : go(Cover<T, 1, 32, 256>{});
}

template <typename T, bool COMP> int run_backward(const ScanArgs& a, bool flat, bool saved, cudaStream_t st)
{
    int n = 1;
    if (!saved) {
        if (!launch_forward<T, COMP>(a, flat, st)) return -1;   // out and fin are NULL: the states alone
        ++n;
    }
    auto go = [&](auto cover) {
        using V = decltype(cover);
        return launch_walks<V>(flat ? scan_bwd_kernel<V, COMP, true> : scan_bwd_kernel<V, COMP, false>, a, flat, 4 + 2 * sizeof(T),
                               sizeof(Inner<V>), st);
    };
    // fp32: twice the threads, half the rows each, for the registers that a row's values take
    const bool ok = a.C % 4 == 0 ? go(Cover<T, 4, 16, 512>{}) : go(Cover<T, 1, 32, 256>{});
    return ok ? n : -1;
}

template <typename T, int N, bool COMP>
bool launch_step(const osdn_scan_params& p, const void* x, const float* gate, float* state, void* out, cudaStream_t st)
{
    return launch_after(scan_step_kernel<T, N, COMP>, dim3(div_up((long long)p.B * (p.C / N), 128)), dim3(128), 0, st,
                        static_cast<const T*>(x), gate, state, static_cast<T*>(out), p.B, p.T, p.C);
}

template <typename F> int by_type(const osdn_scan_params& p, F f)   // f(element, input gate)
{
    const bool comp = p.input_gate == OSDN_INPUT_COMPLEMENT;
    if (p.io_dtype == OSDN_FP32) return comp ? f(0.f, std::true_type{}) : f(0.f, std::false_type{});
    return comp ? f(__nv_bfloat16{}, std::true_type{}) : f(__nv_bfloat16{}, std::false_type{});
}

}  // namespace

size_t scan_workspace(const osdn_scan_params& p)
{
    const ScanArgs a = make_args(p);
    return align_up((size_t)(is_flat(p) ? 1 : p.B) * a.tiles * p.C * 4, 256);
}

int scan_forward(const osdn_scan_params& p, const void* x, const float* gate, const float* init, void* out, float* fin,
                 void* ws, cudaStream_t st)
{
    ScanArgs a = make_args(p);
    a.x = x; a.gate = gate; a.init = init; a.out = out; a.fin = fin;
    a.saved = static_cast<float*>(ws);
    stage_mark(st, "scan_fwd");
    const int n = by_type(p, [&](auto e, auto comp) { return launch_forward<decltype(e), decltype(comp)::value>(a, is_flat(p), st) ? 1 : -1; });
    stage_end(st);
    return n;
}

int scan_backward(const osdn_scan_params& p, const void* x, const float* gate, const float* init, const void* dout,
                  const float* dfin, void* dx, float* dgate, float* dinit, void* ws, cudaStream_t st)
{
    ScanArgs a = make_args(p);
    a.x = x; a.gate = gate; a.init = init; a.dout = dout; a.dfin = dfin; a.dx = dx; a.dgate = dgate; a.dinit = dinit;
    a.saved = static_cast<float*>(ws);
    const bool saved = (p.flags & OSDN_FLAG_RESIDUALS_VALID) != 0;
    stage_mark(st, "scan_bwd");
    const int n = by_type(p, [&](auto e, auto comp) { return run_backward<decltype(e), decltype(comp)::value>(a, is_flat(p), saved, st); });
    stage_end(st);
    return n;
}

int scan_step(const osdn_scan_params& p, const void* x, const float* gate, float* state, void* out, cudaStream_t st)
{
    stage_mark(st, "scan_step");
    const int n = by_type(p, [&](auto e, auto comp) {
        using T = decltype(e);
        constexpr bool COMP = decltype(comp)::value;
        return (p.C % 4 == 0 ? launch_step<T, 4, COMP>(p, x, gate, state, out, st) : launch_step<T, 1, COMP>(p, x, gate, state, out, st)) ? 1 : -1;
    });
    stage_end(st);
    return n;
}

}  // namespace osdn
