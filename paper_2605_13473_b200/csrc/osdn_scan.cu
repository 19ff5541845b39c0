// Gated linear recurrence h_t = a_t h_{t-1} + b_t, a_t = exp(g_t), channel by channel: forward, backward, decode step.
#include <cfloat>
#include <cstddef>

#include "osdn_rows.cuh"

namespace osdn {
namespace {

constexpr int SIDE = 4;   // rows whose factors are worked out side by side (one by one: forward of 8 x 2048 tokens 36 us, so 27)
// Rows that a warp takes at a time; the forward keeps the state in front of each such stretch for the backward.
constexpr int UNIT = 8;

// exp(g) for g <= 0 as the sum of two floats, hi the nearest one to it:
//   |g| <= 1/4:  from expm1(g) by its Taylor series to g^6 (remainder below 5e-8 of it): the sum keeps the distance from one;
//   else:        hi alone, by the hardware's exponential: 2^-22 of a, and 1.25 |g| 2^-24 by the rounding of g log2(e) (g = -20:
//                2^-20; a is 2e-9 there).  a <= 0.78 forgets either within a few tokens; -inf is zero.
// As one rounded factor, a gate of -3e-4 keeps 1 - a to 1e-4 only, and a product of thousands of them drifts.  Two floats cost
// one packed fma more a step and no selection (with the form chosen at every step 38 instructions an element instead of 29).
template <int N> struct Decay {
    F<N> hi, lo;
    __device__ __forceinline__ static Decay of(const F<N>& g)
    {
        Decay d[1];
        of<1>(&g, d);
        return d[0];
    }
    // K of them step by step side by side: one alone is a chain of ten dependent operations
    template <int K> __device__ __forceinline__ static void of(const F<N>* g, Decay* d)
    {
        F<N> q[K];
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = mul(g[i], all<N>(1.44269504f));
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d[i].hi.x[k]) : "f"(q[i].x[k]));
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = fma(g[i], all<N>(1.f / 720), all<N>(1.f / 120));
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = fma(g[i], q[i], all<N>(1.f / 24));
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = fma(g[i], q[i], all<N>(1.f / 6));
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = fma(g[i], q[i], all<N>(0.5f));
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = mul(g[i], q[i]);
#pragma unroll
        for (int i = 0; i < K; ++i) q[i] = fma(g[i], q[i], g[i]);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const F<N> near = add(q[i], all<N>(1.f));
            const F<N> rest = add(q[i], fma(near, all<N>(-1.f), all<N>(1.f)));   // p - (near - 1), exact
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const bool is = fabsf(g[i].x[k]) <= 0.25f;
                d[i].hi.x[k] = is ? near.x[k] : d[i].hi.x[k];
                d[i].lo.x[k] = is ? rest.x[k] : 0.f;
            }
        }
    }
    __device__ __forceinline__ F<N> complement() const { return fma(lo, all<N>(-1.f), fma(hi, all<N>(-1.f), all<N>(1.f))); }   // 1 - a
    __device__ __forceinline__ F<N> times(const F<N>& y) const { return fma(hi, y, mul(lo, y)); }                    // a y
    __device__ __forceinline__ F<N> step(const F<N>& h, const F<N>& b) const { return fma(hi, h, fma(lo, h, b)); }   // a h + b
};

struct ScanArgs {
    const void *x, *dout;
    const float *gate, *init, *dfin;
    void *out, *dx;
    float *fin, *dgate, *dinit;
    float* saved;    // [units, C] (dense: [S, units, C]) state in front of every UNIT-th row
    const int* cu;   // packed rows; else sequence s of a flat batch begins at row s T
    int S, T;        // sequences; rows of a dense sequence, or all packed rows
    int C, rows;     // rows of a walk: a dense sequence's, or the whole flat batch's
    int units, span; // units of a walk; CTAs that share it
    __device__ __forceinline__ int begin(int s) const { return cu ? cu[s] : s * T; }
};

// How a CTA covers its rows: its warps take units in turn, over CB channels, VEC to a lane.
template <typename T_, int VEC_, int WARPS_, int DEPTH_> struct Cover {
    using T = T_;
    static_assert(WARPS_ <= 16, "a named barrier for each warp");
    static constexpr int VEC = VEC_, WARPS = WARPS_, DEPTH = DEPTH_, CB = 32 * VEC, TPG = UNIT;
    static constexpr bool STAGED = VEC == 2;   // a warp's next unit is on its way in shared memory while it computes one
};
constexpr int MAX_SPAN = 16;

// VEC elements as they come from memory
template <typename T, int VEC> struct Raw;
template <> struct Raw<float, 2> {
    float2 v;
    __device__ __forceinline__ F<2> get() const { return {{v.x, v.y}}; }
};
template <> struct Raw<__nv_bfloat16, 2> {
    uint32_t v;
    __device__ __forceinline__ F<2> get() const { return {{__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)}}; }
};
template <typename T> struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ F<1> get() const { return {{ldf(&v)}}; }
};
template <int N> __device__ __forceinline__ F<N> read(const float* p)
{
    if constexpr (N == 2) {
        const float2 v = *reinterpret_cast<const float2*>(p);
        return {{v.x, v.y}};
    } else {
        return {{*p}};
    }
}
template <int N> __device__ __forceinline__ F<N> read_or_zero(const float* p, size_t at) { return p ? read<N>(p + at) : all<N>(0.f); }
template <int N> __device__ __forceinline__ void write(float* p, const F<N>& a)
{
    if constexpr (N == 2) *reinterpret_cast<float2*>(p) = make_float2(a.x[0], a.x[1]);
    else *p = a.x[0];
}
template <int N> __device__ __forceinline__ void write(__nv_bfloat16* p, const F<N>& a)
{
    if constexpr (N == 2) *reinterpret_cast<uint32_t*>(p) = pair_bf16(a.x[0], a.x[1]);
    else *p = __float2bfloat16_rn(a.x[0]);
}

// A warp's TPG rows of one tensor.  Staged: the warp copies them in 16-byte pieces to its own part of shared memory.
template <typename E, typename V> struct Fetch {
    Raw<E, V::VEC> r[V::TPG];
    static constexpr int ROW = V::CB * (int)sizeof(E), BYTES = V::TPG * ROW;   // of a warp
    // p: the block's first channel of the warp's first row; cols: channels of the block that there are
    __device__ __forceinline__ static void ask(char* part, const E* p, size_t pitch, int live, int cols)
    {
        if constexpr (V::STAGED) {
            constexpr int PIECES = ROW / 16, ROWS = 32 / PIECES, PER = 16 / (int)sizeof(E);
            const int lane = threadIdx.x & 31, row = lane / PIECES;
            const int col = (lane % PIECES) * PER;
            char* const to = part + lane * 16;
            const E* from = p + row * pitch + col;
            if (live >= V::TPG && cols >= V::CB) {   // nearly always
#pragma unroll
                for (int i = 0; i < V::TPG; i += ROWS, from += ROWS * pitch) copy_async16(to + i * ROW, from, true);
                return;
            }
#pragma unroll
            for (int i = 0; i < V::TPG; i += ROWS, from += ROWS * pitch) {
                const bool real = col < cols && i + row < live;
                copy_async16(to + i * ROW, real ? from : p, real);
            }
        }
    }
    __device__ __forceinline__ void take(const char* part, const E* p, size_t pitch, int live, int col, bool in)
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < V::TPG; ++i) {
            if constexpr (V::STAGED) {
                r[i] = *reinterpret_cast<const Raw<E, V::VEC>*>(part + i * ROW + lane * V::VEC * sizeof(E));
            } else {
                r[i] = Raw<E, V::VEC>{};
                if (in && i < live) r[i] = *reinterpret_cast<const Raw<E, V::VEC>*>(p + i * pitch + col);
            }
        }
    }
};

// Where sequences begin and end among a warp's rows t .. t+n-1 (bit i: row t + i); s: the sequence of row t.  The sequence of
// the last search is kept: a warp whose rows lie inside it reads nothing.
struct Marks {
    unsigned first = 0, last = 0;
    int s = 0;
    int begin = 0, end = 0;   // of the sequence last searched for
    __device__ __forceinline__ void find(const ScanArgs& a, int t, int n, int limit)
    {
        first = last = 0;
        if (t >= limit) return;
        n = min(n, limit - t);
        if (t > begin && t + n < end) return;
        if (!a.cu) {
            s = t / a.T;
            begin = s * a.T;
            end = begin + a.T;
            for (int at = begin; at < t + n; at += a.T) {
                if (at >= t) first |= 1u << (at - t);
                if (at + a.T <= t + n) last |= 1u << (at + a.T - 1 - t);
            }
            return;
        }
        // the last sequence that begins at or before t: 32 probes at a time
        const int lane = threadIdx.x & 31;
        int lo = 0, hi = a.S;
        while (hi - lo > 1) {
            const int pitch = (hi - lo + 31) / 32, i = lo + lane * pitch;
            const unsigned before = __ballot_sync(~0u, i < hi && a.cu[i] <= t);
            lo += (max(__popc(before), 1) - 1) * pitch;
            hi = min(hi, lo + pitch);
        }
        s = lo;
        begin = a.cu[s];
        end = a.cu[s + 1];
        for (int q = s; q < a.S; q += 32) {
            const bool in = q + lane < a.S;
            const int b = in ? a.cu[q + lane] : 0, e = in ? a.cu[q + lane + 1] : 0;
            const bool f = e > b && b >= t && b < t + n, l = e > b && e > t && e <= t + n;
            first |= __reduce_or_sync(~0u, f ? 1u << (b - t) : 0u);
            last |= __reduce_or_sync(~0u, l ? 1u << (e - 1 - t) : 0u);
            if (__shfl_sync(~0u, in && e < t + n, 31) == 0) break;
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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
template <int N> __device__ __forceinline__ F<N> read_remote(const float* mine, uint32_t rank)
{
    uint32_t at;
    F<N> a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    if constexpr (N == 2) asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(a.x[0]), "=f"(a.x[1]) : "r"(at) : "memory");
    else asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(a.x[0]) : "r"(at) : "memory");
    return a;
}
// One warp announces, the next one waits: a named barrier of 64 threads for each warp that waits.  A CTA has sixteen of them
// (with a number shared by two warps both may wait on it at once, and take one another for the announcement).
__device__ __forceinline__ void hand_on(int id) { asm volatile("bar.arrive %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void take_over(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
// Both at once, the state stepped in between: h from `mine`, a h + b to `next`.  One block of instructions, because this is
// what every warp of a walk waits for: left to itself the compiler puts work for later rows in between (forward of 8 x 2048
// tokens, 1024 channels: 28 to 41 us with how it happened to be scheduled).
template <int N>
__device__ __forceinline__ F<N> relay(int id, int next_id, const float* mine, float* next, const Decay<N>& d, const F<N>& b, F<N>& behind)
{
    const uint32_t from = (uint32_t)__cvta_generic_to_shared(mine), to = (uint32_t)__cvta_generic_to_shared(next);
    if constexpr (N == 2) {
        unsigned long long h, t;
        asm volatile("bar.sync %2, 64;\n\t"
                     "ld.shared.b64 %0, [%3];\n\t"
                     "fma.rn.f32x2 %1, %6, %0, %7;\n\t"
                     "fma.rn.f32x2 %1, %5, %0, %1;\n\t"
                     "st.shared.b64 [%4], %1;\n\t"
                     "bar.arrive %8, 64;"
                     : "=&l"(h), "=&l"(t) : "r"(id), "r"(from), "r"(to), "l"(pack(d.hi)), "l"(pack(d.lo)), "l"(pack(b)), "r"(next_id) : "memory");
        behind = unpack(t);
        return unpack(h);
    } else {
        float h, t;
        asm volatile("bar.sync %2, 64;\n\t"
                     "ld.shared.f32 %0, [%3];\n\t"
                     "fma.rn.f32 %1, %6, %0, %7;\n\t"
                     "fma.rn.f32 %1, %5, %0, %1;\n\t"
                     "st.shared.f32 [%4], %1;\n\t"
                     "bar.arrive %8, 64;"
                     : "=&f"(h), "=&f"(t) : "r"(id), "r"(from), "r"(to), "f"(d.hi.x[0]), "f"(d.lo.x[0]), "f"(b.x[0]), "r"(next_id) : "memory");
        behind = {{t}};
        return {{h}};
    }
}

// What the second walk over a unit needs is worked out before the wait for the state, and not put off or done again behind it.
template <int N> __device__ __forceinline__ void pin(Decay<N> (&d)[UNIT], F<N> (&y)[UNIT])
{
#pragma unroll
    for (int i = 0; i < UNIT; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) asm volatile("" : "+f"(d[i].hi.x[k]), "+f"(d[i].lo.x[k]), "+f"(y[i].x[k]));
}

// The sequence in front of q that is not empty (one there is: q does not begin the rows).
__device__ __forceinline__ int previous(const ScanArgs& a, int q)
{
    const int t = a.begin(q);
    --q;
    while (q > 0 && a.begin(q) >= t) --q;
    return max(q, 0);
}

template <typename V> struct Hand {
    float state[V::WARPS][V::CB];                    // in front of the unit that warp w takes next
    float g[V::WARPS][V::CB], b[V::WARPS][V::CB];    // a split walk: the maps of the warps' stretches
    float all_g[V::CB], all_b[V::CB];                //   and the CTA's
};

// A state of an empty sequence (or its gradient) passes through; `place` of `places` warps of the walk.
template <int N>
__device__ __forceinline__ void pass_empty(const ScanArgs& a, const float* from, float* to, int place, int places, int c)
{
    for (int s = place; s < a.S; s += places)
        if (a.cu[s + 1] <= a.cu[s]) write<N>(to + (size_t)s * a.C + c, read_or_zero<N>(from, (size_t)s * a.C + c));
}

// Where a CTA stands: its walk, its channels, and the rows that there are.
template <typename V, bool FLAT, bool SPLIT> struct Stand {
    int rank, s, c0, c, warp, limit, first, last;   // units first .. last-1 of the walk are this CTA's
    bool inside, whole;                             // this lane's channels are there; all of the block's are
    size_t row0;                                    // the walk's first row
    __device__ __forceinline__ Stand(const ScanArgs& a)
    {
        rank = SPLIT ? (int)cluster_rank() : 0;
        const int nblk = (a.C + V::CB - 1) / V::CB, walk = SPLIT ? blockIdx.x / a.span : blockIdx.x;
        s = walk / nblk;
        c0 = (walk % nblk) * V::CB;
        c = c0 + (threadIdx.x & 31) * V::VEC;
        warp = threadIdx.x >> 5;
        inside = c < a.C;
        whole = c0 + V::CB <= a.C;
        limit = FLAT && a.cu ? min(max(a.cu[a.S], 0), a.rows) : a.rows;
        row0 = FLAT ? 0 : (size_t)s * a.rows;
        const int per = SPLIT ? (a.units + a.span - 1) / a.span : a.units;
        first = min(rank * per, a.units);
        last = min(first + per, a.units);
    }
    __device__ __forceinline__ int live(int t) const { return min(max(limit - t, 0), UNIT); }
};

// The map (g, b) of a stretch on the state in front of it; one in which a sequence begins (g = -inf) takes nothing from it.  Gates
// that add up to -inf are another thing, a factor of zero: a state that is not finite stays so behind it.
template <int N> __device__ __forceinline__ F<N> apply(const F<N>& g, const F<N>& b, const F<N>& h)
{
    const F<N> y = Decay<N>::of(g).step(h, b);
    F<N> r;
#pragma unroll
    for (int k = 0; k < N; ++k) r.x[k] = g.x[k] == -INFINITY ? b.x[k] : y.x[k];
    return r;
}
template <int N> __device__ __forceinline__ F<N> gate_sum(bool begins, const F<N>& sum)
{
    F<N> r;
#pragma unroll
    for (int k = 0; k < N; ++k) r.x[k] = begins ? -INFINITY : sum.x[k] == -INFINITY ? -FLT_MAX : sum.x[k];
    return r;
}

// A split walk's first pass over the rows of this warp, units lo .. hi-1: what they do to the state in front of them, as (sum of
// gates, b), and from the other CTAs' and warps' the state in front of this warp's.  REVERSE: for e = a (y + e), from the end.
template <typename V, bool COMP, bool FLAT, bool REVERSE, typename S>
__device__ __forceinline__ F<V::VEC> state_in_front(const ScanArgs& a, const S& at, Hand<V>& hand, F<V::VEC> h, const float* gate,
                                                    const typename V::T* x, char* part, int bytes, int lo, int hi)
{
    using FetchG = Fetch<float, V>;
    using FetchX = Fetch<typename V::T, V>;
    constexpr int N = V::VEC;
    const int l = (threadIdx.x & 31) * N;
    auto unit = [&](int i) { return REVERSE ? hi - 1 - i : lo + i; };
    auto ask = [&](int i, int place) {
        if (i < hi - lo) {
            const int t = unit(i) * UNIT, live = at.live(t);
            const size_t row = live ? (size_t)t * a.C : 0;
            FetchG::ask(part + place * bytes, gate + row, a.C, live, a.C - at.c0);
            FetchX::ask(part + place * bytes + FetchG::BYTES, x + row, a.C, live, a.C - at.c0);
        }
        copies_end();
    };
    F<N> mg = all<N>(0.f), mb = mg;
    bool begins = false;   // a sequence, among these rows (REVERSE: ends)
    Marks marks;
    if (V::STAGED)
        for (int i = 0; i < V::DEPTH; ++i) ask(i, i);
    int place = 0;
    for (int i = 0; i < hi - lo; ++i) {
        const int t = unit(i) * UNIT, live = at.live(t);
        const size_t row = live ? (size_t)t * a.C : 0;
        if (FLAT) marks.find(a, t, UNIT, at.limit);
        FetchG fg;
        FetchX fx;
        if (V::STAGED) {
            copies_wait<V::DEPTH - 1>();
            __syncwarp();
        }
        fg.take(part + place * bytes, gate + row, a.C, live, at.c - at.c0, at.inside);
        fx.take(part + place * bytes + FetchG::BYTES, x + row, a.C, live, at.c - at.c0, at.inside);
        __syncwarp();
        if (V::STAGED) ask(i + V::DEPTH, place);
        place = place + 1 < V::DEPTH ? place + 1 : 0;
        if (!FLAT || !(REVERSE ? marks.last : marks.first)) {
            Decay<N> d[UNIT];
            F<N> b[UNIT];
#pragma unroll
            for (int j = 0; j < UNIT; j += SIDE) {
                F<N> g[SIDE];
#pragma unroll
                for (int i = 0; i < SIDE; ++i) g[i] = fg.r[j + i].get();
                mg = add(mg, add(add(g[0], g[1]), add(g[2], g[3])));   // equal gates lose the same way at every addition to a long sum
                static_assert(SIDE == 4, "rows of one addition");
                Decay<N>::template of<SIDE>(g, d + j);
#pragma unroll
                for (int i = j; i < j + SIDE; ++i) b[i] = COMP && !REVERSE ? mul(d[i].complement(), fx.r[i].get()) : fx.r[i].get();
            }
#pragma unroll
            for (int k = 0; k < UNIT; ++k) {
                const int j = REVERSE ? UNIT - 1 - k : k;
                mb = REVERSE ? d[j].times(add(b[j], mb)) : d[j].step(mb, b[j]);
            }
        } else {
            int q = marks.s;
            if (REVERSE)
                for (int k = 1; k < UNIT; ++k)
                    if (marks.first >> k & 1) q = Marks::next(a, q, t + k);
#pragma unroll
            for (int k = 0; k < UNIT; ++k) {
                const int j = REVERSE ? UNIT - 1 - k : k;
                const F<N> y = fx.r[j].get();
                const Decay<N> d = Decay<N>::of(fg.r[j].get());
                if ((REVERSE ? marks.last : marks.first) >> j & 1) {
                    if (!REVERSE && j) q = Marks::next(a, q, t + j);
                    mb = at.inside ? read_or_zero<N>(REVERSE ? a.dfin : a.init, (size_t)q * a.C + at.c) : all<N>(0.f);
                }
                mb = REVERSE ? d.times(add(y, mb)) : d.step(mb, COMP ? mul(d.complement(), y) : y);
                if (REVERSE && j && (marks.first >> j & 1)) q = previous(a, q);
            }
            begins = true;
        }
    }
    write<N>(&hand.g[at.warp][l], gate_sum<N>(begins, mg));
    write<N>(&hand.b[at.warp][l], mb);
    __syncthreads();
    if (at.warp == 0) {
        F<N> g = all<N>(0.f), b = g;
        begins = false;
#pragma unroll
        for (int k = 0; k < V::WARPS; ++k) {
            const int w = REVERSE ? V::WARPS - 1 - k : k;
            const F<N> wg = read<N>(&hand.g[w][l]);
            b = apply<N>(wg, read<N>(&hand.b[w][l]), b);
            g = add(g, wg);
            begins |= wg.x[0] == -INFINITY;   // of all channels alike
        }
        write<N>(&hand.all_g[l], gate_sum<N>(begins, g));
        write<N>(&hand.all_b[l], b);
    }
    cluster_arrive();
    cluster_wait();
    for (int r = REVERSE ? a.span - 1 : 0; r != at.rank; r += REVERSE ? -1 : 1)
        h = apply<N>(read_remote<N>(&hand.all_g[l], r), read_remote<N>(&hand.all_b[l], r), h);
    for (int w = REVERSE ? V::WARPS - 1 : 0; w != at.warp; w += REVERSE ? -1 : 1)
        h = apply<N>(read<N>(&hand.g[w][l]), read<N>(&hand.b[w][l]), h);
    cluster_arrive();   // nobody leaves, or writes there again, before all have read: waited for at the end
    return h;
}

// One walk = one dense sequence, or a whole flat batch with resets where sequences begin, over CB channels.  A CTA's warps take
// units of UNIT rows in turn: a warp maps its rows to (sum of gates, b), waits for the state in front of them, hands the
// state behind them on to the next warp before it does anything else, and walks the rows a second time from registers.  So
// the only thing done one after another is a step of two fmas a unit, from warp to warp by named barriers.  With barriers of
// all warps instead, tile by tile, the warps waited more than they worked (8 x 2048 tokens, 1024 channels, bf16: 38 to 51 us;
// so 27.3, 4.9 TB/s of what has to be read and written, and the backward 41.3, 5.7 TB/s).  28 instructions an element, of which
// the factor takes nine; bound by their issue and latency in bf16, by memory in fp32 (34.2 us, 5.9 TB/s; backward 57.8, 5.8).
// Few walks are split among the warps of a cluster's CTAs, a stretch of rows to each, read once more for the state in front of
// it: then nothing is waited for but rows (131072 tokens, 1024 channels: 414 us, 39 % of the bytes' rate; by the relay 490).
// Rows that are all there and begin and end no sequence take the code without tests.
// out == nullptr: only the states are kept.
template <typename V, bool COMP, bool FLAT, bool SPLIT>
__global__ void __launch_bounds__(32 * V::WARPS, 16 / V::WARPS) scan_fwd_kernel(ScanArgs a)
{
    using T = typename V::T;
    using FetchG = Fetch<float, V>;
    using FetchX = Fetch<T, V>;
    constexpr int N = V::VEC, PART = FetchG::BYTES + FetchX::BYTES;
    extern __shared__ __align__(16) char shared[];
    pdl_wait();
    const Stand<V, FLAT, SPLIT> at(a);
    Hand<V>& hand = *reinterpret_cast<Hand<V>*>(shared);
    char* const part = shared + sizeof(Hand<V>) + at.warp * V::DEPTH * PART;
    const int c = at.c, l = (threadIdx.x & 31) * N;
    const T* x = static_cast<const T*>(a.x) + at.row0 * a.C + at.c0;
    const float* gate = a.gate + at.row0 * a.C + at.c0;
    T* out = static_cast<T*>(a.out) + at.row0 * a.C + c;
    float* saved = a.saved ? a.saved + (FLAT ? 0 : (size_t)at.s * a.units * a.C) + c : nullptr;
    if (FLAT && a.cu && a.fin && at.inside) pass_empty<N>(a, a.init, a.fin, at.rank * V::WARPS + at.warp, a.span * V::WARPS, c);
    F<N> h = all<N>(0.f);
    if (!FLAT && at.inside) h = read_or_zero<N>(a.init, (size_t)at.s * a.C + c);
    // this warp's units: in turn with the others', or a stretch of its own whose state in front is known
    const int per = (at.last - at.first + V::WARPS - 1) / V::WARPS, pitch = SPLIT ? 1 : V::WARPS;
    const int lo = SPLIT ? min(at.first + at.warp * per, at.last) : at.first + at.warp, hi = SPLIT ? min(lo + per, at.last) : at.last;
    if (SPLIT) h = state_in_front<V, COMP, FLAT, false>(a, at, hand, h, gate, x, part, PART, lo, hi);
    auto ask = [&](int u, int place) {
        if (u < hi) {
            const int t = u * UNIT, live = at.live(t);
            const size_t row = live ? (size_t)t * a.C : 0;
            FetchG::ask(part + place * PART, gate + row, a.C, live, a.C - at.c0);
            FetchX::ask(part + place * PART + FetchG::BYTES, x + row, a.C, live, a.C - at.c0);
        }
        copies_end();
    };
    Marks marks;
    int u = lo, place = 0;
    if (V::STAGED)
        for (int i = 0; i < V::DEPTH; ++i) ask(u + i * pitch, i);
    for (; u < hi; u += pitch) {
        const int t = u * UNIT, live = at.live(t);
        const size_t row = (size_t)t * a.C;
        if (FLAT) marks.find(a, t, UNIT, at.limit);
        const bool plain = live == UNIT && at.whole && !(FLAT && (marks.first | marks.last));
        FetchG fg;
        FetchX fx;
        if (V::STAGED) {
            copies_wait<V::DEPTH - 1>();
            __syncwarp();
        }
        fg.take(part + place * PART, gate + row, a.C, live, c - at.c0, at.inside);
        fx.take(part + place * PART + FetchG::BYTES, x + row, a.C, live, c - at.c0, at.inside);
        __syncwarp();
        if (V::STAGED) ask(u + V::DEPTH * pitch, place);
        place = place + 1 < V::DEPTH ? place + 1 : 0;
        Decay<N> d[UNIT];
        F<N> b[UNIT];
        F<N> mg = all<N>(0.f), mb = mg;
#pragma unroll
        for (int j = 0; j < UNIT; j += SIDE) {
            F<N> g[SIDE];
#pragma unroll
            for (int i = 0; i < SIDE; ++i) {
                g[i] = fg.r[j + i].get();
                mg = add(mg, g[i]);
            }
            Decay<N>::template of<SIDE>(g, d + j);
#pragma unroll
            for (int i = j; i < j + SIDE; ++i) b[i] = COMP ? mul(d[i].complement(), fx.r[i].get()) : fx.r[i].get();
#pragma unroll
            for (int i = j; i < j + SIDE; ++i)
                if (!SPLIT) mb = d[i].step(mb, b[i]);
        }
        if (!SPLIT && FLAT && marks.first) {
            int q = marks.s;
#pragma unroll
            for (int i = 0; i < UNIT; ++i) {
                if (marks.first >> i & 1) {
                    if (i) q = Marks::next(a, q, t + i);
                    mb = at.inside ? read_or_zero<N>(a.init, (size_t)q * a.C + c) : all<N>(0.f);
                }
                mb = d[i].step(mb, b[i]);
            }
            mg = all<N>(-INFINITY);
        }
        pin<N>(d, b);
        if constexpr (!SPLIT) {
            const Decay<N> md = Decay<N>::of(mg);
            F<N> behind;
            const int next = at.warp + 1 < V::WARPS ? at.warp + 1 : 0;
            const bool begins = FLAT && marks.first;   // nothing of the state in front reaches the rows behind, not even a NaN
            if (u > at.first && u + 1 < at.last && !begins) {
                h = relay<N>(at.warp, next, &hand.state[at.warp][l], &hand.state[next][l], md, mb, behind);
            } else {
                if (u > at.first) {
                    take_over(at.warp);
                    h = read<N>(&hand.state[at.warp][l]);
                }
                behind = begins ? mb : md.step(h, mb);
                if (u + 1 < at.last) {
                    write<N>(&hand.state[next][l], behind);
                    hand_on(next);
                }
            }
            if (!FLAT && a.fin && u + 1 == a.units && at.inside) write<N>(a.fin + (size_t)at.s * a.C + c, behind);
        }
        if (plain) {
            if (saved) write<N>(saved + (size_t)u * a.C, h);
#pragma unroll
            for (int i = 0; i < UNIT; ++i) {
                h = d[i].step(h, b[i]);
                if (a.out) write<N>(out + row + (size_t)i * a.C, h);
            }
        } else if (at.inside) {
            if (saved) write<N>(saved + (size_t)u * a.C, h);
            int q = marks.s;
#pragma unroll
            for (int i = 0; i < UNIT; ++i) {
                if (i >= live) break;
                if (FLAT && (marks.first >> i & 1)) {
                    if (i) q = Marks::next(a, q, t + i);
                    h = read_or_zero<N>(a.init, (size_t)q * a.C + c);
                }
                h = d[i].step(h, b[i]);
                if (a.out) write<N>(out + row + (size_t)i * a.C, h);
                if (FLAT && a.fin && (marks.last >> i & 1)) write<N>(a.fin + (size_t)q * a.C + c, h);
            }
        }
        if (SPLIT && !FLAT && a.fin && u + 1 == a.units && at.inside) write<N>(a.fin + (size_t)at.s * a.C + c, h);
    }
    if (SPLIT) cluster_wait();
}

// The same walk from the end: e = a (dout + e), the state's gradient as the row before sees it.  Each unit walks its states
// forward again from the one that the forward kept, so that the gates' gradients take fp32 states:
//   dgate_t = (h_{t-1} [- x_t]) e_t,   dx_t = dh_t or (1 - a_t) dh_t,   dh_t = dout_t + e_{t+1}.
template <typename V, bool COMP, bool FLAT, bool SPLIT>
__global__ void __launch_bounds__(32 * V::WARPS, 16 / V::WARPS) scan_bwd_kernel(ScanArgs a)
{
    using T = typename V::T;
    using FetchG = Fetch<float, V>;
    using FetchX = Fetch<T, V>;
    constexpr int N = V::VEC, PART = FetchG::BYTES + 2 * FetchX::BYTES;
    extern __shared__ __align__(16) char shared[];
    pdl_wait();
    const Stand<V, FLAT, SPLIT> at(a);
    Hand<V>& hand = *reinterpret_cast<Hand<V>*>(shared);
    char* const part = shared + sizeof(Hand<V>) + at.warp * V::DEPTH * PART;
    const int c = at.c, l = (threadIdx.x & 31) * N;
    const T* x = static_cast<const T*>(a.x) + at.row0 * a.C + at.c0;
    const T* dout = static_cast<const T*>(a.dout) + at.row0 * a.C + at.c0;
    const float* gate = a.gate + at.row0 * a.C + at.c0;
    T* dx = static_cast<T*>(a.dx) + at.row0 * a.C + c;
    float* dgate = a.dgate + at.row0 * a.C + c;
    const float* saved = a.saved + (FLAT ? 0 : (size_t)at.s * a.units * a.C) + c;
    if (FLAT && a.cu && a.dinit && at.inside) pass_empty<N>(a, a.dfin, a.dinit, at.rank * V::WARPS + at.warp, a.span * V::WARPS, c);
    F<N> e = all<N>(0.f);
    if (!FLAT && at.inside) e = read_or_zero<N>(a.dfin, (size_t)at.s * a.C + c);
    const int per = (at.last - at.first + V::WARPS - 1) / V::WARPS, pitch = SPLIT ? 1 : V::WARPS;
    const int lo = SPLIT ? min(at.first + at.warp * per, at.last) : at.first;
    const int hi = SPLIT ? min(lo + per, at.last) : at.last - at.warp;
    if (SPLIT) e = state_in_front<V, COMP, FLAT, true>(a, at, hand, e, gate, dout, part, PART, lo, hi);
    auto ask = [&](int u, int place) {
        if (u >= lo) {
            const int t = u * UNIT, live = at.live(t);
            const size_t row = live ? (size_t)t * a.C : 0;
            char* const to = part + place * PART;
            FetchG::ask(to, gate + row, a.C, live, a.C - at.c0);
            FetchX::ask(to + FetchG::BYTES, x + row, a.C, live, a.C - at.c0);
            FetchX::ask(to + FetchG::BYTES + FetchX::BYTES, dout + row, a.C, live, a.C - at.c0);
        }
        copies_end();
    };
    Marks marks;
    int u = hi - 1, place = 0;
    if (V::STAGED)
        for (int i = 0; i < V::DEPTH; ++i) ask(u - i * pitch, i);
    for (; u >= lo; u -= pitch) {
        const int t = u * UNIT, live = at.live(t);
        const size_t row = (size_t)t * a.C;
        if (FLAT) marks.find(a, t, UNIT, at.limit);
        const bool plain = live == UNIT && at.whole && !(FLAT && (marks.first | marks.last));
        F<N> h = all<N>(0.f);
        if (at.inside) h = read<N>(saved + (size_t)u * a.C);
        FetchG fg;
        FetchX fx, fy;
        if (V::STAGED) {
            copies_wait<V::DEPTH - 1>();
            __syncwarp();
        }
        const char* const from = part + place * PART;
        fg.take(from, gate + row, a.C, live, c - at.c0, at.inside);
        fx.take(from + FetchG::BYTES, x + row, a.C, live, c - at.c0, at.inside);
        fy.take(from + FetchG::BYTES + FetchX::BYTES, dout + row, a.C, live, c - at.c0, at.inside);
        __syncwarp();
        if (V::STAGED) ask(u - V::DEPTH * pitch, place);
        place = place + 1 < V::DEPTH ? place + 1 : 0;
        Decay<N> d[UNIT];
        F<N> before[UNIT];
        F<N> mg = all<N>(0.f), mb = mg;
#pragma unroll
        for (int j = 0; j < UNIT; j += SIDE) {
            F<N> g[SIDE];
#pragma unroll
            for (int i = 0; i < SIDE; ++i) {
                g[i] = fg.r[j + i].get();
                mg = add(mg, g[i]);
            }
            Decay<N>::template of<SIDE>(g, d + j);
        }
        int qlast = 0;   // against time: the sequence of the last row first
        if (!FLAT || !(marks.first | marks.last)) {
#pragma unroll
            for (int i = 0; i < UNIT; ++i) {
                const F<N> y = fx.r[i].get();
                before[i] = h;
                h = d[i].step(h, COMP ? mul(d[i].complement(), y) : y);
            }
#pragma unroll
            for (int i = UNIT - 1; i >= 0; --i)
                if (!SPLIT) mb = d[i].times(add(fy.r[i].get(), mb));
        } else {
            int q = marks.s;
#pragma unroll
            for (int i = 0; i < UNIT; ++i) {
                if (marks.first >> i & 1) {
                    if (i) q = Marks::next(a, q, t + i);
                    h = at.inside ? read_or_zero<N>(a.init, (size_t)q * a.C + c) : all<N>(0.f);
                }
                const F<N> y = fx.r[i].get();
                before[i] = h;
                h = d[i].step(h, COMP ? mul(d[i].complement(), y) : y);
            }
            qlast = q;
#pragma unroll
            for (int i = UNIT - 1; i >= 0; --i) {
                if (marks.last >> i & 1) {
                    mb = at.inside ? read_or_zero<N>(a.dfin, (size_t)q * a.C + c) : all<N>(0.f);
                    mg = all<N>(-INFINITY);
                }
                mb = d[i].times(add(fy.r[i].get(), mb));
                if (i && (marks.first >> i & 1)) q = previous(a, q);
            }
        }
        pin<N>(d, before);
        if constexpr (!SPLIT) {
            const Decay<N> md = Decay<N>::of(mg);
            F<N> behind;
            const int next = at.warp + 1 < V::WARPS ? at.warp + 1 : 0;
            const bool ends = FLAT && marks.last;
            if (u > at.first && u + 1 < at.last && !ends) {
                e = relay<N>(at.warp, next, &hand.state[at.warp][l], &hand.state[next][l], md, mb, behind);
            } else {
                if (u + 1 < at.last) {
                    take_over(at.warp);
                    e = read<N>(&hand.state[at.warp][l]);
                }
                behind = ends ? mb : md.step(e, mb);
                if (u > at.first) {
                    write<N>(&hand.state[next][l], behind);
                    hand_on(next);
                }
            }
            if (!FLAT && a.dinit && u == 0 && at.inside) write<N>(a.dinit + (size_t)at.s * a.C + c, behind);
        }
        if (plain) {
#pragma unroll
            for (int i = UNIT - 1; i >= 0; --i) {
                const F<N> dh = add(fy.r[i].get(), e);
                e = d[i].times(dh);
                write<N>(dx + row + (size_t)i * a.C, COMP ? mul(d[i].complement(), dh) : dh);
                write<N>(dgate + row + (size_t)i * a.C, mul(COMP ? fma(fx.r[i].get(), all<N>(-1.f), before[i]) : before[i], e));
            }
        } else if (at.inside) {
            int q = qlast;
#pragma unroll
            for (int i = UNIT - 1; i >= 0; --i) {
                if (i >= live) continue;
                if (FLAT && (marks.last >> i & 1)) e = read_or_zero<N>(a.dfin, (size_t)q * a.C + c);
                const F<N> dh = add(fy.r[i].get(), e);
                e = d[i].times(dh);
                write<N>(dx + row + (size_t)i * a.C, COMP ? mul(d[i].complement(), dh) : dh);
                write<N>(dgate + row + (size_t)i * a.C, mul(COMP ? fma(fx.r[i].get(), all<N>(-1.f), before[i]) : before[i], e));
                if (FLAT && (marks.first >> i & 1)) {
                    if (a.dinit) write<N>(a.dinit + (size_t)q * a.C + c, e);
                    if (i) q = previous(a, q);
                }
            }
        }
        if (SPLIT && !FLAT && a.dinit && u == 0 && at.inside) write<N>(a.dinit + (size_t)at.s * a.C + c, e);
    }
    if (SPLIT) cluster_wait();
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
            const Decay<1> d = Decay<1>::of({{g[j]}});
            h[j] = d.step({{h[j]}}, {{COMP ? d.complement().x[0] * y[j] : y[j]}}).x[0];
        }
        store_vec<N>(out + at, h);
    }
    store_vec<N>(state + b * C + c, h);
}

// Short sequences are walked as one flat batch.
bool is_flat(const osdn_scan_params& p) { return p.nseq > 0 || (p.B > 1 && p.T < 64); }

ScanArgs make_args(const osdn_scan_params& p)
{
    ScanArgs a{};
    a.cu = p.nseq > 0 ? p.cu_seqlens : nullptr;
    a.S = p.nseq > 0 ? p.nseq : p.B;
    a.T = p.T;
    a.C = p.C;
    a.rows = p.nseq > 0 || !is_flat(p) ? p.T : p.B * p.T;
    a.units = div_up(a.rows, UNIT);
    return a;
}

// CTAs of a walk.  One, where walks alone give four of five SMs a CTA; else the walk is split, though its CTAs then read their
// rows twice, until there are CTAs for four of five SMs, or for all of them twice over where every warp has many units.  1024
// channels (16 walks), forward / backward with 4, 8 and 16 CTAs to a walk: one prompt of 2048 tokens 14.3 / 16.3, 13.8 / 15.6 and
// 18.9 / 21.2 us (unsplit 25.1 / 29.8); 131072 tokens 503 / 579, 522 / 661 and 414 / 524 (unsplit 1438 / 1758).
int span_of(long long walks, int units, int warps)
{
    int span = 1;
    if (walks < 120)
        while (span < MAX_SPAN && units >= 2 * span * warps && walks * span < (units >= 64 * span * warps ? 240 : 120)) span *= 2;
    return span;
}

// Warps of a CTA.  Sixteen where an SM has one CTA with enough units for them, eight where it has two or the walk is short.
// 1024 channels, forward / backward with sixteen and with eight: 8 x 2048 tokens (128 walks) 27.3 / 41.1 and 28.4 / 46.9 us; 9 x 2048
// 28.7 / 49.0 and 29.5 / 49.5; 16 x 2048 (256 walks) 53.0 / 80.2 and 47.4 / 91.1; 32 x 2048 105 / 159 and 92.7 / 168; 64 x 100 23.7 / 27.1
// and 15.5 / 22.6; one of 2048, split over eight CTAs, 19.8 / 22.8 and 13.8 / 15.6; 131072 over sixteen 416 / 529 and 417 / 567.
// From 149 walks on sixteen warps need a second wave, and eight would be the faster up to the line at 240 as well (10 x 2048 51.7 / 70.1
// and 46.1 / 63.6; 12 x 2048 52.1 / 68.4 and 46.4 / 66.0; 14 x 2048 52.7 / 82.1 and 46.7 / 76.0; in fp32 66.3 / 102 and 66.2 / 110).
struct Shape {
    int warps;
    bool split;
};
Shape shape_of(const ScanArgs& a, bool flat)
{
    const long long walks = (long long)(flat ? 1 : a.S) * div_up(a.C, 64);
    const int span = span_of(walks, a.units, 16);
    const int warps = walks < 240 && a.units / span >= (span > 1 ? 256 : 64) ? 16 : 8;
    return {warps, span_of(walks, a.units, warps) > 1};
}

// Kernel(SPLIT) for the walks of a batch.
template <typename V, typename K> bool launch_walks(K kernel, ScanArgs a, bool flat, int part, cudaStream_t st)
{
    const long long walks = (long long)(flat ? 1 : a.S) * div_up(a.C, V::CB);
    a.span = span_of(walks, a.units, V::WARPS);
    const bool split = a.span > 1;
    const size_t smem = sizeof(Hand<V>) + (V::STAGED ? (size_t)V::WARPS * V::DEPTH * part : 0);
    void (*f)(ScanArgs) = split ? kernel(std::true_type{}) : kernel(std::false_type{});
    if (cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return false;
    if (a.span > 8 && cudaFuncSetAttribute(f, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return false;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(walks * a.span));
    cfg.blockDim = dim3(32 * V::WARPS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.span;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, f, a) == cudaSuccess;
}

template <typename T> bool is_wide(int C) { return C % (16 / (int)sizeof(T)) == 0; }   // rows in pieces of 16 bytes

template <typename T, bool COMP> bool launch_forward(const ScanArgs& a, bool flat, cudaStream_t st)
{
    auto go = [&](auto cover) {
        using V = decltype(cover);
        auto kernel = [&](auto split) {
            constexpr bool SPLIT = decltype(split)::value;
            return flat ? scan_fwd_kernel<V, COMP, true, SPLIT> : scan_fwd_kernel<V, COMP, false, SPLIT>;
        };
        return launch_walks<V>(kernel, a, flat, Fetch<float, V>::BYTES + Fetch<T, V>::BYTES, st);
    };
    if (!is_wide<T>(a.C)) return go(Cover<T, 1, 8, 1>{});
    const Shape f = shape_of(a, flat);   // a split walk's warps wait for nothing but their rows: more of them on their way
    if (f.warps == 16) return f.split ? go(Cover<T, 2, 16, 3>{}) : go(Cover<T, 2, 16, 1>{});
    return f.split ? go(Cover<T, 2, 8, 3>{}) : go(Cover<T, 2, 8, 2>{});
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
        auto kernel = [&](auto split) {
            constexpr bool SPLIT = decltype(split)::value;
            return flat ? scan_bwd_kernel<V, COMP, true, SPLIT> : scan_bwd_kernel<V, COMP, false, SPLIT>;
        };
        return launch_walks<V>(kernel, a, flat, Fetch<float, V>::BYTES + 2 * Fetch<T, V>::BYTES, st);
    };
    constexpr int MORE = sizeof(T) == 2 ? 3 : 2;
    const Shape f = shape_of(a, flat);
    const bool ok = !is_wide<T>(a.C)  ? go(Cover<T, 1, 8, 1>{})
                    : f.warps == 16  ? (f.split ? go(Cover<T, 2, 16, MORE>{}) : go(Cover<T, 2, 16, 2>{}))
                    : f.split        ? go(Cover<T, 2, 8, MORE>{})
                                     : go(Cover<T, 2, 8, 2>{});
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
    return align_up((size_t)(is_flat(p) ? 1 : p.B) * a.units * p.C * 4, 256);
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
