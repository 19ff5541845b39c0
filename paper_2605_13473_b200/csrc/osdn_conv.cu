// Short causal depthwise convolution over the tokens of a sequence: forward, backward, decode step.
#include "osdn_rows.cuh"

namespace osdn {
namespace {

struct ConvArgs {
    const void *x, *init, *dout, *dfin;
    const float *w, *bias;
    void *out, *fin, *dx, *dinit;
    float* partial;   // [gridDim.y, W + 1, C] sums of dweight and dbias
    Rows rows;
    int C, chunk, chunks;   // tokens a thread walks at a time; such chunks of a dense sequence, or of all packed rows
    long long walks;        // chunks of the whole batch
};

// z sigmoid(z) needs 1 / (1 + exp(-z)).  Where results are rounded to bf16 (2^-8 of the value) the hardware's exponential and
// reciprocal (about 2^-21, and 1.25 |z| 2^-24 by the argument) are exact enough; the weights' fp32 sums take them too.
template <typename T, int L> __device__ __forceinline__ F<L> sigmoid(const F<L>& z)
{
    F<L> s;
    if constexpr (sizeof(T) == 2) {
        const F<L> e = mul(z, all<L>(-1.44269504f));
#pragma unroll
        for (int k = 0; k < L; ++k) {
            float x;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(e.x[k]));
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s.x[k]) : "f"(1.f + x));
        }
    } else {
#pragma unroll
        for (int k = 0; k < L; ++k) s.x[k] = 1.f / (1.f + expf(-z.x[k]));
    }
    return s;
}

// Where a walk over the rows of one chunk stands: its sequence and the sequence's first row and end.
struct Place {
    int s, start, end;   // rows of the walk's own tensor part (a dense sequence: 0 .. T)
    __device__ __forceinline__ void enter(const Rows& r, int t, int limit)
    {
        if (!r.cu) return;
        s = seq_of(r, t);
        start = min(max(r.cu[s], 0), t);
        end = min(max(r.cu[s + 1], t + 1), limit);
    }
};

// x row t of the sequence, or the state's row where t lies in front of it.
template <typename T, int N, int W>
__device__ __forceinline__ Channels<T, N> row_before(const ConvArgs& a, const T* x, const Place& at, int t, int c)
{
    if (t >= at.start) return Channels<T, N>::load(x + (size_t)t * a.C + c);
    if (!a.init) return Channels<T, N>::zero();
    return Channels<T, N>::load(static_cast<const T*>(a.init) + ((size_t)at.s * (W - 1) + (W - 1) + (t - at.start)) * a.C + c);
}

// The taps of N channels, in pairs: one after the other in memory, read in 16-byte pieces.
template <int N, int W> struct Taps {
    static constexpr int L = N % 2 == 0 ? 2 : 1, Q = N / L;
    F<L> w[W][Q], b[Q];
    __device__ __forceinline__ void load(const float* weight, const float* bias, int c)
    {
        float f[N * W], g[N];
        load_vec<N * W>(weight + (size_t)c * W, f);
        if (bias) {
            load_vec<N>(bias + c, g);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) g[j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i][j / L].x[j % L] = f[j * W + i];
            b[j / L].x[j % L] = g[j];
        }
    }
};

// A state of an empty sequence (or its gradient) passes through.
template <typename T, int N, int W>
__device__ __forceinline__ void pass_empty(const ConvArgs& a, const void* from, void* to, long long walk, int c)
{
    if (!a.rows.cu || !to) return;
    for (long long s = walk; s < a.rows.S; s += a.walks) {
        if (a.rows.cu[s + 1] > a.rows.cu[s]) continue;
        for (int i = 0; i < W - 1; ++i) {
            const size_t at = ((size_t)s * (W - 1) + i) * a.C + c;
            (from ? Channels<T, N>::load(static_cast<const T*>(from) + at) : Channels<T, N>::zero()).store(static_cast<T*>(to) + at);
        }
    }
}

// One output row from the window of the rows before it (oldest first) and its own; the window moves on.
template <typename T, int N, int W, bool SILU>
__device__ __forceinline__ Channels<T, N> convolve(const Taps<N, W>& k, F<Taps<N, W>::L> (&prev)[W - 1][Taps<N, W>::Q], const Channels<T, N>& row)
{
    Channels<T, N> y;
#pragma unroll
    for (int q = 0; q < Taps<N, W>::Q; ++q) {
        const auto v = row.get(q);
        auto z = k.b[q];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) z = fma(k.w[j][q], prev[j][q], z);
        z = fma(k.w[W - 1][q], v, z);
        y.set(q, SILU ? mul(z, sigmoid<T>(z)) : z);
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) prev[j][q] = prev[j + 1][q];
        prev[W - 2][q] = v;
    }
    return y;
}

// A warp's rows of one tensor, U at a time.  Staged: 16-byte copies to the warp's part of shared memory, DEPTH stretches on
// their way; else (rows that are not whole 16-byte pieces) read where they are.
template <typename T, int N, bool STAGED> struct Stream {
    static constexpr int U = 8, DEPTH = STAGED ? 2 : 1, ROW = 32 * N * (int)sizeof(T), BYTES = U * ROW;
    __device__ __forceinline__ static void ask(char* part, const T* p, size_t pitch, int live, int cols)
    {
        if constexpr (STAGED) {
            constexpr int PIECES = ROW / 16, ROWS = PIECES < 32 ? 32 / PIECES : 1, STEPS = PIECES > 32 ? PIECES / 32 : 1, PER = 16 / (int)sizeof(T);
            const int lane = threadIdx.x & 31, row = lane / PIECES;
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const int piece = lane % PIECES + j * 32, col = piece * PER;
#pragma unroll
                for (int i = 0; i < U; i += ROWS) {
                    const bool real = col < cols && i + row < live;
                    copy_async16(part + (i + row) * ROW + piece * 16, real ? p + (i + row) * pitch + col : p, real);
                }
            }
        }
    }
    __device__ __forceinline__ static Channels<T, N> get(const char* part, const T* p, size_t pitch, int i)   // p: the lane's channels
    {
        if constexpr (STAGED) return Channels<T, N>::load(reinterpret_cast<const T*>(part + i * ROW) + (threadIdx.x & 31) * N);
        else return Channels<T, N>::load(p + i * pitch);
    }
};

// CTAs of four warps to an SM, by the registers that N channels of a lane take.
template <int N> constexpr int FWD_CTAS = N == 4 ? 6 : 8;
template <int N> constexpr int BWD_CTAS = N == 4 ? 4 : 6;

// A warp walks the rows of a chunk over 32 N channels.
template <typename T, int N, int W, bool SILU, bool STAGED>
__global__ void __launch_bounds__(128, FWD_CTAS<N>) conv_fwd_kernel(ConvArgs a)
{
    using Row = Channels<T, N>;
    using In = Stream<T, N, STAGED>;
    constexpr int Q = Row::Q, U = In::U, DEPTH = In::DEPTH;
    extern __shared__ __align__(16) char shared[];
    pdl_wait();
    const int blocks = (a.C + 32 * N - 1) / (32 * N), lane = threadIdx.x & 31;
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (i >= a.walks * blocks) return;
    char* const part = shared + (threadIdx.x >> 5) * DEPTH * In::BYTES;
    const int c0 = (int)(i % blocks) * 32 * N, c = c0 + lane * N;
    const bool inside = c < a.C;
    const long long walk = i / blocks;
    if (inside) pass_empty<T, N, W>(a, a.init, a.fin, walk, c);
    Place at{(int)(walk / a.chunks), 0, a.rows.T};
    const int limit = a.rows.cu ? rows_end(a.rows) : a.rows.T;
    const int t0 = (int)(walk % a.chunks) * a.chunk, t1 = min(t0 + a.chunk, limit);
    if (t0 >= t1) return;
    const size_t base = a.rows.cu ? 0 : (size_t)at.s * a.rows.T * a.C;
    const T* x = static_cast<const T*>(a.x) + base;
    T* out = static_cast<T*>(a.out) + base;
    auto ask = [&](int t, int place) {
        if (t < t1) In::ask(part + place * In::BYTES, x + (size_t)t * a.C + c0, a.C, t1 - t, a.C - c0);
        copies_end();
    };
    if (STAGED)
        for (int d = 0; d < DEPTH; ++d) ask(t0 + d * U, d);
    at.enter(a.rows, t0, limit);
    Taps<N, W> k;
    F<Row::L> prev[W - 1][Q];
    auto refill = [&](int t) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const Row r = row_before<T, N, W>(a, x, at, t - (W - 1) + j, c);
#pragma unroll
            for (int q = 0; q < Q; ++q) prev[j][q] = r.get(q);
        }
    };
    if (inside) {
        k.load(a.w, a.bias, c);
        refill(t0);
    }
    int place = 0;
    for (int t = t0; t < t1; t += U) {
        if (STAGED) {
            copies_wait<DEPTH - 1>();
            __syncwarp();
        }
        const char* const from = part + place * In::BYTES;
        const T* const rows = x + (size_t)t * a.C + c;
        if (!inside) {
        } else if (t + U <= t1 && t + U < at.end) {
#pragma unroll
            for (int u = 0; u < U; ++u) convolve<T, N, W, SILU>(k, prev, In::get(from, rows, a.C, u)).store(out + (size_t)(t + u) * a.C + c);
        } else {
            for (int u = 0; u < U && t + u < t1; ++u) {
                if (t + u >= at.end) {   // the next sequence that is not empty
                    at.enter(a.rows, t + u, limit);
                    refill(t + u);
                }
                convolve<T, N, W, SILU>(k, prev, In::get(from, rows, a.C, u)).store(out + (size_t)(t + u) * a.C + c);
                if (a.fin && t + u + 1 == at.end)
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) {
                        Row r;
#pragma unroll
                        for (int q = 0; q < Q; ++q) r.set(q, prev[j][q]);
                        r.store(static_cast<T*>(a.fin) + ((size_t)at.s * (W - 1) + j) * a.C + c);
                    }
            }
        }
        __syncwarp();
        if (STAGED) ask(t + DEPTH * U, place);
        place = place + 1 < DEPTH ? place + 1 : 0;
    }
}

// A warp walks the rows of its chunk and, for the gradients of the chunk's last rows, up to W-1 behind it.  acc[j] is the
// gradient, so far, of row t - (W-1) + j; it is complete once dz_t is in, or at the sequence's end, where all W-1 last rows
// take the gradient of the state as well.  Rows in front of a sequence are its state's.
template <typename T, int N, int W, bool SILU, bool STAGED>
__global__ void __launch_bounds__(128, BWD_CTAS<N>) conv_bwd_kernel(ConvArgs a)
{
    using Row = Channels<T, N>;
    using In = Stream<T, N, STAGED>;
    constexpr int Q = Row::Q, L = Row::L, U = In::U, DEPTH = In::DEPTH, WIDTH = 32 * N;
    extern __shared__ __align__(16) char shared[];
    __shared__ float sums[4][W + 1][WIDTH];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = blockIdx.x * WIDTH, c = c0 + lane * N;
    const bool inside = c < a.C;
    char* const part = shared + warp * DEPTH * 2 * In::BYTES;
    F<L> dw[W][Q], db[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][q] = all<L>(0.f);
        db[q] = all<L>(0.f);
    }
    Taps<N, W> k;
    if (inside) k.load(a.w, a.bias, c);
    const int limit = a.rows.cu ? rows_end(a.rows) : a.rows.T;
    for (long long walk = (long long)blockIdx.y * 4 + warp; walk < a.walks; walk += (long long)gridDim.y * 4) {
        if (inside) pass_empty<T, N, W>(a, a.dfin, a.dinit, walk, c);
        Place at{(int)(walk / a.chunks), 0, a.rows.T};
        const int t0 = (int)(walk % a.chunks) * a.chunk, t1 = min(t0 + a.chunk, limit);
        if (t0 >= t1) continue;
        const int tend = min(t1 + W - 1, limit);
        const size_t base = a.rows.cu ? 0 : (size_t)at.s * a.rows.T * a.C;
        const T* x = static_cast<const T*>(a.x) + base;
        const T* dout = static_cast<const T*>(a.dout) + base;
        T* dx = static_cast<T*>(a.dx) + base;
        auto ask = [&](int t, int place) {
            if (t < tend) {
                char* const to = part + place * 2 * In::BYTES;
                In::ask(to, x + (size_t)t * a.C + c0, a.C, tend - t, a.C - c0);
                In::ask(to + In::BYTES, dout + (size_t)t * a.C + c0, a.C, tend - t, a.C - c0);
            }
            copies_end();
        };
        if (STAGED)
            for (int d = 0; d < DEPTH; ++d) ask(t0 + d * U, d);
        at.enter(a.rows, t0, limit);
        F<L> prev[W - 1][Q], acc[W][Q];
        auto refill = [&](int t) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const Row r = row_before<T, N, W>(a, x, at, t - (W - 1) + j, c);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    prev[j][q] = r.get(q);
                    acc[j][q] = all<L>(0.f);
                }
            }
        };
        if (inside) refill(t0);
        auto put = [&](int t, const F<L> (&v)[Q]) {   // the gradient of row t is complete
            Row r;
#pragma unroll
            for (int q = 0; q < Q; ++q) r.set(q, v[q]);
            if (t >= at.start) {
                if (t >= t0 && t < t1) r.store(dx + (size_t)t * a.C + c);
            } else if (a.dinit && at.start >= t0 && at.start < t1) {
                r.store(static_cast<T*>(a.dinit) + ((size_t)at.s * (W - 1) + (W - 1) + (t - at.start)) * a.C + c);
            }
        };
        auto take = [&](const Row& xr, const Row& gr, bool own) {   // dz of one row into the sums and the window
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const F<L> v = xr.get(q);
                F<L> g = gr.get(q);
                if (SILU) {
                    F<L> z = k.b[q];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) z = fma(k.w[j][q], prev[j][q], z);
                    z = fma(k.w[W - 1][q], v, z);
                    const F<L> s = sigmoid<T>(z);
                    g = mul(g, mul(s, fma(z, fma(s, all<L>(-1.f), all<L>(1.f)), all<L>(1.f))));
                }
                if (own) {
                    db[q] = add(db[q], g);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) dw[j][q] = fma(g, prev[j][q], dw[j][q]);
                    dw[W - 1][q] = fma(g, v, dw[W - 1][q]);
                }
#pragma unroll
                for (int j = 0; j < W - 1; ++j) acc[j][q] = fma(k.w[j][q], g, acc[j][q]);
                acc[W - 1][q] = mul(k.w[W - 1][q], g);
#pragma unroll
                for (int j = 0; j + 1 < W - 1; ++j) prev[j][q] = prev[j + 1][q];
                prev[W - 2][q] = v;
            }
        };
        auto shift = [&] {
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int q = 0; q < Q; ++q) acc[j][q] = acc[j + 1][q];
        };
        bool over = false;   // the same for the whole warp
        int place = 0;
        for (int t = t0; t < tend; t += U) {
            if (STAGED) {
                copies_wait<DEPTH - 1>();
                __syncwarp();
            }
            const char* const from = part + place * 2 * In::BYTES;
            const T *const xrows = x + (size_t)t * a.C + c, *const grows = dout + (size_t)t * a.C + c;
            if (!inside || over) {
            } else if (t + U <= t1 && t + U < at.end && t - (W - 1) >= t0 && t - (W - 1) >= at.start) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    take(In::get(from, xrows, a.C, u), In::get(from + In::BYTES, grows, a.C, u), true);
                    Row r;
#pragma unroll
                    for (int q = 0; q < Q; ++q) r.set(q, acc[0][q]);
                    r.store(dx + (size_t)(t + u - (W - 1)) * a.C + c);
                    shift();
                }
            } else {
                for (int s = t; s < t + U && s < tend; ++s) {
                    if (s >= at.end) {
                        if (s >= t1) {
                            over = true;
                            break;
                        }
                        at.enter(a.rows, s, limit);
                        refill(s);
                    }
                    take(In::get(from, xrows, a.C, s - t), In::get(from + In::BYTES, grows, a.C, s - t), s < t1);
                    put(s - (W - 1), acc[0]);
                    shift();
                    if (s + 1 == at.end) {
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) {
                            if (a.dfin) {
                                const Row f = Row::load(static_cast<const T*>(a.dfin) + ((size_t)at.s * (W - 1) + j) * a.C + c);
#pragma unroll
                                for (int q = 0; q < Q; ++q) acc[j][q] = add(acc[j][q], f.get(q));
                            }
                            put(s - (W - 2) + j, acc[j]);
                        }
                    }
                }
            }
            __syncwarp();
            if (STAGED) ask(t + DEPTH * U, place);
            place = place + 1 < DEPTH ? place + 1 : 0;
        }
    }
    // the CTA's sums, warp by warp in order
#pragma unroll
    for (int m = 0; m < N; ++m) {
#pragma unroll
        for (int j = 0; j < W; ++j) sums[warp][j][lane * N + m] = dw[j][m / L].x[m % L];
        sums[warp][W][lane * N + m] = db[m / L].x[m % L];
    }
    __syncthreads();
    for (int m = threadIdx.x; m < (W + 1) * WIDTH; m += 128) {
        const int j = m / WIDTH, ch = c0 + m % WIDTH;
        float v = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) v += sums[r][j][m % WIDTH];
        if (ch < a.C) a.partial[((size_t)blockIdx.y * (W + 1) + j) * a.C + ch] = v;
    }
}

// A thread keeps the taps of N channels and takes `each` sequences one after the other.
template <typename T, int N, int W, bool SILU>
__global__ void __launch_bounds__(128) conv_step_kernel(const T* x, const float* weight, const float* bias, T* state, T* out, int B,
                                                        int len, int C, int each)
{
    pdl_wait();
    using Row = Channels<T, N>;
    constexpr int Q = Row::Q;
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const int n = C / N;
    const long long first = i / n * each;
    if (first >= B) return;
    const int c = (int)(i % n) * N;
    Taps<N, W> k;
    k.load(weight, bias, c);
    for (long long s = first; s < first + each && s < B; ++s) {
        F<Row::L> prev[W - 1][Q];
        Row r[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) r[j] = Row::load(state + (s * (W - 1) + j) * C + c);
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
#pragma unroll
            for (int q = 0; q < Q; ++q) prev[j][q] = r[j].get(q);
        for (int t = 0; t < len; ++t)
            convolve<T, N, W, SILU>(k, prev, Row::load(x + (s * len + t) * C + c)).store(out + (s * len + t) * C + c);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
#pragma unroll
            for (int q = 0; q < Q; ++q) r[j].set(q, prev[j][q]);
            r[j].store(state + (s * (W - 1) + j) * C + c);
        }
    }
}

template <typename F> int by_type(const osdn_conv_params& p, F f)   // f(element, taps, activation)
{
    auto taps = [&](auto e, auto act) {
        if (p.W == 2) return f(e, std::integral_constant<int, 2>{}, act);
        if (p.W == 3) return f(e, std::integral_constant<int, 3>{}, act);
        return f(e, std::integral_constant<int, 4>{}, act);
    };
    auto act = [&](auto e) { return p.activation == OSDN_ACT_SILU ? taps(e, std::true_type{}) : taps(e, std::false_type{}); };
    return p.io_dtype == OSDN_FP32 ? act(0.f) : act(__nv_bfloat16{});
}

// Rows of a walk (a multiple of eight): as many as let the walks of 128 rows at most fill every SM's `ctas` CTAs a whole number
// of times.  (8 x 2048 x 2048 in walks of 64 rows, 1.15 times: forward 28.9 us, in walks of 80 26.9.)
void plan_walks(ConvArgs& a, const osdn_conv_params& p, int N, int ctas)
{
    const long long blocks = div_up(p.C, 32 * N), rows = (long long)p.B * p.T * blocks, slots = 148ll * ctas;
    const int B = p.nseq > 0 ? 1 : p.B;
    const long long times = (rows + slots * 4 * 128 - 1) / (slots * 4 * 128);
    int chunk = (int)std::min(128ll, (rows / (slots * 4 * times) + 7) / 8 * 8);
    chunk = std::max(chunk, 8);
    while (chunk < 160 && (((long long)B * div_up(p.T, chunk) + 3) / 4) * blocks > slots * times) chunk += 8;
    a.chunk = chunk;
    a.chunks = div_up(p.T, chunk);
    a.walks = (long long)B * a.chunks;
}

ConvArgs make_args(const osdn_conv_params& p)
{
    ConvArgs a{};
    a.rows = {p.nseq > 0 ? p.cu_seqlens : nullptr, p.nseq > 0 ? p.nseq : p.B, p.T};
    a.C = p.C;
    return a;
}

// Channels to a lane: rows that are whole 16-byte pieces are staged.
int lane_channels(const osdn_conv_params& p)
{
    const int wide = p.io_dtype == OSDN_BF16 ? 4 : 2;   // 8 bytes
    return p.C % (2 * wide) == 0 ? wide : 1;
}

// CTAs of the backward along the rows, and every warp the same number of walks.
int backward_rows(const ConvArgs& a, int N, int ctas)
{
    const long long need = (a.walks + 3) / 4, most = std::max(1, 148 * ctas / div_up(a.C, 32 * N)), rounds = (need + most - 1) / most;
    return (int)((need + rounds - 1) / rounds);
}

}  // namespace

// Columns 32 blockIdx.x .. of row blockIdx.y of the [W + 1, C] sums, in 64-bit offsets: (W + 1) C passes 32 bits before C does.
__global__ void __launch_bounds__(512) sum_rows_kernel(const float* part, int G, int C, int W, float* out0, float* out1)
{
    pdl_wait();
    __shared__ float s[16][33];
    const int c = blockIdx.x * 32 + threadIdx.x, j = blockIdx.y;
    float v = 0.f;
    if (c < C) {
        const size_t row = (size_t)(W + 1) * C;
        const float* p = part + threadIdx.y * row + (size_t)j * C + c;
        for (int g = threadIdx.y; g < G; g += 8 * 16, p += 8 * 16 * row) {   // eight loads on their way, added in order
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = g + 16 * i < G ? p[16 * i * row] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += x[i];
        }
    }
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y || c >= C) return;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += s[r][threadIdx.x];
    if (j < W) {
        if (out0) out0[(size_t)c * W + j] = sum;
    } else if (out1) {
        out1[c] = sum;
    }
}

bool launch_sum_rows(const float* part, int G, int C, int W, float* out0, float* out1, cudaStream_t st)
{
    return launch_after(sum_rows_kernel, dim3(div_up(C, 32), W + 1), dim3(32, 16), 0, st, part, G, C, W, out0, out1);
}

size_t conv_workspace(const osdn_conv_params& p)
{
    ConvArgs a = make_args(p);
    const int N = lane_channels(p), ctas = N == 4 ? BWD_CTAS<4> : BWD_CTAS<2>;
    plan_walks(a, p, N, ctas);
    return align_up((size_t)backward_rows(a, N, ctas) * (p.W + 1) * p.C * 4, 256);
}

template <typename K> bool set_smem(K* kernel, size_t bytes)
{
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

int conv_forward(const osdn_conv_params& p, const void* x, const float* w, const float* bias, const void* init, void* out,
                 void* fin, cudaStream_t st)
{
    ConvArgs a = make_args(p);
    a.x = x; a.w = w; a.bias = bias; a.init = init; a.out = out; a.fin = fin;
    stage_mark(st, "conv_fwd");
    const int launched = by_type(p, [&](auto e, auto taps, auto act) {
        using T = decltype(e);
        auto go = [&](auto vec) {
            constexpr int N = decltype(vec)::value;
            plan_walks(a, p, N, FWD_CTAS<N>);
            using In = Stream<T, N, (N > 1)>;
            constexpr size_t smem = N > 1 ? 4 * In::DEPTH * In::BYTES : 0;
            const auto kernel = conv_fwd_kernel<T, N, decltype(taps)::value, decltype(act)::value, (N > 1)>;
            const dim3 grid(div_up(a.walks * div_up(p.C, 32 * N), 4));
            return set_smem(kernel, smem) && launch_after(kernel, grid, dim3(128), smem, st, a) ? 1 : -1;
        };
        return lane_channels(p) > 1 ? go(std::integral_constant<int, 8 / (int)sizeof(T)>{}) : go(std::integral_constant<int, 1>{});
    });
    stage_end(st);
    return launched;
}

int conv_backward(const osdn_conv_params& p, const void* x, const float* w, const float* bias, const void* init,
                  const void* dout, const void* dfin, void* dx, float* dw, float* dbias, void* dinit, void* ws, cudaStream_t st)
{
    ConvArgs a = make_args(p);
    a.x = x; a.w = w; a.bias = bias; a.init = init; a.dout = dout; a.dfin = dfin; a.dx = dx; a.dinit = dinit;
    a.partial = static_cast<float*>(ws);
    stage_mark(st, "conv_bwd");
    int launched = by_type(p, [&](auto e, auto taps, auto act) {
        using T = decltype(e);
        constexpr int W = decltype(taps)::value;
        auto go = [&](auto vec) {
            constexpr int N = decltype(vec)::value;
            plan_walks(a, p, N, BWD_CTAS<N>);
            using In = Stream<T, N, (N > 1)>;
            constexpr size_t smem = N > 1 ? 4 * In::DEPTH * 2 * In::BYTES : 0;
            const auto kernel = conv_bwd_kernel<T, N, W, decltype(act)::value, (N > 1)>;
            const int rows = backward_rows(a, N, BWD_CTAS<N>);
            if (!set_smem(kernel, smem) || !launch_after(kernel, dim3(div_up(p.C, 32 * N), rows), dim3(128), smem, st, a)) return -1;
            stage_mark(st, "conv_sums");
            return launch_sum_rows(a.partial, rows, p.C, W, dw, dbias, st) ? 2 : -1;
        };
        return lane_channels(p) > 1 ? go(std::integral_constant<int, 8 / (int)sizeof(T)>{}) : go(std::integral_constant<int, 1>{});
    });
    stage_end(st);
    return launched;
}

int conv_step(const osdn_conv_params& p, const void* x, const float* w, const float* bias, void* state, void* out, cudaStream_t st)
{
    stage_mark(st, "conv_step");
    const int launched = by_type(p, [&](auto e, auto taps, auto act) {
        using T = decltype(e);
        constexpr int W = decltype(taps)::value;
        constexpr bool SILU = decltype(act)::value;
        auto go = [&](auto vec) {
            constexpr int N = decltype(vec)::value;
            const long long n = p.C / N;
            // the taps are as many bytes as a row of two sequences (512 sequences, 2048 channels: one to a thread 6.3 us, two 5.3,
            // four 7.0; with eight channels to a lane 7.1 and more)
            const int each = (int)std::max(1ll, std::min(2ll, p.B * n / (148 * 256)));
            return launch_after(conv_step_kernel<T, N, W, SILU>, dim3(div_up(div_up(p.B, each) * n, 128)), dim3(128), 0, st,
                                static_cast<const T*>(x), w, bias, static_cast<T*>(state), static_cast<T*>(out), p.B, p.T, p.C, each)
                       ? 1 : -1;
        };
        return p.C % 4 == 0 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 1>{});
    });
    stage_end(st);
    return launched;
}

}  // namespace osdn
