// Short causal depthwise convolution over the tokens of a sequence: forward, backward, decode step.
#include "osdn_rows.cuh"

#ifndef XMF
#define XMF 4
#endif
#ifndef XUF
#define XUF 4
#endif
#ifndef XMB
#define XMB 4
#endif
#ifndef XUB
#define XUB 4
#endif
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

// z sigmoid(z) needs 1 / (1 + exp(-z)).  Where results are rounded to bf16 (2^-9 of the value) the hardware's exponential and
// reciprocal (about 2^-21) are exact enough.
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

// A thread walks the rows of a chunk over N channels, U rows on their way at a time.
template <typename T, int N, int W, bool SILU>
__global__ void __launch_bounds__(128, XMF) conv_fwd_kernel(ConvArgs a)
{
    pdl_wait();
    using Row = Channels<T, N>;
    constexpr int Q = Row::Q, U = XUF;
    const int n = a.C / N;
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= a.walks * n) return;
    const int c = (int)(i % n) * N;
    const long long walk = i / n;
    pass_empty<T, N, W>(a, a.init, a.fin, walk, c);
    Place at{(int)(walk / a.chunks), 0, a.rows.T};
    const int limit = a.rows.cu ? rows_end(a.rows) : a.rows.T;
    const int t0 = (int)(walk % a.chunks) * a.chunk, t1 = min(t0 + a.chunk, limit);
    if (t0 >= t1) return;
    const size_t base = a.rows.cu ? 0 : (size_t)at.s * a.rows.T * a.C;
    const T* x = static_cast<const T*>(a.x) + base;
    T* out = static_cast<T*>(a.out) + base;
    at.enter(a.rows, t0, limit);
    Taps<N, W> k;
    k.load(a.w, a.bias, c);
    F<Row::L> prev[W - 1][Q];
    auto refill = [&](int t) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const Row r = row_before<T, N, W>(a, x, at, t - (W - 1) + j, c);
#pragma unroll
            for (int q = 0; q < Q; ++q) prev[j][q] = r.get(q);
        }
    };
    refill(t0);
    for (int t = t0; t < t1; t += U) {
        Row v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u < t1) v[u] = Row::load(x + (size_t)(t + u) * a.C + c);
        if (t + U <= t1 && t + U < at.end) {
#pragma unroll
            for (int u = 0; u < U; ++u) convolve<T, N, W, SILU>(k, prev, v[u]).store(out + (size_t)(t + u) * a.C + c);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (t + u >= t1) break;
                if (t + u >= at.end) {   // the next sequence that is not empty
                    at.enter(a.rows, t + u, limit);
                    refill(t + u);
                }
                convolve<T, N, W, SILU>(k, prev, v[u]).store(out + (size_t)(t + u) * a.C + c);
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
    }
}

// A thread walks the rows of its chunk and, for the gradients of the chunk's last rows, up to W-1 behind it.  acc[j] is the
// gradient, so far, of row t - (W-1) + j; it is complete once dz_t is in, or at the sequence's end, where all W-1 last rows
// take the gradient of the state as well.  Rows in front of a sequence are its state's.
template <typename T, int N, int W, bool SILU>
__global__ void __launch_bounds__(128, XMB) conv_bwd_kernel(ConvArgs a, int gx)
{
    extern __shared__ float sums[];   // [128 / gx][W + 1][gx * N]
    pdl_wait();
    using Row = Channels<T, N>;
    constexpr int Q = Row::Q, L = Row::L, U = XUB;
    const int n = a.C / N;
    const int lane = threadIdx.x % gx, row = threadIdx.x / gx, rows = blockDim.x / gx;
    const int group = blockIdx.x * gx + lane;
    const int c = group * N;
    F<L> dw[W][Q], db[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][q] = all<L>(0.f);
        db[q] = all<L>(0.f);
    }
    if (group < n) {
        Taps<N, W> k;
        k.load(a.w, a.bias, c);
        const int limit = a.rows.cu ? rows_end(a.rows) : a.rows.T;
        for (long long walk = (long long)blockIdx.y * rows + row; walk < a.walks; walk += (long long)gridDim.y * rows) {
            pass_empty<T, N, W>(a, a.dfin, a.dinit, walk, c);
            Place at{(int)(walk / a.chunks), 0, a.rows.T};
            const int t0 = (int)(walk % a.chunks) * a.chunk, t1 = min(t0 + a.chunk, limit);
            if (t0 >= t1) continue;
            const size_t base = a.rows.cu ? 0 : (size_t)at.s * a.rows.T * a.C;
            const T* x = static_cast<const T*>(a.x) + base;
            const T* dout = static_cast<const T*>(a.dout) + base;
            T* dx = static_cast<T*>(a.dx) + base;
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
            refill(t0);
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
            const int tend = min(t1 + W - 1, limit);
            bool over = false;
            for (int t = t0; t < tend && !over; t += U) {
                Row xv[U], gv[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (t + u < tend) {
                        xv[u] = Row::load(x + (size_t)(t + u) * a.C + c);
                        gv[u] = Row::load(dout + (size_t)(t + u) * a.C + c);
                    }
                if (t + U <= t1 && t + U < at.end && t - (W - 1) >= t0 && t - (W - 1) >= at.start) {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        take(xv[u], gv[u], true);
                        Row r;
#pragma unroll
                        for (int q = 0; q < Q; ++q) r.set(q, acc[0][q]);
                        r.store(dx + (size_t)(t + u - (W - 1)) * a.C + c);
                        shift();
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int s = t + u;
                        if (s >= tend || over) continue;
                        if (s >= at.end) {
                            if (s >= t1) {
                                over = true;
                                continue;
                            }
                            at.enter(a.rows, s, limit);
                            refill(s);
                        }
                        take(xv[u], gv[u], s < t1);
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
            }
        }
    }
    // the block's sums, row by row in order
    float* mine = sums + (size_t)row * (W + 1) * gx * N;
#pragma unroll
    for (int m = 0; m < N; ++m) {
#pragma unroll
        for (int j = 0; j < W; ++j) mine[(j * gx + lane) * N + m] = dw[j][m / L].x[m % L];
        mine[(W * gx + lane) * N + m] = db[m / L].x[m % L];
    }
    __syncthreads();
    const int width = gx * N;
    for (int m = threadIdx.x; m < (W + 1) * width; m += blockDim.x) {
        float v = 0.f;
        for (int r = 0; r < rows; ++r) v += sums[(size_t)r * (W + 1) * width + m];
        const int j = m / width, ch = blockIdx.x * width + m % width;
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

// Chunks of a walk: long ones read fewer rows twice, short ones make more threads.
void plan_walks(ConvArgs& a, const osdn_conv_params& p, int N, int longest)
{
    const long long rows = (long long)p.B * p.T, n = p.C / N;
    int chunk = longest;
    while (chunk > 8 && rows * n / chunk < 148ll * 512) chunk /= 2;
    a.chunk = chunk;
    a.chunks = div_up(p.T, chunk);
    a.walks = (long long)(p.nseq > 0 ? 1 : p.B) * a.chunks;
}
#ifndef XLF
#define XLF 32
#endif
#ifndef XLB
#define XLB 64
#endif
constexpr int FWD_CHUNK = XLF, BWD_CHUNK = XLB;

ConvArgs make_args(const osdn_conv_params& p)
{
    ConvArgs a{};
    a.rows = {p.nseq > 0 ? p.cu_seqlens : nullptr, p.nseq > 0 ? p.nseq : p.B, p.T};
    a.C = p.C;
    return a;
}

template <typename T> constexpr int kWide = sizeof(T) == 2 ? 8 : 4;   // channels of a 16-byte access

struct BwdPlan {
    int gx, grid_x, grid_y;
};
BwdPlan plan_backward(const ConvArgs& a, const osdn_conv_params& p, int N)
{
    const int n = p.C / N;
    BwdPlan b;
    b.gx = 32;
    while (b.gx > 1 && b.gx / 2 >= n) b.gx /= 2;
    b.grid_x = div_up(n, b.gx);
    const long long blocks = (a.walks + 128 / b.gx - 1) / (128 / b.gx);
    const long long most = std::max(1, 148 * 4 / b.grid_x), rounds = (blocks + most - 1) / most;
    b.grid_y = (int)((blocks + rounds - 1) / rounds);   // the same number of walks for every thread
    return b;
}
int backward_vec(const osdn_conv_params& p) { return p.C % 4 == 0 ? 4 : 1; }

}  // namespace

// out0[(m % C) W + m / C] = sum of column m < W C, out1[m - W C] the others': one block per 32 columns.
__global__ void __launch_bounds__(512) sum_rows_kernel(const float* part, int G, int C, int W, int M, float* out0, float* out1)
{
    pdl_wait();
    __shared__ float s[16][33];
    const int m = blockIdx.x * 32 + threadIdx.x;
    float v = 0.f;
    if (m < M)
        for (int g = threadIdx.y; g < G; g += 16) v += part[(size_t)g * M + m];
    s[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y || m >= M) return;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += s[r][threadIdx.x];
    if (m < W * C) {
        if (out0) out0[(size_t)(m % C) * W + m / C] = sum;
    } else if (out1) {
        out1[m - W * C] = sum;
    }
}

bool launch_sum_rows(const float* part, int G, int C, int W, int M, float* out0, float* out1, cudaStream_t st)
{
    return launch_after(sum_rows_kernel, dim3(div_up(M, 32)), dim3(32, 16), 0, st, part, G, C, W, M, out0, out1);
}

size_t conv_workspace(const osdn_conv_params& p)
{
    ConvArgs a = make_args(p);
    plan_walks(a, p, backward_vec(p), BWD_CHUNK);
    return align_up((size_t)plan_backward(a, p, backward_vec(p)).grid_y * (p.W + 1) * p.C * 4, 256);
}

int conv_forward(const osdn_conv_params& p, const void* x, const float* w, const float* bias, const void* init, void* out,
                 void* fin, cudaStream_t st)
{
    ConvArgs a = make_args(p);
    a.x = x; a.w = w; a.bias = bias; a.init = init; a.out = out; a.fin = fin;
    stage_mark(st, "conv_fwd");
    const int launched = by_type(p, [&](auto e, auto taps, auto act) {
        using T = decltype(e);
        constexpr int W = decltype(taps)::value;
        constexpr bool SILU = decltype(act)::value;
        auto go = [&](auto vec) {
            constexpr int N = decltype(vec)::value;
            plan_walks(a, p, N, FWD_CHUNK);
            return launch_after(conv_fwd_kernel<T, N, W, SILU>, dim3(div_up(a.walks * (p.C / N), 128)), dim3(128), 0, st, a) ? 1 : -1;
        };
        return p.C % kWide<T> == 0 ? go(std::integral_constant<int, kWide<T>>{}) : go(std::integral_constant<int, 1>{});
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
        constexpr bool SILU = decltype(act)::value;
        auto go = [&](auto vec) {
            constexpr int N = decltype(vec)::value;
            plan_walks(a, p, N, BWD_CHUNK);
            const BwdPlan b = plan_backward(a, p, N);
            const size_t smem = (size_t)128 * (W + 1) * N * 4;
            if (!launch_after(conv_bwd_kernel<T, N, W, SILU>, dim3(b.grid_x, b.grid_y), dim3(128), smem, st, a, b.gx)) return -1;
            stage_mark(st, "conv_sums");
            return launch_sum_rows(a.partial, b.grid_y, p.C, W, (W + 1) * p.C, dw, dbias, st) ? 2 : -1;
        };
        return backward_vec(p) == 4 ? go(std::integral_constant<int, 4>{}) : go(std::integral_constant<int, 1>{});
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
            const int each = (int)std::max(1ll, std::min(4ll, p.B * n / (148 * 256)));   // the taps are as many bytes as a row
            return launch_after(conv_step_kernel<T, N, W, SILU>, dim3(div_up(div_up(p.B, each) * n, 128)), dim3(128), 0, st,
                                static_cast<const T*>(x), w, bias, static_cast<T*>(state), static_cast<T*>(out), p.B, p.T, p.C, each)
                       ? 1 : -1;
        };
        return p.C % kWide<T> == 0 ? go(std::integral_constant<int, kWide<T>>{}) : go(std::integral_constant<int, 1>{});
    });
    stage_end(st);
    return launched;
}

}  // namespace osdn
