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

// Where results are rounded to bf16 (2^-9 of the value) the quick exponential and division (about 2^-21) are exact enough.
template <typename T> __device__ __forceinline__ float sigmoid(float z)
{
    if constexpr (sizeof(T) == 2) return __fdividef(1.f, 1.f + __expf(-z));
    else return 1.f / (1.f + expf(-z));
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
__device__ __forceinline__ void row_before(const ConvArgs& a, const T* x, const Place& at, int t, int c, float (&v)[N])
{
    if (t >= at.start) {
        load_vec<N>(x + (size_t)t * a.C + c, v);
    } else if (a.init) {
        load_vec<N>(static_cast<const T*>(a.init) + ((size_t)at.s * (W - 1) + (W - 1) + (t - at.start)) * a.C + c, v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.f;
    }
}

template <typename T, int N, int W>
__device__ __forceinline__ void load_taps(const ConvArgs& a, int c, float (&w)[W][N], float (&b)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i][j] = a.w[(size_t)(c + j) * W + i];
        b[j] = a.bias ? a.bias[c + j] : 0.f;
    }
}

// A state of an empty sequence (or its gradient) passes through.
template <typename T, int N, int W>
__device__ __forceinline__ void pass_empty(const ConvArgs& a, const void* from, void* to, long long walk, int c)
{
    if (!a.rows.cu || !to) return;
    for (long long s = walk; s < a.rows.S; s += a.walks) {
        if (a.rows.cu[s + 1] > a.rows.cu[s]) continue;
        for (int i = 0; i < W - 1; ++i) {
            float v[N] = {};
            const size_t at = ((size_t)s * (W - 1) + i) * a.C + c;
            if (from) load_vec<N>(static_cast<const T*>(from) + at, v);
            store_vec<N>(static_cast<T*>(to) + at, v);
        }
    }
}

template <typename T, int N, int W, bool SILU>
__global__ void __launch_bounds__(128) conv_fwd_kernel(ConvArgs a)
{
    pdl_wait();
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
    float w[W][N], b[N], prev[W - 1][N];
    load_taps<T, N, W>(a, c, w, b);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) row_before<T, N, W>(a, x, at, t0 - (W - 1) + j, c, prev[j]);
    constexpr int U = 4;
    for (int t = t0; t < t1; t += U) {
        float v[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u < t1) load_vec<N>(x + (size_t)(t + u) * a.C + c, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t + u >= t1) break;
            if (t + u >= at.end) {   // the next sequence that is not empty
                at.enter(a.rows, t + u, limit);
#pragma unroll
                for (int j = 0; j < W - 1; ++j) row_before<T, N, W>(a, x, at, t + u - (W - 1) + j, c, prev[j]);
            }
            float z[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float y = b[k];
#pragma unroll
                for (int j = 0; j < W - 1; ++j) y = fmaf(w[j][k], prev[j][k], y);
                y = fmaf(w[W - 1][k], v[u][k], y);
                z[k] = SILU ? y * sigmoid<T>(y) : y;
#pragma unroll
                for (int j = 0; j + 1 < W - 1; ++j) prev[j][k] = prev[j + 1][k];
                prev[W - 2][k] = v[u][k];
            }
            store_vec<N>(out + (size_t)(t + u) * a.C + c, z);
            if (a.fin && t + u + 1 == at.end)
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
                    store_vec<N>(static_cast<T*>(a.fin) + ((size_t)at.s * (W - 1) + j) * a.C + c, prev[j]);
        }
    }
}

// A thread walks the tokens of its chunk and, for the gradients of the chunk's last rows, up to W-1 behind it.  acc[j] is the
// gradient, so far, of row t - (W-1) + j; it is complete once dz_t is in, or at the sequence's end, where all W-1 last rows
// take the gradient of the state as well.  Rows in front of a sequence are its state's.
template <typename T, int N, int W, bool SILU>
__global__ void __launch_bounds__(128) conv_bwd_kernel(ConvArgs a, int gx)
{
    extern __shared__ float sums[];   // [128 / gx][W + 1][gx * N]
    pdl_wait();
    const int n = a.C / N;
    const int lane = threadIdx.x % gx, row = threadIdx.x / gx, rows = blockDim.x / gx;
    const int group = blockIdx.x * gx + lane;
    const int c = group * N;
    float dw[W][N] = {}, db[N] = {};
    if (group < n) {
        float w[W][N], b[N];
        load_taps<T, N, W>(a, c, w, b);
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
            float prev[W - 1][N], acc[W][N] = {};
#pragma unroll
            for (int j = 0; j < W - 1; ++j) row_before<T, N, W>(a, x, at, t0 - (W - 1) + j, c, prev[j]);
            auto put = [&](int t, const float (&v)[N]) {   // the gradient of row t is complete
                if (t >= at.start) {
                    if (t >= t0 && t < t1) store_vec<N>(dx + (size_t)t * a.C + c, v);
                } else if (a.dinit && at.start >= t0 && at.start < t1) {
                    store_vec<N>(static_cast<T*>(a.dinit) + ((size_t)at.s * (W - 1) + (W - 1) + (t - at.start)) * a.C + c, v);
                }
            };
            for (int t = t0; t < t1 + W - 1 && t < limit; ++t) {
                if (t >= at.end) {
                    if (t >= t1) break;
                    at.enter(a.rows, t, limit);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) {
                        row_before<T, N, W>(a, x, at, t - (W - 1) + j, c, prev[j]);
#pragma unroll
                        for (int k = 0; k < N; ++k) acc[j][k] = 0.f;
                    }
                }
                float v[N], g[N];
                load_vec<N>(x + (size_t)t * a.C + c, v);
                load_vec<N>(dout + (size_t)t * a.C + c, g);
                const bool own = t < t1;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    if (SILU) {
                        float z = b[k];
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) z = fmaf(w[j][k], prev[j][k], z);
                        z = fmaf(w[W - 1][k], v[k], z);
                        const float s = sigmoid<T>(z);
                        g[k] *= s * fmaf(z, 1.f - s, 1.f);
                    }
                    const float d = own ? g[k] : 0.f;
                    db[k] += d;
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) {
                        dw[j][k] = fmaf(d, prev[j][k], dw[j][k]);
                        acc[j][k] = fmaf(w[j][k], g[k], acc[j][k]);
                    }
                    dw[W - 1][k] = fmaf(d, v[k], dw[W - 1][k]);
                    acc[W - 1][k] = w[W - 1][k] * g[k];
#pragma unroll
                    for (int j = 0; j + 1 < W - 1; ++j) prev[j][k] = prev[j + 1][k];
                    prev[W - 2][k] = v[k];
                }
                put(t - (W - 1), acc[0]);
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int k = 0; k < N; ++k) acc[j][k] = acc[j + 1][k];
                if (t + 1 == at.end) {
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) {
                        if (a.dfin) {
                            float f[N];
                            load_vec<N>(static_cast<const T*>(a.dfin) + ((size_t)at.s * (W - 1) + j) * a.C + c, f);
#pragma unroll
                            for (int k = 0; k < N; ++k) acc[j][k] += f[k];
                        }
                        put(t - (W - 2) + j, acc[j]);
                    }
                }
            }
        }
    }
    // the block's sums, row by row in order
    float* mine = sums + (size_t)row * (W + 1) * gx * N;
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
        for (int j = 0; j < W; ++j) mine[(j * gx + lane) * N + k] = dw[j][k];
        mine[(W * gx + lane) * N + k] = db[k];
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

template <typename T, int N, int W, bool SILU>
__global__ void __launch_bounds__(128) conv_step_kernel(const T* x, const float* weight, const float* bias, T* state, T* out, int B,
                                                        int L, int C)
{
    pdl_wait();
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    const int n = C / N;
    if (i >= (long long)B * n) return;
    const size_t s = i / n;
    const int c = (int)(i % n) * N;
    ConvArgs a{};
    a.w = weight; a.bias = bias; a.C = C;
    float w[W][N], b[N], prev[W - 1][N];
    load_taps<T, N, W>(a, c, w, b);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) load_vec<N>(state + (s * (W - 1) + j) * C + c, prev[j]);
    for (int t = 0; t < L; ++t) {
        float v[N];
        load_vec<N>(x + (s * L + t) * C + c, v);
        float z[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float y = b[k];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) y = fmaf(w[j][k], prev[j][k], y);
            y = fmaf(w[W - 1][k], v[k], y);
            z[k] = SILU ? y * sigmoid<T>(y) : y;
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) prev[j][k] = prev[j + 1][k];
            prev[W - 2][k] = v[k];
        }
        store_vec<N>(out + (s * L + t) * C + c, z);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_vec<N>(state + (s * (W - 1) + j) * C + c, prev[j]);
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
void plan_walks(ConvArgs& a, const osdn_conv_params& p, int N)
{
    const long long rows = (long long)p.B * p.T, n = p.C / N;
    int chunk = 64;
    while (chunk > 8 && rows * n / chunk < 148ll * 1024) chunk /= 2;
    a.chunk = chunk;
    a.chunks = div_up(p.T, chunk);
    a.walks = (long long)(p.nseq > 0 ? 1 : p.B) * a.chunks;
}

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
    const long long most = std::max(1, 148 * 4 / b.grid_x);
    b.grid_y = (int)std::min(blocks, most);
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
    plan_walks(a, p, backward_vec(p));
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
            plan_walks(a, p, N);
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
            plan_walks(a, p, N);
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
            return launch_after(conv_step_kernel<T, N, W, SILU>, dim3(div_up((long long)p.B * (p.C / N), 128)), dim3(128), 0, st,
                                static_cast<const T*>(x), w, bias, static_cast<T*>(state), static_cast<T*>(out), p.B, p.T, p.C)
                       ? 1 : -1;
        };
        return p.C % kWide<T> == 0 ? go(std::integral_constant<int, kWide<T>>{}) : go(std::integral_constant<int, 1>{});
    });
    stage_end(st);
    return launched;
}

}  // namespace osdn
