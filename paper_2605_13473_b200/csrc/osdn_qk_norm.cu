// Norms of queries and keys, head by head, with the rotation by the position in the same pass: forward and backward.
#include "osdn_rows.cuh"

namespace osdn {
namespace {

constexpr int NONE = 0, HALF = 1, PAIRS = 2;   // rotation

struct NormArgs {
    const void *q, *k, *dqo, *dko;
    void *qo, *ko, *dq, *dk;
    const float *qw, *kw;
    const double* inv_freq;
    const int* pos;
    float* partial;          // [blocks, 2, D] sums of the weights' gradients
    Rows rows;
    long long q_row, k_row, dq_row, dk_row;
    int Hq, Hk, D, R;        // R: features that are turned
    int heads, blocks;       // heads a lane group takes at a time; such blocks of a token's heads
    long long tokens;
    float share, eps;        // 1 or 1 / D
};

// cos and sin of the pairs a lane's eight features belong to.
//   HALF: features f0 .. f0+7 are the first (or second) members of pairs f0 mod R/2 ..;  PAIRS: of the pairs f0/2 .. f0/2+3.
template <int ROT> struct Turn {
    static constexpr int N = ROT == HALF ? 8 : 4;
    float c[N], s[N];
    __device__ __forceinline__ void set(const NormArgs& a, int f0, int pos)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) { c[j] = 1.f; s[j] = 0.f; }
        if (f0 >= a.R) return;
        const int n0 = ROT == HALF ? (f0 < a.R / 2 ? f0 : f0 - a.R / 2) : f0 / 2;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            double t = pos * (a.inv_freq[n0 + j] * 0.15915494309189535);   // turns; 1 / (2 pi)
            t -= rint(t);
            sincospif(2.f * (float)t, &s[j], &c[j]);
        }
    }
};

// Turns a lane's eight features (back: by the opposite angle).  HALF: the other member of a pair is R/16 lanes away.
template <int ROT, bool BACK, int LH>
__device__ __forceinline__ void turn(const Turn<ROT>& r, int f0, int R, float (&x)[8])
{
    if constexpr (ROT == HALF) {
        const int lane = threadIdx.x & (LH - 1);
        const bool first = f0 < R / 2, in = f0 < R;
        const int other = !in ? lane : first ? lane + R / 16 : lane - R / 16;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y = __shfl_sync(0xffffffffu, x[j], other, LH);
            const float s = first != BACK ? -r.s[j] : r.s[j];
            if (in) x[j] = fmaf(x[j], r.c[j], y * s);
        }
    } else if constexpr (ROT == PAIRS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float s = BACK ? -r.s[j] : r.s[j];
            const float p = x[2 * j], q = x[2 * j + 1];
            x[2 * j] = fmaf(p, r.c[j], -q * s);
            x[2 * j + 1] = fmaf(p, s, q * r.c[j]);
        }
    }
}

template <int LH> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = LH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ void load_weight(const float* w, int f0, bool in, float (&x)[8])
{
    if (w && in) {
        load_vec<8>(w + f0, x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 1.f;
    }
}

// The token's place: positions given, or counted from its sequence's start.
__device__ __forceinline__ int place_of(const NormArgs& a, long long token)
{
    if (a.pos) return a.pos[token];
    if (!a.rows.cu) return (int)(token % a.rows.T);
    return (int)token - a.rows.cu[seq_of(a.rows, (int)token)];
}

// LH lanes to a head, eight features to a lane; a lane group takes a token and `heads` of its heads, U loads on their way.
template <typename T, int LH, int ROT>
__global__ void __launch_bounds__(256) qk_norm_fwd_kernel(NormArgs a)
{
    pdl_wait();
    constexpr int U = 4;
    const long long item = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / LH;
    const int f0 = (threadIdx.x & (LH - 1)) * 8;
    const long long token = item / a.blocks;
    const int h0 = (int)(item % a.blocks) * a.heads;
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    const bool live = token < limit, in = live && f0 < a.D;
    const int h1 = live ? min(h0 + a.heads, a.Hq + a.Hk) : h0;
    Turn<ROT> r;
    if constexpr (ROT != NONE) r.set(a, f0, live ? place_of(a, token) : 0);
    float wq[8], wk[8];
    load_weight(a.qw, f0, f0 < a.D, wq);
    load_weight(a.kw, f0, f0 < a.D, wk);
    for (int b = 0; b < a.heads; b += U) {   // the same for every lane of a warp
        float x[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + b + u;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[u][j] = 0.f;
            if (in && h < h1) {
                const T* p = h < a.Hq ? static_cast<const T*>(a.q) + token * a.q_row + (size_t)h * a.D
                                      : static_cast<const T*>(a.k) + token * a.k_row + (size_t)(h - a.Hq) * a.D;
                load_vec<8>(p + f0, x[u]);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b + u >= a.heads) break;
            const int h = h0 + b + u;
            float ss = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) ss = fmaf(x[u][j], x[u][j], ss);
            const float n = rsqrtf(fmaf(group_sum<LH>(ss), a.share, a.eps));
#pragma unroll
            for (int j = 0; j < 8; ++j) x[u][j] *= n * (h < a.Hq ? wq[j] : wk[j]);
            turn<ROT, false, LH>(r, f0, a.R, x[u]);
            if (in && h < h1) {
                T* p = h < a.Hq ? static_cast<T*>(a.qo) + ((size_t)token * a.Hq + h) * a.D
                                : static_cast<T*>(a.ko) + ((size_t)token * a.Hk + (h - a.Hq)) * a.D;
                store_vec<8>(p + f0, x[u]);
            }
        }
    }
}

// Gradients: with dv = Rot^-1 dy, dw = sum dv u, du = dv w, dx = r (du - u <du, u> share).  A lane group walks over tokens
// and keeps the sums of its eight features for queries and for keys; the block adds its groups in order.
template <typename T, int LH, int ROT>
__global__ void __launch_bounds__(256) qk_norm_bwd_kernel(NormArgs a)
{
    __shared__ float sums[256 / LH][2][LH * 8];
    pdl_wait();
    constexpr int U = 2, GROUPS = 256 / LH;
    const int lane = threadIdx.x & (LH - 1), group = threadIdx.x / LH, f0 = lane * 8;
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    float wq[8], wk[8], dwq[8] = {}, dwk[8] = {};
    load_weight(a.qw, f0, f0 < a.D, wq);
    load_weight(a.kw, f0, f0 < a.D, wk);
    const long long items = a.tokens * a.blocks;
    for (long long first = (long long)blockIdx.x * GROUPS; first < items; first += (long long)gridDim.x * GROUPS) {
        const long long item = first + group, token = item / a.blocks;
        const int h0 = (int)(item % a.blocks) * a.heads;
        const bool live = token < limit, in = live && f0 < a.D;
        const int h1 = live ? min(h0 + a.heads, a.Hq + a.Hk) : h0;
        Turn<ROT> r;
        if constexpr (ROT != NONE) r.set(a, f0, live ? place_of(a, token) : 0);
        for (int b = 0; b < a.heads; b += U) {
            float x[U][8], g[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + b + u;
#pragma unroll
                for (int j = 0; j < 8; ++j) { x[u][j] = 0.f; g[u][j] = 0.f; }
                if (in && h < h1) {
                    const bool isq = h < a.Hq;
                    const T* p = isq ? static_cast<const T*>(a.q) + token * a.q_row + (size_t)h * a.D
                                     : static_cast<const T*>(a.k) + token * a.k_row + (size_t)(h - a.Hq) * a.D;
                    const T* d = isq ? static_cast<const T*>(a.dqo) + ((size_t)token * a.Hq + h) * a.D
                                     : static_cast<const T*>(a.dko) + ((size_t)token * a.Hk + (h - a.Hq)) * a.D;
                    load_vec<8>(p + f0, x[u]);
                    load_vec<8>(d + f0, g[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (b + u >= a.heads) break;
                const int h = h0 + b + u;
                const bool isq = h < a.Hq;
                turn<ROT, true, LH>(r, f0, a.R, g[u]);
                float ss = 0.f, dot = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    ss = fmaf(x[u][j], x[u][j], ss);
                    dot = fmaf(g[u][j] * (isq ? wq[j] : wk[j]), x[u][j], dot);
                }
                const float n = rsqrtf(fmaf(group_sum<LH>(ss), a.share, a.eps));
                const float m = group_sum<LH>(dot) * n * n * a.share;   // <du, u> share / |scale of u|
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float s = g[u][j] * x[u][j] * n;
                    if (isq) dwq[j] += s;
                    else dwk[j] += s;
                    g[u][j] = n * (g[u][j] * (isq ? wq[j] : wk[j]) - x[u][j] * m);
                }
                if (in && h < h1) {
                    T* p = isq ? static_cast<T*>(a.dq) + token * a.dq_row + (size_t)h * a.D
                               : static_cast<T*>(a.dk) + token * a.dk_row + (size_t)(h - a.Hq) * a.D;
                    store_vec<8>(p + f0, g[u]);
                }
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sums[group][0][f0 + j] = dwq[j];
        sums[group][1][f0 + j] = dwk[j];
    }
    __syncthreads();
    for (int m = threadIdx.x; m < 2 * a.D; m += 256) {
        float v = 0.f;
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) v += sums[s][m / a.D][m % a.D];
        a.partial[(size_t)blockIdx.x * 2 * a.D + m] = v;
    }
}

NormArgs make_args(const osdn_qk_norm_params& p)
{
    NormArgs a{};
    a.rows = {p.nseq > 0 ? p.cu_seqlens : nullptr, p.nseq > 0 ? p.nseq : p.B, p.T};
    const long long wq = (long long)p.Hq * p.D, wk = (long long)p.Hk * p.D;
    a.q_row = p.q_row ? p.q_row : wq;
    a.k_row = p.k_row ? p.k_row : wk;
    a.dq_row = p.dq_row ? p.dq_row : wq;
    a.dk_row = p.dk_row ? p.dk_row : wk;
    a.Hq = p.Hq; a.Hk = p.Hk; a.D = p.D; a.R = p.rot_dim;
    a.tokens = (long long)p.B * p.T;
    a.share = p.norm == OSDN_NORM_RMS ? 1.f / p.D : 1.f;
    a.eps = p.eps;
    // with many tokens a lane group takes sixteen heads of one (their angles are the same), with few it takes one
    a.heads = 16;
    while (a.heads > 1 && (a.heads >= 2 * (p.Hq + p.Hk) || a.tokens * div_up(p.Hq + p.Hk, a.heads) < 148 * 64)) a.heads /= 2;
    a.blocks = div_up(p.Hq + p.Hk, a.heads);
    return a;
}

int bwd_blocks(const NormArgs& a, int LH)
{
    const long long need = (a.tokens * a.blocks + 256 / LH - 1) / (256 / LH);
    return (int)std::min<long long>(need, 148 * 4);
}
int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }

template <typename F> int by_type(const osdn_qk_norm_params& p, F f)   // f(element, lanes to a head, rotation)
{
    auto rot = [&](auto e, auto lh) {
        if (p.rot_dim == 0) return f(e, lh, std::integral_constant<int, NONE>{});
        if (p.rot_layout == OSDN_ROT_HALF) return f(e, lh, std::integral_constant<int, HALF>{});
        return f(e, lh, std::integral_constant<int, PAIRS>{});
    };
    auto lanes = [&](auto e) {
        if (p.D <= 64) return rot(e, std::integral_constant<int, 8>{});
        if (p.D <= 128) return rot(e, std::integral_constant<int, 16>{});
        return rot(e, std::integral_constant<int, 32>{});
    };
    return p.io_dtype == OSDN_FP32 ? lanes(0.f) : lanes(__nv_bfloat16{});
}

}  // namespace

size_t qk_norm_workspace(const osdn_qk_norm_params& p)
{
    return align_up((size_t)bwd_blocks(make_args(p), lanes_of(p.D)) * 2 * p.D * 4, 256);
}

int qk_norm_forward(const osdn_qk_norm_params& p, const void* q, const void* k, const float* qw, const float* kw,
                    const double* inv_freq, const int* pos, void* qo, void* ko, cudaStream_t st)
{
    NormArgs a = make_args(p);
    a.q = q; a.k = k; a.qw = qw; a.kw = kw; a.inv_freq = inv_freq; a.pos = pos; a.qo = qo; a.ko = ko;
    stage_mark(st, "qk_norm_fwd");
    const int n = by_type(p, [&](auto e, auto lh, auto rot) {
        constexpr int LH = decltype(lh)::value, ROT = decltype(rot)::value;
        const unsigned grid = div_up(a.tokens * a.blocks, 256 / LH);
        return launch_after(qk_norm_fwd_kernel<decltype(e), LH, ROT>, dim3(grid), dim3(256), 0, st, a) ? 1 : -1;
    });
    stage_end(st);
    return n;
}

int qk_norm_backward(const osdn_qk_norm_params& p, const void* q, const void* k, const float* qw, const float* kw,
                     const double* inv_freq, const int* pos, const void* dqo, const void* dko, void* dq, void* dk, float* dqw,
                     float* dkw, void* ws, cudaStream_t st)
{
    NormArgs a = make_args(p);
    a.q = q; a.k = k; a.qw = qw; a.kw = kw; a.inv_freq = inv_freq; a.pos = pos; a.dqo = dqo; a.dko = dko; a.dq = dq; a.dk = dk;
    a.partial = dqw || dkw ? static_cast<float*>(ws) : nullptr;
    stage_mark(st, "qk_norm_bwd");
    int n = by_type(p, [&](auto e, auto lh, auto rot) {
        constexpr int LH = decltype(lh)::value, ROT = decltype(rot)::value;
        const int blocks = bwd_blocks(a, LH);
        if (!launch_after(qk_norm_bwd_kernel<decltype(e), LH, ROT>, dim3(blocks), dim3(256), 0, st, a)) return -1;
        if (!a.partial) return 1;
        stage_mark(st, "qk_norm_sums");
        return launch_sum_rows(a.partial, blocks, p.D, 1, 2 * p.D, dqw, dkw, st) ? 2 : -1;
    });
    stage_end(st);
    return n;
}

}  // namespace osdn
