// Norms of queries and keys, head by head, with the rotation by the position in the same pass: forward and backward.
#include "osdn_rows.cuh"

#ifndef XNF
#define XNF 3
#endif
#ifndef XNB
#define XNB 2
#endif
#ifndef XNG
#define XNG 2
#endif
namespace osdn {
namespace {

constexpr int NONE = 0, HALF = 1, PAIRS = 2;   // rotation

struct NormArgs {
    const void *q, *k, *dqo, *dko;
    void *qo, *ko, *dq, *dk;
    const float *qw, *kw;
    const double* inv_freq;
    const int* pos;
    float* partial;          // [CTAs, 2, D] sums of the weights' gradients
    Rows rows;
    long long q_row, k_row, dq_row, dk_row;
    int Hq, Hk, D, R;        // R: features that are turned
    int heads, q_parts, parts;   // few tokens: a lane group takes `heads` heads, queries' parts first; parts = 0: whole tokens
    long long tokens;
    float share, eps;        // 1 or 1 / D
};

// cos and sin of the pairs a lane's eight features belong to, two at a time.
//   HALF: features f0 .. f0+7 are the first (or second) members of pairs f0 mod R/2 ..;  PAIRS: of the pairs f0/2 .. f0/2+3.
template <int ROT> struct Turn {
    static constexpr int N = ROT == NONE ? 1 : ROT == HALF ? 8 : 4;
    float c[N], s[N];
    __device__ __forceinline__ void set(const NormArgs& a, int f0, int pos)
    {
        if constexpr (ROT != NONE) {
#pragma unroll
            for (int j = 0; j < N; ++j) { c[j] = 1.f; s[j] = 0.f; }
            if (f0 >= a.R) return;
            const bool second = ROT == HALF && f0 >= a.R / 2;
            const int n0 = ROT == HALF ? (second ? f0 - a.R / 2 : f0) : f0 / 2;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                double t = pos * (a.inv_freq[n0 + j] * 0.15915494309189535);   // turns; 1 / (2 pi)
                t -= rint(t);
                sincospif(2.f * (float)t, &s[j], &c[j]);
                if (second) s[j] = -s[j];   // x cos - other sin becomes x cos + other sin
            }
        }
    }
};

// Turns a lane's eight features (BACK: by the opposite angle).  HALF: the other member of a pair is R/16 lanes away.
template <int ROT, bool BACK, int LH> __device__ __forceinline__ void turn(const Turn<ROT>& r, int f0, int R, F<2> (&x)[4])
{
    if constexpr (ROT == HALF) {
        const int lane = threadIdx.x & (LH - 1);
        const int other = f0 >= R ? lane : f0 < R / 2 ? lane + R / 16 : lane - R / 16;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            F<2> y;
            y.x[0] = __shfl_sync(0xffffffffu, x[q].x[0], other, LH);
            y.x[1] = __shfl_sync(0xffffffffu, x[q].x[1], other, LH);
            const F<2> c = {{r.c[2 * q], r.c[2 * q + 1]}}, s = {{BACK ? r.s[2 * q] : -r.s[2 * q], BACK ? r.s[2 * q + 1] : -r.s[2 * q + 1]}};
            x[q] = fma(x[q], c, mul(y, s));
        }
    } else if constexpr (ROT == PAIRS) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float s = BACK ? -r.s[q] : r.s[q];
            const F<2> swapped = {{x[q].x[1], x[q].x[0]}};
            x[q] = fma(x[q], all<2>(r.c[q]), mul(swapped, F<2>{{-s, s}}));
        }
    }
}

template <int LH> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = LH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <bool WEIGHTS> struct Weight {
    F<2> w[WEIGHTS ? 4 : 1];
    __device__ __forceinline__ void load(const float* p, int f0, bool in)
    {
        if constexpr (WEIGHTS) {
            float x[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (p && in) load_vec<8>(p + f0, x);
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = {{x[2 * q], x[2 * q + 1]}};
        }
    }
    __device__ __forceinline__ F<2> times(int q, const F<2>& v) const
    {
        if constexpr (WEIGHTS) return mul(v, w[q]);
        else return v;
    }
};

// The token's place: positions given, or counted from its sequence's start.
__device__ __forceinline__ int place_of(const NormArgs& a, long long token)
{
    if (a.pos) return a.pos[token];
    if (!a.rows.cu) return (int)(token % a.rows.T);
    return (int)token - a.rows.cu[seq_of(a.rows, (int)token)];
}

// n heads of D features, one after the other, with U loads on their way; `trips` >= n is the same for every lane of a warp.
template <typename T, int LH, int ROT, bool WEIGHTS, int U>
__device__ __forceinline__ void norm_heads(const NormArgs& a, const Turn<ROT>& r, const Weight<WEIGHTS>& w, const T* in, T* out, int f0,
                                           int n, int trips)
{
    using Row = Channels<T, 8>;
    for (int h = 0; h < trips; h += U) {
        Row raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = h + u < n ? Row::load(in + (size_t)(h + u) * a.D) : Row::zero();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            F<2> x[4], ss = all<2>(0.f);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                x[q] = raw[u].get(q);
                ss = fma(x[q], x[q], ss);
            }
            const float m = rsqrtf(fmaf(group_sum<LH>(ss.x[0] + ss.x[1]), a.share, a.eps));
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = w.times(q, mul(x[q], all<2>(m)));
            turn<ROT, false, LH>(r, f0, a.R, x);
            if (h + u < n) {
                Row y;
#pragma unroll
                for (int q = 0; q < 4; ++q) y.set(q, x[q]);
                y.store(out + (size_t)(h + u) * a.D);
            }
        }
    }
}

// LH lanes to a head, eight features to a lane; a lane group takes a token (its angles serve all heads) or, where tokens are
// few, a part of its heads.
template <typename T, int LH, int ROT, bool WEIGHTS>
__global__ void __launch_bounds__(256, XNF) qk_norm_fwd_kernel(NormArgs a)
{
    pdl_wait();
    constexpr int U = 4;
    const long long item = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / LH;
    const int f0 = (threadIdx.x & (LH - 1)) * 8;
    const long long token = a.parts ? item / a.parts : item;
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    const bool live = token < limit, in = f0 < a.D;
    Turn<ROT> r;
    r.set(a, f0, ROT != NONE && live ? place_of(a, token) : 0);
    const T* q = static_cast<const T*>(a.q) + token * a.q_row + f0;
    const T* k = static_cast<const T*>(a.k) + token * a.k_row + f0;
    T* qo = static_cast<T*>(a.qo) + (size_t)token * a.Hq * a.D + f0;
    T* ko = static_cast<T*>(a.ko) + (size_t)token * a.Hk * a.D + f0;
    Weight<WEIGHTS> w;
    if (!a.parts) {
        w.load(a.qw, f0, in);
        norm_heads<T, LH, ROT, WEIGHTS, U>(a, r, w, q, qo, f0, live && in ? a.Hq : 0, a.Hq);
        w.load(a.kw, f0, in);
        norm_heads<T, LH, ROT, WEIGHTS, U>(a, r, w, k, ko, f0, live && in ? a.Hk : 0, a.Hk);
    } else {
        const int part = (int)(item % a.parts);
        const bool isq = part < a.q_parts;
        const int h0 = (isq ? part : part - a.q_parts) * a.heads;
        w.load(isq ? a.qw : a.kw, f0, in);
        norm_heads<T, LH, ROT, WEIGHTS, U>(a, r, w, (isq ? q : k) + (size_t)h0 * a.D, (isq ? qo : ko) + (size_t)h0 * a.D, f0,
                                           live && in ? min((isq ? a.Hq : a.Hk) - h0, a.heads) : 0, a.heads);
    }
}

// Gradients of n heads: with dv = Rot^-1 dy, dw = sum dv u, du = dv w, dx = r (du - u <du, u> share).
template <typename T, int LH, int ROT, bool WEIGHTS, int U>
__device__ __forceinline__ void norm_heads_bwd(const NormArgs& a, const Turn<ROT>& r, const Weight<WEIGHTS>& w, F<2> (&dw)[4], const T* in,
                                               const T* dy, T* dx, int f0, int n, int trips)
{
    using Row = Channels<T, 8>;
    for (int h = 0; h < trips; h += U) {
        Row raw[U], graw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = h + u < n ? Row::load(in + (size_t)(h + u) * a.D) : Row::zero();
            graw[u] = h + u < n ? Row::load(dy + (size_t)(h + u) * a.D) : Row::zero();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            F<2> x[4], g[4], ss = all<2>(0.f), dot = all<2>(0.f);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                x[q] = raw[u].get(q);
                g[q] = graw[u].get(q);
                ss = fma(x[q], x[q], ss);
            }
            turn<ROT, true, LH>(r, f0, a.R, g);
            F<2> du[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                du[q] = w.times(q, g[q]);
                dot = fma(du[q], x[q], dot);
            }
            const float m = rsqrtf(fmaf(group_sum<LH>(ss.x[0] + ss.x[1]), a.share, a.eps));
            const float t = group_sum<LH>(dot.x[0] + dot.x[1]) * m * m * a.share;
            Row y;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (WEIGHTS) dw[q] = fma(mul(g[q], x[q]), all<2>(m), dw[q]);
                y.set(q, mul(fma(x[q], all<2>(-t), du[q]), all<2>(m)));
            }
            if (h + u < n) y.store(dx + (size_t)(h + u) * a.D);
        }
    }
}

// A lane group walks over tokens (or parts of them) and keeps the sums of its eight features for queries and for keys; the
// CTA adds its groups in order.
template <typename T, int LH, int ROT, bool WEIGHTS>
__global__ void __launch_bounds__(256, XNB) qk_norm_bwd_kernel(NormArgs a)
{
    constexpr int U = 2, GROUPS = 256 / LH;
    __shared__ float sums[WEIGHTS ? GROUPS : 1][2][LH * 8];
    pdl_wait();
    const int lane = threadIdx.x & (LH - 1), group = threadIdx.x / LH, f0 = lane * 8;
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    const bool in = f0 < a.D;
    Weight<WEIGHTS> wq, wk;
    wq.load(a.qw, f0, in);
    wk.load(a.kw, f0, in);
    F<2> dwq[4], dwk[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) dwq[q] = dwk[q] = all<2>(0.f);
    const int parts = a.parts ? a.parts : 1;
    const long long items = a.tokens * parts;
    for (long long first = (long long)blockIdx.x * GROUPS; first < items; first += (long long)gridDim.x * GROUPS) {
        const long long item = first + group, token = item / parts;
        const bool live = token < limit && in;
        Turn<ROT> r;
        r.set(a, f0, ROT != NONE && token < limit ? place_of(a, token) : 0);
        const T* q = static_cast<const T*>(a.q) + token * a.q_row + f0;
        const T* k = static_cast<const T*>(a.k) + token * a.k_row + f0;
        const T* dqo = static_cast<const T*>(a.dqo) + (size_t)token * a.Hq * a.D + f0;
        const T* dko = static_cast<const T*>(a.dko) + (size_t)token * a.Hk * a.D + f0;
        T* dq = static_cast<T*>(a.dq) + token * a.dq_row + f0;
        T* dk = static_cast<T*>(a.dk) + token * a.dk_row + f0;
        if (!a.parts) {
            norm_heads_bwd<T, LH, ROT, WEIGHTS, U>(a, r, wq, dwq, q, dqo, dq, f0, live ? a.Hq : 0, a.Hq);
            norm_heads_bwd<T, LH, ROT, WEIGHTS, U>(a, r, wk, dwk, k, dko, dk, f0, live ? a.Hk : 0, a.Hk);
        } else {
            const int part = (int)(item % parts);
            const bool isq = part < a.q_parts;
            const int h0 = (isq ? part : part - a.q_parts) * a.heads;
            const size_t off = (size_t)h0 * a.D;
            Weight<WEIGHTS> w = isq ? wq : wk;
            F<2> dw[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) dw[j] = all<2>(0.f);
            norm_heads_bwd<T, LH, ROT, WEIGHTS, U>(a, r, w, dw, (isq ? q : k) + off, (isq ? dqo : dko) + off, (isq ? dq : dk) + off, f0,
                                                   live ? min((isq ? a.Hq : a.Hk) - h0, a.heads) : 0, a.heads);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dwq[j] = isq ? add(dwq[j], dw[j]) : dwq[j];
                dwk[j] = isq ? dwk[j] : add(dwk[j], dw[j]);
            }
        }
    }
    if constexpr (WEIGHTS) {
        if (!a.partial) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sums[group][0][f0 + j] = dwq[j / 2].x[j % 2];
            sums[group][1][f0 + j] = dwk[j / 2].x[j % 2];
        }
        __syncthreads();
        for (int m = threadIdx.x; m < 2 * a.D; m += 256) {
            float v = 0.f;
#pragma unroll
            for (int s = 0; s < GROUPS; ++s) v += sums[s][m / a.D][m % a.D];
            a.partial[(size_t)blockIdx.x * 2 * a.D + m] = v;
        }
    }
}

int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }

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
    // tokens for 512 lanes of each SM: whole ones; else parts of up to eight heads, and of one where there are few of those
    const long long groups = 148ll * 512 / lanes_of(p.D);
    a.heads = 8;
    a.parts = 0;
    if (a.tokens < groups) {
        while (a.heads > 1 && a.tokens * (div_up(p.Hq, a.heads) + div_up(p.Hk, a.heads)) < groups) a.heads /= 2;
        a.q_parts = div_up(p.Hq, a.heads);
        a.parts = a.q_parts + div_up(p.Hk, a.heads);
    }
    return a;
}

// CTAs of the backward: two for each SM, and every lane group the same number of items.
int bwd_blocks(const NormArgs& a, int LH)
{
    const long long need = (a.tokens * (a.parts ? a.parts : 1) + 256 / LH - 1) / (256 / LH), most = 148 * XNG;
    const long long rounds = (need + most - 1) / most;
    return (int)((need + rounds - 1) / rounds);
}

template <typename F> int by_type(const osdn_qk_norm_params& p, bool weights, F f)   // f(element, lanes to a head, rotation, weights)
{
    auto weight = [&](auto e, auto lh, auto rot) { return weights ? f(e, lh, rot, std::true_type{}) : f(e, lh, rot, std::false_type{}); };
    auto rot = [&](auto e, auto lh) {
        if (p.rot_dim == 0) return weight(e, lh, std::integral_constant<int, NONE>{});
        if (p.rot_layout == OSDN_ROT_HALF) return weight(e, lh, std::integral_constant<int, HALF>{});
        return weight(e, lh, std::integral_constant<int, PAIRS>{});
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
    const int n = by_type(p, qw || kw, [&](auto e, auto lh, auto rot, auto weights) {
        constexpr int LH = decltype(lh)::value, ROT = decltype(rot)::value;
        const unsigned grid = div_up(a.tokens * (a.parts ? a.parts : 1), 256 / LH);
        return launch_after(qk_norm_fwd_kernel<decltype(e), LH, ROT, decltype(weights)::value>, dim3(grid), dim3(256), 0, st, a) ? 1 : -1;
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
    int n = by_type(p, qw || kw, [&](auto e, auto lh, auto rot, auto weights) {
        constexpr int LH = decltype(lh)::value, ROT = decltype(rot)::value;
        const int blocks = bwd_blocks(a, LH);
        if (!launch_after(qk_norm_bwd_kernel<decltype(e), LH, ROT, decltype(weights)::value>, dim3(blocks), dim3(256), 0, st, a)) return -1;
        if (!a.partial) return 1;
        stage_mark(st, "qk_norm_sums");
        return launch_sum_rows(a.partial, blocks, p.D, 1, 2 * p.D, dqw, dkw, st) ? 2 : -1;
    });
    stage_end(st);
    return n;
}

}  // namespace osdn
