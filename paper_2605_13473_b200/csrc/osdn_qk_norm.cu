// Norms of queries and keys, head by head, with the rotation by the position in the same pass: forward and backward.
#include "osdn_rows.cuh"

namespace osdn {
namespace {

constexpr int BWD_CTAS = 2, BWD_DEPTH = 4;   // CTAs to an SM; heads on their way
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
    __device__ __forceinline__ static void angle(const NormArgs& a, int n, int pos, float& s, float& c)
    {
        double t = pos * (a.inv_freq[n] * 0.15915494309189535);   // turns; 1 / (2 pi)
        t -= rint(t);
        sincospif(2.f * (float)t, &s, &c);
    }
    template <int LH> __device__ __forceinline__ void set(const NormArgs& a, int f0, int pos)   // by whole warps
    {
        const bool in = f0 < a.R;
        if constexpr (ROT == HALF) {   // the two lanes of a pair work out four pairs each
            const bool second = f0 >= a.R / 2;
            const int n0 = second ? f0 - a.R / 2 + 4 : f0, lane = threadIdx.x & (LH - 1);
            const int other = !in ? lane : second ? lane - a.R / 16 : lane + a.R / 16;
            float mc[4], ms[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mc[j] = 1.f;
                ms[j] = 0.f;
                if (in) angle(a, n0 + j, pos, ms[j], mc[j]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float oc = __shfl_sync(0xffffffffu, mc[j], other, LH), os = __shfl_sync(0xffffffffu, ms[j], other, LH);
                c[j] = second ? oc : mc[j];
                c[j + 4] = second ? mc[j] : oc;
                s[j] = second ? -os : ms[j];   // x cos - other sin becomes x cos + other sin
                s[j + 4] = second ? -ms[j] : os;
            }
        } else if constexpr (ROT == PAIRS) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = 1.f;
                s[j] = 0.f;
                if (in) angle(a, f0 / 2 + j, pos, s[j], c[j]);
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

// One head: its norm, weight and rotation.
template <typename T, int LH, int ROT, bool WEIGHTS>
__device__ __forceinline__ Channels<T, 8> norm_head(const NormArgs& a, const Turn<ROT>& r, const Weight<WEIGHTS>& w, int f0, const Channels<T, 8>& raw)
{
    F<2> x[4], ss = all<2>(0.f);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        x[q] = raw.get(q);
        ss = fma(x[q], x[q], ss);
    }
    const float m = rsqrtf(fmaf(group_sum<LH>(ss.x[0] + ss.x[1]), a.share, a.eps));
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = w.times(q, mul(x[q], all<2>(m)));
    turn<ROT, false, LH>(r, f0, a.R, x);
    Channels<T, 8> y;
#pragma unroll
    for (int q = 0; q < 4; ++q) y.set(q, x[q]);
    return y;
}

// Its gradient: with dv = Rot^-1 dy, dw = sum dv u, du = dv w, dx = r (du - u <du, u> share).
template <typename T, int LH, int ROT, bool WEIGHTS>
__device__ __forceinline__ Channels<T, 8> norm_head_bwd(const NormArgs& a, const Turn<ROT>& r, const Weight<WEIGHTS>& w, F<2> (&dw)[4], int f0,
                                                        const Channels<T, 8>& raw, const Channels<T, 8>& graw)
{
    F<2> x[4], g[4], ss = all<2>(0.f), dot = all<2>(0.f);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        x[q] = raw.get(q);
        g[q] = graw.get(q);
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
    Channels<T, 8> y;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (WEIGHTS) dw[q] = fma(mul(g[q], x[q]), all<2>(m), dw[q]);
        y.set(q, mul(fma(x[q], all<2>(-t), du[q]), all<2>(m)));
    }
    return y;
}

// LH lanes to a head, eight features to a lane.  Few tokens: a lane group takes a part of a token's heads, U loads on their way.
template <typename T, int LH, int ROT, bool WEIGHTS>
__global__ void __launch_bounds__(256) qk_norm_fwd_parts_kernel(NormArgs a)
{
    pdl_wait();
    constexpr int U = 2;
    using Row = Channels<T, 8>;
    const long long item = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / LH, token = item / a.parts;
    const int f0 = (threadIdx.x & (LH - 1)) * 8, part = (int)(item % a.parts);
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    const bool live = token < limit, in = f0 < a.D, isq = part < a.q_parts;
    const int h0 = (isq ? part : part - a.q_parts) * a.heads, H = isq ? a.Hq : a.Hk, n = live && in ? min(H - h0, a.heads) : 0;
    const T* from = (isq ? static_cast<const T*>(a.q) + token * a.q_row : static_cast<const T*>(a.k) + token * a.k_row) + (size_t)h0 * a.D + f0;
    T* to = static_cast<T*>(isq ? a.qo : a.ko) + ((size_t)token * H + h0) * a.D + f0;
    Turn<ROT> r;
    r.template set<LH>(a, f0, ROT != NONE && live ? place_of(a, token) : 0);
    Weight<WEIGHTS> w;
    w.load(isq ? a.qw : a.kw, f0, in);
    for (int h = 0; h < a.heads; h += U) {   // the same for every lane of a warp
        Row raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = h + u < n ? Row::load(from + (size_t)(h + u) * a.D) : Row::zero();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Row y = norm_head<T, LH, ROT, WEIGHTS>(a, r, w, f0, raw[u]);
            if (h + u < n) y.store(to + (size_t)(h + u) * a.D);
        }
    }
}

// Many tokens: a lane group takes whole ones, whose angles serve all their heads.  Four heads' loads on their way in registers
// (through shared memory, as the backward has it, 4 x 4096 tokens of 32 heads took 8 % longer).  55 us there with rotated halves,
// 74 % of the bytes' rate, and 47 with interleaved pairs: bound by the latency of the loads and of the halves' shuffles.
template <typename T, int LH, int ROT, bool WEIGHTS>
__global__ void __launch_bounds__(256, 4) qk_norm_fwd_kernel(NormArgs a)
{
    pdl_wait();
    constexpr int U = 4;
    using Row = Channels<T, 8>;
    const long long token = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / LH;
    const int f0 = (threadIdx.x & (LH - 1)) * 8;
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    const bool in = f0 < a.D, live = token < limit;
    Turn<ROT> r;
    r.template set<LH>(a, f0, ROT != NONE && live ? place_of(a, token) : 0);
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const int H = part ? a.Hk : a.Hq, n = live && in ? H : 0;
        const T* from = (part ? static_cast<const T*>(a.k) + token * a.k_row : static_cast<const T*>(a.q) + token * a.q_row) + f0;
        T* to = static_cast<T*>(part ? a.ko : a.qo) + (size_t)token * H * a.D + f0;
        Weight<WEIGHTS> w;
        w.load(part ? a.kw : a.qw, f0, in);
        for (int h = 0; h < H; h += U) {
            Row raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = h + u < n ? Row::load(from + (size_t)(h + u) * a.D) : Row::zero();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (h + u >= H) break;
                const Row y = norm_head<T, LH, ROT, WEIGHTS>(a, r, w, f0, raw[u]);
                if (h + u < n) y.store(to + (size_t)(h + u) * a.D);
            }
        }
    }
}

// What a lane reads of the heads of its tokens (one every `stride`), queries before keys, TENSORS of them side by side: copied
// to the lane's own places of shared memory DEPTH heads ahead, since the arithmetic of a head is short against memory's latency
// (backward of 4 x 4096 tokens, 32 rotated heads: with loads to registers, two heads at a time, 97 us, so 67).
template <typename T, int TENSORS, int DEPTH_> struct Ahead {
    static constexpr int DEPTH = DEPTH_, PIECES = (int)sizeof(T) / 2;   // of 16 bytes: eight features
    const T *q[TENSORS], *k[TENSORS], *src[TENSORS];
    long long q_row[TENSORS], k_row[TENSORS], token, stride, limit;
    char* place;
    int head, slot;
    bool in;
    __device__ __forceinline__ char* at(int s, int t) const { return place + (size_t)((s * TENSORS + t) * PIECES) * 256 * 16; }
    __device__ __forceinline__ void ask(const NormArgs& a)   // the next head into `slot`, which has been read
    {
        const bool real = in && token < limit;
#pragma unroll
        for (int t = 0; t < TENSORS; ++t)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) copy_async16(at(slot, t) + p * 256 * 16, real ? src[t] + p * 8 / PIECES : q[t], real);
        copies_end();
        if (++head == a.Hq + a.Hk) {
            head = 0;
            token += stride;
#pragma unroll
            for (int t = 0; t < TENSORS; ++t) src[t] = q[t] + token * q_row[t];
        } else if (head == a.Hq) {
#pragma unroll
            for (int t = 0; t < TENSORS; ++t) src[t] = k[t] + token * k_row[t];
        } else {
#pragma unroll
            for (int t = 0; t < TENSORS; ++t) src[t] += a.D;
        }
    }
    __device__ __forceinline__ void start(const NormArgs& a)
    {
        head = 0;
#pragma unroll
        for (int t = 0; t < TENSORS; ++t) src[t] = q[t] + token * q_row[t];
        for (slot = 0; slot < DEPTH; ++slot) ask(a);
        slot = 0;
    }
    __device__ __forceinline__ void read(Channels<T, 8> (&raw)[TENSORS]) const
    {
        copies_wait<DEPTH - 1>();
#pragma unroll
        for (int t = 0; t < TENSORS; ++t)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const uint4 v = *reinterpret_cast<const uint4*>(at(slot, t) + p * 256 * 16);
                raw[t].w[4 * p] = v.x; raw[t].w[4 * p + 1] = v.y; raw[t].w[4 * p + 2] = v.z; raw[t].w[4 * p + 3] = v.w;
            }
    }
    // Behind the store of what was made of the last read: nothing of it is still on its way out of the place.
    __device__ __forceinline__ void refill(const NormArgs& a)
    {
        ask(a);
        slot = slot + 1 < DEPTH ? slot + 1 : 0;
    }
};

// The CTA's sums of the weights' gradients, its lane groups in order.
template <int LH> __device__ __forceinline__ void add_groups(const NormArgs& a, float* sums, const F<2> (&dwq)[4], const F<2> (&dwk)[4])
{
    constexpr int GROUPS = 256 / LH, WIDTH = LH * 8;   // sums: [GROUPS][2][WIDTH]
    const int f0 = (threadIdx.x & (LH - 1)) * 8, group = threadIdx.x / LH;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sums[(group * 2) * WIDTH + f0 + j] = dwq[j / 2].x[j % 2];
        sums[(group * 2 + 1) * WIDTH + f0 + j] = dwk[j / 2].x[j % 2];
    }
    __syncthreads();
    for (int m = threadIdx.x; m < 2 * a.D; m += 256) {
        float v = 0.f;
#pragma unroll
        for (int s = 0; s < GROUPS; ++s) v += sums[(s * 2 + m / a.D) * WIDTH + m % a.D];
        a.partial[(size_t)blockIdx.x * 2 * a.D + m] = v;
    }
}

template <typename T, int LH, int ROT, bool WEIGHTS>
__global__ void __launch_bounds__(256, BWD_CTAS) qk_norm_bwd_kernel(NormArgs a)
{
    extern __shared__ __align__(16) char shared[];
    pdl_wait();
    constexpr int GROUPS = 256 / LH;
    const int f0 = (threadIdx.x & (LH - 1)) * 8;
    Ahead<T, 2, BWD_DEPTH> rows;
    rows.q[0] = static_cast<const T*>(a.q) + f0;
    rows.k[0] = static_cast<const T*>(a.k) + f0;
    rows.q_row[0] = a.q_row;
    rows.k_row[0] = a.k_row;
    rows.q[1] = static_cast<const T*>(a.dqo) + f0;
    rows.k[1] = static_cast<const T*>(a.dko) + f0;
    rows.q_row[1] = (long long)a.Hq * a.D;
    rows.k_row[1] = (long long)a.Hk * a.D;
    rows.limit = a.rows.cu ? rows_end(a.rows) : a.tokens;
    rows.in = f0 < a.D;
    rows.stride = (long long)gridDim.x * GROUPS;
    rows.token = (long long)blockIdx.x * GROUPS + threadIdx.x / LH;
    rows.place = shared + threadIdx.x * 16;
    const long long limit = rows.limit, stride = rows.stride;
    long long token = rows.token;
    rows.start(a);
    F<2> dw[2][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) dw[0][q] = dw[1][q] = all<2>(0.f);
    for (long long first = (long long)blockIdx.x * GROUPS; first < limit; first += stride, token += stride) {
        const bool live = token < limit;
        Turn<ROT> r;
        r.template set<LH>(a, f0, ROT != NONE && live ? place_of(a, token) : 0);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int H = part ? a.Hk : a.Hq;
            T* to = part ? static_cast<T*>(a.dk) + token * a.dk_row + f0 : static_cast<T*>(a.dq) + token * a.dq_row + f0;
            Weight<WEIGHTS> w;
            w.load(part ? a.kw : a.qw, f0, rows.in);
            for (int h = 0; h < H; ++h, to += a.D) {
                Channels<T, 8> raw[2];
                rows.read(raw);
                const Channels<T, 8> y = norm_head_bwd<T, LH, ROT, WEIGHTS>(a, r, w, dw[part], f0, raw[0], raw[1]);
                if (live && rows.in) y.store(to);
                rows.refill(a);
            }
        }
    }
    if constexpr (WEIGHTS) {
        if (!a.partial) return;
        copies_wait<0>();   // nothing lands there any more
        __syncthreads();
        add_groups<LH>(a, reinterpret_cast<float*>(shared), dw[0], dw[1]);
    }
}

template <typename T, int LH, int ROT, bool WEIGHTS>
__global__ void __launch_bounds__(256) qk_norm_bwd_parts_kernel(NormArgs a)
{
    constexpr int GROUPS = 256 / LH;
    __shared__ float sums[WEIGHTS ? GROUPS * 2 * LH * 8 : 1];
    using Row = Channels<T, 8>;
    pdl_wait();
    const int f0 = (threadIdx.x & (LH - 1)) * 8, group = threadIdx.x / LH;
    const long long limit = a.rows.cu ? rows_end(a.rows) : a.tokens, items = a.tokens * a.parts;
    const bool in = f0 < a.D;
    F<2> dwq[4], dwk[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) dwq[q] = dwk[q] = all<2>(0.f);
    for (long long first = (long long)blockIdx.x * GROUPS; first < items; first += (long long)gridDim.x * GROUPS) {
        const long long item = first + group, token = item / a.parts;
        const int part = (int)(item % a.parts);
        const bool isq = part < a.q_parts, live = token < limit && in;
        const int h0 = (isq ? part : part - a.q_parts) * a.heads, H = isq ? a.Hq : a.Hk, n = live ? min(H - h0, a.heads) : 0;
        const size_t off = (size_t)h0 * a.D + f0;
        const T* from = (isq ? static_cast<const T*>(a.q) + token * a.q_row : static_cast<const T*>(a.k) + token * a.k_row) + off;
        const T* dy = static_cast<const T*>(isq ? a.dqo : a.dko) + (size_t)token * H * a.D + off;
        T* to = (isq ? static_cast<T*>(a.dq) + token * a.dq_row : static_cast<T*>(a.dk) + token * a.dk_row) + off;
        Turn<ROT> r;
        r.template set<LH>(a, f0, ROT != NONE && token < limit ? place_of(a, token) : 0);
        Weight<WEIGHTS> w;
        w.load(isq ? a.qw : a.kw, f0, in);
        F<2> dw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[j] = all<2>(0.f);
        for (int h = 0; h < a.heads; ++h) {   // the same for every lane of a warp
            const Row raw = h < n ? Row::load(from + (size_t)h * a.D) : Row::zero(), g = h < n ? Row::load(dy + (size_t)h * a.D) : Row::zero();
            const Row y = norm_head_bwd<T, LH, ROT, WEIGHTS>(a, r, w, dw, f0, raw, g);
            if (h < n) y.store(to + (size_t)h * a.D);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            dwq[j] = isq ? add(dwq[j], dw[j]) : dwq[j];
            dwk[j] = isq ? dwk[j] : add(dwk[j], dw[j]);
        }
    }
    if constexpr (WEIGHTS)
        if (a.partial) add_groups<LH>(a, sums, dwq, dwk);
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

// CTAs for `per_sm` on each SM, with the same number of items for every lane group.
int even_blocks(long long items, int LH, int per_sm)
{
    const long long need = (items + 256 / LH - 1) / (256 / LH), most = 148ll * per_sm, rounds = (need + most - 1) / most;
    return (int)((need + rounds - 1) / rounds);
}
int bwd_blocks(const NormArgs& a, int LH) { return even_blocks(a.tokens * std::max(a.parts, 1), LH, BWD_CTAS); }

template <typename K> bool set_smem(K* kernel, size_t bytes)
{
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
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
        using T = decltype(e);
        constexpr bool WEIGHTS = decltype(weights)::value;
        if (a.parts)
            return launch_after(qk_norm_fwd_parts_kernel<T, LH, ROT, WEIGHTS>, dim3(div_up(a.tokens * a.parts, 256 / LH)), dim3(256), 0, st, a) ? 1 : -1;
        return launch_after(qk_norm_fwd_kernel<T, LH, ROT, WEIGHTS>, dim3(div_up(a.tokens, 256 / LH)), dim3(256), 0, st, a) ? 1 : -1;
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
        using T = decltype(e);
        constexpr bool WEIGHTS = decltype(weights)::value;
        const auto kernel = a.parts ? qk_norm_bwd_parts_kernel<T, LH, ROT, WEIGHTS> : qk_norm_bwd_kernel<T, LH, ROT, WEIGHTS>;
        const size_t smem = a.parts ? 0 : std::max((size_t)(BWD_DEPTH * 2 * 256 * 8 * sizeof(T)), (size_t)(256 * 2 * 8 * 4));
        if (!set_smem(kernel, smem) || !launch_after(kernel, dim3(blocks), dim3(256), smem, st, a)) return -1;
        if (!a.partial) return 1;
        stage_mark(st, "qk_norm_sums");
        return launch_sum_rows(a.partial, blocks, p.D, 1, dqw, dkw, st) ? 2 : -1;
    });
    stage_end(st);
    return n;
}

}  // namespace osdn
