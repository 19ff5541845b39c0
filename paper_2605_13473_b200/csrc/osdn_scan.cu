// Gated linear recurrence h_t = a_t h_{t-1} + b_t, a_t = exp(g_t), channel by channel: forward, backward, decode step.
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
    float* saved;    // [tiles, C] state in front of every TILE-th token
    Rows rows;
    int C, tiles;    // tiles: of a dense sequence, or of all packed rows
};

template <typename T, bool COMP>
__global__ void scan_fwd_simple_kernel(ScanArgs a)
{
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (long long)a.rows.S * a.C) return;
    const int s = (int)(i / a.C), c = (int)(i % a.C);
    const bool packed = a.rows.cu != nullptr;
    const int end = packed ? rows_end(a.rows) : a.rows.T;
    const int t0 = packed ? min(max(a.rows.cu[s], 0), end) : 0, t1 = packed ? min(max(a.rows.cu[s + 1], t0), end) : a.rows.T;
    const size_t base = packed ? 0 : (size_t)s * a.rows.T;
    const size_t tile0 = packed ? 0 : (size_t)s * a.tiles;
    float h = a.init ? a.init[i] : 0.f;
    for (int t = t0; t < t1; ++t) {
        if (a.saved && t % TILE == 0) a.saved[(tile0 + t / TILE) * a.C + c] = h;
        const size_t at = (base + t) * a.C + c;
        const Decay d = Decay::of(a.gate[at]);
        const float x = ldf(static_cast<const T*>(a.x) + at);
        h = d.step(h, COMP ? d.complement() * x : x);
        if (a.out) stf(static_cast<T*>(a.out) + at, h);
    }
    if (a.fin) a.fin[i] = h;
}

template <typename T, bool COMP>
__global__ void scan_bwd_simple_kernel(ScanArgs a)
{
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (long long)a.rows.S * a.C) return;
    const int s = (int)(i / a.C), c = (int)(i % a.C);
    const bool packed = a.rows.cu != nullptr;
    const int end = packed ? rows_end(a.rows) : a.rows.T;
    const int t0 = packed ? min(max(a.rows.cu[s], 0), end) : 0, t1 = packed ? min(max(a.rows.cu[s + 1], t0), end) : a.rows.T;
    const size_t base = packed ? 0 : (size_t)s * a.rows.T;
    const size_t tile0 = packed ? 0 : (size_t)s * a.tiles;
    float before[TILE];
    float e = a.dfin ? a.dfin[i] : 0.f;   // a_{t+1} dh_{t+1}
    for (int hi = t1; hi > t0;) {
        const int lo = max(t0, (hi - 1) / TILE * TILE);
        float h = lo % TILE == 0 ? a.saved[(tile0 + lo / TILE) * a.C + c] : a.init ? a.init[i] : 0.f;
        for (int t = lo; t < hi; ++t) {
            before[t - lo] = h;
            const size_t at = (base + t) * a.C + c;
            const Decay d = Decay::of(a.gate[at]);
            const float x = ldf(static_cast<const T*>(a.x) + at);
            h = d.step(h, COMP ? d.complement() * x : x);
        }
        for (int t = hi - 1; t >= lo; --t) {
            const size_t at = (base + t) * a.C + c;
            const Decay d = Decay::of(a.gate[at]);
            const float dh = ldf(static_cast<const T*>(a.dout) + at) + e;
            e = d.times(dh);
            const float x = ldf(static_cast<const T*>(a.x) + at);
            a.dgate[at] = (COMP ? before[t - lo] - x : before[t - lo]) * e;
            stf(static_cast<T*>(a.dx) + at, COMP ? d.complement() * dh : dh);
        }
        hi = lo;
    }
    if (a.dinit) a.dinit[i] = e;
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

ScanArgs make_args(const osdn_scan_params& p)
{
    ScanArgs a{};
    a.rows = {p.nseq > 0 ? p.cu_seqlens : nullptr, p.nseq > 0 ? p.nseq : p.B, p.T};
    a.C = p.C;
    a.tiles = div_up(p.T, TILE);
    return a;
}

template <typename T, bool COMP> bool launch_forward(const ScanArgs& a, cudaStream_t st)
{
    const unsigned grid = div_up((long long)a.rows.S * a.C, 128);
    scan_fwd_simple_kernel<T, COMP><<<grid, 128, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess;
}

template <typename T, bool COMP> int run_backward(ScanArgs a, bool saved, cudaStream_t st)
{
    int n = 0;
    if (!saved) {
        ScanArgs f = a;
        f.out = nullptr; f.fin = nullptr;
        if (!launch_forward<T, COMP>(f, st)) return -1;
        ++n;
    }
    const unsigned grid = div_up((long long)a.rows.S * a.C, 128);
    scan_bwd_simple_kernel<T, COMP><<<grid, 128, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? n + 1 : -1;
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
    return align_up((size_t)(p.nseq > 0 ? 1 : p.B) * div_up(p.T, TILE) * p.C * 4, 256);
}

int scan_forward(const osdn_scan_params& p, const void* x, const float* gate, const float* init, void* out, float* fin,
                 void* ws, cudaStream_t st)
{
    ScanArgs a = make_args(p);
    a.x = x; a.gate = gate; a.init = init; a.out = out; a.fin = fin;
    a.saved = static_cast<float*>(ws);
    stage_mark(st, "scan_fwd");
    const int n = by_type(p, [&](auto e, auto comp) { return launch_forward<decltype(e), decltype(comp)::value>(a, st) ? 1 : -1; });
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
    const int n = by_type(p, [&](auto e, auto comp) { return run_backward<decltype(e), decltype(comp)::value>(a, saved, st); });
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
