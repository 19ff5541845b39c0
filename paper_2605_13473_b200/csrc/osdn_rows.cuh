// Device helpers of the operators on rows of channels: the recurrence, the convolution, the norms.
#pragma once

#include <algorithm>
#include <type_traits>

#include "osdn_common.cuh"

namespace osdn {

// Sequences of a batch of rows.  Dense: S sequences of T rows; packed (cu != nullptr): rows cu[s] .. cu[s+1]-1 of T.
struct Rows {
    const int* cu;
    int S, T;
};

// First row behind the last sequence, and never behind the tensor.
__device__ __forceinline__ int rows_end(const Rows& r) { return min(max(r.cu[r.S], 0), r.T); }

// The last sequence that begins at or before row t (packed; 0 <= t < cu[S]), so not an empty one where t lies in a sequence.
// Whatever cu holds, the result is one of 0 .. S-1.
__device__ __forceinline__ int seq_of(const Rows& r, int t)
{
    int lo = 0, hi = r.S;   // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (r.cu[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// N consecutive channels as fp32; p is aligned to their size.
template <int N> __device__ __forceinline__ void load_vec(const float* p, float (&x)[N])
{
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const float4 v = reinterpret_cast<const float4*>(p)[i];
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = p[i];
    }
}
__device__ __forceinline__ float2 bf16_pair(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pair_bf16(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <int N> __device__ __forceinline__ void load_vec(const __nv_bfloat16* p, float (&x)[N])
{
    if constexpr (N == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        const float2 a = bf16_pair(v.x), b = bf16_pair(v.y);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = __bfloat162float(p[i]);
    }
}
template <int N> __device__ __forceinline__ void store_vec(float* p, const float (&x)[N])
{
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i)
            reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = x[i];
    }
}
template <int N> __device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&x)[N])
{
    if constexpr (N == 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pair_bf16(x[0], x[1]), pair_bf16(x[2], x[3]));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = __float2bfloat16_rn(x[i]);
    }
}

// N channels at once; two go through the packed fp32 instructions.
template <int N> struct F {
    float x[N];
};
__device__ __forceinline__ unsigned long long pack(const F<2>& a)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x[0]), "f"(a.x[1]));
    return r;
}
__device__ __forceinline__ F<2> unpack(unsigned long long r)
{
    F<2> a;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a.x[0]), "=f"(a.x[1]) : "l"(r));
    return a;
}
template <int N> __device__ __forceinline__ F<N> all(float v)
{
    F<N> a;
#pragma unroll
    for (int k = 0; k < N; ++k) a.x[k] = v;
    return a;
}
template <int N> __device__ __forceinline__ F<N> fma(const F<N>& a, const F<N>& b, const F<N>& c)
{
    if constexpr (N == 2) {
        unsigned long long d;
        asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(pack(a)), "l"(pack(b)), "l"(pack(c)));
        return unpack(d);
    } else {
        return {{fmaf(a.x[0], b.x[0], c.x[0])}};
    }
}
template <int N> __device__ __forceinline__ F<N> add(const F<N>& a, const F<N>& b)
{
    if constexpr (N == 2) {
        unsigned long long d;
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(pack(a)), "l"(pack(b)));
        return unpack(d);
    } else {
        return {{a.x[0] + b.x[0]}};
    }
}
template <int N> __device__ __forceinline__ F<N> mul(const F<N>& a, const F<N>& b)
{
    if constexpr (N == 2) {
        unsigned long long d;
        asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(pack(a)), "l"(pack(b)));
        return unpack(d);
    } else {
        return {{a.x[0] * b.x[0]}};
    }
}

// N consecutive channels as they come from memory, in pairs (N = 1: alone).
template <typename T, int N> struct Channels {
    static constexpr int L = N % 2 == 0 ? 2 : 1, Q = N / L;
    static constexpr int WORDS = N * (int)sizeof(T) / 4 > 0 ? N * (int)sizeof(T) / 4 : 1;
    uint32_t w[WORDS];
    __device__ __forceinline__ static Channels zero()
    {
        Channels c;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) c.w[i] = 0;
        return c;
    }
    __device__ __forceinline__ static Channels load(const T* p)
    {
        Channels c;
        if constexpr (WORDS % 4 == 0) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const uint4 v = reinterpret_cast<const uint4*>(p)[i];
                c.w[4 * i] = v.x; c.w[4 * i + 1] = v.y; c.w[4 * i + 2] = v.z; c.w[4 * i + 3] = v.w;
            }
        } else if constexpr (WORDS == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            c.w[0] = v.x; c.w[1] = v.y;
        } else if constexpr (sizeof(T) == 2 && N == 1) {
            c.w[0] = *reinterpret_cast<const uint16_t*>(p);
        } else {
            c.w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
        return c;
    }
    __device__ __forceinline__ F<L> get(int q) const
    {
        if constexpr (sizeof(T) == 4) {
            if constexpr (L == 2) return {{__uint_as_float(w[2 * q]), __uint_as_float(w[2 * q + 1])}};
            else return {{__uint_as_float(w[q])}};
        } else {
            if constexpr (L == 2) return {{__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u)}};
            else return {{__uint_as_float(w[q] << 16)}};
        }
    }
    __device__ __forceinline__ void set(int q, const F<L>& v)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < L; ++k) w[L * q + k] = __float_as_uint(v.x[k]);
        } else if constexpr (L == 2) {
            w[q] = pair_bf16(v.x[0], v.x[1]);
        } else {
            const __nv_bfloat16 h = __float2bfloat16_rn(v.x[0]);
            w[q] = *reinterpret_cast<const uint16_t*>(&h);
        }
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (WORDS % 4 == 0) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        } else if constexpr (WORDS == 2) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else if constexpr (sizeof(T) == 2 && N == 1) {
            *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
        } else {
            *reinterpret_cast<uint32_t*>(p) = w[0];
        }
    }
};

__device__ __forceinline__ void copy_async16(void* smem, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(src),
                 "r"(real ? 16 : 0) : "memory");   // what is not there is filled with zeros
}
// Stretches of rows come in through several places of shared memory: one group of copies for each, empty ones too.
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LATER> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory"); }

inline int div_up(long long a, long long b) { return (int)((a + b - 1) / b); }

// Entry points of the kernels' files.  The number of launches, or -1 on a launch error.
int scan_forward(const osdn_scan_params& p, const void* x, const float* gate, const float* init, void* out, float* fin,
                 void* ws, cudaStream_t st);
int scan_backward(const osdn_scan_params& p, const void* x, const float* gate, const float* init, const void* dout,
                  const float* dfin, void* dx, float* dgate, float* dinit, void* ws, cudaStream_t st);
int scan_step(const osdn_scan_params& p, const void* x, const float* gate, float* state, void* out, cudaStream_t st);
size_t scan_workspace(const osdn_scan_params& p);
int conv_forward(const osdn_conv_params& p, const void* x, const float* w, const float* bias, const void* init, void* out,
                 void* fin, cudaStream_t st);
int conv_backward(const osdn_conv_params& p, const void* x, const float* w, const float* bias, const void* init,
                  const void* dout, const void* dfin, void* dx, float* dw, float* dbias, void* dinit, void* ws, cudaStream_t st);
int conv_step(const osdn_conv_params& p, const void* x, const float* w, const float* bias, void* state, void* out, cudaStream_t st);
size_t conv_workspace(const osdn_conv_params& p);
int qk_norm_forward(const osdn_qk_norm_params& p, const void* q, const void* k, const float* qw, const float* kw,
                    const double* inv_freq, const int* pos, void* qo, void* ko, cudaStream_t st);
int qk_norm_backward(const osdn_qk_norm_params& p, const void* q, const void* k, const float* qw, const float* kw,
                     const double* inv_freq, const int* pos, const void* dqo, const void* dko, void* dq, void* dk, float* dqw,
                     float* dkw, void* ws, cudaStream_t st);
size_t qk_norm_workspace(const osdn_qk_norm_params& p);

// Sums over the first axis of part [G, W + 1, C], in a fixed order: out0[c W + j] of rows j < W, out1[c] of the last; either may
// be NULL.
bool launch_sum_rows(const float* part, int G, int C, int W, float* out0, float* out1, cudaStream_t st);

// Launch count of the calling thread's last call (osdn_last_launch_count).
int& last_launches();

}  // namespace osdn
