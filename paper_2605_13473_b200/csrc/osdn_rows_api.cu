// C ABI of the operators on rows of channels: argument validation before anything is launched.
#include <cmath>

#include "osdn_rows.cuh"

using namespace osdn;

namespace {

bool aligned(const void* const* ptrs, int n)
{
    for (int i = 0; i < n; ++i)
        if (reinterpret_cast<uintptr_t>(ptrs[i]) & 15u) return false;
    return true;
}

constexpr long long MAX_CHANNELS = (1ll << 31) - 1024;   // the kernels' channel blocks end below 2^31

int validate_batch(int B, int T, long long C, int io, int nseq, const int32_t* cu)
{
    if (io != OSDN_FP32 && io != OSDN_BF16) return OSDN_INVALID_ARG;
    if (B <= 0 || nseq < 0) return OSDN_INVALID_ARG;
    if (nseq > 0 && (B != 1 || !cu)) return OSDN_INVALID_ARG;
    if (T <= 0 || C <= 0 || C > MAX_CHANNELS) return OSDN_UNSUPPORTED_SHAPE;
    const double tokens = (double)B * T;
    if (tokens > 1.0e9 || tokens * (double)C > 2.0e10) return OSDN_UNSUPPORTED_SHAPE;
    if ((double)(nseq > 0 ? nseq : B) * (double)C > 2.0e10) return OSDN_UNSUPPORTED_SHAPE;
    return OSDN_OK;
}

int validate(const osdn_scan_params* p)
{
    if (!p) return OSDN_INVALID_ARG;
    if (p->input_gate != OSDN_INPUT_PLAIN && p->input_gate != OSDN_INPUT_COMPLEMENT) return OSDN_INVALID_ARG;
    return validate_batch(p->B, p->T, p->C, p->io_dtype, p->nseq, p->cu_seqlens);
}

int validate(const osdn_conv_params* p)
{
    if (!p) return OSDN_INVALID_ARG;
    if (p->activation != OSDN_ACT_NONE && p->activation != OSDN_ACT_SILU) return OSDN_INVALID_ARG;
    if (p->W < 2 || p->W > 4) return OSDN_UNSUPPORTED_SHAPE;
    return validate_batch(p->B, p->T, p->C, p->io_dtype, p->nseq, p->cu_seqlens);
}

bool row_ok(long long row, long long width, int io)
{
    if (row == 0) return true;
    const int unit = io == OSDN_BF16 ? 8 : 4;   // elements of 16 bytes
    return row >= width && row % unit == 0 && row <= (1ll << 31);
}

int validate(const osdn_qk_norm_params* p)
{
    if (!p) return OSDN_INVALID_ARG;
    if (p->norm != OSDN_NORM_L2 && p->norm != OSDN_NORM_RMS) return OSDN_INVALID_ARG;
    if (p->rot_layout != OSDN_ROT_HALF && p->rot_layout != OSDN_ROT_PAIRS) return OSDN_INVALID_ARG;
    if (p->Hq <= 0 || p->Hk <= 0 || p->Hq > (1 << 20) || p->Hk > (1 << 20)) return OSDN_INVALID_ARG;
    if (!(p->eps > 0.f) || !std::isfinite(p->eps)) return OSDN_INVALID_ARG;
    if (p->D < 8 || p->D > 256 || p->D % 8) return OSDN_UNSUPPORTED_SHAPE;
    if (p->rot_dim < 0 || p->rot_dim > p->D || p->rot_dim % 16) return OSDN_UNSUPPORTED_SHAPE;
    const int rc = validate_batch(p->B, p->T, ((long long)p->Hq + p->Hk) * p->D, p->io_dtype, p->nseq, p->cu_seqlens);
    if (rc != OSDN_OK) return rc;
    const long long wq = (long long)p->Hq * p->D, wk = (long long)p->Hk * p->D;
    if (!row_ok(p->q_row, wq, p->io_dtype) || !row_ok(p->dq_row, wq, p->io_dtype) || !row_ok(p->k_row, wk, p->io_dtype) ||
        !row_ok(p->dk_row, wk, p->io_dtype))
        return OSDN_INVALID_ARG;
    return OSDN_OK;
}

int done(int launches)
{
    if (launches < 0) return OSDN_CUDA_ERROR;
    last_launches() = launches;
    return OSDN_OK;
}

}  // namespace

extern "C" {

size_t osdn_scan_workspace_bytes(const osdn_scan_params* p) { return validate(p) == OSDN_OK ? scan_workspace(*p) : 0; }

int osdn_scan_fwd(const osdn_scan_params* p, const void* x, const float* gate, const float* init_state, void* out,
                  float* final_state, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    const bool save = (p->flags & OSDN_FLAG_SAVE_RESIDUALS) != 0;
    if (!x || !gate || !out || (save && !workspace)) return OSDN_INVALID_ARG;
    const void* ptrs[] = {x, gate, init_state, out, final_state, workspace};
    if (!aligned(ptrs, 6)) return OSDN_MISALIGNED;
    if (save && workspace_bytes < scan_workspace(*p)) return OSDN_WORKSPACE_TOO_SMALL;
    return done(scan_forward(*p, x, gate, init_state, out, final_state, save ? workspace : nullptr,
                             static_cast<cudaStream_t>(cuda_stream)));
}

int osdn_scan_bwd(const osdn_scan_params* p, const void* x, const float* gate, const float* init_state, const void* dout,
                  const float* dfinal_state, void* dx, float* dgate, float* dinit_state, void* workspace,
                  size_t workspace_bytes, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (!x || !gate || !dout || !dx || !dgate || !workspace) return OSDN_INVALID_ARG;
    const void* ptrs[] = {x, gate, init_state, dout, dfinal_state, dx, dgate, dinit_state, workspace};
    if (!aligned(ptrs, 9)) return OSDN_MISALIGNED;
    if (workspace_bytes < scan_workspace(*p)) return OSDN_WORKSPACE_TOO_SMALL;
    return done(scan_backward(*p, x, gate, init_state, dout, dfinal_state, dx, dgate, dinit_state, workspace,
                              static_cast<cudaStream_t>(cuda_stream)));
}

int osdn_scan_step(const osdn_scan_params* p, const void* x, const float* gate, float* state, void* out, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (p->nseq != 0) return OSDN_INVALID_ARG;   // a dense [B, T, C] block of new tokens
    if (!x || !gate || !state || !out) return OSDN_INVALID_ARG;
    const void* ptrs[] = {x, gate, state, out};
    if (!aligned(ptrs, 4)) return OSDN_MISALIGNED;
    return done(scan_step(*p, x, gate, state, out, static_cast<cudaStream_t>(cuda_stream)));
}

size_t osdn_short_conv_workspace_bytes(const osdn_conv_params* p) { return validate(p) == OSDN_OK ? conv_workspace(*p) : 0; }

int osdn_short_conv_fwd(const osdn_conv_params* p, const void* x, const float* weight, const float* bias,
                        const void* init_state, void* out, void* final_state, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (!x || !weight || !out) return OSDN_INVALID_ARG;
    const void* ptrs[] = {x, weight, bias, init_state, out, final_state};
    if (!aligned(ptrs, 6)) return OSDN_MISALIGNED;
    return done(conv_forward(*p, x, weight, bias, init_state, out, final_state, static_cast<cudaStream_t>(cuda_stream)));
}

int osdn_short_conv_bwd(const osdn_conv_params* p, const void* x, const float* weight, const float* bias,
                        const void* init_state, const void* dout, const void* dfinal_state, void* dx, float* dweight,
                        float* dbias, void* dinit_state, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (!x || !weight || !dout || !dx || !dweight || !workspace) return OSDN_INVALID_ARG;
    const void* ptrs[] = {x, weight, bias, init_state, dout, dfinal_state, dx, dweight, dbias, dinit_state, workspace};
    if (!aligned(ptrs, 11)) return OSDN_MISALIGNED;
    if (workspace_bytes < conv_workspace(*p)) return OSDN_WORKSPACE_TOO_SMALL;
    return done(conv_backward(*p, x, weight, bias, init_state, dout, dfinal_state, dx, dweight, dbias, dinit_state, workspace,
                              static_cast<cudaStream_t>(cuda_stream)));
}

int osdn_short_conv_step(const osdn_conv_params* p, const void* x, const float* weight, const float* bias, void* state,
                         void* out, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (p->nseq != 0) return OSDN_INVALID_ARG;
    if (!x || !weight || !state || !out) return OSDN_INVALID_ARG;
    const void* ptrs[] = {x, weight, bias, state, out};
    if (!aligned(ptrs, 5)) return OSDN_MISALIGNED;
    return done(conv_step(*p, x, weight, bias, state, out, static_cast<cudaStream_t>(cuda_stream)));
}

size_t osdn_qk_norm_workspace_bytes(const osdn_qk_norm_params* p)
{
    return validate(p) == OSDN_OK ? qk_norm_workspace(*p) : 0;
}

int osdn_qk_norm_fwd(const osdn_qk_norm_params* p, const void* q, const void* k, const float* q_weight,
                     const float* k_weight, const double* inv_freq, const int32_t* positions, void* q_out, void* k_out,
                     void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (!q || !k || !q_out || !k_out || (p->rot_dim > 0 && !inv_freq)) return OSDN_INVALID_ARG;
    const void* ptrs[] = {q, k, q_weight, k_weight, inv_freq, positions, q_out, k_out};
    if (!aligned(ptrs, 8)) return OSDN_MISALIGNED;
    return done(qk_norm_forward(*p, q, k, q_weight, k_weight, inv_freq, positions, q_out, k_out,
                                static_cast<cudaStream_t>(cuda_stream)));
}

int osdn_qk_norm_bwd(const osdn_qk_norm_params* p, const void* q, const void* k, const float* q_weight,
                     const float* k_weight, const double* inv_freq, const int32_t* positions, const void* dq_out,
                     const void* dk_out, void* dq, void* dk, float* dq_weight, float* dk_weight, void* workspace,
                     size_t workspace_bytes, void* cuda_stream)
{
    last_launches() = 0;
    const int rc = validate(p);
    if (rc != OSDN_OK) return rc;
    if (!q || !k || !dq_out || !dk_out || !dq || !dk || (p->rot_dim > 0 && !inv_freq)) return OSDN_INVALID_ARG;
    if ((dq_weight && !q_weight) || (dk_weight && !k_weight)) return OSDN_INVALID_ARG;
    const bool sums = dq_weight || dk_weight;
    if (sums && !workspace) return OSDN_INVALID_ARG;
    const void* ptrs[] = {q, k, q_weight, k_weight, inv_freq, positions, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace};
    if (!aligned(ptrs, 13)) return OSDN_MISALIGNED;
    if (sums && workspace_bytes < qk_norm_workspace(*p)) return OSDN_WORKSPACE_TOO_SMALL;
    return done(qk_norm_backward(*p, q, k, q_weight, k_weight, inv_freq, positions, dq_out, dk_out, dq, dk, dq_weight, dk_weight,
                                 workspace, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
