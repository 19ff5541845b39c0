"""B200-native OSDN layer: thin Python binding over the C ABI in ``include/osdn.h``.

The binding only marshals arguments (torch tensors -> device pointers); every step
of the layer runs in the CUDA kernels of ``libosdn.so``.  There is no CPU or eager
fallback: if the library is missing or no CUDA device is present the calls raise.

    from paper_2605_13473_b200 import osdn_fwd, osdn_bwd, osdn_precond_update

Operators beside the layer: ``osdn_scan_*`` (gated linear recurrence), ``osdn_short_conv_*`` (short causal
convolution), ``osdn_qk_norm_*`` (norms of queries and keys with the position rotation).
"""
from .binding import (  # noqa: F401
    FLAG_RESIDUALS_VALID,
    FLAG_SAVE_RESIDUALS,
    ConvParams,
    OsdnParams,
    QkNormParams,
    ScanParams,
    load_library,
    make_conv_params,
    make_params,
    make_qk_norm_params,
    make_scan_params,
    osdn_bwd,
    osdn_fwd,
    osdn_fwd_static,
    osdn_decode_step,
    osdn_precond_update,
    osdn_residual_ratio,
    osdn_qk_norm_bwd,
    osdn_qk_norm_fwd,
    osdn_qk_norm_workspace_bytes,
    osdn_scan_bwd,
    osdn_scan_fwd,
    osdn_scan_step,
    osdn_scan_workspace_bytes,
    osdn_short_conv_bwd,
    osdn_short_conv_fwd,
    osdn_short_conv_step,
    osdn_short_conv_workspace_bytes,
    osdn_step_host,
    osdn_workspace_bytes,
    osdn_host_staging_bytes,
    osdn_last_launch_count,
    osdn_read_device_status,
    status_string,
    run_inputs_fwd,
    run_inputs_bwd,
)
