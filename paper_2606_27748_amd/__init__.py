"""MI355X (gfx950) random-Fourier-feature linear attention (Flexformer, arXiv 2606.27748).

The computation lives in the HIP library ``libflexattn.so`` (C ABI in
include/flex.h); this package is its thin Python binding.
"""
from ._lib import (FlexError, flex_desc, make_desc, workspace_size, flex_feature_map,  # noqa: F401
                   flex_linattn_fwd, flex_linattn_prefill, flex_linattn_fwd_noalloc, flex_linattn_bwd, flex_decode_step,
                   flex_awd_loss, decode_state,
                   flex_attn_desc, make_attn_desc, attn_workspace_size, flex_attn_fwd, flex_attn_bwd,
                   flex_delta_desc, make_delta_desc, delta_workspace_size, delta_saved_size, flex_delta_fwd,
                   flex_delta_bwd, flex_delta_step,
                   flex_conv_desc, make_conv_desc, conv_workspace_size, flex_conv_fwd, flex_conv_bwd, flex_conv_step,
                   flex_scan_desc, make_scan_desc, scan_workspace_size, scan_saved_size, flex_scan_fwd, flex_scan_bwd,
                   flex_scan_step,
                   flex_norm_desc, make_norm_desc, norm_workspace_size, flex_norm_fwd, flex_norm_bwd,
                   decode_state_views, load, status_string,
                   FLEX_OK, FLEX_ERR_INVALID_ARG, FLEX_ERR_UNSUPPORTED, FLEX_ERR_WORKSPACE,
                   FLEX_ERR_HIP, FLEX_PASS_FEATURE_MAP, FLEX_PASS_FWD, FLEX_PASS_BWD, FLEX_PASS_AWD,
                   EXPORTS,
                   KERNELS, flex_timing_enable, flex_timing_read)
