"""MI355X (gfx950) SS2D selective scan: full and VMeanba channel-mean variants.

The computation lives in libvmb.so (hand-written HIP kernels behind the C ABI
declared in include/vmb.h); ``paper_2412_16602_amd.vmb`` is its ctypes
binding. Importing this package does not load the library; the first call
does, and fails loudly if it has not been built.
"""
from .vmb import (VMB_ACT_NONE, VMB_ACT_SILU, VMB_BF16, VMB_F32, VMB_LAYOUT_2D,  # noqa: F401
                  VMB_LAYOUT_SEQ, VmbError, abi_version, load_library, vmb_axis_rotary_bwd,
                  vmb_axis_rotary_fwd, vmb_cross_merge, vmb_cross_scan, vmb_gated_delta_bwd,
                  vmb_gated_delta_fwd, vmb_gated_delta_step, vmb_gated_delta_workspace_bytes,
                  vmb_group_norm_act_bwd, vmb_group_norm_act_fwd,
                  vmb_group_norm_act_workspace_bytes, vmb_mean_scan_fwd,
                  vmb_scan_workspace_bytes, vmb_selective_scan_fwd)
