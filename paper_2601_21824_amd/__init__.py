"""MI355X-native deterministic FlashAttention backward (DASH schedules), over dense
batches and over packed sequences, rotary positions, and attention over a paged key-value cache.

The computation lives in libdash.so (HIP kernels for gfx950 behind the C ABI
in include/dash.h); ``binding`` is its ctypes wrapper and ``synth`` draws the
seeded synthetic inputs.
"""
from . import binding  # noqa: F401
from .binding import (DashError, attn_bwd, attn_decode, attn_fwd, attn_packed_bwd, attn_packed_fwd,  # noqa: F401
                      dash_attn_bwd, dash_attn_decode, dash_attn_fwd, dash_attn_packed_bwd, dash_attn_packed_fwd,
                      dash_bwd_check, dash_bwd_workspace_size, dash_decode_workspace_size, dash_kv_append,
                      dash_last_error, dash_packed_fwd_workspace_size, dash_packed_workspace_size,
                      dash_bwd_placement, dash_mfma_peak, dash_release_workspace, dash_resolve_schedule,
                      dash_schedule_table, attn_prefix_decode, dash_attn_prefix_decode, dash_kv_read,
                      dash_prefix_decode_workspace_size, dash_rotary, dash_rotary_frequencies, kv_read, rotary)
