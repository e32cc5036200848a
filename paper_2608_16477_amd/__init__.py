"""MI355X (gfx950) library for target-side KV-cache reconstruction.

The compute lives in ``libpallas.so`` (hand-written HIP kernels behind a C
ABI declared in ``include/pallas.h``); this package is the thin ctypes
binding that marshals torch device tensors into those calls.  Importing the
binding does not touch the GPU; the first call loads the library and fails
loudly if it has not been built.
"""
from .binding import (  # noqa: F401
    PallasError, Status, lib, library_path,
    pallas_abi_version, pallas_last_error, pallas_check_coverage,
    pallas_model_create, pallas_model_destroy, pallas_workspace_size,
    pallas_prefill_prefix, pallas_prefill_chunk, pallas_pack_suffix_blocks, pallas_assemble_kv,
    pallas_decode_step, pallas_decode_step_static, Model, ChunkDesc, ChunkHeader, EXPORTS, KERNEL_CLASSES,
    pallas_rope_init, pallas_rope_apply, RopePlan, ROPE_LAYOUTS, ROPE_SCALINGS,
    pallas_quant_store, pallas_quant_load, pallas_append_kv, pallas_append_quant,
    pallas_attend_kv, pallas_attend_quant, pallas_attend_workspace_size,
    pallas_bounds_kv, pallas_bounds_quant, pallas_select_blocks, pallas_select_workspace_size,
    pallas_attend_blocks_kv, pallas_attend_blocks_quant,
    pallas_profile_enable, pallas_profile_read, pallas_profile_reset, pallas_profile_clock,
    pallas_window_select, pallas_window_evaluate, pallas_ewma_update, pallas_admit,
    pallas_waste_bound, WindowParams, WindowDecision, Ewma,
)
