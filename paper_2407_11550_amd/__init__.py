"""MI355X-native Ada-KV per-layer cache compression: score, allocate, select, compact.

Decode side of the resulting flattened cache: cache_build, append, decode_attn, decode_step; the same in
8 bits: cache_build_q8, append_q8, decode_attn_q8, decode_step_q8; its sequences forked, dropped and given
other head-room: cache_move, cache_move_q8; a step of sequences that share caches: decode_prefix_attn,
decode_prefix_step.  Attention over the prompt: window_attn.  In front of both: rotary
positions of queries and keys, rotary, and norms of their heads in the same pass, norm_rotary.
All calls run entirely in the HIP library (csrc/); this package only marshals
arguments.  Importing the package does not load the library; the first call does,
and raises if the library has not been built.
"""
from .binding import (PROBE_SINK_BYTES, Q8_BLOCK, STATIC_SCRATCH_BYTES, AdaKVError, KernelTrace, Layer, Prefix, Q8Cache, Rotary,  # noqa: F401
                      allocate, append, append_q8, cache_build, cache_build_q8, cache_move, cache_move_q8, cache_rows, compact,
                      compress, compress_static, decode_attn, decode_attn_q8, decode_prefix_attn, decode_prefix_step, decode_step,
                      decode_step_q8, decode_workspace_bytes, describe, library_path, load_library, norm_rotary,
                      prefix_workspace_bytes, probe_read, pyramid_budgets, q8_cache, q8_scales, rotary, rotary_frequencies, score,
                      select, window_attn, workspace_bytes)
