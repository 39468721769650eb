"""B200 (sm_100a) linear attention for hybrid models behind a C ABI: the chunkwise prefill of the delta rule (GDN and KDA) and its
decoding step, gated linear attention with its backward pass, and the norms on both sides of a block.

`layer` has the latter two; `binding` marshals torch CUDA tensors into the C struct of include/ha_la.h and calls
libha_la.so; `synth` draws the seeded synthetic workloads; `build` compiles the library.
Importing the package loads nothing native; the first call does, and raises if the
library has not been built.
"""
from .binding import (  # noqa: F401
    HaLaError,
    ha_la_debug_wait_timeout,
    ha_la_decode,
    ha_la_decode_args,
    ha_la_decode_raw,
    ha_la_prefill,
    ha_la_prefill_args,
    ha_la_prefill_launch_plan,
    ha_la_prefill_num_launches,
    ha_la_prefill_num_runs,
    ha_la_prefill_num_segments,
    ha_la_prefill_path,
    ha_la_prefill_noalloc,
    ha_la_prefill_noalloc_scratch_bytes,
    ha_la_prefill_raw,
    ha_la_prefill_timed,
    ha_la_prefill_workspace_bytes,
    ha_la_version,
    load_library,
    make_args,
    prepare_args,
    prepare_decode_args,
    status_string,
)
from .layer import (  # noqa: F401
    ha_la_add_norm,
    ha_la_add_norm_args,
    ha_la_add_norm_backward,
    ha_la_add_norm_workspace_bytes,
    ha_la_gated_norm,
    ha_la_gated_norm_args,
    ha_la_gated_norm_backward,
    ha_la_gated_norm_workspace_bytes,
    ha_la_gla_args,
    ha_la_gla_backward,
    ha_la_gla_decode,
    ha_la_gla_path,
    ha_la_gla_prefill,
    ha_la_gla_workspace_bytes,
)
