"""libadacomp for MI355X: AdaComp residual-gradient compression (pack / unpack hot path).

The product is the C library ``libadacomp.so`` (sources in ``csrc/``, ABI in ``include/adacomp.h``);
this package is its ctypes binding.
"""
from .binding import (AdacompError, adacomp_compress, adacomp_compress_static, adacomp_compress_batch, adacomp_compress_batch_lazy, adacomp_compress_variant, adacomp_residue_sync, adacomp_copy_f32, adacomp_triad_f32, adacomp_triad_resident_f32, adacomp_fill_f32, adacomp_debug_keep_gmax, adacomp_debug_wait_polls, adacomp_debug_one_launch, adacomp_packet_bound,  # noqa: F401
                      adacomp_packet_fixed_bytes, adacomp_selftest_binindex, adacomp_timing_enable, adacomp_tuning_unpack_min_groups, adacomp_tuning_fold_scan, adacomp_tuning_place_tiled,
                      adacomp_timing_read, adacomp_unpack_accumulate, adacomp_unpack_update, OPT_SGD_MOMENTUM, OPT_ADAM, adacomp_workspace_bytes, adacomp_workspace_bytes_batch,
                      adacomp_workspace_gmax, adacomp_workspace_init, adacomp_workspace_release,
                      read_packet_summary, RULE_ADACOMP, RULE_PRINTED_COMPARE, RULE_LOCAL_SELECTION)
from .layers import (LAYER_EXPORTS, Dropout, RelativeBias, adacomp_bias_softmax_backward, adacomp_bias_softmax_forward,  # noqa: F401
                     adacomp_bias_softmax_workspace_bytes, adacomp_dropout, adacomp_norm_backward, adacomp_norm_forward,
                     adacomp_norm_workspace_bytes, adacomp_relative_buckets)
from .sequence import (RECURRENCE_KEEP, SEQUENCE_EXPORTS, TEACHER_TOP_MAX, adacomp_distill_backward, adacomp_distill_forward,  # noqa: F401
                       adacomp_embed_backward, adacomp_embed_forward, adacomp_embed_workspace_bytes, adacomp_recurrence_backward, adacomp_recurrence_forward,
                       adacomp_recurrence_kept, adacomp_recurrence_workspace_bytes)
