"""MI355X-native multi-tenant inference worker runtime (HIP, gfx950) and its thin binding."""
from .binding import (Context, MtError, attend_scratch, debug_big_tile_rows, debug_big_tile_walk, debug_conv_frame_ahead, debug_conv_row_tiling, debug_copy, debug_kv_write_places, debug_linear4_shape, debug_mfma_rate, kv_work, layer_spec, load_library, matrix4_footprint, model_footprint, row_groups, sample_scratch, score_scratch, version,  # noqa: F401
                      MT_ACT_GELU, MT_ACT_NONE, MT_ACT_RELU, MT_ADD, MT_BF16, MT_CONV2D, MT_F32, MT_FC, MT_GAP, MT_MAXPOOL,
                      MT_KV8, MT_KV_MAX_DIM, MT_KV_MAX_SEQS, MT_KV_MAX_WIDTH, MT_MAX_LAYERS, MT_MX8, MT_MX_BLOCK, MT_SAMPLE_MAX_CLASSES, MT_SCORE_MAX_GIVEN, MT_SCORE_MAX_TOP, mt_layer_spec)
from .torch_io import (KVCache, Samples, Scores, Served, add_norm, alloc_attend, alloc_kv, alloc_samples, alloc_scores, attend, context_for, kv_compact, kv_copy, kv_fork, kv_free,  # noqa: F401
                       kv_grow, kv_write, linear4, register_tenants, sample, score, serve)
