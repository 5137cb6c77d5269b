"""MI355X-native multi-tenant inference worker runtime (HIP, gfx950) and its thin binding."""
from .binding import (Context, MtError, debug_big_tile_rows, debug_big_tile_walk, debug_conv_frame_ahead, debug_conv_row_tiling, debug_copy, debug_linear4_shape, debug_mfma_rate, layer_spec, load_library, matrix4_footprint, model_footprint, row_groups, score_scratch, version,  # noqa: F401
                      MT_ACT_GELU, MT_ACT_NONE, MT_ACT_RELU, MT_ADD, MT_BF16, MT_CONV2D, MT_F32, MT_FC, MT_GAP, MT_MAXPOOL,
                      MT_MAX_LAYERS, MT_MX8, MT_MX_BLOCK, MT_SCORE_MAX_GIVEN, MT_SCORE_MAX_TOP, mt_layer_spec)
from .torch_io import Scores, Served, add_norm, alloc_scores, context_for, linear4, register_tenants, score, serve  # noqa: F401
