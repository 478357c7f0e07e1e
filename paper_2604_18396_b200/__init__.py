"""B200 (sm_100a) early-exit decode library: thin Python binding over the C ABI in include/river.h."""
from .binding import (argmax_noalloc, RIVER_EXIT_BATCH_MIN, RIVER_EXIT_PER_TOKEN, RIVER_F_GRAPH, RIVER_F_NO_TC, River, RiverError,
                      make_config, river_config)
from .buildlib import build
from .cache_ops import (pages_admit, pages_advance, pages_compact, pages_reorder, pages_slots, prefix_attention, prefix_attention_bytes,
                        prefix_groups, rope_append, rope_frequencies, window_attention)

__all__ = ["rope_frequencies", "rope_append", "window_attention", "pages_advance", "pages_reorder", "pages_compact", "pages_admit", "pages_slots",
           "prefix_groups", "prefix_attention", "prefix_attention_bytes", "River", "argmax_noalloc", "RiverError", "make_config", "river_config", "build", "RIVER_EXIT_PER_TOKEN",
           "RIVER_EXIT_BATCH_MIN", "RIVER_F_GRAPH", "RIVER_F_NO_TC"]
