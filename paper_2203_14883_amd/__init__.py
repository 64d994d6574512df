"""MI355X-native hot path of TGL (Zhou et al., VLDB 2022): T-CSR build and
multi-hop temporal neighbour sampling, and the feature / state lookup of the
sampled slots, as hand-written HIP kernels behind the C
ABI of include/tgl.h.  ``binding`` marshals torch tensors into that ABI;
``layer8`` holds the 8-bit operators that serve a temporal attention layer;
``layer`` those that train one, with gradients;
``workloads`` draws the seeded synthetic graphs and root streams."""
from .binding import (TCSR, Hop, Sampler, TglError, lib, sample, sample_capacity,  # noqa: F401
                      status_str, tcsr_build, tcsr_build_workspace, tcsr_from_host, tcsr_from_columns, tcsr_columns,
                      pack_entries, timer_enable, timer_disable, timer_read, timer_reset, timer_select,
                      gather, time_encode, pointers_reset, mfg_export, MFG, EXPORTS, LIB_PATH, MOST_RECENT, UNIFORM, KEY_NODE, KEY_EDGE)
from .layer import (RowGroups, group_rows, layer_norm, layer_norm_backward, linear_typed,  # noqa: F401
                    linear_typed_backward)
from .layer8 import (HistoryCache, cache_attend, cache_read, cache_write, linear_i8, norm_quant,  # noqa: F401
                     quant_rows)
