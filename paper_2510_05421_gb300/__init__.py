"""GB300 (sm_103a) DVI: self-speculative decode step and online drafter update.

The compute path is libdvi.so (csrc/, C-ABI in include/dvi.h); `dvi` is its
ctypes binding and `build` compiles it in-tree with nvcc.
"""
from .dvi import (DVIEngine, DeviceWeights, DVIError, lib, update_config, LIB_PATH, EXPORTS,  # noqa: F401
                  DVI_F32, DVI_BF16)
from .paged import PagedCache, rotary_table  # noqa: F401
from .pages import PagePool, RowPlan  # noqa: F401
from .sampling import token_probs, verify_drafts  # noqa: F401
