"""GB300-native budget-routed decode (BUDDY, arXiv 2606.09514).

The compute path is libbuddy.so (CUDA kernels for sm_103a behind the C ABI in
include/buddy.h); `binding` marshals arguments to it.  There is no CPU path.
"""
from .binding import (Context, KVCache, KV4Cache, BuddyError, load_library, pack_layer,  # noqa: F401
                      buddy_budget_to_k, buddy_page_plan, buddy_qk_norm_rope, buddy_rope_table)
