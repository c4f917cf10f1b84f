"""fp64 CPU oracle for Flash-ABFT attention.

TEST INFRASTRUCTURE ONLY: imported by tests, the smoke check and the
benchmark's CPU-baseline leg, never by the product path.
"""
from .attention import (visible_mask, sumrow, attention_head, attention,
                        global_check, lazy_softmax_attention,
                        online_checksum_attention, threshold_flags,
                        brute_force_head, alternating_weights,
                        weighted_check_head)
from .cache import cache_k, cache_v, cache_attention, cache_keep

__all__ = ["cache_k", "cache_v", "cache_attention", "cache_keep",
           "visible_mask", "sumrow", "attention_head", "attention",
           "global_check", "lazy_softmax_attention",
           "online_checksum_attention", "threshold_flags", "brute_force_head",
           "alternating_weights", "weighted_check_head"]
