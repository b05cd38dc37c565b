"""MI355X-native batched token sampling (the sampling step that ends every decode iteration), and the vocabulary head
around it.

The product is the C library ``libsip.so`` (sources in ``csrc/``, boundary in
``include/sip.h`` and ``include/sip_head.h``); this package is its thin Python binding."""
from .binding import (SIP_BF16, SIP_F32, SIP_MAX_K_LOGPROBS, SIP_MAX_L, SIP_MAX_SHARDS, SIP_MAX_SLOTS, SIP_MAX_V, ShardTable, SipError, load,
                      sip_call_route, sip_probe_read, sip_profile_kernel_events, sip_publish_ids, sip_sample, sip_init, sip_noalloc_scratch_bytes, sip_sample_noalloc, sip_sample_call, sip_sample_sharded, sip_sample_state, sip_state_assign, sip_state_bytes,
                      sip_state_init, sip_status_string, sip_version, sip_wait_ids, sip_workspace_bytes, sip_workspace_bytes_sharded,
                      state_table_views, state_views)

from .head import (SIP_MAX_D, SIP_MAX_TENSORS, SIP_MAX_TOKENS, GradTable, sip_grad_clip, sip_grad_clip_workspace_bytes,
                   sip_head_logits, sip_head_quantize, sip_head_workspace_bytes, sip_xent_backward, sip_xent_forward,
                   sip_xent_workspace_bytes)

__all__ = ["SIP_BF16", "SIP_F32", "SIP_MAX_K_LOGPROBS", "SIP_MAX_L", "SIP_MAX_SHARDS", "SIP_MAX_SLOTS", "SIP_MAX_V", "ShardTable", "SipError", "load",
           "sip_call_route", "sip_probe_read", "sip_profile_kernel_events", "sip_publish_ids", "sip_sample", "sip_init", "sip_noalloc_scratch_bytes", "sip_sample_noalloc", "sip_sample_call", "sip_sample_sharded", "sip_sample_state", "sip_state_assign", "sip_state_bytes",
           "sip_state_init", "sip_status_string", "sip_version", "sip_wait_ids", "sip_workspace_bytes", "sip_workspace_bytes_sharded", "state_table_views", "state_views"]
__all__ += ["GradTable", "SIP_MAX_D", "SIP_MAX_TENSORS", "SIP_MAX_TOKENS", "sip_grad_clip", "sip_grad_clip_workspace_bytes",
            "sip_head_logits", "sip_head_quantize", "sip_head_workspace_bytes", "sip_xent_backward", "sip_xent_forward",
            "sip_xent_workspace_bytes"]
