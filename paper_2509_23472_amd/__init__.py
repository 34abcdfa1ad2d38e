"""LoRAct activation compression for AMD MI355X: Python binding of the libloract C ABI."""
from .api import (ACTIVATIONS, BF16, F32, MAX_HEAD, MAX_LORA_RANK, MAX_RANK, STATUS_RANK_DEFICIENT, LoractError,
                  AdamwState, MAX_TOP, TokenLogprobs, loract_adamw, loract_adamw_state, loract_compress,
                  loract_compress_adaptive, loract_dropout,
                  loract_gaussian_omega_t, loract_linear, loract_linear_backward, loract_lora_grad, loract_lora_grad_static, loract_lora_requests,
                  loract_static_scratch_bytes, loract_prenorm_backward,
                  loract_prenorm_forward, loract_profile_begin,
                  loract_profile_end, loract_qknorm_rope_backward, loract_qknorm_rope_forward, loract_reconstruct,
                  loract_rope_table, loract_rsvd, loract_sample_indices, loract_token_logprobs,
                  loract_token_logprobs_backward, loract_token_logprobs_grad,
                  loract_version, loract_workspace_bytes, make_params)

__all__ = [
    "ACTIVATIONS", "BF16", "F32", "MAX_HEAD", "MAX_LORA_RANK", "MAX_RANK", "STATUS_RANK_DEFICIENT", "LoractError",
    "AdamwState", "MAX_TOP", "TokenLogprobs", "loract_adamw", "loract_adamw_state",
    "loract_compress", "loract_compress_adaptive", "loract_dropout",
    "loract_gaussian_omega_t", "loract_linear", "loract_linear_backward", "loract_lora_grad", "loract_lora_grad_static", "loract_lora_requests",
    "loract_static_scratch_bytes", "loract_prenorm_backward", "loract_prenorm_forward",
    "loract_profile_begin", "loract_profile_end", "loract_qknorm_rope_backward", "loract_qknorm_rope_forward",
    "loract_reconstruct", "loract_rope_table", "loract_rsvd", "loract_sample_indices", "loract_token_logprobs",
    "loract_token_logprobs_backward", "loract_token_logprobs_grad", "loract_version",
    "loract_workspace_bytes", "make_params",
]
