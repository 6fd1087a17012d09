"""MI355X-native layer-wise post-training quantization solve (libptq bindings)."""
from .binding import (  # noqa: F401
    OP_INT8_LINEAR, OP_PAGED_ATTENTION, OP_SHARED_ATTENTION, PTQ_BF16, PTQ_F32, PTQ_F64, PtqError, lib_path, load_library,
    ptq_activation_abs_sum, ptq_activation_scale, ptq_average_bits, ptq_damped_cholesky_inv, ptq_hessian_accumulate, ptq_layer_error,
    ptq_lopro_column_order, ptq_lopro_linear_forward, ptq_lopro_linear_forward_static, ptq_lopro_linear_forward_static_limit, ptq_lopro_rotate_hessian, ptq_lopro_rotate_weight, ptq_lopro_unrotate_weight,
    PTQ_ROTARY_BASE, PTQ_ROTARY_LINEAR, PTQ_ROTARY_PLAIN, PTQ_ROTARY_TURNS, ptq_kv_cache_copy_pages, ptq_paged_attention_shared, ptq_prompt_attention, ptq_rotary, ptq_rotary_frequencies, ptq_rotary_kv_cache_write,
    ptq_int8_linear, ptq_kv_cache_read, ptq_kv_cache_write, ptq_pack_codes, ptq_paged_attention, ptq_quantize_layer, ptq_quantize_layer_static_groups, ptq_quantize_layer_vq, ptq_rmsnorm_quantize, ptq_scaled_r1svd, ptq_unpack_dequantize, ptq_status_string, ptq_workspace_bytes,
)
