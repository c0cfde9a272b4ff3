"""BiQGEMM lookup-table matrix multiply for AMD MI355X (gfx950).

The product is libbiq.so (HIP kernels behind the C ABI of include/biq.h); this package is the
thin binding plus the synthetic workload generator.
"""
from .binding import (  # noqa: F401
    BIQ_EHIP, BIQ_EINVAL, BIQ_EUNSUPPORTED, BIQ_EWORKSPACE, BIQ_OK, BiqError, BiqPlan, BiqProblem, PreparedGemm, PreparedGroup, PreparedLstmCell, biq_gemm_grouped, biq_lstm_cell,
    biq_build_lut, biq_gemm, biq_gemm_ex, biq_gemm_noalloc, biq_init, biq_noalloc_scratch_bytes, biq_kernel_name, biq_key_row_stride, biq_lut_bytes,
    biq_num_chunks, biq_pack, biq_packed_bytes, biq_plan_check, biq_plan_get, biq_plan_get_lut, biq_plan_get_mfma, biq_plan_workspace_bytes, biq_quantize, biq_query,
    biq_unpack_keys, biq_unpack_keys16, biq_workspace_bytes, load_library, status_str,
)
from .serving import (  # noqa: F401
    KvCache, PreparedAppend, PreparedAttention, PreparedRead, PreparedRotary, PreparedSharedAttention, PreparedVerify, biq_attention,
    biq_attention_shared, biq_attention_shared_workspace_bytes, biq_attention_workspace_bytes, biq_cache_append, biq_cache_page_bytes, biq_cache_read, biq_rotary, biq_rotary_frequencies,
    biq_rotary_table, biq_verify_drafts, biq_verify_workspace_bytes,
)
from .step import (  # noqa: F401
    PreparedGemm4, PreparedLogits, PreparedNorm, biq_gemm4, biq_gemm4_workspace_bytes, biq_logits, biq_logits_workspace_bytes,
    biq_norm, biq_pack4, biq_packed4_bytes, biq_quantize4, biq_unpack4,
)
