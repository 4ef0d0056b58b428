"""What ptxas said of the kernels around the compression step: none of them spills."""
from test_build_report import _spills


def test_attention_and_cache_kernels_do_not_spill():
    for source, kernel, count in [("snapkv_prefill.cu", "prefill_kernel", 12),
                                  ("snapkv_decode_paged.cu", "decode_paged_kernel", 6),
                                  ("snapkv_append.cu", "append_kernel", 8)]:
        kernels = _spills(source, kernel)
        assert len(kernels) == count and not any(kernels.values()), kernels
