"""The host code of the operators around the prefill under AddressSanitizer,
as test_asan_host.py does for the rest of the library: every refusal and the
frequency tables, on the CPU."""
from test_asan_host import _run


def test_serving_validation_under_asan():
    _run("from paper_2504_16083_amd import cache as KV\n"
         "import test_serving_abi as T\n"
         "T.test_symbols_and_structures()\n"
         "T.test_rope_frequencies()\n"
         "T.test_rope_refusals()\n"
         "T.test_cache_refusals()\n"
         "T.test_tree_refusals()\n"
         "T.test_binding_refusals()\n", timeout=300)


def test_serving_limits_under_asan():
    _run("import test_serving_abi as T\n"
         "T.test_rope_frequencies_end_at_2_to_40()\n"
         "for S in (524288, 1 << 21): T.test_rope_takes_long_fused_projections(S)\n"
         "T.test_broadcast_rows_are_refused(64, 8, 2)\n"
         "T.test_mask_without_words_is_refused()\n"
         "T.test_scale_that_overflows_is_refused()\n", timeout=300)
