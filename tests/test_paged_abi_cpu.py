"""The entry points of paged caches and of their operators refuse null handles before any CUDA call."""


def test_null_handles_are_refused_without_a_gpu():
    import paper_2403_18647_gb300 as sd
    lib = sd.lib()
    assert lib.sdsat_kv_create_paged(None, 1, 64, 4, None) == 1
    assert lib.sdsat_kv_pages(None, None, None, None, None) == 1
    assert lib.sdsat_kv_fork(None, None, None, 1) == 1
    assert lib.sdsat_kv_free(None, None, 0) == 1
    assert lib.sdsat_kv_reserve(None, None, 0, 1, 6) == 1
    assert lib.sdsat_kv_compact(None, None, None) == 1
    assert lib.sdsat_op_prefix_attention(None, None, 0, None, None, 1, None, 1, None, None, None, 1, 1, 1, 1, 64, None, 0, 0) == 1
    assert lib.sdsat_op_logprobs(None, None, 0, 0, 1, 100, None, 1.0, 0, None, None, None, None, None) == 1


def test_the_paged_constants_match_the_header():
    import os
    import re
    import paper_2403_18647_gb300 as sd
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sdsat.h")).read()
    value = lambda n: int(re.search(r"#define %s (0x[0-9a-f]+|\d+)" % n, src).group(1).rstrip("u"), 0)  # noqa: E731
    assert (value("SDSAT_PAGE"), value("SDSAT_FP32"), value("SDSAT_BF16")) == (sd.PAGE, sd.FP32, sd.BF16)
    assert value("SDSAT_DEV_PAGE") == sd.DEV_PAGE
