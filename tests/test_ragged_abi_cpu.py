"""The entry points of ragged batches refuse null handles before any CUDA call; constants and structures match the header."""
import ctypes
import os
import re


def test_null_handles_are_refused_without_a_gpu():
    import paper_2403_18647_gb300 as sd
    lib = sd.lib()
    h = ctypes.c_void_p()
    assert lib.sdsat_rope_create(None, ctypes.byref(sd.RopeConfig()), ctypes.byref(h)) == 1
    lib.sdsat_rope_destroy(None)
    assert lib.sdsat_op_rotary_append(None, None, None, 64, None, 64, None, 64, 0, 1, None, None, 1, None, None, None, 1e-5, 1, 1, 64,
                                      None, 64, None, None, 1, None, 1, None) == 1
    assert lib.sdsat_op_chunk_attention(None, None, 64, 1, None, None, 1, None, 1, None, None, 1, 1, 1, 64, None, 64, 0) == 1
    assert lib.sdsat_op_adjust_logits(None, None, 100, 0, 1, 1, 100, None, 0, None, None, None, None, None, None, None, None, None, 0,
                                      None, 0, None, 100) == 1


def test_constants_and_the_structure_match_the_header():
    import paper_2403_18647_gb300 as sd
    src = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sdsat.h")).read()
    for name, value in (("PLAIN", None), ("LINEAR", "linear"), ("PARTS", "parts")):
        assert int(re.search(r"#define SDSAT_ROPE_%s (\d+)" % name, src).group(1)) == sd.ROPE_SCALING[value]
    body = re.search(r"typedef struct \{([^}]*)\} sdsat_rope_config;", src).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip() for d in body.split(";") if d.strip() for n in d.split(None, 1)[1].split(",")]
    assert names == [n for n, _ in sd.RopeConfig._fields_]
