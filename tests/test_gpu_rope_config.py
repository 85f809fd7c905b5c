"""A rotation whose reserved field is set is refused: it may be an option of a later version."""
import ctypes

import pytest

import synth

pytestmark = pytest.mark.gpu


def test_the_reserved_field_is_zero():
    import paper_2403_18647_gb300 as sd
    ctx = sd.Context(synth.SHAPES["tiny"], None, max_position=64)
    for reserved, status in ((1, 1), (-1, 1), (1 << 30, 1), (0, 0)):
        h = ctypes.c_void_p(77)
        cfg = sd.RopeConfig(64, 0, 128, 0, 0, reserved, 1e4, 1.0, 1.0, 32.0, 1.0)
        assert sd.lib().sdsat_rope_create(ctx.handle, ctypes.byref(cfg), ctypes.byref(h)) == status
        assert bool(h.value) == (status == 0)
        sd.lib().sdsat_rope_destroy(h)
    assert ctx.get_error() == 0
