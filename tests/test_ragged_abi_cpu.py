"""The entry points of ragged batches refuse null handles before any CUDA call; constants and structures match the header."""
import ctypes
import os
import re

import pytest


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


class Fake:
    """What the binding asks of a tensor, without memory."""

    def __init__(self, dtype, *shape, cuda=True, contiguous=True, stride=None):
        self.dtype, self.shape, self.is_cuda, self.contiguous = dtype, shape, cuda, contiguous
        self.strides = stride or tuple([shape[1], 1] if len(shape) == 2 else [1] * len(shape))

    def stride(self):
        return self.strides

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 1 << 20


@pytest.fixture()
def calls():
    """The calls with a stream of their own; the handles are null, so that what passes the checks is refused by the library."""
    import torch
    import paper_2403_18647_gb300 as sd
    sd._types()
    sd._calls.types(torch.float32, torch.bfloat16, torch.int32, lambda: 0)
    yield sd._calls
    sd._types()


def rotary(n, **change):
    import torch
    f, h, i = torch.float32, torch.bfloat16, torch.int32
    a = dict(ctx=None, rope=None, q=Fake(f, 6, 256), k=Fake(f, 6, 128), v=Fake(f, 6, 128), q_out=Fake(f, 6, 256), k_pages=Fake(h, 5, 2, 64, 64),
             v_pages=Fake(h, 5, 2, 64, 64), table=Fake(i, 2, 3), lens=Fake(i, 2), starts=Fake(i, 3), H=4, Hk=2, hd=64, positions=Fake(i, 6),
             q_gain=Fake(h, 64), k_gain=None, eps=1e-5, refs=Fake(i, 5))
    a.update(change)
    return n.rotary_append(*a.values())


def chunk(n, **change):
    import torch
    f, h, i = torch.float32, torch.bfloat16, torch.int32
    a = dict(ctx=None, q=Fake(f, 6, 256), k_pages=Fake(h, 5, 2, 64, 64), v_pages=Fake(h, 5, 2, 64, 64), table=Fake(i, 2, 3), lens=Fake(i, 2),
             starts=Fake(i, 3), H=4, Hk=2, hd=64, out=Fake(f, 6, 256))
    a.update(change)
    return n.chunk_attention(*a.values())


def adjust(n, **change):
    import torch
    f, i = torch.float32, torch.int32
    a = dict(ctx=None, logits=Fake(f, 6, 100), out=Fake(f, 6, 100), q=3, history=Fake(i, 2, 9), history_lens=Fake(i, 2), prompt_lens=None,
             tokens=Fake(i, 6), anc=None, repetition=Fake(f, 2), frequency=None, presence=None, bias_ids=Fake(i, 2, 5), bias=Fake(f, 2, 5),
             allowed=Fake(i, 6, 4))
    a.update(change)
    return n.adjust_logits(*a.values())


def test_tensors_are_checked_without_a_gpu(calls):
    import torch
    f, h, i = torch.float32, torch.bfloat16, torch.int32
    assert rotary(calls) == chunk(calls) == adjust(calls) == 1              # null handles: EINVAL
    for call, wrong in (
            (rotary, [dict(q=Fake(h, 6, 256)), dict(q=Fake(f, 6, 255)), dict(q=Fake(f, 6, 4, 64)), dict(q=Fake(f, 6, 256, cuda=False)),
                      dict(q=Fake(f, 6, 256, stride=(1, 6))), dict(k=Fake(f, 5, 128)), dict(v=Fake(f, 6, 127)), dict(q_out=Fake(f, 5, 256)),
                      dict(k_pages=Fake(h, 5, 2, 32, 64)), dict(v_pages=Fake(h, 4, 2, 64, 64)), dict(k_pages=Fake(f, 5, 2, 64, 64)),
                      dict(v_pages=Fake(h, 5, 2, 64, 64, contiguous=False)), dict(table=Fake(i, 6)), dict(table=Fake(torch.int64, 2, 3)),
                      dict(lens=Fake(i, 1)), dict(starts=Fake(i, 2)), dict(positions=Fake(i, 5)), dict(q_gain=Fake(f, 64)), dict(k_gain=Fake(h, 63)),
                      dict(refs=Fake(i, 4)), dict(H=1 << 40), dict(Hk=3), dict(q=Fake(f, 1 << 31, 256), q_out=Fake(f, 1 << 31, 256),
                                                                               k=Fake(f, 1 << 31, 128), v=Fake(f, 1 << 31, 128))]),
            (chunk, [dict(q=Fake(h, 6, 256)), dict(q=Fake(f, 7, 256)), dict(out=Fake(f, 6, 255)), dict(k_pages=Fake(h, 5, 3, 64, 64)),
                     dict(table=Fake(i, 2)), dict(lens=Fake(i, 1)), dict(starts=Fake(i, 2)), dict(starts=Fake(i, 3, cuda=False)), dict(hd=128)]),
            (adjust, [dict(logits=Fake(h, 6, 100)), dict(out=Fake(f, 6, 99)), dict(out=Fake(f, 5, 100)), dict(q=0), dict(q=4), dict(q=-3),
                      dict(history=Fake(i, 1, 9)), dict(history=Fake(i, 18)), dict(history_lens=Fake(i, 1)), dict(tokens=Fake(i, 5)),
                      dict(anc=Fake(f, 6)), dict(presence=Fake(h, 2)), dict(bias=None), dict(bias_ids=None), dict(bias=Fake(f, 2, 4)),
                      dict(allowed=Fake(i, 6, 3)), dict(allowed=Fake(i, 5, 4))])):
        for change in wrong:
            with pytest.raises(ValueError):
                call(calls, **change)
    for call in (rotary, chunk, adjust):
        with pytest.raises(AttributeError):
            call(calls, **{"logits" if call is adjust else "q": "a text"})
    with pytest.raises(TypeError):
        calls.chunk_attention(None)
    with pytest.raises(TypeError):
        rotary(calls, eps="small")
