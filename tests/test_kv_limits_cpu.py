"""Sizes and scales that the attention over the key/value cache refuses, on the host: no device is asked before."""
import ctypes as C
import math

import pytest

from paper_2603_16590_b200 import binding, build

SHAPE = 2


class _Handle(C.Structure):
    """The head of a batq_kv_cache, as far as the host's sizes go by it; the rest is zero."""
    _fields_ = [("device", C.c_int), ("sm_count", C.c_int), ("pages", C.c_int64), ("page_size", C.c_int32), ("page_shift", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("rest", C.c_uint8 * 1024)]


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _calls(lib, kv_heads=8, head_dim=128):
    c = _Handle(device=-1, sm_count=148, pages=1000, page_size=64, page_shift=6, kv_heads=kv_heads, head_dim=head_dim)

    def bytes_of(q_heads, tokens, seqs, max_q, max_kv):
        return lib.batq_attention_kv_mxfp8_workspace_bytes(C.addressof(c), q_heads, tokens, seqs, max_q, max_kv)

    def attend(q_heads, tokens, seqs, max_q, max_kv, scale=0.1):
        width = q_heads * head_dim
        return lib.batq_attention_kv_mxfp8(C.addressof(c), 256, width, q_heads, tokens, 256, 256, 256, 4, seqs, max_q, max_kv, scale, 1,
                                           256, width, None, None, 0, None)
    return c, bytes_of, attend


ACCEPTED = [(32, 1, 1, 1, 1 << 30), (32, 512, 512, 1, 16000000), (32, 5000, 512, 12, 2700000), (32, 100, 1, 100, (1 << 28) - 128),
            (32, 2048, 1, 2048, 100000), (8, 1000, 1000, 1, 16000000)]
REFUSED = [(32, 1, 1, 1, (1 << 30) + 1), (32, 512, 512, 1, 16800000), (32, 100, 1, 100, (1 << 28) - 127), (32, 1 << 30, 1, 1 << 30, 1000),
           (32, 1 << 29, 512, 1 << 20, 1000), (32, 600, 600, 1, 1 << 30)]


@pytest.mark.parametrize("sizes", ACCEPTED)
def test_bounds_within_the_limits(lib, sizes):
    """A workspace is asked for, so the call comes as far as missing it."""
    c, bytes_of, attend = _calls(lib)
    assert bytes_of(*sizes) > 0
    assert attend(*sizes) == 1


@pytest.mark.parametrize("sizes", REFUSED)
def test_bounds_past_the_limits(lib, sizes):
    c, bytes_of, attend = _calls(lib)
    assert bytes_of(*sizes) == 0
    assert attend(*sizes) == SHAPE


@pytest.mark.parametrize("scale", [math.nan, math.inf, -math.inf, 3e38, -2.4e38])
def test_scales_that_are_infinite_in_base_two(lib, scale):
    """The kernels work with scale * log2(e) in fp32: an infinite one would make 0 * infinity of a score of 0."""
    c, _, attend = _calls(lib)
    assert attend(32, 1, 1, 1, 100000, scale=scale) == SHAPE
    assert attend(32, 1, 1, 1, 100000, scale=2.3e38) == 1
