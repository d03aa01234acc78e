"""Key/value cache entry points without a device: what they refuse, before any device work."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv_reference as R
from paper_2603_16590_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_cache_create_refuses(lib):
    h = C.c_void_p()
    make = lambda *a: lib.batq_kv_cache_create(C.byref(h), *a)  # noqa: E731
    assert lib.batq_kv_cache_create(None, 256, 256, 256, 256, 4, 64, 8, 128) == 1
    for i in range(4):
        p = [256] * 4
        p[i] = None
        assert make(*p, 4, 64, 8, 128) == 1
        p[i] = 264
        assert make(*p, 4, 64, 8, 128) == 3
    for sizes in ((0, 64, 8, 128), (-1, 64, 8, 128), (4, 0, 8, 128), (4, 64, 0, 128), (4, 64, 8, 0), (1 << 22, 64, 8, 128), (1 << 40, 64, 8, 128)):
        assert make(256, 256, 256, 256, *sizes) == 2
    for sizes in ((4, 8, 8, 128), (4, 48, 8, 128), (4, 256, 8, 128), (4, 64, 8, 96), (4, 64, 8, 256)):
        assert make(256, 256, 256, 256, *sizes) == 4
    assert not h.value
    assert lib.batq_kv_cache_destroy(None) == 0


def test_null_handles_are_refused(lib):
    assert lib.batq_kv_append_mxfp8(None, None, None, None, 256, 128, 256, 128, None, 0, None, 0, 0, 1, 256, None, None, 0, 0, None) == 1
    assert lib.batq_attention_kv_mxfp8(None, 256, 128, 1, 1, None, 256, 256, 4, 1, 1, 64, 1.0, 1, 256, 128, None, None, 0, None) == 1
    assert lib.batq_attention_kv_mxfp8_workspace_bytes(None, 8, 1, 1, 1, 64) == 0
    h = C.c_void_p()
    assert lib.batq_transform_create_dual(None, None) == 1
    assert lib.batq_transform_create_dual(C.byref(h), None) == 1
    assert binding.STATUS_NAMES[9] == "ERR_INDEX" and lib.batq_status_string(9) == b"index outside its table"


def test_binding_refuses_buffers_of_another_form():
    codes, scales = torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, dtype=torch.uint8)
    with pytest.raises(ValueError):
        binding.batq_kv_cache_create(codes, scales, codes, torch.zeros(4, 2, 16, 4, dtype=torch.uint8))
    with pytest.raises(ValueError):
        binding.batq_kv_cache_create(codes.float(), scales, codes, scales)
    with pytest.raises(ValueError):
        binding.batq_kv_cache_create(codes.transpose(1, 2), scales, codes, scales)


def test_reference_quantiser_against_torch():
    """The tests' MXFP8 against torch's conversion of values that fp32 holds: equal codes below saturation."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(50, 128, generator=g) * torch.exp(3 * torch.randn(50, 128, generator=g))
    codes, scales = R.mxfp8(x.double())
    e = scales.double() - 127
    u = (x.double().unflatten(-1, (-1, 32)) / torch.exp2(e)[..., None]).flatten(-2)
    assert (u.abs() < 512).all()
    assert torch.equal(codes, u.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    y = R.values(codes, scales)
    step = torch.exp2(torch.floor(torch.log2(x.double().abs().clamp(min=1e-30))) - 3)
    least = torch.exp2(e - 9).repeat_interleave(32, -1)
    inside = u.abs() <= 448
    assert ((y - x.double()).abs()[inside] <= (torch.maximum(step, least) / 2)[inside] * (1 + 1e-12)).all()


def test_reference_attention_by_hand():
    """Two keys, one head: out and lse as written down, and an empty row."""
    v = torch.zeros(2, 1, 16, 64, dtype=torch.float64)
    k = torch.zeros(2, 1, 16, 64, dtype=torch.float64)
    k[1, 0, 0, 0], k[1, 0, 1, 0], v[1, 0, 0, 3], v[1, 0, 1, 3] = 1.0, 2.0, 4.0, 8.0
    q = torch.zeros(2, 1, 64)
    q[:, 0, 0] = 1.0
    out, lse, _ = R.attention(q, R.mxfp8(k), R.mxfp8(v), [2], [2], [[1]], 1.0, True)
    e = np.e
    assert abs(out[0, 0, 3] - 4) < 1e-12 and abs(lse[0, 0] - 1) < 1e-12
    assert abs(out[1, 0, 3] - (4 * e + 8 * e * e) / (e + e * e)) < 1e-12 and abs(lse[1, 0] - np.log(e + e * e)) < 1e-12
    out, lse, _ = R.attention(q, R.mxfp8(k), R.mxfp8(v), [2], [1], [[1]], 1.0, True)
    assert out[0].abs().max() == 0 and lse[0, 0] == -np.inf and abs(out[1, 0, 3] - 4) < 1e-12
