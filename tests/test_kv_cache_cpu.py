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


# ------------------------------------------------------------------------------------------------ the binding
class _Cache:
    handle = C.c_void_p(64)
    kv_heads, head_dim = 2, 64


def _call_arguments(monkeypatch, shim):
    """What the two calls hand to their C entry points: through the shim, or through ctypes."""
    seen = []
    P, I64, I32, SZ, F = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t, C.c_float
    append = C.CFUNCTYPE(C.c_int, P, P, P, P, P, I64, P, I64, P, I64, P, I64, I32, I64, P, P, P, I64, I32, P)(lambda *a: seen.append(a) or 0)
    attend = C.CFUNCTYPE(C.c_int, P, P, I64, I32, I64, P, P, P, I64, I32, I32, I32, F, I32, P, I64, P, P, SZ, P)(lambda *a: seen.append(a) or 0)
    if shim:
        monkeypatch.setattr(binding, "_ADDRESS", {"batq_kv_append_mxfp8": C.cast(append, P).value, "batq_attention_kv_mxfp8": C.cast(attend, P).value})
    else:
        monkeypatch.setattr(binding, "_CALL", None)
        monkeypatch.setattr(binding, "_LIB", type("Lib", (), {"batq_kv_append_mxfp8": staticmethod(append), "batq_attention_kv_mxfp8": staticmethod(attend)}))
    monkeypatch.setattr(binding, "_stream", lambda: 7)
    x = torch.zeros(5, 640, dtype=torch.bfloat16)
    q, k, v = x.split([384, 128, 128], 1)
    q_out = torch.zeros(5, 400, dtype=torch.bfloat16)[:, :384]
    slots, pos, rope = torch.zeros(5, dtype=torch.int64), torch.zeros(5, dtype=torch.int32), torch.zeros(9, 32)
    t = type("T", (), {"handle": C.c_void_p(32)})()
    binding.batq_kv_append_mxfp8(_Cache, t, None, k, v, slots, positions=pos, rope=rope, t_q=t, q=q, q_out=q_out)
    binding.batq_kv_append_mxfp8(_Cache, None, t, k, v, slots)
    lens, table, starts = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 11, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    lse, ws = torch.zeros(5, 6), torch.zeros(512, dtype=torch.uint8)
    binding.batq_attention_kv_mxfp8(_Cache, q, q_out, lens, table, 4, 99, ws, q_starts=starts, scale=0.5, causal=False, lse=lse)
    binding.batq_attention_kv_mxfp8(_Cache, q[:3], q_out[:3], lens, table, 1, 99)
    ptr = lambda a: a.data_ptr()  # noqa: E731
    assert seen == [
        (64, 32, None, 32, ptr(k), 640, ptr(v), 640, ptr(q), 640, ptr(q_out), 400, 6, 5, ptr(slots), ptr(pos), ptr(rope), 9, 32, 7),
        (64, None, 32, None, ptr(k), 640, ptr(v), 640, None, 0, None, 0, 0, 5, ptr(slots), None, None, 0, 0, 7),
        (64, ptr(q), 640, 6, 5, ptr(starts), ptr(lens), ptr(table), 11, 3, 4, 99, 0.5, 0, ptr(q_out), 400, ptr(lse), ptr(ws), 512, 7),
        (64, ptr(q), 640, 6, 3, None, ptr(lens), ptr(table), 11, 3, 1, 99, 0.125, 1, ptr(q_out), 400, None, None, 0, 7)]


def test_arguments_through_the_shim(lib, monkeypatch):
    assert binding._CALL is not None
    _call_arguments(monkeypatch, True)


def test_arguments_through_ctypes(lib, monkeypatch):
    _call_arguments(monkeypatch, False)


@pytest.mark.parametrize("shim", [True, False])
def test_tensors_of_another_form_are_refused(lib, monkeypatch, shim):
    """What the kernels would read or write past an end of: refused before the library is called."""
    monkeypatch.setattr(binding, "_stream", lambda: 7)
    called = []
    P, I64, I32, SZ, F = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t, C.c_float
    append = C.CFUNCTYPE(C.c_int, P, P, P, P, P, I64, P, I64, P, I64, P, I64, I32, I64, P, P, P, I64, I32, P)(lambda *a: called.append(a) or 0)
    attend = C.CFUNCTYPE(C.c_int, P, P, I64, I32, I64, P, P, P, I64, I32, I32, I32, F, I32, P, I64, P, P, SZ, P)(lambda *a: called.append(a) or 0)
    monkeypatch.setattr(binding, "_ADDRESS", {"batq_kv_append_mxfp8": C.cast(append, P).value, "batq_attention_kv_mxfp8": C.cast(attend, P).value})
    if not shim:
        monkeypatch.setattr(binding, "_CALL", None)
    monkeypatch.setattr(binding, "_LIB", type("Lib", (), {"batq_kv_append_mxfp8": staticmethod(lambda *a: called.append(a) or 0),
                                                          "batq_attention_kv_mxfp8": staticmethod(lambda *a: called.append(a) or 0)}))
    x = torch.zeros(5, 640, dtype=torch.bfloat16)
    q, k, v = x.split([384, 128, 128], 1)
    slots, pos, rope = torch.zeros(5, dtype=torch.int64), torch.zeros(5, dtype=torch.int32), torch.zeros(9, 32)
    good = dict(positions=pos, rope=rope, q=q, q_out=q)
    binding.batq_kv_append_mxfp8(_Cache, None, None, k, v, slots, **good)
    for bad in (dict(slots=slots[:4]), dict(slots=slots.int()), dict(slots=torch.zeros(10, dtype=torch.int64)[::2]), dict(positions=pos[:4]),
                dict(positions=pos.long()), dict(rope=rope.double()), dict(rope=rope[:, :16]), dict(k=k[:, :64]), dict(k=k.float()),
                dict(v=v[:4]), dict(q_out=q[:4]), dict(q_out=q[:, :320]), dict(q=q[:, :100], q_out=q[:, :100]),
                dict(k=torch.zeros(128, 5, dtype=torch.bfloat16).t())):
        with pytest.raises(ValueError):
            a = {**dict(k=k, v=v, slots=slots), **good, **bad}
            binding.batq_kv_append_mxfp8(_Cache, None, None, a.pop("k"), a.pop("v"), a.pop("slots"), **a)
    lens, table, starts = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 11, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    good = dict(q=q, out=q, kv_lens=lens, page_table=table, max_q=4, max_kv=99, q_starts=starts)
    binding.batq_attention_kv_mxfp8(_Cache, **good)
    for bad in (dict(q=q.float()), dict(out=q[:4]), dict(out=q[:, :320]), dict(kv_lens=lens.long()), dict(q_starts=starts[:3]),
                dict(q_starts=starts.long()), dict(page_table=table[:2]), dict(page_table=table.long()), dict(page_table=table[:, :5]),
                dict(lse=torch.zeros(4, 6)), dict(lse=torch.zeros(5, 6).double()), dict(q=q[:, :100], out=q[:, :100])):
        with pytest.raises(ValueError):
            binding.batq_attention_kv_mxfp8(_Cache, **{**good, **bad})
    assert len(called) == 2
