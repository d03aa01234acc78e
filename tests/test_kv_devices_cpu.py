"""Tensors that are not where the cache is: the binding refuses them before the library is called."""
import ctypes as C

import pytest
import torch

from paper_2603_16590_b200 import binding, build


class _Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


class _Cache:
    handle = C.c_void_p(64)
    kv_heads, head_dim, device_index = 2, 64, -1     # the tensors below are the host's


@pytest.mark.parametrize("shim", [True, False])
def test_tensors_elsewhere_are_refused(monkeypatch, shim):
    build.build()
    binding.load()
    called = []
    P, I64, I32, SZ, F = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t, C.c_float
    append = C.CFUNCTYPE(C.c_int, P, P, P, P, P, I64, P, I64, P, I64, P, I64, I32, I64, P, P, P, I64, I32, P)(lambda *a: called.append(a) or 0)
    attend = C.CFUNCTYPE(C.c_int, P, P, I64, I32, I64, P, P, P, I64, I32, I32, I32, F, I32, P, I64, P, P, SZ, P)(lambda *a: called.append(a) or 0)
    monkeypatch.setattr(binding, "_stream", lambda: 7)
    monkeypatch.setattr(binding, "_ADDRESS", {"batq_kv_append_mxfp8": C.cast(append, P).value, "batq_attention_kv_mxfp8": C.cast(attend, P).value})
    monkeypatch.setattr(binding, "_LIB", type("Lib", (), {"batq_kv_append_mxfp8": staticmethod(append), "batq_attention_kv_mxfp8": staticmethod(attend)}))
    if not shim:
        monkeypatch.setattr(binding, "_CALL", None)
    assert (binding._CALL is not None) == shim
    x = torch.zeros(5, 640, dtype=torch.bfloat16)
    q, k, v = x.split([384, 128, 128], 1)
    calls = [(binding.batq_kv_append_mxfp8,
              dict(t_k=None, t_v=None, k=k, v=v, slots=torch.zeros(5, dtype=torch.int64), positions=torch.zeros(5, dtype=torch.int32),
                   rope=torch.zeros(9, 32), q=q, q_out=torch.zeros(5, 384, dtype=torch.bfloat16))),
             (binding.batq_attention_kv_mxfp8,
              dict(q=q, out=torch.zeros(5, 384, dtype=torch.bfloat16), kv_lens=torch.zeros(3, dtype=torch.int32),
                   page_table=torch.zeros(3, 11, dtype=torch.int32), max_q=4, max_kv=99, workspace=torch.zeros(64, dtype=torch.uint8),
                   q_starts=torch.zeros(4, dtype=torch.int32), lse=torch.zeros(5, 6)))]
    for call, good in calls:
        call(_Cache, **good)
        tensors = [name for name, x in good.items() if isinstance(x, torch.Tensor)]
        assert len(tensors) == 7
        for name in tensors:
            with pytest.raises(ValueError, match=f"{name}: on device 1"):
                call(_Cache, **{**good, name: good[name].as_subclass(_Elsewhere)})
        with pytest.raises(ValueError, match="on device -1, the cache is on 0"):
            call(type("OnGpu", (_Cache,), {"device_index": 0}), **good)
    assert len(called) == 2


def test_cache_buffers_of_the_host_are_refused():
    codes, scales = torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA device"):
        binding.batq_kv_cache_create(codes, scales, codes.clone(), scales.clone())
