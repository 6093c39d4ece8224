"""The calls on draft trees refuse tensors of another device than the current one, by the fast way and by the general one.

There may be only one GPU: a tensor is then given another device's number (through DLPack) over memory of this one."""
import ctypes as C

import pytest
import torch

from paper_2603_11243_b200 import binding as ssd
from tree_ref import Case

pytestmark = pytest.mark.gpu


class DLTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("device_type", C.c_int32), ("device_id", C.c_int32), ("ndim", C.c_int32),
                ("code", C.c_uint8), ("bits", C.c_uint8), ("lanes", C.c_uint16), ("shape", C.POINTER(C.c_int64)),
                ("strides", C.POINTER(C.c_int64)), ("offset", C.c_uint64)]


class DLManaged(C.Structure):
    _fields_ = [("tensor", DLTensor), ("context", C.c_void_p), ("deleter", C.c_void_p)]


CODES = {torch.int32: (0, 32), torch.int64: (0, 64), torch.uint8: (1, 8), torch.float32: (2, 32), torch.float16: (2, 16), torch.bfloat16: (4, 16)}
KEEP = []


def elsewhere(t):
    """t's memory, as a tensor of device 1"""
    code, bits = CODES[t.dtype]
    shape, strides = (C.c_int64 * t.dim())(*t.shape), (C.c_int64 * t.dim())(*t.stride())
    m = DLManaged(DLTensor(t.data_ptr(), 2, 1, t.dim(), code, bits, 1, shape, strides, 0), None, None)
    KEEP.append((m, shape, strides, t))
    new = C.pythonapi.PyCapsule_New
    new.restype, new.argtypes = C.py_object, [C.c_void_p, C.c_char_p, C.c_void_p]
    x = torch._C._from_dlpack(new(C.addressof(m), b"dltensor", None))
    assert x.device == torch.device("cuda:1") and x.data_ptr() == t.data_ptr()
    return x


def calls(dev):
    """name -> (function, arguments, results)"""
    c = Case(50, [5, 3], [20, 30], room=8)
    d = c.on(dev)
    ids, logits = torch.zeros(8, dtype=torch.int32, device=dev), torch.randn(8, 50, device=dev)
    weight, use = torch.zeros(2, 48, device=dev), torch.ones(8, dtype=torch.uint8, device=dev)
    lse = torch.zeros(8, c.Hq, device=dev)
    path_len = torch.ones(2, dtype=torch.int32, device=dev)
    path = torch.zeros(8, dtype=torch.int32, device=dev)
    cache = dict(k_cache=d["k"], v_cache=d["v"], page_table=d["table"], cache_len=d["lens"])
    keys = {k: v for k, v in cache.items() if k != "v_cache"}
    return dict(
        attention=(ssd.ssd_tree_attention, dict(q=d["q"], tree_k=d["tk"], tree_v=d["tv"], tok_off=d["off"], max_nodes=5, parent=d["parent"], **cache),
                   ssd.alloc_tree_attention_outputs(8, 2, c.Hq, c.D, c.dtype, dev)),
        verify=(ssd.ssd_verify_tree, dict(logits=logits, tok_off=d["off"], draft_ids=ids, parent=d["parent"], tau_slm=0.1, skip=use[:2]),
                ssd.alloc_verify_tree_outputs(8, 2, dev, ssd.ssd_verify_workspace_bytes(2, 8, 50, ssd.F32))),
        append=(ssd.ssd_cache_append, dict(tree_k=d["tk"], tree_v=d["tv"], tok_off=d["off"], path=path, path_len=path_len, weight=weight, **cache),
                ssd.alloc_cache_append_outputs(2, dev)),
        weights=(ssd.ssd_cache_weights, dict(q=d["q"], lse=lse, tok_off=d["off"], max_nodes=5, weight=weight, use=use, **keys),
                 ssd.alloc_cache_weights_outputs(2, dev)),
        evict=(ssd.ssd_cache_evict, dict(weight=weight, budget=10, **cache), ssd.alloc_cache_evict_outputs(2, 10, dev)))


@pytest.mark.parametrize("name", ["attention", "verify", "append", "weights", "evict"])
@pytest.mark.parametrize("native", [True, False])
def test_tensors_of_another_device_are_refused(cuda_device, monkeypatch, name, native):
    f, args, out = calls(cuda_device)[name]
    if not native:
        monkeypatch.setattr(ssd, "_call", ssd._Declines())
    f(**args, out=out)
    for key, t in args.items():
        if isinstance(t, torch.Tensor):
            with pytest.raises(ValueError, match="current device"):
                f(**{**args, key: elsewhere(t)}, out=out)
    for key, t in out.items():
        with pytest.raises(ValueError, match="current device"):
            f(**args, out={**out, key: elsewhere(t)})
    torch.cuda.synchronize()
