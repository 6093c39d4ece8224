"""The calls on draft trees and their cache turn bad arguments into error codes on the host (no GPU: they return
before any launch), and the binding refuses tensors that do not fit together."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from paper_2603_11243_b200 import binding as ssd
from paper_2603_11243_b200 import build as ssd_build
import tree_ref


@pytest.fixture(scope="module")
def lib():
    ssd_build.build()
    return ssd.lib()


def heads(data=256, row=512, head=64, n=8):
    return ssd.Heads(data or None, row, head, n)


def cache(**kw):
    d = dict(k=256, v=256, page_stride=2048, slot_stride=128, head_stride=64, pages=4, page_size=16, heads=2, head_dim=64,
             dtype=ssd.BF16, max_pages=3, page_table=256, table_stride=3, len=256)
    d.update(kw)
    return ssd.KvCache(*[d[f] or None if f in ("k", "v", "page_table", "len") else d[f] for f, _ in ssd.KvCache._fields_])


P = C.c_void_p
ref = ssd._ref


def attention(lib, q=None, tk=None, tv=None, c=None, off=8, B=2, M=5, max_nodes=4, scale=0.1, cap=0.0, out=None, status=8,
              ws=256, ws_bytes=1 << 30):
    kv = lambda x: ref(heads(n=2, row=128) if x is None else x)  # noqa: E731
    return lib.ssd_tree_attention(ref(heads() if q is None else q), kv(tk), kv(tv), ref(cache() if c is None else c),
                                  P(off) if off else None, None, B, M, max_nodes, scale, cap,
                                  ref(heads() if out is None else out), None, P(status) if status else None, P(ws) if ws else None,
                                  ws_bytes, None)


BAD_CACHES = [(dict(dtype=ssd.F32), ssd.ERR_DTYPE), (dict(dtype=9), ssd.ERR_DTYPE), (dict(page_size=0), ssd.ERR_ARG),
              (dict(pages=-1), ssd.ERR_ARG), (dict(heads=0), ssd.ERR_ARG), (dict(head_dim=96), ssd.ERR_ARG),
              (dict(max_pages=-1), ssd.ERR_ARG), (dict(table_stride=2), ssd.ERR_ARG), (dict(len=0), ssd.ERR_NULL),
              (dict(page_table=0), ssd.ERR_NULL), (dict(k=0), ssd.ERR_NULL), (dict(k=264), ssd.ERR_ALIGN),
              (dict(slot_stride=132), ssd.ERR_ALIGN), (dict(head_stride=68), ssd.ERR_ALIGN), (dict(page_stride=2052), ssd.ERR_ALIGN),
              (dict(page_stride=-8), ssd.ERR_ARG), (dict(pages=1 << 28, page_size=8), ssd.ERR_ARG), (dict(page_stride=1 << 40), ssd.ERR_ARG)]


@pytest.mark.parametrize("kw,code", BAD_CACHES + [(dict(v=0), ssd.ERR_NULL), (dict(v=264), ssd.ERR_ALIGN)])
def test_attention_refuses_a_bad_cache(lib, kw, code):
    assert attention(lib, c=cache(**kw)) == code


def test_attention_refuses_bad_arguments(lib):
    assert attention(lib, off=0) == ssd.ERR_NULL
    assert attention(lib, status=0) == ssd.ERR_NULL
    assert attention(lib, q=heads(data=0)) == ssd.ERR_NULL
    assert attention(lib, out=heads(data=0)) == ssd.ERR_NULL
    for kw in (dict(B=-1), dict(M=-1), dict(M=1 << 31), dict(max_nodes=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(q=heads(n=3)),
               dict(q=heads(n=0)), dict(q=heads(n=258), out=heads(n=258)), dict(out=heads(n=4)), dict(tk=heads(n=1)), dict(tv=heads(n=4)),
               dict(q=heads(row=-8)), dict(q=heads(row=1 << 40))):
        assert attention(lib, **kw) == ssd.ERR_ARG, kw
    for kw in (dict(q=heads(data=264)), dict(q=heads(row=516)), dict(tk=heads(n=2, head=68)), dict(out=heads(data=258))):
        assert attention(lib, **kw) == ssd.ERR_ALIGN, kw
    need = lib.ssd_tree_attention_workspace_bytes(8, 2, 64, 5, 4)
    assert 0 < need < lib.ssd_tree_attention_workspace_bytes(8, 2, 64, 500, 400) < 1 << 30
    for kw in (dict(ws=0), dict(ws=264), dict(ws_bytes=need - 1)):
        assert attention(lib, **kw) == ssd.ERR_WORKSPACE, kw
    assert lib.ssd_tree_attention_workspace_bytes(8, 3, 64, 5, 4) == 0


def append(lib, tk=None, c=None, off=8, path=8, path_len=512, B=2, M=5, weight=8, stride=50, cols=50, new_len=1024, status=8):
    kv = heads(n=2, row=128)
    return lib.ssd_cache_append(ref(kv if tk is None else tk), ref(kv), ref(cache() if c is None else c), P(off) if off else None,
                                P(path), P(path_len) if path_len else None, B, M, P(weight), stride, cols,
                                P(new_len) if new_len else None, P(status) if status else None, None)


def test_append_refuses_bad_arguments(lib):
    for kw in (dict(off=0), dict(path_len=0), dict(new_len=0), dict(status=0), dict(tk=heads(data=0, n=2))):
        assert append(lib, **kw) == ssd.ERR_NULL, kw
    for kw in (dict(B=-1), dict(M=-1), dict(tk=heads(n=8)), dict(stride=49), dict(cols=-1), dict(new_len=256), dict(new_len=512)):
        assert append(lib, **kw) == ssd.ERR_ARG, kw
    assert append(lib, tk=heads(data=260, n=2)) == ssd.ERR_ALIGN
    for kw, code in BAD_CACHES:
        assert append(lib, c=cache(**kw)) == code, kw


def weights(lib, q=None, lse=8, c=None, off=8, B=2, M=5, max_nodes=4, scale=0.1, cap=0.0, weight=8, stride=50, cols=50, status=8):
    return lib.ssd_cache_weights(ref(heads() if q is None else q), P(lse) if lse else None, ref(cache(v=0) if c is None else c),
                                 P(off) if off else None, B, M, max_nodes, scale, cap, None, P(weight) if weight else None,
                                 stride, cols, P(status) if status else None, None)


def test_weights_refuse_bad_arguments(lib):
    for kw in (dict(off=0), dict(lse=0), dict(weight=0), dict(status=0), dict(q=heads(data=0))):
        assert weights(lib, **kw) == ssd.ERR_NULL, kw
    for kw in (dict(B=-1), dict(M=-1), dict(M=1 << 31), dict(max_nodes=-1), dict(scale=0.0), dict(cap=-1.0), dict(q=heads(n=3)),
               dict(stride=49), dict(cols=-1)):
        assert weights(lib, **kw) == ssd.ERR_ARG, kw
    assert weights(lib, q=heads(data=260)) == ssd.ERR_ALIGN
    for kw, code in BAD_CACHES:
        assert weights(lib, c=cache(v=0, **kw)) == code, kw


def evict(lib, c=None, weight=8, stride=50, cols=50, B=2, budget=10, sink=2, recent=3, kept=16, out=32, out_stride=10, new_len=8, status=8):
    opt = lambda p: P(p) if p else None  # noqa: E731
    return lib.ssd_cache_evict(ref(cache() if c is None else c), opt(weight), stride, cols, B, budget, sink, recent, opt(kept),
                               opt(out), out_stride, opt(new_len), opt(status), None)


def test_evict_refuses_bad_arguments(lib):
    for kw in (dict(weight=0), dict(kept=0), dict(new_len=0), dict(status=0)):
        assert evict(lib, **kw) == ssd.ERR_NULL, kw
    for kw in (dict(B=-1), dict(budget=-1), dict(sink=-1), dict(recent=-1), dict(sink=8), dict(stride=49), dict(cols=-1),
               dict(out_stride=9), dict(out=8)):
        assert evict(lib, **kw) == ssd.ERR_ARG, kw
    for kw, code in BAD_CACHES:
        assert evict(lib, c=cache(**kw)) == code, kw


def tree(lib, logits=8, dtype=ssd.BF16, V=10, ld=10, off=8, ids=8, B=1, M=4, outs=8, path=8, ws=256, ws_bytes=1 << 20, opts=None):
    opt = lambda p: P(p) if p else None  # noqa: E731
    return lib.ssd_verify_tree(opt(logits), dtype, V, ld, opt(off), opt(ids), None, B, M, C.c_float(0.1), None, opt(outs), None,
                               opt(path), opt(outs), opt(outs), opt(outs), opt(ws), ws_bytes, None, ssd._opts(opts))


def test_verify_tree_refuses_bad_arguments(lib):
    assert tree(lib, dtype=ssd.F16) == ssd.ERR_DTYPE
    for kw in (dict(V=0), dict(ld=9), dict(B=-1), dict(M=-1), dict(opts=ssd.LaunchOpts(finish=2))):
        assert tree(lib, **kw) == ssd.ERR_ARG, kw
    for kw in (dict(logits=0), dict(off=0), dict(ids=0), dict(outs=0), dict(path=0)):
        assert tree(lib, **kw) == ssd.ERR_NULL, kw
    assert tree(lib, logits=9) == ssd.ERR_ALIGN
    for kw in (dict(ws=0), dict(ws=264), dict(ws_bytes=64)):
        assert tree(lib, **kw) == ssd.ERR_WORKSPACE, kw


def test_the_binding_refuses_what_does_not_fit_together():
    c = tree_ref.Case(1, [3, 2], [5, 6])
    d = c.on("cpu")
    call = lambda **kw: ssd.ssd_tree_attention(**{**dict(  # noqa: E731
        q=d["q"], tree_k=d["tk"], tree_v=d["tv"], k_cache=d["k"], v_cache=d["v"], page_table=d["table"], cache_len=d["lens"],
        tok_off=d["off"], max_nodes=3, parent=d["parent"]), **kw})
    for kw in (dict(q=d["q"].half()), dict(tree_k=d["tk"].float()), dict(page_table=d["table"].long()), dict(cache_len=d["lens"].long()),
               dict(tok_off=d["off"].int()), dict(parent=d["parent"].long()), dict(parent=d["parent"][:-1])):
        with pytest.raises(TypeError):
            call(**kw)
    for kw in (dict(), dict(tree_v=d["tv"][:-1]), dict(tree_k=d["tk"][..., :32]), dict(q=d["q"].transpose(1, 2)), dict(v_cache=d["v"][:-1]),
               dict(page_table=d["table"][:1]), dict(cache_len=d["lens"][:1]), dict(k_cache=d["k"][0]),
               dict(v_cache=d["v"].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))):
        with pytest.raises(ValueError):                  # host tensors, last of all
            call(**kw)
    with pytest.raises(ValueError):
        ssd.ssd_cache_evict(d["k"], d["v"], d["table"], d["lens"], torch.zeros(3, 9), 4)
    with pytest.raises(TypeError):
        ssd.ssd_cache_append(d["tk"], d["tv"], d["off"], None, d["lens"].long(), d["k"], d["v"], d["table"], d["lens"])
    with pytest.raises(ValueError):
        ssd.ssd_cache_weights(d["q"], torch.zeros(5, 7), d["k"], d["table"], d["lens"], d["off"], 3, torch.zeros(2, 9))


def test_the_plain_reference_itself():
    """The CPU reference that the GPU tests use: a chain is causal attention, and probabilities sum to the rows' count."""
    c = tree_ref.Case(2, [4], [6], Hq=2, Hkv=1, chain=True)
    out, lse = c.attention()
    k = torch.cat([c.slots(c.k, 0), c.tk]).double()[:, 0]
    v = torch.cat([c.slots(c.v, 0), c.tv]).double()[:, 0]
    x = torch.einsum("nhd,ld->hnl", c.q.double(), k) * c.scale
    x = x.masked_fill(~torch.ones(4, 10, dtype=torch.bool).tril(6), -float("inf"))
    assert torch.allclose(torch.einsum("hnl,ld->nhd", torch.softmax(x, -1), v), out, atol=1e-12)
    assert torch.allclose(torch.logsumexp(x, -1).t(), lse, atol=1e-12)
    assert tree_ref.lines([-1, 0, 0, 2, 9]) == [[0], [0, 1], [0, 2], [0, 2, 3], [4]]


def test_the_native_marshalling_declines_what_is_not_plainly_fine():
    call = ssd._native()
    c = tree_ref.Case(1, [3, 2], [5, 6])
    d = c.on("cpu")
    out = ssd.alloc_tree_attention_outputs(5, 2, c.Hq, c.D, c.dtype, "cpu")
    args = [d["q"], d["tk"], d["tv"], d["k"], d["v"], d["table"], d["lens"], d["off"], 3, d["parent"], 0.1, 0.0, out]
    assert call.tree_attention(*args) is None and call.tree_attention(*args[:-1]) is None
    assert call.verify_tree(torch.zeros(5, 9), d["off"], d["parent"], None, 0.1, None, None, out) is None
    assert call.cache_append(d["tk"], d["tv"], d["off"], None, d["lens"], d["k"], d["v"], d["table"], d["lens"], None, {}) is None
    assert call.cache_weights(d["q"], None, d["k"], d["table"], d["lens"], d["off"], 3, None, None, 0.1, 0.0, {}) is None
    assert call.cache_evict(d["k"], d["v"], d["table"], d["lens"], None, 4, 0, 0, {}) is None
    with pytest.raises(ValueError):
        ssd.ssd_tree_attention(*args[:-1], out=out)
