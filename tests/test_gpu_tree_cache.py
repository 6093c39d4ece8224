"""ssd_cache_append, ssd_cache_weights and ssd_cache_evict against the definitions on the CPU, and a whole
verification pass over a draft tree through every call.

Weights: a weight is a sum of up to n * Hq probabilities exp(s - lse).  Their relative error is the absolute error of
s - lse in fp32: s is a sum of D exact products (below 3e-6 at the sizes here), lse is given, the difference is
rounded once (|s - lse| < 32: 2e-6), and ex2 adds 2^-22: 1e-5 relative covers it and the additions."""
import math

import numpy as np
import pytest
import torch

from paper_2603_11243_b200 import binding as ssd
from tree_ref import Case, planted, verify_tree

pytestmark = pytest.mark.gpu


def cpu(d):
    torch.cuda.synchronize()
    return {k: v.cpu() for k, v in d.items()}


# ---- append ------------------------------------------------------------------------------------------

def appended(c, path, path_len):
    k, v = c.k.clone(), c.v.clone()
    for b in range(c.B):
        for i in range(int(path_len[b])):
            s, node = int(c.lens[b]) + i, int(c.off[b]) + int(path[c.off[b] + i])
            k[c.table[b, s // c.page], s % c.page] = c.tk[node]
            v[c.table[b, s // c.page], s % c.page] = c.tv[node]
    return k, v


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,lens,Hkv,D,page", [([1], [0], 1, 64, 16), ([9], [7], 2, 64, 16), ([5, 0, 33, 200], [15, 3, 100, 0], 5, 128, 24),
                                               ([3] * 70, [31] * 70, 8, 128, 1)])
def test_append(cuda_device, dtype, n, lens, Hkv, D, page):
    rng = np.random.default_rng(1)
    c = Case(20, n, lens, Hq=Hkv, Hkv=Hkv, D=D, page=page, dtype=dtype, room=max(n))
    path, path_len = np.full(c.M, -1, np.int32), np.zeros(c.B, np.int32)
    for b in range(c.B):
        p = np.sort(rng.permutation(n[b])[:rng.integers(0, n[b] + 1)])
        path_len[b] = len(p)
        path[c.off[b]:c.off[b] + len(p)] = p
    d, put = c.on(cuda_device), lambda a: torch.from_numpy(a).to(cuda_device)
    weight = torch.ones(c.B, int(max(lens)) + max(n), device=cuda_device)
    r = cpu(ssd.ssd_cache_append(d["tk"], d["tv"], d["off"], put(path), put(path_len), d["k"], d["v"], d["table"], d["lens"], weight))
    k, v = appended(c, path, path_len)
    assert torch.equal(d["k"].cpu(), k) and torch.equal(d["v"].cpu(), v)
    assert r["new_len"].tolist() == (c.lens + path_len).tolist() and not r["utt_status"].any()
    w = weight.cpu()
    for b in range(c.B):
        lo, hi = int(c.lens[b]), int(c.lens[b]) + int(path_len[b])
        assert (w[b, lo:hi] == 0).all() and (w[b, :lo] == 1).all() and (w[b, hi:] == 1).all()


def test_append_refuses_what_does_not_fit(cuda_device):
    c = Case(21, [4, 4, 4, 4, 4], [14, 10, 10, 10, 10], room=4, page=16)
    path = np.tile(np.arange(4, dtype=np.int32), 5)
    path[2 * 4 + 1] = 4                                            # none of utterance 2's nodes
    d, put = c.on(cuda_device), lambda a: torch.from_numpy(a).to(cuda_device)
    table = d["table"].clone()
    table[:, 1:] = c.k.shape[0] + 5                                # a page outside the cache behind slot 16
    table[1, 0] = -1
    lens = d["lens"].clone()
    lens[0], lens[3] = 30, 40                                      # 30 + 4 > 32; 40 > 32
    path_len = torch.tensor([4, 4, 4, 4, 5], dtype=torch.int32, device=cuda_device)
    before = d["k"].clone()
    r = cpu(ssd.ssd_cache_append(d["tk"], d["tv"], d["off"], put(path), path_len, d["k"], d["v"], table, lens))
    assert r["utt_status"].tolist() == [ssd.UTT_CACHE_FULL, ssd.UTT_BAD_CACHE, ssd.UTT_BAD_PARENT, ssd.UTT_BAD_CACHE, ssd.UTT_BAD_PARENT]
    assert r["new_len"].tolist() == [30, 14, 14, 40, 10]
    k = before.cpu()
    for i in (0, 2, 3):
        k[c.table[2, 0], 10 + i] = c.tk[8 + i]
    assert torch.equal(d["k"].cpu(), k)
    with pytest.raises(ssd.SsdError) as e:
        ssd.ssd_cache_append(d["tk"], d["tv"], d["off"], None, path_len, d["k"], d["v"], table, lens,
                             out=dict(new_len=lens, utt_status=path_len.clone()))
    assert e.value.code == ssd.ERR_ARG


# ---- weights -----------------------------------------------------------------------------------------

def weights(c, lse, use, cap):
    w = torch.zeros(c.B, int(c.lens.max(initial=0)), dtype=torch.float64)
    for b in range(c.B):
        rows = [r for r in range(int(c.off[b]), int(c.off[b + 1])) if use is None or use[r]]
        if rows and c.lens[b]:
            x = c.scores(c.q[rows], c.slots(c.k, b), cap)
            w[b, :int(c.lens[b])] = torch.exp(x - lse[rows].double().t()[:, :, None]).sum((0, 1))
    return w


def run_weights(c, dev, lse, use=None, cap=0.0, d=None, weight=None):
    d = d or c.on(dev)
    if weight is None:
        weight = torch.zeros(c.B, int(c.lens.max(initial=0)), device=dev)
    r = ssd.ssd_cache_weights(d["q"], lse.to(dev), d["k"], d["table"], d["lens"], d["off"], c.max_nodes, weight,
                              None if use is None else use.to(dev), c.scale, cap)
    torch.cuda.synchronize()
    return weight, r["utt_status"]


@pytest.mark.parametrize("dtype,cap", [(torch.bfloat16, 0.0), (torch.float16, 0.0), (torch.bfloat16, 15.0)])
@pytest.mark.parametrize("n,lens,Hq,Hkv,D,page", [([1], [1], 1, 1, 64, 16), ([1], [1000], 32, 8, 64, 16), ([3, 0, 9], [100, 50, 0], 8, 2, 128, 8),
                                                  ([20, 70, 5], [300, 129, 640], 28, 4, 64, 24), ([6] * 40, [200] * 40, 4, 4, 128, 200),
                                                  ([1, 2], [333, 40], 64, 1, 64, 100)])
def test_weights(cuda_device, dtype, cap, n, lens, Hq, Hkv, D, page):
    c = Case(22, n, lens, Hq=Hq, Hkv=Hkv, D=D, page=page, dtype=dtype).spoil_unused()
    lse = c.attention(cap)[1].float()
    use = torch.from_numpy((np.random.default_rng(3).random(c.M) < 0.7).astype(np.uint8))
    for u in (None, use):
        got, status = run_weights(c, cuda_device, lse, u, cap)
        want = weights(c, lse, u, cap)
        assert ((got.cpu().double() - want).abs() <= 1e-5 * want + 1e-12).all()
        assert not status.any()
        again, _ = run_weights(c, cuda_device, lse, u, cap, weight=got.clone())       # adds, and to the same bits
        assert torch.equal(again, got + got)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,Hq,Hkv", [([300, 7, 65], 4, 2), ([33, 130], 16, 2), ([9, 17], 96, 1), ([5, 40], 128, 1), ([200], 3, 1)])
def test_weights_of_many_tiles_of_queries(cuda_device, D, n, Hq, Hkv):
    """More tiles of queries to a head than slots for them: its keys have to stay, and nobody may wait for them to go."""
    c = Case(29, n, [150 + 20 * i for i in range(len(n))], Hq=Hq, Hkv=Hkv, D=D, chain=True)
    lse = c.attention()[1].float()
    got, status = run_weights(c, cuda_device, lse)
    want = weights(c, lse, None, 0.0)
    assert not status.any()
    assert ((got.cpu().double() - want).abs() <= 1e-5 * want + 1e-12).all()


def test_weights_of_uncounted_nodes_and_short_arrays(cuda_device):
    c = Case(23, [7, 40], [300, 150])
    lse = c.attention()[1].float()
    use = torch.ones(c.M, dtype=torch.uint8)
    use[[1, 4, 20]] = 0
    want, _ = run_weights(c, cuda_device, lse, use)
    c.q[1], c.q[4] = math.nan, math.inf
    lse[20] = math.nan
    got, _ = run_weights(c, cuda_device, lse, use)
    assert torch.equal(got, want)
    # fewer columns than slots, in the middle of a wider array
    wide = torch.full((2, 400), 5.0, device=cuda_device)
    got, status = run_weights(c, cuda_device, lse, use, weight=wide[:, 10:210])
    assert status.cpu().tolist() == [ssd.UTT_BAD_CACHE, 0]
    assert (wide[:, :10] == 5).all() and (wide[:, 210:] == 5).all() and (wide[1, 160:] == 5).all()
    assert ((wide[0, 10:210] - 5 - want[0, :200]).abs() <= 2e-6).all()


def test_weights_with_malformed_utterances(cuda_device):
    c = Case(24, [3, 4, 5], [20, 30, 40])
    lse = c.attention()[1].float()
    d = c.on(cuda_device)
    d["off"] = torch.tensor([0, 3, 2, 12], dtype=torch.int64, device=cuda_device)
    d["table"] = d["table"].clone()
    d["table"][0, 1] = -3
    weight, status = run_weights(c, cuda_device, lse, d=d)
    assert status.cpu().tolist() == [ssd.UTT_BAD_CACHE, ssd.UTT_BAD_OFFSETS, ssd.UTT_BAD_OFFSETS]
    assert (weight[1:] == 0).all() and (weight[0, :16] > 0).all()


# ---- evict -------------------------------------------------------------------------------------------

def evicted(c, weight, budget, sink, recent):
    """kept lists, by a stable sort"""
    kept = []
    for b in range(c.B):
        L = int(c.lens[b])
        if L <= budget:
            kept.append(np.arange(L))
            continue
        w = weight[b, :L].astype(np.float64)
        w = np.where(np.isnan(w), -np.inf, w)
        nan = np.isnan(weight[b, :L])
        middle = np.arange(sink, L - recent)
        order = middle[np.lexsort((middle, nan[middle], -w[middle]))]
        kept.append(np.concatenate([np.arange(sink), np.sort(order[:budget - sink - recent]), np.arange(L - recent, L)]))
    return kept


def check_evict(c, dev, weight, budget, sink, recent, inplace=False):
    d = c.on(dev)
    w = torch.from_numpy(weight).to(dev)
    out = None
    if inplace:
        out = ssd.alloc_cache_evict_outputs(c.B, budget, dev)
        out["new_len"] = d["lens"]
    r = cpu(ssd.ssd_cache_evict(d["k"], d["v"], d["table"], d["lens"], w, budget, sink, recent, out=out))
    k, v = c.k.clone(), c.v.clone()
    for b, keep in enumerate(evicted(c, weight, budget, sink, recent)):
        m = len(keep)
        assert r["kept"][b, :m].tolist() == keep.tolist() and (r["kept"][b, m:] == -1).all(), b
        assert np.array_equal(r["weight"][b, :m].numpy(), weight[b, keep], equal_nan=True) and (r["weight"][b, m:] == 0).all()
        assert r["new_len"][b] == m
        for pool in (k, v):
            src = pool[torch.from_numpy(c.table[b, keep // c.page].astype(np.int64)), torch.from_numpy(keep % c.page)].clone()
            j = np.arange(m)
            pool[torch.from_numpy(c.table[b, j // c.page].astype(np.int64)), torch.from_numpy(j % c.page)] = src
    assert torch.equal(d["k"].cpu(), k) and torch.equal(d["v"].cpu(), v)
    assert not r["utt_status"].any()


@pytest.mark.parametrize("lens,budget,sink,recent,page,D", [([10], 4, 1, 1, 16, 64), ([0, 1, 5, 6, 7], 6, 0, 6, 8, 64), ([3000, 40, 700], 500, 4, 100, 16, 128),
                                                            ([5000], 1, 0, 0, 64, 64), ([2049, 2048], 2048, 0, 0, 100, 64), ([600], 64, 64, 0, 8, 128),
                                                            ([900], 0, 0, 0, 16, 64), ([300] * 50, 100, 3, 7, 1, 64), ([20000, 9], 6000, 16, 1000, 256, 64)])
def test_evict(cuda_device, lens, budget, sink, recent, page, D):
    rng = np.random.default_rng(4)
    c = Case(25, [1] * len(lens), lens, Hq=3, Hkv=3, D=D, page=page)
    W = max(max(lens), 1)
    check_evict(c, cuda_device, np.exp(2 * rng.standard_normal((c.B, W))).astype(np.float32), budget, sink, recent)
    check_evict(c, cuda_device, rng.integers(0, 4, (c.B, W)).astype(np.float32), budget, sink, recent, inplace=True)     # ties
    check_evict(c, cuda_device, np.zeros((c.B, W), np.float32), budget, sink, recent)
    ramp = np.tile(np.arange(W, dtype=np.float32), (c.B, 1))
    check_evict(c, cuda_device, ramp, budget, sink, recent)                       # the last are kept: the longest moves
    check_evict(c, cuda_device, -ramp, budget, sink, recent)                      # the first are kept: none


def test_evict_with_odd_weights(cuda_device):
    rng = np.random.default_rng(5)
    c = Case(26, [1], [400], Hq=1, Hkv=1)
    w = rng.standard_normal((1, 400)).astype(np.float32)
    w[0, ::7], w[0, 1::7], w[0, 2::7], w[0, 3::7], w[0, 4::7] = np.nan, -0.0, 0.0, -np.inf, np.inf
    for budget in (30, 100, 250, 390):
        check_evict(c, cuda_device, w, budget, 2, 3)


def test_evict_reports_what_is_malformed(cuda_device):
    c = Case(27, [1, 1, 1], [100, 100, 100], Hq=1, Hkv=1)
    d = c.on(cuda_device)
    table, lens = d["table"].clone(), d["lens"].clone()
    table[0, 3] = c.k.shape[0]
    lens[1] = 10_000
    before = d["k"].clone()
    w = torch.rand(3, 100, device=cuda_device)
    r = cpu(ssd.ssd_cache_evict(d["k"], d["v"], table, lens, w, 50, 0, 0))
    assert (r["utt_status"][:2] == ssd.UTT_BAD_CACHE).all() and r["utt_status"][2] == 0
    spare = torch.ones(before.shape[0], dtype=torch.bool)
    spare[torch.from_numpy(c.table[:, :7].astype(np.int64)).flatten()] = False
    assert torch.equal(d["k"].cpu()[spare], before.cpu()[spare])


# ---- together ----------------------------------------------------------------------------------------

def test_a_verification_pass_over_trees(cuda_device):
    """Attention -> (a stand-in for the rest of the model) -> verification along the tree -> append -> attention again
    from the grown cache -> weights of the accepted nodes -> eviction, two steps in a row, captured into a graph
    and checked against the same steps from the definitions."""
    dev = cuda_device
    c = Case(28, [9, 14, 1, 30], [60, 200, 33, 0], Hq=8, Hkv=2, D=64, room=40)
    rng = np.random.default_rng(6)
    x, ids = planted(rng, c.off, c.parent, 700, likely=0.9)
    d = c.on(dev)
    put = lambda a: torch.from_numpy(a).to(dev)  # noqa: E731
    logits, ids_d = torch.from_numpy(x).float().to(dev), put(ids)
    W, budget = 260, 120
    weight = torch.rand(c.B, W, device=dev)
    start = weight.cpu().numpy().copy()
    att = ssd.alloc_tree_attention_outputs(c.M, c.B, c.Hq, c.D, c.dtype, dev)
    ver = ssd.alloc_verify_tree_outputs(c.M, c.B, dev, ssd.ssd_verify_workspace_bytes(c.B, c.M, 700, ssd.F32))
    app = ssd.alloc_cache_append_outputs(c.B, dev)
    wei = ssd.alloc_cache_weights_outputs(c.B, dev)
    evi = ssd.alloc_cache_evict_outputs(c.B, budget, dev)

    def step():
        ssd.ssd_tree_attention(d["q"], d["tk"], d["tv"], d["k"], d["v"], d["table"], d["lens"], d["off"], c.max_nodes, d["parent"], out=att)
        ssd.ssd_verify_tree(logits, d["off"], ids_d, d["parent"], 0.02, out=ver)
        ssd.ssd_cache_weights(d["q"], att["lse"], d["k"], d["table"], d["lens"], d["off"], c.max_nodes, weight, ver["on_path"], out=wei)
        ssd.ssd_cache_append(d["tk"], d["tv"], d["off"], ver["path"], ver["path_len"], d["k"], d["v"], d["table"], d["lens"], weight, out=app)
        ssd.ssd_cache_evict(d["k"], d["v"], d["table"], app["new_len"], weight, budget, 2, 20, out=evi)

    keep = {k: v.clone() for k, v in d.items()}
    step()                                                        # one of each before the capture
    torch.cuda.synchronize()
    for k, v in keep.items():
        d[k].copy_(v)
    weight.copy_(torch.from_numpy(start))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    torch.cuda.synchronize()
    out, lse = c.attention()
    assert ((att["out"].cpu().double() - out).norm() / out.norm()) < 5e-3
    logp, _, path, length, on = verify_tree(x.astype(np.float32).astype(np.float64), c.off, ids, c.parent, 0.02)
    assert np.array_equal(ver["path"].cpu().numpy(), path) and np.array_equal(ver["path_len"].cpu().numpy(), length)
    w = torch.from_numpy(start).double()
    add = weights(c, att["lse"].cpu(), on, 0.0)
    w[:, :add.shape[1]] += add
    k, v = appended(c, path, length)
    for b in range(c.B):
        w[b, int(c.lens[b]):int(c.lens[b]) + int(length[b])] = 0
    got = weight.cpu()
    assert ((got.double() - w).abs() <= 2e-5 * w + 1e-6).all()
    assert app["new_len"].cpu().tolist() == (c.lens + length).tolist()
    c.k, c.v, c.lens = k, v, c.lens + length
    for b, kept in enumerate(evicted(c, got.numpy(), budget, 2, 20)):
        assert evi["kept"][b, :len(kept)].cpu().tolist() == kept.tolist()
        src = c.slots(c.k, b)[kept].clone()
        c.lens[b] = len(kept)
        assert torch.equal(c.slots(d["k"].cpu(), b), src)
    # the next pass reads what this one left
    c.k, c.v = d["k"].cpu(), d["v"].cpu()
    ssd.ssd_tree_attention(d["q"], d["tk"], d["tv"], d["k"], d["v"], d["table"], evi["new_len"], d["off"], c.max_nodes, d["parent"], out=att)
    out, _ = c.attention()
    assert ((att["out"].cpu().double() - out).norm() / out.norm()) < 5e-3


@pytest.mark.parametrize("what", ["lse", "query", "both"])
def test_weights_of_a_counted_node_that_is_nan(cuda_device, what):
    """exp(s - lse) of a counted node is NaN where either is: its utterance's slots become NaN (never a sum without it),
    the other utterance's do not."""
    c = Case(40, [7, 40], [300, 150])
    lse = c.attention()[1].float()
    use = torch.ones(c.M, dtype=torch.uint8)
    use[[2, 9]] = 0
    want, _ = run_weights(c, cuda_device, lse, use)
    if what != "lse":
        c.q[4, 3, 5] = math.nan
    if what != "query":
        lse[4, 3] = math.nan
    got, _ = run_weights(c, cuda_device, lse, use)
    assert torch.isnan(got[0, :300]).all()
    assert torch.equal(got[1, :150], want[1, :150])


def test_weights_of_a_counted_node_with_an_infinite_lse(cuda_device):
    """exp(s - inf) is 0 for a score s, and NaN for one that is NaN: only use == 0 takes a node out."""
    c = Case(41, [7, 40], [300, 150])
    lse = c.attention()[1].float()
    use = torch.ones(c.M, dtype=torch.uint8)
    use[4] = 0
    without, _ = run_weights(c, cuda_device, lse, use)
    lse[4] = math.inf
    got, _ = run_weights(c, cuda_device, lse)
    assert torch.equal(got, without)
    c.q[4, 3, 5] = math.nan
    got, _ = run_weights(c, cuda_device, lse)
    assert torch.isnan(got[0, :300]).all() and torch.equal(got[1, :150], without[1, :150])


@pytest.mark.parametrize("cap", [1e-45, 1e-40, 1e37, 3e38])
def test_weights_at_caps_whose_ratio_to_the_scale_is_no_normal_number(cuda_device, cap):
    c = Case(44, [9, 40], [200, 70]).spoil_unused()
    c.q[3] = 0
    lse = c.attention(cap)[1].float()
    got, status = run_weights(c, cuda_device, lse, cap=cap)
    want = weights(c, lse, None, cap)
    assert ((got.cpu().double() - want).abs() <= 1e-5 * want + 1e-12).all() and not status.any()


@pytest.mark.parametrize("budget,sink,recent", [(20_000, 4, 512), (32_768, 0, 0), (100, 0, 100)])
def test_evict_of_caches_longer_than_shared_memory_holds(cuda_device, budget, sink, recent):
    """Weights of up to 32,768 slots are held in shared memory, longer ones are read where they lie; both in one call."""
    rng = np.random.default_rng(7)
    c = Case(45, [1] * 5, [100_000, 9, 32_768, 32_769, 40_001], Hq=1, Hkv=1, page=64)
    W = 100_000
    w = np.exp(2 * rng.standard_normal((c.B, W))).astype(np.float32)
    check_evict(c, cuda_device, w, budget, sink, recent)
    check_evict(c, cuda_device, rng.integers(0, 4, (c.B, W)).astype(np.float32), budget, sink, recent, inplace=True)     # ties
    w = rng.standard_normal((c.B, W)).astype(np.float32)
    w[:, ::3], w[:, 1::7], w[:, 2::11] = np.nan, -np.inf, -0.0
    check_evict(c, cuda_device, w, budget, sink, recent)


def test_offsets_that_pass_32_bits(cuda_device):
    """A cache of more than 2^31 values whose pages in use are its last ones, and rows of nodes 2^26 values apart: through
    every call on a cache, against the same calls on compact arrays."""
    c = Case(46, [40, 3], [150, 90], Hq=8, Hkv=2, D=128, room=40, chain=True)
    dev, d = cuda_device, c.on(cuda_device)
    pages = 2**31 // c.k[0].numel() + 100
    shift = pages - c.k.shape[0]
    big = {}
    for name in ("k", "v"):
        big[name] = torch.empty((pages, *c.k.shape[1:]), dtype=c.dtype, device=dev)
        big[name][shift:] = d[name]
    assert big["k"].numel() > 2**31
    wide = torch.empty((c.M, 2**26), dtype=c.dtype, device=dev)
    at = 0
    for name, heads in (("q", 8), ("tk", 2), ("tv", 2), ("out", 8)):
        big[name] = wide[:, at:at + heads * 128].view(c.M, heads, 128)
        at += heads * 128
        if name != "out":
            big[name].copy_(d[name])
    used = (torch.arange(c.table.shape[1])[None] < torch.from_numpy(-(-(c.lens + 40) // c.page))[:, None]).to(dev)
    big["table"] = torch.where(used, d["table"] + shift, 2**30)
    path_len = torch.tensor([33, 2], dtype=torch.int32, device=dev)
    results = []
    for x in (d, {**d, **big}):
        att = ssd.alloc_tree_attention_outputs(c.M, 2, 8, 128, c.dtype, dev, 2, c.max_nodes)
        att["out"] = x.get("out", att["out"])
        ssd.ssd_tree_attention(x["q"], x["tk"], x["tv"], x["k"], x["v"], x["table"], x["lens"], x["off"], c.max_nodes, None, out=att)
        weight = torch.zeros(2, 200, device=dev)
        ssd.ssd_cache_weights(x["q"], att["lse"], x["k"], x["table"], x["lens"], x["off"], c.max_nodes, weight)
        app = ssd.ssd_cache_append(x["tk"], x["tv"], x["off"], None, path_len, x["k"], x["v"], x["table"], x["lens"], weight)
        evi = ssd.ssd_cache_evict(x["k"], x["v"], x["table"], app["new_len"], weight, 64, 2, 8)
        results.append(cpu(dict(out=att["out"], lse=att["lse"], weight=weight, k=x["k"][-c.k.shape[0]:], v=x["v"][-c.k.shape[0]:],
                                **{"evict " + k: v for k, v in evi.items()})))
    for k in results[0]:
        assert torch.equal(results[0][k], results[1][k]), k
    assert (results[0]["evict new_len"] == 64).all() and not results[0]["evict utt_status"].any()
