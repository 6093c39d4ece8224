"""ssd_tree_attention against the definition in 64 bits.

Tolerances.  Scores are sums of D exact products of two 16-bit values in fp32 and one fp32 scaling; with
|q.k| terms of a few units their absolute error stays below 1e-5, which is the relative error of every
probability and the absolute error of the log-sum-exp (held to 2e-5 plus 2^-23 of its size).  An output is
a mean of values v with weights p: each p is rounded once to the 16-bit type (relative half step u = 2^-8 or
2^-11, so the error is at most u * sum p |v|), and so is the result (u * |out|): the bound is
u * (mean |v| + |out|) with a tenth more for the rest."""
import numpy as np
import pytest
import torch

from paper_2603_11243_b200 import binding as ssd
from tree_ref import Case, lines

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def run(c, dev, cap=0.0, d=None, **kw):
    d = d or c.on(dev)
    r = ssd.ssd_tree_attention(d["q"], d["tk"], d["tv"], d["k"], d["v"], d["table"], d["lens"], d["off"], c.max_nodes,
                               d["parent"], c.scale, cap, **kw)
    torch.cuda.synchronize()
    return r


def check(c, r, cap=0.0, rows=None):
    out, lse = c.attention(cap)
    keep = c.v, c.tv
    c.v, c.tv = c.v.abs(), c.tv.abs()
    mean, _ = c.attention(cap)
    c.v, c.tv = keep
    u = HALF_STEP[c.dtype]
    rows = slice(None) if rows is None else rows
    got, want = r["out"].cpu().double()[rows], out[rows]
    bound = 1.1 * u * (mean[rows] + want.abs()) + 1e-6
    worst = ((got - want).abs() / bound).max().item() if got.numel() else 0.0
    assert worst <= 1.0, worst
    dl = (r["lse"].cpu().double()[rows] - lse[rows]).abs()
    assert (dl <= 2e-5 + 2.0 ** -23 * lse[rows].abs()).all(), dl.max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,lens", [([1], [1]), ([1], [0]), ([1], [1000]), ([5], [128]), ([7, 0, 3], [130, 50, 0]),
                                    ([20, 31, 17], [700, 127, 257])])
def test_against_64_bits(cuda_device, dtype, D, n, lens):
    c = Case(1, n, lens, D=D, dtype=dtype).spoil_unused()
    r = run(c, cuda_device)
    check(c, r)
    assert (r["utt_status"] == 0).all()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (5, 1), (28, 4), (6, 2), (16, 1), (128, 1)])
def test_head_layouts(cuda_device, Hq, Hkv):
    c = Case(2, [9, 3, 40], [200, 33, 300], Hq=Hq, Hkv=Hkv).spoil_unused()
    check(c, run(c, cuda_device))


@pytest.mark.parametrize("page", [1, 3, 8, 20, 24, 64, 100, 128, 129, 200, 256, 1000])
def test_pages_that_end_inside_a_tile(cuda_device, page):
    c = Case(3, [4, 9, 2], [301, 127, 129], page=page).spoil_unused()
    check(c, run(c, cuda_device))


@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("n", [[33], [64, 65], [130, 1, 257], [300]])
def test_more_nodes_than_a_tile(cuda_device, n, chain):
    """G = 4: 32 nodes a tile, and two tiles to a CTA; over 128 nodes the tree's keys are several tiles, over 256
    its parents are not all in shared memory."""
    c = Case(4, n, [90] * len(n), chain=chain, roots=2 if not chain else 1, dtype=torch.float16, D=128).spoil_unused()
    check(c, run(c, cuda_device))


def test_many_items_leave_no_cluster(cuda_device):
    """More items than multiprocessors: one CTA for each, both with one tile of queries and with two."""
    rng = np.random.default_rng(5)
    c = Case(5, rng.integers(0, 24, 41), rng.integers(0, 400, 41), Hq=16, Hkv=8).spoil_unused()
    check(c, run(c, cuda_device))
    c = Case(6, rng.integers(0, 150, 11), rng.integers(0, 400, 11), Hq=16, Hkv=8, chain=True, D=128).spoil_unused()
    check(c, run(c, cuda_device))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_capped_scores(cuda_device, dtype):
    for spread in (2.0, 30.0):
        c = Case(7, [9, 70], [400, 90], dtype=dtype, spread=spread).spoil_unused()
        check(c, run(c, cuda_device, cap=20.0), cap=20.0)


def test_long_flat_tail_in_fp16(cuda_device):
    """One score far above thousands of equal small ones, whose probabilities fp16 could not hold as they are."""
    c = Case(8, [3], [6000], dtype=torch.float16, Hq=2, Hkv=1)
    c.q.fill_(1.0)
    c.k.normal_(0.0, 0.01)
    c.tk.zero_()
    c.k[c.table[0, 0], 0] = 2.2                                  # score 17.6: the others' p is 2e-8 each
    check(c, run(c, cuda_device))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n,lens", [([6, 5], [20, 0]), ([140, 5], [20, 300]), ([6], [3000])])
def test_what_a_node_does_not_see_cannot_reach_it(cuda_device, bad, n, lens):
    c = Case(9, n, lens).spoil_unused()
    d = c.on(cuda_device)
    clean = run(c, cuda_device, d=d)
    j = 3                                                        # a node of utterance 0, and who descends from it
    below = [i for i in range(n[0]) if any(j == a for a in __import__("tree_ref").lines(c.parent[:n[0]])[i])]
    others = [i for i in range(c.M) if i not in below]
    for name in ("tk", "tv"):
        e = dict(d, **{name: d[name].clone()})
        e[name][j, :, 5] = bad
        r = run(c, cuda_device, d=e)
        assert torch.equal(r["out"][others], clean["out"][others])
        assert torch.equal(r["lse"][others], clean["lse"][others])
        if name == "tv":
            hit = r["out"][below][..., 5].float()
            assert (torch.isnan(hit) if bad != bad else torch.isinf(hit)).all()
            assert torch.isfinite(r["out"][below][..., :5].float()).all()


def test_strided_and_partial_inputs(cuda_device):
    """q, keys and values as slices of one fused projection, K and V caches interleaved, out inside a wider array."""
    c = Case(10, [9, 33], [100, 257], Hq=8, Hkv=2, D=64)
    d = c.on(cuda_device)
    fused = torch.randn(c.M, 8 + 2 + 2, 64, device=cuda_device).to(c.dtype)
    fused[:, :8], fused[:, 8:10], fused[:, 10:] = d["q"], d["tk"], d["tv"]
    d.update(q=fused[:, :8], tk=fused[:, 8:10], tv=fused[:, 10:])
    both = torch.empty(c.k.shape[0], 2, *c.k.shape[1:], dtype=c.dtype, device=cuda_device)
    both[:, 0], both[:, 1] = d["k"], d["v"]
    d.update(k=both[:, 0], v=both[:, 1])
    wide = torch.full((c.M, 10, 72), 7.0, dtype=c.dtype, device=cuda_device)
    out = ssd.alloc_tree_attention_outputs(c.M, 2, 8, 64, c.dtype, cuda_device)
    out["out"] = wide[:, 1:9, :64]
    r = run(c, cuda_device, d=d, out=out)
    check(c, r)
    assert (wide[:, 0] == 7).all() and (wide[:, 9] == 7).all() and (wide[:, :, 64:] == 7).all()


def test_head_major_cache(cuda_device):
    c = Case(11, [3, 4], [40, 70])
    d = c.on(cuda_device)
    for k in ("k", "v"):
        d[k] = d[k].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)          # [pages, heads, slots, D] in memory
    check(c, run(c, cuda_device, d=d))


def test_malformed_utterances(cuda_device):
    c = Case(12, [4, 5, 6, 7], [50, 60, 70, 80])
    d = c.on(cuda_device)
    clean = run(c, cuda_device, d=d)
    # a parent out of range counts as none; a bad page and a bad length are reported and stay inside the cache
    e = dict(d, parent=d["parent"].clone(), table=d["table"].clone(), lens=d["lens"].clone())
    e["parent"][c.off[1] + 2] = 2
    e["parent"][c.off[1] + 3] = -5
    e["table"][2, 1] = c.k.shape[0]
    e["lens"][3] = c.table.shape[1] * c.page + 1
    r = run(c, cuda_device, d=e)
    assert r["utt_status"].cpu().tolist() == [0, ssd.UTT_BAD_PARENT, ssd.UTT_BAD_CACHE, ssd.UTT_BAD_CACHE]
    assert torch.equal(r["out"][:4], clean["out"][:4])
    c.parent[c.off[1] + 2] = c.parent[c.off[1] + 3] = -1
    check(c, dict(out=r["out"], lse=r["lse"]), rows=slice(0, 9))
    # offsets that run backwards, and more nodes than were announced: rows are left as they were
    off = torch.tensor([0, 4, 2, 15, 22], dtype=torch.int64, device=cuda_device)
    out = ssd.alloc_tree_attention_outputs(c.M, c.B, c.Hq, c.D, c.dtype, cuda_device)
    out["out"].fill_(3.0)
    r = ssd.ssd_tree_attention(d["q"], d["tk"], d["tv"], d["k"], d["v"], d["table"], d["lens"], off, 7, d["parent"], out=out)
    assert r["utt_status"].cpu().tolist() == [0, ssd.UTT_BAD_OFFSETS, ssd.UTT_BAD_OFFSETS, 0]
    assert (r["out"][4:15] == 3.0).all() and torch.equal(r["out"][:4], clean["out"][:4])


def test_without_a_cache(cuda_device):
    c = Case(13, [9, 4], [0, 0], D=128)
    d = c.on(cuda_device)
    d.update(k=d["k"][:0], v=d["v"][:0], table=d["table"][:, :0])
    check(c, run(c, cuda_device, d=d))
    none = ssd.ssd_tree_attention(d["q"][:0], d["tk"][:0], d["tv"][:0], d["k"], d["v"], d["table"][:0], d["lens"][:0],
                                  d["off"][:1], 0, None)
    assert none["out"].shape == (0, c.Hq, c.D)


def test_captured_and_on_two_streams(cuda_device):
    c = Case(14, [9, 70, 3], [500, 90, 1200])
    other = Case(15, [30, 2, 50], [100, 1000, 20])
    d, e = c.on(cuda_device), other.on(cuda_device)
    want, want2 = run(c, cuda_device, d=d), run(other, cuda_device, d=e)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(10):
        got = []
        for s, x, y in zip(streams, (c, other), (d, e)):
            with torch.cuda.stream(s):
                got.append(ssd.ssd_tree_attention(y["q"], y["tk"], y["tv"], y["k"], y["v"], y["table"], y["lens"], y["off"],
                                                  x.max_nodes, y["parent"]))
        torch.cuda.synchronize()
        assert torch.equal(got[0]["out"], want["out"]) and torch.equal(got[1]["out"], want2["out"])
    out = ssd.alloc_tree_attention_outputs(c.M, c.B, c.Hq, c.D, c.dtype, cuda_device)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ssd.ssd_tree_attention(d["q"], d["tk"], d["tv"], d["k"], d["v"], d["table"], d["lens"], d["off"], c.max_nodes,
                               d["parent"], out=out)
    out["out"].zero_()
    d["lens"][0] = 77                                              # a replay takes what is in the buffers then
    graph.replay()
    torch.cuda.synchronize()
    c.lens[0] = 77
    check(c, out)


def test_one_long_cache_cut_into_as_many_parts_as_there_are(cuda_device):
    """One kv head and one utterance: every CTA has a part of the same item."""
    c = Case(30, [2], [40_001], Hq=2, Hkv=1, page=64, dtype=torch.float16).spoil_unused()
    check(c, run(c, cuda_device))


def test_more_utterances_than_costs_are_held_for(cuda_device):
    rng = np.random.default_rng(31)
    B = 4500                                                      # 4,096 are held in front of the walk where heads have 64 values
    c = Case(31, rng.integers(0, 3, B), rng.integers(0, 20, B), Hq=2, Hkv=1, page=8)
    r = run(c, cuda_device)
    check(c, r)
    assert (r["utt_status"] == 0).all()


@pytest.mark.parametrize("cap", [1e-30, 1e-3, 1.0, 1e6])
def test_caps_of_any_size(cuda_device, cap):
    c = Case(32, [9, 40], [200, 70], spread=10.0).spoil_unused()
    check(c, run(c, cuda_device, cap=cap), cap=cap)


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1.0])
def test_scales_of_any_size(cuda_device, scale):
    c = Case(33, [9, 40], [200, 70], spread=1.0 if scale < 1 else 0.25).spoil_unused()
    c.scale = scale
    check(c, run(c, cuda_device))


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(cuda_device, seed):
    rng = np.random.default_rng(100 + seed)
    B, Hkv = int(rng.integers(1, 9)), int(rng.integers(1, 5))
    chain = bool(rng.random() < 0.4)
    top = int(rng.choice([1, 4, 40, 140]))
    c = Case(200 + seed, rng.integers(0, top + 1, B), rng.integers(0, int(rng.choice([2, 130, 700])), B), Hq=Hkv * int(rng.choice([1, 2, 3, 4, 8])),
             Hkv=Hkv, D=int(rng.choice([64, 128])), page=int(rng.choice([1, 5, 8, 16, 40, 64, 128, 160])),
             dtype=torch.bfloat16 if rng.random() < 0.5 else torch.float16, chain=chain, roots=1 if chain else int(rng.integers(1, 4))).spoil_unused()
    cap = float(rng.choice([0.0, 0.0, 10.0]))
    r = run(c, cuda_device, cap=cap)
    check(c, r, cap=cap)
    again = run(c, cuda_device, cap=cap)
    assert torch.equal(r["out"], again["out"]) and torch.equal(r["lse"], again["lse"])


def test_rows_behind_the_last_utterance_are_left_alone(cuda_device):
    c = Case(34, [5, 6], [30, 40])
    d = c.on(cuda_device)
    more = lambda x: torch.cat([x, torch.full_like(x[:7], float("nan"))])  # noqa: E731
    e = dict(d, q=more(d["q"]), tk=more(d["tk"]), tv=more(d["tv"]), parent=torch.cat([d["parent"], d["parent"][:7]]))
    out = ssd.alloc_tree_attention_outputs(c.M + 7, c.B, c.Hq, c.D, c.dtype, cuda_device)
    out["out"].fill_(5.0)
    out["lse"].fill_(6.0)
    r = run(c, cuda_device, d=e, out=out)
    check(c, dict(out=r["out"][:c.M], lse=r["lse"][:c.M]))
    assert (r["out"][c.M:] == 5.0).all() and (r["lse"][c.M:] == 6.0).all()


def test_without_lse_and_a_workspace_left_over(cuda_device):
    c = Case(35, [12, 3], [900, 500], Hq=4, Hkv=1)
    want = run(c, cuda_device)["out"]
    out = ssd.alloc_tree_attention_outputs(c.M, c.B, c.Hq, c.D, c.dtype, cuda_device, 1, c.max_nodes)
    out["workspace"].fill_(255)
    del out["lse"]
    assert torch.equal(run(c, cuda_device, out=out)["out"], want)
    out["workspace"] = out["workspace"][:256]
    with pytest.raises(ssd.SsdError) as e:
        run(c, cuda_device, out=out)
    assert e.value.code == ssd.ERR_WORKSPACE


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("n,lens", [([6, 5], [20, 0]), ([140, 5], [20, 300]), ([6], [3000])])
def test_a_query_of_nan_stays_its_own(cuda_device, cap, n, lens):
    """The rows of a tile share their accumulators and their warps' choices: one head of one node is NaN, it alone is in
    the results, and everything else is right."""
    c = Case(36, n, lens).spoil_unused()
    d = c.on(cuda_device)
    d["q"][2, 1, 3] = float("nan")
    r = run(c, cuda_device, cap=cap, d=d)
    assert torch.isnan(r["out"][2, 1].float()).all() and torch.isnan(r["lse"][2, 1])
    whole = run(c, cuda_device, cap=cap)
    r["out"][2, 1], r["lse"][2, 1] = whole["out"][2, 1], whole["lse"][2, 1]
    check(c, r, cap)


@pytest.mark.parametrize("chain", [True, False])
def test_many_items_of_one_and_of_two_tiles(cuda_device, chain):
    """Several items to a multiprocessor, of one tile of queries and of two in any order, trees that are walked and trees
    that are not: what an item leaves in shared memory is not the next one's."""
    rng = np.random.default_rng(37)
    n = rng.choice([1, 5, 31, 33, 40, 64, 65, 100, 130], 160)
    c = Case(37, n, rng.integers(0, 300, 160), Hq=8, Hkv=2, D=64, chain=chain, roots=1 if chain else 3).spoil_unused()
    d = c.on(cuda_device)
    clean = run(c, cuda_device, d=d)
    check(c, clean)
    off = c.off
    d["tv"][torch.as_tensor(off[:-1:7], device=cuda_device), 1, 9] = float("nan")       # an utterance's first node
    r = run(c, cuda_device, d=d)
    hit = torch.zeros(c.M, dtype=torch.bool)
    for b in range(0, 160, 7):
        for i, line in enumerate(lines(c.parent[off[b]:off[b + 1]])):
            hit[off[b] + i] = 0 in line
    got, want = r["out"].cpu(), clean["out"].cpu()
    assert torch.isnan(got[hit][:, 4:, 9]).all()
    got[hit, 4:, 9] = want[hit, 4:, 9]
    assert torch.equal(got, want) and torch.equal(r["lse"], clean["lse"])


@pytest.mark.parametrize("cap", [1e-45, 1e-40, 1e37, 3e38])
def test_caps_whose_ratio_to_the_scale_is_no_normal_number(cuda_device, cap):
    """scale / cap leaves fp32's range: scores of 0 stay 0 (not 0 * inf), and a cap far above every score changes none."""
    c = Case(42, [9, 40], [200, 70], spread=10.0).spoil_unused()
    c.q[3] = 0
    check(c, run(c, cuda_device, cap=cap), cap=cap)


def test_broadcast_heads_and_rows(cuda_device):
    """Strides of 0: one kv head for all (keys, values and cache), one row of queries for every node."""
    c = Case(43, [9, 40], [200, 70], Hq=8, Hkv=2)
    for name in ("k", "v", "tk", "tv"):
        x = getattr(c, name)
        x[..., 1, :] = x[..., 0, :]
    c.q[:] = c.q[:1].clone()
    d = c.on(cuda_device)
    for name in ("k", "v", "tk", "tv"):
        d[name] = d[name][..., :1, :].contiguous().expand(d[name].shape)
    d["q"] = d["q"][:1].contiguous().expand(d["q"].shape)
    assert d["tk"].stride(1) == 0 and d["k"].stride(2) == 0 and d["q"].stride(0) == 0
    check(c, run(c, cuda_device, d=d))
