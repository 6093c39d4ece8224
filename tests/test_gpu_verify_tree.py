"""ssd_verify_tree against the definition in 64 bits.  Float outputs are held to the suite's 1e-4; the paths have to
be what the returned log-likelihoods lead to, bit for bit."""
import numpy as np
import pytest
import torch

import helpers as H
from paper_2603_11243_b200 import binding as ssd
from tree_ref import planted, random_parents, verify_tree

pytestmark = pytest.mark.gpu


def batch(seed, n, V, dtype, chain=False, likely=0.75, roots=1):
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
    parent = np.concatenate([np.arange(-1, k - 1) if chain else random_parents(rng, k, roots) for k in n] +
                            [np.zeros(0)]).astype(np.int32)
    x, ids = planted(rng, off, parent, V, likely)
    t = torch.from_numpy(x).to(dtype)
    return t, off, ids, parent


def run(dev, t, off, ids, parent, tau=0.02, **kw):
    put = lambda a: torch.from_numpy(a).to(dev)  # noqa: E731
    r = ssd.ssd_verify_tree(t.to(dev), put(off), put(ids), None if parent is None else put(parent), tau, **kw)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in r.items()}


def check(r, t, off, ids, parent, tau=0.02):
    logp, lse, path, length, on = verify_tree(t.double().numpy(), off, ids, parent, tau, r["token_logp"])
    fine = np.isfinite(logp)
    assert (np.abs(r["token_logp"][fine] - logp[fine]) <= H.FLOAT_TOL).all()
    assert np.array_equal(r["token_logp"][~fine], logp[~fine])
    assert (np.abs(r["row_lse"] - lse) <= H.FLOAT_TOL).all()
    assert np.array_equal(r["path"], path) and np.array_equal(r["path_len"], length) and np.array_equal(r["on_path"], on)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [([1], 50), ([8], 32000), ([0, 5, 0, 33], 1025), ([31, 32, 33, 64, 65, 200], 349), ([12] * 40, 2048)])
def test_trees(cuda_device, dtype, n, V):
    a = batch(1, n, V, dtype)
    check(run(cuda_device, *a), *a)


@pytest.mark.parametrize("n", [[1, 0, 40, 90], [1024], [1025, 3], [2500]])
@pytest.mark.parametrize("explicit", [True, False])
def test_chains_of_any_length(cuda_device, n, explicit):
    """Also without a reject: the path is then the whole chain.  Over 1,024 nodes the state lies in `path`."""
    for likely in (0.97, 1.0):
        t, off, ids, parent = batch(2, n, 300, torch.float32, chain=True, likely=likely)
        check(run(cuda_device, t, off, ids, parent if explicit else None), t, off, ids, parent)


def test_large_bushy_tree_and_several_given_nodes(cuda_device):
    a = batch(3, [3000, 700], 100, torch.float32, likely=0.9, roots=5)
    check(run(cuda_device, *a), *a)


@pytest.mark.parametrize("tau", [0.0, -1.0, 1.0])
def test_thresholds_that_accept_all_or_nothing(cuda_device, tau):
    a = batch(4, [9, 40, 0], 600, torch.bfloat16)
    check(run(cuda_device, *a, tau=tau), *a, tau=tau)


def test_of_equal_paths_the_lowest_node(cuda_device):
    off, parent = np.array([0, 7], np.int64), np.array([-1, 0, 0, 1, 2, 2, 1], np.int32)
    rng = np.random.default_rng(5)
    x, ids = planted(rng, off, parent, 500, likely=1.0)
    t = torch.from_numpy(x)
    r = run(cuda_device, t.float(), off, ids, parent)
    assert r["path"].tolist() == [0, 1, 3, -1, -1, -1, -1] and r["path_len"].tolist() == [3]


def test_a_chain_is_what_ssd_verify_accepts(cuda_device):
    """ssd_verify's rows predict their own token: a chain with the context's last token in front has them one up."""
    rng = np.random.default_rng(6)
    K, V = 37, 1000
    off, parent = np.array([0, K + 1], np.int64), np.arange(-1, K, dtype=np.int32)
    x, ids = planted(rng, off, parent, V, likely=0.9)
    r = run(cuda_device, torch.from_numpy(x).float(), off, ids, parent)
    v = ssd.ssd_verify(torch.from_numpy(x[:K]).float().to(cuda_device), torch.tensor([0, K], device=cuda_device),
                       torch.from_numpy(ids[1:]).to(cuda_device), 0.02)
    assert np.array_equal(v["token_logp"].cpu().numpy(), r["token_logp"][1:])
    assert int(v["accepted_len"][0]) + 1 == r["path_len"][0]


def test_statuses_and_skip(cuda_device):
    n = [6, 6, 6, 6, 6]
    t, off, ids, parent = batch(7, n, 400, torch.float32, likely=1.0)
    ids[8], parent[off[2] + 3], parent[off[2] + 4] = 400, 3, -7
    t[off[3] + 1, 7] = float("nan")
    skip = np.array([0, 0, 0, 0, 1], np.uint8)
    out = ssd.alloc_verify_tree_outputs(30, 5, cuda_device, ssd.ssd_verify_workspace_bytes(5, 30, 400, ssd.F32))
    out["token_logp"].fill_(9.0)
    r = run(cuda_device, t, off, ids, parent, skip=torch.from_numpy(skip).to(cuda_device), out=out)
    assert r["utt_status"].tolist() == [0, ssd.UTT_BAD_DRAFT_ID, ssd.UTT_BAD_PARENT, ssd.UTT_NONFINITE, 0]
    assert r["token_logp"][8] == -np.inf and (r["token_logp"][off[2] + 3:off[2] + 5] == -np.inf).all()
    assert (r["token_logp"][24:] == 9.0).all() and r["path_len"][4] == 0
    assert (r["path"][24:] == -1).all() and (r["on_path"][24:] == 0).all()
    bad = np.array([0, 6, 3, 18, 31, 30], np.int64)
    r = run(cuda_device, t, bad, ids, parent)
    assert (r["utt_status"][[1, 3, 4]] & ssd.UTT_BAD_OFFSETS).all() and (r["path_len"][[1, 3, 4]] == 0).all()


def test_padded_rows_and_launch_options(cuda_device):
    t, off, ids, parent = batch(8, [20, 3, 11], 515, torch.bfloat16)
    wide = torch.full((t.shape[0], 600), float("nan"), dtype=t.dtype)
    wide[:, 3:518] = t
    x = wide.to(cuda_device)[:, 3:518]
    put = lambda a: torch.from_numpy(a).to(cuda_device)  # noqa: E731
    for o in (None, H.opts(kernel=1), H.opts(split=3, warps=8)):
        r = ssd.ssd_verify_tree(x, put(off), put(ids), put(parent), 0.02, opts=o)
        check({k: v.cpu().numpy() for k, v in r.items()}, t, off, ids, parent)
    with pytest.raises(ssd.SsdError) as e:
        ssd.ssd_verify_tree(x, put(off), put(ids), put(parent), 0.02, opts=H.opts(finish=2))
    assert e.value.code == ssd.ERR_ARG
