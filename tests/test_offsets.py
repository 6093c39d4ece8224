"""Utterance offsets are the caller's data: which row a closing kernel fetches ahead of the streaming
kernel's end, for offsets of every kind, from the very functions the kernels call."""
import ctypes as C
import itertools
import os
import subprocess

import pytest
import torch

import helpers as H
from conftest import ROOT
from paper_2603_11243_b200 import binding as ssd

INT64_MAX, INT64_MIN = (1 << 63) - 1, -(1 << 63)
SOURCE = """
#include "ssd_ranges.cuh"
extern "C" long long row(long long i0, long long i1, long long M, int k) {
    return ssd::ranges::row_of_utterance(i0, i1, M, k);
}
extern "C" int path(int *p, unsigned char *on, int n, int node, int depth, const int *parent) {
    return ssd::ranges::write_path(p, on, n, node, depth, [&](int j) { return parent[j]; });
}
extern "C" void tell(unsigned *status, int B, unsigned bits, int first, int step) {
    ssd::ranges::tell_all(status, B, bits, first, step);
}
extern "C" int sound(long long i0, long long i1, long long M) { return ssd::ranges::rows_sound(i0, i1, M); }
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("ranges")
    (d / "r.cpp").write_text(SOURCE)
    # -ftrapv: signed arithmetic that overflows on the way ends the process
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-ftrapv", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2603_11243_b200", "csrc"), str(d / "r.cpp"), "-o", str(d / "r.so")],
                   check=True)
    lib = C.CDLL(str(d / "r.so"))
    lib.row.restype = C.c_longlong
    lib.row.argtypes = [C.c_longlong, C.c_longlong, C.c_longlong, C.c_int]
    lib.sound.argtypes = [C.c_longlong] * 3
    return lib


def test_rows_fetched_ahead_lie_inside_the_matrix(host):
    ends = [INT64_MIN, INT64_MIN + 500, -1, 0, 1, 3, 7, 30, 31, 1 << 31, INT64_MAX - 1024, INT64_MAX - 5, INT64_MAX]
    for M, i0, i1 in itertools.product((0, 1, 7, 30), ends, ends):
        inside = 0 <= i0 <= i1 <= M
        assert bool(host.sound(i0, i1, M)) == inside
        for k in (0, 1, 6, 29, 30, 511, 1023):
            want = i0 + k if inside and k < i1 - i0 else -1
            assert host.row(i0, i1, M, k) == want, (M, i0, i1, k)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", [0, 1, 2])
def test_offsets_at_the_ends_of_int64(cuda_device, kernel):
    """Flagged and treated as empty, the sound utterances beside them unharmed."""
    M, V, dev = 30, 900, cuda_device
    g = torch.Generator().manual_seed(9)
    x = torch.randn((M, V), generator=g).bfloat16().to(dev)
    ids = x.float().argmax(1).to(torch.int32)
    off = torch.tensor([0, 10, INT64_MAX - 100, 20, 30, INT64_MIN + 100, 5, INT64_MAX, INT64_MAX - 1000, 12, 30],
                       dtype=torch.int64, device=dev)
    bad = [0, 1, 1, 0, 1, 1, 1, 1, 1, 0]
    lens = [10, 0, 0, 10, 0, 0, 0, 0, 0, 18]
    o = H.opts(kernel=kernel)
    v = ssd.ssd_verify(x, off, ids, 0.0, opts=o)
    e = ssd.ssd_verify_early_exit(x, off, ids, 0.0, opts=o)
    stats = ssd.ssd_verify_shard(x, 0, off, ids, opts=o)
    c = ssd.ssd_verify_combine(stats[None], V, off, ids, 0.0)
    torch.cuda.synchronize()
    for out in (v, e, c):
        assert H.status_u32(out["utt_status"]).tolist() == [ssd.UTT_BAD_OFFSETS * b for b in bad]
        assert out["accepted_len"].tolist() == lens
        assert out["all_accepted"].tolist() == [1 - b for b in bad]


def test_a_path_stays_inside_its_utterance(host):
    """Whatever a tree's closing kernel is left with where utterances name the same rows: depths above the number of
    nodes, parents out of range, nodes that are none."""
    wild = [-(1 << 31), -7, -1, 0, 1, 2, 3, 4, 5, 6, 900, (1 << 31) - 1]
    guard = 16
    for n, node, depth in itertools.product((0, 1, 5), wild, wild):
        for up in wild:
            parents = (C.c_int * (n + 2 * guard))(*[up] * (n + 2 * guard))
            p, on = (C.c_int * (n + 2 * guard))(*[77] * (n + 2 * guard)), (C.c_ubyte * (n + 2 * guard))(*[77] * (n + 2 * guard))
            at = lambda a, size: C.byref(a, guard * size)  # noqa: E731
            length = host.path(at(p, 4), at(on, 1), n, node, depth, at(parents, 4))
            assert 0 <= length <= n
            for a in (p, on):
                assert list(a[:guard]) == [77] * guard and list(a[guard + n:]) == [77] * guard
    parents = (C.c_int * 6)(-1, 0, 0, 2, 1, 3)
    p, on = (C.c_int * 6)(*[-1] * 6), (C.c_ubyte * 6)()
    assert host.path(p, on, 6, 5, 4, parents) == 4 and list(p) == [0, 2, 3, 5, -1, -1] and list(on) == [1, 0, 1, 1, 0, 1]


def test_every_utterance_is_told_that_a_wait_ran_out(host):
    """Those that the failing CTA never began among them."""
    for B in (0, 1, 255, 256, 257, 4500):
        status = (C.c_uint * (B + 300))(*[5] * (B + 300))
        for thread in range(256):
            host.tell(status, B, C.c_uint(ssd.UTT_INTERNAL), thread, 256)
        assert list(status) == [ssd.UTT_INTERNAL] * B + [5] * 300
    source = open(os.path.join(ROOT, "paper_2603_11243_b200", "csrc", "ssd_tree.cu")).read()
    assert "if (cut.failed && slice == 0) ranges::tell_all(p.status, p.B, SSD_UTT_INTERNAL," in source


@pytest.mark.gpu
@pytest.mark.parametrize("chain", [True, False])
def test_trees_of_utterances_that_name_the_same_rows(cuda_device, chain):
    """More nodes than are held in shared memory, so that the two utterances overwrite each other's depths: lengths and
    entries stay in range, and nothing beside the rows is touched."""
    V, n, dev = 40, 3000, cuda_device
    off = torch.tensor([0, 2400, 300, n], dtype=torch.int64, device=dev)      # [0, 2400), malformed, [300, 3000)
    g = torch.Generator().manual_seed(12)
    x = torch.randn((n, V), generator=g).to(dev)
    ids = x.argmax(1).to(torch.int32)
    parent = None if chain else (torch.arange(n, dtype=torch.int32, device=dev) - 1) // 3 - 120
    wide = {k: torch.full((n + 512,), 77, dtype=t, device=dev) for k, t in (("path", torch.int32), ("on_path", torch.uint8))}
    out = ssd.alloc_verify_tree_outputs(n, 3, dev, ssd.ssd_verify_workspace_bytes(3, n, V, ssd.F32))
    for k in wide:
        out[k] = wide[k][256:256 + n]
    for _ in range(20):
        ssd.ssd_verify_tree(x, off, ids, parent, 0.0, out=out)
    torch.cuda.synchronize()
    length = out["path_len"].tolist()
    assert 0 <= length[0] <= 2400 and length[1] == 0 and 0 <= length[2] <= 2700
    assert out["path"].min() >= -1 and out["path"].max() < 2700 and out["on_path"].max() <= 1
    for w in wide.values():
        assert (w[:256] == 77).all() and (w[256 + n:] == 77).all()
