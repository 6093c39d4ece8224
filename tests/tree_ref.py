"""Draft trees and their cache in 64 bits on the CPU, utterance by utterance from the definitions, and
random cases of them.  Nothing here uses the library."""
import math

import numpy as np
import torch


def lines(parent):
    """Every node's line of descent, first node first; a parent out of range is none."""
    out = []
    for i, p in enumerate(parent):
        out.append((out[p] if 0 <= p < i else []) + [i])
    return out


def random_parents(rng, n, roots=1):
    p = np.full(n, -1, np.int32)
    for i in range(roots, n):
        p[i] = i - 1 if rng.random() < 0.5 else rng.integers(0, i)
    return p


class Case:
    """A batch: nodes, trees and a paged cache with pages in random order.  Tensors lie on the CPU."""

    def __init__(self, seed, n, lens, Hq=8, Hkv=2, D=64, page=16, dtype=torch.bfloat16, chain=False, room=0, spread=2.0,
                 spare=3, roots=1):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.n, self.lens = np.asarray(n, np.int64), np.asarray(lens, np.int64)
        self.B, self.M = len(n), int(np.sum(n))
        self.Hq, self.Hkv, self.D, self.page, self.dtype, self.chain = Hq, Hkv, D, page, dtype, chain
        self.off = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int64)
        self.parent = np.concatenate([np.arange(-1, k - 1, dtype=np.int32) if chain else random_parents(rng, k, roots)
                                      for k in n] + [np.zeros(0, np.int32)]).astype(np.int32)
        need = -(-(self.lens + room) // page)
        pages = int(need.sum()) + spare
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((self.B, max(1, int(need.max(initial=0)))), 2**30, np.int32)      # behind the length: never looked at
        at = 0
        for b in range(self.B):
            self.table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
        r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.q = (spread * r(self.M, Hq, D)).to(dtype)
        self.tk, self.tv = r(self.M, Hkv, D).to(dtype), r(self.M, Hkv, D).to(dtype)
        self.k, self.v = r(pages, page, Hkv, D).to(dtype), r(pages, page, Hkv, D).to(dtype)
        self.scale = D ** -0.5
        self.max_nodes = int(self.n.max(initial=0))

    def spoil_unused(self):
        """NaN in every slot of the cache that no utterance uses."""
        used = torch.zeros(self.k.shape[:2], dtype=torch.bool)
        for b in range(self.B):
            for s in range(int(self.lens[b])):
                used[self.table[b, s // self.page], s % self.page] = True
        self.k[~used] = math.nan
        self.v[~used] = math.inf
        return self

    def slots(self, pool, b):
        s = np.arange(int(self.lens[b]))
        return pool[torch.from_numpy(self.table[b, s // self.page].astype(np.int64)), torch.from_numpy(s % self.page)]

    def on(self, device):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
        return dict(q=self.q.to(device), tk=self.tk.to(device), tv=self.tv.to(device), k=self.k.to(device),
                    v=self.v.to(device), table=t(self.table), lens=t(self.lens.astype(np.int32)), off=t(self.off),
                    parent=None if self.chain else t(self.parent))

    def scores(self, q, k, cap):
        """[heads, rows, keys] in 64 bits"""
        x = torch.einsum("nhd,lhd->hnl", q.double(), k.double().repeat_interleave(self.Hq // self.Hkv, 1)) * self.scale
        return cap * torch.tanh(x / cap) if cap > 0 else x

    def attention(self, cap=0.0):
        """out [M, Hq, D] and lse [M, Hq] in 64 bits; what a node does not see is not looked at."""
        out, lse = torch.zeros(self.M, self.Hq, self.D, dtype=torch.float64), torch.zeros(self.M, self.Hq, dtype=torch.float64)
        for b in range(self.B):
            lo, hi = int(self.off[b]), int(self.off[b + 1])
            ck, cv = self.slots(self.k, b), self.slots(self.v, b)
            for i, line in enumerate(lines(self.parent[lo:hi])):
                at = torch.tensor([lo + j for j in line])
                k, v = torch.cat([ck, self.tk[at]]), torch.cat([cv, self.tv[at]])
                x = self.scores(self.q[lo + i:lo + i + 1], k, cap)[:, 0]
                out[lo + i] = torch.einsum("hl,lhd->hd", torch.softmax(x, -1), v.double().repeat_interleave(self.Hq // self.Hkv, 1))
                lse[lo + i] = torch.logsumexp(x, -1)
        return out, lse


def verify_tree(logits, off, ids, parent, tau, judged=None):
    """token_logp, row_lse, path, path_len, on_path in 64 bits; logits [M, V] float64.  A node whose parent is out of
    range is rejected.  judged: float32 log-likelihoods to take the decisions by, in float32, instead of these."""
    M = logits.shape[0]
    with np.errstate(all="ignore"):
        top = logits.max(1, keepdims=True)
        lse = (top + np.log(np.exp(logits - top).sum(1, keepdims=True)))[:, 0]
    logp, path, on = np.zeros(M), np.full(M, -1, np.int32), np.zeros(M, np.uint8)
    length = np.zeros(len(off) - 1, np.int32)
    for b in range(len(off) - 1):
        lo, n = off[b], off[b + 1] - off[b]
        line = [None] * n
        best = []
        for i in range(n):
            p = parent[lo + i]
            if p == -1:
                line[i] = [i]
            elif not 0 <= p < i:
                logp[lo + i] = -np.inf
            else:
                logp[lo + i] = logits[lo + p, ids[lo + i]] - lse[lo + p]
                if judged is None:
                    over = tau <= 0 or (tau < 1 and logp[lo + i] > math.log(tau))
                else:
                    over = tau <= 0 or (tau < 1 and judged[lo + i] > np.float32(math.log(np.float32(tau))))
                if line[p] is not None and over:
                    line[i] = line[p] + [i]
            if line[i] is not None and len(line[i]) > len(best):
                best = line[i]
        length[b] = len(best)
        path[lo:lo + len(best)] = best
        on[lo + np.array(best, np.int64)] = 1
    return logp, lse, path, length, on


def planted(rng, off, parent, V, likely=0.75):
    """Logits and ids whose nodes are clearly likely (p of 0.1 and more at up to three children) or at noise level."""
    M = int(off[-1])
    x = rng.standard_normal((M, V))
    ids = np.zeros(M, np.int32)
    for b in range(len(off) - 1):
        for r in range(off[b], off[b + 1]):
            ids[r] = rng.integers(0, V)
            if parent[r] >= 0 and rng.random() < likely:
                x[off[b] + parent[r], ids[r]] = math.log(V) + 2.0 + rng.random()
    return x, ids
