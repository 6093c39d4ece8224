"""Performance cases of drafts that branch and of the key/value cache they are verified against.

Five kinds of pass, each through the public binding:

  attention  ssd_tree_attention: the nodes of every utterance's draft tree (or chain) attend to the
             utterance's paged cache and to their own ancestors; one layer of a verification pass
  verify     ssd_verify_tree: the LLM's logits behind every node -> the longest accepted path
  append     ssd_cache_append: the accepted path's keys and values enter the cache, one layer
  weights    ssd_cache_weights: attention weight that every cached slot has received, accumulated
  evict      ssd_cache_evict: the slots that have received the most are kept, the cache compacted

The shape of a batch (lengths, trees, pages) comes from the case alone, the values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda"


def case(name, kind, **kw):
    """Grouped heads of 128, bf16, pages of 16 slots, trees (not chains), one utterance unless said."""
    c = dict(kind=kind, B=1, n_lo=1, n_hi=1, len_lo=1000, len_hi=1000, Hq=32, Hkv=8, D=128, page=16, chain=False,
             cap=0.0, dtype="bf16", shape=1)
    if kind == "verify":
        c = dict(kind=kind, B=1, n_lo=8, n_hi=8, V=32000, pad=0, tau=0.1, dtype="bf16", shape=1)
    if kind == "evict":
        c.update(budget=512, sink=4, recent=128)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one utterance, one token, behind a prompt of 20 s of audio: a step of the auto-regressive fallback
        case("attn_1_token", "attention", D=64),
        # an ordinary serving batch: trees of up to 32 nodes over prompts of 10 to 60 s
        case("attn_trees_b64", "attention", B=64, n_lo=5, n_hi=32, len_lo=500, len_hi=3001, shape=2),
        # whole CTC drafts, up to 200 tokens each in a chain, verified in one pass: bound by the products
        case("attn_chains_b128", "attention", B=128, n_lo=50, n_hi=200, len_lo=250, len_hi=1500, chain=True, shape=3),
        # an hour of audio in the cache; capped scores, an odd number of heads to a group, fp16, pages of 64
        case("attn_long_cap_f16", "attention", B=4, n_lo=33, n_hi=64, len_lo=60001, len_hi=100003, Hq=28, Hkv=4,
             page=64, cap=50.0, dtype="f16", shape=4),
        # one utterance, a tree of eight nodes, fp32 logits: latency
        case("verify_8_nodes_f32", "verify", dtype="f32"),
        # a batch of trees against a wide vocabulary of odd size, a slice of a padded matrix
        case("verify_trees_b64", "verify", B=64, n_lo=5, n_hi=32, V=100353, pad=3, shape=2),
        # a few accepted tokens of one utterance
        case("append_1", "append", n_lo=8, n_hi=8, D=64, shape=5),
        # long accepted chains of a whole batch
        case("append_chains_b512", "append", B=512, n_lo=50, n_hi=200, len_lo=250, len_hi=1500, chain=True, shape=6),
        # one token's weights of a small batch
        case("weights_1_token_b8", "weights", B=8, len_lo=800, len_hi=2000, D=64, shape=7),
        # trees of a batch, fp16, no grouped heads
        case("weights_trees_b32", "weights", B=32, n_lo=5, n_hi=32, len_lo=500, len_hi=3001, Hq=16, Hkv=16,
             dtype="f16", shape=8),
        # one utterance's cache down to an eighth
        case("evict_1", "evict", len_lo=4096, len_hi=4096, budget=512, D=64, shape=9),
        # a batch of long caches down to a quarter and less; some are short enough to stay as they are
        case("evict_b64", "evict", B=64, len_lo=1500, len_hi=12001, budget=2048, recent=512, page=64, shape=10),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "verify", "append", "weights", "evict"])
    shape = rng.randrange(1 << 20)
    if kind == "verify":
        B = log_int(rng, 1, 64)
        return case("", kind, B=B, n_lo=rng.randint(1, 5), n_hi=log_int(rng, 6, 32), V=log_int(rng, 1000, 100353),
                    pad=rng.choice([0, 0, 1, 3]), dtype=rng.choice(["bf16", "bf16", "f32"]), shape=shape)
    Hkv, G = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 2, 3, 4, 7, 8])
    kw = dict(Hq=Hkv * G, Hkv=Hkv, D=rng.choice([64, 128]), page=rng.choice([8, 16, 32, 64, 128, 256]),
              dtype=rng.choice(["bf16", "f16"]), shape=shape)
    if kind == "evict":
        top = log_int(rng, 600, 12000)
        budget = log_int(rng, 64, top)
        return case("", kind, B=log_int(rng, 1, 64), len_lo=max(1, top // rng.choice([1, 2, 10])), len_hi=top,
                    budget=budget, sink=rng.choice([0, 4, 16]), recent=rng.randint(0, budget - 16), **kw)
    chain = rng.random() < 0.4
    n_hi = log_int(rng, 1, 200 if chain else 64)
    kw.update(chain=chain, n_hi=n_hi, n_lo=rng.randint(0, n_hi), cap=rng.choice([0.0, 0.0, 0.0, 30.0]))
    B = log_int(rng, 1, 128)
    most = 300_000 if kind == "append" else max(64, min(40_000, int(4e8 / (B * kw["Hq"] * n_hi))))
    top = min(log_int(rng, 40, 40_000), most, 400_000 // B + 40)
    return case("", kind, B=B, len_lo=rng.choice([0, top // 4, top]), len_hi=top, **kw)


# ---- the shape of a batch, from the case alone --------------------------------------------------

def shape_of(c):
    r = np.random.RandomState(c["shape"])
    B = c["B"]
    n = r.randint(c["n_lo"], c["n_hi"] + 1, B)
    n[r.randint(B)] = c["n_hi"]
    off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
    parent = np.full(int(off[-1]), -1, np.int32)
    for b in range(B):
        for i in range(1, n[b]):                       # a few hypotheses that share prefixes
            parent[off[b] + i] = i - 1 if c.get("chain") else max(0, i - 1 - int(r.geometric(0.55) - 1))
    lens = None
    if "len_lo" in c:
        lens = r.randint(c["len_lo"], c["len_hi"] + 1, B).astype(np.int32)
        lens[r.randint(B)] = c["len_hi"]
    return n, off, parent, lens


def pages_of(c, lens, room):
    """A page table [B, P] of pages handed out in random order, with `room` slots left behind each cache, and their number."""
    r = np.random.RandomState(c["shape"] + 1)
    need = -(-(lens.astype(np.int64) + room) // c["page"])
    P, total = int(need.max()), int(need.sum())
    order = r.permutation(total).astype(np.int32)
    table = np.zeros((c["B"], max(P, 1)), np.int32)
    at = 0
    for b in range(c["B"]):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    return table, total


def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = TORCH[c["dtype"]]
    n, off, parent, lens = shape_of(c)
    M, B = int(off[-1]), c["B"]
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    s = dict(c=c, kind=c["kind"], n=n, tok_off=put(off), parent=put(parent), B=B, M=M, n_max=int(n.max()))
    if c["kind"] == "verify":
        V = c["V"]
        x = torch.randn((M, V + c["pad"]), generator=g, device=DEV, dtype=torch.float32 if c["dtype"] == "f32" else dt)[:, :V]
        ids = torch.randint(0, V, (M,), generator=g, device=DEV, dtype=torch.int32)
        # two nodes in three are likely behind their parent, the others are at the noise's level
        start = torch.repeat_interleave(s["tok_off"][:-1], s["tok_off"].diff())
        up = start + s["parent"].clamp(min=0)
        likely = (torch.rand((M,), generator=g, device=DEV) < 0.8) & (s["parent"] >= 0)
        boost = math.log(V) + 0.5 + 1.0 + torch.rand((M,), generator=g, device=DEV) * 0.5
        x[up[likely], ids[likely].long()] = boost[likely].to(x.dtype)
        s.update(x=x, ids=ids, tau=c["tau"])
        return s
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    room = c["n_hi"] if c["kind"] == "append" else 0
    table, total = pages_of(c, lens, room)
    pool = (max(total, 1), c["page"], Hkv, D)
    s.update(table=put(table), lens=put(lens), len_max=int(lens.max()), k=torch.randn(pool, generator=g, device=DEV, dtype=dt),
             scale=D ** -0.5, cap=c["cap"])
    if c["kind"] != "weights":
        s["v"] = torch.randn(pool, generator=g, device=DEV, dtype=dt)
    if c["kind"] == "evict":
        # heavy-tailed, as attention weight is: a few slots hold most of it
        s["weight"] = torch.exp(2.0 * torch.randn((B, s["len_max"]), generator=g, device=DEV))
        return s
    s["tk"] = torch.randn((M, Hkv, D), generator=g, device=DEV, dtype=dt)
    s["tv"] = torch.randn((M, Hkv, D), generator=g, device=DEV, dtype=dt)
    if c["kind"] == "append":
        keep = torch.randint(0, 1 << 30, (B,), generator=g, device=DEV) % torch.from_numpy(n + 1).to(DEV)
        pos = torch.arange(M, device=DEV) - torch.repeat_interleave(s["tok_off"][:-1], s["tok_off"].diff())
        kept = torch.repeat_interleave(keep, s["tok_off"].diff())
        # a path of every tree: its first nodes, as an accepted chain has them
        s["path"] = torch.where(pos < kept, pos, -1).to(torch.int32)
        s["path_len"] = keep.to(torch.int32)
        s["weight"] = torch.rand((B, s["len_max"] + room), generator=g, device=DEV)
        return s
    s["q"] = (2.0 * torch.randn((M, Hq, D), generator=g, device=DEV)).to(dt)
    if c["kind"] == "weights":
        s["lse"] = cache_lse(s)
        s["use"] = (torch.rand((M,), generator=g, device=DEV) < 0.7).to(torch.uint8)
        s["weight"] = torch.rand((B, max(s["len_max"], 1)), generator=g, device=DEV)
    return s


# ---- the plain forms ------------------------------------------------------------------------------

def padded(s):
    """Node numbers [B, n] of every utterance, and which of them are there."""
    n = s["tok_off"].diff()
    at = torch.arange(s["n_max"], device=DEV)
    there = at[None, :] < n[:, None]
    return torch.where(there, s["tok_off"][:-1, None] + at[None, :], 0), there


def ancestors(s, at, there):
    """[B, n, n]: whether node j is node i or above it."""
    n = s["n_max"]
    up = torch.where(there, s["parent"][at].long(), -1)
    a = torch.nn.functional.one_hot(up + 1, n + 1)[:, :, 1:].float() + torch.eye(n, device=DEV)
    for _ in range(n.bit_length()):
        a = torch.matmul(a, a).clamp(max=1.0)
    return (a > 0) & there[:, :, None] & there[:, None, :]


def slots(s, pool, length):
    """[B, length, Hkv, D]: the first slots of every utterance's cache, in 32 bits."""
    page = pool.shape[1]
    pages = s["table"][:, :max(1, -(-length // page))].long()
    return pool[pages].flatten(1, 2)[:, :length].float()


def capped(x, cap):
    return cap * torch.tanh(x / cap) if cap > 0 else x


def cache_scores(s, at):
    """[B, Hkv, G, n, len]: every node's scores against its utterance's cache."""
    q = s["q"][at].float().unflatten(2, (s["k"].shape[2], -1)).permute(0, 2, 3, 1, 4)
    k = slots(s, s["k"], s["len_max"]).permute(0, 2, 3, 1)
    x = torch.matmul(q.flatten(2, 3), k).unflatten(2, q.shape[2:4])
    return capped(x * s["scale"], s["cap"]), q


def cached(s):
    return torch.arange(s["len_max"], device=DEV)[None, :] < s["lens"][:, None]


def cache_lse(s):
    """[M, Hq]: the log-sum-exp of the nodes' scores against cache and node itself, as the attention's."""
    at, there = padded(s)
    x, q = cache_scores(s, at)
    x = x.masked_fill(~cached(s)[:, None, None, None, :], -math.inf)
    k = s["tk"][at].float().permute(0, 2, 1, 3)[:, :, None]
    mine = capped((q * k).sum(-1, keepdim=True) * s["scale"], s["cap"])
    lse = torch.logsumexp(torch.cat([x, mine], -1), -1)
    return lse.permute(0, 3, 1, 2).flatten(2, 3)[there].contiguous()


def plain_attention(s):
    at, there = padded(s)
    x, q = cache_scores(s, at)
    x = x.masked_fill(~cached(s)[:, None, None, None, :], -math.inf)
    k = s["tk"][at].float().permute(0, 2, 3, 1)
    y = capped(torch.matmul(q.flatten(2, 3), k).unflatten(2, q.shape[2:4]) * s["scale"], s["cap"])
    y = y.masked_fill(~ancestors(s, at, there)[:, None, None], -math.inf)
    x = torch.cat([x, y], -1)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    v = torch.cat([slots(s, s["v"], s["len_max"]) * cached(s)[:, :, None, None],
                   s["tv"][at].float() * there[:, :, None, None]], 1).permute(0, 2, 1, 3)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, q.shape[2:4]) / total
    out = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[there]
    lse = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).flatten(2, 3)[there]
    return dict(out=out.to(s["q"].dtype), lse=lse)


def plain_verify(s):
    x = s["x"].float()
    top = x.amax(-1, keepdim=True)
    lse = (top + torch.log(torch.exp(x - top).sum(-1, keepdim=True)))[:, 0]
    at, there = padded(s)
    start = s["tok_off"][:-1, None]
    up = torch.where(there, s["parent"][at].long(), -1)
    row = (start + up.clamp(min=0)).clamp(max=s["M"] - 1)
    logp = torch.where(up >= 0, x[row, s["ids"][at].long()] - lse[row], 0.0)
    fine = (logp > math.log(s["tau"])) | (up < 0)
    anc = ancestors(s, at, there)
    taken = there & (anc <= fine[:, None, :]).all(-1)
    deep = torch.where(taken, anc.sum(-1), 0)
    length, best = deep.max(1)
    best = (deep == length[:, None]).int().argmax(1)       # the lowest of equals
    on = torch.gather(anc, 1, best[:, None, None].expand(-1, 1, s["n_max"]))[:, 0] & (length > 0)[:, None]
    order = torch.sort(torch.where(on, torch.arange(s["n_max"], device=DEV), s["n_max"]), dim=1).values
    return dict(token_logp=logp[there], row_lse=lse, path=torch.where(order < s["n_max"], order, -1)[there].int(),
                path_len=length.int(), on_path=on[there].to(torch.uint8))


def places(s, slot, table):
    """Page and slot in the page, of slots [B, n]."""
    page = s["k"].shape[1]
    return torch.gather(table.long(), 1, (slot // page).clamp(max=table.shape[1] - 1)), slot % page


def plain_append(s):
    at, there = padded(s)
    k = torch.arange(s["n_max"], device=DEV)[None, :].expand(s["B"], -1)
    take = there & (k < s["path_len"][:, None])
    node = (s["tok_off"][:-1, None] + s["path"][at])[take]
    slot = s["lens"].long()[:, None] + k
    page, place = places(s, slot, s["table"])
    s["k"][page[take], place[take]] = s["tk"][node]
    s["v"][page[take], place[take]] = s["tv"][node]
    b = torch.arange(s["B"], device=DEV)[:, None].expand_as(slot)
    s["weight"][b[take], slot[take]] = 0.0
    return dict(k=s["k"], v=s["v"], weight=s["weight"], new_len=s["lens"] + s["path_len"])


def plain_weights(s):
    at, there = padded(s)
    x, _ = cache_scores(s, at)
    lse = s["lse"][at].unflatten(2, (s["k"].shape[2], -1)).permute(0, 2, 3, 1)[..., None]
    use = there & (s["use"][at] != 0)
    p = torch.where(use[:, None, None, :, None] & cached(s)[:, None, None, None, :], torch.exp(x - lse), 0.0)
    s["weight"][:, :s["len_max"]] += p.sum((1, 2, 3))
    return dict(weight=s["weight"])


def plain_evict(s):
    c, L = s["c"], s["len_max"]
    at = torch.arange(L, device=DEV)[None, :]
    n = s["lens"].long()[:, None]
    key = torch.where((at < c["sink"]) | (at >= n - c["recent"]), math.inf, s["weight"])
    key = torch.where(at < n, key, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :c["budget"]]
    j = torch.arange(order.shape[1], device=DEV)[None, :]
    new = n.clamp(max=c["budget"])
    # caches within the budget keep every slot in its place
    kept = torch.sort(torch.where(j < new, order, L), dim=1).values
    there = j < new
    kept = torch.where(there, kept, 0)
    page, place = places(s, kept, s["table"])
    k, v = s["k"][page, place], s["v"][page, place]
    page, place = places(s, j.expand_as(kept), s["table"])
    s["k"][page[there], place[there]] = k[there]
    s["v"][page[there], place[there]] = v[there]
    fill = (0, c["budget"] - kept.shape[1])
    weight = torch.where(there, torch.gather(s["weight"], 1, kept), 0.0)
    return dict(k=s["k"], v=s["v"], weight=torch.nn.functional.pad(weight, fill),
                kept=torch.nn.functional.pad(torch.where(there, kept, -1), fill, value=-1).int(), new_len=new[:, 0].int())


# ---- the framework's calls --------------------------------------------------------------------------

def buffers(s):
    """Result buffers, which a serving program keeps from step to step."""
    from paper_2603_11243_b200 import binding as ssd
    if "out" not in s:
        c, B, M = s["c"], s["B"], s["M"]
        if s["kind"] == "attention":
            s["out"] = ssd.alloc_tree_attention_outputs(M, B, c["Hq"], c["D"], TORCH[c["dtype"]], DEV)
        elif s["kind"] == "verify":
            code = ssd.F32 if c["dtype"] == "f32" else ssd.BF16
            s["out"] = ssd.alloc_verify_tree_outputs(M, B, DEV, ssd.ssd_verify_workspace_bytes(B, M, c["V"], code))
        elif s["kind"] == "append":
            s["out"] = ssd.alloc_cache_append_outputs(B, DEV)
        elif s["kind"] == "weights":
            s["out"] = ssd.alloc_cache_weights_outputs(B, DEV)
        else:
            s["out"] = ssd.alloc_cache_evict_outputs(B, c["budget"], DEV)
    return ssd, s["out"]


def own_attention(s):
    ssd, out = buffers(s)
    ssd.ssd_tree_attention(s["q"], s["tk"], s["tv"], s["k"], s["v"], s["table"], s["lens"], s["tok_off"], s["n_max"],
                           None if s["c"]["chain"] else s["parent"], s["scale"], s["cap"], out=out)
    return dict(out=out["out"], lse=out["lse"])


def own_verify(s):
    ssd, out = buffers(s)
    ssd.ssd_verify_tree(s["x"], s["tok_off"], s["ids"], s["parent"], s["tau"], out=out)
    return {k: out[k] for k in ("token_logp", "row_lse", "path", "path_len", "on_path")}


def own_append(s):
    ssd, out = buffers(s)
    ssd.ssd_cache_append(s["tk"], s["tv"], s["tok_off"], s["path"], s["path_len"], s["k"], s["v"], s["table"],
                         s["lens"], s["weight"], out=out)
    return dict(k=s["k"], v=s["v"], weight=s["weight"], new_len=out["new_len"])


def own_weights(s):
    ssd, out = buffers(s)
    ssd.ssd_cache_weights(s["q"], s["lse"], s["k"], s["table"], s["lens"], s["tok_off"], s["n_max"], s["weight"],
                          s["use"], s["scale"], s["cap"], out=out)
    return dict(weight=s["weight"])


def own_evict(s):
    ssd, out = buffers(s)
    c = s["c"]
    ssd.ssd_cache_evict(s["k"], s["v"], s["table"], s["lens"], s["weight"], c["budget"], c["sink"], c["recent"], out=out)
    return dict(k=s["k"], v=s["v"], weight=out["weight"], kept=out["kept"], new_len=out["new_len"])


def run(s):
    if own:
        return {"attention": own_attention, "verify": own_verify, "append": own_append, "weights": own_weights,
                "evict": own_evict}[s["kind"]](s)
    return {"attention": plain_attention, "verify": plain_verify, "append": plain_append, "weights": plain_weights,
            "evict": plain_evict}[s["kind"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(c):
    n, off, parent, lens = shape_of(c)
    M, B, e = int(off[-1]), c["B"], BYTES[c["dtype"]]
    if c["kind"] == "verify":
        return dict(bytes=float(M * c["V"] * e + M * 21 + B * 12), flops=float(3 * M * c["V"]))
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    row = Hkv * D * e
    if c["kind"] == "evict":
        new = np.minimum(lens, c["budget"])
        moved = np.where(lens > c["budget"], np.maximum(new - c["sink"], 0), 0).sum()
        return dict(bytes=float(4 * row * moved + 4 * lens.sum() + 8 * new.sum()), flops=float(lens.sum()))
    if c["kind"] == "append":
        return dict(bytes=float(2 * row * M + 4 * M), flops=0.0)       # about half of the nodes: read and written, K and V
    if c["kind"] == "weights":
        return dict(bytes=float(row * lens.sum() + M * Hq * (D * e + 4) + 8 * lens.sum()),
                    flops=float(2 * Hq * D * (n.astype(float) * lens).sum()))
    depth = np.ones(M)
    for b in range(B):
        for i in range(1, n[b]):
            depth[off[b] + i] += depth[off[b] + parent[off[b] + i]]
    pairs = (n.astype(float) * lens).sum() + depth.sum()
    return dict(bytes=float(2 * row * (lens.sum() + M) + 2 * M * Hq * D * e + 4 * M * Hq), flops=float(4 * Hq * D * pairs))


# ---- in 64 bits, utterance by utterance, from the definitions ----------------------------------------

def lines_of_descent(parent):
    """Every node's line, root first."""
    lines = []
    for i, p in enumerate(parent):
        lines.append((lines[p] if p >= 0 else []) + [i])
    return lines


def exact(c, seed):
    s = prepare(c, seed)
    n, off, parent, lens = shape_of(c)
    if c["kind"] == "verify":
        lse = torch.cat([torch.logsumexp(rows.double(), 1) for rows in s["x"].split(64)])
        up = torch.from_numpy(np.repeat(off[:-1], n) + np.maximum(parent, 0)).to(DEV)
        logp = s["x"][up, s["ids"].long()].double() - lse[up]
        logp[s["parent"] < 0] = 0.0
        good = (logp > math.log(c["tau"])).cpu().numpy()
        path, length, on = np.full(s["M"], -1, np.int32), np.zeros(c["B"], np.int32), np.zeros(s["M"], np.uint8)
        for b in range(c["B"]):
            lines = lines_of_descent(parent[off[b]:off[b + 1]])
            best = []
            for line in lines:
                if all(good[off[b] + i] or parent[off[b] + i] < 0 for i in line) and len(line) > len(best):
                    best = line
            length[b] = len(best)
            path[off[b]:off[b] + len(best)] = best
            on[off[b] + np.array(best, np.int64)] = 1
        put = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
        return dict(token_logp=logp, row_lse=lse, path=put(path), path_len=put(length), on_path=put(on))
    table = s["table"].long()

    def own_slots(pool, b):
        return pool[table[b]].flatten(0, 1)[:int(lens[b])]

    if c["kind"] == "append":
        for b in range(c["B"]):
            for j in range(int(s["path_len"][b])):
                slot = int(lens[b]) + j
                page, node = int(table[b, slot // c["page"]]), int(off[b]) + j
                s["k"][page, slot % c["page"]] = s["tk"][node]
                s["v"][page, slot % c["page"]] = s["tv"][node]
                s["weight"][b, slot] = 0.0
            if b >= 64:
                return None
        return dict(k=s["k"], v=s["v"], weight=s["weight"].double(), new_len=s["lens"] + s["path_len"])
    if c["kind"] == "evict":
        weight = torch.zeros((c["B"], c["budget"]), dtype=torch.float64, device=DEV)
        kept = torch.full((c["B"], c["budget"]), -1, dtype=torch.int32, device=DEV)
        for b in range(c["B"]):
            L = int(lens[b])
            w = s["weight"][b, :L].cpu().numpy()
            if L <= c["budget"]:
                keep = np.arange(L)
            else:
                tail = min(c["recent"], L - c["sink"])
                middle = np.arange(c["sink"], L - tail)
                chosen = middle[np.lexsort((middle, -w[middle]))][:c["budget"] - c["sink"] - tail]
                keep = np.concatenate([np.arange(c["sink"]), np.sort(chosen), np.arange(L - tail, L)])
            m = len(keep)
            at = torch.from_numpy(keep).to(DEV)
            to = torch.arange(m, device=DEV)
            kept[b, :m] = at.int()
            weight[b, :m] = s["weight"][b, at].double()
            for pool in (s["k"], s["v"]):
                pool[table[b][to // c["page"]], to % c["page"]] = own_slots(pool, b)[at].clone()
        return dict(k=s["k"], v=s["v"], weight=weight, kept=kept,
                    new_len=torch.from_numpy(np.minimum(lens, c["budget"]).astype(np.int32)).to(DEV))
    G = c["Hq"] // c["Hkv"]

    def scores(q, k):
        x = torch.einsum("nhd,lhd->hnl", q, k.repeat_interleave(G, 1)) * s["scale"]
        return c["cap"] * torch.tanh(x / c["cap"]) if c["cap"] > 0 else x

    if c["kind"] == "weights":
        w = s["weight"].double()
        for b in range(c["B"]):
            rows = torch.arange(off[b], off[b + 1], device=DEV)
            rows = rows[s["use"][rows] != 0]
            x = scores(s["q"][rows].double(), own_slots(s["k"], b).double())
            w[b, :int(lens[b])] += torch.exp(x - s["lse"][rows].double().t()[:, :, None]).sum((0, 1))
        return dict(weight=w)
    out, lse = [], []
    for b in range(c["B"]):
        lo, hi, L = int(off[b]), int(off[b + 1]), int(lens[b])
        if hi == lo:
            continue
        see = np.zeros((hi - lo, L + hi - lo), bool)
        see[:, :L] = True
        for i, line in enumerate(lines_of_descent(parent[lo:hi])):
            see[i, L + np.array(line)] = True
        see = torch.from_numpy(see).to(DEV)
        k = torch.cat([own_slots(s["k"], b), s["tk"][lo:hi]]).double()
        v = torch.cat([own_slots(s["v"], b), s["tv"][lo:hi]]).double()
        x = scores(s["q"][lo:hi].double(), k).masked_fill(~see, -math.inf)
        out.append(torch.einsum("hnl,lhd->nhd", torch.softmax(x, -1), v.repeat_interleave(G, 1)))
        lse.append(torch.logsumexp(x, -1).t())
    if not out:
        return None
    return dict(out=torch.cat(out), lse=torch.cat(lse))


if __name__ == "__main__":
    for _c in listed() + [draw(random.Random(0))]:
        print(_c, work(_c))
