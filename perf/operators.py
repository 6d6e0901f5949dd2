"""The cache operators as timed cases: rows stored into a cache, attention of a tree of drafted tokens over it, attention over
blocks of it that a cheap score selects, and the verification of a tree with the move of the accepted rows.

A cache of bf16 heads of 64 or 128 dimensions lies in operand order: groups of 32 keys, of K
    [key tile t][dimensions 32 s ..][q][a][r][e]      key 8 a + 4 t + r, dimension 32 s + 8 q + e   (t < 2, q, a, r < 4, e < 8)
and of V
    [dimensions 16 s ..][q][c][e]                     key 8 q + e, dimension 16 s + c                (q < 4, c < 16, e < 8)
as tensors [layers, B, heads, groups, 32, D]; every other cache is [layers, B, rows, heads, D].  The summaries of blocks of rows are
    [B, heads, blocks / 64, 2 (smallest, largest), D / 8, 64, 8].
Lengths, trees and sizes depend on the case alone; keys, values, queries, tokens on the seed.
"""
import math

import numpy as np
import torch

own = False

DEFAULTS = dict(call="tree", batch=1, rows=1, heads=8, kv=8, dim=64, length=64, dtype="bf16", chain=False, ragged=False, layers=1,
                block=0, first=0, recent=0, top=0)


def case(**kw):
    return dict(DEFAULTS, **kw)


def listed():
    return [
        # greedy decoding of one sentence with the big translation model: one token, one layer's self-attention
        case(name="tree-one-token", heads=16, kv=16, length=40, chain=True),
        # ten intensities of eight images, the drafts a tree
        case(name="tree-image-batch8", batch=8, rows=10, length=2999),
        # long documents, four query heads to a key head, drafts of ragged lengths
        case(name="tree-long-grouped", batch=8, rows=12, heads=32, kv=8, dim=128, length=32000, ragged=True),
        # wide trees, eight query heads to a key head: as many rows as a tree has
        case(name="tree-wide", batch=4, rows=64, heads=32, kv=4, dim=128, length=16381),
        # the small fp32 model
        case(name="tree-fp32", batch=4, rows=4, heads=4, kv=4, dim=16, length=130, dtype="f32"),
        # images once more, a third of the keys
        case(name="sparse-image-batch8", call="sparse", batch=8, rows=10, length=2999, block=32, first=1, recent=4, top=24),
        # one token far into a long document, and a few of them at once with trees
        case(name="sparse-one-token-long", call="sparse", heads=32, kv=8, dim=128, length=120001, chain=True, block=64, first=1, recent=4, top=59),
        case(name="sparse-long-batch4", call="sparse", batch=4, rows=7, heads=16, kv=8, dim=128, length=64000, ragged=True, block=64, first=1, recent=2, top=32),
        # verification: one sentence, and a batch with wide trees and many layers
        case(name="commit-sentence", call="commit", rows=10, heads=16, kv=16, length=90, layers=6),
        case(name="commit-batch16", call="commit", batch=16, rows=48, kv=8, dim=128, length=200, layers=24, ragged=True),
        # prompts into the cache of one layer, a short and a long ragged one
        case(name="store-prompt", call="store", batch=1, rows=37, kv=16),
        case(name="store-prompts-batch4", call="store", batch=4, rows=8100, kv=8, dim=128, ragged=True),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    most = [work(c) for c in listed()]
    while True:
        call = rng.choice(["tree", "tree", "tree", "sparse", "sparse", "commit", "store"])
        kv, dim = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 128])
        c = case(call=call, batch=log(1, 24), rows=log(1, 64), kv=kv, dim=dim, heads=kv * rng.choice([1, 1, 2, 3, 4, 8]), length=log(1, 70000), ragged=rng.random() < 0.5,
                 chain=rng.random() < 0.3)
        if call in ("tree", "sparse") and rng.random() < 0.2:
            c.update(dtype="f32", dim=rng.choice([16, 64, 128]), length=log(1, 3000))
        if call == "sparse":
            c.update(block=rng.choice([32, 64, 128]), first=rng.randint(0, 2), recent=rng.randint(0, 4), top=log(1, 64))
        elif call == "commit":
            c.update(heads=kv, layers=log(1, 24), length=log(1, 300))
        elif call == "store":
            c.update(heads=kv, rows=log(1, 8000), length=1, chain=False)
        w = work(c)
        if w["bytes"] <= max(x["bytes"] for x in most) and w["flops"] <= max(x["flops"] for x in most):
            return c


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(c):
    """Committed rows per sequence: as given, or from a quarter of that on."""
    b, n = c["batch"], c["length"]
    if not c["ragged"] or b == 1:
        return np.full(b, n, np.int64)
    return np.random.default_rng(b * 7 + n).integers(max(1, n // 4), n + 1, b).astype(np.int64)


def _counts(c):
    """Rows to be stored per sequence: of a prompt ragged, of a tree all."""
    b, t = c["batch"], c["rows"]
    if c["call"] != "store" or not c["ragged"]:
        return np.full(b, t, np.int64)
    return np.random.default_rng(b * 11 + t).integers(max(1, t // 3), t + 1, b).astype(np.int64)


def _parents(c):
    """Parents of the drafted nodes, [B, T]: a chain, or long branches with others beside them; ragged: some have fewer nodes."""
    b, t = c["batch"], c["rows"]
    p = np.tile(np.arange(t) - 1, (b, 1))
    if c["chain"]:
        return p
    rng = np.random.default_rng(b * 13 + t)
    other = rng.integers(-1, np.maximum(np.arange(t), 1), (b, t))
    p = np.where(rng.random((b, t)) < 0.5, p, np.minimum(other, np.arange(t) - 1))
    if c["ragged"]:
        p = np.where(np.arange(t)[None, :] < rng.integers(max(1, t // 2), t + 1, b)[:, None], p, -2)
    return p


def _capacity(c):
    """Rows of a cache: what the longest sequence needs, and a few more."""
    most = c["rows"] if c["call"] == "store" else c["length"] + c["rows"]
    return (most + 5 + 31) // 32 * 32


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _inputs(c, seed):
    """Keys, values and what else a call takes, a row a key.  Keys of a long text come in runs that resemble each other; queries look for some of them."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, b, t, kv, d, cap, nl = _dtype(c), c["batch"], c["rows"], c["kv"], c["dim"], _capacity(c), c["layers"]

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen, dtype=torch.float32)

    x = {}
    runs = (cap + 47) // 48
    x["k"] = torch.empty((nl, b, cap, kv, d), device="cuda", dtype=dt)
    x["v"] = torch.empty((nl, b, cap, kv, d), device="cuda", dtype=dt)
    for layer in range(nl):
        for s in range(b):
            theme = normal(runs, 1, kv, d).expand(runs, 48, kv, d).reshape(runs * 48, kv, d)[:cap]
            x["k"][layer, s] = (theme + normal(cap, kv, d) * 0.7).to(dt)
            x["v"][layer, s] = normal(cap, kv, d).to(dt)
    x["length"] = torch.from_numpy(_lengths(c).astype(np.int32)).cuda()
    x["parent"] = torch.from_numpy(_parents(c).astype(np.int32)).cuda()
    if c["call"] in ("tree", "sparse"):
        at = torch.randint(0, max(1, int(_lengths(c).min())), (b, 1), device="cuda", generator=gen).expand(b, c["heads"] // kv)
        seq = torch.arange(b, device="cuda")[:, None].expand_as(at)
        near = x["k"][0][seq, at].float().permute(0, 2, 1, 3).reshape(b, 1, c["heads"], d)          # a key that the heads of a group look for
        x["q"] = (near * 0.4 + normal(b, 1, c["heads"], d) * 0.6 + normal(b, t, c["heads"], d) * 0.5).to(dt)
        x["added"] = torch.full((b,), min(7, t), dtype=torch.int32, device="cuda")
    else:                                                     # K and V of the new rows, side by side as a projection leaves them
        kvs = normal(nl, b, t, 3, kv, d).to(dt)
        x["new_k"], x["new_v"] = kvs[:, :, :, 1], kvs[:, :, :, 2]
        x["start"] = torch.zeros(b, dtype=torch.int32, device="cuda") if c["call"] == "store" else x["length"]
        x["count"] = torch.from_numpy(_counts(c).astype(np.int32)).cuda()
    if c["call"] == "commit":
        x["best"] = torch.randint(3, 32000, (b, t), device="cuda", generator=gen, dtype=torch.int32)
        x["expect"] = torch.randint(3, 32000, (b,), device="cuda", generator=gen, dtype=torch.int32)
        want = torch.cat([x["expect"][:, None], x["best"]], 1).gather(1, x["parent"].clamp(min=-1).long() + 1)
        said = torch.rand((b, t), device="cuda", generator=gen) < 0.75
        x["token"] = torch.where(said, want, torch.randint(3, 32000, (b, t), device="cuda", generator=gen, dtype=torch.int32))
        x["room"] = torch.randint(1, t + 4, (b,), device="cuda", generator=gen, dtype=torch.int32)
    return x


def _grouped(k):
    return k.dtype == torch.bfloat16 and k.shape[-1] in (64, 128)


def _pack(k, v):
    """Caches [layers, B, rows, heads, D] as they lie in memory."""
    if not _grouped(k):
        return k, v
    nl, b, cap, h, d = k.shape
    g = cap // 32
    kk = k.view(nl, b, g, 4, 2, 4, h, d // 32, 4, 8).permute(0, 1, 6, 2, 4, 7, 8, 3, 5, 9)        # (a, t, r, s, q, e) -> t s q a r e
    vv = v.view(nl, b, g, 4, 8, h, d // 16, 16).permute(0, 1, 5, 2, 6, 3, 7, 4)                   # (q, e, s, c) -> s q c e
    return kk.reshape(nl, b, h, g, 32, d), vv.reshape(nl, b, h, g, 32, d)


def _summaries(k, block, length=None, added=None):
    """Smallest and largest key per block and dimension of a cache [B, rows, heads, D], as they lie in memory; without those of complete blocks among whose
    rows are the last `added`."""
    b, cap, h, d = k.shape
    n = cap // block
    tiles = (n + 63) // 64
    x = k[:, :n * block].view(b, n, block, h, d)
    both = torch.stack([x.amin(2), x.amax(2)], 1).permute(0, 3, 2, 1, 4)                          # [b, h, n, 2, d]
    if added is not None:
        at = torch.arange(n, device=k.device)
        both = both * ~((at >= ((length - added).clamp(min=0) // block)[:, None]) & (at < (length // block)[:, None]))[:, None, :, None, None]
    both = torch.cat([both, torch.zeros((b, h, tiles * 64 - n, 2, d), device=k.device, dtype=k.dtype)], 2)
    return both.reshape(b, h, tiles, 64, 2, d // 8, 8).permute(0, 1, 2, 4, 5, 3, 6).contiguous()


def prepare(case, seed):
    c = case
    state = _inputs(c, seed)
    state["c"] = c
    if c["call"] == "sparse":
        state["summaries"] = _summaries(state["k"][0], c["block"], state["length"], state["added"])
    state["k"], state["v"] = _pack(state["k"], state["v"])
    return state


# ------------------------------------------------------------------------------------------------ the operators, plainly

def _k_rows(k):
    """Keys of a packed cache [.., groups, 32, D], a row a key, in 32 bits."""
    lead, d = k.shape[:-2], k.shape[-1]
    n = len(lead)
    x = k.view(*lead, 2, d // 32, 4, 4, 4, 8).permute(*range(n), n + 3, n, n + 4, n + 1, n + 2, n + 5)
    return x.reshape(*lead[:-1], lead[-1] * 32, d).float()


def _v_rows(v):
    lead, d = v.shape[:-2], v.shape[-1]
    n = len(lead)
    x = v.view(*lead, d // 16, 4, 16, 8).permute(*range(n), n + 1, n + 3, n, n + 2)
    return x.reshape(*lead[:-1], lead[-1] * 32, d).float()


def _rows_of(k, v):
    """Both of one layer as [B, heads, rows, D] in 32 bits."""
    if _grouped(k):
        return _k_rows(k[0]), _v_rows(v[0])
    return k[0].transpose(1, 2).float(), v[0].transpose(1, 2).float()


def _ancestors(parent):
    """[B, T, T]: node j is node i or above it; absent nodes have none."""
    t = parent.shape[1]
    i = torch.arange(t, device=parent.device)
    there = (parent >= -1) & (parent < i)
    step = ((parent[:, :, None] == i) & there[:, :, None]).float() + torch.eye(t, device=parent.device)
    reach = torch.matrix_power(step, max(1, t)) > 0.5
    whole = ~(reach & ~there[:, None, :]).any(2)              # no absent node above
    return reach & whole[:, :, None]


def _attend(q, k, v, seen):
    """Softmax over the keys that are seen ([B, 1 or heads of K, T, keys]); rows that see none are zero."""
    b, t, h, d = q.shape
    kv, n = k.shape[1], k.shape[2]
    x = q.float().view(b, t, kv, h // kv, d).permute(0, 2, 1, 3, 4).reshape(b, kv, t * (h // kv), d)
    s = torch.matmul(x, k.transpose(2, 3).contiguous()) * (1 / math.sqrt(d))
    s = s.view(b, kv, t, h // kv, n).masked_fill_(~seen[:, :, :, None, :], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = e.sum(-1, keepdim=True)
    e = (e / torch.where(total == 0, torch.ones_like(total), total)).view(b, kv, t * (h // kv), n)
    o = torch.matmul(e, v)
    return o.view(b, kv, t, h // kv, d).permute(0, 2, 1, 3, 4).reshape(b, t, h, d).to(q.dtype)


def _seen(length, parent, n):
    """Prefix [B, 1, keys] and ancestors [B, T, keys] among the cache's rows."""
    anc = _ancestors(parent)
    at = torch.arange(n, device=length.device)[None, :] - length[:, None]
    node = at.clamp(0, parent.shape[1] - 1)[:, None, :].expand(-1, parent.shape[1], -1)
    own_rows = anc.gather(2, node) & ((at >= 0) & (at < parent.shape[1]))[:, None, :]
    return (at < 0)[:, None, :] & anc.any(2)[:, :, None], own_rows


def _plain_tree(s):
    k, v = _rows_of(s["k"], s["v"])
    prefix, above = _seen(s["length"], s["parent"], k.shape[2])
    return _attend(s["q"], k, v, (prefix | above)[:, None])


def _plain_sparse(s):
    c, q, length = s["c"], s["q"], s["length"].long()
    k, v = _rows_of(s["k"], s["v"])
    b, kv, n, d = k.shape
    t, group, block = q.shape[1], q.shape[2] // kv, c["block"]
    blocks = n // block
    tiles = s["summaries"].shape[2]
    # summaries of the complete blocks that rows length - added .. length - 1 have touched
    fresh = k[:, :, :blocks * block].view(b, kv, blocks, block, d)
    fresh = torch.stack([fresh.amin(3), fresh.amax(3)], 3).to(s["summaries"].dtype)                # [b, kv, blocks, 2, d]
    at = torch.arange(blocks, device=q.device)
    done = length // block
    again = (at >= ((length - s["added"].long()).clamp(min=0) // block)[:, None]) & (at < done[:, None])
    kept = s["summaries"].permute(0, 1, 2, 5, 3, 4, 6).reshape(b, kv, tiles * 64, 2, d)
    both = torch.where(again[:, None, :, None, None], fresh, kept[:, :, :blocks])
    kept[:, :, :blocks] = both
    s["summaries"].copy_(kept.view(b, kv, tiles, 64, 2, d // 8, 8).permute(0, 1, 2, 4, 5, 3, 6))
    # the bound of the scores in a block; in 64 bits, for which blocks are taken
    x = q.double().view(b, t, kv, group, d).permute(0, 2, 1, 3, 4).reshape(b, kv, t * group, d)
    low, high = both[:, :, :, 0].double(), both[:, :, :, 1].double()
    score = torch.matmul(x.clamp(min=0), high.transpose(2, 3).contiguous()) + torch.matmul(x.clamp(max=0), low.transpose(2, 3).contiguous())
    score = score.view(b, kv, t, group, blocks).sum(3)
    always = ((at < c["first"]) | (at >= (done - c["recent"])[:, None])) & (at < done[:, None])
    open_ = ((at < done[:, None]) & ~always)[:, None, None, :]
    order = torch.sort(torch.where(open_, score, torch.full_like(score, -math.inf)), dim=3, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(3, order, at.expand_as(order).contiguous())
    chosen = (open_ & (rank < c["top"])) | always[:, None, None, :]
    prefix, above = _seen(s["length"], s["parent"], n)
    chosen = chosen & prefix.any(2)[:, None, :, None]
    key = torch.arange(n, device=q.device)
    tail = key >= (done * block)[:, None]                     # behind the last complete block
    picked = chosen.gather(3, (key // block).clamp(max=max(0, blocks - 1)).expand(b, kv, t, n)) if blocks else torch.zeros((b, kv, t, n), dtype=torch.bool, device=q.device)
    seen = (prefix[:, None] & (picked | tail[:, None, None, :])) | above[:, None]
    return [_attend(q, k, v, seen), _words(chosen), s["summaries"]]


def _words(chosen):
    """Truth values over blocks as bits of 32-bit words."""
    b, kv, t, n = chosen.shape
    w = (n + 31) // 32
    bits = torch.zeros((b, kv, t, w * 32), dtype=torch.int64, device=chosen.device)
    bits[..., :n] = chosen
    word = (bits.view(b, kv, t, w, 32) << torch.arange(32, device=chosen.device)).sum(4)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)


def _take(k, is_v, b, key):
    """Rows `key` [B, T] of sequences b [B, 1] of all layers, D last."""
    if not _grouped(k):
        return k[:, b, key]
    lead, d = k.shape[:4], k.shape[-1]
    if is_v:
        return k.view(*lead, d // 16, 4, 16, 8)[:, b, :, key // 32, :, (key // 8) % 4, :, key % 8]
    return k.view(*lead, 2, d // 32, 4, 4, 4, 8)[:, b, :, key // 32, (key // 4) % 2, :, :, (key // 8) % 4, key % 4, :]


def _put(k, is_v, b, key, rows):
    if not _grouped(k):
        k[:, b, key] = rows
    elif is_v:
        k.view(*k.shape[:4], k.shape[-1] // 16, 4, 16, 8)[:, b, :, key // 32, :, (key // 8) % 4, :, key % 8] = rows
    else:
        k.view(*k.shape[:4], 2, k.shape[-1] // 32, 4, 4, 4, 8)[:, b, :, key // 32, (key // 4) % 2, :, :, (key // 8) % 4, key % 4, :] = rows


def _new_rows(new, k, is_v):
    """New rows [layers, B, T, heads, D] as _take() gives them."""
    if not _grouped(k):
        return new.to(k.dtype)
    x = new.to(k.dtype).permute(1, 2, 0, 3, 4)
    d = k.shape[-1]
    return x.reshape(*x.shape[:-1], d // 16, 16) if is_v else x.reshape(*x.shape[:-1], d // 32, 4, 8)


def _plain_store(s):
    b, t = s["new_k"].shape[1:3]
    seq, i = torch.arange(b, device=s["k"].device)[:, None], torch.arange(t, device=s["k"].device)
    key, there = s["start"].long()[:, None] + i, i < s["count"][:, None]
    for cache, new, is_v in ((s["k"], s["new_k"], False), (s["v"], s["new_v"], True)):
        rows = _new_rows(new, cache, is_v)
        at = 0 if _grouped(cache) else 1
        there_ = there.view((1,) * at + (b, t) + (1,) * (rows.dim() - 2 - at))
        _put(cache, is_v, seq, key, torch.where(there_, rows, _take(cache, is_v, seq, key)))


def _plain_commit(s):
    _plain_store(s)
    c, parent, token = s["c"], s["parent"].long(), s["token"].long()
    b, t = parent.shape
    i = torch.arange(t, device=parent.device)
    there = (parent >= -1) & (parent < i)
    want = torch.cat([s["expect"][:, None], s["best"]], 1).long().gather(1, parent.clamp(-1, t - 1) + 1)
    match = there & (token == want)
    rival = (parent[:, :, None] == parent[:, None, :]) & match[:, None, :] & (i[None, :] < i[:, None])
    match = match & ~rival.any(2)
    anc = _ancestors(s["parent"])
    good = anc.any(2) & (~anc | match[:, None, :]).all(2)
    order = torch.sort(torch.where(good, i, i + t), dim=1).values
    node = order % t
    end = (token.gather(1, node) == 2) & (order < t)
    kept = (order < t) & (torch.cumsum(end.long(), 1) - end.long() == 0) & (i < s["room"][:, None])
    accepted = kept.sum(1)
    path = torch.where(kept, node, torch.full_like(node, -1))
    last = torch.where(accepted > 0, node.gather(1, (accepted - 1).clamp(min=0)[:, None])[:, 0], torch.full_like(accepted, -1))
    following = torch.cat([s["expect"][:, None], s["best"]], 1).gather(1, last[:, None] + 1)[:, 0]
    seq, length = torch.arange(b, device=parent.device)[:, None], s["length"].long()[:, None]
    source = length + torch.where(kept, node, i.expand_as(node))
    for cache, is_v in ((s["k"], False), (s["v"], True)):
        _put(cache, is_v, seq, length + i, _take(cache, is_v, seq, source))
    return [path.to(torch.int32), accepted.to(torch.int32), following.to(torch.int32), (s["length"] + accepted).to(torch.int32), s["k"], s["v"]]


def run(state):
    s, c = state, state["c"]
    if not own:
        if c["call"] == "store":
            _plain_store(s)
            return [s["k"], s["v"]]
        return {"tree": _plain_tree, "sparse": _plain_sparse, "commit": _plain_commit}[c["call"]](s)
    from paper_1811_03115_amd.binding import Context as bpd
    cache = (s["k"], s["v"])
    if c["call"] == "tree":
        return bpd.bpd_tree_attention(cache, s["q"], s["length"], None if c["chain"] else s["parent"])
    if c["call"] == "sparse":
        out, chosen = bpd.bpd_sparse_attention(cache, s["q"], s["length"], s["summaries"], block=c["block"], first=c["first"], recent=c["recent"], top=c["top"],
                                               parent=None if c["chain"] else s["parent"], added=s["added"])
        return [out, chosen, s["summaries"]]
    bpd.bpd_cache_store(cache, s["new_k"], s["new_v"], s["start"], s["count"])
    if c["call"] == "store":
        return [s["k"], s["v"]]
    return [*bpd.bpd_tree_accept(s["parent"], s["token"], s["expect"], s["best"], s["length"], cache=cache, room=s["room"], eos_id=2), s["k"], s["v"]]


# ------------------------------------------------------------------------------------------------ what they have to do

def work(case):
    """Every key and value that a call has to see read once, what it makes written once.  Of chosen blocks those of one row, which the others may share."""
    c = case
    size, b, t, kv, d = 4 if c["dtype"] == "f32" else 2, c["batch"], c["rows"], c["kv"], c["dim"]
    n = _lengths(c).astype(float)
    row = 2.0 * kv * d * size
    if c["call"] == "store":
        return {"bytes": 2 * float(_counts(c).sum()) * row, "flops": 0.0}
    if c["call"] == "commit":                                 # stored once; half of a tree at most moves
        return {"bytes": 2.0 * b * t * row * c["layers"], "flops": 0.0}
    io = 2.0 * b * t * c["heads"] * d * size
    if c["call"] == "tree":
        return {"bytes": float((n + t).sum()) * row + io, "flops": float((4 * (n + 1) * t * c["heads"] * d).sum())}
    done = n // c["block"]
    seen = np.minimum(done, c["first"] + c["recent"] + c["top"]) * c["block"] + n % c["block"]
    return {"bytes": float((done + seen + t).sum()) * row + io, "flops": float((4 * (done + seen + 1) * t * c["heads"] * d).sum())}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits

def _exact_rows(parent, i):
    """Nodes above node i and i itself, None if one of them is absent."""
    got = []
    while i != -1:
        p = int(parent[i])
        if p < -1 or p >= i:
            return None
        got.append(i)
        i = p
    return got


def _exact_chosen(q, k, c, n):
    """Blocks that the row's heads q [heads, D] of one key head see, of n committed rows: keys k [rows, D], all in 64 bits."""
    done = n // c["block"]
    always = set(range(min(c["first"], done))) | set(range(max(0, done - c["recent"]), done))
    if not done:
        return []
    x = k[:done * c["block"]].view(done, c["block"], -1)
    low, high = x.amin(1), x.amax(1)
    bound = sum(torch.maximum(h * low, h * high).sum(1) for h in q).cpu().numpy()
    rest = sorted((j for j in range(done) if j not in always), key=lambda j: (-bound[j], j))
    return sorted(always | set(rest[:c["top"]]))


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    b, t, kv, group, d = c["batch"], c["rows"], c["kv"], c["heads"] // c["kv"], c["dim"]
    parents, lengths = _parents(c), _lengths(c)
    if c["call"] in ("tree", "sparse"):
        if c["call"] == "sparse" and b * kv * t > 3000:
            return None
        out = torch.zeros((b, t, c["heads"], d), dtype=torch.float64, device="cuda")
        blocks = _capacity(c) // c["block"] if c["block"] else 0
        words = np.zeros((b, kv, t, (blocks + 31) // 32, 32), bool)
        for s in range(b):
            n = int(lengths[s])
            above = [_exact_rows(parents[s], i) for i in range(t)]
            for h in range(kv):
                k, v = x["k"][0, s, :n + t, h].double(), x["v"][0, s, :n + t, h].double()
                q = x["q"][s, :, h * group:(h + 1) * group].double()
                seen = torch.zeros((t, n + t), dtype=torch.bool)
                for i in range(t):
                    if above[i] is None:
                        continue
                    seen[i, :n] = True
                    if c["call"] == "sparse":
                        picks = _exact_chosen(q[i], k, c, n)
                        seen[i, :n // c["block"] * c["block"]] = False
                        for j in picks:
                            seen[i, j * c["block"]:(j + 1) * c["block"]] = True
                            words[s, h, i, j // 32, j % 32] = True
                    seen[i, [n + a for a in above[i]]] = True
                seen = seen.cuda()
                score = (q.reshape(t * group, d) @ k.T / math.sqrt(d)).view(t, group, -1)
                p = torch.softmax(torch.where(seen[:, None], score, torch.full_like(score, -1e300)), 2) * seen.any(1)[:, None, None]
                out[s, :, h * group:(h + 1) * group] = (p.view(t * group, -1) @ v).view(t, group, d)
        if c["call"] == "tree":
            return out
        word = (words.astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)
        return [out, torch.from_numpy(word).cuda(), _summaries(x["k"][0], c["block"])]
    k, v = x["k"], x["v"]
    start, count = x["start"].tolist(), x["count"].tolist()
    for s in range(b):
        k[:, s, start[s]:start[s] + count[s]] = x["new_k"][:, s, :count[s]]
        v[:, s, start[s]:start[s] + count[s]] = x["new_v"][:, s, :count[s]]
    if c["call"] == "store":
        return [*_pack(k, v)]
    path, token, best, expect, room = np.full((b, t), -1, np.int32), x["token"].cpu().numpy(), x["best"].cpu().numpy(), x["expect"].cpu().numpy(), x["room"].cpu().numpy()
    accepted, following, after = np.zeros(b, np.int32), expect.copy(), lengths.astype(np.int32)
    for s in range(b):
        at = -1
        while accepted[s] < room[s] and not (at >= 0 and token[s, at] == 2):
            step = [i for i in range(at + 1, t) if parents[s, i] == at and token[s, i] == following[s]]
            if not step:
                break
            at = step[0]
            path[s, accepted[s]] = at
            accepted[s] += 1
            following[s] = best[s, at]
        n, a = int(lengths[s]), int(accepted[s])
        rows = torch.from_numpy(path[s, :a].astype(np.int64)).cuda() + n
        k[:, s, n:n + a], v[:, s, n:n + a] = k[:, s, rows].clone(), v[:, s, rows].clone()
        after[s] += a
    return [torch.from_numpy(path).cuda(), torch.from_numpy(accepted).cuda(), torch.from_numpy(following).cuda(), torch.from_numpy(after).cuda(), *_pack(k, v)]
