"""The cache operators (rows stored, attention of a tree of drafts, over chosen blocks, trees verified) against their plain definition in 64 bits
(cache_reference.py), through the public entry points."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from paper_1811_03115_amd import binding
from paper_1811_03115_amd.binding import Context as bpd

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def tree(rng, b, t, kind):
    if kind == "chain":
        return None
    p = np.tile(np.arange(t) - 1, (b, 1))
    p = np.where(rng.random((b, t)) < 0.5, p, np.minimum(rng.integers(-1, np.maximum(1, np.arange(t)), (b, t)), np.arange(t) - 1))
    if kind == "odd":                              # absent nodes in the middle and at the end, by every kind of parent that is none
        p = np.where(rng.random((b, t)) < 0.15, rng.choice([-2, -7, 64, 1 << 30, -(1 << 31)], (b, t)), p)
        p = np.where(rng.random((b, t)) < 0.05, np.arange(t), p)
    return p.astype(np.int32)


def rows(rng, *shape, dtype=BF, peak=1.0):
    return (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)) * peak).to(dtype)


def cuda(x):
    return None if x is None else (torch.from_numpy(x).cuda() if isinstance(x, np.ndarray) else x.cuda())


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache_of(rng, b, cap, kv, d, dtype, lengths, t, parent=None):
    """Random keys and values, NaN where nothing has been stored and where a node is absent."""
    k, v = rows(rng, b, cap, kv, d, dtype=dtype), rows(rng, b, cap, kv, d, dtype=dtype)
    for s, n in enumerate(lengths):
        end = 0 if n < 0 else min(cap, n + t)
        none = list(range(end, cap))
        if parent is not None and n >= 0:
            none += [n + i for i, a in enumerate(ref.ancestors(parent[s], t)) if a is None and n + i < cap]
        k[s, none], v[s, none] = float("nan"), float("nan")
    return k, v


def same_bits(a, b):
    kind = torch.int16 if a.element_size() == 2 else torch.int32
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


# heads of K, heads per head of K, nodes, lengths, capacity, tree
SHAPES = [
    (1, 1, 1, [0], 32, "chain"), (2, 1, 1, [1, 31], 32, "chain"), (1, 1, 3, [29, 30, -1, 32], 32, "chain"), (3, 1, 10, [0, 33, 95, 64], 128, "tree"),
    (2, 4, 12, [130, 7], 160, "odd"), (1, 8, 64, [100], 192, "tree"), (5, 1, 16, [31, 32, 33], 64, "odd"), (1, 3, 11, [200, 255], 288, "tree"),
    (2, 1, 7, [700, 1017, 1024, 3], 1024, "tree"), (1, 3, 16, [90, 31], 128, "odd"), (1, 7, 7, [500], 544, "tree"), (1, 1, 17, [5000, 40], 5056, "tree"), (1, 1, 3, [4700, 4097, 1, -1], 4704, "tree"), (1, 1, 33, [2000], 2048, "odd"), (1, 64, 1, [77], 96, "chain"), (2, 2, 64, [1500, 0], 1600, "odd"),
]


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 64), (F32, 128), (BF, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("kv,g,t,lengths,cap,kind", SHAPES, ids=lambda x: str(x).replace(" ", ""))
def test_tree_attention(dtype, d, kv, g, t, lengths, cap, kind):
    rng = np.random.default_rng(d + t + cap)
    b = len(lengths)
    parent = tree(rng, b, t, kind)
    k, v = cache_of(rng, b, cap, kv, d, dtype, lengths, t, parent)
    q = rows(rng, b, t, kv * g, d, dtype=dtype, peak=1.5)
    want, off, _ = ref.attention(q, k, v, lengths, parent)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    got = bpd.bpd_tree_attention(cache, cuda(q), ints(lengths), cuda(parent))
    ref.check(got, want, off)
    again = bpd.bpd_tree_attention(cache, cuda(q), ints(lengths), cuda(parent))
    assert torch.equal(got, again)


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("q_type,o_type", [(F32, F32), (F32, BF), (BF, F32)])
def test_tree_attention_types(d, q_type, o_type):
    """Queries and results of other types than the cache's, and a scale of its own."""
    rng = np.random.default_rng(d)
    for lengths, t, kv, g in (([40, 300], 5, 2, 2), ([333], 40, 1, 1)):
        b, cap = len(lengths), 384
        k, v = cache_of(rng, b, cap, kv, d, BF, lengths, t)
        q, parent = rows(rng, b, t, kv * g, d, dtype=q_type), tree(rng, b, t, "tree")
        want, off, _ = ref.attention(q, k, v, lengths, parent, scale=0.2)
        out = torch.empty(q.shape, dtype=o_type, device="cuda")
        assert bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k, v)), cuda(q), ints(lengths), cuda(parent), scale=0.2, out=out) is out
        ref.check(out, want, off)


@pytest.mark.parametrize("shift", [0, 1, 3, 8])
def test_tree_attention_strides(shift):
    """Queries inside a projection of all three, at any element; results into a larger array, whose other elements stay."""
    rng = np.random.default_rng(5)
    b, t, kv, g, d, cap, lengths = 2, 9, 2, 3, 64, 96, [50, 61]
    k, v = cache_of(rng, b, cap, kv, d, BF, lengths, t)
    h = kv * g
    fused = rows(rng, b, t, shift + (h + 2 * kv) * d + 5).cuda()
    q = fused[:, :, shift:shift + h * d].view(b, t, h, d) if shift == 0 else fused[:, :, shift:shift + h * d].unflatten(2, (h, d))
    parent = tree(rng, b, t, "tree")
    want, off, _ = ref.attention(q.cpu(), k, v, lengths, parent)
    big = torch.full((t, b, h, d + shift), 7.0, dtype=BF, device="cuda")
    out = big.permute(1, 0, 2, 3)[..., shift:]
    bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k, v)), q, ints(lengths), cuda(parent), out=out)
    ref.check(out.contiguous(), want, off)
    assert bool((big[..., :shift] == 7).all())


def test_tree_attention_layer_and_stream():
    """A layer of several; a stream of its own."""
    rng = np.random.default_rng(6)
    b, t, kv, d, cap, lengths = 2, 4, 2, 64, 64, [20, 50]
    k, v = rows(rng, 3, b, cap, kv, d), rows(rng, 3, b, cap, kv, d)
    q = rows(rng, b, t, kv, d)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    qd, n = cuda(q), ints(lengths)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for layer in range(3):
        want, off, _ = ref.attention(q, k[layer], v[layer], lengths, None)
        with torch.cuda.stream(side):
            got = bpd.bpd_tree_attention(cache, qd, n, layer=layer)
        side.synchronize()
        ref.check(got, want, off)


@pytest.mark.parametrize("d,dtype", [(64, BF), (128, BF), (16, F32)])
def test_extreme_scores(d, dtype):
    """Scores that overflow exp if no maximum is subtracted, one key that takes all, equal keys, values of one size (the weights add up to one)."""
    rng = np.random.default_rng(7)
    b, t, kv, cap, lengths = 1, 6, 1, 320, [300]
    k, v = cache_of(rng, b, cap, kv, d, dtype, lengths, t)
    k[0, 17], k[0, 200] = k[0, 17] * 30, k[0, 201]
    q = rows(rng, b, t, kv, d, dtype=dtype, peak=8.0)
    q[0, 3] = 0
    parent = tree(rng, b, t, "tree")
    want, off, _ = ref.attention(q, k, v, lengths, parent)
    ref.check(bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k, v)), cuda(q), ints(lengths), cuda(parent)), want, off)
    v[:, :lengths[0] + t] = 3.0
    want, off, _ = ref.attention(q, k, v, lengths, parent)
    got = bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k, v)), cuda(q), ints(lengths), cuda(parent))
    ref.check(got, want, off)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 64), (BF, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("kv,g,t,n,cap", [(2, 1, 9, 70, 96), (1, 2, 13, 400, 448), (1, 3, 20, 700, 1024), (1, 8, 12, 333, 1024), (1, 1, 2, 31, 64)])
def test_what_others_see_does_not_matter(dtype, d, kv, g, t, n, cap):
    """Keys and values that are not finite, in drafts of other branches, in absent nodes and in blocks that only other nodes chose: results as without them; who sees them gets what
    the formula gives."""
    rng = np.random.default_rng(d + t)
    parent = np.array([[-1] + [max(0, i - 2) for i in range(1, t)]], np.int32)          # two branches
    if t > 3:
        parent[0, t - 1] = -3
    k, v = cache_of(rng, 1, cap, kv, d, dtype, [n], t, parent)
    q = rows(rng, 1, t, kv * g, d, dtype=dtype)
    bad = t - 2 if t > 3 else t - 1                # a leaf
    sees = [i for i, a in enumerate(ref.ancestors(parent[0], t)) if a is not None and bad in a]
    clean = ref.attention(q, k, v, [n], parent)
    for value in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        v2[0, n + bad, :, ::3] = value
        if value != value:
            k2[0, n + bad, :, 5] = value
        got = bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k2, v2)), cuda(q), ints([n]), cuda(parent)).cpu()
        others = [i for i in range(t) if i not in sees]
        ref.check(got[:, others], clean[0][:, others], clean[1][:, others], what=str(value))
        want = ref.attention(q, k2, v2, [n], parent)[0]
        hit = ~torch.isfinite(want)
        assert hit.any() and torch.equal(torch.isnan(got.double()), torch.isnan(want)) and torch.equal(got.double()[hit & ~torch.isnan(want)], want[hit & ~torch.isnan(want)])
        # a block that some of the nodes choose
        what = dict(block=32, first=0, recent=0, top=1)
        _, _, picks = ref.attention(q, k, v, [n], parent, blocks=what)
        words = picks.numpy().view(np.uint32)[0, 0]
        block = next((j for j in range(n // 32) if 0 < sum(int(w[j // 32]) >> (j % 32) & 1 for w in words) < len(words)), None)
        if block is None or kv > 1:
            continue
        v2 = v.clone()
        v2[0, block * 32 + 3, 0, 1::2] = value
        cache = tuple(cuda(x) for x in ref.pack(k, v2))
        got, chosen = bpd.bpd_sparse_attention(cache, cuda(q), ints([n]), binding.new_summaries(cache, 32), parent=cuda(parent), **what)
        assert torch.equal(chosen.cpu(), picks)
        want, off, _ = ref.attention(q, k, v2, [n], parent, blocks=what)
        fine = torch.isfinite(want).all(3).all(2)[0]
        assert fine.any() and not fine.all()
        ref.check(got[:, fine], want[:, fine], off[:, fine])
        assert torch.equal(torch.isnan(got.cpu().double()), torch.isnan(want))


def test_many_rows_and_fewer_sequences():
    """64 nodes times 64 heads on a key head; fewer sequences than the cache has; lengths past its end; results in the queries' place."""
    rng = np.random.default_rng(12)
    for d, dtype in ((64, BF), (128, BF), (16, F32)):
        b, t, kv, g, cap, lengths = 2, 64, 1, 64, 160, [90, 161]
        k, v = rows(rng, 4, cap, kv, d, dtype=dtype), rows(rng, 4, cap, kv, d, dtype=dtype)
        q, parent = rows(rng, b, t, kv * g, d, dtype=dtype), tree(rng, b, t, "tree")
        want, off, _ = ref.attention(q, k[:b], v[:b], lengths, parent)
        out = cuda(q).clone()
        got = bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k, v)), out, ints(lengths), cuda(parent), out=out)
        ref.check(got, want, off)
        assert not bool(got[1].any())


def test_negative_and_zero_scales():
    rng = np.random.default_rng(13)
    for d, dtype in ((64, BF), (128, BF), (16, F32)):
        k, v = rows(rng, 1, 320, 1, d, dtype=dtype), rows(rng, 1, 320, 1, d, dtype=dtype)
        q = rows(rng, 1, 5, 2, d, dtype=dtype)
        for scale in (-0.3, 0.0, 2.0, 1e-20):
            want, off, _ = ref.attention(q, k, v, [300], None, scale=scale)
            ref.check(bpd.bpd_tree_attention(tuple(cuda(x) for x in ref.pack(k, v)), cuda(q), ints([300]), scale=scale), want, off, what=str(scale))


def test_far_offsets():
    """A cache of more than 2^32 bytes: the last sequence's rows are read, stored and moved where they are."""
    rng = np.random.default_rng(8)
    b, kv, d, cap, t = 37, 8, 128, 65536, 5
    k, v = binding.new_cache(b, kv, d, cap)
    assert k.numel() * 2 > 1 << 32
    n = 300
    lengths, first = torch.full((b,), -1, dtype=torch.int32), torch.full((b,), -1, dtype=torch.int32)
    lengths[-1], first[-1] = n, 0
    kk, vv = rows(rng, 1, n + t, kv, d), rows(rng, 1, n + t, kv, d)
    bpd.bpd_cache_store((k, v), cuda(kk).expand(b, -1, -1, -1), cuda(vv).expand(b, -1, -1, -1), cuda(first))
    q = rows(rng, 1, t, kv, d)
    got = bpd.bpd_tree_attention((k, v), cuda(q).expand(b, -1, -1, -1), cuda(lengths))
    want, off, _ = ref.attention(q, kk, vv, [n], None)
    ref.check(got[-1:], want, off)
    assert not bool(got[:-1].any())
    # the far end of a sequence
    first[-1] = cap - t - 3
    bpd.bpd_cache_store((k, v), cuda(kk)[:, :3 + t].expand(b, -1, -1, -1), cuda(vv)[:, :3 + t].expand(b, -1, -1, -1), cuda(first))
    tail = ref.unpack(k[-1:, :, -1:].cpu(), v[-1:, :, -1:].cpu())
    assert torch.equal(tail[0][0, 32 - t - 3:], kk[0, :t + 3]) and torch.equal(tail[1][0, 32 - t - 3:], vv[0, :t + 3])


# ------------------------------------------------------------------------------------------------ store

def test_largest_capacity():
    """2^24 rows, all of them the same row, stored by one call and attended to: sums of 2^24 powers of two of one size are exact in 32 bits, and what
    is left is the rounding of a quotient, less than half a step of bf16."""
    n = 1 << 24
    cache = binding.new_cache(1, 1, 16, n)
    row = torch.tensor([2.0 ** (i % 5 - 2) * (-1) ** (i // 5) for i in range(16)], dtype=BF, device="cuda")
    bpd.bpd_cache_store(cache, row.expand(1, n, 1, 16), row.expand(1, n, 1, 16), ints([0]))
    for x in cache:
        assert bool((x.view(n, 16) == row).all())
    for length, t in ((n, 1), (n - 2, 2)):
        out = bpd.bpd_tree_attention(cache, torch.zeros(1, t, 1, 16, dtype=BF, device="cuda"), ints([length]))
        want = [row * 0 if length + i >= n else row for i in range(t)]
        assert torch.equal(out[0, :, 0], torch.stack(want))


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 64), (F32, 128), (BF, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("src", [BF, F32], ids=["from_bf16", "from_f32"])
@pytest.mark.parametrize("layers", [0, 3])
def test_store(dtype, d, src, layers):
    rng = np.random.default_rng(d)
    b, kv, cap, t = 7, 3, 160, 45
    lead = (layers,) if layers else ()
    k, v = rows(rng, *lead, b, cap, kv, d, dtype=dtype), rows(rng, *lead, b, cap, kv, d, dtype=dtype)
    start, count = [0, 1, 31, 130, -1, 159, 64], [45, 0, 33, 45, 45, 45, 1]
    cache = tuple(cuda(x).clone() for x in ref.pack(k, v))
    fused = rows(rng, *lead, b, t, 3 * kv, d, dtype=src).cuda()
    nk, nv = fused[..., kv:2 * kv, :], fused[..., 2 * kv:, :]
    for counts in (None, count, [t + 9, -5, 2, 3, 4, 5, 6]):
        bpd.bpd_cache_store(cache, nk, nv, ints(start), None if counts is None else ints(counts))
        for s in range(b):
            c = t if counts is None else max(0, min(t, counts[s]))
            end = min(cap, start[s] + c) if start[s] >= 0 else start[s]
            if end > start[s]:
                at = (slice(None),) * len(lead) + (s, slice(start[s], end))
                of = (slice(None),) * len(lead) + (s, slice(0, end - start[s]))
                k[at], v[at] = nk.cpu()[of].to(dtype), nv.cpu()[of].to(dtype)
        got = ref.unpack(*(x.cpu() for x in cache))
        assert torch.equal(got[0], k) and torch.equal(got[1], v)
        nk, nv = nv, nk


def test_store_unaligned():
    rng = np.random.default_rng(1)
    b, kv, d, cap, t = 2, 2, 64, 64, 20
    cache = binding.new_cache(b, kv, d, cap)
    for x in cache:
        x.zero_()
    flat = rows(rng, b, t, 1 + 2 * kv * d + 3).cuda()
    nk, nv = flat[..., 1:1 + kv * d].unflatten(2, (kv, d)), flat[..., 1 + kv * d:1 + 2 * kv * d].unflatten(2, (kv, d))
    bpd.bpd_cache_store(cache, nk, nv, ints([3, 44]))
    got = ref.unpack(*(x.cpu() for x in cache))
    for g, n in zip(got, (nk, nv)):
        want = torch.zeros((b, cap, kv, d), dtype=BF)
        want[0, 3:23], want[1, 44:64] = n.cpu()[0], n.cpu()[1]
        assert torch.equal(g, want)


# ------------------------------------------------------------------------------------------------ sparse

SPARSE = [
    # kv, g, T, lengths, capacity, tree, block, first, recent, top
    (2, 1, 1, [500], 512, "chain", 32, 1, 1, 4), (1, 4, 6, [300, 31, 32, 0], 320, "tree", 32, 0, 0, 3), (2, 2, 9, [1000, 640, -1], 1056, "odd", 64, 1, 2, 2),
    (1, 1, 20, [2200], 2304, "tree", 32, 2, 3, 20), (1, 2, 5, [400, 900], 960, "tree", 128, 0, 1, 1), (2, 1, 3, [90], 96, "chain", 64, 1, 1, 0),
    (1, 1, 2, [100, 20], 128, "chain", 32, 50, 50, 50), (1, 3, 17, [700], 736, "odd", 32, 0, 0, 0), (1, 8, 4, [4200], 4256, "tree", 32, 1, 4, 27),
    (1, 1, 4, [40], 64, "tree", 128, 1, 1, 1),
]


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 64), (BF, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("kv,g,t,lengths,cap,kind,block,first,recent,top", SPARSE, ids=lambda x: str(x).replace(" ", ""))
def test_sparse_attention(dtype, d, kv, g, t, lengths, cap, kind, block, first, recent, top):
    rng = np.random.default_rng(d + t + cap)
    b = len(lengths)
    parent = tree(rng, b, t, kind)
    k, v = cache_of(rng, b, cap, kv, d, dtype, lengths, t, parent)
    if cap > 200 and max(lengths) > 160:                                  # blocks with the same bound: the lower one goes first
        k[:, 96:128], k[:, 32:64] = k[:, 128:160], k[:, 128:160]
    q = rows(rng, b, t, kv * g, d, dtype=dtype)
    what = dict(block=block, first=first, recent=recent, top=top)
    want, off, picks = ref.attention(q, k, v, lengths, parent, blocks=what)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    summ = binding.new_summaries(cache, block)
    summ.fill_(float("nan"))
    got, chosen = bpd.bpd_sparse_attention(cache, cuda(q), ints(lengths), summ, parent=cuda(parent), **what)
    assert torch.equal(chosen.cpu(), picks)
    ref.check(got, want, off)
    kept = ref.summaries_unpacked(summ.cpu(), cap // block)
    for s, n in enumerate(lengths):
        done = max(0, min(n, cap)) // block
        assert torch.equal(kept[s, :, :done], ref.summaries(k[s:s + 1], block)[0, :, :done])
    # from the next call on only what has been added
    if min(lengths) >= 0:
        for added in ([0] * b, [min(n, 40) for n in lengths], [1 << 30] * b):
            got2, chosen2 = bpd.bpd_sparse_attention(cache, cuda(q), ints(lengths), summ, parent=cuda(parent), added=ints(added), **what)
            assert torch.equal(chosen2, chosen) and same_bits(got2, got)


def test_sparse_sees_only_what_was_added():
    """Summaries of blocks that no new row lies in are the caller's."""
    rng = np.random.default_rng(3)
    b, kv, d, cap, block = 1, 1, 64, 320, 32
    k, v = rows(rng, b, cap, kv, d), rows(rng, b, cap, kv, d)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    summ = binding.new_summaries(cache, block)
    summ.fill_(5.0)
    q = rows(rng, b, 1, kv, d)
    bpd.bpd_sparse_attention(cache, cuda(q), ints([200]), summ, block=block, first=0, recent=0, top=2, added=ints([10]))
    kept, fresh = ref.summaries_unpacked(summ.cpu(), cap // block), ref.summaries(k, block)
    assert bool((kept[0, 0, :5] == 5).all()) and torch.equal(kept[0, 0, 5], fresh[0, 0, 5]) and bool((kept[0, 0, 6:] == 5).all())


def test_sparse_many_blocks():
    """As many blocks as are allowed, bounds that differ in their last bits only, and all the same."""
    d, block, cap = 64, 32, binding.BLOCKS_MAX * 32
    k = torch.zeros((1, cap, 1, d), dtype=BF)
    q = torch.zeros((1, 2, 1, d), dtype=BF)
    q[0, 0, 0, 0], q[0, 0, 0, 1], q[0, 1, 0, 2] = 1.0, 1.0, 1.0
    rng = np.random.default_rng(4)
    order = rng.permutation(binding.BLOCKS_MAX)
    first = torch.arange(cap) // block
    k[0, :, 0, 0] = 128.0
    k[0, :, 0, 1] = ((torch.from_numpy(order)[first] // 16).float() / 256).to(BF)          # 256 values, sixteen blocks of each
    v = rows(rng, 1, cap, 1, d)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    summ = binding.new_summaries(cache, block)
    n = cap - 7
    for top in (1, 37, 1000, 4095):
        want, off, picks = ref.attention(q, k, v, [n - 2], None, blocks=dict(block=block, first=0, recent=0, top=top))
        got, chosen = bpd.bpd_sparse_attention(cache, cuda(q), ints([n - 2]), summ, block=block, first=0, recent=0, top=top)
        assert torch.equal(chosen.cpu(), picks), top
        ref.check(got, want, off)


@pytest.mark.parametrize("blocks", [1, 64, 65, 128, 129, 500, 512, 513, 1600])
def test_sparse_which_blocks(blocks):
    """Which blocks are chosen, in one tile and in many: bounds of both signs, with many ties, infinite ones and ones that are no number."""
    rng = np.random.default_rng(blocks)
    d, block, kv, b = 64, 32, 2, 2
    cap = blocks * block
    k = torch.from_numpy(rng.integers(-2, 3, (b, blocks, 1, kv, d)).astype(np.float32)).repeat(1, 1, block, 1, 1).reshape(b, cap, kv, d)
    k[:, :, :, 2:] *= 0.125
    k[0, ::max(1, cap // 7), 0, 0] = float("inf")
    k[1, cap // 3:cap // 3 + 40, 1, 1] = float("-inf")
    k = k.to(BF)
    v = rows(rng, b, cap, kv, d)
    q = torch.zeros((b, 4, kv, d))
    q[:, 0, :, :2] = torch.tensor([1.0, -1.0])
    q[:, 1, :, :2] = torch.tensor([-3.0, 2.0])
    q[:, 2] = rows(rng, b, kv, d, dtype=F32)
    q = q.to(BF)                                                          # (node 3: bounds of zero, or none)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    parent = np.full((b, 4), -1, np.int32)
    summ = binding.new_summaries(cache, block)
    lengths = [max(0, cap - 4), cap // 2]
    for first, recent, top in ((0, 0, 1), (1, 2, max(1, blocks // 3)), (0, 0, blocks), (2, 1, 0)):
        what = dict(block=block, first=first, recent=recent, top=top)
        _, _, picks = ref.attention(q, k, v, lengths, parent, blocks=what)
        _, chosen = bpd.bpd_sparse_attention(cache, cuda(q), ints(lengths), summ, parent=cuda(parent), **what)
        assert torch.equal(chosen.cpu(), picks), what


# ------------------------------------------------------------------------------------------------ accept

@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 128), (BF, 16), (None, 0)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("t,kind", [(1, "tree"), (10, "tree"), (10, "odd"), (64, "tree"), (64, "odd"), (33, "chain")])
def test_accept(dtype, d, t, kind):
    rng = np.random.default_rng(t + d)
    b, kv, cap, nl = 40, 2, 96, 2
    parent = tree(rng, b, t, kind)
    if parent is None:
        parent = np.tile(np.arange(t, dtype=np.int32) - 1, (b, 1))
    best, expect = rng.integers(0, 3, (b, t)).astype(np.int32), rng.integers(0, 3, b).astype(np.int32)
    token = rng.integers(0, 3, (b, t)).astype(np.int32)
    sure = rng.random((b, t)) < 0.6
    chain = np.concatenate([expect[:, None], best], 1)
    token = np.where(sure, np.take_along_axis(chain, np.clip(parent, -1, t - 1) + 1, 1), token).astype(np.int32)
    length = rng.integers(-1, cap - 20, b).astype(np.int32)
    length[:4] = [0, cap - 3, cap, -5]
    room = rng.integers(-1, t + 3, b).astype(np.int32)
    cache = None
    if dtype is not None:
        k, v = rows(rng, nl, b, cap, kv, d, dtype=dtype), rows(rng, nl, b, cap, kv, d, dtype=dtype)
        cache = tuple(cuda(x).clone() for x in ref.pack(k, v))
    eos = 1 if kind == "tree" else -1
    for r in (None, room):
        path, accepted, following, after = (x.cpu().numpy() for x in bpd.bpd_tree_accept(cuda(parent), cuda(token), cuda(expect), cuda(best), cuda(length), cache=cache, room=cuda(r), eos_id=eos))
        moved = 0
        for s in range(b):
            p, nxt = ref.accept(parent[s], token[s], expect[s], best[s], length[s], None if r is None else r[s], eos, None if cache is None else cap)
            assert path[s].tolist() == p + [-1] * (t - len(p)) and accepted[s] == len(p) and following[s] == nxt and after[s] == length[s] + len(p), s
            if cache is not None and p:
                at = torch.tensor(p) + int(length[s])
                k[:, s, length[s]:length[s] + len(p)], v[:, s, length[s]:length[s] + len(p)] = k[:, s, at].clone(), v[:, s, at].clone()
                moved += p[-1] != len(p) - 1
        if cache is not None:
            got = ref.unpack(*(x.cpu() for x in cache))
            assert torch.equal(got[0], k) and torch.equal(got[1], v)
            assert moved or t == 1 or kind == "chain"


# ------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("d,dtype", [(64, BF), (128, BF), (16, F32)])
def test_steps_with_trees(d, dtype):
    """A serving loop: a prompt stored, then drafts stored, attended to, verified, moved.  The prefix is always the accepted rows, in order."""
    rng = np.random.default_rng(9)
    b, kv, g, t, cap = 3, 2, 2, 9, 256
    cache = binding.new_cache(b, kv, d, cap, dtype=dtype)
    if dtype == BF and d == 64:
        for x in cache:
            x.fill_(float("nan"))
    summ = binding.new_summaries(cache, 32)
    prefix_k, prefix_v = [[] for _ in range(b)], [[] for _ in range(b)]
    length = ints([0] * b)
    pk, pv, count = rows(rng, b, 70, kv, d, dtype=dtype), rows(rng, b, 70, kv, d, dtype=dtype), [70, 1, 33]
    bpd.bpd_cache_store(cache, cuda(pk), cuda(pv), length, ints(count))
    for s in range(b):
        prefix_k[s], prefix_v[s] = list(pk[s, :count[s]]), list(pv[s, :count[s]])
    length, added = ints(count), None
    for step in range(12):
        parent = tree(rng, b, t, "odd" if step % 3 == 2 else "tree")
        nk, nv, q = rows(rng, b, t, kv, d, dtype=dtype), rows(rng, b, t, kv, d, dtype=dtype), rows(rng, b, t, kv * g, d, dtype=dtype)
        bpd.bpd_cache_store(cache, cuda(nk), cuda(nv), length)
        got = bpd.bpd_tree_attention(cache, cuda(q), length, cuda(parent))
        what = dict(block=32, first=1, recent=1, top=1)
        some, chosen = bpd.bpd_sparse_attention(cache, cuda(q), length, summ, parent=cuda(parent), added=added, **what)
        n = [len(x) for x in prefix_k]
        k, v = torch.zeros((b, cap, kv, d), dtype=dtype), torch.zeros((b, cap, kv, d), dtype=dtype)
        for s in range(b):
            k[s, :n[s]], v[s, :n[s]] = torch.stack(prefix_k[s]), torch.stack(prefix_v[s])
            k[s, n[s]:n[s] + t], v[s, n[s]:n[s] + t] = nk[s], nv[s]
        ref.check(got, *ref.attention(q, k, v, n, parent)[:2], what=f"step {step}")
        want, off, picks = ref.attention(q, k, v, n, parent, blocks=what)
        assert torch.equal(chosen.cpu(), picks), step
        ref.check(some, want, off, what=f"step {step}, chosen blocks")
        best, expect = rng.integers(0, 2, (b, t)).astype(np.int32), rng.integers(0, 2, b).astype(np.int32)
        token = rng.integers(0, 2, (b, t)).astype(np.int32)
        path, accepted, following, length = bpd.bpd_tree_accept(cuda(parent), cuda(token), cuda(expect), cuda(best), length, cache=cache)
        added = accepted
        for s in range(b):
            p, _ = ref.accept(parent[s], token[s], expect[s], best[s], n[s], None, -1, cap)
            assert int(accepted[s]) == len(p)
            prefix_k[s] += [nk[s, i] for i in p]
            prefix_v[s] += [nv[s, i] for i in p]
    assert length.tolist() == [len(x) for x in prefix_k] and max(length.tolist()) > 80


def test_captured_steps():
    """Store, both attentions and the verification in a graph, replayed with other rows, lengths and trees, eager calls in between."""
    rng = np.random.default_rng(10)
    b, kv, g, t, d, cap = 2, 2, 2, 6, 64, 1024
    k, v = rows(rng, b, cap, kv, d), rows(rng, b, cap, kv, d)
    cache = tuple(cuda(x) for x in ref.pack(k, v))
    nk, nv, q = (torch.zeros((b, t, h, d), dtype=BF, device="cuda") for h in (kv, kv, kv * g))
    length, parent, added = ints([0, 0]), torch.zeros((b, t), dtype=torch.int32, device="cuda"), ints([1 << 30] * 2)
    token, best, expect = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((b, t), (b, t), (b,)))
    summ = binding.new_summaries(cache, 32)
    out, out2 = torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(bpd.bpd_attention_workspace_bytes(cache, b, t, kv * g, 32), dtype=torch.uint8, device="cuda")

    def step(out, out2):
        bpd.bpd_cache_store(cache, nk, nv, length)
        bpd.bpd_tree_attention(cache, q, length, parent, out=out, workspace=ws)
        _, chosen = bpd.bpd_sparse_attention(cache, q, length, summ, block=32, first=1, recent=1, top=4, parent=parent, added=added, out=out2, workspace=ws)
        return [out, out2, chosen, *bpd.bpd_tree_accept(parent, token, expect, best, length, cache=cache), *cache]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, out2)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step(out, out2)
    for n in ([0, 1], [900, 33], [1018, 500], [-1, 64]):
        for x in (nk, nv, q):
            x.copy_(rows(rng, *x.shape))
        length.copy_(ints(n)), parent.copy_(cuda(tree(rng, b, t, "tree")))
        for x in (token, best, expect):
            x.copy_(torch.from_numpy(rng.integers(0, 2, tuple(x.shape)).astype(np.int32)))
        before = [x.clone() for x in cache]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in res]
        for x, y in zip(cache, before):
            x.copy_(y)
        want = step(torch.empty_like(q), torch.empty_like(q))
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_refusals():
    """What the wrappers refuse before they call."""
    cache = binding.new_cache(2, 2, 64, 64)
    q, n = torch.zeros((2, 3, 4, 64), dtype=BF, device="cuda"), ints([0, 0])
    for call in (
        lambda: bpd.bpd_tree_attention(cache, q.half(), n), lambda: bpd.bpd_tree_attention(cache, q[..., :32], n), lambda: bpd.bpd_tree_attention(cache, q[:, :, :3], n),
        lambda: bpd.bpd_tree_attention(cache, q, n.long()), lambda: bpd.bpd_tree_attention(cache, q, n[:1]), lambda: bpd.bpd_tree_attention(cache, q.cpu(), n),
        lambda: bpd.bpd_tree_attention(cache, q, n, layer=1), lambda: bpd.bpd_tree_attention((cache[0], cache[1][:1]), q, n),
        lambda: bpd.bpd_tree_attention(cache, q, n, workspace=n[:0], scale=float("nan")),
        lambda: bpd.bpd_tree_attention(cache, torch.zeros((2, 65, 4, 64), dtype=BF, device="cuda"), n), lambda: bpd.bpd_tree_attention(cache, q.transpose(2, 3).contiguous().transpose(2, 3), n),
        lambda: bpd.bpd_cache_store(cache, q, q, n), lambda: bpd.bpd_cache_store(cache, q[:, :, :2], q[:, :, :2], n, ints([1])),
        lambda: bpd.bpd_sparse_attention(cache, q, n, binding.new_summaries(cache, 32), block=48, first=0, recent=0, top=1),
        lambda: bpd.bpd_sparse_attention(cache, q, n, binding.new_summaries(cache, 32)[:1], block=32, first=0, recent=0, top=1),
        lambda: bpd.bpd_sparse_attention(cache, q, n, binding.new_summaries(cache, 32), block=32, first=0, recent=-1, top=1),
    ):
        with pytest.raises(binding.BpdError):
            call()
    p = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    with pytest.raises(binding.BpdError):
        bpd.bpd_tree_accept(p, p, n, p, n, out=(torch.empty_like(p), n, torch.empty_like(n), torch.empty_like(n)))
    with pytest.raises(binding.BpdError):
        bpd.bpd_tree_accept(p, p, n, p[:, :2], n)
    assert bpd.bpd_tree_attention(cache, q[:0], n[:0]).shape == (0, 3, 4, 64)
    assert bpd.bpd_tree_attention(cache, q[:, :0], n).shape == (2, 0, 4, 64)
