"""The cache operators where keys, queries and scales are not the usual ones."""
import math

import numpy as np
import pytest
import torch

import cache_reference as ref
from paper_1811_03115_amd import binding
from paper_1811_03115_amd.binding import Context as bpd

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def rows(rng, *shape, dtype=BF):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def packed(k, v):
    return tuple(x.cuda() for x in ref.pack(k, v))


# ------------------------------------------------------------------------------------------------ bounds that are not finite

def bound(q, block):
    """Of the heads q [G, D] and a block's keys [rows, D], as bpd.h has it: NaN keys aside, no number where a dimension has no key but those."""
    none = torch.isnan(block)
    lo, hi = torch.where(none, torch.full_like(block, INF), block).amin(0), torch.where(none, torch.full_like(block, -INF), block).amax(0)
    one = torch.maximum(q * lo, q * hi)
    return float(torch.where(none.all(0), torch.full_like(one, NAN), one).sum())


def chosen_of(q, k, n, block, first, recent, top):
    done = n // block
    always = [j for j in range(done) if j < first or j >= done - recent]
    rest = [(bound(q, k[j * block:(j + 1) * block]), j) for j in range(done) if j not in always]
    rest.sort(key=lambda x: (math.isnan(x[0]), -x[0] if not math.isnan(x[0]) else 0, x[1]))
    return sorted(always + [j for _, j in rest[:top]])


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("g", [1, 2, 3])
@pytest.mark.parametrize("blocks,t", [(9, 4), (9, 1), (150, 5), (530, 2)])
def test_which_blocks_with_heads_that_share_keys(dtype, d, g, blocks, t):
    """Infinite keys beside heads of zero, dimensions of nothing but NaN beside heads of both signs: what the sum is defined to be ranks the block, not what the heads add up to.
    (Small whole numbers: sums are exact in any order.)"""
    rng = np.random.default_rng(blocks + 7 * g + d)
    block, kv = 32, 2
    cap = (blocks + 1) * block
    k = torch.from_numpy(rng.integers(-3, 4, (1, cap, kv, d)).astype(np.float32)) * 0.125
    for j in range(blocks):
        part = k[0, j * block:(j + 1) * block]
        kind = int(rng.integers(0, 8))
        if kind == 0:
            part[5, :, 0] = INF
        elif kind == 1:
            part[:, :, 1] = NAN
        elif kind == 2:
            part[9, :, 2] = -INF
        elif kind == 3:
            part[3:20, :, 3] = NAN
        elif kind == 4:
            part[7, :, 0], part[8, :, 2] = INF, -INF
    k = k.to(dtype)
    q = torch.from_numpy(rng.integers(-3, 4, (1, t, kv * g, d)).astype(np.float32))
    q[0, 0, :, :4] = 0
    q[0, 0, ::2, :4] = torch.tensor([1.0, 2.0, -1.0, 1.0])               # the other heads of a group: exactly zero there
    if g > 1:
        q[0, 0, 1::g, 1] = -2.0
    if t > 2:
        q[0, 2] = 0
    q = q.to(dtype)
    cache = packed(k, rows(rng, *k.shape, dtype=dtype))
    n = blocks * block + 3
    parent = np.full((1, t), -1, np.int32)
    for first, recent, top in ((0, 0, 1), (0, 0, blocks // 2), (1, 1, 3), (0, 0, blocks - 1)):
        _, chosen = bpd.bpd_sparse_attention(cache, q.cuda(), ints([n]), binding.new_summaries(cache, block), block=block, first=first, recent=recent, top=top, parent=torch.from_numpy(parent).cuda())
        got = chosen.cpu().numpy().view(np.uint32)
        for i in range(t):
            for h in range(kv):
                want = chosen_of(q[0, i, h * g:(h + 1) * g].double(), k[0, :, h].double(), n, block, first, recent, top)
                assert [j for j in range(blocks) if int(got[0, h, i, j // 32]) >> (j % 32) & 1] == want, (first, recent, top, i, h)


# ------------------------------------------------------------------------------------------------ scales

@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 64), (BF, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("kv,g,t,n,cap", [(2, 2, 6, 700, 736), (1, 1, 1, 2500, 2560), (1, 3, 19, 4100, 4160)])
def test_chosen_blocks_of_other_scales(dtype, d, kv, g, t, n, cap):
    """The blocks are those with the largest bounds of the SCORES: under a negative scale those of the queries turned round, under none all are alike."""
    rng = np.random.default_rng(d + t)
    k, v = rows(rng, 1, cap, kv, d, dtype=dtype), rows(rng, 1, cap, kv, d, dtype=dtype)
    q = rows(rng, 1, t, kv * g, d, dtype=dtype)
    parent = np.array([[-1] + [i // 2 for i in range(t - 1)]], np.int32)
    cache = packed(k, v)
    what = dict(block=32, first=1, recent=1, top=5)
    for scale in (-0.3, 0.0, -2.0, 0.3):
        sign = (scale > 0) - (scale < 0)
        want, off, picks = ref.attention(q * sign, k, v, [n], parent, scale=abs(scale) or 1.0, blocks=what)
        got, chosen = bpd.bpd_sparse_attention(cache, q.cuda(), ints([n]), binding.new_summaries(cache, 32), scale=scale, parent=torch.from_numpy(parent).cuda(), **what)
        assert torch.equal(chosen.cpu(), picks), scale
        ref.check(got, want, off, what=str(scale))


# ------------------------------------------------------------------------------------------------ scores that are not finite

# heads of K, heads per head of K, nodes, length, capacity: one part and several of the keys, rows that share keys through LDS and not
PLACES = [(2, 2, 5, 40, 64), (1, 1, 1, 0, 32), (1, 1, 3, 3000, 8192), (1, 8, 12, 900, 992), (1, 4, 30, 5000, 5056)]


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16), (F32, 64), (BF, 16)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("kv,g,t,n,cap", PLACES)
@pytest.mark.parametrize("sparse", [False, True], ids=["all", "blocks"])
def test_all_scores_minus_infinite(dtype, d, kv, g, t, n, cap, sparse):
    """A node all of whose scores are -inf has no weights (0 / 0): no number, as the formula gives; an absent one stays zero; one that sees a finite score is as ever."""
    rng = np.random.default_rng(t + n)
    k, v = rows(rng, 1, cap, kv, d, dtype=dtype), rows(rng, 1, cap, kv, d, dtype=dtype)
    k[..., 0] = -INF
    q = rows(rng, 1, t, kv * g, d, dtype=dtype)
    q[..., 0] = 1.0
    parent = np.full((1, t), -1, np.int32)
    if t > 2:
        parent[0, 1] = -7                          # absent
        k[0, n + 2, :, 0] = 0.5                    # a finite score of its own
    what = dict(block=32, first=1, recent=1, top=1) if sparse else None
    want, off, _ = ref.attention(q, k, v, [n], parent, blocks=what)
    assert bool(torch.isnan(want[0, 0]).all()) and (t <= 2 or (not bool(want[0, 1].any()) and bool(torch.isfinite(want[0, 2]).all())))
    off = torch.where(torch.isfinite(off), off, torch.full_like(off, 2.0 ** -20 * float(v.float().abs().max())))   # (the bound is of infinite scores: one key has all the weight, or none does)
    cache = packed(k, v)
    if sparse:
        got, _ = bpd.bpd_sparse_attention(cache, q.cuda(), ints([n]), binding.new_summaries(cache, 32), parent=torch.from_numpy(parent).cuda(), **what)
    else:
        got = bpd.bpd_tree_attention(cache, q.cuda(), ints([n]), torch.from_numpy(parent).cuda())
    ref.check(got, want, off)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv,g,t,n,cap", PLACES[:1] + PLACES[2:])
def test_infinite_keys_under_fp32_queries(d, kv, g, t, n, cap):
    """Keys with an infinite dimension under queries of fp32: a score of -inf has no weight and leaves the others theirs, one of +inf leaves no number, whatever the queries round to."""
    rng = np.random.default_rng(t + n + d)
    k, v = rows(rng, 1, cap, kv, d), rows(rng, 1, cap, kv, d)
    q = rows(rng, 1, t, kv * g, d, dtype=F32)
    q[..., 0] = 1.0                                # exact in fewer bits
    q[..., 1] = 1.0 + 2.0 ** -20
    bad = [i for i in range(0, n, 7)]
    k[0, bad, :, 0] = -INF
    k[0, [i + 1 for i in bad if i + 1 < n], :, 1] = -INF
    want = ref.attention(q, k, v, [n], None)[0]
    fine = [i for i in range(n + t) if bool(torch.isfinite(k[0, i]).all())]
    seen = len([i for i in fine if i < n])
    kept = torch.tensor(fine)
    less, off, _ = ref.attention(q, k[:, kept], v[:, kept], [seen], None)
    assert torch.allclose(want, less, rtol=1e-12, atol=1e-14)
    off = off * ((n + t) / (seen + 1))             # (as many terms as there are keys)
    out = torch.empty(q.shape, dtype=F32, device="cuda")
    bpd.bpd_tree_attention(packed(k, v), q.cuda(), ints([n]), out=out)
    ref.check(out, less, off)
    k[0, n, 0, 0] = INF                            # the first node's own key: for it and all below it
    got = bpd.bpd_tree_attention(packed(k, v), q.cuda(), ints([n]), out=out).cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(ref.attention(q, k, v, [n], None)[0]))


# ------------------------------------------------------------------------------------------------ captured steps that carry their state

@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 16)], ids=lambda x: str(x).replace("torch.", ""))
def test_replays_summarise_what_the_one_before_has_added(dtype, d):
    """A serving step in a graph: rows stored, chosen blocks with the rows that the replay before has accepted as `added`, the tree verified, lengths moved on.  Each replay against the
    same step called directly on a state of its own, and summaries against those of the keys."""
    rng = np.random.default_rng(14)
    b, kv, g, t, cap, block = 3, 2, 2, 6, 320, 32
    names = ("nk", "nv", "q", "parent", "token", "best", "expect")

    def state(k, v):
        s = dict(cache=tuple(x.clone() for x in packed(k, v)), length=ints([40, 0, 95]), added=ints([1 << 30] * b))
        s.update(nk=torch.zeros((b, t, kv, d), dtype=dtype, device="cuda"), nv=torch.zeros((b, t, kv, d), dtype=dtype, device="cuda"), q=torch.zeros((b, t, kv * g, d), dtype=dtype, device="cuda"))
        s.update({n: torch.zeros((b, t), dtype=torch.int32, device="cuda") for n in ("parent", "token", "best")}, expect=ints([0] * b))
        s["summaries"] = binding.new_summaries(s["cache"], block)
        return s

    def step(s):
        bpd.bpd_cache_store(s["cache"], s["nk"], s["nv"], s["length"])
        out, chosen = bpd.bpd_sparse_attention(s["cache"], s["q"], s["length"], s["summaries"], block=block, first=0, recent=1, top=2, parent=s["parent"], added=s["added"])
        path, accepted, following, after = bpd.bpd_tree_accept(s["parent"], s["token"], s["expect"], s["best"], s["length"], cache=s["cache"])
        s["length"].copy_(after)
        s["added"].copy_(accepted)
        return out, chosen, path, accepted

    k, v = rows(rng, b, cap, kv, d, dtype=dtype), rows(rng, b, cap, kv, d, dtype=dtype)
    warm, one, two = state(k, v), state(k, v), state(k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step(one)
    for turn in range(60):
        parent = np.array([[-1] + [int(rng.integers(max(0, i - 2), i)) for i in range(1, t)] for _ in range(b)], np.int32)
        new = dict(nk=rows(rng, b, t, kv, d, dtype=dtype), nv=rows(rng, b, t, kv, d, dtype=dtype), q=rows(rng, b, t, kv * g, d, dtype=dtype), parent=torch.from_numpy(parent))
        new.update({n: torch.from_numpy(rng.integers(0, 2, tuple(one[n].shape)).astype(np.int32)) for n in ("token", "best", "expect")})
        for s in (one, two):
            for n in names:
                s[n].copy_(new[n])
        before = two["length"].clone()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(res, step(two)):
            assert torch.equal(x, y), turn
        for n in ("length", "added"):
            assert torch.equal(one[n], two[n])
        keys = ref.unpack(*(x.cpu() for x in two["cache"]))[0]
        for s in (one, two):
            kept = ref.summaries_unpacked(s["summaries"].cpu(), cap // block)
            for i, n in enumerate(before.tolist()):
                assert torch.equal(kept[i, :, :n // block], ref.summaries(keys[i:i + 1], block)[0, :, :n // block]), (turn, i)
        if max(two["length"].tolist()) > cap - t:
            break
    assert all(n // block > m // block for n, m in zip(two["length"].tolist(), (40, 0, 95)))       # (blocks have become complete)
