"""Steps of a tree of drafts (bpd_step_tree) and decoder self-attention by chosen blocks (bpd_set_sparse_attention), through the C ABI, against
the oracle."""
import math

import numpy as np
import pytest
import torch

import cache_reference as ref
import workloads as wl
from harness import TOL, check_argmax, gpu_context, oracle_model, tol_of
from oracle import greedy_decode, scorers
from oracle.transformer import softmax_rows
from paper_1811_03115_amd import binding

pytestmark = pytest.mark.gpu

F32 = wl.Config("ts-f32", 61, 1, 2, 64, 4, 128, 96, 8, 5, 9, 40, "f32", 2, src_len_kind="lognormal")
F32_LONG = wl.Config("ts-f32-long", 62, 1, 1, 64, 4, 128, 96, 10, 2, 8, 300, "f32", -1, src_kind="uniform0")
BF16 = wl.Config("ts-bf16", 63, 1, 2, 128, 2, 512, 272, 8, 5, 12, 40, "bf16", 2, src_len_kind="lognormal")             # 64-wide heads, kernels of constant K
BF16_ONE = wl.Config("ts-bf16-one", 64, 1, 2, 128, 2, 512, 272, 10, 1, 12, 60, "bf16", 2, src_kind="uniform3")
BF16_ODD = wl.Config("ts-bf16-odd", 65, 1, 2, 192, 3, 288, 272, 7, 3, 12, 40, "bf16", 2, src_kind="uniform3")              # 64-wide heads, other widths: one to two row tiles
BF16_16 = wl.Config("ts-bf16-16", 66, 1, 2, 64, 4, 128, 272, 6, 4, 12, 40, "bf16", 2, src_kind="uniform3")                # 16-wide heads
BF16_16_LEAN = wl.Config("ts-bf16-16-lean", 71, 1, 2, 128, 8, 512, 272, 8, 4, 12, 40, "bf16", 2, src_kind="uniform3")         # 16-wide heads, kernels of constant K
LAYERS = wl.Config("ts-layers", 67, 1, 2, 512, 8, 2048, 512, 8, 2, 12, 40, "bf16", 2, src_kind="uniform3")                # the shape whose chains run as one kernel
ALL = [F32, F32_LONG, BF16, BF16_ONE, BF16_ODD, BF16_16, BF16_16_LEAN, LAYERS]


def trees(k, seed, n=3):
    rng = np.random.default_rng(seed)
    out = [[-1] + [i for i in range(k - 1)], [-1] + [0] * (k - 1)]
    out += [[-1] + [int(rng.integers(max(0, i - 3), i)) for i in range(1, k)] for _ in range(n)]
    return out


def depth(parent, i):
    e = 0
    while i > 0:
        i, e = parent[i], e + 1
    return e


def walk(parent, tok, A, room, eos):
    """Taken nodes of one sequence, as bpd.h says, by the table that the step has left."""
    path = [0]
    while len(path) < room and not (eos >= 0 and tok[path[-1]] == eos):
        nxt = [i for i in range(1, len(parent)) if parent[i] == path[-1] and tok[i] == A[path[-1]][0]]
        if not nxt:
            break
        path.append(nxt[0])
    return path


def next_proposals(parent, path, A):
    out = []
    for i in range(len(parent)):
        e, r = depth(parent, i), sum(parent[q] == parent[i] for q in range(1, i))
        if len(path) - 1 - r < 0 or e + r >= len(parent):
            r = 0
        out.append(int(A[path[len(path) - 1 - r]][e + r]))
    return out


@pytest.mark.parametrize("cfg", ALL, ids=lambda c: c.name)
def test_steps_are_greedy_decoding(cfg):
    """Whatever trees are verified, the tokens are p_1's own choices (exactly greedy decoding's in fp32, within the tolerance of bf16 otherwise), and the bookkeeping is that of the
    definition: nodes taken, lengths, next proposals.  Half of the steps get proposals with the right tokens beside wrong ones, so that rows have to move."""
    weights = wl.make_weights(cfg)
    ctx, model = gpu_context(cfg, weights), oracle_model(cfg, weights)
    src, n = wl.make_sources(cfg)
    rng = np.random.default_rng(cfg.index)
    B, k, budget = cfg.batch, cfg.k, np.minimum(cfg.max_out, rng.integers(cfg.max_out // 2, cfg.max_out + 1, cfg.batch)).astype(np.int32)
    ctx.bpd_encode(src, n, budget)
    fns = [scorers(model, src[b, :n[b]]) for b in range(B)]
    ctx.bpd_step(k)                                 # (from an ordinary step on)
    taken, moved, done = [ctx.bpd_get_output()[0][b, :ctx.bpd_get_output()[1][b]].tolist() for b in range(B)], 0, False
    for step in range(60):
        P, _, j, fin = ctx.bpd_get_state()
        if fin.all():
            done = True
            break
        parent = trees(k, step + 100 * cfg.index)[step % 5]
        if step % 2 == 0:                           # the right continuation along one branch, something else in all other nodes
            P = P.copy()
            for b in range(B):
                if fin[b]:
                    continue
                line, tip = [0], 0
                while True:
                    kids = [i for i in range(1, k) if parent[i] == tip]
                    if not kids:
                        break
                    tip = int(rng.choice(kids[-2:]))
                    line.append(tip)
                prefix = taken[b] + [int(P[b, 0])]
                P[b, 1:k] = rng.integers(3, cfg.vocab, k - 1)
                for i in line[1:1 + int(rng.integers(1, 5))]:
                    P[b, i] = int(fns[b][0](prefix)[0].argmax())
                    prefix.append(int(P[b, i]))
            ctx.bpd_set_proposals(P)
        acc = torch.full((B,), -1, dtype=torch.int32, device="cuda")
        ctx.bpd_step_tree(k, parent, acc)
        P2, A, j2, fin2 = ctx.bpd_get_state()
        ids, lens = ctx.bpd_get_output()
        for b in range(B):
            if fin[b]:
                assert int(acc[b]) == 0 and fin2[b]
                continue
            path = walk(parent, P[b].tolist(), A[b].tolist(), int(budget[b]) - int(j[b]), cfg.eos_id)
            new = [int(P[b, i]) for i in path]
            assert int(acc[b]) == len(path) and j2[b] == j[b] + len(path) == lens[b], (step, b)
            assert ids[b, j[b]:j2[b]].tolist() == new
            assert P2[b, :k].tolist() == next_proposals(parent, path, A[b].tolist())
            assert bool(fin2[b]) == (j2[b] >= budget[b] or (cfg.eos_id >= 0 and new[-1] == cfg.eos_id))
            moved += path[-1] != len(path) - 1
            taken[b] += new
        if step % 7 == 6:
            ctx.bpd_step(k)                         # an ordinary step in between
            ids, lens = ctx.bpd_get_output()
            taken = [ids[b, :lens[b]].tolist() for b in range(B)]
    assert moved >= min(4, 2 * B)                   # (rows did move)
    if not done:
        ids, lens, _ = ctx.bpd_decode(k)            # ... and the rest
        taken = [ids[b, :lens[b]].tolist() for b in range(B)]
    for b in range(B):
        if cfg.dtype == "f32":
            assert taken[b] == greedy_decode(fns[b][0], int(budget[b]), cfg.eos_id).tokens
        else:
            z = model.all_position_logits(model.encode(src[b, :n[b]]), taken[b][:-1], k=1)[:, 0]
            check_argmax(np.array(taken[b]), z, tol_of(cfg), f"tokens of {b}")
    st = ctx.bpd_get_stats()
    assert st.accepted_total == sum(len(t) for t in taken) and st.finished == B


@pytest.mark.parametrize("cfg", [F32, BF16, BF16_ONE], ids=lambda c: c.name)
def test_scores_of_a_tree(cfg):
    """The table of a tree step: every entry is an arg-max of the oracle's scores behind the node's ancestors."""
    weights = wl.make_weights(cfg)
    ctx, model = gpu_context(cfg, weights), oracle_model(cfg, weights)
    src, n = wl.make_sources(cfg)
    rng = np.random.default_rng(7)
    B, k = cfg.batch, cfg.k
    ctx.bpd_encode(src, n)
    for _ in range(2):
        ctx.bpd_step(k)
    prefix = [ctx.bpd_get_output()[0][b, :ctx.bpd_get_output()[1][b]].tolist() for b in range(B)]
    P, _, j, fin = ctx.bpd_get_state()
    for parent in trees(k, 3)[1:]:
        P[:, 1:k] = rng.integers(3, cfg.vocab, (B, k - 1))
        ctx.bpd_set_proposals(P)
        ctx.bpd_step_tree(k, parent)
        P2, A, j2, fin2 = ctx.bpd_get_state()
        for b in range(B):
            if fin[b]:
                continue
            for i in range(k):
                line, q = [], i
                while q > 0:
                    line, q = [q] + line, parent[q]
                z = model.next_logits(model.encode(src[b, :n[b]]), prefix[b] + [int(P[b, x]) for x in [0] + line], k)
                check_argmax(A[b, i, :k], z, tol_of(cfg), f"node {i} of {b}")
            prefix[b] += [int(t) for t in ctx.bpd_get_output()[0][b, j[b]:j2[b]]]
        P, j, fin = P2.copy(), j2, fin2


def test_chain_is_an_ordinary_step():
    cfg = F32
    weights = wl.make_weights(cfg)
    a, b = gpu_context(cfg, weights), gpu_context(cfg, weights)
    src, n = wl.make_sources(cfg)
    for c in (a, b):
        c.bpd_encode(src, n)
    for k in (8, 8, 5, 1, 8):
        a.bpd_step(k)
        b.bpd_step_tree(k, [-1] + list(range(k - 1)))
        for x, y in zip(a.bpd_get_state() + a.bpd_get_output(), b.bpd_get_state() + b.bpd_get_output()):
            np.testing.assert_array_equal(x, y)
    assert bytes(a.bpd_get_stats()) == bytes(b.bpd_get_stats())


@pytest.mark.parametrize("cfg", [BF16, F32], ids=lambda c: c.name)
def test_captured_tree_steps(cfg):
    """A step of a tree in a graph, replayed with direct calls in between, against direct calls alone."""
    weights = wl.make_weights(cfg)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctxs = [binding.Context(binding.config_from_workload(cfg), stream=side) for _ in range(2)]
        for c in ctxs:
            c.bpd_load_weights(weights)
    src, n = wl.make_sources(cfg)
    parent = trees(cfg.k, 5)[3]
    for c in ctxs:
        c.bpd_encode(src, n)
        c.bpd_step(cfg.k)
        c.bpd_step_tree(cfg.k, parent)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctxs[0].bpd_step_tree(cfg.k, parent)
    for step in range(5):
        with torch.cuda.stream(side):
            graph.replay()
        ctxs[1].bpd_step_tree(cfg.k, parent)
        if step == 2:
            for c in ctxs:
                c.bpd_step(cfg.k)
        side.synchronize()
        for x, y in zip(ctxs[0].bpd_get_state() + ctxs[0].bpd_get_output(), ctxs[1].bpd_get_state() + ctxs[1].bpd_get_output()):
            np.testing.assert_array_equal(x, y, err_msg=f"step {step}")


def test_tree_step_refusals():
    cfg = F32
    ctx = gpu_context(cfg, wl.make_weights(cfg))
    with pytest.raises(binding.BpdError) as e:
        ctx.bpd_step_tree(2, [-1, 0])
    assert e.value.code == -2
    ctx.bpd_encode(*wl.make_sources(cfg))
    before = [np.array(x) for x in ctx.bpd_get_state()]
    for k, parent in ((3, [-1, 0, 2]), (3, [-1, 0, -1]), (3, [0, 0, 1]), (2, [-1, 1]), (3, [-1, 0]), (9, [-1] + [0] * 8), (0, [])):
        with pytest.raises(binding.BpdError) as e:
            ctx.bpd_step_tree(k, parent)
        assert e.value.code == -1
    for on, off in ((lambda: ctx.bpd_set_acceptance(1, 1), lambda: ctx.bpd_set_acceptance(0, 1)), (lambda: ctx.bpd_set_top_n(2), lambda: ctx.bpd_set_top_n(1)),
                    (lambda: ctx.bpd_set_acceptance(0, 2), lambda: ctx.bpd_set_acceptance(0, 1)), (lambda: ctx.bpd_set_local_attention(8, 8), lambda: ctx.bpd_set_local_attention(0, 0))):
        on()
        with pytest.raises(binding.BpdError) as e:
            ctx.bpd_step_tree(2, [-1, 0])
        assert e.value.code == -1
        off()
    for x, y in zip(before, ctx.bpd_get_state()):
        np.testing.assert_array_equal(x, y)


# ------------------------------------------------------------------------------------------------ chosen blocks

def sparse_logits(model, memory, committed, block_tokens, what):
    """Scores of the block rows of a model of one decoder layer, whose rows see the first len(committed) + 1 positions by chosen blocks (in 64 bits).  One layer: what the
    earlier rows saw in their own steps does not reach their keys and values."""
    w, dh = model.w, model.d // model.n_heads
    y = np.array(list(committed) + list(block_tokens))
    t1, L = len(y) + 1, len(committed) + 1
    u = np.zeros((t1, model.d))
    u[1:] = math.sqrt(model.d) * w["emb"][y]
    x = u + w["pos_tgt"][:t1]
    a = model._ln(x, "dec.0.ln1")
    q, k, v = ((a @ w[f"dec.0.self.{m}"]).reshape(t1, model.n_heads, dh) for m in ("wq", "wk", "wv"))
    out = np.zeros((t1, model.n_heads, dh))
    for s in range(L, t1):
        for h in range(model.n_heads):
            vis = np.zeros((1, t1), bool)
            for j in ref.choose(torch.from_numpy(q[s, h][None]), torch.from_numpy(k[:, h]), L, **what):
                vis[0, j * what["block"]:(j + 1) * what["block"]] = True
            vis[0, L // what["block"] * what["block"]:s + 1] = True
            out[s, h] = softmax_rows((q[s, h] @ k[:, h].T / math.sqrt(dh))[None], vis)[0] @ v[:, h]
    x = (x + out.reshape(t1, -1) @ w["dec.0.self.wo"])[L:]
    x = x + model._attn(model._ln(x, "dec.0.ln2"), memory, "dec.0.cross", np.ones((t1 - L, memory.shape[0]), bool))
    x = x + model._ffn(model._ln(x, "dec.0.ln3"), "dec.0.ffn")
    return model.logits(model._ln(x, "dec.lnf"), model.k)


def forced(ctx, cfg, rng, steps):
    """Steps that take whole blocks of random tokens; returns what has been committed, and the block that follows."""
    taken = [[] for _ in range(cfg.batch)]
    P = rng.integers(3, cfg.vocab, (cfg.batch, cfg.k)).astype(np.int32)
    ctx.bpd_set_proposals(P)
    whole = np.full(cfg.batch, cfg.k, np.int32)
    for _ in range(steps):
        ctx.bpd_step(cfg.k, whole)
        for b in range(cfg.batch):
            taken[b] += P[b].tolist()
        P = rng.integers(3, cfg.vocab, (cfg.batch, cfg.k)).astype(np.int32)
        ctx.bpd_set_proposals(P)
    return taken, P


@pytest.mark.parametrize("what", [dict(block=32, first=1, recent=1, top=2), dict(block=32, first=0, recent=0, top=1), dict(block=64, first=0, recent=1, top=1)], ids=str)
def test_sparse_scores(what):
    """Scores by few blocks against the oracle's, the setting switched on from the start, late, and off again."""
    cfg = F32_LONG
    weights = wl.make_weights(cfg)
    model = oracle_model(cfg, weights)
    src, n = wl.make_sources(cfg)
    for late in (False, True):
        ctx = gpu_context(cfg, weights)
        rng = np.random.default_rng(11)
        ctx.bpd_encode(src, n)
        if not late:
            ctx.bpd_set_sparse_attention(**what)
        taken, P = forced(ctx, cfg, rng, 23)
        if late:
            ctx.bpd_set_sparse_attention(**what)
        got = ctx.bpd_debug_step_logits(cfg.k).cpu().numpy()
        for b in range(cfg.batch):
            want = sparse_logits(model, model.encode(src[b, :n[b]]), taken[b], P[b], what)
            assert np.abs(got[b] - want).max() <= TOL["f32"], (late, b)
        ctx.bpd_set_sparse_attention(0)
        got = ctx.bpd_debug_step_logits(cfg.k).cpu().numpy()
        for b in range(cfg.batch):
            want = model.all_position_logits(model.encode(src[b, :n[b]]), taken[b] + P[b].tolist(), first=len(taken[b]) + 1)
            assert np.abs(got[b] - want).max() <= TOL["f32"], (late, b)


BF16_LONG = wl.Config("ts-bf16-long", 68, 1, 2, 128, 2, 512, 272, 8, 3, 12, 400, "bf16", -1, src_kind="uniform3")
BF16_16_LONG = wl.Config("ts-bf16-16-long", 69, 1, 2, 64, 4, 128, 272, 8, 3, 12, 400, "bf16", -1, src_kind="uniform3")


@pytest.mark.parametrize("cfg", [BF16_LONG, BF16_16_LONG, F32_LONG], ids=lambda c: c.name)
def test_all_blocks_is_full_attention(cfg):
    """With as many blocks as there are nothing is left out: scores within the tolerance of the oracle's full attention at every depth, also those of trees and ragged batches."""
    weights = wl.make_weights(cfg)
    model = oracle_model(cfg, weights)
    src, n = wl.make_sources(cfg)
    ctx = gpu_context(cfg, weights)
    ctx.bpd_set_sparse_attention(32, 1, 1, 100)
    ctx.bpd_encode(src, n)
    rng = np.random.default_rng(3)
    taken = [[] for _ in range(cfg.batch)]
    P = ctx.bpd_get_state()[0]
    for step in range(30):
        if step in (5, 18, 29):
            got = ctx.bpd_debug_step_logits(cfg.k).cpu().numpy()
            for b in range(cfg.batch):
                want = model.all_position_logits(model.encode(src[b, :n[b]]), taken[b] + P[b, :cfg.k].tolist(), first=len(taken[b]) + 1)
                assert np.abs(got[b] - want).max() <= tol_of(cfg), (step, b)
        acc = rng.integers(1, cfg.k + 1, cfg.batch).astype(np.int32)
        ctx.bpd_step(cfg.k, acc)
        for b in range(cfg.batch):
            taken[b] += P[b, :acc[b]].tolist()
        P = rng.integers(3, cfg.vocab, (cfg.batch, cfg.k)).astype(np.int32)
        ctx.bpd_set_proposals(P)


def test_sparse_decode_with_ended_sequences():
    """A batch whose sequences end one after the other, by chosen blocks: as many tokens as the budgets, each p_1's choice (all blocks chosen), tree steps in between."""
    cfg = wl.scaled(BF16_LONG, eos_id=2, batch=6, index=70)
    weights = wl.make_weights(cfg)
    model = oracle_model(cfg, weights)
    src, n = wl.make_sources(cfg)
    budget = np.array([9, 120, 40, 77, 1, 100], np.int32)
    ctx = gpu_context(cfg, weights)
    ctx.bpd_set_sparse_attention(32, 0, 2, 9)
    ctx.bpd_encode(src, n, budget)
    for step in range(4):
        ctx.bpd_step_tree(cfg.k, trees(cfg.k, step)[2])
    ids, lens, st = ctx.bpd_decode(cfg.k)
    for b in range(cfg.batch):
        got = ids[b, :lens[b]]
        assert lens[b] == budget[b] or (got[-1] == cfg.eos_id and lens[b] < budget[b])
        assert not (got[:-1] == cfg.eos_id).any()
        z = model.all_position_logits(model.encode(src[b, :n[b]]), got[:-1].tolist(), k=1)[:, 0]
        check_argmax(got, z, tol_of(cfg), f"tokens of {b}")
    assert st.finished == cfg.batch


@pytest.mark.parametrize("cfg", [BF16, BF16_ODD, F32_LONG], ids=lambda c: c.name)
def test_encodes_recorded_under_the_setting(cfg):
    """Encodes that come again are recorded: under the setting they are those without it, and outlive its buffer."""
    weights = wl.make_weights(cfg)
    src, n = wl.make_sources(cfg)
    plain, ctx = gpu_context(cfg, weights), gpu_context(cfg, weights)
    plain.bpd_encode(src, n)
    want = [np.array(x) for x in plain.bpd_get_state()]
    ctx.bpd_set_sparse_attention(32, 1, 1, 4)
    for _ in range(10):
        ctx.bpd_encode(src, n)
    ctx.bpd_step(cfg.k)
    ctx.bpd_set_sparse_attention(0)
    torch.cuda.synchronize()
    junk = torch.full((1 << 22,), float("nan"), device="cuda")
    for _ in range(2):
        ctx.bpd_encode(src, n)
        for x, y in zip(want, ctx.bpd_get_state()):
            np.testing.assert_array_equal(x, y)
    assert bool(torch.isnan(junk).all())


def test_captured_sparse_steps():
    """Steps by chosen blocks in a graph, replayed, with direct steps in between, against direct calls alone."""
    cfg = F32_LONG
    weights = wl.make_weights(cfg)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctxs = [binding.Context(binding.config_from_workload(cfg), stream=side) for _ in range(2)]
    src, n = wl.make_sources(cfg)
    whole = torch.full((cfg.batch,), cfg.k, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for c in ctxs:
        c.bpd_load_weights(weights)
        c.bpd_set_sparse_attention(32, 1, 1, 1)
        c.bpd_encode(src, n)
        c.bpd_step(cfg.k, whole)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctxs[0].bpd_step(cfg.k, whole)
    for step in range(25):
        with torch.cuda.stream(side):
            graph.replay()
        ctxs[1].bpd_step(cfg.k, whole)
        if step % 6 == 5:
            for c in ctxs:
                c.bpd_step(cfg.k, whole)
        side.synchronize()
        for x, y in zip(ctxs[0].bpd_get_state(), ctxs[1].bpd_get_state()):
            np.testing.assert_array_equal(x, y, err_msg=f"step {step}")


def test_sparse_refusals():
    cfg = F32
    ctx = gpu_context(cfg, wl.make_weights(cfg))
    L, h = binding.lib(), ctx.h
    need = ctx.bpd_sparse_buffer_bytes(32)
    buf = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    at = (buf.data_ptr() + 255) // 256 * 256
    assert need > 0 and ctx.bpd_sparse_buffer_bytes(48) == 0
    for args, code in (((48, 1, 1, 1, at, need), -1), ((32, -1, 1, 1, at, need), -1), ((32, 1, -1, 1, at, need), -1), ((32, 1, 1, -1, at, need), -1), ((-32, 1, 1, 1, at, need), -1),
                       ((32, 1, 1, 1, None, need), -3), ((32, 1, 1, 1, at + 128, need), -3), ((32, 1, 1, 1, at, need - 1), -3)):
        assert L.bpd_set_sparse_attention(h, *args) == code, args
    assert L.bpd_set_sparse_attention(None, 32, 1, 1, 1, at, need) == -1
    ctx.bpd_set_local_attention(8, 8)
    with pytest.raises(binding.BpdError):
        ctx.bpd_set_sparse_attention(32)
    ctx.bpd_set_local_attention(0, 0)
    ctx.bpd_set_sparse_attention(32)
    with pytest.raises(binding.BpdError):
        ctx.bpd_set_local_attention(8, 8)
    ctx.bpd_set_sparse_attention(0)
    ctx.bpd_set_local_attention(8, 8)
