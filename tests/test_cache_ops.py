"""The cache operators' checks of their arguments and their sizes, without a GPU: every call here is refused before anything is enqueued, or has nothing to do."""
import ctypes as C

import pytest
import torch

import cache_reference as ref
from paper_1811_03115_amd import binding

P = 1 << 20          # an aligned address that nothing dereferences
BF, F32 = binding.BPD_BF16, binding.BPD_F32


def cache(**kw):
    return binding.bpd_cache(**dict(dict(k=P, v=P, dtype=BF, n_layers=2, max_batch=4, n_kv_heads=2, head_dim=64, capacity=256), **kw))


def rows(**kw):
    return binding.bpd_rows(**dict(dict(data=P, dtype=BF, layer=0, seq=1024, row=256, head=64), **kw))


def ref_of(x):
    return None if x is None else C.byref(x)


BAD_CACHES = [dict(k=None), dict(v=None), dict(k=P + 8), dict(dtype=2), dict(n_layers=0), dict(max_batch=0), dict(max_batch=65536), dict(n_kv_heads=0), dict(n_kv_heads=1025),
              dict(head_dim=32), dict(head_dim=0), dict(capacity=0), dict(capacity=250), dict(capacity=(1 << 24) + 32), dict(dtype=F32, head_dim=256)]


def attend(c=None, q=None, out=None, length=P, parent=P, b=2, t=3, heads=4, scale=0.1, ws=P, n=1 << 40, blocks=None, null=False):
    L = binding.lib()
    c, q, out = c or cache(), q or rows(), out or rows()
    args = [None if null else C.byref(c), C.byref(q), C.byref(out), length, parent, b, t, heads, scale]
    if blocks is None:
        return L.bpd_tree_attention(*args, ws, n, None)
    return L.bpd_sparse_attention(*args, C.byref(blocks), ws, n, None)


def blocks(**kw):
    return binding.bpd_blocks(**dict(dict(block=32, first=1, recent=1, top=2, summaries=P, added=None, chosen=None), **kw))


@pytest.mark.parametrize("sparse", [False, True])
def test_attention_refusals(sparse):
    b = blocks() if sparse else None
    bad = [dict(null=True), dict(length=None), dict(b=5), dict(b=-1), dict(t=65), dict(t=-1), dict(heads=0), dict(heads=3), dict(heads=130), dict(heads=-2), dict(scale=float("nan")),
           dict(scale=float("inf")), dict(q=rows(data=None)), dict(q=rows(dtype=5)), dict(q=rows(data=P + 1)), dict(out=rows(data=None)), dict(out=rows(dtype=F32, data=P + 2))]
    for kw in bad + [dict(c=cache(**x)) for x in BAD_CACHES]:
        assert attend(blocks=b, **kw) == -1, kw
        assert binding.lib().bpd_op_error()
    for kw in (dict(b=0), dict(t=0), dict(b=0, length=None, ws=None, n=0)):
        assert attend(blocks=b, **kw) == 0, kw
    # the workspace: of a long cache, whose keys are split
    long = cache(capacity=1 << 16)
    need = binding.lib().bpd_attention_workspace_bytes(C.byref(long), 2, 3, 4, 32 if sparse else 0)
    assert need > 0
    for kw in (dict(ws=None), dict(n=need - 1), dict(ws=P + 4)):
        assert attend(blocks=b, c=long, **kw) == -3, kw


def test_sparse_refusals():
    for kw in (dict(block=0), dict(block=48), dict(block=256), dict(block=-32), dict(first=-1), dict(recent=-1), dict(top=-1), dict(summaries=None), dict(summaries=P + 4)):
        assert attend(blocks=blocks(**kw)) == -1, kw
    assert attend(c=cache(capacity=32 * 4097), blocks=blocks()) == -3
    assert binding.lib().bpd_sparse_attention(C.byref(cache()), C.byref(rows()), C.byref(rows()), P, P, 2, 3, 4, 0.1, None, P, 1 << 40, None) == -1


def test_store_refusals():
    L = binding.lib()

    def store(c=None, k=None, v=None, start=P, b=2, t=3):
        return L.bpd_cache_store(C.byref(c or cache()), C.byref(k or rows()), C.byref(v or rows()), start, None, b, t, None)

    for kw in [dict(c=cache(**x)) for x in BAD_CACHES] + [dict(k=rows(data=None)), dict(v=rows(dtype=7)), dict(v=rows(data=P + 1)), dict(start=None), dict(b=5), dict(b=-1), dict(t=-1)]:
        assert store(**kw) == -1, kw
    assert store(t=257) == -3 and store(c=cache(n_layers=40000)) == -3
    assert store(b=0) == 0 and store(t=0) == 0
    assert L.bpd_cache_store(None, C.byref(rows()), C.byref(rows()), P, None, 1, 1, None) == -1
    assert L.bpd_cache_store(C.byref(cache()), None, C.byref(rows()), P, None, 1, 1, None) == -1


def test_accept_refusals():
    L = binding.lib()
    far = [P * (i + 1) for i in range(10)]

    def accept(b=2, t=3, c=None, **kw):
        a = dict(zip(("parent", "token", "expect", "best", "length", "room"), far)) | dict(zip(("path", "accepted", "next", "new_length"), far[6:])) | kw
        return L.bpd_tree_accept(a["parent"], a["token"], a["expect"], a["best"], a["length"], a["room"], 2, b, t, a["path"], a["accepted"], a["next"], a["new_length"], ref_of(c), None)

    for name in ("parent", "token", "expect", "best", "length", "path", "accepted", "next", "new_length"):
        assert accept(**{name: None}) == -1, name
    for kw in (dict(b=-1), dict(b=65536), dict(t=-1), dict(t=65), dict(b=5, c=cache())) + tuple(dict(c=cache(**x)) for x in BAD_CACHES):
        assert accept(**kw) == -1, kw
    # results over what every workgroup reads
    for kw in (dict(new_length=far[4]), dict(next=far[2]), dict(next=far[2] + 4), dict(path=far[1] - 8), dict(accepted=far[5]), dict(path=far[0]), dict(new_length=far[3] + 20)):
        assert accept(**kw) == -1, kw
    assert accept(c=cache(n_layers=65536)) == -3
    assert accept(b=0) == 0


def test_sizes():
    L = binding.lib()
    assert L.bpd_cache_bytes(C.byref(cache(k=None))) == 2 * 4 * 2 * 256 * 64 * 2
    assert L.bpd_cache_bytes(C.byref(cache(dtype=F32, head_dim=16, capacity=37))) == 2 * 4 * 2 * 37 * 16 * 4
    assert L.bpd_summaries_bytes(C.byref(cache()), 32) == 4 * 2 * 1 * 64 * 2 * 64 * 2
    assert L.bpd_summaries_bytes(C.byref(cache(capacity=64)), 128) == 0
    for bad in (dict(capacity=33), dict(head_dim=8), dict(dtype=9)):
        assert L.bpd_cache_bytes(C.byref(cache(**bad))) == 0 and L.bpd_summaries_bytes(C.byref(cache(**bad)), 32) == 0
        assert L.bpd_attention_workspace_bytes(C.byref(cache(**bad)), 1, 1, 2, 0) == 0
    assert L.bpd_summaries_bytes(C.byref(cache()), 40) == 0 and L.bpd_attention_workspace_bytes(C.byref(cache()), 1, 65, 2, 0) == 0


def test_layout():
    """bpd_cache's order of elements, by the formulas of the header, both ways."""
    for d in (64, 128):
        k, v = torch.randn(2, 3, 64, 2, d).bfloat16(), torch.randn(2, 3, 64, 2, d).bfloat16()
        pk, pv = ref.pack(k, v)
        shape = binding.new_cache(3, 2, d, 50, device="cpu", n_layers=2)[0].shape
        assert pk.shape == shape and pv.shape == shape
        uk, uv = ref.unpack(pk, pv)
        assert torch.equal(uk, k) and torch.equal(uv, v)
        # group 1, K [t 1][s 1][q 2][a 3][r 0][e 5]: key 8 * 3 + 4, dimension 32 + 16 + 5
        flat = pk[1, 2, 1, 1].reshape(-1)
        assert flat[(((1 * (d // 32) + 1) * 4 + 2) * 4 + 3) * 32 + 5] == k[1, 2, 32 + 28, 1, 53]
        assert pv[1, 2, 1, 1].reshape(-1)[((2 * 4 + 1) * 16 + 9) * 8 + 6] == v[1, 2, 32 + 14, 1, 41]
    assert binding.new_cache(3, 2, 16, 50, device="cpu")[0].shape == (3, 50, 2, 16)
    assert binding.new_cache(3, 2, 64, 50, dtype=torch.float32, device="cpu", n_layers=4)[1].shape == (4, 3, 50, 2, 64)


def test_wrappers_want_a_gpu():
    c = binding.new_cache(2, 2, 64, 64, device="cpu")
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(binding.BpdError):
        binding.Context.bpd_tree_attention(c, torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), n)
    with pytest.raises(binding.BpdError):
        binding.Context.bpd_cache_store(c, torch.zeros(2, 3, 2, 64), torch.zeros(2, 3, 2, 64), n)


def test_packed_structures():
    """What the wrappers pack as bytes is what the structures hold."""
    for pack, kind, values in ((binding._PACK_CACHE, binding.bpd_cache, (P, 2 * P, 1, 2, 3, 4, 64, 96)), (binding._PACK_ROWS, binding.bpd_rows, (P, 1, 1 << 40, -5, 7, 64)),
                               (binding._PACK_BLOCKS, binding.bpd_blocks, (32, 1, 2, 3, P, 2 * P, 3 * P))):
        got = kind.from_buffer_copy(pack.pack(*values))
        assert pack.size == C.sizeof(kind) and tuple(getattr(got, f[0]) for f in kind._fields_) == values
