"""Drafted tokens, host side, no GPU: refusals of the entry points (device pointers are opaque, nothing is launched), sizes,
and the oracle's trees by hand."""
import ctypes as C

import numpy as np
import pytest

from oracle import tree
from paper_2510_18546_amd import binding as B

P = 0x10000      # an address that nobody looks at


def handles(dtype=B.EN_BF16, n_new=20, lens=(30, 5), d=64, hkv=2, hq=4, cap=40):
    pool = B.kv_pool_create(None, None, list(lens), hq, 1e4, 4096, dtype=dtype, shape=(len(lens), hkv, cap, d), k_ptr=0x1000,
                            v_ptr=0x2000)
    return pool, B.segment_select(pool, list(range(len(lens))), list(range(len(lens) + 1)), n_new)


def code(rc):
    return B.STATUS[rc].replace("EN_ERR_", "")


def attention(pool, plan, n=4, done=P, parent=P, q=P, k=P, v=P, kc=P, vt=P, out=P, ws=P, ws_bytes=1 << 40):
    h = lambda x: x.handle if x is not None else None
    return code(B.load().segmented_tree_attention(h(pool), h(plan), n, done, parent, q, k, v, kc, vt, out, ws, ws_bytes, None))


def test_attention_refusals():
    pool, plan = handles()
    other, _ = handles()
    assert attention(None, plan) == attention(pool, None) == attention(other, plan) == "INVALID_ARG"
    for name in ("done", "parent", "q", "k", "v", "kc", "vt", "out"):
        assert attention(pool, plan, **{name: None}) == "INVALID_ARG", name
    for name in ("q", "k", "v", "kc", "vt", "out", "ws"):
        assert attention(pool, plan, **{name: P + 8}) == "INVALID_ARG", name
    for name in ("done", "parent"):
        assert attention(pool, plan, **{name: P + 2}) == "INVALID_ARG", name
    assert attention(pool, plan, n=0) == attention(pool, plan, n=-5) == "INVALID_ARG"
    assert attention(pool, plan, n=B.TREE_MAX_NODES + 1) == "UNSUPPORTED"
    need = B.tree_workspace_bytes(pool, plan, 4)
    if need:
        assert attention(pool, plan, ws=None) == "INVALID_ARG"
        assert attention(pool, plan, ws_bytes=need - 1) == "CAPACITY"
    big, its = handles(lens=(3_000,), d=128, cap=4000, n_new=60)
    its.values_from_pool(True)
    assert attention(big, its) == "UNSUPPORTED"


def test_attention_refuses_contexts_that_offsets_cannot_reach():
    pool = B.kv_pool_create(None, None, [0], 1, 1e4, 1 << 30, dtype=B.EN_BF16, shape=(1, 1, 4, 128), k_ptr=0x1000, v_ptr=0x2000)
    plan = B.segment_select(pool, [0], [0, 1], 1 << 24)
    assert attention(pool, plan) == "UNSUPPORTED"


def test_workspace_sizes():
    pool, plan = handles()
    assert B.tree_workspace_bytes(pool, plan, 0) == B.tree_workspace_bytes(pool, plan, 65) == 0
    assert B.tree_accept_workspace_bytes(plan, 0, 10) == B.tree_accept_workspace_bytes(plan, 65, 10) == 0
    assert B.tree_accept_workspace_bytes(plan, 3, 0) == 0 and B.tree_accept_workspace_bytes(plan, 3, 1) > 0


def commit(pool, plan, n=4, layers=2, done=P, count=P, path=P, change=None):
    arrays = [[P] * max(0, layers) for _ in range(4)]
    if change:
        arrays[change[0]][change[1]] = change[2]
    ptrs = [(C.c_void_p * len(x))(*x) for x in arrays]
    return code(B.load().segmented_tree_commit(pool.handle if pool else None, plan.handle if plan else None, n, layers, done, count, path,
                                               *ptrs, None))


def test_commit_refusals():
    pool, plan = handles()
    other, _ = handles()
    assert commit(None, plan) == commit(pool, None) == commit(other, plan) == "INVALID_ARG"
    for name in ("done", "count", "path"):
        assert commit(pool, plan, **{name: None}) == commit(pool, plan, **{name: P + 1}) == "INVALID_ARG"
    assert commit(pool, plan, n=0) == commit(pool, plan, layers=-1) == "INVALID_ARG"
    assert commit(pool, plan, n=65) == "UNSUPPORTED"
    for which in range(4):
        assert commit(pool, plan, change=(which, 1, None)) == commit(pool, plan, change=(which, 0, P + 8)) == "INVALID_ARG"
    assert code(B.load().segmented_tree_commit(pool.handle, plan.handle, 4, 1, P, P, P, None, None, None, None, None)) == "INVALID_ARG"
    big, its = handles(lens=(3_000,), d=128, cap=4000, n_new=60)
    its.values_from_pool(True)
    assert commit(big, its) == "UNSUPPORTED"


def rules(**kw):
    r = B._TokenRules()
    for name, x in kw.items():
        setattr(r, name, x)
    return r


def apply(r=None, agents=2, n=3, vocab=100, dtype=B.EN_BF16, parent=P, tokens=P, x=P, stride=100, out=P + 4096, out_stride=100):
    return code(B.load().token_rules_apply(None if r is None else C.addressof(r), agents, n, vocab, dtype, parent, tokens, x, stride, out,
                                           out_stride, None))


def bad_rules():
    yield rules(reserved=1)
    yield rules(history_stride=-1)
    yield rules(history_dev=P, history_stride=5)
    yield rules(bias_dev=P, bias_agent_stride=99)
    yield rules(bias_dev=P + 2)
    yield rules(mask_dev=P, mask_agent_stride=3)
    yield rules(mask_dev=P, mask_node_stride=-4)
    yield rules(mask_dev=P + 1)
    yield rules(penalties_dev=P + 3)
    yield rules(history_dev=P, history_len_dev=P + 2)


def test_rules_refusals():
    fine = rules()
    assert apply(None) == apply(fine, x=None) == apply(fine, out=None) == apply(fine, agents=0) == "INVALID_ARG"
    assert apply(fine, parent=None) == apply(fine, tokens=None) == "INVALID_ARG"
    assert apply(fine, parent=P + 1) == apply(fine, tokens=P + 2) == "INVALID_ARG"
    assert apply(fine, n=0) == apply(fine, vocab=0) == apply(fine, stride=99) == apply(fine, out_stride=99) == "INVALID_ARG"
    assert apply(fine, x=P + 1) == apply(fine, out=P + 1) == apply(fine, x=P + 2, dtype=B.EN_F32) == "INVALID_ARG"
    assert apply(fine, n=65) == apply(fine, dtype=B.EN_I8) == apply(fine, dtype=7) == "UNSUPPORTED"
    assert apply(fine, out=P, out_stride=200) == "INVALID_ARG"
    for r in bad_rules():
        assert apply(r) == "INVALID_ARG"


def accept(plan, r=None, n=3, vocab=100, dtype=B.EN_BF16, done=P, parent=P, tokens=P, x=P, stride=100, choice=P, path=P, count=P, token=P,
           done_out=P, ws=P, ws_bytes=1 << 30):
    return code(B.load().token_tree_accept(plan.handle if plan else None, None if r is None else C.addressof(r), n, vocab, dtype, done, parent,
                                           tokens, x, stride, choice, path, count, token, done_out, ws, ws_bytes, None))


def test_accept_refusals():
    _, plan = handles()
    assert accept(None) == "INVALID_ARG"
    for name in ("done", "parent", "tokens", "path", "count", "token", "done_out"):
        assert accept(plan, **{name: None}) == accept(plan, **{name: P + 2}) == "INVALID_ARG", name
    assert accept(plan, choice=P + 1) == accept(plan, x=None, choice=None) == "INVALID_ARG"
    assert accept(plan, n=0) == accept(plan, vocab=0) == accept(plan, stride=99) == accept(plan, x=P + 1) == "INVALID_ARG"
    assert accept(plan, n=65) == accept(plan, dtype=B.EN_I8) == "UNSUPPORTED"
    assert accept(plan, ws=None) == accept(plan, ws=P + 4) == "INVALID_ARG"
    assert accept(plan, ws_bytes=B.tree_accept_workspace_bytes(plan, 3, 100) - 1) == "CAPACITY"
    for r in bad_rules():
        assert accept(plan, r) == "INVALID_ARG"


def test_more_agents_or_tokens_than_a_launch_counts():
    fine, most = rules(), 65535 * 4096
    assert apply(fine, agents=65536) == "UNSUPPORTED"
    assert apply(fine, vocab=most + 1, stride=most + 1, out_stride=most + 1) == "UNSUPPORTED"
    pool, _ = handles(lens=(1,), cap=1, n_new=1)
    plan = B.segment_select(pool, [0] * 65536, list(range(65537)), 1)
    assert accept(plan) == accept(plan, x=None) == commit(pool, plan) == "UNSUPPORTED"
    _, plan = handles()
    assert accept(plan, vocab=most + 1, stride=most + 1, ws_bytes=1 << 50) == "UNSUPPORTED"


def test_calls_after_the_pool_is_gone():
    pool, plan = handles()
    lib = B.load()
    lib.kv_pool_destroy(pool.handle)
    pool.handle = None
    assert accept(plan) == "INVALID_ARG"


def test_binding_refusals():
    import torch
    x = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError):
        B.token_rules_apply(B.token_rules(), x, x)                       # not on a GPU
    with pytest.raises(ValueError):
        B.token_rules_apply(B.token_rules(), x.half(), x.half())
    for kw in (dict(penalties=torch.zeros(2, 2)), dict(penalties=torch.zeros(2, 3, dtype=torch.float64)), dict(bias=torch.zeros(2, 2, 2)),
               dict(history=torch.zeros(2, 5, dtype=torch.int32)), dict(history=torch.zeros(2, 5), history_len=torch.zeros(2)),
               dict(mask=torch.zeros(2, 5, dtype=torch.int32)), dict(penalties=torch.zeros(3, 2).t())):
        with pytest.raises(ValueError):
            B.token_rules(**kw)


def layered(monkeypatch):
    """Calls of the binding up to the library, whose part takes everything: (pool, plan, the right arguments)."""
    import types

    import torch
    pool, plan = handles(lens=(30, 5), d=64, hkv=2, hq=4)
    ctx = plan.context_bytes
    taken = types.SimpleNamespace(segmented_tree_commit=lambda *a: 0, segmented_tree_attention=lambda *a: 0)
    monkeypatch.setattr(B, "load", lambda path=None: taken)
    monkeypatch.setattr(B, "_device", lambda: -1)            # (a CPU tensor's)
    some = dict(dtype=torch.bfloat16)
    return pool, plan, ctx, dict(rows=[torch.zeros(2, 3, 2, 64, **some) for _ in range(3)],
                                 contexts=[torch.zeros(ctx // 2, **some) for _ in range(3)], ints=torch.zeros(2, dtype=torch.int32),
                                 tree=torch.zeros(2, 3, dtype=torch.int32), q=torch.zeros(2, 3, 4, 64, **some))


def unfit_rows(x):
    """The same bytes as rows [B, n, Hkv, D], or as many, that are none."""
    import torch
    b, n, h, d = x.shape
    return [x.transpose(1, 2).contiguous(), x.view(b, n, h * d), x.view(b * n, h, d), x.to(torch.float16), x.view(torch.int16),
            torch.zeros(b, n, h, 2 * d, dtype=x.dtype)[..., :d], x[:, :2].contiguous()]


def unfit_contexts(x):
    import torch
    return [x.float(), x.to(torch.float16), x.double(), x.to(torch.complex64), x[:-1], torch.zeros(x.numel(), 2, dtype=x.dtype)[:, 0]]


def test_binding_commit_looks_at_shape_and_type_of_every_layer(monkeypatch):
    pool, plan, _, a = layered(monkeypatch)

    def commit(**other):
        x = {"k": list(a["rows"]), "v": list(a["rows"]), "kc": list(a["contexts"]), "vt": list(a["contexts"])}
        for name, tensor in other.items():
            x[name][1] = tensor
        B.segmented_tree_commit(pool, plan, a["ints"], a["ints"], a["tree"], x["k"], x["v"], x["kc"], x["vt"], stream=0)

    commit()
    commit(kc=a["contexts"][0].view(B._torch().uint8), vt=a["contexts"][0].view(B._torch().int16))
    for bad in unfit_rows(a["rows"][0]):
        for name in ("k", "v"):
            with pytest.raises(ValueError):
                commit(**{name: bad})
    for bad in unfit_contexts(a["contexts"][0]):
        for name in ("kc", "vt"):
            with pytest.raises(ValueError):
                commit(**{name: bad})


def test_binding_attention_looks_at_shape_and_type(monkeypatch):
    pool, plan, _, a = layered(monkeypatch)

    def attend(**other):
        x = {"k": a["rows"][0], "v": a["rows"][1], "kc": a["contexts"][0], "vt": a["contexts"][1], **other}
        B.segmented_tree_attention(pool, plan, a["ints"], a["tree"], a["q"], x["k"], x["v"], x["kc"], x["vt"], a["q"].clone(), stream=0)

    attend()
    attend(kc=a["contexts"][0].view(B._torch().uint8), vt=a["contexts"][0].view(B._torch().int16))
    for name in ("k", "v"):
        for bad in unfit_rows(a["rows"][0]):
            with pytest.raises(ValueError):
                attend(**{name: bad})
    for name in ("kc", "vt"):
        for bad in unfit_contexts(a["contexts"][0]):
            with pytest.raises(ValueError):
                attend(**{name: bad})


def test_oracle_trees_by_hand():
    assert tree.ways([-1, 0, 0, 1, -1, 4]) == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5]]
    assert tree.ways([-1, -2, 1, 3, 5, 0]) == [[0], [], [], [], [], [0, 5]]
    assert tree.ways([-1, 0, 1, 2], room=2) == [[0], [0, 1], [], []]
    assert [tree.room_of(d, 5) for d in (-1, 0, 4, 5, 6)] == [0, 5, 1, 0, 0]
    assert tree.accept([[3, 9, 8, 1]], [0], 10, [[-1, 0, 0, 2]], [[0, 4, 3, 8]]) == [([0, 2, 3], 1)]
    assert tree.accept([[3, 9]], [0], 10, [[-2, 0]], [[0, 3]]) == [([], -1)]
    assert tree.choose(np.array([1.0, np.nan, 3.0, 3.0])) == 2 and tree.choose(np.array([-np.inf, np.nan])) == -1
