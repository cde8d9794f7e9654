"""Attention over trees of drafted tokens (segmented_tree_attention) against the float64 oracle, which goes along each
node's way by itself. Tolerances: tree_cases.near."""
import numpy as np
import pytest

from tree_cases import BASE, TREES, Tree, bf16, chain, column, comb, near

pytestmark = pytest.mark.gpu


def check(t, layer=0):
    import torch
    got = t.attend(layer)
    torch.cuda.synchronize()
    near(got.float().cpu().numpy(), t.expected(layer), t.f32)


def forest(agents, n, kinds=("comb", "chain", "broken", "star")):
    return [TREES[kinds[b % len(kinds)]](n) for b in range(agents)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16, 31, 33, 64])
def test_nodes(dtype, d, n):
    check(Tree(n, dtype, [200, 77, 0, 129], [3, 0, 1, 5], 80, forest(4, n), r=2, kv=2, d=d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,kv,n,d", [(1, 1, 1, 64), (1, 3, 5, 128), (3, 2, 11, 64), (4, 8, 8, 128), (7, 1, 13, 128), (8, 2, 64, 64),
                                      (7, 2, 64, 128), (16, 1, 4, 128), (32, 1, 1, 128), (5, 1, 40, 64), (20, 1, 64, 128)])
def test_heads(dtype, r, kv, n, d):
    check(Tree(r + n, dtype, [300, 65], [2, 7], 90, forest(2, n), r=r, kv=kv, d=d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 193, 255, 256, 257, 320, 511, 513, 1000, 2047])
def test_lengths(dtype, length):
    check(Tree(length, dtype, [length, max(0, length - 40)], [0, 17], 40, forest(2, 6), r=4, kv=1, d=128 if length % 2 else 64))


@pytest.mark.parametrize("dtype,r,kv,n,d,lens", [("bf16", 4, 2, 8, 128, [9000]), ("bf16", 7, 1, 64, 128, [5000, 100]),
                                                 ("bf16", 2, 1, 3, 64, [20000, 12000, 1]), ("f32", 2, 1, 9, 64, [6000, 33]),
                                                 ("f32", 1, 1, 2, 128, [4000]), ("bf16", 1, 4, 64, 64, [3500, 3000])])
def test_long_contexts(dtype, r, kv, n, d, lens):
    check(Tree(n, dtype, lens, [5 * b for b in range(len(lens))], 100, forest(len(lens), n), r=r, kv=kv, d=d))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("agents", [33, 150])
def test_many_agents(dtype, agents):
    rng = np.random.default_rng(agents)
    check(Tree(agents, dtype, rng.integers(0, 400, agents), rng.integers(0, 9, agents), 20, forest(agents, 5), r=2, kv=2, d=64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_absent_nodes_idle_agents_and_the_reserve(dtype):
    """Rows without a node are zero, whatever their inputs hold; nodes that the reserve has no room for are absent."""
    n = 12
    done = [-1, 31, 2**31 - 1, -2**31, 30, 25, 0, 29]          # N_q = 30: idle x 4, full, 5 left, all left, one left
    t = Tree(1, dtype, [100] * 8, done, 30, [chain(n)] * 6 + [np.full(n, -2), comb(n)], d=64)
    want = t.expected()
    assert not want[:5].any() and want[5, :5].any() and not want[5, 5:].any() and not want[6].any() and want[7, 0].any()
    gone = (want == 0).all((2, 3))
    for x in (t.q, t.k, t.v):
        x[0][gone] = np.nan
    t.up()
    import torch
    got = t.attend()
    torch.cuda.synchronize()
    got = got.float().cpu().numpy()
    near(got, want, t.f32)
    assert not got[gone].any()


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,r,d", [(9, 3, 64), (40, 3, 64), (64, 7, 128), (30, 2, 128)])
def test_rows_that_are_no_numbers_reach_their_descendants_only(dtype, value, n, r, d):
    """A drafted token's rows of NaN or infinity: nodes beside it are what they are without it."""
    t = Tree(n, dtype, [130, 50], [1, 0], 70, [comb(n), comb(n)], r=r, kv=1, d=d)
    want = t.expected()
    t.k[0][0, 4, 0, 5] = value
    t.v[0][1, 5, 0, ::3] = value
    t.up()
    import torch
    got = t.attend()
    torch.cuda.synchronize()
    got = got.float().cpu().numpy()
    from oracle import tree
    for b, bad in ((0, 4), (1, 5)):
        ways = tree.ways(t.parent[b])
        clean = [i for i in range(n) if bad not in ways[i]]
        dirty = [i for i in range(n) if bad in ways[i]]
        near(got[b, clean], want[b, clean], t.f32)
        if b == 1:
            # an infinite value with a weight above 0 is infinite, NaN is NaN; the other dimensions are as they were
            assert not np.isfinite(got[b][dirty][..., ::3]).any()
            rest = np.arange(t.d) % 3 != 0
            near(got[b, dirty][..., rest], want[b, dirty][..., rest], t.f32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,r,d", [(9, 3, 64), (4, 2, 128), (13, 4, 128), (32, 4, 64), (64, 2, 128), (64, 7, 128), (64, 4, 64)])
def test_visible_keys_of_minus_infinity_have_no_weight(dtype, n, r, d):
    """A key with a component of minus infinity where the query's is positive has a score of minus infinity: it takes no
    part, and the rows that see it are finite. In the context, and in the tree, where the turned key is minus infinity in
    both halves of its pair. (The pair is the slowest one, which no position here turns by more than 0.001.)"""
    import torch
    t = Tree(n, dtype, [150, 70], [0, 3], 80, [comb(n), comb(n)], r=r, kv=1, d=d)
    first, second = d // 2 - 1, d - 1
    for half in (first, second):
        t.q[..., half] = np.abs(t.q[..., half]) + 0.5
    if not t.f32:
        t.q = bf16(t.q)
    t.keys[0][0, 0, [3, 64, 149], first] = -np.inf
    t.keys[0][1, 0, [0, 72], second] = -np.inf
    t.k[0][1, min(n - 1, 2), 0, first] = -np.inf
    t.up()
    t.kc = [t.device(x) for x in t.keys]
    got, want = t.attend(), t.expected()
    torch.cuda.synchronize()
    assert np.isfinite(want).all()
    near(got.float().cpu().numpy(), want, t.f32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,r,d", [(9, 2, 64), (16, 4, 128), (64, 7, 128), (64, 4, 64)])
def test_context_rows_behind_the_last_token_are_not_looked_at(dtype, n, r, d):
    import torch
    outs = [Tree(5, dtype, [97, 64, 0], [3, 0, 1], 70, forest(3, n), r=r, d=d, fill=fill).attend() for fill in (np.nan, np.inf, 0.0)]
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of several hundred, from both sides, in the context and in the tree."""
    t = Tree(8, dtype, [300, 10], [0, 4], 40, forest(2, 10), r=2, kv=1, d=64)
    t.q *= 64.0
    t.up()
    import torch
    got = t.attend()
    torch.cuda.synchronize()
    got, want = got.float().cpu().numpy(), t.expected()
    assert np.isfinite(got).all()
    if t.f32:
        # scores of +-800: 2^-24 of them, a few times over, is 1e-4 of a weight
        assert np.abs(got - want).max() <= 1e-3 * np.abs(want).max()
    else:
        # a rounded query's score is off by 64 * 0.02 (see near): weights by factors, outputs stay within the values
        assert np.abs(got).max() <= np.abs(t.values[0][np.isfinite(t.values[0])]).max() + np.abs(t.v).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,r,d", [(4, 2, 64), (13, 4, 128), (32, 4, 128), (64, 8, 128), (64, 4, 64)])
@pytest.mark.parametrize("direction", [1, -1])
def test_scores_that_grow_or_fall_along_the_context(dtype, n, r, d, direction):
    """Along the context the keys turn from pointing away from every query to pointing at it, scores from -100 to 100 in steps
    of two per 64 keys, or the other way round: references have to follow, by factors far beyond what an exponent holds.
    The direction that the scores come from is one that no position turns (the last pair's angle is below 0.02 here)."""
    length = 6400
    t = Tree(2, dtype, [length, 320], [0, 3], 80, forest(2, n, ("comb", "chain")), r=r, kv=1, d=d)
    u = np.zeros(d, np.float32)
    u[d // 2 - 1] = 1.0
    ramp = (np.arange(t.T, dtype=np.float32) / length * 2 - 1) * 100 * direction
    t.q[:] = 0.25 * t.q + np.sqrt(d) * u / 2
    t.keys[:] = 0.25 * t.keys + ramp[:, None] * u * 2
    t.k[:] = 0.25 * t.k
    if dtype == "bf16":
        from tree_cases import bf16
        t.q, t.keys, t.k = bf16(t.q), bf16(t.keys), bf16(t.k)
    t.up()
    t.kc = [t.device(x) for x in t.keys]
    import torch
    got = t.attend()
    torch.cuda.synchronize()
    got, want = got.float().cpu().numpy(), t.expected()
    assert np.isfinite(got).all()
    # a score of 100 is known to 100 * 2^-24 * a few roundings in fp32, to 100 * 2^-8 / sqrt(3) of the one product that makes it
    # in bf16 (the query is rounded, by the same factor for all keys): neighbours in weight differ by steps of 2 / 64 a key,
    # so that weights over some 30 keys are off by a tenth at most
    err = np.abs(got - want)
    assert (err <= (2e-4 if t.f32 else 0.25) * np.maximum(1.0, np.abs(want))).all(), err.max()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("n", [1, 5, 16])
def test_a_chain_is_a_decode_step(dtype, d, n):
    """With parent i - 1 the rows are those of segmented_decode_step(q_first = done)."""
    import torch
    from paper_2510_18546_amd import binding as B
    t = Tree(n, dtype, [333, 333], [4, 4], 40, [chain(n)] * 2, r=2, kv=2, d=d, fill=0.0)
    got = t.attend()
    step = torch.empty_like(got)
    ws = torch.empty(max(256, B.decode_workspace_bytes(t.pool, t.plan, n)), dtype=torch.uint8, device="cuda:0")
    B.segmented_decode_step(t.pool, t.plan, 4, t.dq[0], t.dk[0], t.dv[0], t.kc[0], t.vt[0], step, ws)
    torch.cuda.synchronize()
    near(got.float().cpu().numpy(), t.expected(), t.f32)
    near(step.float().cpu().numpy(), t.expected(), t.f32)


def test_an_8_bit_pool_has_bf16_contexts():
    import torch
    from paper_2510_18546_amd import binding as B
    t = Tree(3, "bf16", [150, 20], [2, 0], 30, forest(2, 8), d=128)
    want = t.attend()
    cap = 150
    pool = B.kv_pool_create(None, None, t.lens, t.hq, 500000.0, cap + 30, dtype=B.EN_I8, k_ptr=t.block.data_ptr(),
                            v_ptr=t.block.data_ptr(), shape=(2, t.kv, cap, t.d))
    plan = B.segment_select(pool, [0, 1], [0, 1, 2], 30)
    out = torch.empty_like(want)
    ws = torch.empty(max(256, B.tree_workspace_bytes(pool, plan, 8)), dtype=torch.uint8, device="cuda:0")
    B.segmented_tree_attention(pool, plan, t.ddone, t.dparent, t.dq[0], t.dk[0], t.dv[0], t.kc[0], t.vt[0], out, ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_twice_the_same_bits_and_another_stream(dtype):
    import torch
    t = Tree(9, dtype, [1500, 700], [3, 8], 60, forest(2, 20), r=4, kv=2, d=128)
    first = t.attend()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = t.attend()
    torch.cuda.synchronize()
    assert torch.equal(first, second)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(dtype):
    """What changes from step to step is device memory: the graph follows it."""
    import torch
    t = Tree(4, dtype, [400, 90, 10], [0, 2, 5], 60, forest(3, 10), r=2, kv=2, d=64, fill=0.0)
    out = t.attend()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        t.attend(out=out)
    for step in range(4):
        done = np.array([step, 7 * step - 1, 20], np.int32)
        parent = np.stack(forest(3, 10, [("chain", "comb", "star", "broken")[(step + k) % 4] for k in range(3)])).astype(np.int32)
        t.ddone.copy_(t.device(done))
        t.dparent.copy_(t.device(parent))
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.float().cpu().numpy()
        eager = t.attend()
        torch.cuda.synchronize()
        assert np.array_equal(got, eager.float().cpu().numpy())
        t.done, t.parent = done, parent
        near(got, t.expected(), t.f32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_calls_at_once(dtype):
    """Two streams, two scratch buffers, one plan: the calls only read what they share."""
    import torch
    t = Tree(3, dtype, [3000, 900], [3, 8], 60, forest(2, 33), r=4, kv=2, d=64)
    want = t.attend()
    torch.cuda.synchronize()
    streams, outs, scratch = [torch.cuda.Stream() for _ in range(2)], [], [t.ws, t.ws.clone()]
    for _ in range(4):
        for s, ws in zip(streams, scratch):
            t.ws = ws
            with torch.cuda.stream(s):
                outs.append(t.attend())
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in outs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,n_new", [(64, 5), (64, 1), (10, 10)])
def test_more_nodes_than_the_reserve(dtype, n, n_new):
    check(Tree(n, dtype, [77, 5, 64], [0, n_new - 1, n_new // 2], n_new, forest(3, n, ("star", "comb", "chain"))))


def test_timed_like_the_other_attention_calls():
    import torch
    from paper_2510_18546_amd import binding as B
    t = Tree(2, "bf16", [200], [0], 20, [comb(6)])
    B.timing_enable(t.pool, 4)
    t.attend()
    t.attend()
    torch.cuda.synchronize()
    ms = B.timing_collect(t.pool, 4)
    assert len(ms) == 2 and (ms > 0).all()


def test_contexts_of_more_than_4_gib():
    """The last of 70 agents over 32 K tokens lies 2.3e9 elements into the buffers; its rows and its commit are right, and the
    other rows of its context are as they were."""
    import torch
    from oracle import tree
    from paper_2510_18546_amd import binding as B
    agents, kv, d, n, length, n_new = 70, 8, 128, 3, 32_000, 8
    block = torch.zeros(64, device="cuda:0")
    pool = B.kv_pool_create(None, None, np.array([length]), kv, BASE, length + n_new, dtype=B.EN_BF16, k_ptr=block.data_ptr(),
                            v_ptr=block.data_ptr(), shape=(1, kv, length, d))
    plan = B.segment_select(pool, np.zeros(agents, np.int32), np.arange(agents + 1), n_new)
    T = plan.info.ctx_stride
    torch.manual_seed(5)
    some = dict(dtype=torch.bfloat16, device="cuda:0")
    kc, vt = torch.zeros(agents, kv, T, d, **some), torch.zeros(agents, kv, d, T, **some)
    assert kc.numel() > 2**31
    kc[-1].normal_()
    vt[-1].normal_()
    keys = kc[-1].float().cpu().numpy()[None]
    values = np.moveaxis(vt[-1].float().cpu().numpy()[..., column(np.arange(T))], -1, -2)[None]
    q, k, v = (torch.randn(agents, n, kv, d, **some) for _ in range(3))
    i32 = dict(dtype=torch.int32, device="cuda:0")
    parent = torch.tensor(np.stack([chain(n)] * agents), **i32)
    done = torch.full((agents,), 2, **i32)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, B.tree_workspace_bytes(pool, plan, n)), dtype=torch.uint8, device="cuda:0")
    B.segmented_tree_attention(pool, plan, done, parent, q, k, v, kc, vt, out, ws)
    torch.cuda.synchronize()
    last = [x[-1:].float().cpu().numpy() for x in (q, k, v)]
    want = tree.attention(keys, values, [length], [2], n_new, parent[-1:].cpu().numpy(), *last, BASE)
    near(out[-1:].float().cpu().numpy(), want, False)

    path = torch.tensor([[0, 2, -1]] * agents, **i32)
    B.segmented_tree_commit(pool, plan, done + 2, done, path, [k], [v], [kc], [vt])
    torch.cuda.synchronize()
    now = np.moveaxis(vt[-1].float().cpu().numpy()[..., column(np.arange(T))], -1, -2)
    values[0][:, length + 2:length + 4] = np.moveaxis(last[2][0, [0, 2]], 0, 1)
    assert np.array_equal(now, values[0])
    now = kc[-1].float().cpu().numpy()
    for j, node in ((0, 0), (1, 2)):
        key = tree.rope(last[1][0, node], length + 2 + j, BASE)
        # half a step of bf16, and the rotation in float32 as in the tests of the commit
        assert (np.abs(now[:, length + 2 + j] - key) <= 4 * 2.0 ** -24 * 10 + 2.0 ** -8 * np.abs(key)).all()
        now[:, length + 2 + j] = keys[0][:, length + 2 + j]
    assert np.array_equal(now, keys[0])
