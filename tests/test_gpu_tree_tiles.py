"""Attention over trees of drafted tokens where a workgroup takes many tiles, one behind the other: many agents, so that
the keys are cut into few splits, for each number of row blocks that a workgroup may take. A few agents differ, the others
are copies of them whose rows have to be the same bits.

Tolerance, bf16, per row in the 2-norm. The output is rounded once: 2^-8 of it at most. A weight p_j is off by a relative
e_j: its own rounding, at most 2^-8 and in the mean square 2^-8 / sqrt(3), and the query's in its score, as much for scores
of standard normal numbers (their D products over sqrt(D) are off by 2^-8 / sqrt(3) each in the mean square). The weights'
sum is off by the same, so that the row is off by sum p_j e_j (v_j - out): in the mean square 2^-8 sqrt(2 / 3) times
sqrt(sum p_j^2 |v_j - out|^2), which is computed beside the expected row; six times that is allowed. Drafted keys are
rounded in the expected rows as they are held. A tile that is left out moves every row by more than that: by 2.4 to 16
times as much, row by row, of the largest number here, 47, by 5 to 28 times as much of 13. fp32: as in tree_cases.near."""
import numpy as np
import pytest

from oracle import tree
from tree_cases import BASE, TREES, Tree, bf16, near

MERGE_WIDE = 2048      # groups of values from which on a wave of the merge has one to itself


def exact_rows(t, b, layer=0):
    """Agent b's rows [n, Hq, D] in 64 bits, and what the errors of their weights are measured in."""
    d, length = t.d, int(t.lens[b] + t.done[b])
    ways = tree.ways(t.parent[b], tree.room_of(int(t.done[b]), t.n_new))
    out, spread = np.zeros((t.n, t.hq, d)), np.zeros((t.n, t.hq))
    held = [i for i, w in enumerate(ways) if w]
    if not held:
        return out, spread
    sees = np.full((len(held), t.n), -np.inf)
    for row, i in enumerate(held):
        sees[row, ways[i]] = 0.0
    as_held = (lambda x: x) if t.f32 else (lambda x: bf16(x).astype(np.float64))
    for g in range(t.kv):
        own = np.zeros((t.n, d))
        for i in held:
            own[i] = as_held(tree.rope(t.k[layer][b, i, g], length + len(ways[i]) - 1, BASE))
        keys = np.concatenate([t.keys[layer][b, g, :length].astype(np.float64), own])
        values = np.concatenate([t.values[layer][b, g, :length], t.v[layer][b, :, g]]).astype(np.float64)
        for h in range(g * t.r, (g + 1) * t.r):
            q = np.stack([tree.rope(t.q[layer][b, i, h], length + len(ways[i]) - 1, BASE) for i in held])
            s = q @ keys.T / np.sqrt(d)
            s[:, length:] += sees
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o = p @ values
            out[held, h] = o
            p2 = p * p
            square = p2 @ (values * values).sum(1) - 2 * (o * (p2 @ values)).sum(1) + p2.sum(1) * (o * o).sum(1)
            spread[held, h] = np.sqrt(np.maximum(square, 0.0))
    return out, spread


class Copies(Tree):
    """`agents` agents, agent b a copy of agent b % m of the m that `lens` and the others name."""

    def __init__(self, seed, dtype, agents, lens, done, n_new, parent, change=None, **kw):
        import torch
        from paper_2510_18546_amd import binding as B
        super().__init__(seed, dtype, lens, done, n_new, parent, **kw)
        if change:
            change(self)
        self.up()
        self.m, self.of = len(lens), np.arange(agents) % len(lens)
        of = torch.from_numpy(self.of).to("cuda:0")
        more = lambda xs: [x[of].contiguous() for x in xs]
        self.kc, self.vt = more([self.device(x) for x in self.keys]), more(self.vt)
        self.dq, self.dk, self.dv = more(self.dq), more(self.dk), more(self.dv)
        self.ddone, self.dparent = self.ddone[of].contiguous(), self.dparent[of].contiguous()
        cap = max(1, int(self.lens.max()))
        self.pool = B.kv_pool_create(None, None, self.lens[self.of], self.hq, BASE, cap + n_new, dtype=self.pool.desc.dtype,
                                     k_ptr=self.block.data_ptr(), v_ptr=self.block.data_ptr(), shape=(agents, self.kv, cap, self.d))
        self.plan = B.segment_select(self.pool, np.arange(agents), np.arange(agents + 1), n_new)
        assert self.plan.info.ctx_stride == self.T
        self.need = B.tree_workspace_bytes(self.pool, self.plan, self.n)
        self.ws = torch.empty(max(256, self.need), dtype=torch.uint8, device="cuda:0")
        self.ws.fill_(0xFF)
        self.blocks = agents * self.kv * -(-self.r * self.n // 32)

    def splits(self):
        """As many as the scratch holds: a reference, a sum and D values for each row of every block."""
        if self.need == 0:
            return 1
        rows = self.blocks * 32
        s, = [s for s in range(2, 65) if (s * rows * 8 + 255) // 256 * 256 + s * rows * self.d * 4 == self.need]
        return s

    def check(self):
        import torch
        got = self.attend()
        torch.cuda.synchronize()
        of = torch.from_numpy(self.of).to("cuda:0")
        assert torch.equal(got, got[:self.m][of])
        got = got[:self.m].double().cpu().numpy()
        for b in range(self.m):
            want, spread = exact_rows(self, b)
            if self.f32:
                near(got[b], want, True)
                continue
            err = np.linalg.norm(got[b] - want, axis=-1)
            most = 2.0 ** -8 * np.linalg.norm(want, axis=-1) + 6 * 2.0 ** -8 * np.sqrt(2 / 3) * spread
            assert (err <= most).all(), (b, np.nanmax(err / np.maximum(most, 1e-30)))


def forest(agents, n):
    return [TREES[("comb", "broken", "chain", "star")[b % 4]](n) for b in range(agents)]


# (r, n): 1, 2, 4 and 8 blocks of 32 rows in a workgroup, 6 of 8, and two workgroups of 7
SHAPES = [(2, 13), (4, 13), (4, 25), (4, 64), (3, 64), (7, 64)]
# agents, KV heads, tiles of the longest agents
MANY = [(260, 1, 3), (260, 1, 4), (260, 1, 5), (130, 2, 10), (260, 1, 13), (100, 1, 11), (70, 1, 30)]
LEVELS = [((-200, -100, 0), -200), ((-200, -100, 0), 0), ((0, -100, -200), 0), ((0, -100, -200), -200), ((-100, 0, -200), -200),
          ((-200, -100, -200), 0), ((-200, 0, 0), -100)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,r,n,agents,kv,tiles",
                         [("bf16", (64, 128)[(i + j) % 2], *shape, *many) for i, shape in enumerate(SHAPES) for j, many in enumerate(MANY)] +
                         [("f32", (64, 128)[i % 2], *SHAPES[i], *MANY[3 * i]) for i in range(3)])
def test_workgroups_of_many_tiles(dtype, d, r, n, agents, kv, tiles):
    """Even and odd numbers of tiles, the last one in part, of agents that differ in how many they have."""
    full = tiles * 64
    lens = [full - 64 + 37, full - 8, full - 128, 70, full - 191]
    t = Copies(tiles + n, dtype, agents, lens, [3, 8, 0, 5, 70], 150, forest(5, n), r=r, kv=kv, d=d)
    if dtype == "bf16":
        assert (tiles + 1) / t.splits() > 3       # for each workgroup of the longest agents
    t.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,r,n,agents,levels,own",
                         [("bf16", (64, 128)[(i + j) % 2], *shape, (260, 90)[(i // 2 + j) % 2], *at) for i, shape in enumerate(SHAPES)
                          for j, at in enumerate(LEVELS)] + [("f32", (64, 128)[j % 2], *SHAPES[j % 3], 90, *at) for j, at in enumerate(LEVELS)])
def test_scores_that_jump_between_the_tiles_of_a_workgroup(dtype, d, r, n, agents, levels, own):
    """Nine context tiles, the scores of each three at a level of its own, and the drafted keys' scores at one: levels are
    100 log2 units and more apart, so that a reference is replaced up to twice in a workgroup and nothing may stay of what
    was summed against the old one. What counts at the end is at a level of 0, whose keys lack the component that makes the
    level: its error in bf16 is in no weight."""
    def change(t):
        c = d // 2 - 1                            # of the slowest pair: no position here turns it by more than 0.002
        t.q[..., c] = 8.0
        level = np.repeat(np.float32(levels), 3 * 64)
        level = np.concatenate([level, np.full(t.T - len(level), levels[-1], np.float32)])
        t.keys[0][..., c] = np.where(np.isnan(t.keys[0][..., c]), np.nan, level)
        t.k[..., c] = own

    t = Copies(n + d, dtype, agents, [9 * 64 - 5, 9 * 64 - 50, 8 * 64 + 3], [2, 0, 1], 80, forest(3, n), change, r=r, kv=1, d=d)
    assert dtype == "f32" or t.splits() <= (1 if agents == 260 else 2)
    t.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,r,n,agents", [("bf16", (64, 128)[(i + j) % 2], *shape, agents) for i, shape in enumerate(SHAPES)
                                                for j, agents in enumerate((2, 260))] + [("f32", 64, 2, 13, 2), ("f32", 128, 4, 25, 260)])
def test_rows_whose_keys_all_have_no_weight_are_zero(dtype, d, r, n, agents):
    """Every score minus infinity, but those of one drafted key: rows that see it are its value's and those that do not are
    zero, with one split and with several."""
    import torch
    first, second = d // 2 - 1, d - 1             # (the slowest pair, see test_scores_that_jump_between_the_tiles_of_a_workgroup)

    def change(t):
        for half in (first, second):
            t.q[..., half] = bf16(np.abs(t.q[..., half]) + 0.5)
        t.keys[..., first] = np.where(np.isnan(t.keys[..., first]), np.nan, -np.inf)
        t.k[:, :, :2, :, first] = t.k[:, :, 3:, :, first] = -np.inf

    t = Copies(n, dtype, agents, [130, 64], [1, 0], 80, forest(1, n) * 2, change, r=r, kv=1, d=d)
    assert dtype == "f32" or (t.splits() == 1) == (agents == 260)
    got = t.attend()
    torch.cuda.synchronize()
    got = got[:2].double().cpu().numpy()
    for b in range(2):
        for i, way in enumerate(tree.ways(t.parent[b])):
            want = np.broadcast_to(t.v[0][b, 2, 0] if 2 in way else 0.0, got[b, i].shape)
            assert np.array_equal(got[b, i], want), (b, i)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,r,n,d,agents,kv,length,wide", [
    ("bf16", 2, 13, 128, 127, 1, 900, False), ("bf16", 2, 13, 128, 128, 1, 900, True), ("bf16", 2, 13, 128, 64, 2, 900, True),
    ("bf16", 4, 25, 64, 63, 1, 1400, False), ("bf16", 4, 25, 64, 64, 1, 1400, True), ("bf16", 4, 64, 128, 16, 1, 3000, True),
    ("bf16", 7, 64, 128, 9, 1, 2500, False), ("bf16", 7, 64, 128, 10, 1, 2500, True),
    ("f32", 2, 8, 64, 170, 1, 7680, False), ("f32", 2, 8, 64, 300, 1, 7680, True), ("f32", 4, 8, 128, 150, 1, 7680, True)])
def test_both_forms_of_the_merge(dtype, r, n, d, agents, kv, length, wide):
    """Just below and above the number of groups of values from which on each is one wave's."""
    t = Copies(agents, dtype, agents, [length, length - 333, 20], [1, 0, 4], 70, forest(3, n), r=r, kv=kv, d=d)
    assert t.splits() > 1 and (t.blocks * (d // 8) >= MERGE_WIDE) == wide
    t.check()


def test_the_expected_rows_are_the_oracles():
    """Without a GPU: the rows above against the oracle that goes node by node."""
    t = Tree.__new__(Tree)
    rng = np.random.default_rng(3)
    t.lens, t.done, t.n_new, t.n, t.r, t.kv, t.hq, t.d, t.f32 = np.array([50, 7]), np.array([2, 0]), 12, 9, 3, 2, 6, 64, False
    t.parent = np.stack([TREES["broken"](9), TREES["comb"](9)]).astype(np.int64).astype(np.int32)
    t.keys, t.values = (bf16(rng.standard_normal((1, 2, 2, 64, 64))) for _ in range(2))
    t.q, t.k, t.v = (bf16(rng.standard_normal((1, 2, 9, h, 64))) for h in (6, 2, 2))
    want = tree.attention(t.keys[0], t.values[0], t.lens, t.done, 12, t.parent, t.q[0], t.k[0], t.v[0], BASE,
                          round_keys=lambda x: bf16(x).astype(np.float64))
    for b in range(2):
        rows, spread = exact_rows(t, b)
        assert np.abs(rows - want[b]).max() < 1e-12
        assert (spread[np.abs(rows).sum(-1) > 0] > 0).all()
