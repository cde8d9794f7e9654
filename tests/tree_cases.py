"""What the tests of drafted tokens share: trees, gathered contexts drawn in their documented layout, the library's
handles around them."""
import numpy as np

from paper_2510_18546_amd import inputs as I

BASE = 500000.0


def chain(n):
    return np.arange(n) - 1


def star(n):
    return np.full(n, -1)


def comb(n):
    """Node 0 the root, the others on one of the six before them; fixed by n."""
    rng = np.random.default_rng(n)
    return np.array([-1] + [i - 1 - rng.integers(0, min(6, i)) for i in range(1, n)])


def broken(n):
    """A tree with what is no link in it: absent nodes, nodes below them, a node that names itself or a later one."""
    p = comb(n)
    for i, x in ((1, -2), (3, 3), (4, n), (6, 2**31 - 1), (7, -2**31), (9, 11)):
        if i < n:
            p[i] = x
    return p


TREES = {f.__name__: f for f in (chain, star, comb, broken)}


def column(t):
    """Column of token t in the transposed values: bits 2 and 3 exchanged."""
    return (t & ~12) | ((t & 4) << 1) | ((t & 8) >> 1)


def bf16(x):
    return I.round_to_bf16(np.asarray(x, np.float32))


class Tree:
    """Agents over gathered contexts: pool, plan, context buffers and a drafted tree on the GPU, and the same numbers on
    the host. Context rows that hold no token are NaN unless `fill` says otherwise."""

    def __init__(self, seed, dtype, lens, done, n_new, parent, r=2, kv=2, d=64, fill=np.nan, layers=1):
        import torch
        from paper_2510_18546_amd import binding as B
        rng = np.random.default_rng(seed)
        self.lens, self.done = np.asarray(lens, np.int32), np.asarray(done, np.int32)
        self.parent = np.asarray(parent, np.int64).astype(np.int32)
        self.agents, self.n = self.parent.shape
        self.r, self.kv, self.hq, self.d, self.n_new, self.layers = r, kv, r * kv, d, n_new, layers
        self.f32 = dtype == "f32"
        self.type = torch.float32 if self.f32 else torch.bfloat16
        cap = max(1, int(self.lens.max()))
        block = torch.zeros(64, device="cuda:0")
        self.pool = B.kv_pool_create(None, None, self.lens, self.hq, BASE, cap + n_new, dtype=B.EN_F32 if self.f32 else B.EN_BF16,
                                     k_ptr=block.data_ptr(), v_ptr=block.data_ptr(), shape=(self.agents, kv, cap, d))
        self.block = block
        self.plan = B.segment_select(self.pool, np.arange(self.agents), np.arange(self.agents + 1), n_new)
        self.T = self.plan.info.ctx_stride
        shape = (layers, self.agents, kv, self.T, d)
        k, v = (rng.standard_normal(shape, dtype=np.float32) for _ in range(2))
        held = np.where((self.done >= 0) & (self.done <= n_new), self.lens + self.done, self.lens)
        empty = np.arange(self.T)[None] >= held[:, None]
        k[:, empty.nonzero()[0], :, empty.nonzero()[1]] = fill
        v[:, empty.nonzero()[0], :, empty.nonzero()[1]] = fill
        rows = [rng.standard_normal((layers, self.agents, self.n, h, d), dtype=np.float32) for h in (self.hq, kv, kv)]
        if not self.f32:
            k, v = bf16(k), bf16(v)
            rows = [bf16(x) for x in rows]
        self.keys, self.values = k, v
        self.q, self.k, self.v = rows
        vt = v
        if not self.f32:
            vt = np.empty((layers, self.agents, kv, d, self.T), np.float32)
            vt[..., column(np.arange(self.T))] = np.moveaxis(v, -1, -2)
        self.up()
        self.kc = [self.device(x) for x in k]
        self.vt = [self.device(x) for x in vt]
        self.ws = torch.empty(max(256, B.tree_workspace_bytes(self.pool, self.plan, self.n)), dtype=torch.uint8, device="cuda:0")
        self.ws.fill_(0xFF)                     # a NaN pattern: nothing is read that was not written

    def device(self, x):
        import torch
        if x.dtype.kind == "i":
            return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to("cuda:0")
        return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to("cuda:0").to(self.type)

    def up(self):
        """The rows and the tree on the device, again after a change on the host."""
        self.dq, self.dk, self.dv = ([self.device(x) for x in rows] for rows in (self.q, self.k, self.v))
        self.ddone, self.dparent = self.device(self.done), self.device(self.parent)

    def attend(self, layer=0, stream=None, out=None):
        import torch
        from paper_2510_18546_amd import binding as B
        if out is None:
            out = torch.full_like(self.dq[layer], 7.0)
        B.segmented_tree_attention(self.pool, self.plan, self.ddone, self.dparent, self.dq[layer], self.dk[layer], self.dv[layer],
                                   self.kc[layer], self.vt[layer], out, self.ws, stream)
        return out

    def expected(self, layer=0):
        from oracle import tree
        return tree.attention(self.keys[layer], self.values[layer], self.lens, self.done, self.n_new, self.parent, self.q[layer],
                              self.k[layer], self.v[layer], BASE)

    def context(self, layer=0):
        """(keys, values) [B, Hkv, T, D] as they are on the device now, float32."""
        k, v = self.kc[layer].float().cpu().numpy(), self.vt[layer].float().cpu().numpy()
        return k, v if self.f32 else np.moveaxis(v[..., column(np.arange(self.T))], -1, -2)


def near(got, want, f32, scale=1.0):
    """Outputs of attention over values of about `scale` (standard normal times it).

    fp32: 1e-5 of the row's largest value, as every fp32 case of this library. bf16: the output is rounded once, at most
    2^-8 of it; a probability and a partial result once each, 2^-8 of sum p |v|, which is below 5 `scale`; queries and
    drafted keys are rounded after their rotation, off by 2^-8 / sqrt(3) of each product of a score in the mean square:
    of D products of standard normal numbers over sqrt(D) that is 0.0023 a side, 0.0032 for both, six times that 0.02, in
    the weight and in their sum. Together 2^-8 |out| + (2^-7 + 2 * 0.02) sum p |v|, with sum p |v| below `scale` on average
    over many keys and up to 4 `scale` over few: 2^-8 |out| + 0.05 * 4 scale bounds a single value, and in the 2-norm,
    where errors of either sign add up as squares, 2^-8 / sqrt(3) times sqrt(5) for the five roundings: 0.0051 of the
    output's norm, which with weights that differ grows by half at most: 0.0076."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got))
    err = np.abs(got - want)
    if f32:
        row = np.abs(np.where(fine, want, 0.0)).max(-1, keepdims=True)
        assert (np.where(fine, err, 0.0) <= 1e-5 * np.maximum(np.abs(np.where(fine, want, 0.0)), row)).all(), err[fine].max()
        return
    assert (err[fine] <= 2.0 ** -8 * np.abs(want[fine]) + 0.2 * scale).all(), err[fine].max()
    norm = np.linalg.norm(want[fine])
    assert np.linalg.norm(err[fine]) <= 0.0076 * norm, (np.linalg.norm(err[fine]) / max(norm, 1e-30))
