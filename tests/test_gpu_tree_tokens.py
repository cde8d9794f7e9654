"""Rules on logits (token_rules_apply) and acceptance (token_tree_accept) against the float64 oracle, and the accepted
tokens' way into the contexts (segmented_tree_commit).

Tolerances. The rules are a division or product, a product, two differences and a sum, each off by 2^-24 of its result at
most, and the results are below |x| max(rep, 1) + c freq + pres + |bias|: 5 * 2^-24 of that, and for bf16 logits 2^-8 of
the result on top. Choices are compared where float32 cannot tell otherwise: exactly, on values whose rules are exact in
float32 (powers of two, small multiples of 1/8)."""
import numpy as np
import pytest

from tree_cases import TREES, Tree, bf16, broken, chain, comb

pytestmark = pytest.mark.gpu


def dev(x):
    import torch
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to("cuda:0")


def logits_on(x, dtype, pad=0, shift=0):
    """[B, n, V] on the device with rows V + pad apart, the first one `shift` elements into its buffer."""
    import torch
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    b, n, v = x.shape
    buf = torch.full((shift + b * n * (v + pad),), float("nan"), dtype=t, device="cuda:0")
    view = buf[shift:].view(b, n, v + pad)[:, :, :v]
    view.copy_(dev(x.astype(np.float32)))
    return view


def drawn(seed, agents, n, vocab, dtype, history=0, bias=None, mask=None, exact=False):
    rng = np.random.default_rng(seed)
    c = {"tokens": rng.integers(-2, vocab + 2, (agents, n)).astype(np.int32)}
    x = rng.standard_normal((agents, n, vocab)).astype(np.float32) * 4
    x = np.round(x * 8) / 8 if exact else x
    c["logits"] = x if dtype == "f32" else bf16(x)
    c["penalties"] = c["history"] = c["history_len"] = c["bias"] = c["mask"] = None
    if history:
        c["history"] = (rng.random((agents, history)) ** 3 * (vocab + 4)).astype(np.int32) - 2
        c["history_len"] = rng.integers(-1, history + 3, agents).astype(np.int32)
    if history is not None:
        c["penalties"] = np.stack([rng.uniform(1.0, 1.5, agents), rng.uniform(0, 0.3, agents), rng.uniform(-0.2, 0.5, agents)], 1)
        if exact:
            c["penalties"] = np.stack([2.0 ** rng.integers(0, 3, agents), rng.integers(0, 4, agents) / 8, rng.integers(-2, 5, agents) / 8], 1)
        c["penalties"] = c["penalties"].astype(np.float32)
    if bias:
        c["bias"] = rng.standard_normal((vocab,) if bias == "all" else (agents, vocab)).astype(np.float32)
        c["bias"] = np.round(c["bias"] * 4) / 4 if exact else c["bias"]
    if mask:
        c["mask"] = rng.integers(-2**31, 2**31, (agents, n if mask == "node" else 1, (vocab + 31) // 32)).astype(np.int32)
    return c


RULES = ("penalties", "history", "history_len", "bias", "mask")


def rules_of(c):
    from paper_2510_18546_amd import binding as B
    return B.token_rules(**{k: dev(c[k]) for k in RULES})


def forest(agents, n):
    kinds = ("comb", "broken", "chain", "star")
    return np.stack([TREES[kinds[b % 4]](n) for b in range(agents)]).astype(np.int64).astype(np.int32)


def check_rules(c, parent, dtype, pad=0, shift=0, in_place=False):
    import torch
    from oracle import tree
    from paper_2510_18546_amd import binding as B
    before = np.full_like(c["logits"], 3.0)
    x = logits_on(c["logits"], dtype, pad, shift)
    out = x if in_place else logits_on(before, dtype, pad, (shift + 1) % 8)
    tokens = c["tokens"] if parent is not None else None
    B.token_rules_apply(rules_of(c), x, out, dev(parent), dev(tokens))
    torch.cuda.synchronize()
    want = tree.rules(c["logits"], parent, tokens, *(c[k] for k in RULES), out=c["logits"] if in_place else before)
    got = out.float().cpu().numpy().astype(np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(np.isneginf(want), np.isneginf(got)) and np.array_equal(fine, np.isfinite(got))
    size = np.abs(c["logits"].astype(np.float64)) * 2 + 2 + 0.3 * (c["history"].shape[1] if c["history"] is not None else 0) + 5
    tol = 5 * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(np.where(fine, want, 0)) if dtype == "bf16" else 0)
    assert (np.abs(got[fine] - want[fine]) <= tol[fine]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 7, 31, 32, 33, 100, 1000, 2047, 2048, 2049, 4099, 32000, 50021])
def test_rules_vocabularies(dtype, vocab):
    c = drawn(vocab, 3, 5, vocab, dtype, history=40, bias="all", mask="node")
    check_rules(c, forest(3, 5), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 13, 64])
@pytest.mark.parametrize("history,bias,mask", [(None, None, None), (0, None, None), (300, None, None), (None, "all", None),
                                               (None, "agent", "agent"), (5000, "agent", "node"), (1, None, "node")])
def test_rules_parts(dtype, n, history, bias, mask):
    c = drawn(n, 3, n, 3001, dtype, history, bias, mask)
    check_rules(c, forest(3, n), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (7, 2), (64, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rules_strides_and_alignment(dtype, pad, shift, in_place):
    c = drawn(pad, 2, 6, 5003, dtype, 77, "all", "node")
    check_rules(c, forest(2, 6), dtype, pad, shift, in_place)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rules_of_rows_by_themselves(dtype):
    check_rules(drawn(1, 5, 1, 4321, dtype, 200, "agent", "agent"), None, dtype)
    check_rules(drawn(2, 2, 3, 777, dtype, 20, None, "node"), None, dtype)


def test_rules_leave_what_lies_between_the_rows():
    import torch
    from paper_2510_18546_amd import binding as B
    c = drawn(3, 2, 4, 1001, "bf16", 10)
    x = logits_on(c["logits"], "bf16")
    buf = torch.full((8 + 8 * 1020,), 5.0, dtype=torch.bfloat16, device="cuda:0")
    out = buf[3:3 + 8 * 1020].view(2, 4, 1020)[:, :, :1001]
    B.token_rules_apply(rules_of(c), x, out, dev(forest(2, 4)), dev(c["tokens"]))
    torch.cuda.synchronize()
    gaps = buf[3:3 + 8 * 1020].view(8, 1020)[:, 1001:]
    assert (gaps == 5.0).all() and (buf[:3] == 5.0).all() and (buf[3 + 8 * 1020:] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("span", [512, 1024])
@pytest.mark.parametrize("different", [126, 127, 128, 129, 255, 256, 257, 512])
def test_rules_where_many_tokens_have_occurred(dtype, span, different):
    """So many different tokens of the first `span`, some more than once, and ways with tokens that are among them or not."""
    vocab, n = 5000, 6
    c = drawn(different, 2, n, vocab, dtype, history=4200, bias="all", mask="node")
    rng = np.random.default_rng(different)
    for b in range(2):
        of = rng.choice(span, min(different, span), replace=False)
        c["history"][b] = rng.choice(of, 4200)
        c["history"][b, :len(of)] = of
        c["tokens"][b] = [of[0], of[0], (of[1] + 1) % span, span, span + 1, of[2]]
    c["history_len"][:] = [4200, 99999]
    check_rules(c, forest(2, n), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rules_count_a_token_as_often_as_the_way_has_it(dtype):
    c = drawn(4, 2, 64, 700, dtype, 0)
    c["tokens"][:] = 5
    c["tokens"][1, ::2] = 699
    check_rules(c, np.stack([chain(64), comb(64)]).astype(np.int32), dtype)


def test_logits_further_apart_than_2_to_the_31():
    """64 rows of a tensor of 2.6e9 elements."""
    import torch
    from oracle import tree
    from paper_2510_18546_amd import binding as B
    n, vocab, apart = 64, 1000, 41_000_003
    c = drawn(6, 1, n, vocab, "bf16", 30, exact=True)
    parent = comb(n)[None].astype(np.int32)
    x = torch.empty(n * apart, dtype=torch.bfloat16, device="cuda:0").as_strided((1, n, vocab), (n * apart, apart, 1))
    x.copy_(dev(c["logits"]))
    t = Tree(2, "bf16", [4], [0], 80, parent, d=64)
    choice = accepted(t, c["tokens"], x, rules_of(c))[0]
    B.token_rules_apply(rules_of(c), x, x, dev(parent), dev(c["tokens"]))
    torch.cuda.synchronize()
    want = tree.rules(c["logits"], parent, c["tokens"], *(c[k] for k in RULES))
    assert list(choice[0]) == [tree.choose(row) for row in want[0]]
    # (exact in float32, rounded to bf16 once)
    assert np.array_equal(x.float().cpu().numpy(), bf16(want))


def accepted(t, tokens, logits, rules=None, choice="out", ws=None, done_out=None):
    import torch
    from paper_2510_18546_amd import binding as B
    i32 = dict(dtype=torch.int32, device="cuda:0")
    shape = (t.agents, t.n)
    choice = torch.full(shape, 99, **i32) if isinstance(choice, str) else choice
    path = torch.full(shape, 99, **i32)
    count, token = torch.full((t.agents,), 99, **i32), torch.full((t.agents,), 99, **i32)
    done = torch.full((t.agents,), 99, **i32) if done_out is None else done_out
    if logits is not None and ws is None:
        ws = torch.empty(max(8, B.tree_accept_workspace_bytes(t.plan, t.n, logits.shape[2])), dtype=torch.uint8, device="cuda:0")
        ws.fill_(0xFF)
    B.token_tree_accept(t.plan, t.ddone, t.dparent, dev(tokens), logits, choice, path, count, token, done, ws, rules)
    torch.cuda.synchronize()
    return [x.cpu().numpy() if x is not None else None for x in (choice, path, count, token, done)]


def check_accept(t, c, dtype, pad=0, shift=0):
    from oracle import tree
    want_x = tree.rules(c["logits"], t.parent, c["tokens"], *(c[k] for k in RULES))
    want_choice = np.full((t.agents, t.n), -1)
    for b in range(t.agents):
        for i, way in enumerate(tree.ways(t.parent[b], tree.room_of(int(t.done[b]), t.n_new))):
            if way:
                want_choice[b, i] = tree.choose(want_x[b, i])
    want = tree.accept(want_choice, t.done, t.n_new, t.parent, c["tokens"])
    choice, path, count, token, done = accepted(t, c["tokens"], logits_on(c["logits"], dtype, pad, shift), rules_of(c))
    assert np.array_equal(choice, want_choice)
    for b, (p, nxt) in enumerate(want):
        assert count[b] == len(p) and list(path[b]) == p + [-1] * (t.n - len(p)) and token[b] == nxt
        assert done[b] == t.done[b] + len(p)
    return want


def agree(c, t, rng, share=0.7, much=64.0):
    """The drafted tokens stand out at their parents, most of them."""
    for b in range(t.agents):
        for i in range(t.n):
            p = int(t.parent[b, i])
            c["tokens"][b, i] = rng.integers(0, c["logits"].shape[2])
            if 0 <= p < i and rng.random() < share:
                c["logits"][b, p, c["tokens"][b, i]] += much


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", [(1, 100), (2, 5000), (8, 2048), (13, 2049), (31, 999), (64, 3000), (5, 70001)])
@pytest.mark.parametrize("history,bias,mask", [(None, None, None), (100, "all", "node"), (9, "agent", "agent")])
def test_accept(dtype, n, vocab, history, bias, mask):
    rng = np.random.default_rng(n)
    agents = 5
    t = Tree(n, "bf16", [10] * agents, [0, 5, -1, 70, 78], 80, forest(agents, n), d=64)
    c = drawn(vocab, agents, n, vocab, dtype, history, bias, mask, exact=True)
    agree(c, t, rng)
    check_accept(t, c, dtype, pad=vocab % 3, shift=vocab % 2)


@pytest.mark.parametrize("different", [255, 256, 257])
def test_accept_where_many_tokens_have_occurred(different):
    c = drawn(different, 2, 9, 3000, "f32", 3000, None, "agent", exact=True)
    rng = np.random.default_rng(1)
    for b in range(2):
        c["history"][b] = rng.choice(rng.choice(1024, different, replace=False), 3000)
    c["history_len"][:] = 3000
    t = Tree(9, "bf16", [10] * 2, [0, 5], 80, forest(2, 9), d=64)
    agree(c, t, rng)
    check_accept(t, c, "f32")


def test_accept_goes_deep():
    """A chain that is right throughout, one that ends at the reserve, siblings with the same token."""
    rng = np.random.default_rng(0)
    n = 40
    twin = np.array([-1] + [0] * 5 + [1, 2, 3] * 11 + [4])
    t = Tree(n, "bf16", [10] * 4, [0, 41, 50, 3], 60, [chain(n), chain(n), chain(n), twin], d=64)
    c = drawn(5, 4, n, 500, "bf16", None, exact=True)
    agree(c, t, rng, share=1.0)
    c["tokens"][3] = 7
    c["logits"][3, :, 7] = 200.0
    want = check_accept(t, c, "bf16")
    assert [len(p) for p, _ in want[:3]] == [40, 19, 10] and want[3][0] == [0, 1, 6]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accept_ties_zeros_and_what_is_no_number(dtype):
    vocab = 6000
    t = Tree(1, "bf16", [4] * 8, [0] * 8, 4, [[-1]] * 8, d=64)
    x = np.full((8, 1, vocab), -5.0, np.float32)
    x[0, 0, [4000, 17, 5999]] = 2.0              # ties in several chunks
    x[1, 0] = -np.inf
    x[2, 0] = np.nan
    x[3, 0, 100], x[3, 0, 50], x[3, 0, 70] = -0.0, 0.0, -0.0
    x[3, 0, 40] = -0.0                           # -0 equals +0: the lowest of them
    x[4, 0, 10], x[4, 0, 11] = np.nan, 1.0
    x[5, 0, [20, 3000]] = np.inf
    x[6, 0] = -np.inf
    x[6, 0, 5999] = -3e38
    x[7, 0, :] = np.nan
    x[7, 0, 3] = -np.inf
    want = [17, -1, -1, 40, 11, 20, 5999, -1]
    choice, path, count, token, done = accepted(t, np.zeros((8, 1), np.int32), logits_on(x, dtype))
    assert list(choice[:, 0]) == want and list(token) == want and (count == 1).all() and (path[:, 0] == 0).all() and (done == 1).all()


def put_signalling(view, at, sign):
    """Signalling NaN, which no arithmetic brings forth, into logits on the device."""
    import torch
    if view.dtype == torch.float32:
        view.view(torch.int32)[at] = 0x7F800001 - (2**31 if sign else 0)
    else:
        view.view(torch.int16)[at] = 0x7F81 - (2**15 if sign else 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [0, 1])
@pytest.mark.parametrize("ruled", ["none", "mask", "penalties", "bias"])
@pytest.mark.parametrize("vocab,base", [(3000, 1480), (3000, 2992), (2053, 2045), (5000, 600)])
def test_accept_signalling_nan(dtype, sign, ruled, vocab, base):
    """The largest logit at every place of a run of eight, a signalling NaN at every other one."""
    places = [(i, j) for i in range(8) for j in range(8) if i != j]
    agents = len(places)
    t = Tree(1, "bf16", [4] * agents, [0] * agents, 4, [[-1]] * agents, d=64)
    c = drawn(3, agents, 1, vocab, dtype, 0 if ruled == "penalties" else None, "all" if ruled == "bias" else None)
    c["logits"][:] = -5.0
    c["tokens"][:] = 17
    if ruled == "mask":
        c["mask"] = np.full((agents, 1, (vocab + 31) // 32), -1, np.int32)
    if ruled == "bias":
        c["bias"][:] = 0.25
    for b, (i, _) in enumerate(places):
        c["logits"][b, 0, base + i] = 2.0
    x = logits_on(c["logits"], dtype)
    for b, (_, j) in enumerate(places):
        put_signalling(x, (b, 0, base + j), sign)
    choice, _, _, token, _ = accepted(t, c["tokens"], x, rules_of(c) if ruled != "none" else None)
    want = [base + i for i, _ in places]
    assert list(choice[:, 0]) == want and list(token) == want


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accept_signalling_nan_everywhere(dtype):
    vocab = 2500
    t = Tree(1, "bf16", [4] * 2, [0] * 2, 4, [[-1]] * 2, d=64)
    x = logits_on(np.zeros((2, 1, vocab), np.float32), dtype)
    put_signalling(x, slice(None), 0)
    x[1, 0, 1234] = -3.0
    choice = accepted(t, np.zeros((2, 1), np.int32), x)[0]
    assert list(choice[:, 0]) == [-1, 1234]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ruled", ["mask", "penalties"])
def test_rules_signalling_nan_stays_nan(dtype, ruled):
    """Written out it is still no number, unless the mask hides it; its neighbours are what they are."""
    import torch
    from oracle import tree
    from paper_2510_18546_amd import binding as B
    c = drawn(7, 2, 1, 1500, dtype, 0 if ruled == "penalties" else None, None, "agent" if ruled == "mask" else None)
    at = np.array([0, 3, 511, 700, 1499])
    x = logits_on(c["logits"], dtype)
    put_signalling(x, (slice(None), slice(None), torch.tensor(at, device="cuda:0")), 0)
    c["logits"][..., at] = np.nan
    out = torch.empty_like(x)
    B.token_rules_apply(rules_of(c), x, out)
    torch.cuda.synchronize()
    want = tree.rules(c["logits"], None, None, *(c[k] for k in RULES))
    assert np.array_equal(out.double().cpu().numpy(), want, equal_nan=True)


def test_accept_where_a_mask_leaves_nothing():
    t = Tree(1, "bf16", [4] * 2, [0] * 2, 8, [chain(3)] * 2, d=64)
    c = drawn(2, 2, 3, 300, "f32", None, None, "node", exact=True)
    c["tokens"][:] = 5
    c["mask"][0, 0] = 0
    c["mask"][1] = 0
    c["mask"][1, 0, 0] = 1 << 5
    check_accept(t, c, "f32")
    choice, path, count, token, _ = accepted(t, c["tokens"], logits_on(c["logits"], "f32"), rules_of(c))
    assert choice[0, 0] == -1 and count[0] == 1 and token[0] == -1 and count[1] == 2 and token[1] == -1


def test_accept_choices_of_the_caller():
    from oracle import tree
    n = 20
    rng = np.random.default_rng(3)
    t = Tree(2, "bf16", [4] * 6, [0, 3, 1, -4, 25, 26], 30, forest(6, n), d=64)
    tokens = rng.integers(0, 3, (6, n)).astype(np.int32)
    choice = rng.integers(-1, 3, (6, n)).astype(np.int32)
    tokens[0, 5], choice[0, 0] = -1, -1
    want = tree.accept(choice, t.done, 30, t.parent, tokens)
    got = accepted(t, tokens, None, choice=dev(choice))
    assert np.array_equal(got[0], choice)
    for b, (p, nxt) in enumerate(want):
        assert got[2][b] == len(p) and list(got[1][b]) == p + [-1] * (n - len(p)) and got[3][b] == nxt and got[4][b] == t.done[b] + len(p)


def test_accept_in_place_and_without_choices():
    t = Tree(2, "bf16", [4] * 2, [2, 3], 30, [comb(6)] * 2, d=64)
    c = drawn(1, 2, 6, 999, "f32", None, exact=True)
    agree(c, t, np.random.default_rng(1), 1.0)
    x = logits_on(c["logits"], "f32")
    _, path, count, token, done = accepted(t, c["tokens"], x)
    none, path2, count2, token2, done2 = accepted(t, c["tokens"], x, choice=None, done_out=t.ddone)
    assert none is None and all(np.array_equal(p, q) for p, q in ((path, path2), (count, count2), (token, token2), (done, done2)))


# ---------------------------------------------------------------------------------------------------------------
# commit
# ---------------------------------------------------------------------------------------------------------------
def commit(t, path, count, done):
    import torch
    from paper_2510_18546_amd import binding as B
    B.segmented_tree_commit(t.pool, t.plan, dev(done), dev(count), dev(path), t.dk, t.dv, t.kc, t.vt)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,d,kv,layers", [("bf16", 64, 2, 1), ("bf16", 128, 3, 5), ("f32", 64, 1, 2), ("f32", 128, 2, 3),
                                               ("bf16", 64, 1, 64), ("bf16", 128, 1, 131)])
@pytest.mark.parametrize("n", [1, 9, 64])
def test_commit(dtype, d, kv, layers, n):
    """Accepted rows are those that a decode step writes, bit for bit (bf16: to half a step of the rotated key; the values
    as they are); every other row is as it was."""
    from oracle import tree
    rng = np.random.default_rng(n + layers)
    agents, n_new = 4, 80
    count = np.array([1, min(n, 7), 0, n], np.int32)
    t = Tree(n, dtype, [70, 3, 9, 0], np.array([5, 11, 2, 0]), n_new, [chain(n)] * agents, kv=kv, d=d, layers=layers, fill=0.25)
    path = np.full((agents, n), -1, np.int32)
    for b in range(agents):
        path[b, :count[b]] = np.sort(rng.choice(n, count[b], replace=False))
    commit(t, path, count, t.done + count)
    for layer in range(layers):
        keys, values = t.context(layer)
        want_k, want_v = t.keys[layer].astype(np.float64), t.values[layer].copy()
        touched = np.zeros((agents, t.T), bool)
        for b in range(agents):
            for j in range(count[b]):
                row = t.lens[b] + t.done[b] + j
                touched[b, row] = True
                want_k[b, :, row] = tree.rope(t.k[layer][b, path[b, j]], row, 500000.0)
                want_v[b, :, row] = t.v[layer][b, path[b, j]]
        assert np.array_equal(values, want_v)
        same = ~touched[:, None, :, None] & np.ones_like(keys, bool)
        assert np.array_equal(keys[same], want_k[same].astype(np.float32))
        # a rotated key: cosine and sine, two products and a sum off by 2^-24 each, of at most |x1| + |x2| < 10
        err = np.abs(keys - want_k)
        assert (err <= 4 * 2.0 ** -24 * 10 + (0 if t.f32 else 2.0 ** -8 * np.abs(want_k))).all()


def test_commit_leaves_out_what_is_no_row():
    n = 6
    t = Tree(1, "bf16", [20] * 5, [3] * 5, 10, [chain(n)] * 5, fill=0.5)
    path = np.array([[0, 99, 2, -7, 2**31 - 1, 5]] * 5, np.int32)
    count = np.array([6, 6, 100, -3, 2], np.int32)
    done = np.array([9, 12, 3, 3, -5], np.int32)      # the second goes past the reserve, the third begins before it
    before = t.context()
    commit(t, path, count, done)
    after = t.context()
    changed = (before[1] != after[1]).any((1, 3))
    assert sorted(changed[0].nonzero()[0]) == [23, 25, 28]      # entries 0, 2, 5
    assert sorted(changed[1].nonzero()[0]) == [26, 28]          # entry 5 would be row 11 of 10
    assert not changed[2].any() and not changed[3].any() and not changed[4].any()


def test_commit_of_no_layers():
    t = Tree(1, "bf16", [20], [3], 10, [chain(4)])
    t.dk, t.dv, t.kc, t.vt = [], [], [], []
    commit(t, np.zeros((1, 4), np.int32), np.array([2], np.int32), np.array([5], np.int32))


# ---------------------------------------------------------------------------------------------------------------
# all of them together
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,captured", [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)])
def test_a_loop_of_drafted_steps(dtype, captured):
    """Two layers, three agents, several steps: attention over the tree in every layer, acceptance from ruled logits, the
    path into both contexts, all on the device; eagerly, and as one graph that is replayed. Each step against the oracle
    from the contexts that the oracle's own rows built up."""
    import torch
    from oracle import tree
    from paper_2510_18546_amd import binding as B
    rng = np.random.default_rng(11)
    agents, n, vocab, n_new, layers, steps = 3, 12, 1500, 40, 2, 5
    parents = forest(agents, n)
    parents[1] = comb(n)
    t = Tree(6, dtype, [140, 64, 5], [0, 2, 35], n_new, parents, r=2, kv=2, d=64, layers=layers, fill=0.0)
    c = drawn(4, agents, n, vocab, "bf16", 30, "all", "agent", exact=True)
    c["history_len"][:] = 30
    rules = rules_of(c)
    i32 = dict(dtype=torch.int32, device="cuda:0")
    x = logits_on(c["logits"], "bf16")
    tokens = dev(c["tokens"])
    choice, path = (torch.empty(agents, n, **i32) for _ in range(2))
    count, token = (torch.empty(agents, **i32) for _ in range(2))
    ws = torch.empty(B.tree_accept_workspace_bytes(t.plan, n, vocab), dtype=torch.uint8, device="cuda:0")
    outs = [torch.empty_like(q) for q in t.dq]

    def step():
        for layer in range(layers):
            t.attend(layer, out=outs[layer])
        B.token_tree_accept(t.plan, t.ddone, t.dparent, tokens, x, choice, path, count, token, t.ddone, ws, rules)
        B.segmented_tree_commit(t.pool, t.plan, t.ddone, count, path, t.dk, t.dv, t.kc, t.vt)

    graph = None
    if captured:
        kept = [z.clone() for z in (*t.kc, *t.vt, t.ddone)]
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            step()
        for z, was in zip((*t.kc, *t.vt, t.ddone), kept):
            z.copy_(was)
    used = 0
    for _ in range(steps):
        for rows in (t.q, t.k, t.v):
            rows[:] = rng.standard_normal(rows.shape) if t.f32 else bf16(rng.standard_normal(rows.shape))
        c["logits"][:] = bf16(np.round(rng.standard_normal(c["logits"].shape) * 32) / 8)
        agree(c, t, rng)
        for there, here in ((t.dq, t.q), (t.dk, t.k), (t.dv, t.v)):
            for z, y in zip(there, here):
                z.copy_(t.device(y))
        x.copy_(dev(c["logits"]))
        tokens.copy_(dev(c["tokens"]))
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        for layer in range(layers):
            from tree_cases import near
            near(outs[layer].float().cpu().numpy(), t.expected(layer), t.f32)
        want_x = tree.rules(c["logits"], t.parent, c["tokens"], *(c[k] for k in RULES))
        want = tree.accept([[tree.choose(r) for r in a] for a in want_x], t.done, n_new, t.parent, c["tokens"])
        for b, (p, nxt) in enumerate(want):
            assert list(path[b].cpu().numpy()[:len(p)]) == p and int(count[b]) == len(p) and int(token[b]) == nxt
            for j, node in enumerate(p):
                row = t.lens[b] + t.done[b] + j
                for layer in range(layers):
                    k = tree.rope(t.k[layer][b, node], row, 500000.0)
                    t.keys[layer][b, :, row] = k if t.f32 else bf16(k)
                    t.values[layer][b, :, row] = t.v[layer][b, node]
            t.done[b] += len(p)
            used += len(p)
        assert np.array_equal(t.ddone.cpu().numpy(), t.done)
    assert used > steps and t.done[2] == n_new


@pytest.mark.parametrize("captured", [False, True])
def test_a_loop_whose_history_grows(captured):
    """The caller appends the accepted tokens to the history, on the device like everything else: choices of later steps are
    those under all tokens so far. The logits stay what they are, so that without them a step's choices would be the ones
    before again."""
    import torch
    from oracle import tree
    from paper_2510_18546_amd import binding as B
    agents, n, vocab, n_new, steps = 3, 6, 300, 60, 6
    t = Tree(4, "bf16", [20, 3, 9], [0, 2, 5], n_new, [chain(n), comb(n), broken(n)], d=64, fill=0.0)
    c = drawn(9, agents, n, vocab, "f32", 10, exact=True)
    agree(c, t, np.random.default_rng(5), 1.0, much=40.0)
    c["penalties"][:] = [2.0, 1.0, 4.0]
    c["history_len"][:] = [4, 0, 10]
    room = 10 + steps * n + 1                       # the last entry is where nothing is appended to
    c["history"] = np.concatenate([c["history"], np.full((agents, room - 10), -1, np.int32)], 1)
    history, length, penalties = (dev(c[k]) for k in ("history", "history_len", "penalties"))
    rules = B.token_rules(penalties, history, length)
    x, tokens = logits_on(c["logits"], "f32"), dev(c["tokens"])
    i32 = dict(dtype=torch.int32, device="cuda:0")
    choice, path = (torch.empty(agents, n, **i32) for _ in range(2))
    count, token = (torch.empty(agents, **i32) for _ in range(2))
    at = torch.arange(n, device="cuda:0")
    ws = torch.empty(B.tree_accept_workspace_bytes(t.plan, n, vocab), dtype=torch.uint8, device="cuda:0")

    def step():
        B.token_tree_accept(t.plan, t.ddone, t.dparent, tokens, x, choice, path, count, token, t.ddone, ws, rules)
        on = path >= 0
        history.scatter_(1, torch.where(on, length[:, None] + at, room - 1), tokens.gather(1, path.clamp(min=0).long()))
        length.add_(count)

    graph = None
    if captured:
        kept = [z.clone() for z in (history, length, t.ddone)]
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            step()
        for z, was in zip((history, length, t.ddone), kept):
            z.copy_(was)
    first = None
    for _ in range(steps):
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        want_x = tree.rules(c["logits"], t.parent, c["tokens"], c["penalties"], c["history"], c["history_len"])
        want_choice = np.array([[tree.choose(r) for r in a] for a in want_x])
        want = tree.accept(want_choice, t.done, n_new, t.parent, c["tokens"])
        for b, (p, nxt) in enumerate(want):
            assert list(path[b].cpu().numpy()[:len(p)]) == p and int(count[b]) == len(p) and int(token[b]) == nxt
            h = int(c["history_len"][b])
            c["history"][b, h:h + len(p)] = c["tokens"][b, p]
            c["history_len"][b] += len(p)
            t.done[b] += len(p)
        assert np.array_equal(length.cpu().numpy(), c["history_len"])
        assert np.array_equal(history.cpu().numpy()[:, :-1], c["history"][:, :-1])
        first = want if first is None else first
    assert want != first
