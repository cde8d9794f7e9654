"""Decoding with drafted tokens in a tree, as cases that can be timed and compared with plain forms.

A decode step that verifies a tree of drafted tokens reads the gathered context once for all of them. Four
kinds of case, one per operator:

  attention  the drafted tokens attend over the context and over their ancestors in the tree
  rules      penalties for repeated tokens, biases and masks of allowed tokens, on logits
  accept     the best token of every node, and the path through the tree that they confirm
  commit     the accepted tokens' keys and values join the contexts of all layers

A case is a dict of sizes and options; what the work depends on (context lengths, how many nodes of an agent's
tree are present, how much of its reserve is used up) follows from the case alone, everything else from the seed.
"""
import math

import torch

own = False

DEV = "cuda:0"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BASE = 500000.0


def _case(**kw):
    c = {"kind": "attention", "dtype": "bf16", "agents": 1, "q_heads": 32, "kv_heads": 8, "head_dim": 128, "ctx": 1536,
         "ragged": False, "nodes": 8, "reserve": 40, "layers": 1, "vocab": 32000, "history": 0, "bias": False, "mask": "none"}
    assert set(kw) - {"name"} <= set(c)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest: seven drafted tokens on a tiny fp32 layer over four groups of 32 tokens
        _case(name="tree of 7, tiny fp32", dtype="f32", q_heads=4, kv_heads=1, head_dim=64, ctx=128, nodes=7),
        # an ordinary step of one agent's plan: eight drafted tokens over a ragged map of 1.5 K tokens
        _case(name="tree of 8, ragged map", ctx=1531),
        # the widest tree over a large map, on a layer of 56 query heads
        _case(name="tree of 64, 56 heads, 8 K", q_heads=56, ctx=8192, nodes=64, reserve=512),
        # sixteen agents over ragged maps, trees of different sizes padded to 13 nodes
        _case(name="16 agents, trees of 13", agents=16, ctx=1920, ragged=True, nodes=13),
        # 64 agents over 16 K tokens each, four drafted tokens: the context comes from HBM
        _case(name="64 agents, trees of 4, 16 K", agents=64, ctx=16384, nodes=4),
        # plain decoding of one token: a grammar's mask and penalties over the 700 tokens so far
        _case(name="rules, one row", kind="rules", dtype="f32", nodes=1, history=700, mask="agent"),
        # sixteen agents' trees, an odd vocabulary, a mask for every node, long histories
        _case(name="rules, 16 trees of 13", kind="rules", agents=16, ragged=True, nodes=13, vocab=50021, history=4096, bias=True,
              mask="node"),
        # one agent's eight drafted tokens, no rules
        _case(name="accept, one tree of 8", kind="accept"),
        # sixteen agents' trees under penalties and masks
        _case(name="accept, 16 trees, rules", kind="accept", agents=16, ragged=True, nodes=13, vocab=128000, history=2048, bias=True,
              mask="node"),
        # the largest: 64 trees of 32 nodes, half a gigabyte of logits
        _case(name="accept, 64 trees of 32", kind="accept", agents=64, nodes=32, vocab=128000),
        # one agent's accepted tokens join the contexts of 40 layers
        _case(name="commit, one agent, 40 layers", kind="commit", layers=40),
        # the same for sixteen agents
        _case(name="commit, 16 agents, 40 layers", kind="commit", agents=16, ctx=1920, ragged=True, nodes=13, layers=40),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def _held(case):
    """Values in the contexts of all layers."""
    return case["layers"] * case["agents"] * case["kv_heads"] * (case["ctx"] + case["reserve"]) * case["head_dim"]


def draw(rng):
    limit = max(_cost(c) for c in listed())
    room = max(_held(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= limit and _held(case) <= room:
            return case


def _draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "rules", "accept", "accept", "commit"])
    agents = rng.choice([1, 1, 2, 3, _log(rng, 1, 64), _log(rng, 1, 64)])
    nodes = rng.choice([1, _log(rng, 1, 64), _log(rng, 1, 64), _log(rng, 2, 32)])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), agents=agents, ragged=rng.random() < 0.5,
             nodes=nodes, reserve=nodes + rng.randint(0, 64))
    if kind in ("attention", "commit"):
        kv, ratio = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 3, 4, 4, 7, 8])
        if c["dtype"] == "f32":
            kv, ratio, c["agents"] = rng.choice([1, 2]), rng.choice([1, 2, 4]), min(agents, 4)
        c.update(kv_heads=kv, q_heads=kv * ratio, head_dim=rng.choice([64, 128, 128]),
                 ctx=_log(rng, 1, 4096 if c["dtype"] == "f32" else 16384))
    if kind == "commit":
        c.update(layers=_log(rng, 1, 64), ctx=_log(rng, 1, 2048))
    if kind in ("rules", "accept"):
        ruled = kind == "rules" or rng.random() < 0.5
        c.update(vocab=_log(rng, 100, 160000), history=_log(rng, 1, 8192) if ruled else 0, bias=ruled and rng.random() < 0.5,
                 mask=rng.choice(["none", "agent", "node"]) if ruled else "none")
    return _case(**c)


# ---------------------------------------------------------------------------------------------------------------
# what a case's work depends on
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Cached tokens of every agent."""
    n = case["ctx"]
    return [n - (b * 37) % (n // 4 + 1) if case["ragged"] else n for b in range(case["agents"])]


def _present(case):
    """Nodes of every agent's tree that are present."""
    n = case["nodes"]
    return [n - (b * 5) % (n // 2 + 1) if case["ragged"] else n for b in range(case["agents"])]


def _done(case):
    """New tokens that every agent's context holds already."""
    room = case["reserve"] - case["nodes"]
    return [(3 + 7 * b) % (room + 1) for b in range(case["agents"])]


def _accepted(case):
    return [1 + (b * 3 + 4) % min(p, 6) for b, p in enumerate(_present(case))]


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    agents, n, hkv, hq, d, vocab = (case[k] for k in ("agents", "nodes", "kv_heads", "q_heads", "head_dim", "vocab"))
    if case["kind"] == "attention":
        keys = [c + m for c, m in zip(_lengths(case), _done(case))]
        rows = agents * n * d * (2 * hq + 2 * hkv) * e
        # of the tree's own keys a node sees itself at least
        return {"bytes": sum(keys) * hkv * d * 2 * e + rows,
                "flops": 4 * d * hq * sum(p * (k + 1) for p, k in zip(_present(case), keys))}
    if case["kind"] == "commit":
        return {"bytes": 2 * 2 * case["layers"] * sum(_accepted(case)) * hkv * d * e, "flops": 0}
    tables = agents * case["history"] * 4 + (vocab * 4 if case["bias"] else 0)
    tables += {"none": 0, "agent": agents, "node": sum(_present(case))}[case["mask"]] * vocab // 8
    logits = sum(_present(case)) * vocab * e
    return {"bytes": tables + logits * (2 if case["kind"] == "rules" else 1), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _tree(case, gen):
    """Parents, int32 [agents, nodes]: node 0 is the root, the others hang on one of the six nodes before them; the
    nodes that an agent's tree does not have say -2."""
    agents, n = case["agents"], case["nodes"]
    at = torch.arange(n, device=DEV)
    back = (torch.rand(agents, n, generator=gen, device=DEV) * at.clamp(max=6)).long() + 1
    parent = torch.where(at > 0, at - torch.minimum(back, at.clamp(min=1)), -1)
    present = torch.tensor(_present(case), device=DEV)
    return torch.where(at < present[:, None], parent, -2).int()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    t = _TYPES[case["dtype"]]
    agents, n, hkv, hq, d = (case[k] for k in ("agents", "nodes", "kv_heads", "q_heads", "head_dim"))
    s = {"case": case, "parent": _tree(case, gen), "done": _ints(_done(case)), "len": _ints(_lengths(case))}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=t)

    stride = (max(_lengths(case)) + case["reserve"] + 63) // 64 * 64
    if case["kind"] == "attention":
        # a gathered context: keys [.., tokens, D] with their rotation; values the same way in fp32, transposed in bf16
        s["kc"] = normal(agents, hkv, stride, d)
        s["vt"] = normal(agents, hkv, stride, d) if t == torch.float32 else normal(agents, hkv, d, stride)
        s["q"], s["k"], s["v"] = normal(agents, n, hq, d), normal(agents, n, hkv, d), normal(agents, n, hkv, d)
    elif case["kind"] == "commit":
        layers = case["layers"]
        s["kc"] = normal(layers, agents, hkv, stride, d)
        s["vt"] = normal(layers, agents, hkv, stride, d) if t == torch.float32 else normal(layers, agents, hkv, d, stride)
        s["k"], s["v"] = normal(layers, agents, n, hkv, d), normal(layers, agents, n, hkv, d)
        # a path of as many nodes as were accepted, ascending; the counts after the acceptance
        count = _ints(_accepted(case))
        at = torch.rand(agents, n, generator=gen, device=DEV)
        at = torch.where(torch.arange(n, device=DEV) < _ints(_present(case))[:, None], at, 2.0)
        at[:, 0] = -1.0
        nearest = at.argsort(1)
        held = torch.where(torch.arange(n, device=DEV) < count[:, None], nearest, 2 * n).sort(1).values
        s["path"] = torch.where(held < n, held, -1).int()
        s["accepted"], s["done"] = count, s["done"] + count
    else:
        vocab = case["vocab"]
        s["logits"] = normal(agents, n, vocab) * 3
        s["tokens"] = (torch.rand(agents, n, generator=gen, device=DEV) * vocab).int()
        if case["kind"] == "accept":
            # a draft model that is right about two times in three: the node's token stands out at its parent
            right = torch.rand(agents, n, generator=gen, device=DEV) < 0.65
            b, i = (right & (s["parent"] >= 0)).nonzero(as_tuple=True)
            s["logits"].index_put_((b, s["parent"][b, i].long(), s["tokens"][b, i].long()),
                                   torch.full((len(b),), 40.0, device=DEV, dtype=t), accumulate=True)
        s["penalties"] = s["history"] = s["history_len"] = s["bias"] = s["mask"] = None
        if case["history"]:
            # frequent tokens come back: the cube of a uniform number over the vocabulary
            h = case["history"]
            s["history"] = (torch.rand(agents, h, generator=gen, device=DEV) ** 3 * vocab).int()
            s["history_len"] = _ints([h - (b * 11) % (h // 2 + 1) for b in range(agents)])
            s["penalties"] = torch.rand(agents, 3, generator=gen, device=DEV) * torch.tensor([0.3, 0.2, 0.5], device=DEV)
            s["penalties"] += torch.tensor([1.0, 0.0, 0.0], device=DEV)
        if case["bias"]:
            s["bias"] = torch.randn(vocab, generator=gen, device=DEV) * 0.5
        if case["mask"] != "none":
            # half the tokens are allowed; the last node of the first agent allows none
            words = (vocab + 31) // 32
            s["mask"] = torch.randint(-2**31, 2**31, (agents, n if case["mask"] == "node" else 1, words), generator=gen, device=DEV,
                                      dtype=torch.int64).int()
            if case["mask"] == "node" and n > 1:
                s["mask"][0, -1] = 0
        s["out"] = torch.zeros_like(s["logits"]) if case["kind"] == "rules" else None
    if own:
        s["own"] = _handles(s, stride)
    return s


def _handles(s, stride):
    """What a program that uses the library keeps: the pool, the plan, the buffers."""
    from paper_2510_18546_amd import binding as B
    case = s["case"]
    agents, n = case["agents"], case["nodes"]
    h = {}
    # a pool with a group per agent; the contexts are gathered already, so that its blocks are not looked at
    cap = max(_lengths(case))
    block = torch.zeros(64, device=DEV)
    pool = B.kv_pool_create(None, None, _lengths(case), case["q_heads"], _BASE, cap + case["reserve"],
                            dtype=B.EN_F32 if case["dtype"] == "f32" else B.EN_BF16, k_ptr=block.data_ptr(), v_ptr=block.data_ptr(),
                            shape=(agents, case["kv_heads"], cap, case["head_dim"]))
    plan = B.segment_select(pool, list(range(agents)), list(range(agents + 1)), case["reserve"])
    assert plan.info.ctx_stride == stride
    h.update(pool=pool, plan=plan, block=block)
    if case["kind"] == "attention":
        h["out"] = torch.empty_like(s["q"])
        h["ws"] = torch.empty(max(256, B.tree_workspace_bytes(pool, plan, n)), dtype=torch.uint8, device=DEV)
    elif case["kind"] == "commit":
        h["kc"], h["vt"], h["k"], h["v"] = ([x for x in s[k]] for k in ("kc", "vt", "k", "v"))
    else:
        h["rules"] = B.token_rules(penalties=s["penalties"], history=s["history"], history_len=s["history_len"], bias=s["bias"],
                                   mask=s["mask"]) if case["history"] or case["bias"] or case["mask"] != "none" else None
        if case["kind"] == "accept":
            h["out"] = [torch.empty(agents, n, dtype=torch.int32, device=DEV) for _ in range(2)]
            h["out"] += [torch.empty(agents, dtype=torch.int32, device=DEV) for _ in range(3)]
            h["ws"] = torch.empty(max(256, B.tree_accept_workspace_bytes(plan, n, case["vocab"])), dtype=torch.uint8, device=DEV)
    return h


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else {"attention": _attention, "rules": _rules, "accept": _accept, "commit": _commit}[s["case"]["kind"]](s)


def _run_own(s):
    from paper_2510_18546_amd import binding as B
    h, kind = s["own"], s["case"]["kind"]
    if kind == "attention":
        return B.segmented_tree_attention(h["pool"], h["plan"], s["done"], s["parent"], s["q"], s["k"], s["v"], s["kc"], s["vt"],
                                          h["out"], h["ws"])
    if kind == "rules":
        return B.token_rules_apply(h["rules"], s["logits"], s["out"], s["parent"], s["tokens"])
    if kind == "accept":
        choice, path, accepted, token, done = h["out"]
        B.token_tree_accept(h["plan"], s["done"], s["parent"], s["tokens"], s["logits"], choice, path, accepted, token, done, h["ws"],
                            rules=h["rules"])
        return {"choice": choice, "path": path, "accepted": accepted, "next": token, "done": done}
    B.segmented_tree_commit(h["pool"], h["plan"], s["done"], s["accepted"], s["path"], h["k"], h["v"], h["kc"], h["vt"])
    return {"kc": s["kc"], "vt": s["vt"]}


def _lineage(parent, done=None, reserve=None):
    """Of trees [agents, nodes]: whether a node is present, its depth, and which nodes lie on its way from the root,
    [agents, nodes, nodes]. With `done` and `reserve` nodes past the reserve are absent too."""
    n = parent.shape[1]
    at = torch.arange(n, device=parent.device)
    linked = (parent >= 0) & (parent < at)
    up = (parent[..., None] == at) & linked[..., None]
    # powers of (1 + up) count the ways up: positive where one leads there
    reach = torch.matrix_power(torch.eye(n, dtype=torch.float64, device=parent.device) + up.double(), max(n, 1)) > 0
    present = (reach & (parent == -1)[:, None, :]).any(-1)
    depth = reach.sum(-1) - 1
    if done is not None:
        d = done[:, None].long()
        present = present & (d >= 0) & (d <= reserve) & (d + depth < reserve)
    return present, depth, reach & present[..., None]


def _turn(x, pos):
    """Rotary encoding in pairs (k, k + D/2) at positions `pos`, which lack x's last axis."""
    d = x.shape[-1]
    theta = _BASE ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    angle = pos[..., None].double() * theta
    c, s = angle.cos().to(x.dtype), angle.sin().to(x.dtype)
    x1, x2 = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1)


def _column(t):
    """Column of token t in the transposed values: bits 2 and 3 exchanged."""
    return (t & ~12) | ((t & 4) << 1) | ((t & 8) >> 1)


def _attention(s):
    case, parent = s["case"], s["parent"]
    agents, n, hkv, hq, d = (case[k] for k in ("agents", "nodes", "kv_heads", "q_heads", "head_dim"))
    r, stride = hq // hkv, s["kc"].shape[2]
    present, depth, seen = _lineage(parent, s["done"], case["reserve"])
    keys = (s["len"] + s["done"]).long()
    pos = keys[:, None] + depth
    q = _turn(s["q"].float(), pos[:, :, None]).view(agents, n, hkv, r, d).permute(0, 2, 3, 1, 4).reshape(agents, hkv, r * n, d)
    k = _turn(s["k"].float(), pos[:, :, None]).transpose(1, 2)
    v = s["v"].float().transpose(1, 2)
    vc = s["vt"].float()
    if case["dtype"] == "bf16":
        vc = vc[..., _column(torch.arange(stride, device=DEV))].transpose(-1, -2)
    low = torch.finfo(torch.float32).min
    cached = torch.arange(stride, device=DEV) < keys[:, None]
    a = torch.matmul(q, s["kc"].float().transpose(-1, -2)) / math.sqrt(d)
    a = a.masked_fill(~cached[:, None, None, :], low)
    b = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(d)
    b = b.view(agents, hkv, r, n, n).masked_fill(~seen[:, None, None], low).view(agents, hkv, r * n, n)
    top = torch.maximum(a.amax(-1, keepdim=True), b.amax(-1, keepdim=True))
    a, b = torch.exp(a - top), torch.exp(b - top)
    out = (torch.matmul(a, vc) + torch.matmul(b, v)) / (a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True))
    out = out.view(agents, hkv, r, n, d).permute(0, 3, 1, 2, 4).reshape(agents, n, hq, d)
    return torch.where(present[:, :, None, None], out, 0.0).to(s["q"].dtype)


def _ruled(s):
    """The logits in 32 bits under the rules, and the trees' present nodes."""
    x = s["logits"].float()
    agents, n, vocab = x.shape
    present, _, seen = _lineage(s["parent"])
    if s["penalties"] is not None:
        used = torch.arange(s["history"].shape[1], device=DEV) < s["history_len"][:, None]
        said = torch.zeros(agents, vocab, device=DEV).scatter_add_(1, s["history"].long(), used.float())
        count = said[:, None].repeat(1, n, 1).scatter_add_(2, s["tokens"].long()[:, None].expand(-1, n, -1), seen.float())
        rep, freq, pres = (s["penalties"][:, k, None, None] for k in range(3))
        x = torch.where(count > 0, torch.where(x > 0, x / rep, x * rep) - count * freq - pres, x)
    if s["bias"] is not None:
        x = x + s["bias"]
    if s["mask"] is not None:
        v = torch.arange(vocab, device=DEV)
        x = x.masked_fill((s["mask"][..., v >> 5] >> (v & 31)) & 1 == 0, -math.inf)
    return x, present


def _rules(s):
    x, present = _ruled(s)
    return torch.where(present[..., None], x.to(s["logits"].dtype), s["out"])


def _accept(s):
    x, _ = _ruled(s)
    present, depth, seen = _lineage(s["parent"], s["done"], s["case"]["reserve"])
    n = x.shape[1]
    at = torch.arange(n, device=DEV)
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(-1, keepdim=True)
    # the lowest of the tokens that reach the maximum
    choice = torch.where(x == top, torch.arange(x.shape[2], device=DEV), x.shape[2]).amin(-1)
    choice = torch.where(present & (top[..., 0] > -math.inf), choice, -1)
    parent, tokens = s["parent"].long(), s["tokens"].long()
    # a node is confirmed if its parent's choice is its token and no sibling before it has the same one
    twin = (parent[:, :, None] == parent[:, None, :]) & (tokens[:, :, None] == tokens[:, None, :]) & present[:, None, :]
    first = ~(twin & (at < at[:, None])).any(-1)
    confirmed = present & first & (choice.gather(1, parent.clamp(min=0)) == tokens) & (parent >= 0)
    confirmed[:, 0] = present[:, 0] & (parent[:, 0] == -1)
    on_path = present & ((seen & confirmed[:, None, :]).sum(-1) == depth + 1)
    accepted = on_path.sum(-1)
    path = torch.full((x.shape[0], n + 1), -1, device=DEV).scatter_(1, torch.where(on_path, depth, n), torch.where(on_path, at, -1))
    path = path[:, :n]
    last = path.gather(1, (accepted - 1).clamp(min=0)[:, None])
    token = torch.where(accepted > 0, choice.gather(1, last.clamp(min=0))[:, 0], -1)
    return {"choice": choice.int(), "path": path.int(), "accepted": accepted.int(), "next": token.int(),
            "done": (s["done"] + accepted).int()}


def _commit(s):
    b, j = (torch.arange(s["case"]["nodes"], device=DEV) < s["accepted"][:, None]).nonzero(as_tuple=True)
    node = s["path"][b, j].long()
    pos = s["len"][b].long() + (s["done"] - s["accepted"])[b].long() + j
    k = _turn(s["k"][:, b, node].float(), pos[None, :, None])
    v = s["v"][:, b, node]
    s["kc"][:, b, :, pos] = k.to(s["kc"].dtype).transpose(0, 1)
    if s["case"]["dtype"] == "bf16":
        s["vt"][:, b, :, :, _column(pos)] = v.transpose(0, 1)
    else:
        s["vt"][:, b, :, pos] = v.transpose(0, 1)
    return {"kc": s["kc"], "vt": s["vt"]}


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _turned64(x, pos):
    """x [.., D] in 64 bits as complex numbers, turned by pos theta_k."""
    d = x.shape[-1]
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    k = torch.arange(d // 2, device=x.device, dtype=torch.float64)
    z = z * torch.polar(torch.ones_like(k), pos * torch.exp(-2.0 * k / d * math.log(_BASE)))
    return torch.cat([z.real, z.imag], -1)


def _ways(parent, limit):
    """Of one agent's tree, for every node the nodes from the root down to it, or none where it is absent."""
    ways = []
    for i, p in enumerate(parent):
        way = [i] if p == -1 else ways[p] + [i] if 0 <= p < i and ways[p] else []
        ways.append(way if len(way) <= limit else [])
    return ways


def exact(case, seed):
    if case["kind"] == "accept":
        return None          # whole numbers only
    s = prepare(case, seed)
    lens, done, parent = s["len"].tolist(), s["done"].tolist(), s["parent"].tolist()
    if case["kind"] == "commit":
        kc, vt = s["kc"].double(), s["vt"].double()
        path = s["path"].tolist()
        for b, m in enumerate(s["accepted"].tolist()):
            for j in range(m):
                t = lens[b] + done[b] - m + j
                kc[:, b, :, t] = _turned64(s["k"][:, b, path[b][j]], t)
                value = s["v"][:, b, path[b][j]].double()
                if case["dtype"] == "f32":
                    vt[:, b, :, t] = value
                else:
                    vt[:, b, :, :, t - t % 16 + (0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15)[t % 16]] = value
        return {"kc": kc, "vt": vt}
    if case["kind"] == "rules":
        out = s["out"].double()
        for b in range(case["agents"]):
            for i, way in enumerate(_ways(parent[b], case["nodes"])):
                if not way:
                    continue
                x = s["logits"][b, i].double()
                if s["history"] is not None:
                    said = s["history"][b, :int(s["history_len"][b])].long()
                    said = torch.cat([said, s["tokens"][b, torch.tensor(way, device=DEV)].long()])
                    token, count = said.unique(return_counts=True)
                    rep, freq, pres = (float(p) for p in s["penalties"][b])
                    y = x[token]
                    x[token] = y * torch.where(y > 0, 1.0 / rep, rep) - count * freq - pres
                if s["bias"] is not None:
                    x += s["bias"].double()
                if s["mask"] is not None:
                    words = s["mask"][b, i if case["mask"] == "node" else 0]
                    bits = (words[:, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
                    x[bits.reshape(-1)[:case["vocab"]] == 0] = -math.inf
                out[b, i] = x
        return out
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    r = case["q_heads"] // case["kv_heads"]
    for b in range(case["agents"]):
        m = lens[b] + done[b]
        ways = _ways(parent[b], case["reserve"] - done[b])
        held = [i for i, way in enumerate(ways) if way]
        hidden = torch.full((len(held), case["nodes"]), -math.inf, dtype=torch.float64, device=DEV)
        for row, i in enumerate(held):
            hidden[row, ways[i]] = 0.0
        turned = {i: (_turned64(s["q"][b, i], m + len(ways[i]) - 1), _turned64(s["k"][b, i], m + len(ways[i]) - 1)) for i in held}
        none = torch.zeros(case["kv_heads"], case["head_dim"], dtype=torch.float64, device=DEV)
        for h in range(case["kv_heads"]):
            tree = torch.stack([turned[i][1][h] if i in turned else none[h] for i in range(case["nodes"])])
            keys = torch.cat([s["kc"][b, h, :m].double(), tree])
            if case["dtype"] == "f32":
                held_values = s["vt"][b, h, :m].double()
            else:
                held_values = s["vt"][b, h].double().view(case["head_dim"], -1, 2, 2, 4).transpose(2, 3).reshape(case["head_dim"], -1).t()[:m]
            values = torch.cat([held_values, s["v"][b, :, h].double()])
            if not held:
                continue
            q = torch.stack([turned[i][0][h * r:(h + 1) * r] for i in held])            # [rows, r, D]
            score = (q.reshape(-1, case["head_dim"]) @ keys.t()).view(len(held), r, -1) / math.sqrt(case["head_dim"])
            score[..., m:] += hidden[:, None]
            out[b, held, h * r:(h + 1) * r] = (torch.softmax(score, -1).view(len(held) * r, -1) @ values).view(len(held), r, -1)
    return out
