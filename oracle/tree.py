"""Float64 oracle of decoding with drafted tokens in a tree: attention along each node's way, rules on logits,
acceptance and commit, written out node by node (numpy).

TEST INFRASTRUCTURE ONLY, like the rest of this folder; nothing here imports the GPU package.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np


def ways(parent: Sequence[int], room: Optional[int] = None) -> List[List[int]]:
    """For every node its way from a root down to itself, or [] where it is absent: a parent that is neither -1 nor a
    node before it, an absent parent, or a way longer than ``room``."""
    out: List[List[int]] = []
    for i, p in enumerate(parent):
        p = int(p)
        if p == -1:
            way = [i]
        elif 0 <= p < i and out[p]:
            way = out[p] + [i]
        else:
            way = []
        out.append(way)
    return [w if room is None or len(w) <= room else [] for w in out]


def room_of(done: int, n_new: int) -> int:
    return n_new - done if 0 <= done <= n_new else 0


def rope(x: np.ndarray, pos: int, base: float) -> np.ndarray:
    d = x.shape[-1]
    angle = pos * base ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(angle), np.sin(angle)
    x = x.astype(np.float64)
    x1, x2 = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([x1 * c - x2 * s, x2 * c + x1 * s], -1)


def attention(keys, values, lens, done, n_new, parent, q, k, v, base, round_keys=lambda x: x):
    """keys, values: per agent [Hkv, tokens, D], rotated; q [B, n, Hq, D], k, v [B, n, Hkv, D] unrotated. round_keys: what a
    drafted key is held as. Returns [B, n, Hq, D]; absent nodes 0."""
    n_agents, n, hq, d = q.shape
    r = hq // k.shape[2]
    out = np.zeros(q.shape)
    with np.errstate(over="ignore", invalid="ignore"):
        for b in range(n_agents):
            length = int(lens[b]) + int(done[b])
            for i, way in enumerate(ways(parent[b], room_of(int(done[b]), n_new))):
                for h in range(hq if way else 0):
                    g = h // r
                    kk = [np.asarray(keys[b][g][:length], np.float64)]
                    kk += [round_keys(rope(k[b, m, g], length + j, base))[None] for j, m in enumerate(way)]
                    vv = [np.asarray(values[b][g][:length], np.float64)] + [v[b, m, g].astype(np.float64)[None] for m in way]
                    s = np.concatenate(kk) @ rope(q[b, i, h], length + len(way) - 1, base) / np.sqrt(d)
                    p = np.exp(s - s.max())
                    out[b, i, h] = (p / p.sum()) @ np.concatenate(vv)
    return out


def rules(logits, parent=None, tokens=None, penalties=None, history=None, history_len=None, bias=None, mask=None, out=None):
    """Logits [B, n, V] under the rules in 64 bits; rows of absent nodes come from ``out``."""
    n_agents, n, vocab = logits.shape
    res = np.array(logits if out is None else out, np.float64)
    for b in range(n_agents):
        for i, way in enumerate(ways(parent[b]) if parent is not None else [[]] * n):
            if parent is not None and not way:
                continue
            x = logits[b, i].astype(np.float64)
            if penalties is not None:
                said = [] if history is None else list(history[b][:max(0, min(int(history_len[b]), history.shape[1]))])
                said += [tokens[b][m] for m in way]
                said = np.array([t for t in said if 0 <= t < vocab], np.int64)
                c = np.bincount(said, minlength=vocab)
                rep, freq, pres = (float(p) for p in penalties[b])
                with np.errstate(over="ignore", invalid="ignore"):
                    x = np.where(c > 0, np.where(x > 0, x / rep, x * rep) - c * freq - pres, x)
            if bias is not None:
                x = x + (bias if bias.ndim == 1 else bias[b])[:vocab]
            if mask is not None:
                words = mask[b, i if mask.shape[1] > 1 else 0].view(np.uint32)
                t = np.arange(vocab)
                x = np.where(words[t // 32] >> (t % 32).astype(np.uint32) & 1, x, -np.inf)
            res[b, i] = x
    return res


def choose(x: np.ndarray) -> int:
    """The lowest of the tokens with the largest logit; NaN never; -1 where nothing is above -infinity."""
    x = np.where(np.isnan(x), -np.inf, x)
    t = int(np.argmax(x))
    return t if x[t] > -np.inf else -1


def accept(choice, done, n_new, parent, tokens):
    """Per agent (path, next token) for choices [B, n]."""
    res = []
    for b in range(len(done)):
        present = ways(parent[b], room_of(int(done[b]), n_new))
        path, token = [], -1
        at = 0 if present[0] and parent[b][0] == -1 else None
        while at is not None:
            path.append(at)
            token = int(choice[b][at])
            at = next((c for c in range(len(parent[b])) if token >= 0 and present[c] and parent[b][c] == at and tokens[b][c] == token),
                      None)
        res.append((path, token))
    return res
