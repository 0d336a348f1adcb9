"""Inputs of the tests of generation over drafted trees: seeded, with the shapes and routes that a case names."""
import numpy as np

from paper_2602_03681_b200 import inputs


def random_tree(rng, B, T, kind="random"):
    """parent [B,T]: "chain", "star" (every node a child of the context) or "random" (children of one of the last nodes)."""
    par = np.empty((B, T), np.int32)
    for b in range(B):
        for i in range(T):
            par[b, i] = i - 1 if kind == "chain" else -1 if kind == "star" else max(-1, i - 1 - int(rng.exponential(2.5)))
    return par


def paths(rng, parent, n_nodes=None):
    """A path from the context to some node of each tree: path [B,T] (-1 behind its end), n_path [B]."""
    B, T = parent.shape
    path, n = np.full((B, T), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        last = T if n_nodes is None else int(n_nodes[b])
        i = int(rng.integers(0, last)) if last else -1
        p = []
        while i >= 0:
            p.insert(0, i)
            i = int(parent[b, i])
        path[b, :len(p)], n[b] = p, len(p)
    return path, n


def make(seed, B, H, T, d, lengths, cap, dtype, *, tree="random", route="mixed", unit=True, nodes=None):
    """numpy inputs of one tree step.  route: "mixed" (0 and 1), "all" (0, 1 and 2), or a number for every token.  unit: unit-norm
    q and k (otherwise rows of very different lengths, for the normalisation inside)."""
    rng = np.random.default_rng(seed)

    def rows(*s):
        x = rng.standard_normal(s)
        x = x / np.linalg.norm(x, axis=-1, keepdims=True) if unit else x * np.exp(0.7 * rng.standard_normal((*s[:-1], 1)))
        return inputs.round_bf16(x.astype(np.float32)) if dtype == "bf16" else x.astype(np.float32)

    def values(*s):
        x = rng.standard_normal(s).astype(np.float32)
        return inputs.round_bf16(x) if dtype == "bf16" else x

    n = rng.permutation(np.resize(np.asarray(lengths, np.int32), B * H)).reshape(B, H).astype(np.int32)
    x = dict(q=rows(B, T, H, d), k=rows(B, T, H, d), v=values(B, T, H, d), k_cache=rows(B, H, cap, d), v_cache=values(B, H, cap, d))
    x["g"] = -np.log1p(np.exp(rng.standard_normal((B, T, H)))).astype(np.float32)
    x["beta"] = (1 / (1 + np.exp(-rng.standard_normal((B, T, H))))).astype(np.float32)
    x["w"] = rng.dirichlet((1.0, 1.0), (B, T, H)).astype(np.float32)
    x["state"] = (0.3 * rng.standard_normal((B, H, d, d))).astype(np.float32)
    if route == "mixed":
        x["route"] = rng.integers(0, 2, (B, T, H)).astype(np.uint8)
    elif route == "all":
        x["route"] = rng.integers(0, 3, (B, T, H)).astype(np.uint8)
    else:
        x["route"] = np.full((B, T, H), int(route), np.uint8)
    x["parent"] = random_tree(rng, B, T, tree)
    x["n_nodes"] = None if nodes is None else np.resize(np.asarray(nodes, np.int32), B).astype(np.int32)
    x["cache_len"] = n
    x["path"], x["n_path"] = paths(rng, x["parent"], x["n_nodes"])
    return x
