"""The oracle of generation over drafted trees and of eviction, pinned against the oracle of plain generation and against
brute force; and what the library refuses before it launches anything."""
import ctypes

import numpy as np
import pytest

import oracle
from oracle import grouped, tree
from tree_cases import make


@pytest.mark.parametrize("kind", ["chain", "star", "random"])
@pytest.mark.parametrize("route", ["mixed", 0, 1])
def test_every_path_is_plain_generation(kind, route):
    """A node's output is what generation gives after its ancestors; committing a path leaves what generation leaves."""
    B, H, T, d, cap = 2, 2, 7, 8, 20
    x = make(3, B, H, T, d, [0, 1, 5, 9], cap, "f32", tree=kind, route=route)
    kw = dict(scale_la=0.4, scale_sm=1.7)
    got = tree.tree_step(x["q"], x["k"], x["v"], x["g"], x["beta"], x["route"], x["w"], x["parent"], None, x["state"],
                         x["k_cache"], x["v_cache"], x["cache_len"], **kw)

    def generate(b, nodes):
        st = [x[m][b:b + 1].astype(np.float64) for m in ("state", "k_cache", "v_cache")] + [x["cache_len"][b:b + 1].copy()]
        for i in nodes:
            ref = oracle.decode_step(*(x[m][b:b + 1, i] for m in ("q", "k", "v", "g", "beta", "route", "w")), *st, **kw)
        return ref["out"] if nodes else None, st

    for b in range(B):
        for i in range(T):
            nodes, j = [], i
            while j >= 0:
                nodes.insert(0, j)
                j = int(x["parent"][b, j])
            out, _ = generate(b, nodes)
            assert np.abs(got["out"][b, i] - out[0]).max() < 1e-12
    st = [x[m].astype(np.float64) for m in ("state", "k_cache", "v_cache")] + [x["cache_len"].copy()]
    tree.tree_commit(x["k"], x["v"], x["g"], x["beta"], x["route"], x["path"], x["n_path"], *st)
    for b in range(B):
        ref = generate(b, x["path"][b, :x["n_path"][b]].tolist())[1]
        for a, r in zip(st, ref):
            assert np.abs(a[b] - r[0]).max() < 1e-12
    # ... and the state is D S0 + sum_j D_j k_j^T u_j with the u of the tree step
    for b in range(B):
        for h in range(H):
            S = x["state"][b, h].astype(np.float64)
            for i in x["path"][b, :x["n_path"][b]]:
                S = S * np.exp(np.float64(x["g"][b, i, h])) + np.outer(x["k"][b, i, h], got["u"][b, i, h])
            assert np.abs(S - st[0][b, h]).max() < 1e-12


@pytest.mark.parametrize("G,norm", [(1, True), (2, False), (2, True)])
def test_a_chain_is_the_forward(G, norm):
    """Grouped heads and normalised q, k: a chain of tokens from an empty context, against the layer's own oracle."""
    B, H, T, d = 1, 2, 9, 16
    x = make(5, B, H, T, d, [0], 1, "f32", tree="chain", unit=False)
    kw = dict(scale_la=0.3, scale_sm=0.9, G=G, qk_norm=norm)
    got = tree.tree_step(x["q"], x["k"], x["v"], x["g"], x["beta"], x["route"], x["w"], x["parent"], None,
                         np.zeros((B, H, d, d)), x["k_cache"], x["v_cache"], x["cache_len"], **kw)
    ref = grouped.hybrid_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["route"], x["w"], **kw)
    assert np.abs(got["out"] - ref["out"]).max() < 1e-12
    fin = np.isfinite(ref["lse"])
    assert np.array_equal(fin, np.isfinite(got["lse"])) and np.abs(got["lse"][fin] - ref["lse"][fin]).max() < 1e-12
    # the weights of the whole prompt: every row that sees a key hands out one unit per softmax head
    kept = x["route"].transpose(0, 2, 1) != 0
    n = kept.sum(-1).astype(np.int32)
    kc = np.zeros((B, H, T, d))
    for b in range(B):
        for h in range(H):
            kc[b, h, :n[b, h]] = x["k"][b, kept[b, h], h]
    w = tree.cache_weights(x["q"], ref["lse"], x["route"].cumsum(1), kc, n, np.zeros((B, H, T)), scale_sm=0.9, G=G, qk_norm=norm)
    assert np.allclose(w.sum(-1), fin.sum((2, 3)), atol=1e-12)


def test_eviction_order():
    w = np.array([5.0, 1.0, 1.0, np.nan, 7.0, 1.0, -np.inf, 0.0, 9.0])
    assert tree.evict(w, 9, 9, 1, 1) == list(range(9))
    assert tree.evict(w, 9, 5, 1, 1) == [0, 1, 2, 4, 8]
    assert tree.evict(w, 9, 3, 1, 2) == [0, 7, 8]
    assert tree.evict(w, 8, 7, 0, 0) == [0, 1, 2, 4, 5, 6, 7]            # the NaN goes first
    assert tree.evict(w, 8, 6, 0, 0) == [0, 1, 2, 4, 5, 7]


# ---------------------------------------------------------------------------------------------
# Refusals: no GPU is needed, for nothing is launched
# ---------------------------------------------------------------------------------------------
A16, ODD = 1 << 20, (1 << 20) + 8                      # (never dereferenced: the calls come back before a launch)


def _params(**kw):
    from paper_2602_03681_b200 import binding, build
    build.build()
    p = binding.natsl_params()
    p.B, p.H, p.L, p.d, p.C, p.dtype, p.eps, p.scale_la, p.scale_sm, p.G = 2, 3, 16, 128, 64, 1, 1e-5, 1.0, 1.0, 1
    for n, x in kw.items():
        setattr(p, n, x)
    return binding, p


CALLS = {      # pointers (required or not), and where the integers stand
    "natsl_tree_step": [1, 1, 1, 1, 1, 1, 1, 0, 1, 1, 1, 1, "cap", 1, 0, "p", "ws", "size", 0],
    "natsl_tree_commit": [1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, "cap", "p", "ws", "size", 0],
    "natsl_cache_weights": [1, 1, 0, 1, 1, "cap", 1, "p", 0],
    "natsl_cache_evict": [1, 1, 1, 1, "cap", "keep", "first", "recent", 1, "p", 0],
}
ALIGNED = {"natsl_tree_step": [0, 1, 2, 8, 9, 10, 13, 14, 16], "natsl_tree_commit": [0, 1, 4, 7, 8, 9, 13],
           "natsl_cache_weights": [0, 3], "natsl_cache_evict": [0, 1]}


def _call(name, p_kw=None, at=None, value=None, cap=100, keep=50, first=4, recent=8, size=None):
    binding, p = _params(**(p_kw or {}))
    n = ctypes.c_size_t(0)
    lib = binding.lib()
    lib.natsl_workspace_size(ctypes.byref(p), binding.OP_TREE, ctypes.byref(n))
    args = []
    for i, a in enumerate(CALLS[name]):
        x = {"cap": ctypes.c_int32(cap), "keep": ctypes.c_int32(keep), "first": ctypes.c_int32(first), "recent": ctypes.c_int32(recent),
             "p": ctypes.byref(p), "ws": ctypes.c_void_p(A16), "size": ctypes.c_size_t(n.value if size is None else size)}.get(
                 a, ctypes.c_void_p(A16 if a else 0))
        args.append(ctypes.c_void_p(value) if i == at else x)
    return getattr(lib, name)(*args)


@pytest.mark.parametrize("name", CALLS)
def test_refusals(name):
    for i, a in enumerate(CALLS[name]):
        if a == 1:
            assert _call(name, at=i, value=0) == -1, i
    for i in ALIGNED[name]:
        assert _call(name, at=i, value=ODD) == -4, i
    if "ws" in CALLS[name]:
        assert _call(name, at=CALLS[name].index("ws"), value=0) == -5
        assert _call(name, size=255) == -5
    for bad in (dict(B=0), dict(H=-1), dict(d=96), dict(C=32), dict(eps=0.0), dict(G=3), dict(G=-1)):
        assert _call(name, bad) in ((-2, -8) if "G" in bad and bad["G"] > 0 else (-2,)), bad
    if name != "natsl_cache_evict":
        assert _call(name, dict(L=0)) == -2
        assert name == "natsl_tree_commit" or _call(name, dict(d=64, G=4)) == -8
        assert _call(name, dict(flags=128, norm_eps=-1.0)) == -2
    if "tree" in name:
        assert _call(name, dict(L=65)) == -2
    assert _call(name, dict(dtype=5)) == -3
    for cap in (0, -3):
        assert _call(name, cap=cap) == -2


def test_refusals_of_an_eviction():
    for bad in (dict(keep=0), dict(keep=101), dict(first=-1), dict(recent=-1), dict(first=43), dict(recent=2 ** 31 - 1)):
        assert _call("natsl_cache_evict", **bad) == -2, bad


def test_workspace_of_a_tree():
    binding, p = _params()
    p.L = 64
    assert binding.natsl_workspace_size(p, binding.OP_TREE) >= 256
    p.L = 65
    with pytest.raises(binding.NatslError):
        binding.natsl_workspace_size(p, binding.OP_TREE)
    assert "tree" in binding.natsl_strerror(binding.ERR_TREE)
