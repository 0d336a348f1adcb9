"""Generation over drafted trees (natsl_tree_step, natsl_tree_commit) against the fp64 oracle.

Tolerances, from the arithmetic:
* fp32 storage, and every fp32 result: sums of at most 64 + 700 terms and products of at most 128 columns in fp32, whose
  relative error stays below 128 * 2^-24 = 8e-6 per sum, through paths of at most 64 nodes: 1e-4 of the RMS, the project's
  bound for fp32.
* bf16 storage, `out`: the probabilities that meet V on the tensor cores are rounded to bf16, each off by at most 2^-8 of
  itself and independently of the others: a standard deviation of at most 2^-8 / sqrt(3) = 2.3e-3 of the branch's RMS, of
  which 2e-2, the project's bound for bf16, is more than six (weights of at most one); storing adds half an ulp
  (check_stored).
* log-sum-exp: logits of at most 12 in magnitude, each a sum of 128 products in fp32: 12 * 128 * 2^-24 = 9.2e-5."""
import numpy as np
import pytest
import torch

from oracle import tree
from test_gpu_parity import TOL, check_stored, dev, rel_err
from tree_cases import make

pytestmark = pytest.mark.gpu

LENGTHS = [0, 1, 31, 32, 33, 63, 64, 65, 127, 129, 255, 300, 513, 600]
SENTINEL = 768.0                                    # (exact in bf16)


def scales(d, G, norm):
    return d ** -0.5, (d // G) ** -0.5 if norm else d ** 0.5


def upload(x, dtype):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    return {n: None if a is None else dev(a, dt if n in ("q", "k", "v", "k_cache", "v_cache") else None) for n, a in x.items()}


def call(x, dtype, *, G=1, norm=False, flags=0, norm_eps=1e-6, w=True, want_u=True, want_lse=True):
    """One natsl_tree_step: dict of device tensors (out, u, lse, inputs, p, ws)."""
    from paper_2602_03681_b200 import binding
    t = upload(x, dtype)
    B, T, H, d = x["q"].shape
    la, sm = scales(d, G, norm)
    out = torch.full_like(t["q"], SENTINEL)
    u = torch.full((B, T, H, d), SENTINEL, device="cuda") if want_u else None
    lse = torch.full((B, H, G, T) if G > 1 else (B, H, T), SENTINEL, device="cuda") if want_lse else None
    p = binding.make_params(B, H, T, d, binding._dtype_code(t["q"]), la, sm, flags=flags | (binding.QK_NORM if norm else 0),
                            w=t["w"] if w else None, lse=lse, G=G, norm_eps=norm_eps)
    ws = binding.alloc_workspace(p, binding.OP_TREE)
    t.update(out=out, u=u, lse=lse, p=p, ws=ws)
    step(t)
    return t


def step(t):
    from paper_2602_03681_b200 import binding
    binding.natsl_tree_step(t["q"], t["k"], t["v"], t["g"], t["beta"], t["route"], t["parent"], t["n_nodes"], t["state"],
                            t["k_cache"], t["v_cache"], t["cache_len"], t["out"], t["u"], t["p"], t["ws"])


def reference(x, G=1, norm=False, w=True, norm_eps=1e-6):
    la, sm = scales(x["q"].shape[-1], G, norm)
    return tree.tree_step(x["q"], x["k"], x["v"], x["g"], x["beta"], x["route"], x["w"] if w else None, x["parent"], x["n_nodes"],
                          x["state"], x["k_cache"], x["v_cache"], x["cache_len"], scale_la=la, scale_sm=sm, G=G, qk_norm=norm,
                          norm_eps=norm_eps)


def check(t, ref, dtype, status=0):
    from paper_2602_03681_b200 import binding
    assert binding.natsl_device_status(t["ws"]) == status
    live = np.isfinite(ref["u"][..., 0])            # rows behind a tree's last node: as they were
    out = t["out"].float().cpu().numpy()
    assert (out[~live] == SENTINEL).all()
    if live.any():
        check_stored(out[live], ref["out"][live], TOL[dtype], dtype)
    if t["u"] is not None:
        u = t["u"].cpu().numpy()
        assert (u[~live] == SENTINEL).all()
        if live.any() and ref["u"][live].any():
            assert rel_err(u[live], ref["u"][live]) <= 1e-4
    if t["lse"] is not None:
        lse = t["lse"].cpu().numpy().reshape(ref["lse"].shape)
        dead = np.broadcast_to(~live.transpose(0, 2, 1)[:, :, None], lse.shape)
        assert (lse[dead] == SENTINEL).all()
        none = np.isneginf(ref["lse"])
        assert np.array_equal(np.isneginf(lse), none)
        fin = ~dead & ~none
        if fin.any():
            assert np.abs(lse[fin] - ref["lse"][fin]).max() <= 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,kind,route", [(1, "random", "all"), (2, "chain", "mixed"), (3, "star", "mixed"), (7, "random", 2),
                                          (15, "random", "mixed"), (16, "chain", "all"), (17, "random", "all"), (31, "random", 1),
                                          (32, "star", "all"), (33, "chain", "mixed"), (47, "random", 2), (48, "random", 0),
                                          (63, "random", "all"), (64, "chain", "all"), (64, "random", "mixed")])
def test_sizes_and_trees(dtype, T, kind, route):
    x = make(T, 2, 7, T, 128, LENGTHS, 613, dtype, tree=kind, route=route)
    check(call(x, dtype), reference(x), dtype)


@pytest.mark.parametrize("dtype,d,G,norm,flags", [
    ("f32", 64, 1, False, 0), ("f32", 64, 2, True, 0), ("f32", 128, 4, True, 0), ("f32", 128, 2, False, 0),
    ("bf16", 64, 1, False, 0), ("bf16", 64, 1, True, 0), ("bf16", 64, 2, False, 0), ("bf16", 64, 2, True, 0),
    ("bf16", 128, 1, True, 0), ("bf16", 128, 2, False, 0), ("bf16", 128, 2, True, 0), ("bf16", 128, 4, True, 0),
    ("bf16", 128, 4, False, 0), ("bf16", 128, 1, False, 1), ("bf16", 128, 2, True, 1), ("bf16", 64, 1, True, 1)])
@pytest.mark.parametrize("T", [5, 19, 50])
def test_heads_and_normalisation(dtype, d, G, norm, flags, T):
    x = make(T + d + G, 2, 3, T, d, [0, 1, 65, 200, 413, 64], 413, dtype, route="all", unit=not norm)
    check(call(x, dtype, G=G, norm=norm, flags=flags), reference(x, G, norm), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H", [(1, 1), (1, 16), (9, 11), (25, 12), (40, 16)])
def test_numbers_of_pairs(dtype, B, H):
    """A pair's cache is cut by the number of pairs: few, many, and every length."""
    x = make(B, B, H, 4, 64, LENGTHS, 600, dtype, route="mixed")
    check(call(x, dtype), reference(x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_cache(dtype):
    x = make(1, 1, 2, 21, 128, [5000, 4097], 5000, dtype)
    check(call(x, dtype), reference(x), dtype)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,norm", [(1, False), (1, True), (2, False), (2, True)])
@pytest.mark.parametrize("T,cluster", [(33, 8), (64, 4), (49, 2)])
def test_full_trees_over_long_caches(d, G, norm, T, cluster):
    """33 to 64 nodes: several turns of the ring, every number of tiles modulo its places, one to eight CTAs' shares."""
    B, H = {8: (1, 9), 4: (3, 10), 2: (6, 10)}[cluster]
    lengths = [1800, 0, 1, 63, 64, 65, 640, 704, 768, 832, 896, 960, 1024, 1088, 1151, 1153, 1799, 17, 700]
    x = make(T + G, B, H, T, d, lengths, 1800, "bf16", route="all", unit=not norm)
    check(call(x, "bf16", G=G, norm=norm), reference(x, G, norm), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weights_of_the_branches_at_any_address(dtype):
    """p->w is an fp32 array like the others: nothing but its elements' alignment is asked for."""
    from paper_2602_03681_b200 import binding
    x = make(12, 2, 3, 9, 64, [0, 30, 77], 80, dtype)
    t = call(x, dtype)
    first = t["out"].clone()
    shifted = torch.empty(t["w"].numel() + 1, device="cuda")[1:].view_as(t["w"])
    shifted.copy_(t["w"])
    B, T, H, d = x["q"].shape
    la, sm = scales(d, 1, False)
    t["p"] = binding.make_params(B, H, T, d, binding._dtype_code(t["q"]), la, sm, w=shifted, lse=t["lse"])
    t["out"].fill_(SENTINEL)
    step(t)
    assert torch.equal(t["out"], first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nodes", [[0, 5], [13, 1, 7], [0, 0]])
def test_ragged_trees(dtype, nodes):
    """Rows behind a tree's last node are neither read nor written, whatever they hold."""
    x = make(2, len(nodes), 3, 13, 128, [0, 70, 3], 80, dtype, route="all", nodes=nodes)
    for b, n in enumerate(nodes):
        for m in ("q", "k", "v", "g", "beta"):
            x[m][b, n:] = np.nan
        x["parent"][b, n:] = 99
        x["route"][b, n:] = 2
    check(call(x, dtype), reference(x), dtype)


@pytest.mark.parametrize("dtype,G,d", [("f32", 1, 128), ("bf16", 1, 128), ("bf16", 2, 128), ("bf16", 1, 64), ("bf16", 2, 64)])
@pytest.mark.parametrize("T", [12, 40])
def test_nothing_leaks(dtype, G, d, T):
    """NaN and infinities in what a node does not see -- cache rows behind the length, nodes off its path, V of nodes that are
    not retained and K of its softmax -- reach no output."""
    x = make(4, 2, 2, T, d, [0, 5, 66, 190], 200, dtype, route="mixed", tree="random")
    for b in range(2):
        for h in range(2):
            x["k_cache"][b, h, x["cache_len"][b, h]:] = np.nan
            x["v_cache"][b, h, x["cache_len"][b, h]:] = np.inf
    clean = call(x, dtype, G=G)
    bad = 3                                          # this node and its descendants are spoilt, nobody else
    spoilt = np.zeros((2, T), bool)
    for b in range(2):
        for i in range(T):
            spoilt[b, i] = i == bad or (x["parent"][b, i] >= 0 and spoilt[b, x["parent"][b, i]])
    y = dict(x, k=x["k"].copy(), v=x["v"].copy(), q=x["q"].copy())
    y["k"][:, bad], y["v"][:, bad], y["q"][:, bad] = np.nan, np.inf, -np.inf
    got = call(y, dtype, G=G)
    ok = torch.from_numpy(~spoilt).cuda()
    for m in ("out", "u"):
        assert torch.equal(got[m][ok], clean[m][ok]) and torch.isfinite(got[m][ok]).all()
    check(clean, reference(x, G), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_of_zero_and_one(dtype):
    """g = -inf wipes the state for the node and what follows it, g = 0 leaves it."""
    x = make(6, 1, 2, 20, 64, [40], 40, dtype, route="all", tree="chain")
    x["g"][:, ::5] = -np.inf
    x["g"][:, 1::5] = 0.0
    check(call(x, dtype), reference(x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_visible_and_optional_arguments(dtype):
    """Linear tokens over an empty cache: log-sum-exp -inf, the softmax branch zero; no u, no lse, no weights."""
    x = make(8, 1, 3, 9, 64, [0], 10, dtype, route=0)
    t = call(x, dtype)
    assert torch.isneginf(t["lse"]).all()
    check(t, reference(x), dtype)
    check(call(x, dtype, w=False, want_u=False, want_lse=False), reference(x, w=False), dtype)


@pytest.mark.parametrize("T", [6, 50])
def test_large_logits(T):
    """Logits of several hundred: the running maximum keeps exponentials in range."""
    for dtype in ("f32", "bf16"):
        x = make(9, 1, 2, T, 128, [200, 77], 200, dtype)
        x["q"] *= 32
        ref = reference(x)
        t = call(x, dtype, want_lse=False)
        # (a logit of 360 carries up to 360 * 128 * 2^-24 = 2.7e-3, and so does the probability it gives)
        check_stored(t["out"].float().cpu().numpy(), ref["out"], 2e-2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_a_tree_is_reported(dtype):
    from paper_2602_03681_b200 import binding
    x = make(10, 2, 2, 6, 64, [3, 9], 9, dtype)
    ref = reference(x)
    for parent, nodes, length, status in ((4, None, None, binding.ERR_TREE), (-2, None, None, binding.ERR_TREE),
                                          (None, 7, None, binding.ERR_TREE), (None, -1, None, binding.ERR_TREE),
                                          (None, None, 10, binding.ERR_CACHE_FULL), (None, None, -5, binding.ERR_CACHE_FULL)):
        y = dict(x, parent=x["parent"].copy(), cache_len=x["cache_len"].copy())
        z = dict(x, parent=x["parent"].copy(), cache_len=x["cache_len"].copy())
        if parent is not None:
            y["parent"][0, 4], z["parent"][0, 4] = parent, -1
        if nodes is not None:
            y["n_nodes"], z["n_nodes"] = np.array([nodes, 6], np.int32), np.array([max(0, min(6, nodes)), 6], np.int32)
        if length is not None:
            y["cache_len"][0, 0], z["cache_len"][0, 0] = length, max(0, min(9, length))
        check(call(y, dtype), reference(z), dtype, status)
    check(call(x, dtype), ref, dtype)


def test_logits_that_grow_along_the_cache():
    """Every tile raises the running maximum by more than the sums' slack, so that all sums are rescaled again and again."""
    for T, G, d in ((9, 1, 128), (40, 1, 128), (40, 2, 128), (9, 1, 64), (40, 1, 64), (40, 2, 64)):
        x = make(T, 1, 2, T, d, [900, 641], 900, "bf16", unit=True)
        # keys along the first nodes' mean direction, longer from tile to tile: logits grow to about 100
        x["q"][:] = x["q"][:, :1]
        ramp = np.linspace(0.0, 8.0, 900)[:, None]
        x["k_cache"] = (ramp * x["q"][:, 0][:, :, None, :]).astype(np.float32)
        x["k_cache"] = torch.from_numpy(x["k_cache"]).bfloat16().float().numpy().astype(x["v_cache"].dtype)
        ref = reference(x, G)
        t = call(x, "bf16", G=G, want_lse=False)
        # (a logit of 91 carries up to 91 * 128 * 2^-24 = 7e-4, and so does the probability it gives)
        check_stored(t["out"].float().cpu().numpy(), ref["out"], TOL["bf16"], "bf16")


@pytest.mark.parametrize("dtype,G,norm,T", [("f32", 1, False, 24), ("bf16", 1, False, 24), ("bf16", 2, True, 24), ("bf16", 1, False, 64),
                                            ("bf16", 2, True, 64)])
def test_results_do_not_depend_on_who_finishes_last(dtype, G, norm, T):
    x = make(11, 4, 8, T, 128, LENGTHS, 600, dtype, unit=not norm)
    t = call(x, dtype, G=G, norm=norm)
    first = [t[m].clone() for m in ("out", "u", "lse")]
    for _ in range(20):
        step(t)
        assert all(torch.equal(t[m], f) for m, f in zip(("out", "u", "lse"), first))


# ---------------------------------------------------------------------------------------------
# The accepted path
# ---------------------------------------------------------------------------------------------
def commit(t, x):
    from paper_2602_03681_b200 import binding
    binding.natsl_tree_commit(t["k"], t["v"], t["g"], t["route"], t["u"], t["path"], t["n_path"], t["state"], t["k_cache"],
                              t["v_cache"], t["cache_len"], t["p"], t["ws"])


def check_commit(t, x, norm=False, status=0):
    from paper_2602_03681_b200 import binding
    assert binding.natsl_device_status(t["ws"]) == status
    st = [x[m].astype(np.float64) for m in ("state", "k_cache", "v_cache")] + [x["cache_len"].copy()]
    tree.tree_commit(x["k"], x["v"], x["g"], x["beta"], x["route"], x["path"], x["n_path"], *st, qk_norm=norm)
    assert np.array_equal(t["cache_len"].cpu().numpy(), st[3])
    assert np.array_equal(t["k_cache"].double().cpu().numpy(), st[1])
    assert np.array_equal(t["v_cache"].double().cpu().numpy(), st[2])
    assert rel_err(t["state"].cpu().numpy(), st[0]) <= 1e-4


@pytest.mark.parametrize("dtype,d,norm", [("f32", 64, False), ("f32", 128, True), ("bf16", 64, True), ("bf16", 128, False)])
@pytest.mark.parametrize("T,kind,route", [(1, "random", "all"), (6, "random", "mixed"), (33, "random", "all"), (64, "chain", "all"),
                                          (64, "chain", 1), (9, "star", 0)])
def test_commit(dtype, d, norm, T, kind, route):
    x = make(T, 3, 5, T, d, [0, 1, 40], 110, dtype, tree=kind, route=route, unit=not norm)
    if kind == "chain":
        x["path"][0], x["n_path"][0] = np.arange(T), T
    x["n_path"][1] = 0
    t = call(x, dtype, norm=norm)
    commit(t, x)
    check_commit(t, x, norm)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_commit_without_room_or_without_a_path(dtype):
    """A full cache leaves its pair alone, a path that does not climb its sequence."""
    from paper_2602_03681_b200 import binding
    x = make(3, 3, 4, 8, 64, [10, 16, 13, 15], 16, dtype, tree="chain", route="mixed")
    x["path"][:], x["n_path"][:] = np.arange(8), 5
    t = call(x, dtype)
    commit(t, x)
    check_commit(t, x, status=binding.ERR_CACHE_FULL)
    x["cache_len"][:] = 2
    for path, n in (([0, 2, 2, 3], 4), ([3, 1], 2), ([-1], 1), ([0, 8], 2), ([-7, 0], 2), ([0], 9), ([0], -1)):
        y = dict(x, path=x["path"].copy(), n_path=x["n_path"].copy())
        y["path"][1, :len(path)], y["n_path"][1] = path, n
        t = call(y, dtype)
        commit(t, y)
        y["n_path"][1] = 0                           # (for the oracle: that sequence accepts nothing)
        check_commit(t, y, status=binding.ERR_TREE)


@pytest.mark.parametrize("dtype,G,norm", [("f32", 1, False), ("bf16", 1, False), ("bf16", 2, True), ("f32", 4, True)])
def test_step_and_commit_are_generation(dtype, G, norm):
    """The same tokens through natsl_decode_step one at a time: outputs, state, cache and length."""
    from paper_2602_03681_b200 import binding
    B, H, T, d = 2, 3, 11, 128
    x = make(21, B, H, T, d, [0, 64, 130], 160, dtype, tree="random", route="all", unit=not norm)
    t = call(x, dtype, G=G, norm=norm)
    commit(t, x)
    ref = upload(x, dtype)
    la, sm = scales(d, G, norm)
    for b in range(B):
        one = {m: ref[m][b:b + 1].contiguous() for m in ("state", "k_cache", "v_cache", "cache_len")}
        for i in x["path"][b, :x["n_path"][b]]:
            row = {m: ref[m][b:b + 1, i].contiguous() for m in ("q", "k", "v", "g", "beta", "route", "w")}
            p = binding.make_params(1, H, 0, d, binding._dtype_code(row["q"]), la, sm, flags=binding.QK_NORM if norm else 0, w=row["w"],
                                    G=G, norm_eps=1e-6 if norm else 0.0)
            out = torch.empty_like(row["q"])
            binding.natsl_decode_step(row["q"], row["k"], row["v"], row["g"], row["beta"], row["route"], one["state"], one["k_cache"],
                                      one["v_cache"], one["cache_len"], out, p, binding.alloc_workspace(p, binding.OP_DECODE))
            check_stored(t["out"][b, i].float().cpu().numpy(), out[0].double().cpu().numpy(), TOL[dtype], dtype, large_only=False)
        assert torch.equal(one["cache_len"][0], t["cache_len"][b])
        assert torch.equal(one["k_cache"][0], t["k_cache"][b]) and torch.equal(one["v_cache"][0], t["v_cache"][b])
        assert rel_err(t["state"][b].cpu().numpy(), one["state"][0].cpu().numpy()) <= 1e-4


@pytest.mark.parametrize("dtype,T", [("f32", 10), ("bf16", 10), ("bf16", 45)])
def test_captured_and_on_another_stream(dtype, T):
    """Step and commit in a CUDA graph, replayed on new contents; two graphs that share a workspace, one after the other; a
    stream that is not the default one."""
    x = make(31, 2, 4, T, 128, [5, 70, 200, 0], 260, dtype, route="all")
    t = call(x, dtype)
    eager = [t[m].clone() for m in ("out", "u", "lse")]
    start = [t[m].clone() for m in ("state", "k_cache", "v_cache", "cache_len")]
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for _ in range(2):
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=side):
                step(t)
                commit(t, x)
            graphs.append(gr)
    torch.cuda.synchronize()
    for rep in range(4):
        for m, s in zip(("state", "k_cache", "v_cache", "cache_len"), start):
            t[m].copy_(s)
        for m in ("out", "u", "lse"):
            t[m].fill_(SENTINEL)
        torch.cuda.synchronize()
        graphs[rep % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t[m], e) for m, e in zip(("out", "u", "lse"), eager))
        check_commit(t, x)
    for m, s in zip(("state", "k_cache", "v_cache", "cache_len"), start):
        t[m].copy_(s)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(t)
        commit(t, x)
    side.synchronize()
    assert all(torch.equal(t[m], e) for m, e in zip(("out", "u", "lse"), eager))
    check_commit(t, x)


def test_beside_other_users_of_tensor_memory():
    """Full trees, cache weights and the prompt's forward, on three streams at once, each with a workspace of its own."""
    from paper_2602_03681_b200 import binding
    x = make(41, 4, 8, 64, 128, [600, 5, 333, 64], 700, "bf16")
    t = call(x, "bf16")
    B, T, H, d = x["q"].shape
    la, sm = scales(d, 1, False)
    weight = torch.zeros(B, H, 700, device="cuda")
    pw = binding.make_params(B, H, T, d, binding._dtype_code(t["q"]), la, sm)
    L = 512
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(1, L, 4, d, device="cuda", generator=gen) for _ in range(3))
    q, k, v = (torch.nn.functional.normalize(y, dim=-1).bfloat16() for y in (q, k, v))
    g, beta = -torch.rand(1, L, 4, device="cuda", generator=gen), torch.rand(1, L, 4, device="cuda", generator=gen)
    route = (torch.rand(1, L, 4, device="cuda", generator=gen) < 0.3).to(torch.uint8)
    out = torch.empty_like(q)
    pf = binding.make_params(1, 4, L, d, binding._dtype_code(q), la, sm)
    wf = binding.alloc_workspace(pf, binding.OP_FWD)

    def weights():
        binding.natsl_cache_weights(t["q"], t["lse"], None, t["k_cache"], t["cache_len"], weight, pw)

    def forward():
        binding.natsl_hybrid_fwd(q, k, v, g, beta, route, out, pf, wf)

    want = [t[m].clone() for m in ("out", "u")]
    weights()
    forward()
    torch.cuda.synchronize()
    once, fwd = weight.clone(), out.clone()
    weight.zero_()
    lse = t["lse"].clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        with torch.cuda.stream(streams[0]):
            step(t)
        with torch.cuda.stream(streams[1]):
            weight.zero_()
            binding.natsl_cache_weights(t["q"], lse, None, t["k_cache"], t["cache_len"], weight, pw)
        with torch.cuda.stream(streams[2]):
            forward()
    torch.cuda.synchronize()
    assert all(torch.equal(t[m], y) for m, y in zip(("out", "u"), want))
    assert torch.equal(weight, once) and torch.equal(out, fwd)
    assert binding.natsl_device_status(t["ws"]) == 0 and binding.natsl_device_status(wf) == 0


@pytest.mark.parametrize("dtype,T", [("f32", 12), ("bf16", 12), ("bf16", 40)])
@pytest.mark.parametrize("g", [-95.0, -200.0, -1e9, -1e30, float(np.finfo(np.float32).min)])
@pytest.mark.parametrize("times", [1, 2])
def test_decays_that_are_zero_in_fp32(dtype, T, g, times):
    """A finite g whose decay is zero in fp32 (a masked gate, say), once and twice on a path: what comes behind it decays by its own
    g, as in natsl_decode_step, which multiplies the state by exp(g) token by token."""
    x = make(16, 1, 2, T, 64, [40, 0], 40, dtype, route="all", tree="chain")
    x["g"][:, [3, 6][:times]] = g
    check(call(x, dtype), reference(x), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decay_to_nothing_and_generation(dtype):
    """The same through natsl_decode_step: the step's outputs and the committed state."""
    from paper_2602_03681_b200 import binding
    H, T, d = 2, 9, 64
    x = make(17, 1, H, T, d, [20, 0], 40, dtype, route=0, tree="chain")
    x["g"][:, 2], x["g"][:, 5] = -1e30, np.finfo(np.float32).min
    x["path"][0], x["n_path"][0] = np.arange(T), T
    t = call(x, dtype)
    commit(t, x)
    ref = upload(x, dtype)
    la, sm = scales(d, 1, False)
    for i in range(T):
        row = {m: ref[m][:, i].contiguous() for m in ("q", "k", "v", "g", "beta", "route", "w")}
        p = binding.make_params(1, H, 0, d, binding._dtype_code(row["q"]), la, sm, w=row["w"])
        out = torch.empty_like(row["q"])
        binding.natsl_decode_step(row["q"], row["k"], row["v"], row["g"], row["beta"], row["route"], ref["state"], ref["k_cache"],
                                  ref["v_cache"], ref["cache_len"], out, p, binding.alloc_workspace(p, binding.OP_DECODE))
        check_stored(t["out"][0, i].float().cpu().numpy(), out[0].double().cpu().numpy(), TOL[dtype], dtype, large_only=False)
    assert rel_err(t["state"].cpu().numpy(), ref["state"].cpu().numpy()) <= 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [-5, -2 ** 31, 17, 2 ** 31 - 1])
@pytest.mark.parametrize("route", [0, "mixed"])
def test_commit_to_a_length_out_of_range(dtype, length, route):
    """Reported, and nothing of the pair is written, whether or not its path retains a token: with the length put right the
    same commit does what it always does."""
    from paper_2602_03681_b200 import binding
    x = make(5, 2, 2, 8, 64, [3, 5, 0, 7], 16, dtype, tree="chain", route=route)
    x["path"][:], x["n_path"][:] = np.arange(8), 5
    t = call(x, dtype)
    right = t["cache_len"].clone()
    t["cache_len"][1, 0] = length
    before = [t[m][1, 0].clone() for m in ("state", "k_cache", "v_cache", "cache_len")]
    commit(t, x)
    assert binding.natsl_device_status(t["ws"]) == binding.ERR_CACHE_FULL
    assert all(torch.equal(t[m][1, 0], y) for m, y in zip(("state", "k_cache", "v_cache", "cache_len"), before))
    one = {m: t[m][1:, :1].contiguous() for m in ("state", "k_cache", "v_cache")}
    one["cache_len"] = right[1:, :1].contiguous()
    for m in ("k", "v", "g", "route", "u"):
        one[m] = t[m][1:, :, :1].contiguous()
    one["path"], one["n_path"] = t["path"][1:].contiguous(), t["n_path"][1:].contiguous()
    one["p"] = binding.make_params(1, 1, 8, 64, binding._dtype_code(t["k"]), 1.0, 1.0)
    one["ws"] = t["ws"]
    commit(one, x)
    for m in ("state", "k_cache", "v_cache", "cache_len"):
        t[m][1:, :1] = one[m]
    check_commit(t, x)


@pytest.mark.parametrize("dtype,G,norm,T", [("f32", 1, True, 6), ("f32", 4, True, 6), ("bf16", 4, True, 6), ("bf16", 2, True, 6),
                                            ("bf16", 2, True, 40), ("f32", 1, False, 6), ("bf16", 1, False, 40)])
@pytest.mark.parametrize("sm", [0.0, 1e-23, -0.3])
def test_any_logit_scale(dtype, G, norm, T, sm, monkeypatch):
    """Zero (every visible key counts the same), one whose square is zero, and a negative one."""
    import test_gpu_tree
    monkeypatch.setattr(test_gpu_tree, "scales", lambda d, G, norm: (d ** -0.5, sm))
    x = make(3, 1, 2, T, 128, [50, 3], 50, dtype, route="all", unit=not norm)
    check(call(x, dtype, G=G, norm=norm), reference(x, G, norm), dtype)


@pytest.mark.parametrize("d,G", [(128, 1), (128, 2), (64, 1)])
@pytest.mark.parametrize("T", [33, 64])
def test_full_trees_one_behind_the_other(d, G, T):
    """More pairs than are resident at once over long caches of every length modulo the tile, two batches in turns and nothing waited
    for between them: the same bits as alone.  Behind the lengths lies what may not be seen."""
    from paper_2602_03681_b200 import binding
    B, H, cap = 8, 16, 4000
    dev_gen = torch.Generator(device="cuda").manual_seed(T + d + G)
    la, sm = scales(d, G, False)

    def batch():
        def rows(*s):
            return torch.nn.functional.normalize(torch.randn(s, generator=dev_gen, device="cuda"), dim=-1).bfloat16()
        t = dict(q=rows(B, T, H, d), k=rows(B, T, H, d), v=rows(B, T, H, d), k_cache=rows(B, H, cap, d), v_cache=rows(B, H, cap, d))
        t["g"], t["beta"] = -torch.rand(B, T, H, generator=dev_gen, device="cuda"), torch.rand(B, T, H, generator=dev_gen, device="cuda")
        t["route"] = torch.randint(0, 3, (B, T, H), generator=dev_gen, device="cuda").to(torch.uint8)
        t["parent"] = (torch.arange(T, device="cuda", dtype=torch.int32) - 2).clamp(min=-1).repeat(B, 1)
        t["state"] = torch.randn(B, H, d, d, generator=dev_gen, device="cuda")
        t["cache_len"] = (cap - torch.randint(0, cap // 2, (B, H), generator=dev_gen, device="cuda")).to(torch.int32)
        behind = torch.arange(cap, device="cuda") >= t["cache_len"][:, :, None]
        t["k_cache"][behind], t["v_cache"][behind] = float("inf"), float("nan")
        t["n_nodes"], t["out"], t["u"] = None, torch.empty_like(t["q"]), torch.empty(B, T, H, d, device="cuda")
        t["lse"] = torch.empty((B, H, G, T) if G > 1 else (B, H, T), device="cuda")
        t["p"] = binding.make_params(B, H, T, d, binding.NATSL_BF16, la, sm, lse=t["lse"], G=G)
        t["ws"] = binding.alloc_workspace(t["p"], binding.OP_TREE)
        return t

    one, other = batch(), batch()
    alone = []
    for t in (one, other):
        step(t)
        torch.cuda.synchronize()
        alone.append([t[m].clone() for m in ("out", "u", "lse")])
        assert all(torch.isfinite(y).all() for y in alone[-1])
    for _ in range(40):
        for _ in range(5):
            step(one)
            step(other)
        torch.cuda.synchronize()
        for t, want in zip((one, other), alone):
            assert all(torch.equal(t[m], y) for m, y in zip(("out", "u", "lse"), want))
    assert binding.natsl_device_status(one["ws"]) == 0 and binding.natsl_device_status(other["ws"]) == 0
