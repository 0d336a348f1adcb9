"""Attention weights of the retained entries and eviction by them (natsl_cache_weights, natsl_cache_evict) against the fp64
oracle, and a run of everything that generation with a bounded cache calls.

Tolerance of the weights: a probability's relative error is its exponent's absolute one: logits of at most 12, each a sum of
128 products in fp32, 12 * 128 * 2^-24 = 9.2e-5 at worst; entries are compared with 1e-4 of themselves plus the RMS.
An eviction copies: every result is exact."""
import numpy as np
import pytest
import torch

from oracle import tree
from paper_2602_03681_b200 import inputs
from test_gpu_parity import TOL, check_stored, dev, rel_err
from test_gpu_tree import scales
from tree_cases import make, paths, random_tree

pytestmark = pytest.mark.gpu

LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 300, 513, 600]


def logits(x, sm, G, norm):
    """lse [B,H,G,T] of the rows q over the entries they see, fp64."""
    B, T, H, d = x["q"].shape
    out = np.full((B, H, G, T), -np.inf)
    qs, kc = tree._rows(x["q"], G, norm, 1e-6)[1], tree._rows(x["k_cache"], G, norm, 1e-6)[1]
    for b in range(B):
        for h in range(H):
            for t in range(T):
                m = max(0, min(int(x["visible"][b, t, h]), int(x["cache_len"][b, h])))
                for s in range(G):
                    if m:
                        y = sm * (kc[b, h, :m, s] @ qs[b, t, h, s])
                        out[b, h, s, t] = y.max() + np.log(np.exp(y - y.max()).sum())
    return out.astype(np.float32)


def weigh(x, dtype, G=1, norm=False, flags=0, visible=True):
    from paper_2602_03681_b200 import binding
    B, T, H, d = x["q"].shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    la, sm = scales(d, G, norm)
    weight = dev(x["weight"])
    q, kc = dev(x["q"], dt), dev(x["k_cache"], dt)
    p = binding.make_params(B, H, T, d, binding._dtype_code(q), la, sm, flags=flags | (binding.QK_NORM if norm else 0), G=G,
                            norm_eps=1e-6 if norm else 0.0)
    lse = dev(x["lse"] if G > 1 else x["lse"][:, :, 0])
    binding.natsl_cache_weights(q, lse, dev(x["visible"]) if visible else None, kc, dev(x["cache_len"]), weight, p)
    ref = tree.cache_weights(x["q"], x["lse"], x["visible"] if visible else None, x["k_cache"], x["cache_len"], x["weight"],
                             scale_sm=sm, G=G, qk_norm=norm)
    got = weight.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    fin = ~np.isnan(ref)
    rms = np.sqrt((ref[fin] ** 2).mean())
    assert (np.abs(got[fin] - ref[fin]) <= 1e-4 * (np.abs(ref[fin]) + rms)).all()
    for b in range(B):                               # entries behind the length: left alone
        for h in range(H):
            n = x["cache_len"][b, h]
            assert np.array_equal(got[b, h, n:], x["weight"][b, h, n:])


def case(seed, B, H, T, d, lengths, cap, dtype, G=1, norm=False):
    x = make(seed, B, H, T, d, lengths, cap, dtype, unit=not norm)
    rng = np.random.default_rng(seed)
    x["visible"] = rng.integers(-2, cap + 3, (B, T, H)).astype(np.int32)
    x["visible"][0, 0, 0] = [-2 ** 31, 2 ** 31 - 1][seed % 2]
    x["weight"] = rng.random((B, H, cap)).astype(np.float32)
    x["lse"] = logits(x, scales(d, G, norm)[1], G, norm)
    return x


@pytest.mark.parametrize("dtype,d,G,norm,flags", [
    ("f32", 64, 1, False, 0), ("f32", 64, 2, True, 0), ("f32", 128, 4, True, 0), ("f32", 128, 2, False, 0),
    ("bf16", 64, 1, False, 0), ("bf16", 64, 2, True, 0), ("bf16", 128, 1, True, 0), ("bf16", 128, 2, True, 0),
    ("bf16", 128, 2, False, 0), ("bf16", 128, 4, True, 0), ("bf16", 128, 1, False, 1), ("bf16", 128, 1, False, 0)])
@pytest.mark.parametrize("T", [1, 13, 16, 17, 64, 77])
def test_weights(dtype, d, G, norm, flags, T):
    weigh(case(T + d, 2, 3, T, d, [0, 1, 65, 200, 310, 64], 310, dtype, G, norm), dtype, G, norm, flags)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [5, 30, 40])
def test_weights_of_every_length(dtype, T):
    x = case(3, 3, 5, T, 128, LENGTHS, 600, dtype)
    weigh(x, dtype)
    weigh(x, dtype, visible=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,norm", [(1, False), (1, True), (2, False), (2, True)])
@pytest.mark.parametrize("T", [32, 65, 128, 200])
def test_weights_of_many_rows(d, G, norm, T):
    """Rows by the 64, keys by the 128, runs of 256 and more of them."""
    x = case(T, 2, 2, T, d, [1200, 0, 129, 256, 640], 1200, "bf16", G, norm)
    weigh(x, "bf16", G, norm)
    weigh(x, "bf16", G, norm, visible=False)


def test_weights_of_many_pairs():
    """Runs of more than the shortest length."""
    x = case(5, 8, 16, 40, 128, [1500, 31, 800, 1024, 1025], 1500, "bf16")
    weigh(x, "bf16")


@pytest.mark.parametrize("dtype,T,d", [("f32", 9, 64), ("bf16", 9, 64), ("bf16", 70, 64), ("bf16", 70, 128)])
def test_rows_that_count_for_nothing(dtype, T, d):
    """A row whose log-sum-exp is not finite, whatever its query holds; entries behind the length, whatever they hold; an
    entry that is NaN gets a NaN of its own."""
    x = case(4, 1, 2, T, d, [50, 17], 60, dtype)
    x["visible"][:] = 60
    x["lse"] = logits(x, d ** 0.5, 1, False)
    x["lse"][:, :, :, 2], x["lse"][:, :, :, 3], x["lse"][:, :, :, 4] = -np.inf, np.inf, np.nan
    x["q"][:, 2:5] = np.nan
    x["k_cache"][0, 0, 50:], x["k_cache"][0, 1, 17:] = np.nan, np.inf
    weigh(x, dtype)
    x["k_cache"][0, 0, 7] = np.nan
    weigh(x, dtype)


# ---------------------------------------------------------------------------------------------
def evict(k, v, w, n, keep, first, recent, dtype):
    """natsl_cache_evict on copies; checked against the oracle entry by entry."""
    from paper_2602_03681_b200 import binding
    B, H, cap, d = k.shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    kc, vc, weight, length = dev(k, dt), dev(v, dt), dev(w), dev(n)
    kept = torch.full((B, H, keep), -9, dtype=torch.int32, device="cuda")
    p = binding.make_params(B, H, 0, d, binding._dtype_code(kc), 1.0, 1.0)
    want = [x.clone() for x in (kc, vc, weight, length, kept)]
    for b in range(B):
        for h in range(H):
            stay = tree.evict(w[b, h], max(0, min(int(n[b, h]), cap)), keep, first, recent)
            at = torch.tensor(stay, dtype=torch.long, device="cuda")
            for x, y in zip(want[:3], (kc, vc, weight)):
                x[b, h, :len(stay)] = y[b, h, at]
            if n[b, h] > keep:
                want[3][b, h] = keep
            want[4][b, h, :len(stay)] = at.to(torch.int32)
    binding.natsl_cache_evict(kc, vc, weight, length, keep, first, recent, kept, p)
    for name, x, y in zip(("kept", "cache_len", "weight", "k", "v"), (kept, length, weight, kc, vc),
                          (want[4], want[3], want[2], want[0], want[1])):
        assert torch.equal(x.nan_to_num(nan=-5.0), y.nan_to_num(nan=-5.0)), name


def cache(seed, B, H, cap, d, dtype):
    rng = np.random.default_rng(seed)
    k, v = (rng.standard_normal((B, H, cap, d)).astype(np.float32) for _ in range(2))
    if dtype == "bf16":
        k, v = inputs.round_bf16(k), inputs.round_bf16(v)
    return rng, k, v, np.exp(1.5 * rng.standard_normal((B, H, cap))).astype(np.float32)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (1, 0, 1), (16, 4, 4), (63, 0, 63), (64, 1, 0), (200, 4, 50), (599, 0, 0),
                                               (600, 10, 10)])
def test_eviction(dtype, d, keep, first, recent):
    _, k, v, w = cache(keep, 3, 5, 600, d, dtype)
    n = np.random.default_rng(1).permutation(LENGTHS).reshape(3, 5).astype(np.int32)
    evict(k, v, w, n, keep, first, recent, dtype)


@pytest.mark.parametrize("B,H", [(1, 1), (1, 2), (2, 8), (5, 8), (5, 20), (13, 13)])
def test_eviction_by_number_of_pairs(B, H):
    """Few pairs are moved by several CTAs each."""
    rng, k, v, w = cache(B, B, H, 2300, 64, "bf16")
    n = rng.integers(0, 2301, (B, H)).astype(np.int32)
    n[0, 0] = 2300
    evict(k, v, w, n, 1111, 3, 100, "bf16")


@pytest.mark.parametrize("keep,first,recent", [(1500, 1, 5), (1499, 0, 0)])
def test_eviction_with_ties_and_odd_weights(keep, first, recent):
    """Ties go to the lower index; a NaN is the lowest; zeros of both signs are equal; infinities and negative weights count."""
    rng, k, v, w = cache(9, 2, 3, 3001, 64, "f32")
    w[0, 0] = 1.0
    w[0, 1] = rng.integers(0, 3, 3001)
    w[0, 2] = np.where(rng.random(3001) < 0.7, np.nan, w[0, 2])
    w[1, 0] = np.where(rng.random(3001) < 0.5, 0.0, -0.0)
    w[1, 1] = rng.choice([np.inf, -np.inf, np.nan, 1.0, -1.0, 0.0], 3001)
    w[1, 2] = 1.0 + rng.integers(0, 4, 3001) * 2.0 ** -23           # (they differ in the last bits only)
    evict(k, v, w, np.full((2, 3), 3001, np.int32), keep, first, recent, "f32")


@pytest.mark.parametrize("B", [1, 40])
def test_eviction_of_the_tail(B):
    """What stays is already in front: nothing moves, the length does."""
    _, k, v, w = cache(5, B, 4, 500, 64, "bf16")
    w[:] = np.arange(500, 0, -1)
    evict(k, v, w, np.full((B, 4), 500, np.int32), 320, 3, 0, "bf16")
    evict(k, v, w, np.full((B, 4), 500, np.int32), 320, 320, 0, "bf16")


@pytest.mark.parametrize("H", [2, 90, 160])
def test_eviction_of_long_caches(H):
    """More entries than a CTA holds in registers."""
    rng, k, v, w = cache(6, 1, H, 9001, 64, "bf16")
    n = rng.integers(8000, 9002, (1, H)).astype(np.int32)
    evict(k, v, w, n, 6007, 5, 111, "bf16")


def test_eviction_of_stored_lengths_out_of_range():
    _, k, v, w = cache(2, 1, 3, 100, 64, "bf16")
    evict(k, v, w, np.array([[-4, 100, 130]], np.int32), 60, 2, 3, "bf16")


# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,G,norm", [("f32", 1, False), ("bf16", 1, False), ("bf16", 2, True)])
def test_generation_with_a_bounded_cache(dtype, G, norm):
    """As a server would run it: prefill, weights of the last queries, eviction, then rounds of draft, tree step, commit,
    weights of the accepted nodes and eviction -- every round against the oracle, from the device's own state before it."""
    from paper_2602_03681_b200 import binding
    B, H, L, T, d, keep, first, recent = 2, 3, 192, 9, 128, 40, 2, 8
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    la, sm = scales(d, G, norm)
    kw = dict(scale_sm=sm, G=G, qk_norm=norm)
    flags = binding.QK_NORM if norm else 0
    eps = 1e-6 if norm else 0.0
    rng = np.random.default_rng(17)
    x = make(17, B, H, L, d, [0], 1, dtype, unit=not norm, route="mixed")
    res = binding.hybrid_fwd(dev(x["q"], dt), dev(x["k"], dt), dev(x["v"], dt), dev(x["g"]), dev(x["beta"]), dev(x["route"]),
                             dev(x["w"]), scale_la=la, scale_sm=sm, want=("lse", "state_out", "cache"), flags=flags, sm_cap=L + 64,
                             G=G, norm_eps=eps)
    kc, vc, length, state, lse = res["k_sm"], res["v_sm"], res["sm_len"], res["state_out"], res["lse"].reshape(B, H, G, L)
    weight = torch.zeros(kc.shape[:3], device="cuda")
    visible = dev(x["route"]).to(torch.int32).cumsum(1).to(torch.int32)
    W = 32                                           # the prompt's last queries
    args = [a[:, -W:].contiguous() for a in (dev(x["q"], dt), visible)]
    rows = lse[..., -W:].contiguous()

    def weigh_and_evict(q, rows, visible, weight):
        T = q.shape[1]
        p = binding.make_params(B, H, T, d, binding._dtype_code(q), la, sm, flags=flags, G=G, norm_eps=eps)
        ref = tree.cache_weights(q.double().cpu().numpy(), rows.double().cpu().numpy(), visible.cpu().numpy(), kc.double().cpu().numpy(),
                                 length.cpu().numpy(), weight.cpu().numpy(), **kw)
        binding.natsl_cache_weights(q, rows if G > 1 else rows[:, :, 0].contiguous(), visible, kc, length, weight, p)
        got = weight.cpu().numpy()
        assert (np.abs(got - ref) <= 1e-4 * (ref + np.sqrt((ref ** 2).mean()))).all()
        before = [a.clone() for a in (kc, vc, weight)]
        n = length.cpu().numpy()
        kept = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
        binding.natsl_cache_evict(kc, vc, weight, length, keep, first, recent, kept, p)
        for b in range(B):
            for h in range(H):
                stay = tree.evict(got[b, h], int(n[b, h]), keep, first, recent)
                assert int(length[b, h]) == len(stay) and kept[b, h, :len(stay)].tolist() == stay
                for a, was in zip((kc, vc, weight), before):
                    assert torch.equal(a[b, h, :len(stay)], was[b, h, stay])

    weigh_and_evict(args[0], rows, args[1], weight)
    ws = None
    for r in range(4):
        y = make(100 + r, B, H, T, d, [0], 1, dtype, unit=not norm, route="mixed")
        y["parent"] = random_tree(rng, B, T)
        y["path"], y["n_path"] = paths(rng, y["parent"])
        t = {m: dev(y[m], dt if m in ("q", "k", "v") else None) for m in ("q", "k", "v", "g", "beta", "route", "w", "parent", "path", "n_path")}
        out, u = torch.empty_like(t["q"]), torch.empty(t["q"].shape, device="cuda")
        lse = torch.empty((B, H, G, T) if G > 1 else (B, H, T), device="cuda")
        p = binding.make_params(B, H, T, d, binding._dtype_code(out), la, sm, flags=flags, w=t["w"], lse=lse, G=G, norm_eps=eps)
        ws = binding.alloc_workspace(p, binding.OP_TREE) if ws is None else ws
        st = [a.double().cpu().numpy() for a in (state, kc, vc)] + [length.cpu().numpy().copy()]
        ref = tree.tree_step(y["q"], y["k"], y["v"], y["g"], y["beta"], y["route"], y["w"], y["parent"], None, *st, scale_la=la, **kw)
        binding.natsl_tree_step(t["q"], t["k"], t["v"], t["g"], t["beta"], t["route"], t["parent"], None, state, kc, vc, length, out, u,
                                p, ws)
        check_stored(out.float().cpu().numpy(), ref["out"], TOL[dtype], dtype)
        tree.tree_commit(y["k"], y["v"], y["g"], y["beta"], y["route"], y["path"], y["n_path"], *st, qk_norm=norm)
        n_before = length.clone()
        binding.natsl_tree_commit(t["k"], t["v"], t["g"], t["route"], u, t["path"], t["n_path"], state, kc, vc, length, p, ws)
        assert np.array_equal(length.cpu().numpy(), st[3]) and np.array_equal(kc.double().cpu().numpy(), st[1])
        assert rel_err(state.cpu().numpy(), st[0]) <= 1e-4
        # the accepted nodes' rows; behind a sequence's path rows that count for nothing
        m = int(y["n_path"].max())
        at = t["path"][:, :m].clamp(min=0).long()
        live = (torch.arange(m, device="cuda") < t["n_path"][:, None])
        q = out.new_empty((B, m, H, d))
        q.copy_(t["q"].gather(1, at[:, :, None, None].expand(B, m, H, d)))
        rows = lse.reshape(B, H, G, T).gather(3, at[:, None, None].expand(B, H, G, m))
        rows = torch.where(live[:, None, None], rows, -torch.inf).contiguous()
        kept = (t["route"].gather(1, at[:, :, None].expand(B, m, H)) != 0) & live[:, :, None]
        visible = (n_before[:, None] + kept.cumsum(1)).to(torch.int32)
        weigh_and_evict(q, rows, visible, weight)
        assert binding.natsl_device_status(ws) == 0


@pytest.mark.parametrize("dtype,T", [("bf16", 12), ("bf16", 40), ("f32", 12)])
def test_calls_one_behind_the_other(dtype, T):
    """Step, weights, commit and eviction, three rounds of them: enqueued back to back (each may start while the one ahead of it
    ends) and with the GPU waited for after each."""
    from paper_2602_03681_b200 import binding
    B, H, d, cap, keep = 24, 16, 128, 500, 300
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(T)
    x = make(T, B, H, T, d, [0, 290, 300, 300, 299], cap, dtype, route="all")
    t = {n: dev(x[n], dt if n in ("q", "k", "v", "k_cache", "v_cache") else None) for n in x if x[n] is not None}
    weight = dev(rng.random((B, H, cap)).astype(np.float32))
    la, sm = scales(d, 1, False)
    got = []
    for wait in (True, False, False):
        kc, vc, w, n, state = (y.clone() for y in (t["k_cache"], t["v_cache"], weight, t["cache_len"], t["state"]))
        out, u = torch.empty_like(t["q"]), torch.empty(B, T, H, d, device="cuda")
        lse, kept = torch.empty(B, H, T, device="cuda"), torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
        p = binding.make_params(B, H, T, d, binding._dtype_code(out), la, sm, w=t["w"], lse=lse)
        ws = binding.alloc_workspace(p, binding.OP_TREE)
        torch.cuda.synchronize()
        for _ in range(3):
            for f in (lambda: binding.natsl_tree_step(t["q"], t["k"], t["v"], t["g"], t["beta"], t["route"], t["parent"], None, state, kc,
                                                      vc, n, out, u, p, ws),
                      lambda: binding.natsl_cache_weights(t["q"], lse, None, kc, n, w, p),
                      lambda: binding.natsl_tree_commit(t["k"], t["v"], t["g"], t["route"], u, t["path"], t["n_path"], state, kc, vc, n,
                                                        p, ws),
                      lambda: binding.natsl_cache_evict(kc, vc, w, n, keep, 2, 10, kept, p)):
                f()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert binding.natsl_device_status(ws) == 0
        got.append([out, u, lse, state, n, kept, w, kc, vc])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("dtype,T", [("f32", 9), ("bf16", 9), ("bf16", 40)])
def test_captured_and_on_another_stream(dtype, T):
    """Weights and eviction in a CUDA graph, replayed on new contents on a stream of its own, against the calls themselves."""
    from paper_2602_03681_b200 import binding
    B, H, d, cap, keep = 2, 4, 128, 900, 200
    x = case(9, B, H, T, d, [0, 150, 200, 201, 900, 899, 512, 640], cap, dtype)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    la, sm = scales(d, 1, False)
    q, kc, vc = dev(x["q"], dt), dev(x["k_cache"], dt), dev(x["v_cache"], dt)
    lse, visible, weight, n = dev(x["lse"][:, :, 0]), dev(x["visible"]), dev(x["weight"]), dev(x["cache_len"])
    kept = torch.zeros(B, H, keep, dtype=torch.int32, device="cuda")
    p = binding.make_params(B, H, T, d, binding._dtype_code(q), la, sm)
    start = [y.clone() for y in (kc, vc, weight, n, kept)]

    def run():
        binding.natsl_cache_weights(q, lse, visible, kc, n, weight, p)
        binding.natsl_cache_evict(kc, vc, weight, n, keep, 4, 30, kept, p)

    def reset():
        for y, s0 in zip((kc, vc, weight, n, kept), start):
            y.copy_(s0)
        torch.cuda.synchronize()

    run()
    torch.cuda.synchronize()
    want = [y.clone() for y in (kc, vc, weight, n, kept)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(graph, stream=side):
        run()
    for _ in range(3):
        reset()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, w) for y, w in zip((kc, vc, weight, n, kept), want))


@pytest.mark.parametrize("dtype,T", [("bf16", 9), ("bf16", 40), ("f32", 9)])
def test_offsets_past_32_bits(dtype, T):
    """Caches of more than 2^31 elements a pair: the second pair's lies behind them.  All four calls give what they give for
    the same entries in a small cache."""
    from paper_2602_03681_b200 import binding
    d, cap, big, keep = 128, 400, 2 ** 24 + 64, 100
    if torch.cuda.mem_get_info()[0] < 6 * big * d * (2 if dtype == "bf16" else 4):
        pytest.skip("not enough device memory")
    x = make(6, 1, 2, T, d, [300, 290], cap, dtype)
    t = {n: dev(x[n], torch.bfloat16 if dtype == "bf16" and n in ("q", "k", "v", "k_cache", "v_cache") else None) for n in x
         if x[n] is not None}
    la, sm = scales(d, 1, False)
    results = []
    for rows in (cap, big):
        kc = torch.empty(1, 2, rows, d, dtype=t["k_cache"].dtype, device="cuda")
        vc, weight = torch.empty_like(kc), torch.zeros(1, 2, rows, device="cuda")
        kc[:, :, :cap], vc[:, :, :cap] = t["k_cache"], t["v_cache"]
        out, u = torch.empty_like(t["q"]), torch.empty(1, T, 2, d, device="cuda")
        lse, state, length = torch.empty(1, 2, T, device="cuda"), t["state"].clone(), t["cache_len"].clone()
        kept = torch.full((1, 2, keep), -1, dtype=torch.int32, device="cuda")
        p = binding.make_params(1, 2, T, d, binding._dtype_code(out), la, sm, w=t["w"], lse=lse)
        ws = binding.alloc_workspace(p, binding.OP_TREE)
        binding.natsl_tree_step(t["q"], t["k"], t["v"], t["g"], t["beta"], t["route"], t["parent"], None, state, kc, vc, length, out, u,
                                p, ws)
        binding.natsl_tree_commit(t["k"], t["v"], t["g"], t["route"], u, t["path"], t["n_path"], state, kc, vc, length, p, ws)
        binding.natsl_cache_weights(t["q"], lse, None, kc, length, weight, p)
        grown = [kc[:, :, :cap].clone(), vc[:, :, :cap].clone(), length.clone()]
        binding.natsl_cache_evict(kc, vc, weight, length, keep, 2, 10, kept, p)
        assert binding.natsl_device_status(ws) == 0
        results.append([out, u, lse, state, length, kept, weight[:, :, :keep].clone(), kc[:, :, :keep].clone(), vc[:, :, :keep].clone()] +
                       [g[:, h, :grown[2][0, h]] if g.dim() > 2 else g for g in grown for h in range(2)])
        del kc, vc, weight
        torch.cuda.empty_cache()
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dtype,T", [("f32", 6), ("bf16", 6), ("bf16", 40)])
def test_weights_of_what_is_appended_after_an_eviction(dtype, T):
    """The places behind a cut cache keep the weights of what lay there; set to zero, as natsl.h asks, they give the entries that
    are appended next the weights that these rows give them and no others."""
    from paper_2602_03681_b200 import binding
    B, H, d, cap, keep = 1, 3, 64, 200, 50
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = make(T, B, H, T, d, [150, 90, 51], cap, dtype, tree="chain", route=1)
    x["path"][:], x["n_path"][:] = np.arange(T), T
    t = {n: dev(x[n], dt if n in ("q", "k", "v", "k_cache", "v_cache") else None) for n in x if x[n] is not None}
    kc, vc, n, state = t["k_cache"], t["v_cache"], t["cache_len"], t["state"]
    la, sm = scales(d, 1, False)
    weight = torch.rand(B, H, cap, device="cuda") + 1.0
    kept = torch.empty(B, H, keep, dtype=torch.int32, device="cuda")
    out, u = torch.empty_like(t["q"]), torch.empty(B, T, H, d, device="cuda")
    lse = torch.empty(B, H, T, device="cuda")
    p = binding.make_params(B, H, T, d, binding._dtype_code(out), la, sm, lse=lse)
    ws = binding.alloc_workspace(p, binding.OP_TREE)
    binding.natsl_cache_evict(kc, vc, weight, n, keep, 2, 5, kept, p)
    behind = torch.arange(cap, device="cuda") >= n[:, :, None]
    assert (weight[behind] >= 1.0).all()             # (as they were)
    weight.masked_fill_(behind, 0.0)
    binding.natsl_tree_step(t["q"], t["k"], t["v"], t["g"], t["beta"], t["route"], t["parent"], None, state, kc, vc, n, out, u, p, ws)
    binding.natsl_tree_commit(t["k"], t["v"], t["g"], t["route"], u, t["path"], t["n_path"], state, kc, vc, n, p, ws)
    visible = (keep + torch.arange(1, T + 1, device="cuda", dtype=torch.int32))[None, :, None].expand(B, T, H).contiguous()
    before = weight.clone()
    binding.natsl_cache_weights(t["q"], lse, visible, kc, n, weight, p)
    assert binding.natsl_device_status(ws) == 0 and (n == keep + T).all()
    # a row of a chain sees the cache and itself with what lies before it: all of its unit goes to entries
    given = (weight - before)[:, :, :keep + T].double()
    assert torch.equal(weight[:, :, keep + T:], before[:, :, keep + T:])
    assert (given.sum(-1) - T).abs().max() <= 1e-4 * T
    ref = tree.cache_weights(x["q"], lse.double().cpu().numpy()[:, :, None], visible.cpu().numpy(), kc.double().cpu().numpy(),
                             n.cpu().numpy(), np.zeros((B, H, cap)), scale_sm=sm)[:, :, keep:keep + T]
    got = weight[:, :, keep:keep + T].cpu().numpy()
    assert (np.abs(got - ref) <= 1e-4 * (ref + np.sqrt((ref ** 2).mean()))).all()
