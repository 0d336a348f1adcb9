"""Speculative generation on the layer's two hidden states and a cache that stays bounded, each operator in its plain form
and as the call of ``paper_2602_03681_b200.binding`` that a program makes.

A case is a dict of plain values.  ``kind`` says which operator one pass runs:

  tree     the hybrid layer over a tree of ``T`` drafted tokens per sequence (one token: plain generation), state and cache unchanged
  commit   the accepted path of such a tree goes into the linear state and the retained cache
  weights  attention weights of ``T`` query rows, added up per cache entry
  evict    the cache shrinks to ``keep`` entries, by those weights

``mode`` is how the layer is set up: "token" (a route per token, unit-norm q and k, one softmax head per linear head) or
"paper" (the decision of the current block open, q and k normalised by the operator, two softmax heads of 64 columns per
linear head at d = 128 and one at d = 64).  ``ctx`` is the largest number of retained tokens; with ``ragged`` each
(sequence, head) has its own, down to half of it, and some trees have fewer nodes than ``T``.
"""
import math
import random

import torch

own = False

EPS = 1e-5
NORM_EPS = 1e-6
P_KEEP = 0.2            # share of tokens that the softmax branch retains ("token" mode)


def listed():
    return [
        # one user: a tree of 16 drafted tokens over 1638 retained ones (10 % of a context of 16384); latency
        dict(name="tree_one_user", kind="tree", mode="token", dtype="bf16", B=1, H=16, d=128, T=16, ctx=1638, ragged=False),
        # a serving batch of 64, one token each: the operator as plain generation
        dict(name="tree_one_token", kind="tree", mode="token", dtype="bf16", B=64, H=16, d=128, T=1, ctx=1638, ragged=False),
        # the same batch with 32 drafted tokens each: the memory-bound end, the largest case
        dict(name="tree_batch64", kind="tree", mode="token", dtype="bf16", B=64, H=16, d=128, T=32, ctx=1638, ragged=False),
        # full trees over long ragged caches (20 % of a context of 32768)
        dict(name="tree_full_long", kind="tree", mode="token", dtype="bf16", B=8, H=16, d=128, T=64, ctx=6554, ragged=True),
        # a model of the paper's mode, its block open: two softmax heads per linear head, normalised q and k, ragged
        dict(name="tree_paper", kind="tree", mode="paper", dtype="bf16", B=12, H=6, d=128, T=47, ctx=771, ragged=True),
        # fp32 storage, the arithmetic that bf16 results are checked against: two heads, a short cache
        dict(name="tree_f32_tiny", kind="tree", mode="token", dtype="f32", B=1, H=2, d=64, T=7, ctx=100, ragged=True),
        # one user's accepted path, and the batch's
        dict(name="commit_one_user", kind="commit", mode="token", dtype="bf16", B=1, H=16, d=128, T=16, ctx=1638, ragged=False),
        dict(name="commit_batch64", kind="commit", mode="token", dtype="bf16", B=64, H=16, d=128, T=32, ctx=1638, ragged=False),
        # the last 64 queries of four prompts weigh what the prompts retained, before it is cut down
        dict(name="weights_window", kind="weights", mode="paper", dtype="bf16", B=4, H=16, d=128, T=64, ctx=3277, ragged=True),
        # every step of a batch: the accepted nodes' weights
        dict(name="weights_batch64", kind="weights", mode="token", dtype="bf16", B=64, H=16, d=128, T=5, ctx=1638, ragged=False),
        # one user's cache of 8192 entries cut to half
        dict(name="evict_one_user", kind="evict", mode="token", dtype="bf16", B=1, H=16, d=128, ctx=8192, keep=4096, ragged=False),
        # a batch's caches cut to a budget of 1024
        dict(name="evict_batch64", kind="evict", mode="token", dtype="bf16", B=64, H=16, d=128, ctx=1638, keep=1024, ragged=True),
    ]


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, every kind, mode, head size and storage type."""
    def log(a, b):
        return min(b, max(a, int(round(math.exp(rng.uniform(math.log(a), math.log(b + 1)))))))

    most = [work(c) for c in listed()]
    most = {m: max(w[m] for w in most) for m in ("bytes", "flops")}
    while True:
        kind = rng.choice(["tree", "tree", "tree", "commit", "weights", "evict"])
        c = dict(kind=kind, mode=rng.choice(["token", "token", "paper"]), dtype="bf16", B=log(1, 64), H=rng.randint(2, 16),
                 d=rng.choice([64, 128, 128]), ctx=log(1, 8192), ragged=rng.random() < 0.5)
        if kind != "evict":
            c.update(T=log(1, 256 if kind == "weights" else 64))
        else:
            c.update(keep=max(1, int(c["ctx"] * rng.uniform(0.25, 0.95))))
        if rng.random() < 0.15:                                     # fp32 storage: small calls
            c.update(dtype="f32", B=log(1, 4), H=rng.randint(1, 8), ctx=log(1, 1024))
            if kind != "evict":
                c.update(T=log(1, 32))
            else:
                c.update(keep=max(1, int(c["ctx"] * rng.uniform(0.25, 0.95))))
        w = work(c)
        if all(w[m] <= most[m] for m in most):
            return c


def _groups(c):
    return 2 if c["mode"] == "paper" and c["d"] == 128 else 1


def _scales(c):
    """Logit scales: d^-1/2 for the linear read-out; for the softmax branch sqrt(d) on unit-norm q and k, (slice
    width)^-1/2 where the operator normalises."""
    return c["d"] ** -0.5, (c["d"] // _groups(c)) ** -0.5 if c["mode"] == "paper" else c["d"] ** 0.5


def _trees(c, seed):
    """Parents [B,T] (below the node, -1: the context), nodes per tree [B], the path to the deepest node of each tree
    [B,T] and its length [B]: drafts branch off one of the last few nodes, one tree in eight is a chain."""
    rng = random.Random(seed)
    T = c["T"]
    parents, nodes, paths, lengths = [], [], [], []
    for _ in range(c["B"]):
        n = rng.randint((T + 1) // 2, T) if c["ragged"] else T
        par = list(range(-1, T - 1)) if rng.random() < 0.125 else [max(-1, i - 1 - int(rng.expovariate(0.4))) for i in range(T)]
        depth = []
        for i in range(n):
            depth.append(0 if par[i] < 0 else depth[par[i]] + 1)
        path, i = [], depth.index(max(depth))
        while i >= 0:
            path.insert(0, i)
            i = par[i]
        parents.append(par)
        nodes.append(n)
        lengths.append(len(path))
        paths.append(path + [-1] * (T - len(path)))
    return [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (parents, nodes, paths, lengths)]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    B, H, d, ctx, G = c["B"], c["H"], c["d"], c["ctx"], _groups(c)
    kind = c["kind"]
    T = c.get("T", 1)
    unit = c["mode"] == "token"                     # (paper's mode: the operator normalises)

    def n(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def u(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    def rows(*shape):
        x = n(*shape)
        return (torch.nn.functional.normalize(x, dim=-1) if unit else x).to(dt)

    s = dict(kind=kind, G=G, norm=not unit, keep=c.get("keep"))
    s["scale_la"], s["scale_sm"] = _scales(c)
    cap = ctx + T
    length = torch.full((B, H), ctx, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        length -= (u(B, H) * ((ctx + 1) // 2)).to(torch.int32)
    s["length"], s["cache_len"] = length, length.clone()
    inside = torch.arange(cap, device="cuda") < length[:, :, None]
    s["k_cache"] = rows(B, H, cap, d) * inside[..., None]
    s["v_cache"] = n(B, H, cap, d).to(dt) * inside[..., None]
    if kind == "evict":
        # sums of a few hundred queries' probabilities: a few entries carry most of it
        s["weight"] = torch.exp(1.5 * n(B, H, cap)) * inside
        s["first"], s["recent"] = min(4, c["keep"] // 4), c["keep"] // 8
        s["kept"] = torch.zeros((B, H, c["keep"]), dtype=torch.int32, device="cuda")
    elif kind == "weights":
        s["q"] = rows(B, T, H, d)
        kept = u(B, T, H) < P_KEEP
        s["visible"] = (length[:, None] - (kept.sum(1, keepdim=True) - kept.cumsum(1))).clamp_(min=0).to(torch.int32)
        x, _ = _logits(s, _slices(s["q"].float(), s))
        s["lse"] = torch.logsumexp(x, -1).contiguous() if G > 1 else torch.logsumexp(x, -1)[:, :, 0].contiguous()
        s["weight"] = u(B, H, cap) * inside
    else:
        s["parent"], s["n_nodes"], s["path"], s["n_path"] = _trees(c, seed)
        s["q"], s["k"], s["v"] = rows(B, T, H, d), rows(B, T, H, d), n(B, T, H, d).to(dt)
        s["g"] = -torch.nn.functional.softplus(n(B, T, H))
        s["beta"] = torch.sigmoid(n(B, T, H))
        s["route"] = (u(B, T, H) < P_KEEP).to(torch.uint8) if unit else torch.full((B, T, H), 2, dtype=torch.uint8, device="cuda")
        s["w"] = torch.softmax(n(B, T, H, 2), -1).contiguous()
        s["state"] = 0.1 * n(B, H, d, d)
        if kind == "tree":
            s["out"] = torch.zeros((B, T, H, d), dtype=dt, device="cuda")
            s["u"] = torch.zeros((B, T, H, d), dtype=torch.float32, device="cuda")
            s["lse"] = torch.zeros((B, H, G, T) if G > 1 else (B, H, T), dtype=torch.float32, device="cuda")
        else:
            s["u"] = n(B, T, H, d) * (s["route"] != 1)[..., None]        # as a tree step leaves it
    if own:
        from paper_2602_03681_b200 import binding as nb
        code = nb.NATSL_F32 if c["dtype"] == "f32" else nb.NATSL_BF16
        s["p"] = nb.make_params(B, H, T, d, code, s["scale_la"], s["scale_sm"], EPS, flags=nb.QK_NORM if s["norm"] else 0,
                                w=s["w"] if kind == "tree" else None, lse=s["lse"] if kind == "tree" else None, G=G,
                                norm_eps=NORM_EPS if s["norm"] else 0.0)
        if kind in ("tree", "commit"):
            s["ws"] = nb.alloc_workspace(s["p"], nb.OP_TREE)
    return s


# ---------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------
def _heads(x):
    """[B,T,H,...] -> [B,H,T,...]"""
    return x.transpose(1, 2)


def _slices(x, s):
    """[B,T,H,d] -> [B,H,G,T,d/G], RMS-normalised per slice where the operator normalises."""
    B, T, H, d = x.shape
    x = x.reshape(B, T, H, s["G"], d // s["G"]).permute(0, 2, 3, 1, 4)
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + NORM_EPS) if s["norm"] else x


def _unit(x, s):
    return x * torch.rsqrt(x.square().sum(-1, keepdim=True) + NORM_EPS) if s["norm"] else x


def _logits(s, q):
    """Scaled logits of the rows q [B,H,G,T,ds] against the cache, -inf outside it (and beyond ``visible``); the keys."""
    k = _slices(s["k_cache"].float().transpose(1, 2), s)
    x = s["scale_sm"] * (q @ k.transpose(-1, -2))
    at = torch.arange(k.shape[-2], device=k.device)
    seen = at < s["length"][:, :, None, None, None]
    if "visible" in s:
        seen = seen & (at < _heads(s["visible"])[:, :, None, :, None])
    return x.masked_fill(~seen, -math.inf), k


def _plain_tree(s):
    q, k, v = (s[m].float() for m in ("q", "k", "v"))
    B, T, H, d = q.shape
    G, ds = s["G"], d // s["G"]
    at = torch.arange(T, device=q.device)
    eye = torch.eye(T, device=q.device)
    step = (s["parent"][:, :, None] == at).float()
    path = (torch.linalg.matrix_power(eye + step, 64) > 0)[:, None]              # [B,1,T,T]: j is i or above it
    route = _heads(s["route"])
    fold, keep = route != 1, route != 0
    # decays along the paths: differences of their sums, in 64 bits
    total = path.double() @ _heads(s["g"]).double()[..., None]                    # [B,H,T,1]
    decay = torch.exp((total - total.transpose(-1, -2)).masked_fill(~path, -math.inf)).float()
    whole = torch.exp(total).float()
    ql, kl, vh = _heads(_unit(q, s)), _heads(_unit(k, s)), _heads(v)
    beta = _heads(s["beta"])[..., None]
    a = beta * decay * (kl @ kl.transpose(-1, -2)) * fold[:, :, None] * (1 - eye)
    u = torch.linalg.solve_triangular(eye + a, beta * (vh - whole * (kl @ s["state"])), upper=False, unitriangular=True)
    u = u * fold[..., None]
    o_la = s["scale_la"] * (whole * (ql @ s["state"]) + (decay * (ql @ kl.transpose(-1, -2)) * fold[:, :, None]) @ u)
    qs, ks, vs = _slices(q, s), _slices(k, s), vh.reshape(B, H, T, G, ds).transpose(2, 3)
    xc, _ = _logits(s, qs)
    seen = (path & keep[:, :, None])[:, :, None]
    xt = (s["scale_sm"] * (qs @ ks.transpose(-1, -2))).masked_fill(~seen, -math.inf)
    m = torch.maximum(xc.amax(-1, keepdim=True), xt.amax(-1, keepdim=True))
    m0 = m.masked_fill(m == -math.inf, 0.0)
    pc, pt = torch.exp(xc - m0), torch.exp(xt - m0)
    z = pc.sum(-1, keepdim=True) + pt.sum(-1, keepdim=True)
    vc = s["v_cache"].float().reshape(B, H, -1, G, ds).transpose(2, 3)
    o = (pc @ vc + pt @ vs) / z.masked_fill(z == 0, 1.0)
    lse = (m0 + torch.log(z))[..., 0]
    o = (o * torch.rsqrt(o.square().mean(-1, keepdim=True) + EPS)).transpose(2, 3).reshape(B, H, T, d)
    o_la = o_la * torch.rsqrt(o_la.square().mean(-1, keepdim=True) + EPS)
    w = _heads(s["w"])
    out = w[..., :1] * o + w[..., 1:] * o_la
    live = (at < s["n_nodes"][:, None])[:, None, :]                               # rows behind a tree's last node: untouched
    out = (out * live[..., None]).transpose(1, 2).to(s["q"].dtype).contiguous()
    u = (u * live[..., None]).transpose(1, 2).contiguous()
    lse = torch.where(live[:, :, None], lse, 0.0)
    return dict(out=out, u=u, lse=lse if G > 1 else lse[:, :, 0])


def _plain_commit(s):
    s["cache_len"].copy_(s["length"])               # every pass commits to the same cache
    B, T, H, d = s["k"].shape
    live = torch.arange(T, device="cuda") < s["n_path"][:, None]                  # [B,T]
    at = s["path"].clamp(min=0).long()[:, :, None].expand(B, T, H)
    g = torch.where(live[:, None], _heads(s["g"].gather(1, at)), 0.0).double()
    route = _heads(s["route"].gather(1, at))
    rows = at[..., None].expand(B, T, H, d)
    k, v, u = (_heads(s[m].gather(1, rows)) for m in ("k", "v", "u"))
    after = torch.exp(g.flip(-1).cumsum(-1).flip(-1) - g).float()                 # decay behind each token
    fold = after * ((route != 1) & live[:, None])
    s["state"].mul_(torch.exp(g.sum(-1)).float()[..., None, None])
    s["state"].add_((fold[..., None] * _unit(k.float(), s)).transpose(-1, -2) @ u)
    keep = (route != 0) & live[:, None]
    to = s["cache_len"][..., None] + keep.cumsum(-1) - 1
    b, h, t = keep.nonzero(as_tuple=True)
    s["k_cache"][b, h, to[b, h, t]] = k[b, h, t]
    s["v_cache"][b, h, to[b, h, t]] = v[b, h, t]
    s["cache_len"].add_(keep.sum(-1).to(torch.int32))
    return dict(state=s["state"], k_cache=s["k_cache"], v_cache=s["v_cache"], cache_len=s["cache_len"])


def _plain_weights(s):
    x, _ = _logits(s, _slices(s["q"].float(), s))
    lse = s["lse"] if s["G"] > 1 else s["lse"][:, :, None]
    ok = torch.isfinite(lse)[..., None]                                           # (rows that see nothing)
    p = torch.exp((x - torch.where(ok, lse[..., None], 0.0)).masked_fill(~ok, -math.inf))
    s["weight"].add_(p.sum((2, 3)))
    return dict(weight=s["weight"])


def _plain_evict(s):
    s["cache_len"].copy_(s["length"])               # every pass starts from the same lengths
    n, keep = s["length"][..., None], s["keep"]
    d = s["k_cache"].shape[-1]
    at = torch.arange(s["weight"].shape[-1], device="cuda")
    inside = at < n
    safe = inside & ((at < s["first"]) | (at >= n - s["recent"]))
    key = s["weight"].masked_fill(safe, math.inf).masked_fill(~inside, -math.inf)
    best = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :keep]
    order = torch.sort(torch.where(best < n, best, at.numel()), dim=-1).values    # in the cache's order
    new = torch.minimum(s["length"], torch.full_like(s["length"], keep))
    live = at[:keep] < new[..., None]
    order = torch.where(live, order, at[:keep])
    rows = order[..., None].expand(*order.shape, d)
    for m in ("k_cache", "v_cache"):
        s[m][:, :, :keep] = s[m].gather(2, rows)
    s["weight"][:, :, :keep] = s["weight"].gather(2, order)
    s["kept"].copy_(torch.where(live, order, s["kept"]))
    s["cache_len"].copy_(new)
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], weight=s["weight"], cache_len=s["cache_len"], kept=s["kept"])


def run(state):
    s = state
    kind = s["kind"]
    if not own:
        return {"tree": _plain_tree, "commit": _plain_commit, "weights": _plain_weights, "evict": _plain_evict}[kind](s)
    from paper_2602_03681_b200 import binding as nb
    if kind == "tree":
        nb.natsl_tree_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["route"], s["parent"], s["n_nodes"], s["state"],
                           s["k_cache"], s["v_cache"], s["cache_len"], s["out"], s["u"], s["p"], s["ws"])
        return dict(out=s["out"], u=s["u"], lse=s["lse"])
    if kind == "weights":
        nb.natsl_cache_weights(s["q"], s["lse"], s["visible"], s["k_cache"], s["cache_len"], s["weight"], s["p"])
        return dict(weight=s["weight"])
    s["cache_len"].copy_(s["length"])               # every pass starts from the same lengths
    if kind == "commit":
        nb.natsl_tree_commit(s["k"], s["v"], s["g"], s["route"], s["u"], s["path"], s["n_path"], s["state"], s["k_cache"],
                             s["v_cache"], s["cache_len"], s["p"], s["ws"])
        return dict(state=s["state"], k_cache=s["k_cache"], v_cache=s["v_cache"], cache_len=s["cache_len"])
    nb.natsl_cache_evict(s["k_cache"], s["v_cache"], s["weight"], s["cache_len"], s["keep"], s["first"], s["recent"], s["kept"],
                         s["p"])
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], weight=s["weight"], cache_len=s["cache_len"], kept=s["kept"])


def work(case):
    """Inputs read once, outputs written once; 2 operations per multiply-add."""
    c = case
    BH, d = c["B"] * c["H"], c["d"]
    e = 4 if c["dtype"] == "f32" else 2
    n = c["ctx"] * (0.75 if c["ragged"] else 1.0)
    if c["kind"] == "evict":
        stay = min(n, c["keep"])
        moved = stay if n > c["keep"] else 0
        return dict(bytes=BH * (4 * n + moved * (4 * d * e + 4) + 4 * stay), flops=BH * n)
    T = c["T"]
    if c["kind"] == "weights":
        return dict(bytes=BH * (n * d * e + 8 * n + T * (d * e + 8)), flops=BH * 2 * T * n * d)
    t = T * (0.75 if c["ragged"] else 1.0)
    if c["kind"] == "commit":
        m = min(t, 2 + t / 3)                       # a path's length, about
        kept = m * (1.0 if c["mode"] == "paper" else P_KEEP)
        return dict(bytes=BH * (8 * d * d + m * d * (e + 4) + kept * 3 * d * e), flops=BH * 2 * m * d * d)
    return dict(bytes=BH * (2 * n * d * e + 4 * d * d + t * (4 * d * e + 4 * d + 24)),
                flops=BH * (4 * t * n * d + 4 * t * d * d + 4 * t * t * d))


# ---------------------------------------------------------------------------------------------
# From the definitions, in 64 bits: token by token along each path
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, H, d, G = c["B"], c["H"], c["d"], s["G"]
    if c["kind"] == "evict":
        kept, weight, length = s["kept"].cpu(), s["weight"].double().cpu(), s["length"].cpu()
        for b in range(B):
            for h in range(H):
                n = int(length[b, h])
                w = weight[b, h, :n].tolist()
                stay = list(range(n))
                if n > c["keep"]:
                    safe = [j for j in range(n) if j < s["first"] or j >= n - s["recent"]]
                    rest = sorted(range(s["first"], n - s["recent"]), key=lambda j: (-w[j], j))
                    stay = sorted(safe + rest[:c["keep"] - len(safe)])
                kept[b, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
                weight[b, h, :len(stay)] = torch.tensor([w[j] for j in stay], dtype=torch.float64)
        return dict(k_cache=None, v_cache=None, weight=weight, cache_len=length.clamp(max=c["keep"]), kept=kept)

    def norm(x, width, mean):                       # over groups of `width` columns
        if not s["norm"]:
            return x
        y = x.reshape(*x.shape[:-1], -1, width)
        y = y / (y.pow(2).sum(-1, keepdim=True) / (width if mean else 1) + NORM_EPS).sqrt()
        return y.reshape(x.shape)

    ds, T = d // G, c["T"]
    kc = norm(s["k_cache"].double(), ds, True).reshape(B, H, -1, G, ds)
    at = torch.arange(kc.shape[2], device="cuda")
    if c["kind"] == "weights":
        q = norm(s["q"].double(), ds, True).reshape(B, T, H, G, ds)
        lse = (s["lse"] if G > 1 else s["lse"][:, :, None]).double()
        weight = s["weight"].double()
        for t in range(T):
            seen = at < torch.minimum(s["visible"][:, t], s["length"])[..., None]
            for a in range(G):
                x = s["scale_sm"] * torch.einsum("bhd,bhnd->bhn", q[:, t, :, a], kc[:, :, :, a])
                there = seen & torch.isfinite(lse[:, :, a, t])[..., None]
                weight += torch.where(there, torch.exp(x - lse[:, :, a, t, None]), 0.0)
        return dict(weight=weight)
    k, v, g = s["k"].double(), s["v"].double(), s["g"].double()
    kl, alpha = norm(k, d, False), torch.exp(g)
    if c["kind"] == "commit":
        path, state = s["path"].cpu().tolist(), s["state"].double()
        k_cache, v_cache, n = s["k_cache"].double(), s["v_cache"].double(), s["length"].cpu().clone()
        route, u = s["route"].cpu(), s["u"].double()
        for b in range(B):
            for i in path[b][:int(s["n_path"][b])]:
                fold = (s["route"][b, i] != 1).double()[:, None, None]
                state[b] = state[b] * alpha[b, i][:, None, None] + fold * kl[b, i][:, :, None] * u[b, i][:, None, :]
                for h in range(H):
                    if int(route[b, i, h]):
                        k_cache[b, h, int(n[b, h])], v_cache[b, h, int(n[b, h])] = k[b, i, h], v[b, i, h]
                        n[b, h] += 1
        return dict(state=state, k_cache=k_cache, v_cache=v_cache, cache_len=n)
    q = s["q"].double()
    ql, qs, ks = norm(q, d, False), norm(q, ds, True), norm(k, ds, True)
    vc = s["v_cache"].double().reshape(B, H, -1, G, ds)
    seen = at < s["length"][..., None]
    states, above = [], []                          # after each node; the nodes of its path, [B,T] truth values
    out = torch.zeros((B, T, H, d), dtype=torch.float64, device="cuda")
    u_all, lse_all = torch.zeros_like(out), torch.zeros((B, H, G, T), dtype=torch.float64, device="cuda")
    parent, first = s["parent"].cpu(), s["state"].double()
    for i in range(T):
        before = torch.stack([states[int(parent[b, i])][b] if parent[b, i] >= 0 else first[b] for b in range(B)])
        mine = torch.stack([above[int(parent[b, i])][b] if parent[b, i] >= 0 else torch.zeros(T, dtype=torch.bool, device="cuda")
                            for b in range(B)])
        mine[:, i] = True
        before = before * alpha[:, i][:, :, None, None]
        fold, live = (s["route"][:, i] != 1)[..., None], (i < s["n_nodes"])[:, None, None]
        u = s["beta"][:, i].double()[..., None] * (v[:, i] - torch.einsum("bhd,bhdc->bhc", kl[:, i], before)) * fold
        states.append(before + kl[:, i][..., None] * u[:, :, None, :])
        above.append(mine)
        o_la = s["scale_la"] * torch.einsum("bhd,bhdc->bhc", ql[:, i], states[-1])
        o_la = o_la / (o_la.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        o = []
        for a in range(G):
            cols = slice(a * ds, (a + 1) * ds)
            qa = s["scale_sm"] * qs[:, i, :, cols]
            x = torch.einsum("bhd,bhnd->bhn", qa, kc[:, :, :, a]).masked_fill(~seen, -math.inf)
            y = torch.einsum("bhd,bthd->bht", qa, ks[..., cols])
            x = torch.cat([x, y.masked_fill(~(mine[:, None] & (_heads(s["route"]) != 0)), -math.inf)], -1)
            lse = torch.logsumexp(x, -1)
            p = torch.exp(x - lse.masked_fill(lse == -math.inf, 0.0)[..., None])
            oa = torch.einsum("bhn,bhnd->bhd", p[..., :at.numel()], vc[:, :, :, a])
            oa = oa + torch.einsum("bht,bthd->bhd", p[..., at.numel():], v[..., cols])
            o.append(oa / (oa.pow(2).mean(-1, keepdim=True) + EPS).sqrt())
            lse_all[:, :, a, i] = torch.where(live[..., 0], lse, 0.0)
        w = s["w"][:, i].double()
        out[:, i] = (w[..., :1] * torch.cat(o, -1) + w[..., 1:] * o_la) * live
        u_all[:, i] = u * live
    return dict(out=out, u=u_all, lse=lse_all if G > 1 else lse_all[:, :, 0])
