"""fp64 CPU oracle of generation over a tree of drafted tokens and of a cache that stays bounded -- TEST INFRASTRUCTURE
ONLY (see the package docstring for who may import it).

Written node by node from the definitions: a node's state is its parent's after one step of the gated delta rule (Section
4.3), its softmax reads the cache and the retained tokens of its own path (Section 4.1), nothing of any other node.  With
grouped softmax heads and normalised q, k as in ``grouped.py``.  numpy, float64, no batching over nodes."""
from __future__ import annotations

import numpy as np


def _rows(x, G, qk_norm, norm_eps):
    """[..., d] -> (as the linear operation sees it [..., d], as the softmax heads see it [..., G, d / G])."""
    x = np.asarray(x, np.float64)
    s = x.reshape(*x.shape[:-1], G, x.shape[-1] // G)
    if not qk_norm:
        return x, s
    return (x / np.sqrt((x * x).sum(-1, keepdims=True) + norm_eps),
            s / np.sqrt((s * s).mean(-1, keepdims=True) + norm_eps))


def tree_step(q, k, v, g, beta, route, w, parent, n_nodes, state, k_cache, v_cache, cache_len, *, scale_la, scale_sm, eps=1e-5,
              G=1, qk_norm=False, norm_eps=1e-6):
    """q,k,v [B,T,H,d]; g,beta,route [B,T,H]; w [B,T,H,2] or None; parent [B,T]; n_nodes [B] or None.  Returns dict(out, u
    [B,T,H,d], lse [B,H,G,T]); rows behind a tree's last node are NaN."""
    B, T, H, d = np.asarray(q).shape
    out, u_all = np.full((B, T, H, d), np.nan), np.full((B, T, H, d), np.nan)
    lse = np.full((B, H, G, T), np.nan)
    (ql, qs), (kl, ks) = _rows(q, G, qk_norm, norm_eps), _rows(k, G, qk_norm, norm_eps)
    v = np.asarray(v, np.float64)
    vs = v.reshape(B, T, H, G, d // G)
    for b in range(B):
        for h in range(H):
            n = int(cache_len[b, h])
            kc = _rows(k_cache[b, h, :n], G, qk_norm, norm_eps)[1]
            vc = np.asarray(v_cache[b, h, :n], np.float64).reshape(n, G, d // G)
            states, paths = [], []
            for i in range(T if n_nodes is None else int(n_nodes[b])):
                p = int(parent[b, i])
                S = (states[p] if p >= 0 else np.asarray(state[b, h], np.float64)) * np.exp(np.float64(g[b, i, h]))
                path = (paths[p] if p >= 0 else []) + [i]
                r = int(route[b, i, h])
                u = np.zeros(d)
                if r != 1:
                    u = float(beta[b, i, h]) * (v[b, i, h] - kl[b, i, h] @ S)
                    S = S + np.outer(kl[b, i, h], u)
                states.append(S)
                paths.append(path)
                o_la = scale_la * (ql[b, i, h] @ S)
                seen = [j for j in path if route[b, j, h]]
                o = np.zeros((G, d // G))
                for s in range(G):
                    keys = np.concatenate([kc[:, s], ks[b, seen, h, s]])
                    vals = np.concatenate([vc[:, s], vs[b, seen, h, s]])
                    lse[b, h, s, i] = -np.inf
                    if len(keys):
                        x = scale_sm * (keys @ qs[b, i, h, s])
                        e = np.exp(x - x.max())
                        lse[b, h, s, i] = x.max() + np.log(e.sum())
                        o[s] = e @ vals / e.sum()
                y = (o / np.sqrt((o * o).mean(-1, keepdims=True) + eps)).reshape(d)
                wn, wl = (0.5, 0.5) if w is None else (float(w[b, i, h, 0]), float(w[b, i, h, 1]))
                out[b, i, h] = wn * y + wl * o_la / np.sqrt((o_la * o_la).mean() + eps)
                u_all[b, i, h] = u
    return dict(out=out, u=u_all, lse=lse)


def tree_commit(k, v, g, beta, route, path, n_path, state, k_cache, v_cache, cache_len, *, qk_norm=False, norm_eps=1e-6):
    """The accepted tokens one after the other; state, k_cache, v_cache, cache_len are updated in place.  A pair whose
    cache has no room is left untouched."""
    B, T, H, d = np.asarray(k).shape
    kl = _rows(k, 1, qk_norm, norm_eps)[0]
    for b in range(B):
        nodes = [int(i) for i in path[b][:int(n_path[b])]]
        for h in range(H):
            if int(cache_len[b, h]) + sum(int(route[b, i, h]) != 0 for i in nodes) > k_cache.shape[2]:
                continue
            for i in nodes:
                S = state[b, h] * np.exp(np.float64(g[b, i, h]))
                if route[b, i, h] != 1:
                    S = S + float(beta[b, i, h]) * np.outer(kl[b, i, h], np.asarray(v[b, i, h], np.float64) - kl[b, i, h] @ S)
                state[b, h] = S
                if route[b, i, h]:
                    k_cache[b, h, cache_len[b, h]] = k[b, i, h]
                    v_cache[b, h, cache_len[b, h]] = v[b, i, h]
                    cache_len[b, h] += 1


def cache_weights(q, lse, visible, k_cache, cache_len, weight, *, scale_sm, G=1, qk_norm=False, norm_eps=1e-6):
    """q [B,T,H,d]; lse [B,H,G,T]; visible [B,T,H] or None; returns the new weights [B,H,cap]."""
    B, T, H, d = np.asarray(q).shape
    weight = np.array(weight, np.float64)
    qs = _rows(q, G, qk_norm, norm_eps)[1]
    for b in range(B):
        for h in range(H):
            n = int(cache_len[b, h])
            kc = _rows(k_cache[b, h, :n], G, qk_norm, norm_eps)[1]
            for t in range(T):
                m = n if visible is None else max(0, min(n, int(visible[b, t, h])))
                for s in range(G):
                    if np.isfinite(lse[b, h, s, t]):
                        weight[b, h, :m] += np.exp(scale_sm * (kc[:m, s] @ qs[b, t, h, s]) - lse[b, h, s, t])
    return weight


def evict(weight, n, keep, first, recent):
    """The places of the entries of one cache that stay, ascending: weight [n]."""
    if n <= keep:
        return list(range(n))
    w = [-np.inf if np.isnan(x) else float(x) for x in weight[:n]]
    low = [bool(np.isnan(x)) for x in weight[:n]]                     # (below everything, minus infinity included)
    between = sorted(range(first, n - recent), key=lambda j: (low[j], -w[j], j))
    return sorted([*range(first), *range(n - recent, n), *between[:keep - first - recent]])
