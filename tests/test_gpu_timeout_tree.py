"""The time-out path of the tree step beyond 32 nodes and of the cache weights of more than 16 rows, exercised without a fault and
without a hang: natsl_debug_set_wait_limit shortens the bound of every wait to a few milliseconds and withholds arrivals that
other warps wait for (a barrier that nothing completes).  All of a CTA's parts then give up, let what is in flight land,
free tensor memory and return; the next call is right."""
import numpy as np
import pytest
import torch

from test_gpu_evict import case, logits
from test_gpu_parity import dev
from test_gpu_tree import SENTINEL, call, check, reference, scales, step
from tree_cases import make

pytestmark = pytest.mark.gpu


@pytest.fixture
def short_waits():
    """A call of it runs f with arrivals withheld and waits of about 4 ms, and says how long that took (ms)."""
    from paper_2602_03681_b200 import binding

    def run(f):
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        try:
            binding.natsl_debug_set_wait_limit(8192, withhold_scan_flags=True)       # 8 M cycles
            t0.record()
            f()
            t1.record()
            torch.cuda.synchronize()
        finally:
            binding.natsl_debug_set_wait_limit(0, withhold_scan_flags=False)
        return t0.elapsed_time(t1)

    return run


@pytest.mark.parametrize("d,G,norm", [(128, 1, False), (128, 1, True), (128, 2, True), (128, 2, False), (64, 1, True), (64, 2, False)])
@pytest.mark.parametrize("B,H,cap", [(2, 2, 300), (7, 5, 1200)])
def test_tree_step(d, G, norm, B, H, cap, short_waits):
    """Few tiles a CTA and more than the ring holds.  A pair without a cache waits for nothing, and neither does the tree's own
    part: they are right all the same."""
    from paper_2602_03681_b200 import binding
    x = make(d + G, B, H, 40, d, [cap, 0, 65, cap - 1], cap, "bf16", unit=not norm, nodes=[40, 35])
    t = call(x, "bf16", G=G, norm=norm)
    check(t, reference(x, G, norm), "bf16")
    first = {m: t[m].clone() for m in ("out", "u", "lse")}
    for m in first:
        t[m].fill_(SENTINEL)
    took = short_waits(lambda: step(t))
    assert binding.natsl_device_status(t["ws"]) == binding.ERR_TIMEOUT
    assert took < 1000.0                             # the bound, not the default two seconds
    assert torch.equal(t["u"], first["u"])
    live = torch.arange(40, device="cuda") < t["n_nodes"][:, None]
    assert (t["out"][~live] == SENTINEL).all()
    for b, h in np.argwhere(x["cache_len"] == 0):
        assert torch.equal(t["out"][b, :, h], first["out"][b, :, h])
    step(t)
    assert binding.natsl_device_status(t["ws"]) == 0
    assert all(torch.equal(t[m], y) for m, y in first.items())


@pytest.mark.parametrize("d,G,norm", [(128, 1, False), (128, 1, True), (128, 2, True), (128, 2, False), (64, 1, True), (64, 2, False)])
@pytest.mark.parametrize("T", [40, 200])
def test_cache_weights(d, G, norm, T, short_waits):
    """One tile of rows and several.  There is no status word: every entry below the length gets a NaN."""
    from paper_2602_03681_b200 import binding
    x = case(T + d, 2, 2, T, d, [600, 0, 129, 311], 620, "bf16", G, norm)
    la, sm = scales(d, G, norm)
    q, kc = dev(x["q"], torch.bfloat16), dev(x["k_cache"], torch.bfloat16)
    lse, visible, n = dev(x["lse"] if G > 1 else x["lse"][:, :, 0]), dev(x["visible"]), dev(x["cache_len"])
    p = binding.make_params(2, 2, T, d, binding.NATSL_BF16, la, sm, flags=binding.QK_NORM if norm else 0, G=G,
                            norm_eps=1e-6 if norm else 0.0)
    was = dev(x["weight"])
    first, held, again = was.clone(), was.clone(), was.clone()
    binding.natsl_cache_weights(q, lse, visible, kc, n, first, p)
    torch.cuda.synchronize()
    took = short_waits(lambda: binding.natsl_cache_weights(q, lse, visible, kc, n, held, p))
    assert took < 1000.0
    inside = torch.arange(620, device="cuda") < n[:, :, None]
    assert torch.isnan(held[inside]).all() and torch.equal(held[~inside], was[~inside])
    binding.natsl_cache_weights(q, lse, visible, kc, n, again, p)
    assert torch.equal(again, first) and torch.isfinite(first).all()
