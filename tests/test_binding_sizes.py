"""What the binding refuses of the calls of speculative generation and of a bounded cache before a kernel sees an address: a tensor
that is too small for the parameters, caches and weights of different capacities, whole numbers beyond 32 bits.  With tensors
of this host: what is not refused for its size is refused for lying there, and nothing is ever launched."""
import numpy as np
import pytest
import torch

from paper_2602_03681_b200 import binding, build

SHAPE = -2
B, H, L, D, CAP, KEEP = 2, 3, 5, 64, 40, 20


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def tensors(code, G=1, **change):
    """Every tensor of the four calls, as natsl.h has it."""
    dt = torch.bfloat16 if code == binding.NATSL_BF16 else torch.float32
    i32, f32 = torch.int32, torch.float32
    sizes = dict(q=((B, L, H, D), dt), k=((B, L, H, D), dt), v=((B, L, H, D), dt), g=((B, L, H), f32), beta=((B, L, H), f32),
                 route=((B, L, H), torch.uint8), parent=((B, L), i32), n_nodes=((B,), i32), state=((B, H, D, D), f32),
                 k_cache=((B, H, CAP, D), dt), v_cache=((B, H, CAP, D), dt), cache_len=((B, H), i32), out=((B, L, H, D), dt),
                 u=((B, L, H, D), f32), path=((B, L), i32), n_path=((B,), i32), lse=((B, H, G, L), f32), visible=((B, L, H), i32),
                 weight=((B, H, CAP), f32), kept=((B, H, KEEP), i32))
    sizes.update(change)
    return {n: None if s is None else torch.zeros(s[0], dtype=s[1]) for n, s in sizes.items()}


CALLS = {
    "tree_step": "q k v g beta route parent n_nodes state k_cache v_cache cache_len out u",
    "tree_commit": "k v g route u path n_path state k_cache v_cache cache_len",
    "cache_weights": "q lse visible k_cache cache_len weight",
    "cache_evict": "k_cache v_cache weight cache_len kept",
}


def call(name, t, code, G=1, keep=KEEP, first=1, recent=2):
    p = binding.make_params(B, H, L, D, code, 1.0, 1.0, G=G)
    args = [t[n] for n in CALLS[name].split()]
    if name == "cache_evict":
        args[-1:] = [keep, first, recent, args[-1], p]
    else:
        args.append(p)
    if name in ("tree_step", "tree_commit"):
        args.append(torch.zeros(256, dtype=torch.uint8))
    getattr(binding, "natsl_" + name)(*args)


def refused(name, t, code, **kw):
    with pytest.raises(binding.NatslError) as e:
        call(name, t, code, **kw)
    assert e.value.status == SHAPE


def passed_on(name, t, code, **kw):
    """As far as a tensor's place: the next thing that is looked at."""
    with pytest.raises(AssertionError, match="device-resident"):
        call(name, t, code, **kw)


@pytest.mark.parametrize("code", [binding.NATSL_F32, binding.NATSL_BF16])
@pytest.mark.parametrize("name", CALLS)
def test_tensors_that_are_too_small(name, code):
    passed_on(name, tensors(code), code)
    dtypes = tensors(code)
    for n in CALLS[name].split():
        shape = list(dtypes[n].shape)
        for axis in range(len(shape)):                        # one element, row, head, ... less
            less = shape[:axis] + [shape[axis] - 1] + shape[axis + 1:]
            if n == "k_cache" and axis == 2 and name == "cache_weights":
                continue                                      # (a capacity of its own: weight is then the odd one)
            refused(name, tensors(code, **{n: (less, dtypes[n].dtype)}), code)
        if dtypes[n].dtype != torch.uint8:                    # elements of half their size
            half = torch.int16 if dtypes[n].element_size() == 4 else torch.int8
            refused(name, tensors(code, **{n: (shape, half)}), code)


@pytest.mark.parametrize("name", CALLS)
def test_room_for_more_is_no_mistake(name):
    """Buffers for a larger batch, of which a call uses the front; optional tensors left out."""
    code = binding.NATSL_BF16
    t = tensors(code)
    passed_on(name, tensors(code, **{n: ((B + 1, *t[n].shape[1:]), t[n].dtype) for n in CALLS[name].split()}), code)
    passed_on(name, tensors(code, n_nodes=None, visible=None, u=None if name == "tree_step" else ((B, L, H, D), torch.float32)), code)


@pytest.mark.parametrize("name,other", [("tree_step", "v_cache"), ("tree_commit", "v_cache"), ("cache_evict", "v_cache"),
                                        ("cache_weights", "weight"), ("cache_evict", "weight")])
def test_capacities_that_differ(name, other):
    code = binding.NATSL_BF16
    t = tensors(code)[other]
    shape = list(t.shape)
    shape[2] = CAP + 1
    refused(name, tensors(code, **{other: (shape, t.dtype)}), code)
    refused(name, tensors(code, k_cache=((B, H, CAP + 1, D), torch.bfloat16)), code)


def test_lists_and_rows_of_other_widths():
    code = binding.NATSL_F32
    refused("cache_evict", tensors(code, kept=((B, H, KEEP + 1), torch.int32)), code)
    refused("tree_step", tensors(code, k_cache=((B, H, CAP, 2 * D), torch.float32), v_cache=((B, H, CAP, 2 * D), torch.float32)), code)
    refused("cache_weights", tensors(code), code, G=2)        # (log-sum-exps of one head)
    passed_on("cache_weights", tensors(code, G=2), code, G=2)


@pytest.mark.parametrize("which", ["keep", "first", "recent"])
@pytest.mark.parametrize("by", [2 ** 32, -2 ** 32, 2 ** 31])
def test_whole_numbers_beyond_32_bits(which, by):
    code = binding.NATSL_F32
    n = dict(keep=KEEP, first=1, recent=2)
    n[which] += by
    refused("cache_evict", tensors(code), code, **n)
    with pytest.raises(OverflowError):
        call("cache_evict", tensors(code), code, **{**n, which: 2 ** 70})


@pytest.mark.parametrize("name", CALLS)
def test_what_is_missing_or_no_tensor(name):
    """Not a question of sizes: these go on to the checks that were there."""
    code = binding.NATSL_F32
    first = CALLS[name].split()[0]
    t = tensors(code)
    t[first] = np.zeros(3)
    with pytest.raises(TypeError):
        call(name, t, code)
    t = tensors(code, k_cache=((B, CAP), torch.float32))
    with pytest.raises((AssertionError, IndexError)):
        call(name, t, code)
