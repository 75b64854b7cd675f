"""What the Python side of the attention operators hands to the library, and which calls it takes, on the CPU."""
import ctypes as C

import pytest
import torch

from paper_2011_14486_amd import binding as vf


class Thing:
    pass


def handed(monkeypatch, fn, *args, fmt=vf.VF_BF16, **more):
    """The arguments that the library would get for a call on CPU tensors, and the call's result."""
    ctx, cache, seen = Thing(), Thing(), []
    ctx.torch, ctx.device = torch, torch.device("cpu")
    ctx.empty = lambda shape, dtype: torch.empty(shape, dtype=dtype)
    cache.device, cache.head_dim, cache.kv_heads, cache.page, cache.fmt, cache.tensors, cache.ref = ctx.device, 64, 2, 16, fmt, (), None
    monkeypatch.setattr(vf, "lib", lambda: C.CDLL(vf.LIB_PATH))
    monkeypatch.setattr(vf, "_call", lambda c, f, a, tensors: seen.append(a))
    out = fn(ctx, cache, *args, **more)
    return seen[0], out


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("window", [0, 1, 100, (1 << 31) - 1])
def test_a_window_without_causality_is_none(monkeypatch, window):
    """Where every row sees all keys a window has no meaning: the library, which refuses the two together, gets none."""
    q = torch.zeros((6, 512), dtype=torch.bfloat16)
    for causal, want in ((True, window), (False, 0)):
        a, _ = handed(monkeypatch, vf.vf_kv_attend, q, i32(3, 4), i32(3), causal=causal, window=window)
        assert a[6:8] == (1 if causal else 0, want)
    for bad in (-1, 1 << 31):
        with pytest.raises(ValueError):
            handed(monkeypatch, vf.vf_kv_attend, q, i32(3, 4), i32(3), causal=False, window=bad)
