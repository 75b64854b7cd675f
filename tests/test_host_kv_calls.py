"""What the Python side of the attention operators hands to the library, and which calls are taken, on the CPU."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, ROOT)

from paper_2011_14486_amd import binding as vf  # noqa: E402
from tests.test_host_kv import EINVAL, OK, P, call, library, make_library  # noqa: E402
from tests.test_host_ops import stub_path  # noqa: E402, F401


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


def test_rows_are_read_as_the_cache_holds_them(monkeypatch):
    """Without a type rows come out in the cache's own, those of 8 bits in bf16: nothing is rounded unasked."""
    where = i32(3, 4), i32(3), 6
    for fmt, kind, dtype in ((vf.VF_FP32, vf.VF_FP32, torch.float32), (vf.VF_BF16, vf.VF_BF16, torch.bfloat16), (vf.VF_E4M3, vf.VF_BF16, torch.bfloat16)):
        a, out = handed(monkeypatch, vf.vf_kv_read, *where, fmt=fmt)
        assert a[2] == kind and all(t.dtype == dtype for t in out)
        own = torch.empty((6, 128), dtype=dtype), None
        assert handed(monkeypatch, vf.vf_kv_read, *where, fmt=fmt, out=own)[1] is own
        for asked, dt in ((vf.VF_FP32, torch.float32), (vf.VF_BF16, torch.bfloat16)):
            a, out = handed(monkeypatch, vf.vf_kv_read, *where, fmt=fmt, out_type=asked)
            assert a[2] == asked and all(t.dtype == dt for t in out)


def in_place(stub, vf, ctx):  # noqa: F811
    """Outputs in the queries' place have the queries' row distance: with another one rows would lie over queries that are still to be read."""
    stub.stub_clear()
    for other in (513, 1024):
        assert call(vf, ctx, "attend", out=5 * P, ldo=other) == EINVAL
        assert call(vf, ctx, "attend", out=5 * P, ldo=other, n_seq=1, tokens=300) == EINVAL
    assert stub.stub_log() == b""
    assert call(vf, ctx, "attend", out=5 * P) == OK
    assert call(vf, ctx, "attend", out=5 * P, ldq=1024, ldo=1024) == OK
    assert call(vf, ctx, "attend", out=5 * P, ldo=1024, n_seq=1, tokens=1) == OK   # (one row has no distance)
    assert call(vf, ctx, "attend", out=5 * P, ldo=1024, n_seq=1, tokens=0) == OK


@pytest.mark.parametrize("case", ["in_place"])
def test_on_a_runtime_without_a_gpu(stub_path, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub_path, case], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    globals()[sys.argv[2]](*library(*make_library(sys.argv[1])))
