"""GPU: sequences in chunks at the edges of what fp32 and the operands' 16 bits hold, against the recurrence in 64 bits.
Tolerances are those of test_gpu_ssm."""
import numpy as np
import pytest

from tests.test_gpu_ssm import Case, ctx, vf  # noqa: F401

pytestmark = pytest.mark.gpu

# (H, P, G, N, W): both forms of the chunks, with full and with filled-up tiles
SIZES = [(4, 64, 1, 64, 4), (2, 64, 1, 128, 4), (3, 48, 1, 32, 4), (1, 16, 1, 256, 4)]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("lens", [[100], [70, 40], [1100]], ids=str)
@pytest.mark.parametrize("size", [0.0, 1e-36])
def test_rows_of_zeros_behind_large_steps(vf, ctx, sizes, lens, size):  # noqa: F811
    """Channels of x that are zero, or next to it, over whole chunks, and steps of 60: a state of zeros stays zeros, small ones are
    as exact as others.  (1100 tokens run in segments.)"""
    c = Case(vf, sizes, lens, "bf16", plain=True, seed=7)
    P = sizes[1]
    c.xbc[:, 3] = size
    c.xbc[:, P - 2] = -size
    c.dt[:] = 60.0
    new = c.layer.state(len(lens), c.dtype)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), longest=max(lens), offsets=c.offsets, state_out=new)
    c.check(out, c.ref(), True, new)
    if size == 0:
        assert not out[:, [3, P - 2]].any() and not new[1][:, 0, [3, P - 2]].any()
