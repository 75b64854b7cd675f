"""GPU: sequences in chunks at the edges of what fp32 and the operands' 16 bits hold, against the recurrence in 64 bits.
Tolerances are those of test_gpu_ssm."""
import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("lens", [[32, 64, 100], [1100]], ids=str)
@pytest.mark.parametrize("large,small,a", [(60.0, -4.0, None), (1000.0, -4.0, None), (1e35, -10.0, -1e4)], ids=str)
def test_small_steps_behind_large_ones(vf, ctx, sizes, lens, large, small, a):  # noqa: F811
    """Steps that make the state forget, then small ones within the same chunk of 32 tokens: what counts are the decays of the small
    ones alone, which are to be as exact as if the large ones were not there.  (1e35 times -1e4 is infinite in 32 bits.)"""
    c = Case(vf, sizes, lens, "bf16", plain=True, seed=8)
    if a is not None:
        c.layer.tensors[2].fill_(a)
        c.lay["a"][:] = a
    rng = np.random.default_rng(9)
    c.dt[:] = small
    for first, count in zip(c.first, c.lens):
        for chunk in range(first, first + count, 32):
            at = chunk + rng.choice(16, 3, replace=False) + 16 * int(rng.integers(0, 2))   # in a chunk's first or second half
            c.dt[at[at < first + count].tolist()] = large
    new = c.layer.state(len(lens), c.dtype)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), longest=max(lens), offsets=c.offsets, state_out=new)
    c.check(out, c.ref(), True, new)


@pytest.mark.parametrize("sizes", [(4, 64, 1, 64, 3), (2, 64, 2, 128, 2), (3, 48, 1, 32, 1), (1, 16, 1, 256, 3), (4, 32, 2, 64, 4)], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
def test_c_that_is_not_finite_reaches_the_tokens_that_see_it(vf, ctx, sizes, value):  # noqa: F811
    """A column of C at one token is met by the W tokens of the convolution's window from there on, by the heads of its group, and
    nobody else: it does not go into the state."""
    H, P, G, N, W = sizes
    c = Case(vf, sizes, [40, 70], "bf16", seed=6)
    args = dict(n_seq=2, longest=70, offsets=c.offsets)
    clean = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
    for at in (9, 31, 40 + 30, 40 + 63):
        col = H * P + G * N + (G - 1) * N + 5
        kept = c.xbc[at, col].clone()
        c.xbc[at, col] = value
        hurt = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
        c.xbc[at, col] = kept
        seen = torch.zeros_like(clean, dtype=torch.bool)
        seen[at:min(at + W, 40 if at < 40 else 110), H // G * (G - 1) * P:] = True
        assert torch.equal(hurt[~seen], clean[~seen])
        if value != value:
            assert bool(hurt[seen].isnan().all())


@pytest.mark.parametrize("sizes", SIZES + [(7, 16, 1, 160, 3)], ids=str)
@pytest.mark.parametrize("lens", [[20, 50, 33], [1100]], ids=str)
def test_outputs_behind_a_state(vf, ctx, sizes, lens):  # noqa: F811
    """Inputs of zeros, small steps: outputs are the products of the state that the sequences began from with C.  Both are in two parts
    of bf16: what is left out of either, and the product of the two second parts, is 2^-16 each."""
    c = Case(vf, sizes, lens, "bf16", plain=True, slots=len(lens), seed=11)
    H, P, G, N, W = sizes
    c.state[0][:, :H * P] = 0
    c.xbc[:, :H * P] = 0
    c.dt[:] = -9.0
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), longest=max(lens), offsets=c.offsets, state=c.state)
    want, _, _, omag, _ = c.ref()
    err = np.abs(out.double().cpu().numpy() - want)
    tol = (3 * 2.0 ** -16 + (128 + max(lens) + N) * 2.0 ** -24) * omag + 2.0 ** -8 * np.abs(want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("lens", [[32, 64, 100], [1100]], ids=str)
@pytest.mark.parametrize("large", [1000.0, 1e6, 1e12], ids=str)
def test_large_steps_that_meet_zeros(vf, ctx, sizes, lens, large):  # noqa: F811
    """A large step where all of x is zero clears the state and adds nothing: what small steps (1.2e-4) add in the same chunk is as
    exact as without it."""
    c = Case(vf, sizes, lens, "bf16", plain=True, seed=12)
    H, P, G, N, W = sizes
    rng = np.random.default_rng(13)
    c.dt[:] = -9.0
    for first, count in zip(c.first, c.lens):
        for chunk in range(first, first + count, 32):
            t = min(chunk + int(rng.integers(0, 28)), first + count - 1)
            c.dt[t] = large
            c.xbc[max(t - W + 1, first):t + 1, :H * P] = 0.0
    new = c.layer.state(len(lens), c.dtype)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), longest=max(lens), offsets=c.offsets, state_out=new)
    c.check(out, c.ref(), True, new)
