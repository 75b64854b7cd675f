"""GPU: the state-space value network captured into a graph and replayed with other inputs between eager calls."""
import numpy as np
import pytest

from tests.test_gpu_ssm_value_slots import F, WIDTH, vf  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what,n", [("extend", 40), ("extend", 3000), ("score", 40), ("score", 3000), ("ranges", 40), ("ranges", 5000)])
def test_replays_equal_eager_calls(vf, what, n):  # noqa: F811
    import torch
    from paper_2011_14486_amd import inputs, ssm
    side = torch.cuda.Stream()
    ctx = vf.vf_create(0, stream=side)
    net = ssm.SsmValue(ctx, inputs.ssm_weights(F, WIDTH, 2, 2, 32, 1, 16, 4, seed=2))
    rng = np.random.default_rng(n)
    dev = lambda v, t: torch.from_numpy(np.ascontiguousarray(v)).to(t).cuda()   # noqa: E731
    lens = rng.integers(0, 9, n) if what == "ranges" else np.full(n, 1 if what == "extend" else 10)
    x0 = dev(rng.standard_normal((int(lens.sum()), F)), torch.bfloat16)
    offsets = dev(np.concatenate([[0], np.cumsum(lens)]), torch.int32)
    slots, to = dev(rng.integers(-1, 50, n), torch.int32), dev(np.where(rng.random(n) < 0.2, -1, rng.permutation(n)), torch.int32)
    first, left = net.state(50), net.state(n)
    net.score(dev(rng.standard_normal((200, F)), torch.bfloat16), n_seq=50, state_out=first)
    call = lambda x: (net.extend(x, first, slots, left, to) if what == "extend" else   # noqa: E731
                      net.score(x, n, 10, offsets if what == "ranges" else None, first, slots, left, to))
    x = x0.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = call(x)
    for k in (1.0, 0.5, 1.0, -2.0, 0.25):
        x.copy_(x0 * k)
        left.total.zero_()
        g.replay()
        replayed, total = got.clone(), left.total.clone()
        torch.cuda.synchronize()
        eager = call(x0 * k)
        torch.cuda.synchronize()
        assert torch.equal(replayed, eager) and torch.equal(total, left.total)
        x0.float().sum().item()
    vf.vf_destroy(ctx)
