"""GPU: matrices without rows, whatever strides they come with."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_no_rows_with_any_strides():
    import torch
    import paper_2011_14486_amd as pkg
    vf = pkg.load()
    ctx = vf.vf_create(0)
    from_numpy = torch.from_numpy(np.zeros((0, 96))).to(torch.bfloat16).cuda()
    across = torch.zeros((96, 5), dtype=torch.bfloat16, device="cuda")[:, :0].t()
    for x in (from_numpy, across):
        assert x.shape == (0, 96)
        y, s = vf.vf_rms_norm(ctx, x, residual=x)
        assert y.shape == (0, 96) and s.shape == (0, 96)
        q = vf.vf_mx_quantize(ctx, x, vf.VF_E4M3)
        assert q.codes.shape == (0, 96) and q.scales.shape == (0, 3)
        assert vf.vf_mx_dequantize(ctx, q, out=x).shape == (0, 96)
        layer = vf.SsmLayer(1, 32, 1, 32, torch.ones((96, 4), device="cuda"), torch.ones(1, device="cuda"))
        assert vf.vf_ssm_scan(ctx, layer, x, x[:, :1], x[:, :32], n_seq=0).shape == (0, 32)
        assert vf.vf_ssm_step(ctx, layer, x, x[:, :1], None).shape == (0, 32)
    # strides that are refused where there are rows
    with pytest.raises(ValueError):
        vf.vf_mx_quantize(ctx, torch.zeros((96, 5), device="cuda").t(), vf.VF_E4M3)
    torch.cuda.synchronize()
    vf.vf_destroy(ctx)
