"""Scratch of exactly the size that the header asks for, and what lies behind it."""
import numpy as np
import pytest
import torch

import test_gpu_operators as P8
from gpu_util import TDT, ok, stream
from paper_2510_05186_amd import binding as B

pytestmark = pytest.mark.gpu
GPT, LLAMA, FP32, BF16 = 0, 1, 0, 1


@pytest.mark.parametrize("dtype,family,rows,h", [(BF16, GPT, 1, 8192), (BF16, GPT, 255, 8192), (BF16, LLAMA, 257, 8192), (BF16, GPT, 700, 4104), (FP32, GPT, 600, 8192), (FP32, GPT, 300, 4100),
                                                 (BF16, GPT, 3000, 520), (BF16, GPT, 17, 64), (FP32, LLAMA, 2100, 1000), (BF16, LLAMA, 5000, 2040)])
def test_norm_gradient_s_partial_sums(dtype, family, rows, h):
    """2 * min(rows, 256) * hidden floats: twice the same bits, with other values left there.  A column's sum: a wave's rows one after the other (at most
    rows / 64 of them from 64 rows on, 64 below), the waves of a workgroup, 256 rows of sums by eight and over 32 lanes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + h)
    x, dn, gamma, beta = (torch.randn(s, generator=g, device="cuda").to(TDT[dtype]) for s in ((rows, h), (rows, h), (h,), (h,)))
    out, dx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((rows, 2), device="cuda")
    codes, scales, whole = P8.kept(rows, h)
    ok(B.lib().optstage_op_norm_fwd_pack8(dtype, family, x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), out.data_ptr(), stats.data_ptr(), codes.data_ptr(), scales.data_ptr(), rows, h,
                                          1e-5, stream()))
    got = []
    for fill in (float("nan"), 7.0):
        partial, untouched = P8.zone((2 * min(rows, 256) * h,), torch.float32, fill)
        grads, also = P8.zone((2, h), torch.float32, 0.0)
        ok(B.lib().optstage_op_norm_bwd8(dtype, family, dn.data_ptr(), codes.data_ptr(), scales.data_ptr(), stats.data_ptr(), gamma.data_ptr(), beta.data_ptr(), 0, dx.data_ptr(), 0,
                                         partial.data_ptr(), grads[0].data_ptr(), grads[1].data_ptr(), rows, h, stream()))
        torch.cuda.synchronize()
        assert untouched() and also() and whole()
        got.append(grads.clone())
    assert torch.equal(*got) and bool(torch.isfinite(got[0]).all())
    if family == GPT:
        want = dn.double().sum(0)
        assert float(((got[0][1] - want).abs() - (rows / 64 + 80) * 2.0 ** -24 * dn.double().abs().sum(0)).max()) <= 0
    else:
        assert not got[0][1].any()


def test_query_and_key_gradient_s_partial_sums():
    """2 * min(rows, 1024) * head_dim floats, for rows of so many heads that every workgroup is used."""
    for rows in (3, 1023, 1025, 3000):
        H = P8.Heads(BF16, rows, 64, 32, 4, 128)
        y, dx = torch.empty_like(H.X), torch.empty_like(H.X)
        H.fwd(H.X, y, True)
        got = []
        for fill in (float("nan"), 7.0):
            H.partial.fill_(fill)
            H.reset()
            H.bwd(H.DY, None, dx)
            torch.cuda.synchronize()
            got.append(H.DG.clone())
        assert H.untouched() and torch.equal(*got) and np.isfinite(got[0].cpu().numpy()).all()
