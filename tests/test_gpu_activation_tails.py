"""The GELU that keeps its input, against its definition value by value in relative terms, far into the lower tail.

The tail of the normal distribution is exp(-x^2 / 2) F(|x|), F a polynomial that falls from 1 / 2 as 0.4 / |x|.  In units of EPS = 2^-24 of the value: the
exponent's argument is rounded three times (1.5 x^2), exp2 2, the fit 2^-22 (4), the products 4; F's reciprocal and multiply-adds 2 EPS outright, which are 4
of F at 0, 20 at -4 and 5 |x| beyond: below 2 x^2 + 40.  The density has the exponent's and 4 more: below 2 x^2 + 8.  bf16: the fit is good to 2^-12, a
sixteenth of the storage type's rounding.  What lies below 2^-126 may be flushed to zero on the way."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

from oracle import operators_fp64 as P
from paper_2510_05186_amd import binding as B
from gpu_util import TDT, host, ok, stream

GPT, FP32, BF16 = 0, 0, 1
EPS, HALF, LEAST = 2.0 ** -24, {FP32: 2.0 ** -24, BF16: 2.0 ** -8}, 2.0 ** -126


def bounds(x, da, dtype):
    """On x cdf(x) and on da (cdf(x) + x density(x)), ahead of the rounding to the storage type"""
    cdf, density = 0.5 * erfc(-x / np.sqrt(2)), np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    n = (EPS * (2 * x * x + 40) + (2.0 ** -12 if dtype == BF16 else 0)) * cdf + LEAST
    return np.abs(x) * n + 2 * EPS * np.abs(x * cdf) + LEAST, np.abs(da) * (n + np.abs(x) * (EPS * (2 * x * x + 8) * density + LEAST) + 2 * EPS * (cdf + np.abs(x) * density)) + LEAST


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gelu_far_into_its_lower_tail(dtype):
    """Random values from -13 to 13 and every value that is kept exactly, forward and backward."""
    r = np.random.default_rng(31)
    kept = np.concatenate([-P.E4M3[::-1], P.E4M3])[None] * np.array([[2.0 ** -5], [2.0 ** -6], [2.0 ** -7]])
    x = np.concatenate([np.resize(kept[0], (2, 256)), np.resize(kept[1], (2, 256)), np.resize(kept[2], (2, 256)), r.uniform(-13, 13, (60, 256)), r.uniform(-13, -4, (60, 256))])
    X = torch.from_numpy(x).to(TDT[dtype]).cuda()
    x = host(X)
    da = host(torch.from_numpy(r.standard_normal(x.shape)).to(TDT[dtype]))
    DA = torch.from_numpy(da).to(TDT[dtype]).cuda()
    rows, f = x.shape
    codes, scales = torch.empty((rows, f), dtype=torch.uint8, device="cuda"), torch.empty((rows, f // 32), dtype=torch.uint8, device="cuda")
    a, again, dgu = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X)
    ok(B.lib().optstage_op_act_fwd_pack8(dtype, GPT, X.data_ptr(), a.data_ptr(), codes.data_ptr(), scales.data_ptr(), rows, f, stream()))
    ok(B.lib().optstage_op_act_bwd8(dtype, GPT, DA.data_ptr(), codes.data_ptr(), scales.data_ptr(), dgu.data_ptr(), again.data_ptr(), rows, f, stream()))
    torch.cuda.synchronize()
    v = P.pack8(x)[2]
    assert v.min() < -12 and x.min() < -12.9
    for what, got, at, ref, b in (("a", a, x, x * 0.5 * erfc(-x / np.sqrt(2)), bounds(x, da, dtype)[0]), ("a again", again, v, v * 0.5 * erfc(-v / np.sqrt(2)), bounds(v, da, dtype)[0]),
                                  ("dgu", dgu, v, da * (0.5 * erfc(-v / np.sqrt(2)) + v * np.exp(-v * v / 2) / np.sqrt(2 * np.pi)), bounds(v, da, dtype)[1])):
        off, b = np.abs(host(got) - ref), HALF[dtype] * np.abs(ref) + b
        bad = ~(off <= b)
        assert not bad.any(), (what, int(bad.sum()), at[bad][:6], host(got)[bad][:6], ref[bad][:6])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gelu_of_what_is_not_finite_and_of_the_largest_values(dtype):
    """As the plain form: infinity stays, what has no limit is NaN, and the largest values are themselves or zero."""
    top = float(torch.finfo(TDT[dtype]).max)
    x = torch.zeros((1, 32), dtype=TDT[dtype], device="cuda")
    x[0, :8] = torch.tensor([np.inf, -np.inf, np.nan, top, -top, 1e20, -1e20, -200.0])
    a, plain = torch.empty_like(x), torch.empty_like(x)
    codes, scales = torch.empty((1, 32), dtype=torch.uint8, device="cuda"), torch.empty((1, 1), dtype=torch.uint8, device="cuda")
    ok(B.lib().optstage_op_act_fwd_pack8(dtype, GPT, x.data_ptr(), a.data_ptr(), codes.data_ptr(), scales.data_ptr(), 1, 32, stream()))
    ok(B.lib().optstage_op_act_fwd(dtype, GPT, x.data_ptr(), plain.data_ptr(), 1, 32, stream()))
    torch.cuda.synchronize()
    assert np.array_equal(host(a), host(plain), equal_nan=True) and np.isinf(host(a)[0, 0]) and np.isnan(host(a)[0, [1, 2]]).all()
    da, dgu = torch.ones_like(x), torch.empty_like(x)
    for v, want in ((torch.full_like(x, top), 1.0), (torch.full_like(x, -top), 0.0), (torch.zeros_like(x), 0.5)):
        ok(B.lib().optstage_op_act_fwd_pack8(dtype, GPT, v.data_ptr(), a.data_ptr(), codes.data_ptr(), scales.data_ptr(), 1, 32, stream()))
        ok(B.lib().optstage_op_act_bwd8(dtype, GPT, da.data_ptr(), codes.data_ptr(), scales.data_ptr(), dgu.data_ptr(), 0, 1, 32, stream()))
        torch.cuda.synchronize()
        assert np.all(host(dgu) == want), (want, host(dgu)[0, 0])
