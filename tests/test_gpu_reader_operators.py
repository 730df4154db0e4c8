"""Rotary positions with several axes, cross attention and the loss against a teacher's top entries against their fp64 definitions, through the C ABI.

Tolerances are bounds per value.  HALF is half a step of the storage type (2^-8 bf16, 2^-24 fp32) of a value, EPS = 2^-24 one fp32 rounding.  What is rounded on the way is
counted at each test."""
import numpy as np
import pytest
import torch

from oracle import operators_fp64 as P
from paper_2510_05186_amd import binding as B
from gpu_util import TDT, dev, host, ok, q, stream

pytestmark = pytest.mark.gpu
FP32, BF16 = 0, 1
EPS, HALF = 2.0 ** -24, {FP32: 2.0 ** -24, BF16: 2.0 ** -8}
TINY = {FP32: 2.0 ** -149, BF16: 2.0 ** -133}            # the least step: results below the normal numbers
FLUSH = 2.0 ** -126                                       # the least normal number: a factor of a product below it may count as 0


def lib():
    return B.lib()


def rng(*key):
    return np.random.default_rng([79, *(int(k) for k in key)])


def zone(shape, dtype, fill=9.0):
    """A tensor with 64 values behind it that nothing may touch -> (tensor, check)"""
    n = int(np.prod(shape))
    flat = torch.full((n + 64,), fill, dtype=dtype, device="cuda")
    tail = flat[n:].clone()
    return flat[:n].view(shape), lambda: torch.equal(flat[n:].view(torch.uint8), tail.view(torch.uint8))


def within(got, ref, bound, what=""):
    got = host(got) if isinstance(got, torch.Tensor) else got
    end = np.where(ref < 0, -np.inf, np.inf)
    ref = np.where(np.abs(ref) > 2.0 ** 128 - 2.0 ** 103, end, ref)      # past the range of either type: rounds to infinity
    over = (np.abs(ref) + bound > 2.0 ** 128 - 2.0 ** 103) & (got == end)      # or a value within the bound does
    same = (got == ref) | (np.isnan(got) & np.isnan(ref)) | over
    with np.errstate(invalid="ignore"):
        d = np.where(same, 0.0, np.abs(got - ref))
    bad = ~(d <= np.broadcast_to(bound, ref.shape)) & ~same
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], np.broadcast_to(bound, ref.shape)[bad][:4])


# ------------------------------------------------------------------ rotary positions with several axes
def rope_case(dtype, rows, n_rot, n_pass, d, axis, n_axes, n_pos, pad=(0, 0), inplace=False, back=0, seed=0, spread=2):
    r = rng(1, dtype, rows, n_rot, d, seed)
    w = (n_rot + n_pass) * d
    ld_src, ld_dst = w + pad[0], w + pad[1]
    x = q(r.standard_normal((rows, ld_src)), dtype)
    pos = r.integers(-spread, n_pos + spread, (n_axes, rows)).astype(np.int32)
    table = torch.zeros((n_pos, d // 2, 2), dtype=torch.float32, device="cuda")
    ok(lib().optstage_op_rope_table(table.data_ptr(), n_pos, d, 10000.0, stream()))
    flat = torch.zeros(n_axes * rows + 1, dtype=torch.int32, device="cuda")       # an address that is a multiple of 4 and no more
    flat[1:] = torch.from_numpy(pos).flatten().cuda()
    if inplace:
        y, whole = zone((rows, ld_src), TDT[dtype])
        y.copy_(dev(x, dtype))
        src, ld_dst = y, ld_src
    else:
        y, whole = zone((rows, ld_dst), TDT[dtype])
        src = dev(x, dtype)
    ok(lib().optstage_op_rope_axes(dtype, src.data_ptr(), ld_src, y.data_ptr(), ld_dst, table.data_ptr(), n_pos, flat[1:].data_ptr(), n_axes, bytes(axis), rows, n_rot, n_pass, d,
                                   back, stream()))
    torch.cuda.synchronize()
    t = table.double().cpu().numpy()
    xin = x[:, :w].reshape(rows, -1, d)
    ref = P.rope_axes(xin, t, pos, axis, n_rot, -1 if back else 1).reshape(rows, w)
    # two products and a sum in fp32 ahead of the one rounding
    partner = np.concatenate([xin[..., d // 2:], xin[..., :d // 2]], 2)
    bound = 2 * EPS * (np.abs(xin) + np.abs(partner)).reshape(rows, w) + HALF[dtype] * np.abs(ref) + TINY[dtype]
    within(host(y)[:, :w], ref, bound, "rope_axes")
    assert np.array_equal(host(y)[:, n_rot * d:w], x[:, n_rot * d:w]), "heads that are passed on"
    assert np.array_equal(host(y)[:, w:], x[:, w:] if inplace else np.full((rows, ld_dst - w), 9.0)) and whole()


AXES = {32: [0] * 3 + [1] * 6 + [2] * 7, 64: [0, 1, 2, 255] * 8, 128: [0] * 13 + [1] * 26 + [2] * 25, 256: [3, 1, 0, 2] * 32, 96: [0] * 48, 16: [1, 0] * 4, 48: [2] * 10 + [1] * 14,
        8: [0, 1, 255, 0]}


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,n_rot,n_pass,d", [(1, 1, 0, 32), (3, 5, 2, 64), (128, 8, 4, 64), (257, 13, 0, 128), (64, 72, 8, 128), (33, 3, 1, 256), (5, 4, 4, 96), (100, 1, 1, 16),
                                                 (17, 40, 3, 48), (1000, 2, 0, 32)])
@pytest.mark.parametrize("inplace,back", [(False, 0), (True, 0), (False, 1), (True, 1)])
def test_rope_axes(dtype, rows, n_rot, n_pass, d, inplace, back):
    rope_case(dtype, rows, n_rot, n_pass, d, AXES[d], 4, 50, (24, 8) if rows % 2 else (0, 0), inplace, back)


@pytest.mark.parametrize("dtype,rows,n_rot,n_pass,d", [(BF16, 2900, 40, 4, 128), (FP32, 1001, 21, 11, 256), (BF16, 16001, 6, 6, 96)])
@pytest.mark.parametrize("inplace,back", [(False, 0), (True, 1)])
def test_rope_axes_of_rows_that_go_past_the_caches(dtype, rows, n_rot, n_pass, d, inplace, back):
    rope_case(dtype, rows, n_rot, n_pass, d, AXES[d], 4, 300, (0, 0), inplace, back)


@pytest.mark.parametrize("n_rot,n_pass", [(1, 0), (3, 2)])
def test_rope_axes_narrow_fp32_heads(n_rot, n_pass):
    rope_case(FP32, 77, n_rot, n_pass, 8, AXES[8], 2, 9, (4, 0))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("axis", [[0, 255, 1, 1] * 16, [0, 0, 255, 255] * 16])
@pytest.mark.parametrize("back", [0, 1])
def test_rope_axes_leaves_what_does_not_turn_whatever_it_holds(dtype, axis, back):
    """NaN, infinities and zeros of both signs in pairs without an axis and in rows whose position lies outside the table; none reaches a pair that turns."""
    rows, heads, d = 60, 5, 128
    r = rng(7, dtype)
    x = torch.from_numpy(r.standard_normal((rows, heads, d))).to(TDT[dtype]).cuda()
    pos = r.integers(0, 9, (2, rows)).astype(np.int32)
    pos[0, ::3], pos[1, 1::4] = -1, 9
    ax = np.array(axis)
    still = np.array([[a == 255 or not 0 <= pos[a][t] < 9 for a in ax] for t in range(rows)])
    mask = torch.from_numpy(np.concatenate([still, still], 1)).cuda()[:, None, :].expand(rows, heads, d)
    odd = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0, 0.0], dtype=TDT[dtype], device="cuda").repeat(rows * heads * d // 5 + 1)[:rows * heads * d].view(rows, heads, d)
    clean = x.clone()
    x = torch.where(mask, odd, x)
    table = torch.zeros((9, d // 2, 2), device="cuda")
    ok(lib().optstage_op_rope_table(table.data_ptr(), 9, d, 10000.0, stream()))
    P0 = torch.from_numpy(pos).cuda()
    outs = []
    for v in (x, clean):
        y = torch.empty_like(v)
        ok(lib().optstage_op_rope_axes(dtype, v.data_ptr(), heads * d, y.data_ptr(), heads * d, table.data_ptr(), 9, P0.data_ptr(), 2, bytes(axis), rows, heads, 0, d, back, stream()))
        outs.append(y)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == BF16 else torch.int32
    assert torch.equal(outs[0].view(bits)[mask], x.view(bits)[mask]) and torch.equal(outs[0][~mask], outs[1][~mask]) and bool(outs[0][~mask].isfinite().all())


def test_rope_axes_far_positions_and_one_axis():
    rope_case(BF16, 40, 4, 4, 128, [0] * 64, 1, 200_000)
    rope_case(FP32, 40, 4, 0, 64, [0] * 32, 1, 1)


def test_rope_axes_agrees_with_the_rotation_by_rows():
    """Every axis at the row's number: bitwise optstage_op_rope's result."""
    rows, seq, nq, nkv, d = 96, 32, 4, 2, 128
    x = torch.randn((rows, (nq + 2 * nkv) * d), device="cuda").bfloat16()
    table = torch.zeros((seq, d // 2, 2), device="cuda")
    ok(lib().optstage_op_rope_table(table.data_ptr(), seq, d, 10000.0, stream()))
    a, b = torch.empty_like(x), torch.empty_like(x)
    pos = (torch.arange(rows, device="cuda") % seq).to(torch.int32).repeat(2, 1).contiguous()
    ok(lib().optstage_op_rope(BF16, x.data_ptr(), a.data_ptr(), table.data_ptr(), rows, seq, nq, nkv, d, 0, stream()))
    ok(lib().optstage_op_rope_axes(BF16, x.data_ptr(), x.shape[1], b.data_ptr(), x.shape[1], table.data_ptr(), seq, pos.data_ptr(), 2, bytes([0, 1] * 32), rows, nq + nkv, nkv, d, 0,
                                   stream()))
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_rope_axes_offsets_beyond_32_bits():
    """Rows that lie 2^31 values and more from the first."""
    rows, d, ld = 70, 64, 1 << 25
    if torch.cuda.mem_get_info()[0] < 12 * 2 ** 30:
        pytest.skip("too little memory free")
    x = torch.zeros((rows, ld), dtype=torch.bfloat16, device="cuda")
    x[:, :2 * d] = torch.randn((rows, 2 * d), device="cuda").bfloat16()
    y = torch.empty((rows, 2 * d), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((rows, d // 2, 2), device="cuda")
    ok(lib().optstage_op_rope_table(table.data_ptr(), rows, d, 10000.0, stream()))
    pos = torch.arange(rows, device="cuda", dtype=torch.int32)
    ok(lib().optstage_op_rope_axes(BF16, x.data_ptr(), ld, y.data_ptr(), 2 * d, table.data_ptr(), rows, pos.data_ptr(), 1, bytes([0] * 32), rows, 1, 1, d, 0, stream()))
    torch.cuda.synchronize()
    xin = host(x[:, :2 * d]).reshape(rows, 2, d)
    ref = P.rope_axes(xin, table.double().cpu().numpy(), [np.arange(rows)], [0] * 32, 1).reshape(rows, -1)
    within(y, ref, HALF[BF16] * np.abs(ref) + 4 * EPS * np.abs(xin).max())


# ------------------------------------------------------------------ cross attention
class Cross:
    """Operands on the device, what the calls give, and the definition with a bound for every value."""

    def __init__(self, dtype, b, nq, nk, hq, hkv, d, lens=None, pad=(0, 0), packed=True, seed=0, size=1.0):
        r = rng(2, dtype, b, nq, nk, hq, d, seed)
        self.shape, self.dtype = (nq, nk, b, hq, hkv, d), dtype
        self.ldq, wk = hq * d + pad[0], hkv * d
        self.ldkv = (2 * wk if packed else wk) + pad[1]
        self.Q = q(size * r.standard_normal((b * nq, self.ldq)), dtype)
        self.KV = q(r.standard_normal((b * nk, self.ldkv)), dtype)
        self.V2 = None if packed else q(r.standard_normal((b * nk, self.ldkv)), dtype)
        self.G = q(r.standard_normal((b * nq, hq * d)), dtype)
        self.lens = np.full(b, nk) if lens is None else np.asarray(lens)
        n = np.clip(self.lens, 0, nk)
        dirty = self.KV.reshape(b, nk, -1).copy(), (self.KV if packed else self.V2).reshape(b, nk, -1).copy()
        for i in range(b):                                       # what lies behind a sequence's states
            for t in dirty:
                t[i, n[i]:, 0::3], t[i, n[i]:, 1::3], t[i, n[i]:, 2::3] = np.nan, np.inf, -np.inf
        self.q, self.g = dev(self.Q, dtype), dev(self.G, dtype)
        self.kv = torch.from_numpy(dirty[0].reshape(b * nk, -1)).to(TDT[dtype]).cuda()
        self.v2 = None if packed else torch.from_numpy(dirty[1].reshape(b * nk, -1)).to(TDT[dtype]).cuda()
        self.kl = None
        if lens is not None:
            self.kl = torch.zeros(b + 1, dtype=torch.int32, device="cuda")[1:]
            self.kl.copy_(torch.from_numpy(self.lens.astype(np.int32)))
        e = self.kv.element_size()
        self.pk = self.kv.data_ptr()
        self.pv = self.kv.data_ptr() + wk * e if packed else self.v2.data_ptr()
        self.wk, self.packed, self.pad = wk, packed, pad
        self.o, self.c_o = zone((b * nq, hq * d), TDT[dtype])
        self.lse, self.c_l = zone((b, hq, nq), torch.float32)
        self.dq, self.c_q = zone((b * nq, self.ldq), TDT[dtype])
        self.dkv, self.c_k = zone((b * nk, self.ldkv), TDT[dtype])
        self.dv2, self.c_v = (None, lambda: True) if packed else zone((b * nk, self.ldkv), TDT[dtype])
        self.pdv = self.dkv.data_ptr() + wk * e if packed else self.dv2.data_ptr()
        nbytes = lib().optstage_op_cross_attn_ws_bytes(dtype, *self.shape)
        self.ws, self.c_w = zone((nbytes,), torch.uint8, 0xA5)

    def fwd(self, at=None):
        ok(lib().optstage_op_cross_attn_fwd(self.dtype, self.q.data_ptr(), self.ldq, self.pk, self.pv, self.ldkv, 0 if self.kl is None else self.kl.data_ptr(), self.o.data_ptr(),
                                            self.lse.data_ptr(), self.ws.data_ptr(), self.ws.numel(), *self.shape, at or stream()))

    def bwd(self, at=None):
        ok(lib().optstage_op_cross_attn_bwd(self.dtype, self.q.data_ptr(), self.ldq, self.pk, self.pv, self.ldkv, 0 if self.kl is None else self.kl.data_ptr(), self.o.data_ptr(),
                                            self.g.data_ptr(), self.lse.data_ptr(), self.dq.data_ptr(), self.dkv.data_ptr(), self.pdv, self.ws.data_ptr(), self.ws.numel(), *self.shape,
                                            at or stream()))

    def outputs(self):
        v = self.dkv[:, self.wk:2 * self.wk] if self.packed else self.dv2[:, :self.wk]
        return {"o": self.o, "lse": self.lse, "dq": self.dq[:, :self.shape[3] * self.shape[5]], "dk": self.dkv[:, :self.wk], "dv": v}

    def untouched(self):
        w = 2 * self.wk if self.packed else self.wk
        assert self.c_o() and self.c_l() and self.c_q() and self.c_k() and self.c_v() and self.c_w()
        assert bool((self.dq[:, self.shape[3] * self.shape[5]:] == 9.0).all()) and bool((self.dkv[:, w:] == 9.0).all())

    def check(self, back=True):
        """Bounds.  A score is a sum of d products in fp32; a weight p = exp(score - lse) is off by e_p of itself: the score's error, the exponent's rounding (fp32, a few
        steps of |score| + |lse|) and the exponential's.  bf16: weights and dS enter the second products rounded (HALF each).  A sum of N products in fp32 is off by N EPS
        of the sum of their sizes.  D = <dout, o> is formed from the stored o.  A weight or a dS below the least normal number has no relative precision left: its
        steps are 2^-149 wide, and the hardware's exponential and products may give 0 for it, so each is off by up to FLUSH besides."""
        nq, nk, b, hq, hkv, d = self.shape
        low = HALF[BF16] if self.dtype == BF16 else 0.0
        store = HALF[self.dtype]
        o, lse = host(self.o).reshape(b, nq, hq, d), host(self.lse)
        if back:
            dq = host(self.dq)[:, :hq * d].reshape(b, nq, hq, d)
            out = self.outputs()
            dk, dv = host(out["dk"]).reshape(b, nk, hkv, d), host(out["dv"]).reshape(b, nk, hkv, d)
        Q, K = self.Q[:, :hq * d].reshape(b, nq, hq, d), self.KV[:, :self.wk].reshape(b, nk, hkv, d)
        V = (self.KV[:, self.wk:2 * self.wk] if self.packed else self.V2[:, :self.wk]).reshape(b, nk, hkv, d)
        G = self.G.reshape(b, nq, hq, d)
        for i in range(b):
            n = min(max(int(self.lens[i]), 0), nk)
            for h in range(hkv):
                k, v = K[i, :n, h], V[i, :n, h]
                rk = rv = bk = bv = np.zeros((n, d))
                for a in range(h * hq // hkv, (h + 1) * hq // hkv):
                    p, L = P.cross_weights(Q[i, :, a], K[i, :, h], n)
                    size = np.abs(Q[i, :, a]) @ np.abs(k).T / np.sqrt(d)
                    if n == 0:
                        assert np.all(lse[i, a] == -np.inf) and not o[i, :, a].any()
                        if back:
                            assert not dq[i, :, a].any()
                        continue
                    e_s = EPS * ((d + 4) * size + 8)
                    e_p = e_s + EPS * 4 * (size + np.abs(L)[:, None]) + EPS * 8
                    within(lse[i, a], L, (p * e_p + FLUSH).sum(1) + EPS * (np.abs(L) + 4) + n * EPS, ("lse", i, a))
                    pv = p @ np.abs(v)
                    within(o[i, :, a], p @ v, (p * e_p + FLUSH) @ np.abs(v) + (p * e_p).sum(1, keepdims=True) * pv + (low + (n + 16) * EPS) * pv + n * EPS * pv + store * np.abs(p @ v) + TINY[self.dtype], ("o", i, a))
                    if not back:
                        continue
                    g = G[i, :, a]
                    dp = g @ v.T
                    D = (p * dp).sum(1, keepdims=True)
                    ds = p * (dp - D)
                    e_D = np.abs((g * o[i, :, a]).sum(1, keepdims=True) - D) + (d + 4) * EPS * (np.abs(g) * np.abs(o[i, :, a])).sum(1, keepdims=True)
                    if self.dtype == BF16 and n <= 64:
                        # few states: D0 = <dout, o> is corrected by the sum of p (dp - D0), off by what its terms and their sum are, and by what the sum of p lacks of one
                        D0 = (g * o[i, :, a]).sum(1, keepdims=True)
                        off = (e_p + (n + d + 16) * EPS) * p
                        e_D = (off * (np.abs(dp - D0) + np.abs(D0))).sum(1, keepdims=True) + (d + 4) * EPS * (p * (np.abs(g) @ np.abs(v).T)).sum(1, keepdims=True) + FLUSH
                        e_D = e_D + (d + 8) * EPS * (np.abs(g) * np.abs(o[i, :, a])).sum(1, keepdims=True)
                    e_ds = np.abs(ds) * (e_p + low + 4 * EPS) + p * (1 + e_p) * (e_D + (d + 4) * EPS * (np.abs(g) @ np.abs(v).T))
                    e_ds = e_ds + FLUSH * (2 + np.abs(dp - D))
                    if n == 1:
                        e_ds = np.zeros_like(e_ds)
                    s = 1 / np.sqrt(d)
                    ref = ds @ k * s
                    within(dq[i, :, a], ref, s * (e_ds @ np.abs(k) + (n + 16) * EPS * ((np.abs(ds) + e_ds) @ np.abs(k))) + (store + 4 * EPS) * np.abs(ref) + TINY[self.dtype], ("dq", i, a))
                    rows = nq * hq // hkv + 16
                    rk, rv = rk + ds.T @ Q[i, :, a] * s, rv + p.T @ g
                    bk = bk + s * (e_ds.T @ np.abs(Q[i, :, a]) + rows * EPS * ((np.abs(ds) + e_ds).T @ np.abs(Q[i, :, a])))
                    bv = bv + (p * (e_p + low + 4 * EPS) + FLUSH).T @ np.abs(g) + rows * EPS * p.T @ np.abs(g)
                if back:
                    within(dk[i, :n, h], rk, bk + (store + 4 * EPS) * np.abs(rk) + TINY[self.dtype], ("dk", i, h))
                    within(dv[i, :n, h], rv, bv + (store + 4 * EPS) * np.abs(rv) + TINY[self.dtype], ("dv", i, h))
                    assert not dk[i, n:, h].any() and not dv[i, n:, h].any(), ("gradients behind the states", i, h)
        return self


def cross_both(c):
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check()
    c.untouched()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("b,nq,nk,hq,hkv,d", [(1, 1, 1, 1, 1, 64), (1, 1, 2, 1, 1, 128), (2, 3, 5, 4, 2, 64), (1, 31, 63, 2, 2, 128), (1, 32, 64, 2, 1, 64), (1, 33, 65, 2, 2, 128),
                                              (3, 63, 31, 6, 3, 64), (2, 64, 129, 4, 4, 128), (1, 65, 200, 8, 1, 128), (1, 128, 77, 4, 4, 64), (2, 130, 257, 3, 1, 128), (1, 257, 16, 2, 2, 64),
                                              (1, 300, 1, 2, 1, 128), (4, 1, 700, 8, 2, 128), (5, 7, 130, 6, 3, 64), (1, 5, 1500, 2, 2, 128), (1, 1000, 40, 1, 1, 64)])
def test_cross_attention(dtype, b, nq, nk, hq, hkv, d):
    cross_both(Cross(dtype, b, nq, nk, hq, hkv, d))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[0, 1, 2, 150], [64, 63, 65, 128], [0, 0, 0, 0], [1, 1, 1, 1], [-3, 1000, 127, 33]])
def test_cross_attention_of_a_padded_batch(dtype, d, lens):
    """Lengths of zero, one, at and around a tile, outside their range; NaN and infinities behind the states."""
    cross_both(Cross(dtype, 4, 70, 150, 4, 2, d, lens))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pad,packed", [((0, 0), False), ((8, 24), True), ((136, 8), False)])
def test_cross_attention_of_rows_that_are_part_of_wider_ones(dtype, d, pad, packed):
    cross_both(Cross(dtype, 2, 40, 90, 4, 2, d, [90, 37], pad, packed))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("b,nq,nk,hq,hkv,d,lens", [(1, 1, 4099, 8, 1, 128, None), (2, 1, 6000, 4, 4, 64, [5999, 3]), (3, 2, 3001, 12, 4, 128, [0, 3001, 64]), (1, 16, 5000, 2, 1, 64, None)])
def test_cross_attention_of_a_few_queries_over_many_states(dtype, b, nq, nk, hq, hkv, d, lens):
    cross_both(Cross(dtype, b, nq, nk, hq, hkv, d, lens))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("b,nq,nk,hq,hkv,d", [(1, 3000, 50, 2, 1, 128), (1, 2500, 130, 2, 2, 64), (2, 1100, 300, 8, 2, 128)])
def test_cross_attention_of_many_queries_over_a_few_states(dtype, b, nq, nk, hq, hkv, d):
    cross_both(Cross(dtype, b, nq, nk, hq, hkv, d))


# (batch, queries, states, heads, kv heads, head size) -> the forms that they take: test_reader_operators_refusals.py holds them to that
FORMS = {(4, 520, 100, 4, 4, 64): None, (4, 520, 400, 4, 4, 64): [400, 77, 0, 399], (4, 520, 600, 4, 4, 128): [1, 600, 130, 64], (4, 100, 600, 8, 4, 64): [600, 599, 2, 31], (4, 300, 600, 4, 4, 64): None,
         (2, 1100, 700, 4, 2, 64): [700, 65], (1, 1100, 2300, 4, 1, 128): None}


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("shape", FORMS)
def test_cross_attention_of_every_division(dtype, shape):
    cross_both(Cross(dtype, *shape, FORMS[shape]))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("b,nq,nk,hq,hkv,d,lens", [(16, 1, 300, 32, 16, 64, None), (12, 15, 140, 16, 16, 128, [140, 0, 1, 16, 17, 139, 64, 33, 140, 2, 128, 100]), (16, 3, 5, 12, 12, 64, None),
                                                   (16, 70, 4, 16, 16, 64, [4, 3, 2, 1] * 4), (12, 100, 20, 12, 12, 128, [0, 20, 1, 16, 17, 19, 20, 5, 20, 2, 15, 20])])
def test_cross_attention_of_many_short_sequences(dtype, b, nq, nk, hq, hkv, d, lens):
    """So many sequences and heads that every one has a workgroup of its own with 1 to 20 rows, or states, of 64 (or of 16) in it."""
    cross_both(Cross(dtype, b, nq, nk, hq, hkv, d, lens))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [8.0, 60.0])
def test_cross_attention_of_large_scores(dtype, d, size):
    """Scores of some hundred: a weight is one, the others vanish; the running maximum is raised in many tiles."""
    c = Cross(dtype, 1, 90, 500, 2, 1, d, size=size)
    ramp = np.linspace(0.2, 1.0, 500)[:, None]
    c.KV[:, :c.wk] = q(c.KV[:, :c.wk] * ramp, dtype)
    c.kv.copy_(dev(c.KV, dtype))
    cross_both(c)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_cross_attention_gives_the_same_bits_every_time(dtype):
    c = Cross(dtype, 2, 300, 900, 8, 2, 128, [900, 411])
    c.fwd(); c.bwd()
    first = {k: v.clone() for k, v in c.outputs().items()}
    for fill in (0.0, float("nan")):
        c.ws.view(torch.uint8)[:c.ws.numel() // 4 * 4].view(torch.float32).fill_(fill)
        for t in (c.o, c.lse, c.dq, c.dkv):
            t.fill_(7.0)
        c.fwd(); c.bwd()
        torch.cuda.synchronize()
        assert all(torch.equal(v, first[k]) for k, v in c.outputs().items())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_cross_attention_what_is_not_finite_stays_with_its_row(dtype):
    """A NaN in a query: its row and, in the gradient, dk and dv of its head group; other rows and heads as without it."""
    c = Cross(dtype, 2, 100, 150, 4, 2, 128, [150, 60])
    c.fwd(); c.bwd()
    clean = {k: v.clone() for k, v in c.outputs().items()}
    c.q[37, 128] = float("nan")                     # sequence 0, query 37, head 1
    c.fwd(); c.bwd()
    torch.cuda.synchronize()
    out = c.outputs()
    view = lambda t, h: t.view(2, -1, h, 128)  # noqa: E731
    hit = torch.zeros((2, 100, 4), dtype=torch.bool, device="cuda")
    hit[0, 37, 1] = True
    for k in ("o", "dq"):
        a, b = view(out[k], 4), view(clean[k], 4)
        assert bool(a[hit].isnan().all()) and torch.equal(a[~hit], b[~hit]), k
    assert bool(out["lse"][0, 1, 37].isnan())
    for k in ("dk", "dv"):
        a, b = view(out[k].contiguous(), 2), view(clean[k].contiguous(), 2)
        assert bool(a[0, :, 0].isnan().any()) and torch.equal(a[:, :, 1], b[:, :, 1]) and torch.equal(a[1], b[1]), k


def test_cross_attention_of_one_state_has_no_gradient_of_scores():
    c = Cross(BF16, 2, 50, 9, 2, 1, 64, [1, 1])
    cross_both(c)
    assert not host(c.outputs()["dq"]).any() and not host(c.outputs()["dk"]).any()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("b,nq,nk,hq,hkv,d", [(2, 200, 500, 4, 2, 128), (3, 1, 3000, 8, 2, 64), (1, 1500, 70, 2, 1, 64)])
def test_cross_attention_captured_and_replayed(dtype, b, nq, nk, hq, hkv, d):
    """Replays with eager calls, other lengths and synchronizations between them."""
    c = Cross(dtype, b, nq, nk, hq, hkv, d, [nk] * b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.fwd(); c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c.fwd(); c.bwd()
    r = rng(9)
    other = Cross(dtype, b, nq, nk, hq, hkv, d, [nk] * b, seed=5)
    for turn in range(4):
        n = torch.from_numpy(r.integers(0, nk + 1, b).astype(np.int32)).cuda()
        c.kl.copy_(n); other.kl.copy_(n)
        c.q.copy_(other.q * (turn + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in c.outputs().items()}
        c.ws.fill_(0x7F)
        c.fwd(); c.bwd()
        other.fwd(); other.bwd()
        torch.cuda.synchronize()
        assert all(torch.equal(v, got[k]) for k, v in c.outputs().items()), turn


def test_cross_attention_two_calls_at_once():
    """Two streams, each call with a workspace of its own."""
    cs = [Cross(BF16, 2, 400, 900, 8, 2, 128, [900, 500], seed=1), Cross(BF16, 4, 1, 4000, 8, 2, 128, seed=2)]
    for c in cs:
        c.fwd(); c.bwd()
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in c.outputs().items()} for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        for c, s in zip(cs, streams):
            c.fwd(s.cuda_stream); c.bwd(s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(v, w[k]) for c, w in zip(cs, want) for k, v in c.outputs().items())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_cross_attention_offsets_beyond_32_bits(dtype):
    """States whose last rows lie more than 2^32 bytes behind the first: a few distinct rows repeated, against the same rows close together."""
    nk, hkv, d, e = 1200, 1, 64, 2 if dtype == BF16 else 4
    ld = (1 << 23) // e - 64
    if torch.cuda.mem_get_info()[0] < 2 * nk * ld * e + (4 << 30):
        pytest.skip("too little memory free")
    a = Cross(dtype, 1, 33, nk, 2, hkv, d)
    a.fwd(); a.bwd()
    big, grad = torch.empty((nk, ld), dtype=TDT[dtype], device="cuda"), torch.empty((nk, ld), dtype=TDT[dtype], device="cuda")
    big[:, :2 * d] = a.kv
    nbytes = lib().optstage_op_cross_attn_ws_bytes(dtype, *a.shape)
    o, lse, dq = torch.empty_like(a.o), torch.empty_like(a.lse), torch.empty_like(a.dq)
    lens = torch.tensor([nk], dtype=torch.int32, device="cuda")
    ok(lib().optstage_op_cross_attn_fwd(dtype, a.q.data_ptr(), a.ldq, big.data_ptr(), big.data_ptr() + d * e, ld, lens.data_ptr(), o.data_ptr(), lse.data_ptr(), a.ws.data_ptr(), nbytes,
                                        *a.shape, stream()))
    ok(lib().optstage_op_cross_attn_bwd(dtype, a.q.data_ptr(), a.ldq, big.data_ptr(), big.data_ptr() + d * e, ld, lens.data_ptr(), o.data_ptr(), a.g.data_ptr(), lse.data_ptr(),
                                        dq.data_ptr(), grad.data_ptr(), grad.data_ptr() + d * e, a.ws.data_ptr(), nbytes, *a.shape, stream()))
    torch.cuda.synchronize()
    assert torch.equal(o, a.o) and torch.equal(lse, a.lse) and torch.equal(dq, a.dq) and torch.equal(grad[:, :2 * d], a.dkv)


def test_cross_attention_gradient_against_differences():
    """fp32: the change of <o, g> along a direction, from the forward calls alone."""
    c = Cross(FP32, 2, 20, 37, 4, 2, 64, [37, 11], size=0.7)
    c.fwd(); c.bwd()
    torch.cuda.synchronize()
    grads = {k: v.double() for k, v in c.outputs().items()}
    r = rng(12)
    for name, base in (("dq", c.q), ("dkv", c.kv)):
        clean = base.clone()
        step = torch.from_numpy(r.standard_normal(tuple(base.shape))).float().cuda()
        ends = []
        for h in (2.0 ** -7, -2.0 ** -7):
            base.copy_(torch.where(clean.isfinite(), clean + h * step, clean))
            c.fwd()
            torch.cuda.synchronize()
            ends.append((c.o.double() * c.g.double()).sum().item())
        base.copy_(clean)
        g = grads["dq"] if name == "dq" else torch.cat([grads["dk"], grads["dv"]], 1)
        want = (g * torch.where(clean.isfinite(), step, torch.zeros_like(step)).double()).sum().item()
        # the difference's own error: h^2 / 6 of the third derivative (sums of a few thousand products of order one, 2^-16.6 of them) and
        # fp32 results' 2^-24 times some sqrt(10240) over 2 h = 2^-6
        assert abs((ends[0] - ends[1]) * 2 ** 6 - want) < 0.05 + 1e-3 * abs(want), name


# ------------------------------------------------------------------ the loss against a teacher's top entries
class Distill:
    def __init__(self, dtype, rows, vocab, k, temperature=1.0, log_probs=0, pad=(0, 0), seed=0, bare=False):
        r = rng(3, dtype, rows, vocab, k, seed)
        self.dtype, self.shape, self.pad = dtype, (rows, vocab, k, temperature, log_probs), pad
        self.Z = q(3.0 * r.standard_normal((rows, vocab + pad[0])), dtype)
        self.ids = r.integers(0, vocab, (rows, k)).astype(np.int32)          # words given twice among them
        self.T = (2.0 * r.standard_normal((rows, k)) - (3.0 + np.log(k) if log_probs else 0.0)).astype(np.float32)
        self.w = r.standard_normal(rows).astype(np.float32)
        if not bare:
            drop = r.random((rows, k))
            self.ids[drop < 0.1] = -1
            self.ids[(drop >= 0.1) & (drop < 0.15)] = vocab + r.integers(0, 5)
            self.T[r.random((rows, k)) < 0.05] = -np.inf
            if rows > 2:
                self.ids[1], self.w[2] = -1, 0.0
        self.upload()
        self.loss, self.c1 = zone((rows,), torch.float32)
        self.lse, self.c2 = zone((rows,), torch.float32)
        self.dz, self.c3 = zone((rows, vocab + pad[1]), TDT[dtype])
        self.ws, self.c4 = zone((lib().optstage_op_distill_ws_bytes(rows, vocab, k),), torch.uint8, 0xA5)

    def upload(self):
        off = lambda a, t: torch.cat([torch.zeros(1, dtype=t), torch.from_numpy(np.ascontiguousarray(a)).flatten()]).cuda()[1:]  # noqa: E731
        self.z = torch.from_numpy(self.Z).to(TDT[self.dtype]).cuda()
        self.i, self.t, self.g = off(self.ids, torch.int32), off(self.T, torch.float32), off(self.w, torch.float32)

    def call(self, how, inplace=False, at=None):
        rows, vocab, k, temperature, log_probs = self.shape
        ld = self.z.shape[1]
        dz, lddz = (self.z, ld) if inplace else (self.dz, self.dz.shape[1])
        at = at or stream()
        head = (self.dtype, self.z.data_ptr(), ld, self.i.data_ptr(), self.t.data_ptr())
        if how == "both":
            ok(lib().optstage_op_distill(*head, self.g.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(), dz.data_ptr(), lddz, self.ws.data_ptr(), self.ws.numel(), *self.shape, at))
            return dz
        ok(lib().optstage_op_distill_fwd(*head, self.loss.data_ptr(), self.lse.data_ptr(), self.ws.data_ptr(), self.ws.numel(), *self.shape, at))
        ok(lib().optstage_op_distill_bwd(*head, self.lse.data_ptr(), self.g.data_ptr(), dz.data_ptr(), lddz, *self.shape, at))
        return dz

    def check(self, dz):
        """Bounds.  exp((z - m) / T) is off by a few fp32 roundings of the exponent (its size |z - m| / T and, from a stored lse, |lse|), the sum of vocab of them by what each is off
        and log2-many to vocab / 64 additions (512 roundings are more than any division of the row makes); the loss is a sum in 64 bits of 32-bit t.  A t is an exponential (2 EPS) times
        one plus a rest (2 EPS); the teacher's normalisation is a sum of such numbers, rounded (1 EPS), and its logarithm (2^-26): with that 10 EPS of t in all, and 6 EPS of log t."""
        rows, vocab, k, T, log_probs = self.shape
        z = self.Z[:, :vocab]
        loss, lse = P.distill(z, self.ids, self.T, T, log_probs)
        ref = P.distill_bwd(z, self.ids, self.T, T, log_probs, self.w.astype(np.float64))
        with np.errstate(invalid="ignore"):
            spread = np.where(np.isfinite(z), np.abs(z - z.max(1, keepdims=True)) / T, 0.0)
        p = np.exp(z / T - lse[:, None])
        e_sum = EPS * ((p * (4 * spread + 4)).sum(1) + 512)
        e_lse = e_sum + 2 * EPS * np.abs(lse)
        ts = [P.teacher_weights(self.ids[r], self.T[r], vocab, T, log_probs)[0] for r in range(rows)]
        mass = np.array([t.sum() for t in ts])
        within(self.lse, lse, e_lse, "lse")
        terms = np.zeros(rows)
        for r in range(rows):
            t, log_t = P.teacher_weights(self.ids[r], self.T[r], vocab, T, log_probs)
            for j in np.nonzero(t)[0]:
                terms[r] += t[j] * abs(log_t[j] - (z[r, self.ids[r, j]] / T - lse[r]))
        within(self.loss, loss, (e_lse + 6 * EPS) * mass + 10 * EPS * terms + EPS * np.abs(loss) + 1e-12, "loss")
        top = np.zeros_like(z)
        for r in range(rows):
            for j in np.nonzero(ts[r])[0]:
                top[r, self.ids[r, j]] += ts[r][j]
        # (a probability below the least normal number is off by up to that number: its steps are 2^-149 wide, and the hardware's exponential gives 0)
        # (from an lse of up to 16, or 4096 in bf16, its rounding comes in; rows beyond have their own sum)
        near = e_sum + 2 * EPS * np.minimum(np.abs(lse), 16.0 if self.dtype == FP32 else 4096.0)
        e_p = ((EPS * (6 * spread + 16) + 2 * near[:, None]) * p + FLUSH) * mass[:, None] + FLUSH + 12 * EPS * (p * mass[:, None] + top)
        within(host(dz)[:, :vocab], ref, np.abs(self.w.astype(np.float64))[:, None] / T * e_p + (HALF[self.dtype] + 2 * EPS) * np.abs(ref) + TINY[self.dtype], "dz")

    def untouched(self, inplace=False):
        vocab = self.shape[1]
        assert self.c1() and self.c2() and self.c3() and self.c4()
        if inplace:
            assert np.array_equal(host(self.z)[:, vocab:], self.Z[:, vocab:])
        else:
            assert bool((self.dz[:, vocab:] == 9.0).all()) and np.array_equal(host(self.z), self.Z)


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab,k,pad", [(1, 1, 1, (0, 0)), (3, 2, 3, (0, 0)), (5, 7, 4, (1, 3)), (128, 1000, 8, (0, 0)), (9, 1001, 64, (0, 0)), (4, 4096, 100, (8, 16)), (300, 513, 5, (7, 0)),
                                              (2, 32000, 64, (0, 0)), (7, 50001, 50, (23, 0)), (3, 151003, 300, (5, 9)), (1, 262144, 1024, (0, 0)), (600, 3001, 17, (3, 3)), (270, 66000, 9, (0, 8)),
                                              (5, 9000, 300, (0, 0)), (200, 9000, 300, (0, 1)), (200, 1500, 1024, (0, 0))])   # many words given twice
def test_distillation(how, dtype, rows, vocab, k, pad):
    c = Distill(dtype, rows, vocab, k, pad=pad)
    dz = c.call(how)
    torch.cuda.synchronize()
    c.check(dz)
    c.untouched()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("vocab", [300, 600, 2048, 2049, 4096, 4097, 7001, 9000, 13001, 20011, 30011, 40009, 45001, 55001, 60001, 70001, 90001, 100003, 120011])
def test_distillation_of_every_length_of_row(dtype, vocab):
    c = Distill(dtype, 161, vocab, 5, pad=(3, 1), seed=4)
    dz = c.call("both")
    torch.cuda.synchronize()
    c.check(dz)
    c.untouched()


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("temperature,log_probs", [(2.0, 0), (0.25, 0), (1.0, 1), (3.0, 1)])
def test_distillation_temperatures_and_forms_in_place(how, dtype, temperature, log_probs):
    for rows, vocab, k, pad in ((20, 2000, 33, 0), (3, 40007, 40, 1), (300, 9000, 3, 8)):
        c = Distill(dtype, rows, vocab, k, temperature, log_probs, (pad, 0), seed=3)
        dz = c.call(how, inplace=True)
        torch.cuda.synchronize()
        c.check(dz)
        c.untouched(True)


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab", [(6, 500), (6, 70001), (300, 8200)])
def test_distillation_of_rows_that_are_not_finite(how, dtype, rows, vocab):
    """Masked words (minus infinity), NaN and plus infinity in a row, a row of which nothing is left: that row's loss and gradient and no other's; none where dloss is 0."""
    c = Distill(dtype, rows, vocab, 4, bare=True)
    c.Z[0, ::3] = -np.inf
    c.ids[0] = [1, 2, 4, 5]
    c.Z[1, vocab // 2] = np.nan
    c.Z[2, vocab - 1] = np.inf
    c.Z[3] = -np.inf
    c.w[4], c.Z[4, 3], c.Z[4, 4] = 0.0, np.nan, np.inf
    c.Z[5, c.ids[5, 0]] = -np.inf
    c.upload()
    dz = c.call(how)
    torch.cuda.synchronize()
    loss, lse, dz = host(c.loss), host(c.lse), host(dz)
    for r in (1, 2, 3):
        assert np.isnan(loss[r]) and np.isnan(dz[r]).any() and not np.isfinite(lse[r]), r
    assert not dz[4].any() and np.isposinf(loss[5]) and np.isfinite(dz[5]).all() and np.isnan(loss[4])
    assert not dz[0, 0::3].any()
    fine = [0] + list(range(6, rows))
    for a in ("Z", "ids", "T", "w"):
        setattr(c, a, getattr(c, a)[fine])
    c.shape = (len(fine),) + c.shape[1:]
    c.loss, c.lse = torch.from_numpy(loss[fine]), torch.from_numpy(lse[fine])
    c.check(torch.from_numpy(dz[fine]))


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab", [(9, 700), (9, 40009), (9, 131200), (170, 9001), (170, 70003)])
@pytest.mark.parametrize("temperature", [1.0, 0.125])
def test_distillation_of_rows_of_every_range(how, dtype, rows, vocab, temperature):
    """Logits that rise by hundreds behind the first words, fall behind them, lie far from zero, are masked by minus infinity or by the type's lowest value in front, behind or nearly everywhere,
    are all alike, or all the lowest value."""
    c = Distill(dtype, rows, vocab, 6, temperature, bare=True, seed=8)
    low = float(torch.finfo(TDT[dtype]).min)
    base = c.Z[:9].copy()
    half = vocab // 2
    c.Z[0, half:] += 300.0
    c.Z[1, :half] += 300.0
    c.Z[2] += 4096.0
    c.Z[3, :half] = -np.inf
    c.Z[4, half:] = low
    c.Z[5] = np.where(np.arange(vocab) == vocab - 2, base[5], low)
    c.Z[6] = 3.0
    c.Z[7, :min(600, half)] = low
    c.Z[8] -= 2048.0
    c.ids[3] = half + np.arange(6)
    c.Z = q(c.Z, dtype)
    c.Z[3, :half] = -np.inf
    c.upload()
    dz = c.call(how)
    torch.cuda.synchronize()
    c.check(dz)                                         # (the rows far from zero have no rounding of lse in their bounds)
    c.untouched()


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", ["lowest", 2.0 ** 35, -(2.0 ** 40), 2.0 ** 90])
@pytest.mark.parametrize("rows,vocab", [(3, 900), (3, 50000), (170, 9001), (170, 131073)])
def test_distillation_of_a_row_of_alike_values(how, dtype, rows, vocab, size):
    """All words masked by the type's lowest value, or as far from zero as only sums of differences bear: the distribution is even."""
    c = Distill(dtype, rows, vocab, 4, bare=True)
    c.Z[1], c.ids[1], c.T[1] = float(torch.finfo(TDT[dtype]).min) if size == "lowest" else size, [0, 1, vocab // 2, vocab - 1], 0.0
    c.upload()
    dz = host(c.call(how))
    torch.cuda.synchronize()
    w = float(c.w[1])
    want = np.full(vocab, w / vocab)
    want[c.ids[1]] -= w / 4
    within(dz[1], want, np.abs(want) * (HALF[dtype] + 16 * EPS) + 16 * EPS * abs(w) / vocab, "even")
    within(host(c.loss)[1:2], np.array([np.log(vocab / 4)]), 1e-5)
    fine = [0] + list(range(2, rows))
    for a in ("Z", "ids", "T", "w"):
        setattr(c, a, getattr(c, a)[fine])
    c.shape = (len(fine),) + c.shape[1:]
    c.loss, c.lse = c.loss[fine], c.lse[fine]
    c.check(torch.from_numpy(dz[fine]))


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab,every", [(3, 50000, 2000), (100, 50000, 4552), (161, 9001, 4000), (161, 40009, 12000)])
@pytest.mark.parametrize("gap", [75.0, 88.0])
@pytest.mark.parametrize("dloss", [1.0 / 4096, 1e-8])
def test_distillation_of_words_whose_exponential_is_just_within_range(how, dtype, rows, vocab, every, gap, dloss):
    """Logits that lie almost as far above the first words' as an exponential in 32 bits reaches (88.7): one of them at the end, and one in every stretch of words that few rows are divided into, whose
    sums come together; against weights of the loss with which 1 / the sum against the first words is below the normal numbers."""
    c = Distill(dtype, rows, vocab, 6, bare=True, seed=9)
    c.Z /= 64
    at = np.arange(3 * every // 4, vocab, every)
    c.Z[0, vocab - 5] = gap
    c.Z[1, at] = gap
    c.Z[2, at] = gap - np.arange(len(at)) % 3
    c.Z = q(c.Z, dtype)
    c.ids[0, 0], c.ids[1, :2], c.ids[2, :2] = vocab - 5, at[:2], at[-2:]
    c.w = (np.float32(dloss) * np.sign(c.w)).astype(np.float32)
    c.upload()
    dz = c.call(how)
    torch.cuda.synchronize()
    c.check(dz)
    c.untouched()


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab", [(3, 900), (3, 50000), (161, 9001), (161, 40009)])
def test_distillation_of_weights_near_the_least_numbers(how, dtype, rows, vocab):
    """The gradient's values are numbers of 32 bits as long as weight times probability is; weight over the sum against the first words need not be."""
    c = Distill(dtype, rows, vocab, 6, bare=True, seed=10)
    c.Z[:2] /= 64
    c.Z[:2, vocab - 5] = 20.0
    c.Z = q(c.Z, dtype)
    c.ids[:2, 0] = vocab - 5
    c.w = (np.float32(1e-35) * np.sign(c.w)).astype(np.float32)
    c.upload()
    dz = c.call(how)
    torch.cuda.synchronize()
    c.check(dz)
    c.untouched()


@pytest.mark.parametrize("how", ["both", "apart"])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab", [(5, 500), (5, 9001), (200, 9001)])
@pytest.mark.parametrize("offset,size,temperature", [(1e4, 1.0, 0.7), (-3e5, 1.0, 3.0), (0.0, 1e9, 1e-30)])
def test_distillation_of_teacher_logits_far_from_zero(how, dtype, rows, vocab, offset, size, temperature):
    """What a teacher's logits have in common does not show in its probabilities, nor does their size over the temperature have to be a number of 32 bits."""
    c = Distill(dtype, rows, vocab, 12, float(np.float32(temperature)), seed=10)
    c.T = (c.T * np.float32(size) + np.float32(offset)).astype(np.float32)
    c.upload()
    dz = c.call(how)
    torch.cuda.synchronize()
    c.check(dz)
    c.untouched()


@pytest.mark.parametrize("rows,vocab,k", [(40, 3000, 20), (2, 100003, 64), (700, 20000, 9), (301, 900, 1024)])
def test_distillation_captured_replayed_and_repeated(rows, vocab, k):
    a, b = Distill(BF16, rows, vocab, k), Distill(BF16, rows, vocab, k, seed=1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.call("both"); a.call("apart")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a.call("both")
    for turn in range(4):
        a.z.copy_(b.z * (0.5 + 0.5 * turn)); a.i.copy_(b.i); a.t.copy_(b.t)
        a.ws.fill_(0x7F)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (a.loss, a.lse, a.dz)]
        b.call("both")
        a.call("both")
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (a.loss, a.lse, a.dz))), turn


def test_distillation_two_calls_at_once():
    cs = [Distill(BF16, 3, 90001, 64, seed=1), Distill(FP32, 500, 5000, 33, seed=2), Distill(BF16, 5, 131072, 8, seed=4)]
    for c in cs:
        c.call("both")
    torch.cuda.synchronize()
    want = [[t.clone() for t in (c.loss, c.lse, c.dz)] for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(5):
        for c, s in zip(cs, streams):
            c.call("both", at=s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for c, w in zip(cs, want) for x, y in zip((c.loss, c.lse, c.dz), w))


def test_distillation_offsets_beyond_32_bits():
    """Logits of more than 2^31 values: rows of a few patterns, their results equal."""
    rows, vocab, k = 16411, 131080, 6
    if torch.cuda.mem_get_info()[0] < 16 * 2 ** 30:
        pytest.skip("too little memory free")
    c = Distill(BF16, 5, vocab, k, bare=True)
    dz5 = c.call("both").clone()
    torch.cuda.synchronize()
    c.check(dz5)
    z = c.z.repeat(rows // 5 + 1, 1)[:rows].contiguous()
    rep = lambda t, n: t.view(5, -1).repeat(n, 1)[:rows].contiguous()  # noqa: E731
    i, t, g = (rep(x, rows // 5 + 1) for x in (c.i, c.t, c.g))
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ws = torch.empty(lib().optstage_op_distill_ws_bytes(rows, vocab, k), dtype=torch.uint8, device="cuda")
    ok(lib().optstage_op_distill(BF16, z.data_ptr(), vocab, i.data_ptr(), t.data_ptr(), g.data_ptr(), loss.data_ptr(), lse.data_ptr(), z.data_ptr(), vocab, ws.data_ptr(), ws.numel(), rows,
                                 vocab, k, 1.0, 0, stream()))
    torch.cuda.synchronize()
    d = (z[-5:].float() - dz5.repeat(2, 1)[rows % 5:rows % 5 + 5].float()).abs().max().item()
    assert d <= 2.0 ** -7 * dz5.abs().max().item()                          # another division of the row: at most a step apart
    assert torch.allclose(loss[-5:], c.loss.repeat(2)[rows % 5:rows % 5 + 5], rtol=1e-5)


@pytest.mark.parametrize("dtype,rows,vocab", [(BF16, 640, 131080), (FP32, 330, 131075), (BF16, 300, 66001)])
def test_distillation_gradient_of_logits_that_go_past_the_caches(dtype, rows, vocab):
    """Rows of a few patterns: from lse, a row's gradient is the same bits however many rows there are."""
    c = Distill(dtype, 5, vocab, 7, bare=True)
    want = c.call("apart").clone()
    torch.cuda.synchronize()
    c.check(want)
    rep = lambda t: t.view(5, -1).repeat(rows // 5, 1).contiguous()  # noqa: E731
    z, i, t, g, lse = (rep(x) for x in (c.z, c.i, c.t, c.g, c.lse))
    for dz in (torch.empty_like(z), z):
        ok(lib().optstage_op_distill_bwd(dtype, z.data_ptr(), vocab, i.data_ptr(), t.data_ptr(), lse.data_ptr(), g.data_ptr(), dz.data_ptr(), vocab, rows, vocab, 7, 1.0, 0, stream()))
        torch.cuda.synchronize()
        assert torch.equal(dz.view(-1, 5, vocab), want.view(1, 5, vocab).expand(rows // 5, 5, vocab))


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_training_step_of_a_reading_layer_with_a_teacher(dtype):
    """Queries and keys turned by three axes, causal attention, cross attention to an encoder's states, the head's product and the teacher's loss, all the way back to the packed qkv rows, the
    states' packed rows and the head's weight, against the same chain in fp64."""
    r = rng(20, dtype)
    b, seq, nk, hq, hkv, d, vocab, k = 2, 64, 45, 4, 2, 64, 520, 6
    rows, w, wk = b * seq, hq * d, hkv * d
    width = w + 2 * wk
    lens = [45, 17]
    qkv, kv, head = (q(s * r.standard_normal(shape), dtype) for s, shape in ((1.0, (rows, width)), (1.0, (b * nk, 2 * wk)), (0.3, (vocab, w))))
    ids, teacher = np.stack([r.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32), r.standard_normal((rows, k)).astype(np.float32)
    dloss = np.full(rows, 1.0 / 64, dtype=np.float32)
    pos = np.stack([np.arange(rows) % seq, np.arange(rows) % 8, np.arange(rows) // 8 % 8]).astype(np.int32)
    axis = [0] * 8 + [1] * 12 + [2] * 12
    L, s = lib(), stream()
    t = {n: torch.empty(sh, dtype=TDT[dtype], device="cuda") for n, sh in (("turned", (rows, width)), ("o1", (rows, w)), ("o2", (rows, w)), ("z", (rows, vocab)), ("dz", (rows, vocab)), ("do2", (rows, w)),
                                                                           ("do1", (rows, w)), ("dkv", (b * nk, 2 * wk)), ("dturned", (rows, width)), ("dqkv", (rows, width)))}
    f = {n: torch.empty(sh, dtype=torch.float32, device="cuda") for n, sh in (("lse1", (b, hq, seq)), ("lse2", (b, hq, seq)), ("loss", (rows,)), ("lsez", (rows,)))}
    t["table"] = torch.empty((seq, d // 2, 2), device="cuda")
    X, KV, W = dev(qkv, dtype), dev(kv, dtype), dev(head, dtype)
    Wt = W.T.contiguous()
    I, Te, G, Po = (torch.from_numpy(a).cuda() for a in (ids, teacher, dloss, pos))
    Ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    dW = torch.zeros((vocab, w), device="cuda")
    e = KV.element_size()
    ws = torch.empty(max(L.optstage_op_cross_attn_ws_bytes(dtype, seq, nk, b, hq, hkv, d), 4 * L.optstage_op_attn_bwd_ws_floats(seq, b, hq, hkv, d), L.optstage_op_distill_ws_bytes(rows, vocab, k)),
                     dtype=torch.uint8, device="cuda")
    at = {n: v.data_ptr() for n, v in {**t, **f}.items()}
    ok(L.optstage_op_rope_table(at["table"], seq, d, 10000.0, s))
    ok(L.optstage_op_rope_axes(dtype, X.data_ptr(), width, at["turned"], width, at["table"], seq, Po.data_ptr(), 3, bytes(axis), rows, hq + hkv, hkv, d, 0, s))
    ok(L.optstage_op_attn_fwd(dtype, at["turned"], at["o1"], at["lse1"], seq, b, hq, hkv, d, s))
    shape = (seq, nk, b, hq, hkv, d)
    ok(L.optstage_op_cross_attn_fwd(dtype, at["o1"], w, KV.data_ptr(), KV.data_ptr() + wk * e, 2 * wk, Ln.data_ptr(), at["o2"], at["lse2"], ws.data_ptr(), ws.numel(), *shape, s))
    ok(L.optstage_op_gemm(dtype, 0, 0, at["o2"], W.data_ptr(), at["z"], 0, rows, vocab, w, w, w, vocab, s))
    ok(L.optstage_op_distill(dtype, at["z"], vocab, I.data_ptr(), Te.data_ptr(), G.data_ptr(), at["loss"], at["lsez"], at["dz"], vocab, ws.data_ptr(), ws.numel(), rows, vocab, k, 2.0, 0, s))
    ok(L.optstage_op_gemm(dtype, 0, 0, at["dz"], Wt.data_ptr(), at["do2"], 0, rows, w, vocab, vocab, vocab, w, s))
    ok(L.optstage_op_gemm(dtype, 1, 2, at["dz"], at["o2"], dW.data_ptr(), 0, vocab, w, rows, vocab, w, w, s))
    ok(L.optstage_op_cross_attn_bwd(dtype, at["o1"], w, KV.data_ptr(), KV.data_ptr() + wk * e, 2 * wk, Ln.data_ptr(), at["o2"], at["do2"], at["lse2"], at["do1"], at["dkv"], at["dkv"] + wk * e,
                                    ws.data_ptr(), ws.numel(), *shape, s))
    ok(L.optstage_op_attn_bwd(dtype, at["turned"], at["o1"], at["do1"], at["lse1"], at["dturned"], ws.data_ptr(), seq, b, hq, hkv, d, s))
    ok(L.optstage_op_rope_axes(dtype, at["dturned"], width, at["dqkv"], width, at["table"], seq, Po.data_ptr(), 3, bytes(axis), rows, hq + hkv, hkv, d, 1, s))
    torch.cuda.synchronize()
    # the same chain in fp64, by autograd where attention is causal
    A = torch.tensor(qkv, requires_grad=True)
    C = torch.tensor(kv, requires_grad=True)
    H = torch.tensor(head, requires_grad=True)
    tab = t["table"].double().cpu()
    ang = tab[torch.tensor(pos[axis].T.copy()).long(), torch.arange(d // 2)][:, None]
    h = A.view(rows, -1, d)
    lo, hi = h[:, :hq + hkv].split(d // 2, 2)
    turned = torch.cat([torch.cat([lo * ang[..., 0] - hi * ang[..., 1], hi * ang[..., 0] + lo * ang[..., 1]], 2), h[:, hq + hkv:]], 1).view(b, seq, -1, d).transpose(1, 2)
    rep = lambda x: x.repeat_interleave(hq // hkv, 1)  # noqa: E731
    sdpa = torch.nn.functional.scaled_dot_product_attention
    o1 = sdpa(turned[:, :hq], rep(turned[:, hq:hq + hkv]), rep(turned[:, hq + hkv:]), is_causal=True)
    st = C.view(b, nk, 2 * hkv, d).transpose(1, 2)
    mask = (torch.arange(nk)[None, :] < torch.tensor(lens)[:, None])[:, None, None, :]
    o2 = sdpa(o1, rep(st[:, :hkv]), rep(st[:, hkv:]), attn_mask=mask).transpose(1, 2).reshape(rows, w)
    z = o2 @ H.T / 2.0
    tw = torch.softmax(torch.tensor(teacher.astype(np.float64)) / 2.0, 1)
    loss = (tw * (tw.log() - torch.log_softmax(z, 1).gather(1, torch.tensor(ids).long()))).sum(1)
    (loss * torch.tensor(dloss.astype(np.float64))).sum().backward()
    # Relative to the tensor's norm.  fp32: some hundred roundings of 2^-24 in a row, no cancellation that costs more than a factor of ten.  bf16: stored tensors each off by at most 2^-8 of
    # their values, twelve of them (four forward, the weights and dS of two attentions twice, five gradients) on the longest way, added up as if all pointed one way: 13 x 2^-8 = 5e-2
    tol = 2e-5 if dtype == FP32 else 5e-2
    for name, got, want in (("loss", f["loss"], loss), ("dhead", dW, H.grad), ("dstates", t["dkv"], C.grad), ("dqkv", t["dqkv"], A.grad), ("o", t["o2"], o2)):
        want = want.detach().numpy()
        err = np.linalg.norm(host(got) - want) / np.linalg.norm(want)
        assert err < tol, (name, err)
