"""Pins of the operators' definitions (oracle/operators_fp64.py): the 8-bit rounding against torch's own type and against its error
bound, every gradient against differences, and what the entry points refuse (no GPU needed: nothing is launched)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import operators_fp64 as P
from paper_2510_05186_amd import binding as B

RNG = np.random.default_rng(11)


def test_e4m3_table_is_torch_s_type():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(t[:0x7F], P.E4M3) and np.array_equal(t[0x80:0xFF], -P.E4M3) and np.isnan(t[[0x7F, 0xFF]]).all()
    y = np.concatenate([RNG.standard_normal(20000) * 40, RNG.standard_normal(20000) * 2.0 ** -8, (P.E4M3[:-1] + P.E4M3[1:]) / 2, P.E4M3, [0.0, -0.0, 448.0, -448.0]])
    y = np.clip(y, -448, 448).astype(np.float32)
    assert np.array_equal(P.round_e4m3(y.astype(np.float64)), torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("cols", [1, 31, 32, 33, 64, 100])
def test_pack8_is_off_by_half_a_step_at_most_and_is_a_bf16_number(cols):
    x = RNG.standard_normal((50, cols)) * 2.0 ** RNG.integers(-30, 30, (50, 1))
    x[3] = 0
    codes, scales, v = P.pack8(x)
    k = np.repeat(scales.astype(float) - 127, P.BLOCK, axis=1)[:, :cols]
    assert np.all(np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (k - 10)))
    most = np.array([[np.abs(x[r, b * 32:(b + 1) * 32]).max() for b in range(scales.shape[1])] for r in range(50)])
    power = 2.0 ** (scales.astype(float) - 127)
    assert np.all(most <= 448 * power) and np.all((most > 224 * power) | (scales == 10))            # the least power that does
    assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)
    again = P.pack8(v)
    assert np.array_equal(again[2], v)                                                              # what is kept is kept exactly


def test_pack8_at_the_ends_of_the_range():
    big, small = float(np.finfo(np.float32).max), 2.0 ** -140
    x = np.array([[big, -1.75 * 2.0 ** 127, 2.0 ** 120], [small, 2.0 ** -126, 2.0 ** -127], [np.inf, -3.0, np.nan], [np.inf, -np.inf, np.nan], [0.0, -0.0, 0.0],
                  [448.0, 449.0, 1.0]])
    codes, scales, v = P.pack8(x)
    assert list(scales[:, 0]) == [246, 10, 120, 10, 10, 128]
    assert v[0].tolist() == [1.75 * 2.0 ** 127, -1.75 * 2.0 ** 127, 2.0 ** 120] and np.all(np.isfinite(v[0].astype(np.float32)))
    assert v[1].tolist() == [0.0, 2.0 ** -126, 0.0]                                                  # half of the least value goes to the even one, 0
    assert np.isnan(v[2][[0, 2]]).all() and v[2][1] == -3.0 and list(codes[2][[0, 2]]) == [0x7F, 0x7F]
    assert np.isnan(v[3]).all() and codes[3][1] == 0xFF and codes[4][1] == 0x80
    assert v[5].tolist() == [448.0, 448.0, 1.0]


def _differences(f, x, dy, h=1e-6):
    """gradient of <f(x), dy> by central differences"""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        a = (f(x) * dy).sum()
        x[i] = keep - h
        g[i] = (a - (f(x) * dy).sum()) / (2 * h)
        x[i] = keep
    return g


def _near(a, b):
    assert np.max(np.abs(a - b)) <= 1e-7 * max(1.0, np.max(np.abs(b)))


@pytest.mark.parametrize("family", [P.GPT, P.LLAMA])
def test_gradients_are_those_of_differences(family):
    gu, da = RNG.standard_normal((3, 12)), RNG.standard_normal((3, 6 if family == P.LLAMA else 12))
    _near(P.activation_bwd(family, gu, da), _differences(lambda x: P.activation(family, x), gu.copy(), da))
    x, gamma, beta, dn, dres = RNG.standard_normal((3, 10)), 1 + 0.1 * RNG.standard_normal(10), RNG.standard_normal(10), RNG.standard_normal((3, 10)), RNG.standard_normal((3, 10))
    full = lambda x, g, b: P.norm(family, x, g, b, *P.norm_stats(family, x, 1e-3))  # noqa: E731
    dx, dg, db = P.norm_bwd(family, dn, x, *P.norm_stats(family, x, 1e-3), gamma, dres)
    _near(dx - dres, _differences(lambda v: full(v, gamma, beta), x.copy(), dn))
    _near(dg, _differences(lambda v: full(x, v, beta), gamma.copy(), dn))
    if family == P.GPT:
        _near(db, _differences(lambda v: full(x, gamma, v), beta.copy(), dn))


def test_qknorm_gradients_are_those_of_differences():
    n_q, n_kv, d, seq, rows = 4, 2, 8, 3, 5
    x, dy = RNG.standard_normal((2, rows, (n_q + 2 * n_kv) * d))
    gq, gk = 1 + 0.1 * RNG.standard_normal((2, d))
    table = P.rope_table(seq, d, 100.0)
    full = lambda x, gq, gk: P.qknorm(x, P.qknorm_stats(x, n_q + n_kv, d, 1e-3), gq, gk, table, seq, n_q, n_kv, d)  # noqa: E731
    dx, dgq, dgk = P.qknorm_bwd(dy, x, P.qknorm_stats(x, n_q + n_kv, d, 1e-3), gq, gk, table, seq, n_q, n_kv, d)
    _near(dx, _differences(lambda v: full(v, gq, gk), x.copy(), dy))
    _near(dgq, _differences(lambda v: full(x, v, gk), gq.copy(), dy))
    _near(dgk, _differences(lambda v: full(x, gq, v), gk.copy(), dy))
    y = full(x, gq * 0 + 1, gk * 0 + 1).reshape(rows, -1, d)
    assert np.allclose((y[:, :n_q + n_kv] ** 2).mean(2), 1, atol=2e-2)                               # normed, and the rotation keeps the length


def test_embedding_gradient_is_that_of_differences():
    ids, w, dy = np.array([3, 0, 3, -1, 5, 3]), RNG.standard_normal((5, 4)), RNG.standard_normal((6, 4))
    _near(P.embed_bwd(ids, dy, 5, 2.5), _differences(lambda v: P.embed(ids, v, 2.5), w.copy(), dy))
    assert np.all(P.embed(ids, w, 2.5)[[3, 4]] == 0)


# ---- refusals: every entry point, one bad argument at a time.  Pointers are addresses that nothing reads: a refused call launches nothing.
A = 1 << 20
CALLS = {
    "optstage_op_pack8": dict(dtype=1, x=A, ldx=64, codes=A, scales=A, rows=4, cols=64, stream=0),
    "optstage_op_unpack8": dict(dtype=1, codes=A, scales=A, x=A, ldx=64, rows=4, cols=64, stream=0),
    "optstage_op_norm_fwd_pack8": dict(dtype=1, family=0, x=A, gamma=A, beta=A, out=2 * A, stats=A, codes=A, scales=A, rows=4, hidden=64, eps=1e-5,
                                       stream=0),
    "optstage_op_norm_bwd8": dict(dtype=1, family=0, dn=A, codes=A, scales=A, stats=A, gamma=A, beta=A, dres=A, dx=A, out=2 * A, partial=A, dgamma=A, dbeta=2 * A, rows=4, hidden=64,
                                  stream=0),
    "optstage_op_act_fwd_pack8": dict(dtype=1, family=1, gu=A, a=2 * A, codes=A, scales=A, rows=4, ffn=64, stream=0),
    "optstage_op_act_bwd8": dict(dtype=1, family=1, da=A, codes=A, scales=A, dgu=2 * A, a=A, rows=4, ffn=64, stream=0),
    "optstage_op_qknorm_rope": dict(dtype=1, src=A, dst=A, gamma_q=A, gamma_k=A, table=A, stats=A, codes=A, scales=A, rows=4, seq=4, n_q=2, n_kv=1, head_dim=64, eps=1e-5,
                                    stream=0),
    "optstage_op_qknorm_rope8": dict(dtype=1, codes=A, scales=A, stats=A, gamma_q=A, gamma_k=A, table=A, dst=A, rows=4, seq=4, n_q=2, n_kv=1, head_dim=64, stream=0),
    "optstage_op_qknorm_rope_bwd": dict(dtype=1, dy=A, x=A, codes=0, scales=0, stats=A, gamma_q=A, gamma_k=A, table=A, dx=A, partial=A, dgamma_q=A, dgamma_k=2 * A, rows=4, seq=4,
                                        n_q=2, n_kv=1, head_dim=64, stream=0),
    "optstage_op_embed_fwd": dict(dtype=1, ids=A, weight=A, out=A, rows=4, vocab=10, hidden=64, scale=1.0, stream=0),
    "optstage_op_embed_bwd": dict(dtype=1, ids=A, dy=A, grad=A, ws=A, ws_bytes=1 << 30, rows=4, vocab=10, hidden=64, scale=1.0, stream=0),
}
MAY_BE_NULL = {("optstage_op_norm_bwd8", "dres"), ("optstage_op_norm_bwd8", "out"), ("optstage_op_act_bwd8", "a")}
MORE = [
    ("optstage_op_pack8", dict(ldx=63)), ("optstage_op_unpack8", dict(ldx=63)), ("optstage_op_pack8", dict(cols=1 << 30, ldx=1 << 30)), ("optstage_op_pack8", dict(rows=1 << 30)),
    ("optstage_op_norm_fwd_pack8", dict(hidden=60)), ("optstage_op_norm_fwd_pack8", dict(out=A)), ("optstage_op_norm_fwd_pack8", dict(hidden=8200)), ("optstage_op_norm_fwd_pack8", dict(family=2)),
    ("optstage_op_norm_fwd_pack8", dict(dtype=0, hidden=62)), ("optstage_op_norm_fwd_pack8", dict(hidden=(1 << 32) - 8)),
    ("optstage_op_norm_bwd8", dict(hidden=60)), ("optstage_op_norm_bwd8", dict(hidden=8200)), ("optstage_op_norm_bwd8", dict(out=A)), ("optstage_op_norm_bwd8", dict(dx=2 * A)),
    ("optstage_op_act_fwd_pack8", dict(ffn=60)), ("optstage_op_act_fwd_pack8", dict(family=2)), ("optstage_op_act_fwd_pack8", dict(ffn=1 << 29)),
    ("optstage_op_act_fwd_pack8", dict(a=A)), ("optstage_op_norm_bwd8", dict(dbeta=A)), ("optstage_op_qknorm_rope_bwd", dict(dgamma_k=A)),
    ("optstage_op_act_bwd8", dict(ffn=60)), ("optstage_op_act_bwd8", dict(dgu=A)), ("optstage_op_act_bwd8", dict(a=2 * A)), ("optstage_op_act_bwd8", dict(dtype=0, ffn=62)),
    ("optstage_op_qknorm_rope", dict(codes=0)), ("optstage_op_qknorm_rope", dict(scales=0)), ("optstage_op_qknorm_rope", dict(head_dim=96)),
    ("optstage_op_qknorm_rope", dict(head_dim=320)), ("optstage_op_qknorm_rope", dict(n_q=65536)), ("optstage_op_qknorm_rope8", dict(head_dim=32)),
    ("optstage_op_qknorm_rope_bwd", dict(codes=A, scales=A)), ("optstage_op_qknorm_rope_bwd", dict(x=0)), ("optstage_op_qknorm_rope_bwd", dict(x=0, codes=A)),
    ("optstage_op_qknorm_rope_bwd", dict(head_dim=96)), ("optstage_op_qknorm_rope_bwd", dict(seq=1 << 24)),
    ("optstage_op_embed_fwd", dict(hidden=60)), ("optstage_op_embed_fwd", dict(vocab=1 << 31)), ("optstage_op_embed_fwd", dict(rows=1 << 26)),
    ("optstage_op_embed_bwd", dict(hidden=60)), ("optstage_op_embed_bwd", dict(rows=1 << 26)), ("optstage_op_embed_bwd", dict(ws_bytes=16)),
]


def _one_bad_argument():
    for name, args in CALLS.items():
        for key, v in args.items():
            if key == "stream":
                continue
            if v in (A, 2 * A):
                if (name, key) not in MAY_BE_NULL:
                    yield name, {key: 0}
                yield name, {key: v + (2 if key == "ids" else 8)}        # 16-byte alignment; ids of 4 bytes
            elif key == "dtype":
                yield name, {key: 2}
            elif key in ("rows", "cols", "hidden", "ffn", "seq", "n_q", "n_kv", "head_dim", "vocab"):
                yield name, {key: 0}
    yield from MORE


@pytest.mark.parametrize("name,bad", list(_one_bad_argument()), ids=lambda v: v if isinstance(v, str) else ",".join(f"{k}={x}" for k, x in v.items()))
def test_refused_with_a_message(name, bad):
    args = dict(CALLS[name], **bad)
    assert getattr(B.lib(), name)(*args.values()) == B.E_ARG
    assert name.replace("optstage_op_", "").encode() in B.lib().optstage_last_error()


def test_refusals_have_the_arguments_of_the_header():
    for name, args in CALLS.items():
        assert len(args) == len(B._SIGS[name])
        for v, t in zip(args.values(), B._SIGS[name]):
            assert isinstance(v, float) == (t is ctypes.c_float)


def test_embed_workspace_holds_the_sorted_tokens():
    f = B.lib().optstage_op_embed_bwd_ws_bytes
    assert f(1, 8) >= 8 and f(100000, 4096) >= 8 * 100000 and f(1 << 26, 8) == 0
    sizes = [f(n, 4096) for n in range(1, 40000, 97)]
    assert sizes == sorted(sizes)
