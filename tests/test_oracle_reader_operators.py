"""Pins of the fp64 definitions of rotary positions with several axes, cross attention and the loss against a teacher's top entries: differences,
torch's autograd of stock operations, identities."""
import numpy as np
import pytest
import torch

from oracle import operators_fp64 as P


def rng(*key):
    return np.random.default_rng([78, *key])


def differences(f, x, dy, h=1e-6):
    """Central differences of <f(x), dy>, element by element."""
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += h
        lo[i] -= h
        g[i] = ((f(hi) - f(lo)) * dy).sum() / (2 * h)
    return g


def test_axes_that_agree_are_the_rotation_by_the_row_s_position():
    r = rng(1)
    x, table = r.standard_normal((12, 5, 16)), P.rope_table(6, 16, 10000.0)
    pos = np.tile(np.arange(12) % 6, (3, 1))
    want = P.rotate(x[:, :3], table, 6)
    got = P.rope_axes(x, table, pos, [0, 1, 2, 2, 1, 0, 1, 2], 3)
    assert np.allclose(got[:, :3], want, atol=1e-14) and np.array_equal(got[:, 3:], x[:, 3:])


def test_rotation_by_axes_keeps_lengths_turns_back_and_leaves_padding():
    r = rng(2)
    x, table = r.standard_normal((7, 2, 8)), P.rope_table(9, 8, 100.0)
    pos, axis = r.integers(-2, 11, (2, 7)), [0, 255, 1, 0]
    y = P.rope_axes(x, table, pos, axis, 2)
    assert np.allclose((y ** 2).sum(2), (x ** 2).sum(2)) and np.allclose(P.rope_axes(y, table, pos, axis, 2, -1), x, atol=1e-14)
    assert np.array_equal(y[..., [1, 5]], x[..., [1, 5]])
    off = (pos[0] < 0) | (pos[0] >= 9)
    assert off.any() and np.array_equal(y[off][..., [0, 3, 4, 7]], x[off][..., [0, 3, 4, 7]])
    # scores of two turned heads go by the difference of positions
    a, b = np.ones((1, 1, 8)), np.ones((1, 1, 8))
    s = [(P.rope_axes(a, table, [[p], [p + 1]], axis, 1) * P.rope_axes(b, table, [[p + 2], [p + 4]], axis, 1)).sum() for p in range(4)]
    assert np.allclose(s, s[0])


@pytest.mark.parametrize("heads,n_kv,lens", [(2, 2, (5, 3)), (4, 2, (0, 5)), (3, 1, (1, 4))])
def test_cross_attention_against_autograd_and_differences(heads, n_kv, lens):
    r = rng(3, heads)
    q, k, v, g = r.standard_normal((2, 4, heads, 6)), r.standard_normal((2, 5, n_kv, 6)), r.standard_normal((2, 5, n_kv, 6)), r.standard_normal((2, 4, heads, 6))
    o, lse = P.cross_attn(q, k, v, lens)
    dq, dk, dv = P.cross_attn_bwd(q, k, v, lens, g)
    for f, x, d in ((lambda x: P.cross_attn(x, k, v, lens)[0], q, dq), (lambda x: P.cross_attn(q, x, v, lens)[0], k, dk), (lambda x: P.cross_attn(q, k, x, lens)[0], v, dv)):
        assert np.allclose(d, differences(f, x, g), atol=1e-8)
    for i, n in enumerate(lens):
        if n == 0:
            assert not o[i].any() and np.all(lse[i] == -np.inf) and not dq[i].any() and not dk[i].any() and not dv[i].any()
            continue
        T = [torch.tensor(t, requires_grad=True) for t in (q[i], k[i, :n], v[i, :n])]
        rep = heads // n_kv
        att = torch.nn.functional.scaled_dot_product_attention(T[0].transpose(0, 1), T[1].transpose(0, 1).repeat_interleave(rep, 0), T[2].transpose(0, 1).repeat_interleave(rep, 0))
        att.transpose(0, 1).backward(torch.tensor(g[i]))
        assert np.allclose(att.detach().transpose(0, 1).numpy(), o[i], atol=1e-12)
        for got, t in ((dq[i], T[0]), (dk[i, :n], T[1]), (dv[i, :n], T[2])):
            assert np.allclose(got, t.grad.numpy(), atol=1e-12)
        assert not dk[i, n:].any() and not dv[i, n:].any()


def test_cross_attention_ignores_what_lies_behind_the_states():
    r = rng(4)
    q, k, v, g = r.standard_normal((1, 3, 2, 4)), r.standard_normal((1, 6, 2, 4)), r.standard_normal((1, 6, 2, 4)), r.standard_normal((1, 3, 2, 4))
    a = P.cross_attn(q, k, v, [4]) + P.cross_attn_bwd(q, k, v, [4], g)
    k[0, 4:], v[0, 4:] = np.nan, np.inf
    b = P.cross_attn(q, k, v, [4]) + P.cross_attn_bwd(q, k, v, [4], g)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))
    one = P.cross_attn_bwd(q, k, v, [1], g)
    assert not one[0].any() and not one[1].any() and np.allclose(one[2][0, 0], g[0].sum(0))


@pytest.mark.parametrize("temperature,log_probs", [(1.0, 0), (2.0, 0), (1.0, 1), (0.5, 1)])
def test_distillation_against_autograd_and_differences(temperature, log_probs):
    r = rng(5, int(10 * temperature), log_probs)
    z, teacher, dloss = 2 * r.standard_normal((6, 11)), r.standard_normal((6, 5)), r.standard_normal(6)
    ids = r.integers(-2, 13, (6, 5))
    ids[0] = [3, 3, 1, 3, 1]                # words given twice
    ids[1] = -1                             # a row without entries
    teacher[2, 1:3] = -np.inf
    if log_probs:
        teacher -= 3.0
    loss, lse = P.distill(z, ids, teacher, temperature, log_probs)
    dz = P.distill_bwd(z, ids, teacher, temperature, log_probs, dloss)
    assert np.allclose(dz, differences(lambda x: P.distill(x, ids, teacher, temperature, log_probs)[0][:, None], z, dloss[:, None]), atol=1e-8)
    assert loss[1] == 0 and not dz[1].any()
    Z = torch.tensor(z, requires_grad=True)
    logp = torch.log_softmax(Z / temperature, 1)
    assert np.allclose(lse, torch.logsumexp(torch.tensor(z) / temperature, 1).numpy())
    total = 0
    for row in range(6):
        ok = (ids[row] >= 0) & (ids[row] < 11) & np.isfinite(teacher[row])
        if not ok.any():
            continue
        t = torch.tensor(teacher[row][ok])
        t = torch.exp(t) if log_probs else torch.softmax(t / temperature, 0)
        kl = (t * (torch.log(t) - logp[row, torch.tensor(ids[row][ok])])).sum()
        assert np.isclose(kl.item(), loss[row])
        total = total + dloss[row] * kl
    total.backward()
    assert np.allclose(Z.grad.numpy(), dz, atol=1e-12)


def test_distillation_is_zero_where_student_and_teacher_agree():
    r = rng(6)
    z = r.standard_normal((2, 7))
    ids = np.tile(np.arange(7), (2, 1))
    loss, lse = P.distill(z, ids, z, 1.7, 0)
    assert np.allclose(loss, 0, atol=1e-15) and np.allclose(P.distill_bwd(z, ids, z, 1.7, 0, np.ones(2)), 0, atol=1e-16)
    logp = z - lse[:, None]                  # lse is of z / 1.7: at temperature 1 the log-probabilities are others
    assert not np.allclose(np.exp(logp).sum(1), 1)
