"""The embedding's gradient on every route that its tokens can take: which one a call takes goes by its sizes alone (embed_bwd_order,
embed_bwd_places), and the cases below say which they are for, so that one that no longer gets there fails.

Tolerances are bounds per value, EPS = 2^-24 for every fp32 rounding that reaches it: a piece of a run adds up to 32 rows one after the other, a
wave of the join every eighth piece, then eight waves, the scale and the accumulator: min(count, 45 + count / 256) + 3 roundings; a few
tokens (448 at most) are added one after the other.  1.01 covers the products of those roundings."""
import ctypes

import numpy as np
import pytest
import torch

import test_gpu_operators as P8
from gpu_util import TDT, ok, stream
from paper_2510_05186_amd import binding as B

FP32, BF16 = 0, 1
EPS = 2.0 ** -24
FEW, PLACED = "few", "placed"


def route(dtype, rows, vocab, h):
    """-> (how the tokens are ordered: FEW, PLACED or the number of the sort's passes; whether a launch counts ahead of each; places of a wave of the sums)"""
    order, places = (ctypes.CDLL(B.LIB_PATH)[n] for n in ("_Z15embed_bwd_orderij", "_Z16embed_bwd_placesiiji"))
    order.argtypes, places.argtypes = [ctypes.c_int, ctypes.c_uint32], [ctypes.c_int, ctypes.c_int, ctypes.c_uint32, ctypes.c_int]
    n = order(rows, vocab)
    if n == 0:
        return FEW, False, 0
    return PLACED if n < 0 else n, n > 0 and rows > 16384, places(dtype, rows, vocab, h)


# ------------------------------------------------------------------ passes of the sort
# dtype, rows, vocab, hidden, ids, passes; a launch counts ahead of a pass beyond 16384 tokens
PASSES = [(BF16, 9000, 400, 16, "padded", 1), (FP32, 16384, 513, 8, "padded", 2), (BF16, 16385, 513, 8, "padded", 2), (BF16, 10001, (1 << 18) + 1, 8, "padded", 3),
          (FP32, 20000, 1 << 20, 4, "zipf", 3), (BF16, 30011, 1 << 27, 8, "words", 3), (FP32, 9000, 1 << 28, 4, "words", 4), (BF16, 8193, (1 << 27) + 1, 8, "words", 4),
          (FP32, 20000, 1 << 28, 4, "words", 4), (BF16, 33003, (1 << 27) + 1, 8, "words", 4), (FP32, 12345, (1 << 31) - 1, 4, "words", 4), (FP32, 3000, (1 << 31) - 1, 4, "words", PLACED)]


def ids_for(kind, rows, vocab, r):
    """As for the other tests, and "words": some words all over the vocabulary, its ends and padding among them, in no order; "lengths": runs of lengths around
    the pieces of 32, their rows in no order."""
    if kind == "words":
        w = np.concatenate([r.integers(0, vocab, 60), [0, vocab - 1, vocab // 2, vocab // 2 - 1, vocab, -1, np.iinfo(np.int32).min]])
        return w[np.minimum(r.geometric(0.06, rows) - 1, len(w) - 1)].astype(np.int64).clip(-(1 << 31), (1 << 31) - 1).astype(np.int32)
    if kind == "lengths":
        n, t = [1, 2, 31, 32, 33, 7, 34, 63, 64, 65, 1, 1, 95, 96, 97, 3, 8, 128, 9, 200, 24, 40], []
        while len(t) < rows:
            t += [len(set(t)) % vocab] * n[len(set(t)) % len(n)]
        return r.permutation(np.array(t[:rows], np.int32))
    return P8.ids_of(kind, rows, vocab, r)


class Gradient:
    """The buffers of a call: random rows and accumulator, 64 values behind each that nothing may touch."""

    def __init__(self, dtype, rows, vocab, h, kind, seed=0):
        self.shape, self.dtype, self.scale = (rows, vocab, h), dtype, float(np.float32(np.sqrt(h)))
        g = torch.Generator(device="cuda")
        g.manual_seed(1000 * rows + vocab % 997 + 7 * h + seed)
        self.dy = torch.randn((rows, h), generator=g, device="cuda").to(TDT[dtype])
        self.ids = torch.from_numpy(ids_for(kind, rows, vocab, np.random.default_rng([88, rows, vocab, h, seed]))).cuda()
        self.grad, self.c1 = P8.zone((vocab, h), torch.float32, 0.0)
        self.start = None
        if vocab * h < 1 << 28:
            self.grad.copy_(torch.randn((vocab, h), generator=g, device="cuda"))
            self.start = self.grad.clone()
        self.need = B.lib().optstage_op_embed_bwd_ws_bytes(rows, h)
        self.ws, self.c2 = P8.zone((self.need,), torch.uint8, 0xC3)

    def reset(self):
        self.grad.zero_() if self.start is None else self.grad.copy_(self.start)

    def call(self, s=None):
        rows, vocab, h = self.shape
        ok(B.lib().optstage_op_embed_bwd(self.dtype, self.ids.data_ptr(), self.dy.data_ptr(), self.grad.data_ptr(), self.ws.data_ptr(), self.need, rows, vocab, h, self.scale,
                                         stream() if s is None else s))

    def check(self):
        """The rows of all tokens that occur against sums in 64 bits; the others as they were.  Leaves the accumulator as it was."""
        rows, vocab, h = self.shape
        torch.cuda.synchronize()
        ids = self.ids.long().cpu()
        valid = (ids >= 0) & (ids < vocab)
        words, run, count = torch.unique(ids[valid], return_inverse=True, return_counts=True)
        dy = self.dy.cpu()[valid].double()
        sums = torch.zeros((len(words), h), dtype=torch.float64).index_add_(0, run, dy)
        sizes = torch.zeros((len(words), h), dtype=torch.float64).index_add_(0, run, dy.abs())
        at = words.cuda()
        was = torch.zeros((len(words), h), dtype=torch.float64) if self.start is None else self.start[at].double().cpu()
        k = (count if rows <= 448 else torch.minimum(count, 45 + count // 256)) + 3
        bound = 1.01 * EPS * k[:, None] * (self.scale * sizes + was.abs())
        if len(words):
            off = (self.grad[at].double().cpu() - (was + self.scale * sums)).abs()
            bad = ~(off <= bound)
            assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:4].tolist(), words[torch.nonzero(bad)[:4, 0]].tolist(), off[bad][:4], bound[bad][:4])
            got = self.grad[at].clone()
            self.grad[at] = was.float().cuda()
        else:
            got = self.grad[:0].clone()
        assert not self.grad.any() if self.start is None else torch.equal(self.grad, self.start)
        assert self.c1() and self.c2()
        return at, got


@pytest.mark.parametrize("dtype,rows,vocab,h,kind,passes", PASSES)
def test_a_case_for_a_number_of_passes_takes_them(dtype, rows, vocab, h, kind, passes):
    assert route(dtype, rows, vocab, h)[:2] == (passes, passes != PLACED and rows > 16384)


def test_the_cases_reach_every_number_of_passes():
    """One to four, with and without the launch that counts; padding among the tokens of each form of the sort."""
    reached = {route(*c[:4])[:2] for c in PASSES}
    assert reached >= {(n, counted) for n in (2, 3, 4) for counted in (False, True)} | {(1, False)}
    assert {(c[5] == 1, c[1] > 16384) for c in PASSES if c[4] in ("padded", "words")} >= {(True, False), (False, False), (False, True)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,vocab,h,kind,passes", PASSES)
def test_gradient_by_passes_of_the_sort(dtype, rows, vocab, h, kind, passes):
    P8.room(16 + vocab * h * 4 * 1.5 / 2 ** 30)
    g = Gradient(dtype, rows, vocab, h, kind)
    g.call()
    at, first = g.check()
    g.call()
    torch.cuda.synchronize()
    assert torch.equal(g.grad[at], first)


# ------------------------------------------------------------------ rows of several waves, runs around the pieces, every number of places
# dtype, rows, vocab, hidden, ids, places of a wave.  More than 2048 columns (fp32: 1024) take workgroups side by side
SUMS = [(BF16, 600, 900, 4104, "zipf", 8), (BF16, 2100, 7, 2056, "one", 8), (BF16, 1500, 300, 1544, "lengths", 8), (BF16, 5000, 300, 2056, "zipf", 16), (BF16, 5000, 300, 2056, "padded", 16),
        (BF16, 9000, 2000, 2056, "lengths", 16), (BF16, 33000, 500, 1032, "padded", 32), (BF16, 20000, 3, 2600, "zipf", 32), (BF16, 25000, 1100, 2056, "lengths", 32),
        (FP32, 2000, 50, 1352, "zipf", 8), (FP32, 2000, 50, 1352, "one", 8), (FP32, 2000, 5000, 516, "lengths", 8), (FP32, 3000, 64, 1352, "padded", 16), (FP32, 4097, 5000, 1100, "all", 16),
        (FP32, 4500, 200, 1028, "lengths", 16), (FP32, 17000, 821, 1352, "zipf", 32), (FP32, 20000, 900, 1284, "lengths", 32), (FP32, 17000, 40, 1352, "one", 32)]


@pytest.mark.parametrize("dtype,rows,vocab,h,kind,places", SUMS)
def test_a_case_for_a_number_of_places_takes_them(dtype, rows, vocab, h, kind, places):
    assert route(dtype, rows, vocab, h)[2] == places


def test_the_cases_reach_every_number_of_places_in_rows_of_several_workgroups():
    for dtype, one_group in ((BF16, 2048), (FP32, 1024)):
        assert {c[5] for c in SUMS if c[0] == dtype and c[3] > one_group} == {8, 16, 32}
        assert {c[5] for c in SUMS if c[0] == dtype and c[4] == "lengths"} == {8, 16, 32}
    ids = ids_for("lengths", 25000, 1100, np.random.default_rng(1))
    assert set(np.bincount(ids)) >= {1, 31, 32, 33, 63, 64, 65, 96, 200}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,rows,vocab,h,kind,places", SUMS)
def test_gradient_of_rows_of_several_waves(dtype, rows, vocab, h, kind, places):
    g = Gradient(dtype, rows, vocab, h, kind)
    g.call()
    at, first = g.check()
    g.call()
    torch.cuda.synchronize()
    assert torch.equal(g.grad[at], first)


# ------------------------------------------------------------------ replayed with other tokens, and several calls at once
# counting the keys ahead; the sort by itself; with a launch that counts: all of them several launches that leave their order, and how many runs
# are long, in the workspace for the next one
LAUNCHES = [(BF16, 600, 500, 264, PLACED), (FP32, 9000, 2000, 36, 2), (BF16, 20000, 2000, 40, 2)]


def test_the_cases_for_replays_take_several_launches():
    assert [route(*c[:4])[:2] for c in LAUNCHES] == [(PLACED, False), (2, False), (2, True)]


@pytest.mark.gpu
@pytest.mark.parametrize("shared", [False, True], ids=["own workspaces", "one workspace after the other"])
def test_gradient_captured_once_and_replayed_with_other_tokens(shared):
    """Long runs, none, tokens of one word, padding alone: every replay gives what the eager call gives for those tokens."""
    sets = [Gradient(*c[:4], "none", seed=3) for c in LAUNCHES]
    if shared:
        most = max(sets, key=lambda g: g.need)
        for g in sets:
            g.ws, g.c2 = most.ws, most.c2
    side = torch.cuda.Stream()
    graphs = []
    for g in sets:
        g.call()                                                   # once before the capture, which may load no code
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            g.call(torch.cuda.current_stream().cuda_stream)
    for turn, kind in enumerate(["zipf", "all", "one", "none", "lengths", "padded", "one", "all"]):
        for g in sets:
            rows, vocab, _ = g.shape
            g.ids.copy_(torch.from_numpy(ids_for(kind, rows, vocab, np.random.default_rng([89, rows, turn]))))
            g.reset()
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        replayed = [g.check() for g in sets]
        for g, (at, got) in zip(sets, replayed):
            g.reset()
            g.call()
            torch.cuda.synchronize()
            assert torch.equal(g.grad[at], got), (g.shape, kind)
        torch.ones(1 << 20, device="cuda").sum().item()


@pytest.mark.gpu
def test_gradients_of_many_tokens_on_two_streams_at_once():
    sets = [[Gradient(*c[:4], kind, seed=4 + k) for c in LAUNCHES] for k, kind in enumerate(("zipf", "lengths"))]
    streams = [torch.cuda.Stream() for _ in sets]
    alone = []
    for k in range(2):
        for g in sets[k]:
            g.call()
        alone.append([g.check() for g in sets[k]])
    for _ in range(4):
        for g in sets[0] + sets[1]:
            g.reset()
        torch.cuda.synchronize()
        for i in range(len(LAUNCHES)):
            for k in range(2):
                sets[k][i].call(streams[k].cuda_stream)
        torch.cuda.synchronize()
        for k in range(2):
            for g, (at, got) in zip(sets[k], alone[k]):
                assert torch.equal(g.grad[at], got), (g.shape, k)
