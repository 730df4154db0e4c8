"""Timed cases of what a stage needs whose model reads images or states of an encoder and learns from a teacher: rotary positions with several axes,
cross attention, and the loss against a teacher's top logits.

A pass is what a training step does with an operator: forward, and backward from what forward left.  "kind":
  cross    attention of queries to the states of another sequence, of which the first kv_len count; with "train" its gradients
  rope     rotation of query and key heads by positions of several axes, and its gradient
  distill  Kullback-Leibler loss against a teacher's top entries and its gradient in the logits; "fused": both from one reading of the logits
"""
import math
from types import SimpleNamespace

import torch

own = False

FP32, BF16 = 0, 1
TORCH = {FP32: torch.float32, BF16: torch.bfloat16}
ROPE_BASE = 10000.0


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the tiny fp32 stage's heads over the states of a short sentence: latency
        {"name": "cross_tiny_fp32", "kind": "cross", "dtype": FP32, "batch": 1, "seq_q": 128, "seq_kv": 77, "n_q": 4, "n_kv": 4, "head_dim": 64, "ragged": False, "train": True},
        # the Llama-style layer reading the patches of four images
        {"name": "cross_images", "kind": "cross", "dtype": BF16, "batch": 1, "seq_q": 4096, "seq_kv": 2305, "n_q": 32, "n_kv": 32, "head_dim": 128, "ragged": False, "train": True},
        # the grouped-query stage reading states as long as its own sequence: the largest
        {"name": "cross_gqa_4k", "kind": "cross", "dtype": BF16, "batch": 1, "seq_q": 4096, "seq_kv": 4096, "n_q": 64, "n_kv": 8, "head_dim": 128, "ragged": False, "train": True},
        # the micro-batch of eight sequences, each with as many states as its source has, one of them with none: a padded batch
        {"name": "cross_padded_batch", "kind": "cross", "dtype": BF16, "batch": 8, "seq_q": 1024, "seq_kv": 1500, "n_q": 16, "n_kv": 8, "head_dim": 64, "ragged": True, "train": True},
        # one new token of each of sixteen answers over long sources: evaluation between training steps
        {"name": "cross_one_token", "kind": "cross", "dtype": BF16, "batch": 16, "seq_q": 1, "seq_kv": 16384, "n_q": 32, "n_kv": 8, "head_dim": 128, "ragged": True, "train": False},
        # a few heads of 64 in fp32: a small model or a debugging session
        {"name": "rope_tiny_fp32", "kind": "rope", "dtype": FP32, "rows": 128, "n_rot": 8, "n_pass": 4, "head_dim": 64, "axes": 3, "interleaved": False, "pad": 0},
        # queries and keys of the grouped-query stage, text around a film
        {"name": "rope_gqa_film", "kind": "rope", "dtype": BF16, "rows": 8192, "n_rot": 72, "n_pass": 8, "head_dim": 128, "axes": 3, "interleaved": False, "pad": 0},
        # an odd number of tokens and heads, axes taking turns over the pairs, rows that are part of wider ones
        {"name": "rope_ragged", "kind": "rope", "dtype": BF16, "rows": 2999, "n_rot": 13, "n_pass": 0, "head_dim": 128, "axes": 2, "interleaved": True, "pad": 136},
        # the tiny stage's tokens over a small vocabulary
        {"name": "distill_tiny_fp32", "kind": "distill", "dtype": FP32, "rows": 128, "vocab": 1000, "pad": 0, "k": 8, "temperature": 1.0, "log_probs": False, "fused": False, "masked": 0.0},
        # a micro-batch of the Llama-style model: 4096 tokens of a 32000-word vocabulary, forward and backward as two calls
        {"name": "distill_32k", "kind": "distill", "dtype": BF16, "rows": 4096, "vocab": 32000, "pad": 0, "k": 64, "temperature": 2.0, "log_probs": False, "fused": False, "masked": 0.0},
        # a large vocabulary, the teacher's stored log-probabilities, the last three tenths of the tokens padding
        {"name": "distill_128k_masked", "kind": "distill", "dtype": BF16, "rows": 4096, "vocab": 131072, "pad": 0, "k": 128, "temperature": 1.0, "log_probs": True, "fused": True, "masked": 0.3},
        # the last few tokens of a batch over a vocabulary of no round size
        {"name": "distill_few_rows", "kind": "distill", "dtype": BF16, "rows": 7, "vocab": 150001, "pad": 23, "k": 50, "temperature": 1.0, "log_probs": False, "fused": True, "masked": 0.0},
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step) * step))


def draw(rng):
    kind = rng.choice(["cross", "cross", "cross", "rope", "distill", "distill"])
    dtype = BF16 if rng.random() < 0.75 else FP32
    if kind == "cross":
        n_kv, d = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 128, 128])
        n_q, batch = n_kv * rng.choice([1, 1, 2, 4, 8]), rng.choice([1, 1, 2, 3, 4, 8, 16])
        train = rng.random() < 0.75
        seq_q, seq_kv = (_log_int(rng, 16, 8192) if train else _log_int(rng, 1, 64)), _log_int(rng, 2, 16384)
        most = 64 * 4096 * 4096 if dtype == BF16 else 4 * 4096 * 4096
        while batch * n_q * seq_q * seq_kv > most:
            batch, seq_q, seq_kv = max(1, batch // 2), max(1, seq_q * 3 // 4), max(2, seq_kv * 3 // 4)
        return {"kind": kind, "dtype": dtype, "batch": batch, "seq_q": seq_q, "seq_kv": seq_kv, "n_q": n_q, "n_kv": n_kv, "head_dim": d,
                "ragged": rng.random() < 0.4, "train": train}
    if kind == "rope":
        d, n_kv = rng.choice([32, 64, 128, 128, 256]), rng.choice([1, 2, 4, 5, 8])
        n_rot, n_pass = n_kv * rng.choice([1, 2, 3, 5, 9]), n_kv * rng.choice([0, 1])
        return {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, min(16384, 80_000_000 // ((n_rot + n_pass) * d))), "n_rot": n_rot, "n_pass": n_pass, "head_dim": d,
                "axes": rng.choice([1, 2, 3, 3, 4]), "interleaved": rng.random() < 0.4, "pad": rng.choice([0, 0, 8, 72])}
    vocab = _log_int(rng, 100, 262144)
    if rng.random() < 0.5:
        vocab = -(-vocab // 64) * 64
    return {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, min(16384, 500_000_000 // vocab // (1 if dtype == BF16 else 2))), "vocab": vocab, "pad": rng.choice([0, 0, 0, 5, 64]),
            "k": min(vocab, _log_int(rng, 1, 256)), "temperature": rng.choice([1.0, 1.0, 2.0, 0.7]), "log_probs": rng.random() < 0.4, "fused": rng.random() < 0.6,
            "masked": rng.choice([0.0, 0.0, 0.1, 0.5])}


# ---------------------------------------------------------------------------------------------- inputs
class _Draw:
    """Seeded normal tensors on the device."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(0xC805 + 7919 * int(seed))

    def __call__(self, shape, dtype, std=1.0, mean=0.0):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(TORCH[dtype])

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def whole(self, lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=torch.int64)


def _axis_of_pairs(case):
    """The axis of each of a head's pairs: in turn, or one run of pairs each, the first (time) half as long as the others where there are several."""
    half, axes = case["head_dim"] // 2, case["axes"]
    if case["interleaved"]:
        return [p % axes for p in range(half)]
    parts = 2 * axes - 1
    return [min(axes - 1, (p * parts // half + 1) // 2) for p in range(half)]


def _positions(rows, axes):
    """Text (all axes alike), a film's patches (time, height, width, and a fourth axis that counts films), text again, one row of int32 per axis."""
    r = torch.arange(rows, device="cuda")
    first, last = rows // 4, rows - rows // 4
    side = max(1, math.isqrt(max(1, (last - first) // 8)))
    p = r - first
    film = torch.stack([first + p // (side * side), first + p // side % side, first + p % side, first + 0 * p])
    after = first + max(side, (last - first) // (side * side) + 1)
    return torch.where(r < first, r, torch.where(r < last, film, after + r - last))[:axes].to(torch.int32).contiguous()


def _cross_ws_bytes(case):
    """At least optstage_op_cross_attn_ws_bytes: a number per query row and head, and up to 256 MiB of partial sums."""
    return 8 * case["batch"] * case["n_q"] * case["seq_q"] + (257 << 20)


def prepare(case, seed):
    d, kind, dt = _Draw(seed), case["kind"], case["dtype"]
    s = SimpleNamespace(case=case)
    empty = lambda *shape, dtype=TORCH[dt]: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "cross":
        b, hd, wq, wk = case["batch"], case["head_dim"], case["n_q"] * case["head_dim"], case["n_kv"] * case["head_dim"]
        s.q, s.kv = d((b * case["seq_q"], wq), dt), d((b * case["seq_kv"], 2 * wk), dt)     # kv: a state's key heads, then its value heads
        s.o, s.lse = empty(b * case["seq_q"], wq), empty(b, case["n_q"], case["seq_q"], dtype=torch.float32)
        if case["ragged"]:
            s.kv_len = d.whole(1, case["seq_kv"] + 1, (b,)).to(torch.int32)
            if b > 2:
                s.kv_len[1] = 0
        if case["train"]:
            s.dout = d((b * case["seq_q"], wq), dt, 1e-3)
            s.dq, s.dkv = empty(b * case["seq_q"], wq), empty(b * case["seq_kv"], 2 * wk)
        s.ws = empty(_cross_ws_bytes(case), dtype=torch.uint8)
    elif kind == "rope":
        hd, rows = case["head_dim"], case["rows"]
        s.width = (case["n_rot"] + case["n_pass"]) * hd
        ld = s.width + case["pad"]
        s.x, s.dy = d((rows, ld), dt), d((rows, ld), dt, 1e-3)
        s.positions = _positions(rows, case["axes"])
        angle = torch.arange(rows + 8, dtype=torch.float64, device="cuda")[:, None] * torch.pow(
            torch.tensor(ROPE_BASE, dtype=torch.float64, device="cuda"), -torch.arange(hd // 2, dtype=torch.float64, device="cuda") * 2 / hd)
        s.table = torch.stack([torch.cos(angle), torch.sin(angle)], -1).float().contiguous()
        s.axis = bytes(_axis_of_pairs(case))
        s.y, s.dx = empty(rows, s.width), empty(rows, s.width)
    else:
        rows, vocab, k, ld = case["rows"], case["vocab"], case["k"], case["vocab"] + case["pad"]
        s.z = d((rows, ld), dt, 2.0)
        # the teacher's entries: k different words a row, logits that fall off with the rank; the student is about right there
        step = 1 + d.whole(0, max(1, vocab // k), (rows, 1))
        ids = (d.whole(0, vocab, (rows, 1)) + step * torch.arange(k, device="cuda")) % vocab
        value = 12.0 - 1.5 * torch.log1p(torch.arange(k, device="cuda", dtype=torch.float32)) + 0.3 * d((rows, k), FP32)
        s.z.scatter_(1, ids, (value + d((rows, k), FP32)).to(TORCH[dt]))
        if case["log_probs"]:                                               # of all words, those beyond the top k have some of it
            value = value - torch.log(torch.exp(value).sum(1, keepdim=True) * 1.05)
        ids = torch.where(d.uniform((rows, k)) < 0.02, torch.full_like(ids, -1), ids)      # a teacher that gave fewer
        s.ids, s.teacher = ids.to(torch.int32), value.contiguous()
        s.dloss = torch.full((rows,), 1.0 / rows, dtype=torch.float32, device="cuda")
        s.dloss[rows - int(case["masked"] * rows):] = 0.0
        s.loss, s.lse = empty(rows, dtype=torch.float32), empty(rows, dtype=torch.float32)
        s.dz = empty(rows, vocab)
        s.ws = empty(1 << 20, dtype=torch.uint8)                            # at least optstage_op_distill_ws_bytes
    s.at = {k: v.data_ptr() for k, v in vars(s).items() if isinstance(v, torch.Tensor)}     # the buffers stay where they are
    return s


# ---------------------------------------------------------------------------------------------- the plain form
def _by_kv_head(case, t, heads):
    """[batch * seq, heads * d] -> [batch, n_kv, rows of all its heads, d] in 32 bits"""
    b, d, n_kv = case["batch"], case["head_dim"], case["n_kv"]
    t = t.float().view(b, -1, heads, d).transpose(1, 2)
    return t.reshape(b, n_kv, -1, d)


def _by_row(case, t, heads):
    b, d = case["batch"], case["head_dim"]
    return t.reshape(b, heads, -1, d).transpose(1, 2).reshape(-1, heads * d)


def _cross_plain(s):
    case = s.case
    dtype, n_q, n_kv, wk = TORCH[case["dtype"]], case["n_q"], case["n_kv"], case["n_kv"] * case["head_dim"]
    scale = 1.0 / math.sqrt(case["head_dim"])
    q, k, v = _by_kv_head(case, s.q, n_q), _by_kv_head(case, s.kv[:, :wk], n_kv), _by_kv_head(case, s.kv[:, wk:], n_kv)
    seen = None
    if case["ragged"]:
        seen = torch.arange(case["seq_kv"], device="cuda")[None, :] < s.kv_len[:, None]
        seen = seen[:, None, None, :]
        v = torch.where(seen.transpose(2, 3), v, torch.zeros((), device="cuda"))
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    if seen is not None:
        p = p.masked_fill_(~seen, -math.inf)
    most = p.amax(3, keepdim=True)
    most = torch.where(most == -math.inf, torch.zeros_like(most), most)
    p = p.sub_(most).exp_()
    total = p.sum(3, keepdim=True)
    some = torch.where(total > 0, total, torch.ones_like(total))
    p = p.div_(some)
    o = torch.matmul(p, v)
    got = {"o": _by_row(case, o, n_q).to(dtype), "lse": (most + torch.log(total)).reshape(case["batch"], n_q, -1)}
    if not case["train"]:
        return got
    do = _by_kv_head(case, s.dout, n_q)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(3, keepdim=True)).mul_(p)
    if seen is not None:
        k = torch.where(seen.transpose(2, 3), k, torch.zeros((), device="cuda"))
    dq, dk = torch.matmul(ds, k) * scale, torch.matmul(ds.transpose(2, 3).contiguous(), q) * scale
    return dict(got, dq=_by_row(case, dq, n_q).to(dtype), dk=_by_row(case, dk, n_kv).to(dtype), dv=_by_row(case, dv, n_kv).to(dtype))


def _rope_plain(s):
    case = s.case
    rows, n_rot, dtype = case["rows"], case["n_rot"], TORCH[case["dtype"]]
    at = s.positions[torch.tensor(list(s.axis), device="cuda")].long().T                  # [rows, pairs]
    angle = s.table[at, torch.arange(at.shape[1], device="cuda")]
    c, sn = angle[:, None, :, 0], angle[:, None, :, 1]

    def turned(t, sign):
        t = t[:, :s.width].float().view(rows, -1, case["head_dim"])
        lo, hi = t[:, :n_rot].chunk(2, 2)
        return torch.cat([torch.cat([lo * c - sign * hi * sn, hi * c + sign * lo * sn], 2), t[:, n_rot:]], 1).to(dtype).view(rows, -1)
    return {"y": turned(s.x, 1.0), "dx": turned(s.dy, -1.0)}


def _distill_plain(s):
    case = s.case
    z, ids, dtype = s.z[:, :case["vocab"]].float() / case["temperature"], s.ids.long(), TORCH[case["dtype"]]
    given = (ids >= 0) & (ids < case["vocab"])
    at = torch.where(given, ids, torch.zeros_like(ids))
    if case["log_probs"]:
        log_t = s.teacher.double()
        t = torch.where(given, torch.exp(log_t), torch.zeros_like(log_t))
    else:
        v = torch.where(given, s.teacher.double() / case["temperature"], torch.full((), -math.inf, device="cuda", dtype=torch.float64))
        most = v.amax(1, keepdim=True)
        most = torch.where(most == -math.inf, torch.zeros_like(most), most)
        total = torch.exp(v - most).sum(1, keepdim=True)
        total = torch.where(total > 0, total, torch.ones_like(total))
        t, log_t = torch.exp(v - most) / total, v - most - torch.log(total)
    most = z.amax(1, keepdim=True)
    e = torch.exp(z - most)
    total = e.sum(1, keepdim=True)
    lse = most.double() + torch.log(total.double())
    loss = torch.where(t > 0, t * (log_t - z.gather(1, at).double() + lse), torch.zeros_like(t)).sum(1)
    p = e.div_(total)
    weight = (s.dloss / case["temperature"])[:, None]
    dz = p.mul_(t.sum(1, keepdim=True).float()).scatter_add_(1, at, -t.float()).mul_(weight)
    dz = torch.where(weight != 0, dz, torch.zeros((), device="cuda"))
    return {"loss": loss.float(), "lse": lse[:, 0].float(), "dz": dz.to(dtype)}


# ---------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2510_05186_amd import binding as B
    lib, case, at = B.lib(), s.case, s.at
    kind, dt, stream = case["kind"], case["dtype"], torch.cuda.current_stream().cuda_stream
    if kind == "cross":
        shape = (case["seq_q"], case["seq_kv"], case["batch"], case["n_q"], case["n_kv"], case["head_dim"])
        wq, wk = case["n_q"] * case["head_dim"], case["n_kv"] * case["head_dim"]
        values, lens = wk * s.kv.element_size(), at.get("kv_len", 0)       # the value heads behind the key heads
        B.check(lib.optstage_op_cross_attn_fwd(dt, at["q"], wq, at["kv"], at["kv"] + values, 2 * wk, lens, at["o"], at["lse"], at["ws"], s.ws.numel(), *shape, stream))
        got = {"o": s.o, "lse": s.lse}
        if case["train"]:
            B.check(lib.optstage_op_cross_attn_bwd(dt, at["q"], wq, at["kv"], at["kv"] + values, 2 * wk, lens, at["o"], at["dout"], at["lse"], at["dq"], at["dkv"],
                                                   at["dkv"] + values, at["ws"], s.ws.numel(), *shape, stream))
            got |= {"dq": s.dq, "dk": s.dkv[:, :wk], "dv": s.dkv[:, wk:]}
        return got
    if kind == "rope":
        shape = (case["rows"], case["n_rot"], case["n_pass"], case["head_dim"])
        ld = s.x.shape[1]
        B.check(lib.optstage_op_rope_axes(dt, at["x"], ld, at["y"], s.width, at["table"], s.table.shape[0], at["positions"], case["axes"], s.axis, *shape, 0, stream))
        B.check(lib.optstage_op_rope_axes(dt, at["dy"], ld, at["dx"], s.width, at["table"], s.table.shape[0], at["positions"], case["axes"], s.axis, *shape, 1, stream))
        return {"y": s.y, "dx": s.dx}
    shape = (case["rows"], case["vocab"], case["k"], case["temperature"], int(case["log_probs"]))
    ld = s.z.shape[1]
    if case["fused"]:
        B.check(lib.optstage_op_distill(dt, at["z"], ld, at["ids"], at["teacher"], at["dloss"], at["loss"], at["lse"], at["dz"], case["vocab"], at["ws"], s.ws.numel(), *shape, stream))
    else:
        B.check(lib.optstage_op_distill_fwd(dt, at["z"], ld, at["ids"], at["teacher"], at["loss"], at["lse"], at["ws"], s.ws.numel(), *shape, stream))
        B.check(lib.optstage_op_distill_bwd(dt, at["z"], ld, at["ids"], at["teacher"], at["lse"], at["dloss"], at["dz"], case["vocab"], *shape, stream))
    return {"loss": s.loss, "lse": s.lse, "dz": s.dz}


def run(state):
    if own:
        return _own(state)
    return {"cross": _cross_plain, "rope": _rope_plain, "distill": _distill_plain}[state.case["kind"]](state)


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits
def _cross_exact(s):
    """Head by head, a query's weights as exp(score - log of the sum of exp(score)) over the states that count."""
    case = s.case
    b, hd, n_q, n_kv, nq, nk = (case[x] for x in ("batch", "head_dim", "n_q", "n_kv", "seq_q", "seq_kv"))
    q, kv = s.q.view(b, nq, n_q, hd), s.kv.view(b, nk, 2 * n_kv, hd)
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    got = {"o": zeros(b, nq, n_q, hd), "lse": zeros(b, n_q, nq) - math.inf}
    if case["train"]:
        dout = s.dout.view(b, nq, n_q, hd)
        got |= {"dq": zeros(b, nq, n_q, hd), "dk": zeros(b, nk, n_kv, hd), "dv": zeros(b, nk, n_kv, hd)}
    lens = s.kv_len.tolist() if case["ragged"] else [nk] * b
    for i, n in enumerate(lens):
        for a in range(n_q if n else 0):
            h = a * n_kv // n_q
            Q, K, V = q[i, :, a].double() / math.sqrt(hd), kv[i, :n, h].double(), kv[i, :n, n_kv + h].double()
            score = Q @ K.T
            got["lse"][i, a] = torch.logsumexp(score, 1)
            w = torch.exp(score - got["lse"][i, a][:, None])
            got["o"][i, :, a] = w @ V
            if case["train"]:
                g = dout[i, :, a].double()
                dw = g @ V.T
                dscore = w * (dw - torch.linalg.vecdot(w, dw)[:, None])
                got["dv"][i, :n, h] += w.T @ g
                got["dk"][i, :n, h] += dscore.T @ Q
                got["dq"][i, :, a] = dscore @ K / math.sqrt(hd)
    return {x: t if x == "lse" else t.flatten(2).flatten(0, 1) for x, t in got.items()}


def _rope_exact(s):
    """The rotation as a product of complex numbers."""
    case = s.case
    half, n = case["head_dim"] // 2, case["n_rot"]
    entries = torch.view_as_complex(s.table.double())
    turn = torch.stack([entries[s.positions[a].long(), p] for p, a in enumerate(s.axis)], 1).unsqueeze(1)

    def turned(t, w):
        t = t[:, :s.width].double().unflatten(1, (-1, 2, half))
        z = torch.complex(t[:, :n, 0], t[:, :n, 1]) * w
        return torch.cat([torch.stack([z.real, z.imag], 2), t[:, n:]], 1).flatten(1)
    return {"y": turned(s.x, turn), "dx": turned(s.dy, turn.conj())}


def _distill_exact(s):
    """A piece of rows at a time: -sum of t log p and sum of t log t, over the entries that are given."""
    case = s.case
    vocab, T, rows = case["vocab"], case["temperature"], case["rows"]
    out = {"loss": [], "lse": [], "dz": []}
    size = max(1, 100_000_000 // vocab)
    for r in range(0, rows, size):
        part = slice(r, min(rows, r + size))
        z = s.z[part, :vocab].double() / T
        log_p = z - torch.logsumexp(z, 1, keepdim=True)
        ids, value = s.ids[part].long(), s.teacher[part].double()
        value = value.masked_fill((ids < 0) | (ids >= vocab), -math.inf)
        if not case["log_probs"]:
            value = torch.log_softmax(value / T, 1).masked_fill((value == -math.inf), -math.inf)
        t = torch.exp(value)
        at = ids.clamp(0, vocab - 1)
        dense = torch.zeros_like(z).scatter_add_(1, at, t)
        out["loss"].append(torch.special.entr(t).sum(1).neg() - torch.where(t > 0, t * log_p.gather(1, at), 0.0).sum(1))
        out["lse"].append(torch.logsumexp(z, 1))
        dz = torch.exp(log_p).mul_(t.sum(1, keepdim=True)).sub_(dense).mul_(s.dloss[part].double()[:, None] / T)
        out["dz"].append(dz)
    return {k: torch.cat(v) for k, v in out.items()}


def exact(case, seed):
    return {"cross": _cross_exact, "rope": _rope_exact, "distill": _distill_exact}[case["kind"]](prepare(case, seed))


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Inputs read once by each direction that needs them, outputs written once; operations by the formulas."""
    kind, e = case["kind"], 2 if case["dtype"] == BF16 else 4
    if kind == "cross":
        # of a ragged batch half of the states are to be expected, and a batch of more than two has one sequence without any
        share = 1.0 if not case["ragged"] else 0.5 * ((case["batch"] - 1) / case["batch"] if case["batch"] > 2 else 1.0)
        q, kv = case["batch"] * case["seq_q"] * case["n_q"] * case["head_dim"], case["batch"] * case["seq_kv"] * case["n_kv"] * case["head_dim"] * 2
        lse = 4 * case["batch"] * case["seq_q"] * case["n_q"]
        product = 2 * q * case["seq_kv"] * share
        # forward: q and states in, o and lse out, two products; backward: q, states, o, dout and lse in, dq and the states' gradients out, five
        if not case["train"]:
            return {"bytes": (2 * q + kv * share) * e + lse, "flops": 2 * product}
        return {"bytes": (2 * q + kv * share) * e + lse + (4 * q + kv * share + kv) * e + lse, "flops": 7 * product}
    if kind == "rope":
        n = case["rows"] * (case["n_rot"] + case["n_pass"]) * case["head_dim"]
        angles = case["rows"] * case["head_dim"] * 4 + case["rows"] * case["axes"] * 4
        return {"bytes": 4 * n * e + 2 * angles, "flops": 6 * case["rows"] * case["n_rot"] * case["head_dim"]}
    n, top = case["rows"] * case["vocab"], case["rows"] * case["k"] * 8
    live = 1.0 - int(case["masked"] * case["rows"]) / case["rows"]
    # logits in once (fused), or once forward and, of the rows that have a gradient, once backward; their gradient out
    reads = 1.0 if case["fused"] else 1.0 + live
    return {"bytes": (reads * n + n) * e + (1 if case["fused"] else 2) * top + 16 * case["rows"], "flops": 6 * n}
