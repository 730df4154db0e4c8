"""Timed cases of the operators around a layer's products: activations kept in 8 bits and used from there in the backward
pass, norms of queries and keys with the position rotation, and the embedding with its gradient.

A pass is what a training step does with an operator: forward with what it keeps, and backward from what was kept.  "kind":
  keep    a tensor kept in 8 bits (blocks of 32 values of a row share a power of two) and restored
  mlp     the MLP activation that keeps its input in 8 bits; its gradient, and its value again for the weight gradient, from there
  norm    RMSNorm / LayerNorm that keeps its input in 8 bits; its gradients, and its value again, from there
  qknorm  RMSNorm of every query and key head with the rotation; with "keep" the projection's output is kept in 8 bits, the
          attention's operands are rebuilt from there, and the gradients read it; without, the gradients read the projection's output
  embed   the scaled embedding of tokens and its gradient, added to the table's fp32 accumulator
Gradients of gains, biases and of the table are added to accumulators, which a pass leaves in the state.
"""
import math
from types import SimpleNamespace

import torch

own = False

GPT, LLAMA = 0, 1
FP32, BF16 = 0, 1
EPS, ROPE_BASE = 1e-5, 10000.0
TORCH = {FP32: torch.float32, BF16: torch.bfloat16}


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the smallest stage's input (fp32, hidden 256): latency of two launches
        {"name": "keep_tiny_fp32", "kind": "keep", "dtype": FP32, "rows": 128, "cols": 256, "ld": 256},
        # the QKV rows of the long-sequence stage (40 heads of 128, 16384 tokens): the largest tensor that a layer keeps
        {"name": "keep_qkv_16k", "kind": "keep", "dtype": BF16, "rows": 16384, "cols": 15360, "ld": 15360},
        # the tiny fp32 stage's MLP activation (GELU)
        {"name": "mlp_tiny_fp32", "kind": "mlp", "family": GPT, "dtype": FP32, "rows": 128, "ffn": 1024},
        # the Llama-style layer's SwiGLU, the ordinary training size
        {"name": "mlp_swiglu", "kind": "mlp", "family": LLAMA, "dtype": BF16, "rows": 4096, "ffn": 11008},
        # the GPT-style layer's GELU on a ragged number of tokens and a width whose last block of 32 is cut
        {"name": "mlp_gelu_ragged", "kind": "mlp", "family": GPT, "dtype": BF16, "rows": 4999, "ffn": 4088},
        # the grouped-query stage's RMSNorm with its residual: the widest rows
        {"name": "norm_rms_8192", "kind": "norm", "family": LLAMA, "dtype": BF16, "rows": 4096, "hidden": 8192},
        # LayerNorm of a ragged batch at an odd width
        {"name": "norm_layer_ragged", "kind": "norm", "family": GPT, "dtype": BF16, "rows": 1237, "hidden": 2040},
        # queries and keys of the grouped-query stage, kept in 8 bits: forward, rebuilt for the attention's gradient, backward
        {"name": "qknorm_gqa_keep", "kind": "qknorm", "dtype": BF16, "rows": 8192, "seq": 4096, "n_q": 64, "n_kv": 8, "head_dim": 128, "keep": True},
        # a few heads of 64 in fp32, nothing kept: a small model or a debugging session
        {"name": "qknorm_tiny_fp32", "kind": "qknorm", "dtype": FP32, "rows": 128, "seq": 128, "n_q": 4, "n_kv": 4, "head_dim": 64, "keep": False},
        # a micro-batch of the tiny stage: 128 tokens
        {"name": "embed_tiny_fp32", "kind": "embed", "dtype": FP32, "rows": 128, "vocab": 1000, "hidden": 256, "scaled": False, "pad": 0.0},
        # a micro-batch of the Llama-style model: 4096 tokens of a 32000-word vocabulary, frequent words often
        {"name": "embed_4k", "kind": "embed", "dtype": BF16, "rows": 4096, "vocab": 32000, "hidden": 4096, "scaled": True, "pad": 0.0},
        # the long-sequence micro-batch over a large vocabulary, the last three tenths padding (no token there)
        {"name": "embed_16k_padded", "kind": "embed", "dtype": BF16, "rows": 16384, "vocab": 131072, "hidden": 5120, "scaled": True, "pad": 0.3},
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step) * step))


def draw(rng):
    kind = rng.choice(["keep", "mlp", "norm", "qknorm", "embed"])
    dtype = BF16 if rng.random() < 0.75 else FP32
    family, step = rng.choice([GPT, LLAMA]), 8 if dtype == BF16 else 4
    most = 1 if dtype == BF16 else 2
    if kind == "keep":
        cols = _log_int(rng, 1, 16384)
        if rng.random() < 0.5:
            cols = -(-cols // 8) * 8
        rows = _log_int(rng, 1, max(1, min(65536, 250_000_000 // cols // most)))
        return {"kind": kind, "dtype": dtype, "rows": rows, "cols": cols, "ld": cols + rng.choice([0, 0, 0, 8, 128, 1])}
    if kind == "mlp":
        ffn = _log_int(rng, 64, 28672, step)
        return {"kind": kind, "family": family, "dtype": dtype, "rows": _log_int(rng, 1, max(1, min(16384, 100_000_000 // ffn // most))), "ffn": ffn}
    if kind == "norm":
        hidden = _log_int(rng, 64, 8192, step)
        return {"kind": kind, "family": family, "dtype": dtype, "rows": _log_int(rng, 1, 16384), "hidden": hidden}
    if kind == "qknorm":
        n_kv, d = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 128, 256])
        n_q, seq = n_kv * rng.choice([1, 2, 3, 4, 8]), _log_int(rng, 1, 8192)
        rows = seq * rng.choice([1, 1, 2, 3])
        while rows * (n_q + 2 * n_kv) * d * most > 120_000_000:
            seq, rows = max(1, seq // 2), max(1, seq // 2)
        return {"kind": kind, "dtype": dtype, "rows": rows, "seq": seq, "n_q": n_q, "n_kv": n_kv, "head_dim": d, "keep": rng.random() < 0.6}
    hidden = _log_int(rng, 64, 8192, step)
    vocab = _log_int(rng, 100, min(262144, 1_000_000_000 // hidden // 2))
    return {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, min(65536, 160_000_000 // hidden // most)), "vocab": vocab, "hidden": hidden,
            "scaled": rng.random() < 0.5, "pad": rng.choice([0.0, 0.0, 0.1, 0.5])}


# ---------------------------------------------------------------------------------------------- inputs
class _Draw:
    """Seeded normal tensors on the device."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(0x0DD5 + 7919 * int(seed))

    def __call__(self, shape, dtype, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32) * std + mean).to(TORCH[dtype])

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def activations(self, rows, cols, dtype):
        """Normal values whose columns differ in size by a few octaves, as the columns of a trained layer's activations do."""
        x = torch.randn((rows, cols), generator=self.g, device="cuda", dtype=torch.float32)
        x *= torch.exp2(1.5 * torch.randn((cols,), generator=self.g, device="cuda", dtype=torch.float32))
        return x.to(TORCH[dtype])


def _width(case):
    return 2 * case["ffn"] if case["family"] == LLAMA else case["ffn"]


def _blocks(cols):
    return (cols + 31) // 32


def _kept(s, rows, cols):
    s.codes = torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
    s.scales = torch.empty((rows, _blocks(cols)), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    d, kind, dt = _Draw(seed), case["kind"], case["dtype"]
    s = SimpleNamespace(case=case)
    rows = case["rows"]
    empty = lambda *shape, dtype=TORCH[dt]: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "keep":
        s.x = d.activations(rows, case["ld"], dt)
        s.y = empty(rows, case["cols"])
        _kept(s, rows, case["cols"])
    elif kind == "mlp":
        f = case["ffn"]
        s.gu, s.da = d((rows, _width(case)), dt, 1.5), d((rows, f), dt, 1e-3)
        s.a, s.a_again, s.dgu = empty(rows, f), empty(rows, f), empty(rows, _width(case))
        _kept(s, rows * (_width(case) // f), f)
    elif kind == "norm":
        h, two = case["hidden"], case["family"] == GPT
        s.x, s.dn, s.dres = d.activations(rows, h, dt), d((rows, h), dt, 1e-3), d((rows, h), dt, 1e-3)
        s.gamma = d((h,), dt, 0.02, 1.0)
        s.beta = d((h,), dt, 0.02) if two else None
        s.dgamma = d((h,), FP32, 1e-3)
        s.dbeta = d((h,), FP32, 1e-3) if two else None
        s.out, s.out_again, s.dx = empty(rows, h), empty(rows, h), empty(rows, h)
        s.stats = empty(rows, 2 if two else 1, dtype=torch.float32)
        s.partial = empty(2 * min(rows, 512) * h, dtype=torch.float32)
        _kept(s, rows, h)
    elif kind == "qknorm":
        hd, n_rot = case["head_dim"], case["n_q"] + case["n_kv"]
        w = (n_rot + case["n_kv"]) * hd
        s.x, s.dy = d.activations(rows, w, dt), d((rows, w), dt, 1e-3)
        s.gq, s.gk = d((hd,), dt, 0.1, 1.0), d((hd,), dt, 0.1, 1.0)
        s.dgq, s.dgk = d((hd,), FP32, 1e-3), d((hd,), FP32, 1e-3)
        angle = torch.arange(case["seq"], dtype=torch.float64, device="cuda")[:, None] * torch.pow(
            torch.tensor(ROPE_BASE, dtype=torch.float64, device="cuda"), -torch.arange(hd // 2, dtype=torch.float64, device="cuda") * 2 / hd)
        s.table = torch.stack([torch.cos(angle), torch.sin(angle)], -1).float().contiguous()
        s.y, s.y_again, s.dx = empty(rows, w), empty(rows, w), empty(rows, w)
        s.stats = empty(rows, n_rot, dtype=torch.float32)
        s.partial = empty(2 * min(rows, 1024) * hd, dtype=torch.float32)
        if case["keep"]:
            _kept(s, rows, w)
    else:
        vocab, h = case["vocab"], case["hidden"]
        s.weight, s.grad, s.dy = d((vocab, h), dt, 0.02), d((vocab, h), FP32, 1e-3), d((rows, h), dt, 1e-3)
        # the k-th most frequent word about 1 / k as often as the first; the words in the vocabulary in no order of frequency
        rank = (torch.exp(d.uniform((rows,)) * math.log(vocab + 1.0)) - 1.0).long().clamp(0, vocab - 1)
        order = torch.argsort(d.uniform((vocab,)))
        s.ids = order[rank].to(torch.int32)
        s.ids[rows - int(case["pad"] * rows):] = -1
        s.scale = math.sqrt(h) if case["scaled"] else 1.0
        s.out = empty(rows, h)
        s.ws = empty(_embed_ws_bytes(rows, h), dtype=torch.uint8)
    s.at = {k: v.data_ptr() for k, v in vars(s).items() if isinstance(v, torch.Tensor)}     # the buffers stay where they are
    return s


def _embed_ws_bytes(rows, hidden):
    """At least optstage_op_embed_bwd_ws_bytes(rows, hidden): the sorted tokens, the sort's counts, and two partial rows for every 32 tokens."""
    return 64 * rows + (1 << 20) + 2 * ((rows + 31) // 32) * hidden * 4


# ---------------------------------------------------------------------------------------------- the plain form
def _stands_for(x):
    """What x kept in 8 bits stands for, in 32 bits: blocks of 32 along the rows, e4m3 values times the least power of two 2^k with
    max |x| <= 448 * 2^k (k from -117 to 119); what is not finite becomes NaN and does not count for the maximum."""
    f = x.float()
    rows, cols = f.shape
    f = torch.cat([f, f.new_zeros((rows, _blocks(cols) * 32 - cols))], 1).view(rows, -1, 32)
    finite = torch.isfinite(f)
    most = torch.where(finite, f.abs(), torch.zeros_like(f)).amax(-1, keepdim=True).view(torch.int32)
    k = ((most >> 23) - 135 + ((most & 0x7FFFFF) > 0x600000).int()).clamp(-117, 119)
    power = lambda e: ((e + 127) << 23).view(torch.float32)  # noqa: E731
    v = (f * power(-k)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() * power(k)
    return torch.where(finite, v, torch.full_like(v, float("nan"))).view(rows, -1)[:, :cols]


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _activation(family, gu):
    if family == LLAMA:
        g, u = gu.chunk(2, 1)
        return g * _sigmoid(g) * u
    return gu * (0.5 * (1.0 + torch.erf(gu * math.sqrt(0.5))))


def _activation_gradient(family, gu, da):
    if family == LLAMA:
        g, u = gu.chunk(2, 1)
        sg = _sigmoid(g)
        return torch.cat([da * u * sg * (1.0 + g * (1.0 - sg)), da * g * sg], 1)
    return da * (0.5 * (1.0 + torch.erf(gu * math.sqrt(0.5))) + gu * torch.exp(-0.5 * gu * gu) / math.sqrt(2.0 * math.pi))


def _heads(case, t):
    return t.view(case["rows"], -1, case["head_dim"])


def _rotate(case, t, table, sign):
    """Element k of a head with element k + head_dim / 2, by the angles of position = row % seq."""
    pos = torch.arange(case["rows"], device=t.device) % case["seq"]
    c, s = table[pos][:, None, :, 0], sign * table[pos][:, None, :, 1]
    lo, hi = t.chunk(2, 2)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], 2)


def _qknorm_plain(case, s, x, r, dtype):
    """The rotated, normed heads beside the values as they are, from x in 32 bits and 1 / rms of every head."""
    nq, n_rot = case["n_q"], case["n_q"] + case["n_kv"]
    n = x[:, :n_rot] * r[:, :, None]
    n = torch.cat([n[:, :nq] * s.gq.float(), n[:, nq:] * s.gk.float()], 1)
    return torch.cat([_rotate(case, n, s.table, 1.0), x[:, n_rot:]], 1).to(dtype).view(case["rows"], -1)


def _plain(s):
    case = s.case
    kind, dtype = case["kind"], TORCH[case["dtype"]]
    if kind == "keep":
        return {"x": _stands_for(s.x[:, :case["cols"]]).to(dtype)}
    if kind == "mlp":
        f = case["ffn"]
        kept = _stands_for(s.gu.view(-1, f)).reshape(case["rows"], -1)
        return {"a": _activation(case["family"], s.gu.float()).to(dtype), "dgu": _activation_gradient(case["family"], kept, s.da.float()).to(dtype),
                "a_again": _activation(case["family"], kept).to(dtype)}
    if kind == "norm":
        x, kept, two = s.x.float(), _stands_for(s.x), case["family"] == GPT
        mean = x.mean(1, keepdim=True) if two else torch.zeros_like(x[:, :1])
        r = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        gamma, beta = s.gamma.float(), s.beta.float() if two else 0.0
        xh, dn = (kept - mean) * r, s.dn.float()
        g = dn * gamma
        dx = r * (g - (g.mean(1, keepdim=True) if two else 0.0) - xh * (g * xh).mean(1, keepdim=True)) + s.dres.float()
        s.dgamma += (dn * xh).sum(0, dtype=torch.float64).float()
        got = {"out": ((x - mean) * r * gamma + beta).to(dtype), "stats": torch.cat([mean, r], 1) if two else r, "dx": dx.to(dtype),
               "out_again": (xh * gamma + beta).to(dtype), "dgamma": s.dgamma}
        if two:
            s.dbeta += dn.sum(0, dtype=torch.float64).float()
            got["dbeta"] = s.dbeta
        return got
    if kind == "qknorm":
        nq, n_rot = case["n_q"], case["n_q"] + case["n_kv"]
        x = _heads(case, s.x.float())
        r = 1.0 / torch.sqrt(x[:, :n_rot].square().mean(2) + EPS)
        got = {"y": _qknorm_plain(case, s, x, r, dtype), "stats": r}
        if case["keep"]:
            x = _heads(case, _stands_for(s.x))
            got["y_again"] = _qknorm_plain(case, s, x, r, dtype)
        dy = _heads(case, s.dy.float())
        dn, xh = _rotate(case, dy[:, :n_rot], s.table, -1.0), x[:, :n_rot] * r[:, :, None]
        s.dgq += (dn[:, :nq] * xh[:, :nq]).sum((0, 1), dtype=torch.float64).float()
        s.dgk += (dn[:, nq:] * xh[:, nq:]).sum((0, 1), dtype=torch.float64).float()
        g = torch.cat([dn[:, :nq] * s.gq.float(), dn[:, nq:] * s.gk.float()], 1)
        dx = r[:, :, None] * (g - xh * (g * xh).mean(2, keepdim=True))
        return dict(got, dx=torch.cat([dx, dy[:, n_rot:]], 1).to(dtype).view(case["rows"], -1), dgamma_q=s.dgq, dgamma_k=s.dgk)
    ids, vocab = s.ids.long(), case["vocab"]
    valid = (ids >= 0) & (ids < vocab)
    at = torch.where(valid, ids, torch.zeros_like(ids))
    out = torch.where(valid[:, None], s.weight[at].float() * s.scale, torch.zeros((), device="cuda")).to(dtype)
    # equal tokens side by side, their rows added in 64 bits, then one addition to the accumulator
    key, order = torch.sort(torch.where(valid, ids, torch.full_like(ids, vocab)), stable=True)
    first = torch.ones_like(key)
    first[1:] = (key[1:] != key[:-1]) | (key[1:] == vocab)
    run_of = torch.cumsum(first, 0) - 1
    sums = torch.zeros((case["rows"], case["hidden"]), dtype=torch.float64, device="cuda").index_add_(0, run_of, s.dy[order].double())
    token = torch.full_like(key, vocab).scatter_(0, run_of, key)
    anywhere = torch.arange(case["rows"], device="cuda") % vocab         # where there is no token, zeros are added
    s.grad.index_add_(0, torch.where(token < vocab, token, anywhere), torch.where((token < vocab)[:, None], sums * s.scale, 0.0).float())
    return {"out": out, "grad": s.grad}


# ---------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2510_05186_amd import binding as B
    lib, case, at = B.lib(), s.case, s.at
    kind, dt, rows, stream = case["kind"], case["dtype"], case["rows"], torch.cuda.current_stream().cuda_stream
    if kind == "keep":
        B.check(lib.optstage_op_pack8(dt, at["x"], case["ld"], at["codes"], at["scales"], rows, case["cols"], stream))
        B.check(lib.optstage_op_unpack8(dt, at["codes"], at["scales"], at["y"], case["cols"], rows, case["cols"], stream))
        return {"x": s.y}
    if kind == "mlp":
        B.check(lib.optstage_op_act_fwd_pack8(dt, case["family"], at["gu"], at["a"], at["codes"], at["scales"], rows, case["ffn"], stream))
        B.check(lib.optstage_op_act_bwd8(dt, case["family"], at["da"], at["codes"], at["scales"], at["dgu"], at["a_again"], rows, case["ffn"], stream))
        return {"a": s.a, "dgu": s.dgu, "a_again": s.a_again}
    if kind == "norm":
        beta, dbeta = at.get("beta", 0), at.get("dbeta", 0)
        B.check(lib.optstage_op_norm_fwd_pack8(dt, case["family"], at["x"], at["gamma"], beta, at["out"], at["stats"], at["codes"], at["scales"], rows,
                                               case["hidden"], EPS, stream))
        B.check(lib.optstage_op_norm_bwd8(dt, case["family"], at["dn"], at["codes"], at["scales"], at["stats"], at["gamma"], beta, at["dres"], at["dx"],
                                          at["out_again"], at["partial"], at["dgamma"], dbeta, rows, case["hidden"], stream))
        got = {"out": s.out, "stats": s.stats, "dx": s.dx, "out_again": s.out_again, "dgamma": s.dgamma}
        if s.dbeta is not None:
            got["dbeta"] = s.dbeta
        return got
    if kind == "qknorm":
        shape = (rows, case["seq"], case["n_q"], case["n_kv"], case["head_dim"])
        codes, scales = at.get("codes", 0), at.get("scales", 0)
        B.check(lib.optstage_op_qknorm_rope(dt, at["x"], at["y"], at["gq"], at["gk"], at["table"], at["stats"], codes, scales, *shape, EPS, stream))
        got = {"y": s.y, "stats": s.stats}
        if case["keep"]:
            B.check(lib.optstage_op_qknorm_rope8(dt, codes, scales, at["stats"], at["gq"], at["gk"], at["table"], at["y_again"], *shape, stream))
            got["y_again"] = s.y_again
        B.check(lib.optstage_op_qknorm_rope_bwd(dt, at["dy"], 0 if case["keep"] else at["x"], codes, scales, at["stats"], at["gq"], at["gk"], at["table"], at["dx"],
                                                at["partial"], at["dgq"], at["dgk"], *shape, stream))
        return dict(got, dx=s.dx, dgamma_q=s.dgq, dgamma_k=s.dgk)
    B.check(lib.optstage_op_embed_fwd(dt, at["ids"], at["weight"], at["out"], rows, case["vocab"], case["hidden"], s.scale, stream))
    B.check(lib.optstage_op_embed_bwd(dt, at["ids"], at["dy"], at["grad"], at["ws"], s.ws.numel(), rows, case["vocab"], case["hidden"], s.scale, stream))
    return {"out": s.out, "grad": s.grad}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits
def _two64(k):
    return ((k.long() + 1023) << 52).view(torch.float64)


def _stands_for64(x):
    """The same rounding from its definition: v = 2^k y with y a whole multiple of 2^(max(exponent of y, -6) - 3), ties to even."""
    x = x.double()
    rows, cols = x.shape
    y = x.new_zeros((rows, _blocks(cols) * 32))
    y[:, :cols] = x
    y = y.reshape(-1, 32)
    bad = ~torch.isfinite(y)
    most = y.masked_fill(bad, 0.0).abs().max(1, keepdim=True).values
    m, e = torch.frexp(most)                                            # most = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    k = torch.where(most > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -117)).clamp(-117, 119)
    y = (y.masked_fill(bad, 0.0) * _two64(-k)).clamp(-448.0, 448.0)
    step = _two64((torch.frexp(y).exponent - 1).clamp(min=-6) - 3)
    v = (torch.round(y / step) * step * _two64(k)).masked_fill(bad, float("nan"))
    return v.reshape(rows, -1)[:, :cols]


def _turn64(case, t, table, back=False):
    """The rotation as a product of complex numbers."""
    z = torch.complex(*t.split(case["head_dim"] // 2, 2))
    w = torch.view_as_complex(table.double())[torch.arange(case["rows"], device="cuda") % case["seq"]].unsqueeze(1)
    z = z * (w.conj() if back else w)
    return torch.cat([z.real, z.imag], 2)


def exact(case, seed):
    s = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind == "keep":
        return {"x": _stands_for64(s.x[:, :case["cols"]])}
    if kind == "mlp":
        f, da = case["ffn"], s.da.double()
        given, kept = s.gu.double(), _stands_for64(s.gu.reshape(-1, f)).reshape(rows, -1)
        if case["family"] == GPT:
            cdf = lambda v: 0.5 * torch.erfc(v * -math.sqrt(0.5))  # noqa: E731
            return {"a": given * cdf(given), "dgu": da * (cdf(kept) + kept * torch.exp(kept * kept * -0.5) * (1 / math.sqrt(2 * math.pi))), "a_again": kept * cdf(kept)}
        silu = lambda v: v / (1 + torch.exp(-v))  # noqa: E731
        g, u = kept[:, :f], kept[:, f:]
        low = 1 / (1 + torch.exp(g))                                    # 1 - sigmoid
        slope = (1 - low) + g * low * (1 - low)
        return {"a": silu(given[:, :f]) * given[:, f:], "dgu": torch.cat([da * u * slope, da * silu(g)], 1), "a_again": silu(g) * u}
    if kind == "norm":
        x, kept, dn, gamma = s.x.double(), _stands_for64(s.x), s.dn.double(), s.gamma.double()
        h, two = case["hidden"], case["family"] == GPT
        mean = x.sum(1, keepdim=True) / h if two else 0.0
        r = torch.rsqrt((x - mean).pow(2).sum(1, keepdim=True) / h + EPS)
        again = (kept - mean) * r
        dxh = gamma * dn
        dx = dxh - again * ((dxh * again).sum(1, keepdim=True) / h)
        if two:
            dx = dx - dxh.sum(1, keepdim=True) / h
        beta = s.beta.double() if two else 0.0
        got = {"out": (x - mean) * r * gamma + beta, "stats": torch.cat([mean, r], 1) if two else r, "dx": s.dres.double() + r * dx, "out_again": again * gamma + beta,
               "dgamma": s.dgamma.double() + (again * dn).sum(0)}
        return dict(got, dbeta=s.dbeta.double() + dn.sum(0)) if two else got
    if kind == "qknorm":
        nq, n_rot, hd = case["n_q"], case["n_q"] + case["n_kv"], case["head_dim"]
        x = s.x.double().reshape(rows, -1, hd)
        gain = torch.cat([s.gq.double().expand(nq, hd), s.gk.double().expand(case["n_kv"], hd)])
        r = torch.rsqrt(torch.linalg.vecdot(x[:, :n_rot], x[:, :n_rot]) / hd + EPS)
        value = lambda t: torch.cat([_turn64(case, t[:, :n_rot] * r.unsqueeze(2) * gain, s.table), t[:, n_rot:]], 1).reshape(rows, -1)  # noqa: E731
        got = {"y": value(x), "stats": r}
        if case["keep"]:
            x = _stands_for64(s.x).reshape(rows, -1, hd)
            got["y_again"] = value(x)
        dy = s.dy.double().reshape(rows, -1, hd)
        dn, xh = _turn64(case, dy[:, :n_rot], s.table, back=True), x[:, :n_rot] * r.unsqueeze(2)
        dgain = (dn * xh).sum(0)
        g = dn * gain
        dx = (g - xh * (torch.linalg.vecdot(g, xh) / hd).unsqueeze(2)) * r.unsqueeze(2)
        return dict(got, dx=torch.cat([dx, dy[:, n_rot:]], 1).reshape(rows, -1), dgamma_q=s.dgq.double() + dgain[:nq].sum(0), dgamma_k=s.dgk.double() + dgain[nq:].sum(0))
    out = torch.zeros((rows, case["hidden"]), dtype=torch.float64, device="cuda")
    here = torch.nonzero((s.ids >= 0) & (s.ids < case["vocab"])).squeeze(1)
    token = s.ids[here].long()
    out[here] = s.weight[token].double() * s.scale
    grad = s.grad.double()
    grad.index_put_((token,), s.dy[here].double() * s.scale, accumulate=True)
    return {"out": out, "grad": grad}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Inputs read once by each direction that needs them, outputs and what is kept written once; operations by the formulas."""
    kind, rows, e = case["kind"], case["rows"], 2 if case["dtype"] == BF16 else 4
    kept = lambda r, c: r * (c + _blocks(c))  # noqa: E731
    if kind == "keep":
        n = rows * case["cols"]
        return {"bytes": 2 * n * e + 2 * kept(rows, case["cols"]), "flops": 4 * n}
    if kind == "mlp":
        n, w = rows * case["ffn"], _width(case)
        # gu in, a out, kept out; da and kept in, dgu and a out
        return {"bytes": (rows * w + n) * e + 2 * kept(rows * w // case["ffn"], case["ffn"]) + (2 * n + rows * w) * e, "flops": 30 * n}
    if kind == "norm":
        n, h, two = rows * case["hidden"], case["hidden"], 2 if case["family"] == GPT else 1
        # x in, out, kept and statistics out; dn, residual, kept and statistics in, dx and out again out; gains, and their gradients in and out
        return {"bytes": 6 * n * e + 2 * kept(rows, h) + 2 * rows * two * 4 + two * h * (2 * e + 8), "flops": 25 * n}
    if kind == "qknorm":
        w = (case["n_q"] + 2 * case["n_kv"]) * case["head_dim"]
        n, stats, table = rows * w, rows * (case["n_q"] + case["n_kv"]) * 4, min(rows, case["seq"]) * case["head_dim"] * 4
        passes = 3 if case["keep"] else 2
        forward = 2 * n * e + stats + table
        again = kept(rows, w) + n * e + stats + table if case["keep"] else 0
        backward = 2 * n * e + (kept(rows, w) if case["keep"] else n * e) + stats + table
        return {"bytes": forward + (kept(rows, w) if case["keep"] else 0) + again + backward + passes * 2 * case["head_dim"] * e + 16 * case["head_dim"], "flops": 30 * n}
    h = case["hidden"]
    tokens = rows - int(case["pad"] * rows)
    # different tokens to be expected of ranks drawn as vocab^u: rank k has the share log((k + 1) / k) / log(vocab + 1)
    different, k, total = 0.0, 1.0, math.log(case["vocab"] + 1.0)
    while k <= case["vocab"]:
        many = max(1.0, math.floor(k / 64))
        many = min(many, case["vocab"] + 1 - k)
        p = math.log((k + many) / k) / total / many
        different += many * -math.expm1(tokens * math.log1p(-min(p, 1 - 1e-12)))
        k += many
    # forward: the tokens, each different row of the table once, the output; backward: dy once, each different accumulator row in and out
    return {"bytes": 8 * rows + different * h * e + rows * h * e + tokens * h * e + different * h * 8, "flops": 3 * tokens * h}
