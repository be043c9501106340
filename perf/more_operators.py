"""Timed cases of the operators of a step in 8 bits and of its output end: normalisation (with the residual sum) into 8-bit
codes with a scale per row (``dare_k_norm_q8``), the projection of such codes (``dare_k_linear_q8``), and log-probabilities,
entropy and top alternatives of logits (``dare_k_logprobs``).

A case is a dict of plain values.  ``op`` names the operator, ``dtype`` is "bf16" or "f32".

  norm      s = x + o (in the type; stored where keep), y = the norm of s ("rms", "layer", or "none": s itself), with a gain, and a
            bias where "layer"; scale = fp32(max |y| / 127) per row, codes y / scale to the nearest whole number, ties to even.
            rows of `dim` channels, pad: elements behind every row of x that do not belong to it.  The codes are returned as the values they stand for
  linear    out = act(sa sw (A W) + bias) + residual, A [m, k] and W [n, k] codes, sa a scale per row, sw one per column;
            act "none", "silu", "gelu" (erf) or "gelu_tanh"; pad: codes behind every row of A that do not belong to it
  logprobs  rows of `vocab` logits times `scale`: the log-probability of one given token per row, the entropy, and the `top` largest with
            their ids, equal ones by their ids.  spread: standard deviation of the logits; lead: one logit of a row is up to this
            much above; banned: ids whose logits are -infinity; pad: logits behind every row that do not belong to it
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def _norm(name, kind, rows, dim, residual=True, keep=True, dtype="bf16", pad=0):
    c = dict(op="norm", dtype=dtype, kind=kind, rows=rows, dim=dim, residual=residual, keep=keep, pad=pad)
    return dict(c, name=name) if name else c


def _linear(name, m, n, k, bias=False, act="none", residual=False, dtype="bf16", pad=0):
    c = dict(op="linear", dtype=dtype, m=m, n=n, k=k, bias=bias, act=act, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _logprobs(name, rows, vocab, top, scale=1.0, spread=2.0, lead=0.0, banned=0, dtype="bf16", pad=0):
    c = dict(op="logprobs", dtype=dtype, rows=rows, vocab=vocab, top=top, scale=scale, spread=spread, lead=lead,
             banned=banned, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the residual sum and norm in front of a layer, one token each of eight sequences: a call bound by its launch
        _norm("norm_step", "rms", 8, 4096),
        # the same for a batch of prompts
        _norm("norm_prompt", "rms", 16384, 4096),
        # activations of a feed-forward on their way into its second product: no norm, long rows, cut from a wider buffer
        _norm("norm_none", "none", 1000, 12288, residual=False, keep=False, pad=64),
        # the fp32 path that results are checked on
        _norm("norm_layer_f32", "layer", 333, 1544, dtype="f32"),
        # the output projection of one decoded token, added to the residual stream: a stream over the weights
        _linear("linear_token", 1, 4096, 4096, residual=True),
        # Q, K and V with their biases for a prompt of odd length, 32 query and 8 key heads
        _linear("linear_qkv_bias", 777, 6144, 4096, bias=True),
        # the first feed-forward product of a batch of long prompts
        _linear("linear_up_gelu", 16384, 12288, 4096, bias=True, act="gelu"),
        # logits of a block of 32 positions over the whole vocabulary
        _linear("linear_head", 32, 126464, 4096),
        # fp32 outputs, a narrow layer, codes cut from a wider buffer
        _linear("linear_f32", 201, 512, 1536, bias=True, act="silu", residual=True, dtype="f32", pad=64),
        # one position of one sequence: whether to unmask it, and with what
        _logprobs("logprobs_token", 1, 126464, 2, lead=12.0, banned=1),
        # all positions of a sequence that are still masked
        _logprobs("logprobs_block", 2048, 126464, 8, lead=12.0, banned=1),
        # fp32 logits of an odd vocabulary, cooled, with many alternatives
        _logprobs("logprobs_f32", 300, 32003, 20, scale=1.4, spread=3.0, banned=500, dtype="f32", pad=1),
    ]


def draw(rng):
    """One more case of the ranges above; it costs no more than the largest listed one of its operator."""
    logu = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    op = rng.choice(["norm", "linear", "linear", "logprobs"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    top = max(work(c)["flops"] for c in listed() if c["op"] == op)
    while True:
        if op == "norm":
            kind = rng.choice(["rms", "rms", "layer", "none"])
            residual = rng.random() < 0.6
            c = _norm(None, kind, logu(1, 16384), 8 * logu(8, 1536), residual, residual and rng.random() < 0.8, dtype,
                      rng.choice([0, 0, 8, 200]))
        elif op == "linear":
            head = rng.random() < 0.2
            m = logu(1, 128 if head else 2048 if dtype == "f32" else 16384)
            c = _linear(None, m, 64 * (logu(192, 1976) if head else logu(1, 192)), 128 * logu(1, 96), rng.random() < 0.5,
                        rng.choice(["none", "none", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.5, dtype,
                        rng.choice([0, 0, 64, 208]))
        else:
            vocab = logu(100, 130000)
            c = _logprobs(None, logu(1, 4096), vocab, rng.choice([0, 1, 2, 5, 8, 20, 32]), rng.choice([1.0, 1.0, 0.7, 1.5]),
                          rng.choice([1.0, 2.0, 4.0]), rng.choice([0.0, 5.0, 15.0]), rng.choice([0, 1, vocab // 8]), dtype,
                          rng.choice([0, 0, 1, 8]))
        if work(c)["flops"] <= top:
            return c


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["op"] == "norm":
        n = c["rows"] * c["dim"]
        vectors = {"none": 0, "rms": 1, "layer": 2}[c["kind"]]
        return {"bytes": n * (e * (1 + c["residual"] + c["keep"]) + 1) + 4 * c["rows"] + e * vectors * c["dim"], "flops": 8 * n}
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": m * k + n * k + 4 * (m + n) + e * (m * n * (1 + c["residual"]) + (n if c["bias"] else 0)),
                "flops": 2 * m * n * k}
    return {"bytes": c["rows"] * (e * c["vocab"] + 4 + 4 + 4 + 8 * c["top"]), "flops": 6 * c["rows"] * c["vocab"]}


# ---- inputs ------------------------------------------------------------------------------

def _codes(x):
    """Codes and scales of rows."""
    scale = x.abs().amax(1) / 127.0
    return torch.round(x / scale[:, None]).to(torch.int8), scale


def _inputs(c, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    td = DTYPES[c["dtype"]]
    rn = lambda *shape, dtype=td: torch.randn(shape, device=dev, dtype=dtype, generator=gen)
    if c["op"] == "norm":
        rows, d = c["rows"], c["dim"]
        x = rn(rows, d + c["pad"])
        x[:, :d // 64 + 1] *= 8   # (a few channels are far larger than the others)
        return {"x": x[:, :d], "o": rn(rows, d) if c["residual"] else None,
                "gain": None if c["kind"] == "none" else rn(d).mul_(0.1).add_(1.0), "bias": rn(d).mul_(0.1) if c["kind"] == "layer" else None}
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        a, sa = _codes(rn(m, k + c["pad"], dtype=torch.float32))
        w, sw = _codes(rn(n, k, dtype=torch.float32).mul_(k ** -0.5))
        return {"a": a[:, :k], "sa": sa, "w": w, "sw": sw, "bias": rn(n).mul_(0.5) if c["bias"] else None,
                "residual": rn(m, n) if c["residual"] else None}
    rows, vocab = c["rows"], c["vocab"]
    z = rn(rows, vocab + c["pad"]).mul_(c["spread"])
    ids = lambda n: torch.randint(0, vocab, (n,), device=dev, generator=gen)
    lead = ids(rows)
    z[torch.arange(rows, device=dev), lead] += (torch.rand(rows, device=dev, generator=gen) * c["lead"]).to(td)
    if c["banned"]:
        z[:, ids(c["banned"])] = float("-inf")
    tokens = torch.where(torch.rand(rows, device=dev, generator=gen) < 0.5, lead, ids(rows))
    return {"z": z[:, :vocab], "tokens": tokens.to(torch.int32)}


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    empty = lambda like, dtype, *shape: torch.empty(shape, dtype=dtype, device=like.device)
    if case["op"] == "norm":
        x = st["x"]
        st["codes"], st["scales"] = empty(x, torch.int8, *x.shape), empty(x, torch.float32, x.shape[0])
        st["sum"] = empty(x, x.dtype, *x.shape) if case["keep"] else None
        st["values"] = empty(x, x.dtype, *x.shape)
    elif case["op"] == "linear":
        st["out"] = empty(st["a"], DTYPES[case["dtype"]], case["m"], case["n"])
    else:
        z, rows, top = st["z"], case["rows"], case["top"]
        st["logprobs"], st["entropy"] = empty(z, torch.float32, rows), empty(z, torch.float32, rows)
        st["ids"], st["tops"] = empty(z, torch.int32, rows, top), empty(z, torch.float32, rows, top)
    return st


# ---- one pass ------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _run_own(c, state)
    return {"norm": _plain_norm, "linear": _plain_linear, "logprobs": _plain_logprobs}[c["op"]](c, state)


def _run_own(c, st):
    from paper_2605_08134_amd import binding as B
    if c["op"] == "norm":
        B.dare_k_norm_q8(None if c["kind"] == "none" else c["kind"], st["x"], st["codes"], st["scales"], o=st["o"], x_out=st["sum"],
                         gain=st["gain"], bias=st["bias"], eps=EPS)
        return _values(st)
    if c["op"] == "linear":
        B.dare_k_linear_q8(st["a"], st["sa"], st["w"], st["sw"], st["out"], bias=st["bias"],
                           act=None if c["act"] == "none" else c["act"], residual=st["residual"])
        return st["out"]
    B.dare_k_logprobs(st["z"], st["tokens"], st["logprobs"], st["entropy"], st["ids"], st["tops"], scale=c["scale"])
    return st["logprobs"], st["entropy"], st["ids"], st["tops"]


def _values(st):
    """What the codes stand for, with the scales and the sum."""
    torch.mul(st["codes"], st["scales"][:, None], out=st["values"])
    return [st["values"], st["scales"]] + ([] if st["sum"] is None else [st["sum"]])


def _plain_norm(c, st):
    # (in 64 bits: in 32 a value next to the middle between two codes goes to the wrong one)
    s = st["x"]
    if c["residual"]:
        s = (s.float() + st["o"].float()).to(s.dtype)
    if c["keep"]:
        st["sum"].copy_(s)
    y = s.double()
    if c["kind"] == "layer":
        y = y - y.mean(1, keepdim=True)
    if c["kind"] != "none":
        y = y / torch.sqrt((y * y).mean(1, keepdim=True) + EPS) * st["gain"].double()
    if c["kind"] == "layer":
        y = y + st["bias"].double()
    st["scales"].copy_(y.abs().amax(1) / 127.0)
    st["codes"].copy_(torch.round(y / st["scales"].double()[:, None]))
    return _values(st)


def _plain_linear(c, st):
    y = st["a"].float() @ st["w"].float().t()
    y = y * st["sa"][:, None] * st["sw"]
    if st["bias"] is not None:
        y += st["bias"].float()
    if c["act"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    elif c["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif c["act"] == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if st["residual"] is not None:
        y += st["residual"].float()
    st["out"].copy_(y)
    return st["out"]


def _plain_logprobs(c, st):
    z = st["z"].float() * c["scale"]
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1)
    lse = torch.log(total)
    st["logprobs"].copy_(z.gather(1, st["tokens"].long()[:, None])[:, 0] - lse)
    # (a place of probability 0 adds nothing: its -infinity is not multiplied)
    st["entropy"].copy_(lse - (e * torch.where(e > 0, z, 0.0)).sum(1) / total)
    if c["top"]:
        value, at = torch.sort(st["z"].float() + 0.0, dim=1, descending=True, stable=True)
        st["ids"].copy_(at[:, :c["top"]])
        st["tops"].copy_(z.gather(1, at[:, :c["top"]]) - lse[:, None])
    return st["logprobs"], st["entropy"], st["ids"], st["tops"]


# ---- the same in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["op"] == "norm":
        s = x["x"].double()
        if c["residual"]:
            s = s + x["o"].double()
        kept = s
        if c["residual"]:   # the sum is a stored tensor
            s = s.to(DTYPES[c["dtype"]]).double()
        if c["kind"] == "rms":
            y = x["gain"].double() * s * torch.rsqrt(torch.linalg.vecdot(s, s)[:, None] / c["dim"] + EPS)
        elif c["kind"] == "layer":
            var, mean = torch.var_mean(s, dim=1, correction=0, keepdim=True)
            y = torch.addcmul(x["bias"].double(), (s - mean) * torch.rsqrt(var + EPS), x["gain"].double())
        else:
            y = s
        scale = torch.linalg.vector_norm(y, torch.inf, dim=1) / 127.0
        step = scale.float().double()[:, None]
        values = torch.round(y / step) * step
        return [values, scale] + ([kept] if c["keep"] else [])
    if c["op"] == "linear":
        z = torch.matmul(x["a"].double(), x["w"].double().mT.contiguous())
        z = x["sa"].double()[:, None] * z * x["sw"].double()
        if x["bias"] is not None:
            z = z + x["bias"].double()
        if c["act"] == "silu":
            z = z * torch.special.expit(z)
        elif c["act"] == "gelu":
            z = z * torch.special.erfc(-z / 2.0 ** 0.5) / 2.0
        elif c["act"] == "gelu_tanh":
            z = z * torch.special.expit(2.0 * (2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
        return z if x["residual"] is None else z + x["residual"].double()
    z = x["z"].double() * c["scale"]
    lp = z - torch.logsumexp(z, 1, keepdim=True)
    entropy = torch.special.entr(torch.exp(lp)).sum(1)
    tops = torch.topk(lp, c["top"], dim=1).values
    return lp[torch.arange(c["rows"], device=lp.device), x["tokens"].long()], entropy, None, tops
