"""Timed cases of the operators of a decoder layer with shared key heads: the projection with bias, activation and
residual sum (``dare_k_linear``), the rotary embedding by positions with its cache writes (``dare_k_rope``) and
attention over packed sequences and caches, causal or in blocks (``dare_k_attention_packed``).

A case is a dict of plain values.  ``op`` names the operator, ``dtype`` is "bf16" or "f32".

  linear  out = act(a W + bias) + residual.  m rows, n columns, sum over k; bias, residual: truth values; act: "none",
          "silu", "gelu" (erf) or "gelu_tanh"; pad: elements behind every row of a that do not belong to it
  rope    tokens rows of `heads` query and `kv` key and value heads of `dim` channels, of which the first `rot` are
          rotated by position * frequency; layout "half" (pair i: channels i, i + rot / 2) or "pairs" (2 i, 2 i + 1).
          q, k and v are parts of one projection's output.  K and V rows go to the cache rows of their tokens: `batch`
          sequences with `room` rows each, every sequence gets tokens / batch of them (the first ones one more), behind
          `front` that it holds already.  scaling "none", "linear" or "turns" by `factor`; magnitude scales cos and sin
  attn    `batch` sequences with q_lo .. q_hi query tokens behind ctx_lo .. ctx_hi earlier keys (spread over the range
          by their logarithm); `idle` of them have no query.  heads, kv, dim as above.  block 0: every query sees all
          keys of its sequence; block b: those up to the end of its own block of b positions (1: causal).  cache: keys
          in a cache of ctx_hi + q_hi rows per sequence (behind the last key of a sequence stale values), else in the
          same buffer as the queries.  spread: standard deviation of the logits
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _linear(name, m, n, k, bias=False, act="none", residual=False, dtype="bf16", pad=0):
    c = dict(op="linear", dtype=dtype, m=m, n=n, k=k, bias=bias, act=act, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _rope(name, tokens, heads, kv, dim, rot, layout, batch, front, room, scaling="none", factor=1.0, magnitude=1.0,
          base=10000.0, dtype="bf16"):
    c = dict(op="rope", dtype=dtype, tokens=tokens, heads=heads, kv=kv, dim=dim, rot=rot, layout=layout, batch=batch,
             front=front, room=room, scaling=scaling, factor=factor, magnitude=magnitude, base=base)
    return dict(c, name=name) if name else c


def _attn(name, batch, q_lo, q_hi, ctx_lo, ctx_hi, heads, kv, dim, block, cache, idle=0, spread=1.0, dtype="bf16"):
    c = dict(op="attn", dtype=dtype, batch=batch, q_lo=q_lo, q_hi=q_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, heads=heads,
             kv=kv, dim=dim, block=block, cache=cache, idle=idle, spread=spread)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the output projection of one decoded token, added to the residual stream: a stream over the weights
        _linear("linear_token", 1, 4096, 4096, residual=True),
        # Q, K and V with their biases for a prompt of odd length, 32 query and 8 key heads
        _linear("linear_qkv_bias", 777, 6144, 4096, bias=True),
        # the first feed-forward product of a batch of long prompts
        _linear("linear_up_gelu", 16384, 12288, 4096, bias=True, act="gelu"),
        # the fp32 path that results are checked on, a narrow layer, rows cut from a wider buffer
        _linear("linear_f32", 201, 512, 1536, bias=True, act="silu", residual=True, dtype="f32", pad=64),
        # one token each of eight sequences far into a long context: a call bound by its launch
        _rope("rope_step", 8, 32, 8, 128, 128, "half", 8, 6001, 8192, "turns", 8.0, 1.0, 500000.0),
        # a batch of prompts at the start of their caches
        _rope("rope_prompt", 16384, 32, 8, 128, 128, "half", 4, 0, 4224, "none", 1.0, 1.0, 10000.0),
        # interleaved pairs, a part of a narrow head, positions interpolated, fp32
        _rope("rope_part_f32", 1111, 12, 4, 64, 32, "pairs", 3, 17, 512, "linear", 4.0, 1.1, 10000.0, dtype="f32"),
        # single tokens of a running batch whose sequences differ in length, some slots idle
        _attn("attn_step", 32, 1, 1, 40, 4000, 32, 8, 128, 1, True, idle=3),
        # a single token of one very long sequence: the cache is read by all of the chip
        _attn("attn_step_long", 1, 1, 1, 131071, 131071, 32, 8, 128, 1, True),
        # the current block of 32 positions of every sequence, refined together over the cache of finished blocks
        _attn("attn_block_32", 16, 32, 32, 256, 2016, 32, 8, 128, 32, True, spread=2.0),
        # prompts of many lengths packed one behind the other, causal
        _attn("attn_prompts", 12, 33, 4096, 0, 0, 32, 8, 128, 1, False, spread=2.0),
        # the fp32 path: narrow heads, blocks that do not divide the lengths, a part of the keys cached
        _attn("attn_f32", 3, 7, 130, 5, 300, 12, 4, 64, 32, True, dtype="f32"),
    ]


def draw(rng):
    """One more case of the ranges above; it costs no more than the largest listed one of its operator."""
    logu = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    op = rng.choice(["linear", "rope", "attn", "attn"])
    top = max(work(c)["flops"] for c in listed() if c["op"] == op)
    while True:
        f32 = rng.random() < 0.2
        dtype = "f32" if f32 else "bf16"
        if op == "linear":
            wide = 1536 if f32 else 12288
            c = _linear(None, logu(1, 300 if f32 else 16384), 64 * logu(4, wide // 64), 64 * logu(2, wide // 64),
                        rng.random() < 0.6, rng.choice(["none", "none", "silu", "gelu", "gelu_tanh"]),
                        rng.random() < 0.5, dtype, rng.choice([0, 0, 64, 200]))
        else:
            dim = 64 if f32 else rng.choice([64, 128, 128])
            kv = rng.choice([1, 2, 4, 8])
            heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
            if heads * dim > 4096:
                continue
            if op == "rope":
                batch, tokens = logu(1, 64), logu(1, 2000 if f32 else 16384)
                if tokens < batch:
                    continue
                front = rng.choice([0, logu(1, 100000 // batch)])
                room = front + tokens // batch + 1 + rng.randint(0, 200)
                c = _rope(None, tokens, heads, kv, dim, rng.choice([dim, dim, dim // 2, dim // 4 + 2]),
                          rng.choice(["half", "half", "pairs"]), batch, front, room,
                          rng.choice(["none", "linear", "turns"]), rng.choice([2.0, 4.0, 8.0]), rng.choice([1.0, 1.2]),
                          rng.choice([10000.0, 500000.0]), dtype)
            else:
                kind = rng.choice(["step", "block", "prompts"])
                if kind == "prompts":
                    hi = logu(1, 300 if f32 else 8192)
                    lo, batch = logu(1, hi), logu(1, 3 if f32 else 24)
                    c = _attn(None, batch, lo, hi, 0, 0, heads, kv, dim, rng.choice([0, 1, 1, 8, 32]), False,
                              spread=rng.choice([1.0, 2.0, 4.0]), dtype=dtype)
                else:
                    ctx_hi = logu(1, 400 if f32 else 131071)
                    ctx_lo, batch = logu(1, ctx_hi), logu(1, 4 if f32 else 64)
                    q = 1 if kind == "step" else rng.choice([2, 5, 8, 17, 32, 64])
                    c = _attn(None, batch, q, q, ctx_lo, ctx_hi, heads, kv, dim, rng.choice([0, 1, q]), True,
                              rng.randint(0, batch // 4), rng.choice([1.0, 2.0, 4.0]), dtype)
                if (c["ctx_hi"] + c["q_hi"]) * c["batch"] * kv * dim > 1 << 28 or c["q_hi"] * c["batch"] > 40000:
                    continue
        if work(c)["flops"] <= top:
            return c


# ---- the sizes of a case -----------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers between lo and hi, spread over the logarithm, the largest one first."""
    if lo < 1:
        return [hi] * n
    at = lambda i: 1.0 if i == 0 else (i * 0.6180339887498949) % 1.0
    return [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * at(i)))) for i in range(n)]


def _lengths(c):
    """Query tokens and keys of every sequence of an attention case."""
    q = _spread(c["q_lo"], c["q_hi"], c["batch"])
    ctx = _spread(c["ctx_lo"], c["ctx_hi"], c["batch"])
    keys = [a + b for a, b in zip(q, ctx)]
    for i in range(c["idle"]):  # idle slots, none of them the first
        q[1 + i * (c["batch"] - 1) // c["idle"]] = 0
    return q, keys


def _pairs(c, lq, lk):
    """(query, key) pairs of one head of one sequence that the mask lets through."""
    if c["block"] == 0:
        return lq * lk
    return sum(min(lk, ((i + lk - lq) // c["block"] + 1) * c["block"]) for i in range(lq))


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": e * (m * k + n * k + m * n * (2 if c["residual"] else 1) + (n if c["bias"] else 0)),
                "flops": 2 * m * n * k}
    if c["op"] == "rope":
        t = c["tokens"]
        return {"bytes": t * (e * 2 * (c["heads"] + 2 * c["kv"]) * c["dim"] + 8) + 4 * c["rot"],
                "flops": t * 3 * (c["heads"] + c["kv"]) * c["rot"]}
    q, keys = _lengths(c)
    seen = sum(lk for lq, lk in zip(q, keys) if lq)
    return {"bytes": e * c["dim"] * 2 * (sum(q) * c["heads"] + seen * c["kv"]),
            "flops": 4 * c["dim"] * c["heads"] * sum(_pairs(c, lq, lk) for lq, lk in zip(q, keys))}


def _frequencies(c):
    """Angle per position of every channel pair.  Scaled by turns: pairs that turn 4 times and more within a context of
    8192 positions keep their frequency, those that turn once or less are divided by the factor, between the two
    both are mixed."""
    f = [c["base"] ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]
    if c["scaling"] == "linear":
        f = [x / c["factor"] for x in f]
    elif c["scaling"] == "turns":
        mix = [min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1.0) / 3.0)) for x in f]
        f = [x * (g + (1.0 - g) / c["factor"]) for x, g in zip(f, mix)]
    return f


# ---- inputs ------------------------------------------------------------------------------

def _inputs(c, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    td = DTYPES[c["dtype"]]
    rn = lambda *shape: torch.randn(shape, device=dev, dtype=td, generator=gen)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        return {"a": rn(m, k + c["pad"])[:, :k], "wt": rn(n, k).mul_(k ** -0.5),
                "bias": rn(n).mul_(0.5) if c["bias"] else None, "residual": rn(m, n) if c["residual"] else None}
    if c["op"] == "rope":
        t, h, kv, d, b = c["tokens"], c["heads"], c["kv"], c["dim"], c["batch"]
        qkv = rn(t, h + 2 * kv, d)
        # token i belongs to sequence i % batch
        i = torch.arange(t)
        pos = c["front"] + i // b
        return {"q": qkv[:, :h], "k": qkv[:, h:h + kv], "v": qkv[:, h + kv:],
                "k_cache": rn(b * c["room"], kv, d), "v_cache": rn(b * c["room"], kv, d),
                "pos": pos.to(torch.int32).to(dev), "rows": ((i % b) * c["room"] + pos).to(torch.int32).to(dev),
                "freqs": torch.tensor(_frequencies(c), dtype=torch.float64, device=dev)}
    lq, lk = _lengths(c)
    h, kv, d, n = c["heads"], c["kv"], c["dim"], sum(lq)
    off = [0]
    for x in lq:
        off.append(off[-1] + x)
    if c["cache"]:
        room = c["ctx_hi"] + c["q_hi"]
        q, k, v = rn(n, h, d), rn(c["batch"] * room, kv, d), rn(c["batch"] * room, kv, d)
        begin = [i * room for i in range(c["batch"])]
    else:
        qkv = rn(n, h + 2 * kv, d)
        q, k, v = qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]
        begin = off[:-1]
    q.mul_(c["spread"])
    return {"q": q, "k": k, "v": v, "q_off": ints(off), "k_begin": ints(begin),
            "k_end": ints([b + x for b, x in zip(begin, lk)]), "host": (off, begin, lk), "max_q": max(lq), "max_k": max(lk)}


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["op"] == "linear":
        st["out"] = torch.empty(case["m"], case["n"], dtype=st["wt"].dtype, device=st["wt"].device)
    else:
        st["out"] = torch.empty(st["q"].shape, dtype=st["q"].dtype, device=st["q"].device)
    return st


# ---- one pass ------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _run_own(c, state)
    return {"linear": _plain_linear, "rope": _plain_rope, "attn": _plain_attn}[c["op"]](c, state)


def _run_own(c, st):
    from paper_2605_08134_amd import binding as B
    if c["op"] == "linear":
        B.dare_k_linear(st["a"], st["wt"], st["out"], bias=st["bias"], act=None if c["act"] == "none" else c["act"],
                        residual=st["residual"])
        return st["out"]
    if c["op"] == "rope":
        B.dare_k_rope(st["pos"], st["freqs"], c["layout"], q=st["q"], q_out=st["out"], k=st["k"], k_out=st["k_cache"],
                      v=st["v"], v_out=st["v_cache"], rows=st["rows"], magnitude=c["magnitude"])
        return st["out"], st["k_cache"], st["v_cache"]
    B.dare_k_attention_packed(st["q"], st["k"], st["v"], st["out"], st["q_off"], st["k_begin"], st["k_end"],
                              st["max_q"], st["max_k"], causal_block=c["block"])
    return st["out"]


def _plain_linear(c, st):
    y = st["a"].float() @ st["wt"].float().t()
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


def _plain_rope(c, st):
    # (angles in 64 bits: in 32 a position of 100000 loses what its fastest pair turns)
    angle = st["pos"].double()[:, None] * st["freqs"][None, :]
    cos, sin = (torch.cos(angle) * c["magnitude"]).float()[:, None], (torch.sin(angle) * c["magnitude"]).float()[:, None]
    rot = c["rot"]

    def turn(x):
        x = x.float()
        out = x.clone()
        first, second = ((slice(0, rot, 2), slice(1, rot, 2)) if c["layout"] == "pairs" else
                         (slice(0, rot // 2), slice(rot // 2, rot)))
        a, b = x[..., first], x[..., second]
        out[..., first] = a * cos - b * sin
        out[..., second] = b * cos + a * sin
        return out

    rows = st["rows"].long()
    st["out"].copy_(turn(st["q"]))
    st["k_cache"][rows] = turn(st["k"]).to(st["k_cache"].dtype)
    st["v_cache"][rows] = st["v"]
    return st["out"], st["k_cache"], st["v_cache"]


def _plain_attn(c, st):
    off, begin, lks = st["host"]
    h, kv, d, g = c["heads"], c["kv"], c["dim"], c["heads"] // c["kv"]
    for b, lk in enumerate(lks):
        lq = off[b + 1] - off[b]
        if lq == 0:
            continue
        k = st["k"][begin[b]:begin[b] + lk].float().permute(1, 2, 0).contiguous()  # [kv, d, lk]
        v = st["v"][begin[b]:begin[b] + lk].float().transpose(0, 1).contiguous()   # [kv, lk, d]
        step = max(1, (1 << 28) // (h * lk))  # query tokens whose logits are held at once
        for i in range(0, lq, step):
            j = min(lq, i + step)
            q = st["q"][off[b] + i:off[b] + j].float().view(j - i, kv, g, d).permute(1, 0, 2, 3).reshape(kv, -1, d)
            s = (q @ k) * d ** -0.5
            if c["block"]:
                pos = torch.arange(i, j, device=s.device) + (lk - lq)
                end = (pos // c["block"] + 1) * c["block"]
                seen = torch.arange(lk, device=s.device)[None, :] < end[:, None]
                s = s.view(kv, j - i, g, lk).masked_fill_(~seen[None, :, None, :], float("-inf")).view(kv, -1, lk)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            o = (p @ v) / p.sum(-1, keepdim=True)
            st["out"][off[b] + i:off[b] + j] = o.view(kv, j - i, g, d).permute(1, 0, 2, 3).reshape(j - i, h, d).to(
                st["out"].dtype)
    return st["out"]


# ---- the same in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["op"] == "linear":
        z = torch.matmul(x["a"].double(), x["wt"].double().mT.contiguous())
        if x["bias"] is not None:
            z = z + x["bias"].double()
        if c["act"] == "silu":
            z = z * torch.special.expit(z)
        elif c["act"] == "gelu":
            z = z * torch.special.erfc(-z / 2.0 ** 0.5) / 2.0
        elif c["act"] == "gelu_tanh":
            z = z * torch.special.expit(2.0 * (2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))
        return z if x["residual"] is None else z + x["residual"].double()
    if c["op"] == "rope":
        half = c["rot"] // 2
        z = torch.polar(torch.full((c["tokens"], half), c["magnitude"], dtype=torch.float64, device=x["q"].device),
                        torch.outer(x["pos"].double(), x["freqs"]))
        where = torch.arange(c["rot"], device=x["q"].device)
        where = where.view(half, 2) if c["layout"] == "pairs" else where.view(2, half).t()

        def turned(t):
            w = t.double()
            both = torch.view_as_complex(w[:, :, where].contiguous()) * z[:, None, :]
            w = w.clone()
            w[:, :, where.reshape(-1)] = torch.view_as_real(both).flatten(-2)
            return w

        kc, vc, rows = x["k_cache"].double(), x["v_cache"].double(), x["rows"].long()
        kc.index_copy_(0, rows, turned(x["k"]))
        vc.index_copy_(0, rows, x["v"].double())
        return turned(x["q"]), kc, vc
    off, begin, lks = x["host"]
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device=x["q"].device)
    group = c["heads"] // c["kv"]
    for b, lk in enumerate(lks):
        lq = off[b + 1] - off[b]
        rows = max(1, (1 << 27) // lk)
        for h in range(c["heads"]):
            if lq == 0:
                break
            key = x["k"][begin[b]:begin[b] + lk, h // group].double()
            value = x["v"][begin[b]:begin[b] + lk, h // group].double()
            for i in range(0, lq, rows):
                n = min(rows, lq - i)
                logits = torch.mm(x["q"][off[b] + i:off[b] + i + n, h].double(), key.t()) / math.sqrt(c["dim"])
                if c["block"]:
                    at = torch.arange(lk - lq + i, lk - lq + i + n, device=logits.device)
                    hidden = torch.arange(lk, device=logits.device) // c["block"] > (at // c["block"])[:, None]
                    logits[hidden] = -torch.inf
                out[off[b] + i:off[b] + i + n, h] = torch.mm(torch.softmax(logits, -1), value)
    return out
