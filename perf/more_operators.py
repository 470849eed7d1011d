"""Timed cases of the operators between a language model's embedding and its
loss: layer norm, attention over packed sequences, the log-probabilities of
given tokens and distillation from a teacher's top logits.

A case is one call, or the calls of one training step through an operator:

  norm      onebit_layer_norm_forward(): rows normalised, scaled and shifted
  normgrad  onebit_layer_norm_grad(): gradients of the rows, weight and bias
  attn      onebit_attention_forward(), followed with grad by
            onebit_attention_grad(): gradients of queries, keys and values
  logp      onebit_logprobs_forward(): log-probabilities of given tokens, the
            rows' entropies and their top alternatives; with grad
            onebit_logprobs_grad(), which gives the log-probabilities and the
            logits' gradient
  distill   onebit_distill_forward(): the divergence from a teacher's top
            logits; with grad onebit_distill_grad(), loss and gradient

Lengths of packed sequences are written "count x length", apart by spaces (the
count left out where it is 1).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
VOCAB = 30522
EPS = 1e-5
MOST_PAIRS = 4.0e11  # flops of the largest attention case, about
MOST_LOGITS = 8192 * VOCAB


def _norm(rows, width, x, y):
    return dict(kind="norm", rows=rows, width=width, x=x, y=y)


def _normgrad(rows, width, x, y, accumulate=False):
    return dict(kind="normgrad", rows=rows, width=width, x=x, y=y, accumulate=accumulate)


def _attn(lengths, heads, kv, dim, dtype, causal=True, grad=False):
    return dict(kind="attn", lengths=lengths, heads=heads, kv=kv, dim=dim, dtype=dtype,
                causal=causal, grad=grad)


def _logp(rows, vocab, dtype, top=0, ids="i64", masked=0.0, scale=1.0, grad=False):
    return dict(kind="logp", rows=rows, vocab=vocab, dtype=dtype, top=top, ids=ids, masked=masked,
                scale=scale, grad=grad)


def _distill(rows, vocab, dtype, top, scale=1.0, grad=False):
    return dict(kind="distill", rows=rows, vocab=vocab, dtype=dtype, top=top, scale=scale,
                grad=grad)


def listed():
    return [
        # a few rows of the BERT-Large width: latency
        dict(_norm(16, 1024, "bf16", "bf16"), name="norm-16"),
        # 256 sequences of 512 tokens through one layer's norm, backwards
        dict(_normgrad(131072, 1024, "bf16", "bf16"), name="normgrad-131072"),
        # rows of an odd width, an fp32 residual stream, added to gradients of another part
        dict(_normgrad(10007, 771, "f32", "bf16", True), name="normgrad-odd"),
        # one short prompt, the heads of BERT-Large
        dict(_attn("1x512", 16, 16, 64, "bf16"), name="attn-512"),
        # prompts of very different lengths in one call, four query heads to a key head
        dict(_attn("8192 4096 2500 1000 333 4x77 1", 16, 4, 128, "bf16"), name="attn-packed"),
        # a BERT-Large batch of 64 sequences, every token sees every other, training
        dict(_attn("64x512", 16, 16, 64, "bf16", False, True), name="attn-train-64x512"),
        # training on packed documents, heads of a size that fills no tile
        dict(_attn("2047 1500 900 3x411 130 65 17 2x1", 12, 4, 80, "f16", True, True),
             name="attn-train-odd"),
        # one step of generation: the next token's distribution, fp32 logits
        dict(_logp(1, VOCAB, "f32", 5), name="logp-1"),
        # scoring eight sequences of 512 tokens: log-probabilities, entropies, 20 alternatives
        dict(_logp(4096, VOCAB, "bf16", 20), name="logp-4096"),
        # training on 16 sequences of 512 tokens, padded places masked
        dict(_logp(8192, VOCAB, "bf16", masked=0.1, grad=True), name="logp-train-8192"),
        # training a student on a teacher's 64 best tokens, the same batch
        dict(_distill(8192, VOCAB, "bf16", 64, 0.5, True), name="distill-train-8192"),
        # fp32 logits of an odd vocabulary, a short list
        dict(_distill(1001, 50001, "f32", 7, grad=True), name="distill-train-odd"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["norm", "normgrad", "attn", "attn", "logp", "logp", "distill"])
    if kind in ("norm", "normgrad"):
        width = rng.choice([768, 1024, _log(rng, 16, 16384)])
        rows = _log(rng, 1, min(131072, 131072 * 1024 // width))
        types = [rng.choice(["f32", "bf16", "bf16", "f16"]) for _ in range(2)]
        if kind == "norm":
            return _norm(rows, width, *types)
        return _normgrad(rows, width, *types, rng.random() < 0.3)
    if kind == "attn":
        dim = rng.choice([64, 64, 128, 128, _log(rng, 8, 128)])
        kv = rng.choice([1, 2, 4, 8, 12])
        heads = kv * rng.choice([1, 1, 2, 4])
        grad, causal = rng.random() < 0.5, rng.random() < 0.7
        tokens = _log(rng, 64, 32768)
        lengths, left, flops = [], tokens, 0
        while left > 0 and len(lengths) < 64:
            n = min(left, _log(rng, 1, min(8192, tokens)))
            more = (14 if grad else 4) * heads * dim * n * n
            if flops + more > MOST_PAIRS:
                break
            flops += more
            left -= n
            lengths.append(str(n))
        return _attn(" ".join(lengths or ["64"]), heads, kv, dim, rng.choice(["bf16", "bf16", "f16"]),
                     causal, grad)
    vocab = rng.choice([VOCAB, VOCAB, _log(rng, 100, 150000)])
    rows = _log(rng, 1, min(8192, MOST_LOGITS // vocab))
    dtype, scale = rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice([1.0, 1.0, 0.5, 1.25])
    grad = rng.random() < 0.5
    if kind == "logp":
        return _logp(rows, vocab, dtype, 0 if grad else rng.choice([0, 1, 5, 20, 64]),
                     rng.choice(["i32", "i64"]), rng.choice([0.0, 0.1]), scale, grad)
    return _distill(rows, vocab, dtype, _log(rng, 1, 64), scale, grad)


# ---------------------------------------------------------------------------
# Inputs: every array is a seeded draw of its own
# ---------------------------------------------------------------------------

def _lengths(case):
    got = []
    for text in case["lengths"].split():
        count, _, n = text.rpartition("x")
        got += [int(n)] * int(count or 1)
    return got


def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 64 + what) & ((1 << 62) - 1))
    return g


def _normal(size, std, seed, what, dtype=torch.float32, mean=0.0):
    return torch.empty(size, dtype=dtype, device="cuda").normal_(mean, std, generator=_gen(seed, what))


def _logits(case, seed, what=1):
    """Logits as a trained model gives them: spread by a few units around an
    offset, and each row's token several units above the others."""
    x = _normal((case["rows"], case["vocab"]), 2.5, seed, what, TYPES[case["dtype"]], -1.0)
    ids = _tokens(case, seed)
    lift = 8.0 + 3.0 * torch.randn(case["rows"], device="cuda", generator=_gen(seed, 2))
    x[torch.arange(case["rows"], device="cuda"), ids] += lift.to(x.dtype)
    return x, ids


def _tokens(case, seed):
    u = torch.rand(case["rows"], dtype=torch.float64, device="cuda", generator=_gen(seed, 3))
    return (torch.exp(u * math.log(case["vocab"] + 1)) - 1).long().clamp_(0, case["vocab"] - 1)


def prepare(case, seed):
    kind, dev = case["kind"], torch.device("cuda", torch.cuda.current_device())
    s = {"case": case}
    if own:
        import paper_2102_02888_amd as ob
        s["ob"] = ob
    if kind in ("norm", "normgrad"):
        rows, width = case["rows"], case["width"]
        s["x"] = _normal((rows, width), 1.0, seed, 1, TYPES[case["x"]], 0.1)
        s["weight"] = _normal((width,), 0.1, seed, 2, mean=1.0)
        s["bias"] = _normal((width,), 0.1, seed, 3)
        if kind == "norm":
            s["y"] = torch.empty((rows, width), dtype=TYPES[case["y"]], device=dev)
        else:
            s["dy"] = _normal((rows, width), 1e-3, seed, 4, TYPES[case["y"]])
            s["dx"] = torch.empty_like(s["x"])
            s["dw"] = _normal((width,), 1e-2, seed, 5)
            s["db"] = _normal((width,), 1e-2, seed, 6)
            if own:
                s["work"] = s["ob"].layer_norm_workspace(rows, width, dev)
    elif kind == "attn":
        lengths = _lengths(case)
        tokens, dtype = sum(lengths), TYPES[case["dtype"]]
        at = [0]
        for n in lengths:
            at.append(at[-1] + n)
        s["at"], s["starts"] = at, torch.tensor(at, dtype=torch.int32, device=dev)
        # one projection's output: queries, keys and values of a token side by side
        sides = [case["heads"], case["kv"], case["kv"]]
        qkv = _normal((tokens, sum(sides), case["dim"]), 1.0, seed, 1, dtype)
        s["q"], s["k"], s["v"] = qkv.split(sides, dim=1)
        s["out"] = torch.empty((tokens, case["heads"], case["dim"]), dtype=dtype, device=dev)
        if case["grad"]:
            s["dout"] = _normal(s["out"].shape, 1e-2, seed, 2, dtype)
            s["dqkv"] = torch.empty_like(qkv)
            s["dq"], s["dk"], s["dv"] = s["dqkv"].split(sides, dim=1)
            s["lse"] = torch.empty((tokens, case["heads"]), dtype=torch.float32, device=dev)
            if own:
                s["work"] = s["ob"].attention_workspace(tokens, case["heads"], dev)
    else:
        rows, vocab, k = case["rows"], case["vocab"], case["top"]
        s["logits"], ids = _logits(case, seed)
        if case["grad"]:
            # a mean over the rows, of different weights
            s["weight"] = torch.rand(rows, device=dev, generator=_gen(seed, 4)) / rows
            s["dlogits"] = torch.empty_like(s["logits"])
        s["value"] = torch.empty(rows, dtype=torch.float32, device=dev)
        if kind == "logp":
            if case["masked"]:
                drop = torch.rand(rows, device=dev, generator=_gen(seed, 5)) < case["masked"]
                ids = ids.masked_fill(drop, -1)
            s["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
            if not case["grad"]:
                s["entropy"] = torch.empty(rows, dtype=torch.float32, device=dev)
                s["top_ids"] = torch.empty((rows, k), dtype=s["ids"].dtype, device=dev)
                s["top_logprobs"] = torch.empty((rows, k), dtype=torch.float32, device=dev)
        else:
            other = s["logits"].float()
            for part in other.split(1024):  # the teacher is another model of the same tokens
                part.add_(torch.randn(part.shape, device=dev, generator=_gen(seed, 6)))
            teacher = other.topk(min(k, vocab), dim=1)
            s["t_ids"] = teacher.indices.contiguous()
            s["t_logits"] = teacher.values.to(s["logits"].dtype).contiguous()
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _run_own(s):
    case, ob = s["case"], s["ob"]
    kind = case["kind"]
    if kind == "norm":
        ob.onebit_layer_norm_forward(s["x"], s["y"], s["weight"], s["bias"], eps=EPS)
        return s["y"]
    if kind == "normgrad":
        ob.onebit_layer_norm_grad(s["dy"], s["x"], s["dx"], s["work"], s["weight"], s["dw"],
                                  s["db"], eps=EPS, accumulate=case["accumulate"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if kind == "attn":
        if not case["grad"]:
            ob.onebit_attention_forward(s["q"], s["k"], s["v"], s["starts"], s["out"],
                                        causal=case["causal"])
            return s["out"]
        ob.onebit_attention_forward(s["q"], s["k"], s["v"], s["starts"], s["out"], s["lse"],
                                    causal=case["causal"])
        ob.onebit_attention_grad(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"],
                                 s["starts"], s["dq"], s["dk"], s["dv"], s["work"],
                                 causal=case["causal"])
        return {"out": s["out"], "dqkv": s["dqkv"]}
    if kind == "logp" and not case["grad"]:
        ob.onebit_logprobs_forward(s["logits"], s["ids"], s["value"], scale=case["scale"],
                                   entropy=s["entropy"], top_ids=s["top_ids"],
                                   top_logprobs=s["top_logprobs"])
        return {"logprobs": s["value"], "entropy": s["entropy"], "top_ids": s["top_ids"],
                "top_logprobs": s["top_logprobs"]}
    if kind == "logp":
        ob.onebit_logprobs_grad(s["logits"], s["ids"], s["weight"], s["dlogits"],
                                scale=case["scale"], logprobs=s["value"])
        return {"logprobs": s["value"], "dlogits": s["dlogits"]}
    if not case["grad"]:
        ob.onebit_distill_forward(s["logits"], s["t_ids"], s["t_logits"], s["value"],
                                  scale=case["scale"])
        return s["value"]
    ob.onebit_distill_grad(s["logits"], s["t_ids"], s["t_logits"], s["weight"], s["dlogits"],
                           scale=case["scale"], loss=s["value"])
    return {"loss": s["value"], "dlogits": s["dlogits"]}


def _normalised(x):
    x = x.float()
    x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    return x * r, r


def _run_norm(s):
    case = s["case"]
    z, r = _normalised(s["x"])
    if case["kind"] == "norm":
        return (z * s["weight"] + s["bias"]).to(s["y"].dtype)
    dy = s["dy"].float()
    g = dy * s["weight"]
    dx = r * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    dw, db = (dy * z).sum(0), dy.sum(0)
    if case["accumulate"]:
        dw, db = s["dw"].add_(dw), s["db"].add_(db)
    return {"dx": dx.to(s["dx"].dtype), "dw": dw, "db": db}


def _heads_first(x, group=1):
    """[tokens, heads, dim] as contiguous fp32 [heads * group, tokens, dim]."""
    return x.float().transpose(0, 1).repeat_interleave(group, 0).contiguous()


def _run_attn(s):
    case = s["case"]
    group, scale = case["heads"] // case["kv"], case["dim"] ** -0.5
    for a, b in zip(s["at"], s["at"][1:]):
        q, k, v = _heads_first(s["q"][a:b]), _heads_first(s["k"][a:b], group), _heads_first(s["v"][a:b], group)
        p = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale)
        if case["causal"]:
            p.masked_fill_(torch.ones(b - a, b - a, dtype=torch.bool, device=p.device).triu_(1), -math.inf)
        p = p.sub_(p.amax(2, keepdim=True)).exp_()
        p /= p.sum(2, keepdim=True)
        s["out"][a:b] = torch.bmm(p, v).transpose(0, 1)
        if not case["grad"]:
            continue
        do = _heads_first(s["dout"][a:b])
        dp = torch.bmm(do, v.transpose(1, 2).contiguous())
        dv = torch.bmm(p.transpose(1, 2).contiguous(), do)
        ds = dp.sub_((dp * p).sum(2, keepdim=True)).mul_(p).mul_(scale)
        dq = torch.bmm(ds, k)
        dk = torch.bmm(ds.transpose(1, 2).contiguous(), q)
        s["dq"][a:b] = dq.transpose(0, 1)
        for whole, part in ((s["dk"], dk), (s["dv"], dv)):
            whole[a:b] = part.view(case["kv"], group, b - a, case["dim"]).sum(1).transpose(0, 1)
    return {"out": s["out"], "dqkv": s["dqkv"]} if case["grad"] else s["out"]


def _log_softmax(x, scale):
    x = x.float() * scale
    x = x - x.amax(1, keepdim=True)
    return x.sub_(x.exp().sum(1, keepdim=True).log_())


def _top(x, k):
    """The k largest of each row, the lowest index first among equal ones: the
    numbers' order as integers, and the index, in one key."""
    bits = (x.float() + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    key = (key << 32) - torch.arange(x.shape[1], device=x.device)
    return key.topk(min(k, x.shape[1]), dim=1).indices


def _run_loss(s):
    case = s["case"]
    rows = torch.arange(case["rows"], device=s["logits"].device)
    logp = _log_softmax(s["logits"], case["scale"])
    if case["kind"] == "logp":
        on = s["ids"] >= 0
        ids = torch.where(on, s["ids"], 0).long()
        value = torch.where(on, logp[rows, ids], 0.0)
        if not case["grad"]:
            top = _top(s["logits"], case["top"])
            got = torch.gather(logp, 1, top)
            return {"logprobs": value, "entropy": -(logp.exp() * logp).sum(1),
                    "top_ids": top.to(s["ids"].dtype), "top_logprobs": got}
        w = torch.where(on, s["weight"], 0.0) * case["scale"]
        d = logp.exp_().mul_(-w[:, None])
        d[rows, ids] += w
        return {"logprobs": value, "dlogits": d.to(s["logits"].dtype)}
    logq = _log_softmax(s["t_logits"], case["scale"])
    q = logq.exp()
    value = (q * (logq - torch.gather(logp, 1, s["t_ids"]))).sum(1)
    if not case["grad"]:
        return value
    w = (s["weight"] * case["scale"])[:, None]
    d = logp.exp_().mul_(w).scatter_add_(1, s["t_ids"], -w * q)
    return {"loss": value, "dlogits": d.to(s["logits"].dtype)}


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    return _run_norm(s) if kind in ("norm", "normgrad") else _run_attn(s) if kind == "attn" else _run_loss(s)


def work(case):
    """Each input read once and each output written once; attention's products
    over the pairs that its mask leaves: two forwards, five backwards."""
    kind = case["kind"]
    if kind in ("norm", "normgrad"):
        n, w = case["rows"] * case["width"], case["width"]
        x, y = BYTES[case["x"]], BYTES[case["y"]]
        if kind == "norm":
            return {"bytes": n * (x + y) + 8 * w, "flops": 8 * n}
        return {"bytes": n * (2 * x + y) + (20 if case["accumulate"] else 12) * w, "flops": 17 * n}
    if kind == "attn":
        lengths = _lengths(case)
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lengths)
        row = (2 * case["heads"] + 2 * case["kv"]) * case["dim"] * BYTES[case["dtype"]]
        return {"bytes": sum(lengths) * row * (2 if case["grad"] else 1),
                "flops": (14 if case["grad"] else 4) * pairs * case["heads"] * case["dim"]}
    n, b = case["rows"] * case["vocab"], BYTES[case["dtype"]]
    each = 4 + (4 if case["grad"] else 0)
    if kind == "logp":
        idb = 4 if case["ids"] == "i32" else 8
        each += idb + (0 if case["grad"] else 4 + case["top"] * (4 + idb))
    else:
        each += case["top"] * (8 + b)
    return {"bytes": n * b * (2 if case["grad"] else 1) + case["rows"] * each,
            "flops": (8 if case["grad"] else 5) * n}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _exact_norm(s):
    case = s["case"]
    x = s["x"].double().requires_grad_()
    w, b = (s[k].double().requires_grad_() for k in ("weight", "bias"))
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    y = (x - mean) / torch.sqrt(var + EPS) * w + b
    if case["kind"] == "norm":
        return y.detach()
    dx, dw, db = torch.autograd.grad(y, [x, w, b], s["dy"].double())
    if case["accumulate"]:
        dw, db = dw + s["dw"].double(), db + s["db"].double()
    return {"dx": dx, "dw": dw, "db": db}


def _exact_attn(s):
    """Head by head: softmax over the keys that a token sees, by autograd."""
    case = s["case"]
    tokens, kv, dim = s["k"].shape
    group = case["heads"] // kv
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=s["out"].device)
    grads = torch.zeros(tokens, case["heads"] + 2 * kv, dim, dtype=torch.float64, device=out.device)
    for a, b in zip(s["at"], s["at"][1:]):
        hidden = None
        if case["causal"]:
            at = torch.arange(b - a, device=out.device)
            hidden = at[None, :] > at[:, None]
        for h in range(case["heads"]):
            g = h // group
            q, k, v = (t.double().contiguous().requires_grad_(case["grad"])
                       for t in (s["q"][a:b, h], s["k"][a:b, g], s["v"][a:b, g]))
            w = (q @ k.t()) / math.sqrt(dim)
            if hidden is not None:
                w = w.masked_fill(hidden, -math.inf)
            o = torch.softmax(w, 1) @ v
            out[a:b, h] = o.detach()
            if case["grad"]:
                d = torch.autograd.grad(o, [q, k, v], s["dout"][a:b, h].double())
                for row, part in zip((h, case["heads"] + g, case["heads"] + kv + g), d):
                    grads[a:b, row] += part
    return {"out": out, "dqkv": grads} if case["grad"] else out


def _exact_loss(s):
    case, parts = s["case"], []
    step = max(1, (1 << 26) // case["vocab"])
    for a in range(0, case["rows"], step):
        x = s["logits"][a:a + step].double().requires_grad_(case["grad"])
        lse = torch.logsumexp(x * case["scale"], 1, keepdim=True)
        logp = x * case["scale"] - lse
        if case["kind"] == "logp":
            ids = s["ids"][a:a + step].long()
            value = torch.where(ids >= 0, logp.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0)
            if not case["grad"]:
                top = torch.sort(s["logits"][a:a + step].double(), dim=1, descending=True,
                                 stable=True).indices[:, :case["top"]]
                parts.append({"logprobs": value, "entropy": torch.special.entr(logp.exp()).sum(1),
                              "top_ids": top.to(s["ids"].dtype), "top_logprobs": logp.gather(1, top)})
                continue
            name = "logprobs"
        else:
            t = s["t_logits"][a:a + step].double() * case["scale"]
            q = torch.softmax(t, 1)
            value = torch.nn.functional.kl_div(logp.gather(1, s["t_ids"][a:a + step]), q,
                                               reduction="none").sum(1)
            if not case["grad"]:
                parts.append({"": value})
                continue
            name = "loss"
        d = torch.autograd.grad(value, x, s["weight"][a:a + step].double())[0]
        parts.append({name: value.detach(), "dlogits": d})
    got = {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
    return got[""] if "" in got else got


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    kind = case["kind"]
    return _exact_norm(s) if kind in ("norm", "normgrad") else _exact_attn(s) if kind == "attn" else _exact_loss(s)
