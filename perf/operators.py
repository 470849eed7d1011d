"""Timed cases of the operators beside the 1-bit Adam path that a language
model's training step is made of on this package: the token embedding, whose
gradient is the largest tensor that the optimizer compresses, and the
orthogonalised (Muon) step of the hidden matrices.

A case is one call:

  embed    onebit_embedding_forward(): rows of a table for a batch of tokens
  embgrad  onebit_embedding_grad(): the table's gradient, every row of it
  ortho    onebit_orthogonalize(): Newton-Schulz products of a list of matrices
  muon     onebit_muon_step(): the workers' mean gradient, momentum,
           orthogonalised update and the parameters

Matrices are written "count x rows x columns", groups apart by spaces; matrix
k + 1 starts at the next multiple of 64 elements after matrix k.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
VOCAB = 30522
STEPS, COEFFICIENTS, NORM_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LR, MOMENTUM, WEIGHT_DECAY = 2e-3, 0.95, 0.01
BERT_LARGE = "96x1024x1024 24x4096x1024 24x1024x4096"


def _embed(tokens, width, table, out, vocab=VOCAB, ids="i64", masked=0.0, scale=1.0):
    return dict(kind="embed", tokens=tokens, width=width, table=table, out=out, vocab=vocab,
                ids=ids, masked=masked, scale=scale)


def _embgrad(tokens, width, dout, grad, vocab=VOCAB, ids="i64", masked=0.0, scale=1.0,
             padding=-1, accumulate=False):
    return dict(kind="embgrad", tokens=tokens, width=width, dout=dout, grad=grad, vocab=vocab,
                ids=ids, masked=masked, scale=scale, padding=padding, accumulate=accumulate)


def _ortho(matrices, grad, out):
    return dict(kind="ortho", matrices=matrices, grad=grad, out=out)


def _muon(matrices, n, grad, nesterov=True):
    return dict(kind="muon", matrices=matrices, n=n, grad=grad, nesterov=nesterov)


def listed():
    return [
        # one sequence of 512 tokens, BERT-Large table, bf16 activations: latency
        dict(_embed(512, 1024, "f32", "bf16"), name="embed-512"),
        # a batch of 256 sequences of 512 tokens
        dict(_embed(131072, 1024, "f32", "bf16"), name="embed-131072"),
        # rows of an odd width, a bf16 table, padded places masked, scaled by sqrt(width)
        dict(_embed(10007, 771, "bf16", "f32", 50001, "i32", 0.2, 27.75), name="embed-odd-masked"),
        # one sequence's gradient: nearly all of the table's gradient is zeros to write
        dict(_embgrad(512, 1024, "bf16", "f32"), name="embgrad-512"),
        # 256 sequences of 512 tokens, Zipf-distributed: a few rows have thousands of tokens
        dict(_embgrad(131072, 1024, "bf16", "f32"), name="embgrad-131072"),
        # an odd width, masked places, a padding row, added to a tied table's gradient
        dict(_embgrad(33333, 771, "f32", "f32", 5003, "i32", 0.2, 27.75, 0, True),
             name="embgrad-odd-tied"),
        # the matrices of a small network, fp32 in and out: launches and latency
        dict(_ortho("8x128x128 2x512x128 2x128x512", "f32", "f32"), name="ortho-small-f32"),
        # one hidden matrix of the BERT-Large shape, bf16 in and out
        dict(_ortho("1x1024x1024", "bf16", "bf16"), name="ortho-1024-bf16"),
        # all 144 hidden matrices of the BERT-Large shape, as a rank would send them on
        dict(_ortho(BERT_LARGE, "f32", "bf16"), name="ortho-bert-large-bf16"),
        # ragged matrices, four workers' fp32 gradients
        dict(_muon("3x300x1000 2x1001x257 5x63x65 1x17x4000", 4, "f32"), name="muon-ragged"),
        # four layers' attention and feed-forward matrices, eight workers' bf16 gradients
        dict(_muon("16x1024x1024 4x4096x1024 4x1024x4096", 8, "bf16"), name="muon-4-layers-bf16"),
        # the whole BERT-Large shape, one bf16 gradient row (averaged before the call)
        dict(_muon(BERT_LARGE, 1, "bf16"), name="muon-bert-large-bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["embed", "embgrad", "embgrad", "ortho", "ortho", "muon", "muon"])
    if kind in ("embed", "embgrad"):
        width = rng.choice([64, 768, 1024, _log(rng, 32, 2048)])
        vocab = rng.choice([VOCAB, _log(rng, 100, 60000)])
        tokens = _log(rng, 1, min(131072, 131072 * 1024 // width))
        types = [rng.choice(["f32", "bf16", "f16"]) for _ in range(2)]
        more = dict(ids=rng.choice(["i32", "i64"]), masked=rng.choice([0.0, 0.0, 0.3]),
                    scale=rng.choice([1.0, 27.75]))
        if kind == "embed":
            return _embed(tokens, width, *types, vocab, **more)
        # a tied table's gradient is added to in fp32: the others are written anew
        more.update(padding=rng.choice([-1, -1, 0]), accumulate=types[1] == "f32" and
                    rng.random() < 0.5)
        return _embgrad(tokens, width, *types, vocab, **more)
    groups, macs = [], 0.0
    for _ in range(rng.choice([1, 1, 2, 3])):
        r, c = _log(rng, 16, 4096), _log(rng, 16, 4096)
        if rng.random() < 0.4:  # the usual multiples of 64
            r, c = max(64, r // 64 * 64), max(64, c // 64 * 64)
        one = STEPS * (2 * min(r, c) * r * c + min(r, c) ** 3)
        count = _log(rng, 1, 24)
        while count > 1 and (macs + one * count > 1.5e12 or count * r * c > 40_000_000):
            count -= 1
        macs += one * count
        groups.append("%dx%dx%d" % (count, r, c))
    grad = rng.choice(["f32", "bf16", "f16"])
    if kind == "ortho":
        return _ortho(" ".join(groups), grad, rng.choice(["f32", "bf16", "bf16", "f16"]))
    return _muon(" ".join(groups), rng.choice([1, 1, 2, 4, 8]), grad, rng.random() < 0.7)


# ---------------------------------------------------------------------------
# Layout and inputs: every array is a seeded draw of its own
# ---------------------------------------------------------------------------

def _groups(case):
    """[(count, rows, columns, offset of the first, elements from one to the next)]"""
    got, at = [], 0
    for text in case["matrices"].split():
        count, r, c = (int(v) for v in text.split("x"))
        pitch = (r * c + 63) // 64 * 64
        got.append((count, r, c, at, pitch))
        at += count * pitch
    return got, at


def _views(flat, groups):
    """Each group's matrices in a flat buffer, as [count, rows, columns]."""
    return [flat.as_strided((n, r, c), (pitch, c, 1), flat.storage_offset() + at)
            for n, r, c, at, pitch in groups]


def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 64 + what) & ((1 << 62) - 1))
    return g


def _normal(size, std, seed, what, dtype=torch.float32):
    return torch.empty(size, dtype=dtype, device="cuda").normal_(0.0, std, generator=_gen(seed, what))


def _ids(case, seed):
    """Tokens of a Zipf distribution: id k with a probability of about 1 / k;
    a share `masked` of the places holds -1, as padded places of a batch do."""
    u = torch.rand(case["tokens"], dtype=torch.float64, device="cuda", generator=_gen(seed, 1))
    ids = (torch.exp(u * math.log(case["vocab"] + 1)) - 1).long().clamp_(0, case["vocab"] - 1)
    if case["masked"]:
        drop = torch.rand(case["tokens"], device="cuda", generator=_gen(seed, 2)) < case["masked"]
        ids.masked_fill_(drop, -1)
    return ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _gradient(groups, extent, seed, what, dtype):
    """A minibatch gradient's two parts: a few directions and noise over all."""
    flat = torch.zeros(extent, dtype=torch.float32, device="cuda")
    for k, v in enumerate(_views(flat, groups)):
        n, r, c = v.shape
        rank = min(16, r, c)
        v.copy_(_normal((n, r, c), 1e-3, seed, what + 3 * k))
        v.add_(torch.bmm(_normal((n, r, rank), 1e-3, seed, what + 3 * k + 1),
                         _normal((n, rank, c), 1.0, seed, what + 3 * k + 2)))
    return flat.to(dtype)


def prepare(case, seed):
    kind, dev = case["kind"], torch.device("cuda", torch.cuda.current_device())
    s = {"case": case}
    if own:
        import paper_2102_02888_amd as ob
        s["ob"] = ob
    if kind == "embed":
        s["ids"] = _ids(case, seed)
        s["table"] = _normal((case["vocab"], case["width"]), 0.02, seed, 3, TYPES[case["table"]])
        s["out"] = torch.empty((case["tokens"], case["width"]), dtype=TYPES[case["out"]], device=dev)
    elif kind == "embgrad":
        s["ids"] = _ids(case, seed)
        s["dout"] = _normal((case["tokens"], case["width"]), 1e-3, seed, 3, TYPES[case["dout"]])
        s["grad"] = _normal((case["vocab"], case["width"]), 1e-3, seed, 4, TYPES[case["grad"]])
        if own:
            s["work"] = s["ob"].embedding_workspace(case["tokens"], case["vocab"], case["width"], dev)
    else:
        s["groups"], s["extent"] = groups, extent = _groups(case)
        dtype = TYPES[case["grad"]]
        if kind == "ortho":
            s["grad"] = _gradient(groups, extent, seed, 8, dtype)
            s["out"] = torch.zeros(extent, dtype=TYPES[case["out"]], device=dev)
        else:
            s["x"] = _normal(extent, 0.02, seed, 3)
            s["m"] = _gradient(groups, extent, seed, 8, torch.float32).mul_(5.0)
            s["grads"] = torch.stack([_gradient(groups, extent, seed, 32 + 16 * i, dtype)
                                      for i in range(case["n"])])
        if own:
            s["mats"] = s["ob"].Matrices([(r, c) for n, r, c, _, _ in groups for _ in range(n)])
            products = s["ob"].products_for(s["out"].dtype if kind == "ortho" else torch.float32)
            s["work"] = s["mats"].workspace(dev, products)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _run_own(s):
    case, ob = s["case"], s["ob"]
    if case["kind"] == "embed":
        ob.onebit_embedding_forward(s["table"], s["ids"], s["out"], scale=case["scale"])
        return s["out"]
    if case["kind"] == "embgrad":
        ob.onebit_embedding_grad(s["dout"], s["ids"], s["grad"], s["work"], scale=case["scale"],
                                 padding_idx=case["padding"], accumulate=case["accumulate"])
        return s["grad"]
    if case["kind"] == "ortho":
        ob.onebit_orthogonalize(s["mats"], s["grad"], s["out"], s["work"])
        return s["out"]
    ob.onebit_muon_step(s["mats"], s["x"], s["m"], s["grads"], LR, MOMENTUM, s["work"],
                        nesterov=case["nesterov"], weight_decay=WEIGHT_DECAY,
                        scale=ob.MUON_SCALE_RMS)
    return {"x": s["x"], "m": s["m"]}


def _newton_schulz(u):
    """Five Newton-Schulz steps on [count, rows, columns] in fp32."""
    wide = u.shape[1] <= u.shape[2]
    a, b, c = COEFFICIENTS
    x = u if wide else u.mT
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NORM_EPS)
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x if wide else x.mT


def _taken(case, ids):
    """Which places hold a token of the table, and their ids with 0 elsewhere."""
    on = (ids >= 0) & (ids < case["vocab"])
    return on, torch.where(on, ids, 0).long()


def _update_group(x, m, u, lr):
    """x - lr (0.2 sqrt(max(rows, columns)) O + weight decay x), in place."""
    o = _newton_schulz(u)
    x.mul_(1 - lr * WEIGHT_DECAY).sub_(o, alpha=lr * 0.2 * math.sqrt(max(x.shape[1:])))


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["kind"] == "embed":
        on, ids = _taken(case, s["ids"])
        rows = s["table"][ids].float() * case["scale"]
        return torch.where(on[:, None], rows, 0.0).to(s["out"].dtype)
    if case["kind"] == "embgrad":
        on, ids = _taken(case, s["ids"])
        rows = s["dout"].float() * case["scale"]
        rows = torch.where((on & (ids != case["padding"]))[:, None], rows, 0.0)
        if case["accumulate"]:
            return s["grad"].index_add_(0, ids, rows)
        return torch.zeros_like(s["grad"], dtype=torch.float32).index_add_(0, ids, rows).to(s["grad"].dtype)
    groups = s["groups"]
    if case["kind"] == "ortho":
        for u, out in zip(_views(s["grad"], groups), _views(s["out"], groups)):
            out.copy_(_newton_schulz(u.float()))
        return s["out"]
    g = s["grads"].float().mean(0)
    s["m"].mul_(MOMENTUM).add_(g)
    u = g + MOMENTUM * s["m"] if case["nesterov"] else s["m"]
    for views in zip(*(_views(t, groups) for t in (s["x"], s["m"], u))):
        _update_group(*views, LR)
    return {"x": s["x"], "m": s["m"]}


def work(case):
    """Each input read once and each output written once; a Gram matrix and its
    square are symmetric, so that half of their products are enough."""
    kind = case["kind"]
    if kind in ("embed", "embgrad"):
        t, w, v = case["tokens"], case["width"], case["vocab"]
        idb = 4 if case["ids"] == "i32" else 8
        if kind == "embed":
            # at most each token's row, at most the whole table
            rows = min(t, v) * w * BYTES[case["table"]]
            return {"bytes": t * idb + rows + t * w * BYTES[case["out"]], "flops": t * w}
        grad = v * w * BYTES[case["grad"]] * (2 if case["accumulate"] else 1)
        return {"bytes": t * idb + t * w * BYTES[case["dout"]] + grad, "flops": 2 * t * w}
    groups, _ = _groups(case)
    elems = sum(n * r * c for n, r, c, _, _ in groups)
    flops = sum(n * STEPS * 2 * (1.5 * min(r, c) * r * c + 0.5 * min(r, c) ** 3)
                for n, r, c, _, _ in groups)
    if kind == "ortho":
        return {"bytes": elems * (BYTES[case["grad"]] + BYTES[case["out"]]), "flops": flops}
    return {"bytes": elems * (case["n"] * BYTES[case["grad"]] + 16),
            "flops": flops + elems * (case["n"] + 6)}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def _polar64(u):
    """The Newton-Schulz polynomial applied five times to u / (|u| + eps), one
    matrix after another: X <- a X + b (X X') X + c (X X') (X X') X."""
    out = torch.empty_like(u)
    for k in range(u.shape[0]):
        x = u[k] / (torch.linalg.matrix_norm(u[k]) + NORM_EPS)
        flip = x.shape[0] > x.shape[1]
        for _ in range(STEPS):
            if flip:  # the same polynomial with the smaller Gram matrix on the right
                g = x.t().contiguous() @ x
                gx = x @ g
                x = COEFFICIENTS[0] * x + COEFFICIENTS[1] * gx + COEFFICIENTS[2] * (gx @ g)
            else:
                g = x @ x.t().contiguous()
                gx = g @ x
                x = COEFFICIENTS[0] * x + COEFFICIENTS[1] * gx + COEFFICIENTS[2] * (g @ gx)
        out[k] = x
    return out


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    kind = case["kind"]
    if kind == "embed":
        padded = torch.zeros((case["vocab"] + 1, case["width"]), dtype=torch.float64, device="cuda")
        padded[:-1] = s["table"].double() * case["scale"]
        ids = s["ids"].long()
        ids[(ids < 0) | (ids >= case["vocab"])] = case["vocab"]  # the row of zeros
        return padded[ids]
    if kind == "embgrad":
        ids = s["ids"].long()
        ids[(ids < 0) | (ids >= case["vocab"]) | (ids == case["padding"])] = case["vocab"]
        total = torch.zeros((case["vocab"] + 1, case["width"]), dtype=torch.float64, device="cuda")
        total.index_put_((ids,), s["dout"].double() * case["scale"], accumulate=True)
        return total[:-1] + s["grad"].double() if case["accumulate"] else total[:-1]
    groups, extent = s["groups"], s["extent"]
    if kind == "ortho":
        out = torch.zeros(extent, dtype=torch.float64, device="cuda")
        for u, o in zip(_views(s["grad"], groups), _views(out, groups)):
            o.copy_(_polar64(u.double()))
        return out
    g = torch.zeros(extent, dtype=torch.float64, device="cuda")
    for row in s["grads"]:
        g += row.double() / case["n"]
    m = MOMENTUM * s["m"].double() + g
    u = g + MOMENTUM * m if case["nesterov"] else m
    x = s["x"].double()
    for xv, uv in zip(_views(x, groups), _views(u, groups)):
        r, c = xv.shape[1:]
        xv.copy_(xv - LR * (WEIGHT_DECAY * xv + 0.2 * math.sqrt(max(r, c)) * _polar64(uv)))
    return {"x": x, "m": m}
