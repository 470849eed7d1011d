"""Attention in fp16 where its numbers span more than fp16 holds: gradients of very
different size in one call, weights far below the largest, and values near its largest
number; against plain 64-bit formulas.

Tolerances.  u = 2^-11 is half a step of fp16, 2^-25 half of its least number.  Scores and
exponentials are off by off = 2^-16 max A + 2^-21, as for any operands, A the products of
magnitudes.  Before a number between two products is rounded it is brought up by a power of
two: the forward's weights so that a row's largest is 2^7 or more (they stay below 2^16),
P by 2^15 for dv, dS so that the largest of its query (for dk, of its key over the heads that
share it) is 2^7 or more.  What is left of the least number is 2^-32 of the largest
weight, 2^-40 of P and 2^-32 of the query's (key's) largest dS; everything else is u of the
number itself.  D is off by sum |dout| times what the results may be off by, and by
2^-17 of its terms' magnitudes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -11


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _reference(q, k, v, dout, at, causal, scale):
    """Results and what each may be off by, in 64 bits."""
    heads, group = q.shape[1], q.shape[1] // k.shape[1]
    got = {name: torch.zeros(t.shape, dtype=torch.float64, device=q.device)
           for name, t in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {name: torch.zeros_like(t) for name, t in got.items()}
    for a, b in zip(at, at[1:]):
        seen = torch.ones(b - a, b - a, dtype=torch.bool, device=q.device)
        if causal:
            seen = seen.tril()
        for g in range(k.shape[1]):
            ki, vi = (t[a:b, g].double().contiguous() for t in (k, v))
            parts = []
            for h in range(g * group, (g + 1) * group):
                qi, di = (t[a:b, h].double().contiguous() for t in (q, dout))
                s = torch.where(seen, qi @ ki.t().contiguous() * scale, -torch.inf)
                p = torch.softmax(s, 1)
                off = 2.0 ** -16 * float((qi.abs() @ ki.t().abs().contiguous()).max()) * scale + 2.0 ** -21
                o, size = p @ vi, p @ vi.abs()
                got["out"][a:b, h] = o
                tol["out"][a:b, h] = (U + 2 * off) * size + 2.0 ** -32 * (seen.double() @ vi.abs()) + U * o.abs()
                dp, d = di @ vi.t().contiguous(), (di * o).sum(1, keepdim=True)
                ds = p * (dp - d)
                mag = di.abs() @ vi.abs().t().contiguous() + d.abs()
                d_off = (di.abs() * tol["out"][a:b, h]).sum(1, keepdim=True)
                ds_off = p * ((2 * off + 2.0 ** -17) * mag + d_off) + U * ds.abs()
                p_off = (U + 2 * off) * p + 2.0 ** -40 * seen
                parts.append((h, qi, di, p, p_off, ds, ds_off))
            largest = torch.stack([ds.abs().amax(0) for _, _, _, _, _, ds, _ in parts]).amax(0)
            for h, qi, di, p, p_off, ds, ds_off in parts:
                got["dq"][a:b, h] = ds @ ki * scale
                of_query = 2.0 ** -32 * ds.abs().amax(1, keepdim=True) * seen
                tol["dq"][a:b, h] = (ds_off + of_query) @ ki.abs() * scale
                got["dk"][a:b, g] += ds.t().contiguous() @ qi * scale
                tol["dk"][a:b, g] += (ds_off + 2.0 ** -32 * largest * seen).t().contiguous() @ qi.abs() * scale
                got["dv"][a:b, g] += p.t().contiguous() @ di
                tol["dv"][a:b, g] += p_off.t().contiguous() @ di.abs()
    for name in ("dq", "dk", "dv"):
        tol[name] += U * got[name].abs()
    return got, {name: t + 2.0 ** -25 for name, t in tol.items()}


def _check(dev, q, k, v, dout, at, causal, scale=None):
    import paper_2102_02888_amd as ob
    tokens, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    starts = torch.tensor(at, dtype=torch.int32, device=dev)
    out, lse = torch.empty_like(q), torch.empty(tokens, heads, device=dev)
    ob.onebit_attention_forward(q, k, v, starts, out, lse, causal=causal, scale=scale)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    ob.onebit_attention_grad(dout, q, k, v, out, lse, starts, *grads, ob.attention_workspace(tokens, heads, dev),
                             causal=causal, scale=scale)
    want, tol = _reference(q, k, v, dout, at, causal, scale)
    for name, t in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        held = want[name].abs() < 6e4  # (a result of 65,520 and more is infinity in fp16)
        ratio = torch.where(held, (t.double() - want[name]).abs() / tol[name], 0.0)
        assert bool((ratio <= 1).all()), (name, float(ratio.max()))
    return out, grads


def _operands(dev, tokens, heads, kv, dim):
    return [torch.randn(tokens, h, dim, device=dev, generator=_gen(dev, s)).half()
            for s, h in enumerate((heads, kv, kv, heads))]


@pytest.mark.parametrize("lengths,heads,kv,dim", [([300, 700, 90], 4, 2, 64), ([300, 700, 90], 4, 1, 40),
                                                  ([257, 64, 130], 64, 64, 64), ([257, 64, 130], 120, 60, 80),
                                                  ([300, 500], 2, 2, 128), ([130, 200, 3], 120, 120, 128),
                                                  ([150, 200], 2, 1, 33)])
@pytest.mark.parametrize("causal", [True, False])
def test_gradients_of_different_size_in_one_call(dev, lengths, heads, kv, dim, causal):
    """Sequences whose gradients differ by 1e4 and heads whose differ by 30: each has its
    own, within what its own size leaves, and the same bits as in a call of its own
    sizes whatever it is packed with."""
    import paper_2102_02888_amd as ob
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    q, k, v, dout = _operands(dev, at[-1], heads, kv, dim)
    for n, (a, b) in enumerate(zip(at, at[1:])):
        dout[a:b] *= (300.0, 0.03, 10.0)[n]
    dout[:, 1::2] *= 1 / 30
    out, grads = _check(dev, q, k, v, dout, at, causal)
    dout[:lengths[0]] *= 2.0 ** -14  # another neighbour: the second sequence stays as it is
    lse, starts = torch.empty(at[-1], heads, device=dev), torch.tensor(at, dtype=torch.int32, device=dev)
    ob.onebit_attention_forward(q, k, v, starts, out, lse, causal=causal)
    others = [torch.empty_like(t) for t in grads]
    ob.onebit_attention_grad(dout, q, k, v, out, lse, starts, *others,
                             ob.attention_workspace(at[-1], heads, dev), causal=causal)
    for x, y in zip(grads, others):
        assert torch.equal(x[at[1]:], y[at[1]:])


@pytest.mark.parametrize("heads", [1, 300])
def test_values_near_the_largest_number(dev, heads):
    """dP of up to 128 * 6e4: dS is far outside fp16, its products with small keys and
    queries are not."""
    q, k, v, dout = _operands(dev, 44, heads, heads, 128)
    q *= 1e-3
    k *= 1e-3
    v[:4] = 6e4
    v[0:4:2] *= -1
    dout *= 0.1
    dout[:4] = 1.0
    _check(dev, q, k, v, dout, [0, 2, 4, 44], False)


@pytest.mark.parametrize("n,heads", [(4096, 1), (1500, 40)])
@pytest.mark.parametrize("dim", [8, 64, 128])
def test_weights_far_below_the_largest(dev, n, heads, dim):
    """Every query sees one key with nearly all the weight; the others have 1.45 * 2^-24 of
    it each, which fp16 would round to 2^-24: the gradients of their values."""
    q, k, v, dout = _operands(dev, n, heads, heads, dim)
    q *= 1e-3
    k *= 1e-3
    q[:, :, 0], k[:, :, 0] = 1.0, 0.0
    k[0, :, 0] = (24 * math.log(2) - math.log(1.45)) * 8
    dout = (dout.abs() * 2000).half()
    _check(dev, q, k, v, dout, [0, n], False, scale=1 / 8)


@pytest.mark.parametrize("n,heads", [(4096, 1), (1500, 40)])
@pytest.mark.parametrize("dim", [8, 64, 128])
def test_many_keys_of_little_weight(dev, n, heads, dim):
    """Weights of 2^-25.5 of the largest, which fp16 would round to nothing, and what
    thousands of them add up to."""
    import paper_2102_02888_amd as ob
    q, k, v, dout = _operands(dev, n, heads, heads, dim)
    q *= 1e-3
    k *= 1e-3
    q[:, :, 0], k[:, :, 0] = 1.0, 0.0
    k[0, :, 0] = 25.5 * math.log(2) * 8
    v = (v * 10 + 5000).half()
    v[0] = 0.0
    dout *= 1e-2
    _check(dev, q, k, v, dout, [0, n], False, scale=1 / 8)


@pytest.mark.parametrize("heads", [2, 300])
@pytest.mark.parametrize("causal", [True, False])
def test_no_gradient_and_some(dev, heads, causal):
    """Gradients of nothing are nothing; with some queries that have none, the others' are
    within their own size."""
    import paper_2102_02888_amd as ob
    q, k, v, dout = _operands(dev, 150, heads, heads, 64)
    dout[:64] = 0.0
    dout[100:130] = 0.0
    _check(dev, q, k, v, dout, [0, 90, 91, 150], causal)
    starts = torch.tensor([0, 90, 91, 150], dtype=torch.int32, device=dev)
    out, lse = torch.empty_like(q), torch.empty(150, heads, device=dev)
    ob.onebit_attention_forward(q, k, v, starts, out, lse, causal=causal)
    grads = [torch.full_like(q, 7.0) for _ in range(3)]
    ob.onebit_attention_grad(torch.zeros_like(dout), q, k, v, out, lse, starts, *grads,
                             ob.attention_workspace(150, heads, dev), causal=causal)
    assert not any(bool(g.any()) for g in grads)


@pytest.mark.parametrize("heads", [4, 200])
def test_nan_and_infinity_stay_in_their_sequence_and_head(dev, heads):
    """Other sequences and heads have the same bits as without them."""
    import paper_2102_02888_amd as ob
    at = [0, 100, 230, 300]
    starts = torch.tensor(at, dtype=torch.int32, device=dev)
    work = ob.attention_workspace(300, heads, dev)

    def calls(sides):
        q, k, v, dout = sides
        out, lse = torch.empty_like(q), torch.empty(300, heads, device=dev)
        ob.onebit_attention_forward(q, k, v, starts, out, lse)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        ob.onebit_attention_grad(dout, q, k, v, out, lse, starts, *grads, work)
        return (out, *grads)
    want = calls(_operands(dev, 300, heads, heads // 2, 64))
    for bad in range(4):
        for value in (float("nan"), float("inf"), -float("inf")):
            sides = _operands(dev, 300, heads, heads // 2, 64)
            sides[bad][150, 1, 3] = value
            # head 1 of the queries, head 1 of the keys with heads 2 and 3 on it
            touched = {heads: [1] if bad in (0, 3) else [2, 3], heads // 2: [0] if bad in (0, 3) else [1]}
            for a, b in zip(want, calls(sides)):
                clean = torch.ones(300, a.shape[1], dtype=torch.bool, device=dev)
                for h in touched[a.shape[1]]:
                    clean[100:230, h] = False
                assert torch.equal(a[clean], b[clean]), (bad, value)
                assert not bool(a.isnan().any())
