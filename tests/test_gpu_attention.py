"""Attention over packed sequences (onebit_attention_forward, onebit_attention_grad)
against plain 64-bit formulas, and its refusals.

Tolerances.  u is half a step of the operands' type (bf16 2^-8, fp16 2^-11).
Scores are products of 16-bit numbers added in fp32, at most 128 of them: off by
128 * 2^-24 = 2^-17 of the sum of magnitudes A_ij = scale |q_i| |k_j|.  An exponential
is off by that, by 2^-22 |score| and by the rounding of the maximum's (lse's) product,
together at most off = 2^-16 max A + 2^-21.  P is rounded once (u) and normalised by a
sum of the unrounded: out is off by (u + 2 off) * sum P |v|, then u of itself.
D adds 128 products of rounded results: off by u * sum |dout| |out| + 2^-17 of it.  dS =
P (dP - D) is then off by P ((2 off + 2^-17)(|dout| |v| + |D|) + D's), rounded by u of
itself; for fp16, by half of its least number 2^-24 over the scale that brings the
largest of dout to 2^-5: 2^-20 of that largest.  Each product adds these magnitudes times
the other operand's, and the result is rounded by u of itself; sums over n tokens add
n 2^-24 of the magnitudes, within what 2 off leaves."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _side(tokens, heads, dim, dtype, dev, extra, seed, std=1.0, shift=0):
    """[tokens, heads, dim], `extra` elements between tokens, from element `shift` on."""
    flat = torch.randn(tokens * (heads * dim + extra) + shift, device=dev, generator=_gen(dev, seed)) * std
    return flat.to(dtype)[shift:].view(tokens, heads * dim + extra)[:, :heads * dim].unflatten(1, (heads, dim))


def _reference(q, k, v, at, causal, scale, dout=None, kind="bf16"):
    """Results and what each may be off by, in 64 bits, head by head."""
    u = U[kind]
    tokens, heads, dim = q.shape
    group = heads // k.shape[1]
    got = {name: torch.zeros(t.shape, dtype=torch.float64, device=q.device)
           for name, t in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {name: torch.zeros_like(t) for name, t in got.items()}
    lse = torch.zeros(tokens, heads, dtype=torch.float64, device=q.device)
    lse_off = 0.0
    least = 0.0
    if kind == "f16" and dout is not None:
        inside = dout[at[0]:at[-1]]
        least = 2.0 ** -20 * float(inside.abs().max()) if inside.numel() else 0.0
    for a, b in zip(at, at[1:]):
        if a == b:
            continue
        seen = torch.ones(b - a, b - a, dtype=torch.bool, device=q.device)
        if causal:
            seen = seen.tril()
        for h in range(heads):
            g = h // group
            qi, ki, vi = (t.double().contiguous() for t in (q[a:b, h], k[a:b, g], v[a:b, g]))
            s = torch.where(seen, qi @ ki.t().contiguous() * scale, -torch.inf)
            lse[a:b, h] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[a:b, h, None])
            size = float((qi.abs() @ ki.t().abs().contiguous()).max()) * scale
            off = 2.0 ** -16 * size + 2.0 ** -21
            lse_off = max(lse_off, off)
            o = p @ vi
            got["out"][a:b, h] = o
            tol["out"][a:b, h] = (u + 2 * off) * (p @ vi.abs()) + u * o.abs() + 2.0 ** -24
            if dout is None:
                continue
            di = dout[a:b, h].double().contiguous()
            dp, d = di @ vi.t().contiguous(), (di * o).sum(1, keepdim=True)
            ds = p * (dp - d)
            d_off = u * 2 * (di.abs() * (p @ vi.abs())).sum(1, keepdim=True)
            mag = di.abs() @ vi.abs().t().contiguous() + d.abs()
            ds_off = p * ((2 * off + 2.0 ** -17) * mag + d_off) + u * ds.abs() + torch.where(seen, least, 0.0)
            for name, row, x, x_off, y, y_size in (
                    ("dv", g, p.t(), ((u + 2 * off) * p + 2.0 ** -24).t(), di, 1.0),
                    ("dq", h, ds, ds_off, ki, scale), ("dk", g, ds.t(), ds_off.t(), qi, scale)):
                got[name][a:b, row] += x.contiguous() @ y * y_size
                tol[name][a:b, row] += x_off.contiguous() @ y.abs() * y_size
    for name in ("dq", "dk", "dv"):
        tol[name] += u * got[name].abs() + 2.0 ** -24
    return got, tol, lse, lse_off


def _check(dev, lengths, heads, kv, dim, kind, causal, extra=0, scale=None, before=0, after=0,
           std=1.0, dstd=1.0, shift=0):
    """Forward and backward over sequences of these lengths, with tokens in front of and
    behind them that belong to none and hold NaN."""
    import paper_2102_02888_amd as ob
    dtype, at = TYPES[kind], [before]
    for n in lengths:
        at.append(at[-1] + n)
    tokens = at[-1] + after
    starts = torch.tensor(at, dtype=torch.int32, device=dev)
    q, k, v, dout = (_side(tokens, h, dim, dtype, dev, extra, 1 + s, std if s < 2 else 1.0, shift)
                     for s, h in enumerate((heads, kv, kv, heads)))
    dout *= dstd
    none = torch.ones(tokens, dtype=torch.bool, device=dev)
    none[at[0]:at[-1]] = False
    for t in (q, k, v, dout):
        t[none] = float("nan")
    out = torch.full((tokens, heads, dim), 7.0, dtype=dtype, device=dev)
    lse = torch.full((tokens, heads), 7.0, device=dev)
    ob.onebit_attention_forward(q, k, v, starts, out, lse, causal=causal, scale=scale)
    scale64 = dim ** -0.5 if scale is None else scale
    want, tol, lse64, lse_off = _reference(q, k, v, at, causal, scale64, dout, kind)
    on = ~none

    def near(name, t):
        bad = ((t.double() - want[name]).abs() > tol[name])[on]
        assert not bool(bad.any()), (name, float(((t.double() - want[name]).abs() / tol[name])[on].max()))
        assert bool((t[none] == 7.0).all())
    near("out", out)
    assert bool(((lse - lse64).abs() <= lse_off + 2.0 ** -21 * (1 + lse64.abs()))[on].all())
    assert bool((lse[none] == 7.0).all())
    again = torch.full_like(out, 7.0)
    ob.onebit_attention_forward(q, k, v, starts, again, causal=causal, scale=scale)
    assert torch.equal(again, out)
    out[none] = float("nan")
    lse[none] = float("nan")
    need = (1024 + tokens * heads) * 4
    whole = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=dev)
    grads = [torch.full(t.shape, 7.0, dtype=dtype, device=dev) for t in (q, k, v)]
    for _ in range(2):
        kept = [g.clone() for g in grads]
        ob.onebit_attention_grad(dout, q, k, v, out, lse, starts, *grads, whole[:need], causal=causal,
                                 scale=scale)
        if _ == 0:
            for name, t in zip(("dq", "dk", "dv"), grads):
                near(name, t)
    assert all(torch.equal(a, b) for a, b in zip(kept, grads))  # bit for bit
    assert bool((whole[need:] == 0xA5).all())


@pytest.mark.parametrize("lengths,heads,kv,dim", [
    ([1], 1, 1, 1), ([1, 1, 0, 1], 2, 1, 8), ([5, 0, 31, 32, 33], 3, 1, 20), ([63, 64, 65], 4, 2, 64),
    ([127, 128, 129], 2, 2, 32), ([200], 6, 2, 33), ([300, 7], 2, 1, 65), ([257], 4, 4, 96),
    ([511, 3, 120], 4, 1, 128), ([130], 2, 2, 97), ([700], 1, 1, 80), ([1000, 24], 2, 1, 127),
    ([0], 2, 2, 16), ([0, 0, 0], 1, 1, 64),
])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
def test_attention(dev, lengths, heads, kv, dim, kind, causal):
    _check(dev, lengths, heads, kv, dim, kind, causal, extra=dim % 2 * 3)


@pytest.mark.parametrize("heads,kv", [(64, 64), (120, 60)])
@pytest.mark.parametrize("dim,shift", [(16, 0), (33, 0), (64, 0), (64, 1), (80, 0), (128, 0), (128, 1)])
@pytest.mark.parametrize("kind,causal", [("bf16", True), ("f16", False)])
def test_calls_of_many_tiles(dev, heads, kv, dim, shift, kind, causal):
    """More than 320 tiles of 128 tokens and a head: whole tiles go through the keys (the
    other tests' calls are small, and their waves share them)."""
    _check(dev, [130, 64, 257], heads, kv, dim, kind, causal, extra=2, shift=shift)


@pytest.mark.parametrize("dim", [8, 32, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("extra,shift", [(1, 0), (0, 1), (2, 2), (16, 8)])
def test_alignments(dev, dim, extra, shift):
    """Rows on 16-byte, 4-byte and odd borders: whole pieces go straight to LDS, others
    through registers."""
    _check(dev, [150, 33], 2, 1, dim, "bf16", True, extra=extra, shift=shift)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
def test_tokens_outside_the_sequences(dev, kind, causal):
    """Neither read, NaN as they are, nor written."""
    _check(dev, [70, 1, 200], 4, 2, 64, kind, causal, extra=5, before=3, after=130, shift=1)
    _check(dev, [70, 1, 200], 4, 2, 64, kind, causal, extra=8, before=3, after=130)
    _check(dev, [40], 2, 2, 128, kind, causal, before=129, after=1)


def test_one_token_of_a_wide_row(dev):
    """The distance to a next token means nothing where there is none."""
    import paper_2102_02888_amd as ob
    q = torch.randn(4, 2, 64, device=dev, generator=_gen(dev, 1)).bfloat16()
    starts = torch.tensor([0, 1], dtype=torch.int32, device=dev)
    for t in (q[:1], q[:1].as_strided((1, 2, 64), (0, 64, 1)), q[:1].as_strided((1, 2, 64), (3, 64, 1))):
        out, lse = torch.empty_like(q[:1]), torch.empty(1, 2, device=dev)
        ob.onebit_attention_forward(t, t, t, starts, out, lse)
        assert torch.equal(out, q[:1])  # the one key has all the weight
        L, p = ob.lib(), t.data_ptr()
        for ld in (-4, 0, 1 << 50):
            out.zero_()
            assert L.onebit_attention_forward(p, ld, p, ld, p, ld, 1, 1, 2, 2, 64, starts.data_ptr(), 1, 1,
                                              0.125, out.data_ptr(), ld, None,
                                              torch.cuda.current_stream().cuda_stream) == 0
            assert torch.equal(out, q[:1])


def test_many_short_sequences(dev):
    """More sequences than a wave looks at in a round, and than 64 rounds of it."""
    _check(dev, [1 + k % 5 for k in range(70)], 2, 1, 16, "bf16", True)
    _check(dev, [k % 3 for k in range(4200)], 1, 1, 8, "bf16", False)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_sharp_softmax_and_given_scale(dev, kind):
    """Scores of up to some hundreds: one key has nearly all the weight, and the running
    maximum moves by far more than a factor of 2^127."""
    _check(dev, [300, 64], 2, 1, 64, kind, True, scale=0.7, std=3.0)
    _check(dev, [300, 64], 2, 1, 64, kind, False, scale=1.3)


@pytest.mark.parametrize("tokens,heads", [(300, 2), (300, 200)])
@pytest.mark.parametrize("causal", [True, False])
def test_scores_below_fp32(dev, tokens, heads, causal):
    """Keys whose scores are below fp32's least number, -infinity, have no weight, also
    where a query sees nothing else in many tiles.  The other scores are 0, each of which
    has the same weight: out is the mean of their values, all of which are 1, and
    lse the logarithm of their number, within its 2^-21 (1 + |lse|) of rounding.  A query
    that sees no other key has no softmax: NaN, and lse -infinity."""
    import paper_2102_02888_amd as ob
    q, k, v = (torch.zeros(tokens, heads, 64, dtype=torch.bfloat16, device=dev) for _ in range(3))
    starts = torch.tensor([0, tokens], dtype=torch.int32, device=dev)
    q[:, :, 0] = 3e38
    v += 1
    low = torch.zeros(tokens, dtype=torch.bool, device=dev)
    low[:200] = True
    low[210:250] = True
    k[low, :, 0] = -3e38
    v[low] = 5.0
    out, lse = torch.empty_like(q), torch.empty(tokens, heads, device=dev)
    ob.onebit_attention_forward(q, k, v, starts, out, lse, causal=causal)
    n = (~low).cumsum(0) if causal else (~low).sum().expand(tokens)
    some = n > 0
    assert bool((out[some] == 1).all())
    want = n[some].double().log()[:, None]
    assert bool(((lse[some] - want).abs() <= 2.0 ** -21 * (1 + want)).all())
    assert bool(out[~some].isnan().all()) and bool((lse[~some] == -torch.inf).all())


@pytest.mark.parametrize("dstd", [1e-6, 3e-5, 300.0])
def test_gradients_of_any_size_in_fp16(dev, dstd):
    """dS is scaled before it is rounded to fp16, whose least number is 6e-8."""
    _check(dev, [200, 90], 2, 1, 64, "f16", True, dstd=dstd)


def test_nan_stays_in_its_sequence_and_head(dev):
    import paper_2102_02888_amd as ob
    at = [0, 100, 230, 300]
    starts = torch.tensor(at, dtype=torch.int32, device=dev)
    for bad in range(4):
        sides = [_side(300, h, 32, torch.bfloat16, dev, 0, s) for s, h in enumerate((4, 2, 2, 4))]
        sides[bad][150, 1, 3] = float("nan")
        sides[bad][160, 1, 5] = float("inf")
        q, k, v, dout = sides
        out, lse = torch.empty_like(q), torch.empty(300, 4, device=dev)
        ob.onebit_attention_forward(q, k, v, starts, out, lse)
        grads = [torch.empty_like(t) for t in (q, k, v)]
        ob.onebit_attention_grad(dout, q, k, v, out, lse, starts, *grads, ob.attention_workspace(300, 4, dev))
        for t in (out, *grads):
            nan = t.isnan().any(2)
            assert not bool(nan[:100].any()) and not bool(nan[230:].any())
            heads = {4: {0: (0, 2, 3), 1: (0, 1), 2: (0, 1), 3: (0, 2, 3)}, 2: {}}[t.shape[1]]
            clean = heads.get(bad, (0,) if bad in (1, 2) else (1,))
            assert not bool(nan[:, list(clean)].any()), (bad, t.shape)


def test_starts_out_of_range_are_cut(dev):
    """Nothing outside the tensors is read or written; ranges inside are as given."""
    import paper_2102_02888_amd as ob
    q, k, v = (_side(100, 2, 32, torch.bfloat16, dev, 0, s) for s in range(3))
    want, out = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    ob.onebit_attention_forward(q, k, v, torch.tensor([0, 40, 100], dtype=torch.int32, device=dev), want)
    ob.onebit_attention_forward(q, k, v, torch.tensor([-5, 40, 1 << 30], dtype=torch.int32, device=dev), out)
    assert torch.equal(out, want)
    lse = torch.zeros(100, 2, device=dev)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    for bad in ([90, 10, 50], [2147483647, -2147483648], [-7, -3], [200, 300]):
        s = torch.tensor(bad, dtype=torch.int32, device=dev)
        ob.onebit_attention_forward(q, k, v, s, out, lse)
        ob.onebit_attention_grad(out, q, k, v, out, lse, s, *grads, ob.attention_workspace(100, 2, dev))
    torch.cuda.synchronize()


def test_gradients_against_differences(dev):
    """Central differences of the 64-bit value along a direction, h = 1e-6, at operands
    that the type holds: within the sum of the gradient's tolerances times the direction."""
    import paper_2102_02888_amd as ob
    at = [0, 50, 51, 90]
    starts = torch.tensor(at, dtype=torch.int32, device=dev)
    q, k, v, dout = (_side(90, h, 24, torch.float16, dev, 0, s) for s, h in enumerate((4, 2, 2, 4)))
    out, lse = torch.empty_like(q), torch.empty(90, 4, device=dev)
    ob.onebit_attention_forward(q, k, v, starts, out, lse)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    ob.onebit_attention_grad(dout, q, k, v, out, lse, starts, *grads, ob.attention_workspace(90, 4, dev))
    _, tol, _, _ = _reference(q, k, v, at, True, 24 ** -0.5, dout, "f16")
    x = [t.double() for t in (q, k, v)]
    for n, (name, grad) in enumerate(zip(("dq", "dk", "dv"), grads)):
        d = torch.randn(grad.shape, dtype=torch.float64, device=dev, generator=_gen(dev, 40 + n))
        slope = 0.0
        for h in (1e-6, -1e-6):
            moved = _reference(*x[:n], x[n] + h * d, *x[n + 1:], at, True, 24 ** -0.5)[0]["out"]
            slope += float((moved * dout.double()).sum()) / (2 * h)
        assert abs(float((grad.double() * d).sum()) - slope) <= float((tol[name] * d.abs()).sum()) + 1e-6


def test_parts_of_one_projection_streams_and_graph(dev):
    """q, k, v and their gradients inside rows of one tensor each; another stream; a
    graph replayed with other sequences and numbers against the eager result."""
    import paper_2102_02888_amd as ob
    heads, kv, dim, tokens = 4, 2, 64, 500
    qkv = torch.randn(tokens, (heads + 2 * kv) * dim, device=dev, generator=_gen(dev, 1)).bfloat16()
    dqkv, out = torch.zeros_like(qkv), torch.empty(tokens, heads, dim, device=dev, dtype=torch.bfloat16)
    dout, lse = torch.randn_like(out), torch.empty(tokens, heads, device=dev)
    parts = qkv.view(tokens, -1, dim).split([heads, kv, kv], 1)
    grads = dqkv.view(tokens, -1, dim).split([heads, kv, kv], 1)
    starts = torch.tensor([0, 123, 124, 400, 500], dtype=torch.int32, device=dev)
    work = ob.attention_workspace(tokens, heads, dev)

    def calls(stream=None):
        ob.onebit_attention_forward(*parts, starts, out, lse, stream=stream)
        ob.onebit_attention_grad(dout, *parts, out, lse, starts, *grads, work, stream=stream)
    calls()
    whole = [t.contiguous() for t in parts]
    out2, grads2 = torch.empty_like(out), [torch.empty_like(t) for t in whole]
    ob.onebit_attention_forward(*whole, starts, out2)
    ob.onebit_attention_grad(dout, *whole, out, lse, starts, *grads2, work)
    assert torch.equal(out, out2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    kept = out.clone(), dqkv.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(kept[0], out) and torch.equal(kept[1], dqkv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed, at in ((4, [0, 1, 2, 3, 500]), (5, [0, 250, 250, 499, 500]), (6, [0, 100, 200, 300, 500])):
        qkv.copy_(torch.randn(qkv.shape, device=dev, generator=_gen(dev, seed)))
        starts.copy_(torch.tensor(at, dtype=torch.int32))
        calls()
        kept = out.clone(), dqkv.clone()
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(kept[0], out) and torch.equal(kept[1], dqkv), seed


def test_rows_past_32_bits(dev):
    """Tokens far apart: 2^31 and more elements from the first to the last."""
    import paper_2102_02888_amd as ob
    tokens, heads, dim, ld = 70000, 2, 64, 32768
    sides = [torch.zeros(tokens, ld, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    qkv = sides[0][:, :3 * heads * dim].unflatten(1, (3 * heads, dim))
    parts = qkv.split(heads, 1)
    n = 200
    qkv[-n:] = torch.randn(n, 3 * heads, dim, device=dev, generator=_gen(dev, 1)).bfloat16()
    starts = torch.tensor([tokens - n, tokens], dtype=torch.int32, device=dev)
    results = sides[1][:, :4 * heads * dim].unflatten(1, (4 * heads, dim)).split(heads, 1)
    lse = torch.zeros(tokens, heads, device=dev)
    ob.onebit_attention_forward(*parts, starts, results[0], lse)
    # the same tokens side by side (which kernels run goes by the number of tokens, too)
    small = [t.contiguous() for t in parts]
    out, l2 = torch.empty_like(small[0]), torch.empty(tokens, heads, device=dev)
    ob.onebit_attention_forward(*small, starts, out, l2)
    assert torch.equal(results[0][-n:], out[-n:]) and torch.equal(lse[-n:], l2[-n:])
    grads, work = [torch.empty_like(t) for t in small], ob.attention_workspace(tokens, heads, dev)
    ob.onebit_attention_grad(parts[0], *parts, results[0], lse, starts, *results[1:], work)
    ob.onebit_attention_grad(small[0], *small, out, l2, starts, *grads, work)
    assert all(torch.equal(a[-n:], b[-n:]) for a, b in zip(results[1:], grads))
    assert not bool(sides[1][:-n].any())


def test_refusals(dev):
    import paper_2102_02888_amd as ob
    q = torch.zeros(10, 4, 16, dtype=torch.bfloat16, device=dev)
    k, lse = torch.zeros(10, 2, 16, dtype=torch.bfloat16, device=dev), torch.zeros(10, 4, device=dev)
    starts, work = torch.tensor([0, 10], dtype=torch.int32, device=dev), ob.attention_workspace(10, 4, dev)
    fwd, bwd = ob.onebit_attention_forward, ob.onebit_attention_grad
    with pytest.raises(TypeError, match="q must be bfloat16 or float16"):
        fwd(q.float(), k, k, starts, q)
    with pytest.raises(TypeError, match="k must be"):
        fwd(q, k.half(), k, starts, q)
    with pytest.raises(ValueError, match="kv_heads a divisor"):
        fwd(q, torch.zeros(10, 3, 16, dtype=torch.bfloat16, device=dev), k, starts, q)
    with pytest.raises(ValueError, match="v is"):
        fwd(q, k, k[:9], starts, q)
    with pytest.raises(ValueError, match="side by side"):
        fwd(q, k.transpose(1, 2).contiguous().transpose(1, 2), k, starts, q)
    with pytest.raises(ValueError, match="overlapping"):
        fwd(q, k[:1].expand(10, 2, 16), k, starts, q)
    with pytest.raises(ValueError, match="GPU tensor"):
        fwd(q, k, k, starts.cpu(), q)
    with pytest.raises(TypeError, match="starts must be an int32"):
        fwd(q, k, k, starts.long(), q)
    with pytest.raises(ValueError, match="starts must be 1-D"):
        fwd(q, k, k, starts[:0], q)
    with pytest.raises(ValueError, match="lse must be contiguous"):
        fwd(q, k, k, starts, q, lse[:9])
    with pytest.raises(ob.OnebitError, match="scale"):
        fwd(q, k, k, starts, q, scale=0.0)
    with pytest.raises(ob.OnebitError, match="dim"):
        wide = torch.zeros(4, 1, 129, dtype=torch.bfloat16, device=dev)
        fwd(wide, wide, wide, starts, wide)
    with pytest.raises(ob.OnebitError, match="lse is NULL"):
        bwd(q, q, k, k, q, None, starts, q, k, k, work)
    with pytest.raises(ValueError, match="workspace has"):
        bwd(q, q, k, k, q, lse, starts, q, k, k, work[:64])
    with pytest.raises(ValueError, match="grad_k is"):
        bwd(q, q, k, k, q, lse, starts, q, q, k, work)


def _guarded(shape, dtype, dev, fill, inner):
    """A tensor filled with `inner` inside a larger one filled with `fill`: (it, whole)."""
    n = 1
    for s in shape:
        n *= s
    whole = torch.full((n + 16384,), fill, dtype=dtype, device=dev)
    whole[8192:8192 + n] = inner
    return whole[8192:8192 + n].view(shape), whole


def test_nothing_outside_the_tensors_with_starts_out_of_range(dev):
    """Starts that decrease or lie outside the tokens: what lies around results, gradients
    and workspace stays, NaN around the operands is not read; where the cut leaves no
    token nothing is written, and ranges that are cut give the gradients of the cut ones."""
    import paper_2102_02888_amd as ob
    tokens, heads, dim = 100, 2, 32
    nan = float("nan")

    def calls(at):
        s = torch.tensor(at, dtype=torch.int32, device=dev)
        q, k, v, dout = (_guarded((tokens, heads, dim), torch.bfloat16, dev, nan, 0.0)[0] for _ in range(4))
        for i, t in enumerate((q, k, v, dout)):
            t.copy_(_side(tokens, heads, dim, torch.bfloat16, dev, 0, i))
        results = [_guarded((tokens, heads, dim), torch.bfloat16, dev, 7.0, 7.0) for _ in range(4)]
        results.append(_guarded((tokens, heads), torch.float32, dev, 7.0, 7.0))
        need = ob.attention_workspace(tokens, heads, dev).numel()
        work, whole = _guarded((need,), torch.uint8, dev, 0xA5, 0)
        out, dq, dk, dv, lse = (t for t, _ in results)
        ob.onebit_attention_forward(q, k, v, s, out, lse)
        ob.onebit_attention_grad(dout, q, k, v, out, lse, s, dq, dk, dv, work)
        for t, around in results:
            n = t.numel()
            assert bool((around[:8192] == 7.0).all()) and bool((around[8192 + n:] == 7.0).all()), at
        assert bool((whole[:8192] == 0xA5).all()) and bool((whole[8192 + need:] == 0xA5).all()), at
        return [t for t, _ in results]
    want = calls([0, 40, 100])
    assert not any(bool(t.isnan().any()) for t in want)
    for a, b in zip(want, calls([-5, 40, 1 << 30])):
        assert torch.equal(a, b)
    for at in ([-7, -3], [200, 300], [2147483647, -2147483648], [100, 100], [0, 0]):
        assert all(bool((t == 7.0).all()) for t in calls(at)), at
    calls([90, 10, 50])
    calls([60, 90, 30, 100, -4])
