"""The calls over logits (onebit_logprobs_*, onebit_distill_*) against plain 64-bit
formulas, at sizes, masks and numbers where they can go wrong, and their refusals.

Tolerances.  The sum S of n numbers e is at most 64 (n / 1,024 where the row does not
fit registers), 6 and 16 additions deep: off by at most 150 * 2^-24 = 9e-6 of itself
here.  An e is off by the roundings of d c, 3 * 2^-24 |d scale| of itself, and one of
the exponential, so that S is off by 2^-22 of the mean E of |d scale| under p besides.
log p is then off by 1.2e-5 + 2^-22 (E + |log p|), p by that much of itself, and the
entropy by it times (E + 1).  Gradients add products of these, then one rounding to the
type.  Numbers e below 2^-126 may count as zero."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 1e-36, "bf16": 1e-36, "f16": 2.0 ** -25}
INF = float("inf")

SHAPES = [(1, 1, 0), (5, 3, 2), (40, 65, 0), (9, 511, 1), (9, 512, 0), (9, 513, 0), (7, 2048, 0),
          (7, 2049, 3), (6, 8192, 0), (6, 8193, 0), (1, 30522, 0), (33, 30522, 1), (4, 32768, 0),
          (4, 32769, 0), (3, 65536, 0), (3, 65537, 1), (2, 150001, 0)]


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _logits(rows, vocab, dtype, dev, extra, seed, masked=False):
    """Rows with one number above the others, `extra` elements apart, from an odd
    element on; masked: some of -infinity and of the type's lowest number."""
    flat = torch.randn(rows * (vocab + extra) + 1, device=dev, generator=_gen(dev, seed)) * 3
    x = flat.to(dtype)[1:].view(rows, vocab + extra)[:, :vocab]
    x[torch.arange(rows), torch.randint(vocab, (rows,), device=dev, generator=_gen(dev, seed + 1))] += 6
    if masked and vocab > 2:
        r = torch.rand(rows, vocab, device=dev, generator=_gen(dev, seed + 2))
        x[r < 0.3] = -INF
        x[(r >= 0.3) & (r < 0.5)] = torch.finfo(dtype).min
        x[:, vocab // 2] = 1.5
    return x


def _ids(rows, vocab, dev, seed, dtype=torch.int64):
    ids = torch.randint(-1, vocab + 1, (rows,), device=dev, generator=_gen(dev, seed))
    ids[0] = min(3, vocab - 1)
    return ids.to(dtype)


class Row64:
    """log p, p and what a call is allowed to be off by, of [rows, vocab] logits."""

    def __init__(self, x, scale):
        x = x.double()
        most = x.max(1, keepdim=True).values
        d = torch.where(x == -INF, -INF, (x - most) * scale)
        self.logp = d - d.exp().sum(1, keepdim=True).log()
        self.p = self.logp.exp()
        self.entropy = -torch.where(self.p > 0, self.p * self.logp, 0.0).sum(1)
        self.mean = torch.where(self.p > 0, self.p * -d, 0.0).sum(1)  # E
        size = torch.where(self.logp == -INF, 0.0, self.logp.abs())  # also where p underflows
        self.off = 1.2e-5 + 2.0 ** -22 * (self.mean[:, None] + size)


def _near(got, want, tol):
    same = (got.double() == want) | ((got.double() - want).abs() <= tol)
    assert bool(same.all()), float((got.double() - want).abs()[~same].max())


@pytest.mark.parametrize("rows,vocab,extra", SHAPES)
@pytest.mark.parametrize("kind,idt,masked,scale", [("f32", torch.int64, False, 1.0),
                                                   ("bf16", torch.int32, True, 0.5),
                                                   ("f16", torch.int64, True, 1.7),
                                                   ("bf16", torch.int64, False, 1.0)])
def test_logprobs(dev, rows, vocab, extra, kind, idt, masked, scale):
    """Log-probabilities, entropies and alternatives; ties, which 16-bit logits are full
    of, go to the lowest index; -0 and 0 are equal."""
    import paper_2102_02888_amd as ob
    x = _logits(rows, vocab, TYPES[kind], dev, extra, 1, masked)
    if vocab > 8:
        x[-1, 3], x[-1, 7] = 0.0, -0.0
    ids = _ids(rows, vocab, dev, 5, idt)
    got, entropy = (torch.full((rows + 1,), 7.0, device=dev) for _ in range(2))
    want = Row64(x, scale)
    on = (ids >= 0) & (ids < vocab)
    at = torch.where(on, ids, 0).long()[:, None]
    for k in (0, 1, 5, 64):
        top = torch.full((rows, k), 99, dtype=idt, device=dev)
        logp = torch.full((rows, k), 9.0, device=dev)
        ob.onebit_logprobs_forward(x, ids, got[:rows], scale=scale, entropy=entropy[:rows],
                                   top_ids=top, top_logprobs=logp)
        _near(got[:rows], torch.where(on, want.logp.gather(1, at)[:, 0], 0.0),
              want.off.gather(1, at)[:, 0])
        _near(entropy[:rows], want.entropy, want.off[:, 0] * 0 + (want.mean + 1) * 2.5e-5)
        n = min(k, vocab)
        best = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :n]
        assert torch.equal(top[:, :n].long(), best), k
        _near(logp[:, :n], want.logp.gather(1, best), want.off.gather(1, best))
        assert bool((top[:, n:] == -1).all()) and bool((logp[:, n:] == -INF).all())
    assert float(got[rows]) == 7.0 and float(entropy[rows]) == 7.0


@pytest.mark.parametrize("rows,vocab,extra", SHAPES)
@pytest.mark.parametrize("kind,idt,masked,scale,more", [
    ("f32", torch.int64, False, 1.0, False), ("bf16", torch.int32, True, 0.5, False),
    ("f16", torch.int64, True, 1.7, True), ("f32", torch.int32, True, 1.0, True)])
def test_logprobs_gradient(dev, rows, vocab, extra, kind, idt, masked, scale, more):
    import paper_2102_02888_amd as ob
    x = _logits(rows, vocab, TYPES[kind], dev, extra, 1, masked)
    ids = _ids(rows, vocab, dev, 5, idt)
    g, h = (torch.randn(rows, device=dev, generator=_gen(dev, s)) for s in (6, 7))
    d = _logits(rows, vocab, TYPES[kind], dev, extra, 8)
    got, entropy = torch.full((rows,), 7.0, device=dev), torch.full((rows,), 7.0, device=dev)
    ob.onebit_logprobs_grad(x, ids, g, d, scale=scale, grad_entropy=h if more else None,
                            logprobs=got, entropy=entropy if more else None)
    r = Row64(x, scale)
    on = (ids >= 0) & (ids < vocab)
    at = torch.where(on, ids, 0).long()[:, None]
    _near(got, torch.where(on, r.logp.gather(1, at)[:, 0], 0.0), r.off.gather(1, at)[:, 0])
    one = torch.zeros_like(r.p).scatter_(1, at, 1.0)
    logp = torch.where(r.p > 0, r.logp, 0.0)
    g64 = torch.where(on, g.double(), 0.0)[:, None] * scale
    want = g64 * (one - r.p)
    tol = g64.abs() * (r.p * (r.off + 2.0 ** -22) + 2.0 ** -22 * one)
    if more:
        h64 = torch.where(on, h.double(), 0.0)[:, None] * scale
        term = r.p * (logp + r.entropy[:, None])
        want = want - h64 * term
        size = r.p * (logp.abs() + r.entropy[:, None] + 1 + r.mean[:, None])
        tol = tol + h64.abs() * size * (2 * r.off + 4e-5)
        _near(entropy, r.entropy, (r.mean + 1) * 2.5e-5)
    _near(d, want, tol + want.abs() * ULP[kind] + LEAST[kind])
    assert not bool(d[~on].any())
    inplace = x.clone()  # over the logits
    ob.onebit_logprobs_grad(inplace, ids, g, inplace, scale=scale, grad_entropy=h if more else None)
    assert torch.equal(inplace, d)


def _teacher(rows, vocab, k, dev, seed, idt, dtype):
    ids = torch.randint(vocab, (rows, k), device=dev, generator=_gen(dev, seed))
    z = (torch.randn(rows, k, device=dev, generator=_gen(dev, seed + 1)) * 2).to(dtype)
    if k > 4:
        ids[:, 3] = ids[:, 1]  # named twice
        ids[0, 2], ids[0, 0] = -1, vocab  # not tokens
        z[:, 4] = -INF
    return ids.to(idt), z


def _distill64(x, ids, z, scale):
    """(loss, what it may be off by, q per alternative, Row64)"""
    vocab, r = x.shape[1], Row64(x, scale)
    on = (ids >= 0) & (ids < vocab)
    at = torch.where(on, ids, 0).long()
    t = torch.where(on, z.double() * scale, -INF)
    logq = t - torch.logsumexp(t, 1, keepdim=True)
    logq = torch.where(logq.isnan(), -INF, logq)  # no alternative
    q = logq.exp()
    logp = r.logp.gather(1, at)
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    size = torch.where(q > 0, q * (logq.abs() + logp.abs() + 1), 0.0).sum(1)
    off = torch.where(q > 0, q * r.off.gather(1, at), 0.0).sum(1)
    return loss, off + size * 2e-5, q, at, r


@pytest.mark.parametrize("rows,vocab,extra", SHAPES)
@pytest.mark.parametrize("kind,teacher,idt,k,scale", [
    ("f32", "f32", torch.int64, 1, 1.0), ("bf16", "f32", torch.int32, 64, 0.5),
    ("f16", "f16", torch.int64, 7, 1.7), ("f32", "bf16", torch.int32, 256, 1.0)])
def test_distillation(dev, rows, vocab, extra, kind, teacher, idt, k, scale):
    import paper_2102_02888_amd as ob
    x = _logits(rows, vocab, TYPES[kind], dev, extra, 1)
    ids, z = _teacher(rows, vocab, k, dev, 3, idt, TYPES[teacher])
    g = torch.randn(rows, device=dev, generator=_gen(dev, 6))
    d = _logits(rows, vocab, TYPES[kind], dev, extra, 8)
    one, two = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
    ob.onebit_distill_forward(x, ids, z, one, scale=scale)
    ob.onebit_distill_grad(x, ids, z, g, d, scale=scale, loss=two)
    loss, off, q, at, r = _distill64(x, ids, z, scale)
    _near(one, loss, off)
    assert torch.equal(one, two)
    all_q = torch.zeros_like(r.p).scatter_add_(1, at, q)
    g64 = g.double()[:, None] * scale
    want = g64 * (r.p - all_q)
    tol = g64.abs() * (r.p * (r.off + 2.0 ** -22) + all_q * 2e-5)
    _near(d, want, tol + want.abs() * ULP[kind] + LEAST[kind])
    inplace = x.clone()
    ob.onebit_distill_grad(inplace, ids, z, g, inplace, scale=scale)
    assert torch.equal(inplace, d)


def _special(vocab, dtype, dev):
    """Rows: 0 all -infinity, 1 all the lowest number, 2 all equal, 3 two left by a mask,
    4 a NaN, 5 +infinity, 6 ordinary, 7 one left by a mask, 8 large numbers."""
    x = torch.randn(9, vocab, device=dev, generator=_gen(dev, 1)).to(dtype)
    x[0], x[1], x[2] = -INF, torch.finfo(dtype).min, 1.25
    x[3], x[7] = -INF, -INF
    x[3, vocab - 1], x[3, 1], x[7, vocab // 2] = 2.0, 1.0, -3.0
    x[4, 2], x[5, 3] = float("nan"), INF
    x[8] = 6e4
    x[8, 4] = 6.0032e4
    return x


@pytest.mark.parametrize("vocab", [9, 300, 3000, 30522, 40000, 70000])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_rows_that_masks_leave_empty_and_numbers_out_of_range(dev, vocab, kind):
    import paper_2102_02888_amd as ob
    x = _special(vocab, TYPES[kind], dev)
    ids = torch.full((9,), vocab - 1, device=dev)
    value, entropy = torch.empty(9, device=dev), torch.empty(9, device=dev)
    top, logp = torch.empty(9, 6, dtype=torch.int64, device=dev), torch.empty(9, 6, device=dev)
    ob.onebit_logprobs_forward(x, ids, value, entropy=entropy, top_ids=top, top_logprobs=logp)
    v, e = value.tolist(), entropy.tolist()
    uniform = math.log(vocab)
    assert v[0] == -INF and e[0] == 0
    for r in (1, 2):
        assert abs(v[r] + uniform) < 2e-5 and abs(e[r] - uniform) < 2e-5
    assert abs(v[3] + math.log1p(math.exp(-1))) < 2e-5 and v[7] == -INF and abs(e[7]) < 1e-6
    assert all(math.isnan(t) for t in (v[4], v[5], e[4], e[5]))
    assert torch.equal(top, torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :6])
    assert logp[3, 2:].eq(-INF).all() and logp[7, 1:].eq(-INF).all() and float(logp[7, 0]) == 0
    assert logp[0].eq(-INF).all() and logp[4].isnan().all()
    want = Row64(x, 1.0)
    _near(value[[6, 8]], want.logp[[6, 8], -1], want.off[[6, 8], -1])
    g, d = torch.ones(9, device=dev), torch.empty_like(x)
    for h in (None, g):
        ob.onebit_logprobs_grad(x, ids, g, d, grad_entropy=h)
        assert not bool(d[0].any())  # no distribution
        assert d[4].isnan().any() and d[5].isnan().any()
        assert not bool(d[[1, 2, 3, 6, 7, 8]].isnan().any())
        assert not bool(d[3, 2:-1].any()) and not bool(d[7, :vocab // 2].any())
        assert float(d[7, -1]) == 1.0  # scale g ([v = t] - p)
    t_ids = torch.tensor([[1, vocab - 1]], device=dev).expand(9, 2).contiguous()
    z = torch.tensor([[0.5, 0.25]], device=dev).repeat(9, 1)
    z[6] = -INF
    ob.onebit_distill_forward(x, t_ids, z, value)
    v = value.tolist()
    assert v[0] == INF and v[7] == INF and math.isnan(v[4]) and math.isnan(v[5]) and v[6] == 0
    ob.onebit_distill_grad(x, t_ids, z, g, d)
    assert not bool(d[0].any()) and not bool(d[6].any())
    assert not bool(d[[1, 2, 3, 7, 8]].isnan().any())
    t_ids[2] = -1  # no alternative
    ob.onebit_distill_grad(x, t_ids, z, g, d, loss=value)
    assert float(value[2]) == 0 and not bool(d[2].any())


def test_masked_places_are_not_read(dev):
    """A row whose id is not a token may hold anything: its gradient is zero."""
    import paper_2102_02888_amd as ob
    x = torch.full((3, 1000), float("nan"), device=dev)
    x[1] = 1.0
    ids = torch.tensor([-1, 5, 1000], device=dev)
    g, d, v = torch.full((3,), float("nan"), device=dev), torch.empty_like(x), torch.empty(3, device=dev)
    g[1] = 2.0
    ob.onebit_logprobs_grad(x, ids, g, d, logprobs=v)
    assert not bool(d[0].any()) and not bool(d[2].any()) and abs(float(d[1, 5]) - 2 * 0.999) < 1e-5
    assert float(v[0]) == 0 and float(v[2]) == 0


def test_rows_without_logits(dev):
    """A vocabulary of none: no token, no distribution, no alternative."""
    import paper_2102_02888_amd as ob
    x, ids = torch.zeros(3, 0, device=dev), torch.zeros(3, dtype=torch.int64, device=dev)
    v, e = torch.full((3,), 7.0, device=dev), torch.full((3,), 7.0, device=dev)
    top, logp = torch.zeros(3, 2, dtype=torch.int64, device=dev), torch.zeros(3, 2, device=dev)
    ob.onebit_logprobs_forward(x, ids, v, entropy=e, top_ids=top, top_logprobs=logp)
    assert not bool(v.any()) and not bool(e.any())
    assert bool((top == -1).all()) and bool((logp == -INF).all())
    ob.onebit_logprobs_grad(x, ids, v, x, logprobs=v)
    v.fill_(7.0)
    ob.onebit_distill_grad(x, top, logp, e, x, loss=v)
    assert not bool(v.any())


def test_outputs_that_are_left_out(dev):
    import paper_2102_02888_amd as ob
    x = _logits(20, 5000, torch.bfloat16, dev, 0, 1)
    ids = _ids(20, 5000, dev, 2)
    a, b, c, d = (torch.empty(20, device=dev) for _ in range(4))
    top, logp = torch.empty(20, 3, dtype=torch.int64, device=dev), torch.empty(20, 3, device=dev)
    ob.onebit_logprobs_forward(x, ids, a, entropy=b, top_ids=top, top_logprobs=logp)
    ob.onebit_logprobs_forward(x, ids, c)
    assert torch.equal(a, c)
    ob.onebit_logprobs_forward(x, None, None, entropy=d)
    assert torch.equal(b, d)
    t2, l2 = torch.empty(20, 3, dtype=torch.int32, device=dev), torch.empty(20, 3, device=dev)
    ob.onebit_logprobs_forward(x, None, None, top_ids=t2)
    assert torch.equal(top, t2.long())
    ob.onebit_logprobs_forward(x, None, None, top_logprobs=l2)
    assert torch.equal(logp, l2)
    ob.onebit_logprobs_forward(x[:0], ids[:0], a[:0])
    grad = torch.empty_like(x)
    ob.onebit_logprobs_grad(x, ids, None, grad, grad_entropy=torch.zeros(20, device=dev))
    assert not bool(grad.any())


@pytest.mark.parametrize("what", ["logprobs", "entropy", "distill"])
def test_gradients_against_differences(dev, what):
    """Central differences of the 64-bit value along a direction, h = 1e-6; the fp32
    gradient's own tolerance, 1e-4 of |gradient| |direction|."""
    import paper_2102_02888_amd as ob
    rows, vocab = 6, 700
    x = _logits(rows, vocab, torch.float32, dev, 0, 1)
    ids = torch.randint(vocab, (rows,), device=dev, generator=_gen(dev, 2))
    t_ids, z = _teacher(rows, vocab, 9, dev, 3, torch.int64, torch.float32)
    g, d = torch.randn(rows, device=dev, generator=_gen(dev, 4)), torch.empty_like(x)
    if what == "distill":
        ob.onebit_distill_grad(x, t_ids, z, g, d, scale=0.8)
    else:
        pair = (g, None) if what == "logprobs" else (None, g)
        ob.onebit_logprobs_grad(x, ids, pair[0], d, scale=0.8, grad_entropy=pair[1])

    def value(y):
        r = Row64(y, 0.8)
        each = (_distill64(y, t_ids, z, 0.8)[0] if what == "distill" else
                r.entropy if what == "entropy" else r.logp.gather(1, ids[:, None])[:, 0])
        return float((each * g.double()).sum())
    for seed in range(3):
        e = torch.randn(x.shape, dtype=torch.float64, device=dev, generator=_gen(dev, 20 + seed))
        slope = (value(x.double() + 1e-6 * e) - value(x.double() - 1e-6 * e)) / 2e-6
        assert abs(float((d.double() * e).sum()) - slope) < 1e-4 * float(d.norm()) * float(e.norm())


def test_a_teachers_alternatives_teach_a_student(dev):
    """The calls as they are used together: a teacher's top alternatives, whose
    log-probabilities serve as its logits, and the student's loss and gradient; on
    another stream and replayed from a graph."""
    import paper_2102_02888_amd as ob
    rows, vocab, k = 300, 1500, 16
    teacher, student = (_logits(rows, vocab, torch.bfloat16, dev, 0, s) for s in (1, 9))
    ids = torch.empty(rows, k, dtype=torch.int32, device=dev)
    logp, loss = torch.empty(rows, k, device=dev), torch.empty(rows, device=dev)
    g, d = torch.full((rows,), 1 / rows, device=dev), torch.empty_like(student)

    def calls(stream=None):
        ob.onebit_logprobs_forward(teacher, None, None, top_ids=ids, top_logprobs=logp,
                                   stream=stream)
        ob.onebit_distill_grad(student, ids, logp, g, d, loss=loss, stream=stream)
    calls()
    best = torch.sort(teacher.float(), dim=1, descending=True, stable=True)
    want, off = _distill64(student, best.indices[:, :k], best.values[:, :k], 1.0)[:2]
    _near(loss, want, off + 2e-5)
    kept = loss.clone(), d.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(kept[0], loss) and torch.equal(kept[1], d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (11, 12, 13):
        teacher.copy_(_logits(rows, vocab, torch.bfloat16, dev, 0, seed))
        calls()
        kept = loss.clone(), d.clone(), ids.clone()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(kept, (loss, d, ids))), seed


def test_logits_past_32_bits(dev):
    """2^31 and more elements: the last rows at their places; more rows than a launch
    has workgroups."""
    import paper_2102_02888_amd as ob
    rows, vocab = 72000, 30522
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=dev)
    x[-1, 7] = 5.0
    ids = torch.full((rows,), 7, device=dev, dtype=torch.int32)
    v, top = torch.empty(rows, device=dev), torch.empty(rows, 1, dtype=torch.int32, device=dev)
    ob.onebit_logprobs_forward(x, ids, v, top_ids=top)
    assert abs(float(v[-1]) - (5 - math.log(vocab - 1 + math.exp(5)))) < 2e-5
    assert bool((v[:-1] == v[0]).all()) and int(top[-1]) == 7 and not bool(top[:-1].any())
    ob.onebit_logprobs_grad(x, ids, torch.ones(rows, device=dev), x)
    assert bool((x[:-1] == x[0]).all()) and not torch.equal(x[-1], x[0])
    rows = (1 << 21) + 3
    x = torch.zeros(rows, 3, device=dev)
    x[-1, 1] = 1.0
    v, top = torch.empty(rows, device=dev), torch.empty(rows, 2, dtype=torch.int32, device=dev)
    ids = torch.full((rows,), 1, device=dev, dtype=torch.int32)
    ob.onebit_logprobs_forward(x, ids, v, top_ids=top)
    assert bool((v[:-1] == v[0]).all()) and abs(float(v[-1]) - (1 - math.log(2 + math.e))) < 2e-5
    assert top[-1].tolist() == [1, 0] and bool((top[:-1] == top[0]).all())


def test_refusals(dev):
    import paper_2102_02888_amd as ob
    x, ids = torch.zeros(5, 8, device=dev), torch.zeros(5, dtype=torch.int64, device=dev)
    v = torch.zeros(5, device=dev)
    fwd, bwd = ob.onebit_logprobs_forward, ob.onebit_logprobs_grad
    with pytest.raises(TypeError, match="logits must"):
        fwd(x.double(), ids, v)
    with pytest.raises(TypeError, match="ids"):
        fwd(x, ids.float(), v)
    with pytest.raises(TypeError, match="ids"):
        fwd(x, None, v)
    with pytest.raises(ValueError, match="ids has"):
        fwd(x, ids[:4], v)
    with pytest.raises(TypeError, match="logprobs must be a float32"):
        fwd(x, ids, v.double())
    with pytest.raises(ValueError, match="logprobs must be contiguous"):
        fwd(x, ids, v[:4])
    with pytest.raises(ValueError, match="GPU tensor"):
        fwd(x, ids, v.cpu())
    with pytest.raises(ob.OnebitError, match="scale"):
        fwd(x, ids, v, scale=0.0)
    with pytest.raises(ob.OnebitError, match="scale"):
        fwd(x, ids, v, scale=float("nan"))
    with pytest.raises(ob.OnebitError, match="top"):
        fwd(x, ids, v, top_logprobs=torch.zeros(5, 65, device=dev))
    with pytest.raises(ValueError, match="as many columns"):
        fwd(x, ids, v, top_ids=torch.zeros(5, 2, dtype=torch.int64, device=dev),
            top_logprobs=torch.zeros(5, 3, device=dev))
    with pytest.raises(TypeError, match="top_ids must be of ids' type"):
        fwd(x, ids, v, top_ids=torch.zeros(5, 2, dtype=torch.int32, device=dev))
    with pytest.raises(TypeError, match="grad_logits must be of the logits' type"):
        bwd(x, ids, v, x.bfloat16())
    with pytest.raises(ValueError, match="grad_logits is"):
        bwd(x, ids, v, x[:4])
    t_ids, z = torch.zeros(5, 3, dtype=torch.int64, device=dev), torch.zeros(5, 3, device=dev)
    with pytest.raises(ValueError, match="teacher_ids has"):
        ob.onebit_distill_forward(x, t_ids[:, :2].contiguous(), z, v)
    with pytest.raises(ValueError, match="teacher_logits is"):
        ob.onebit_distill_forward(x, t_ids, z[:4], v)
    with pytest.raises(ob.OnebitError, match="top"):
        ob.onebit_distill_forward(x, t_ids[:, :0].contiguous(), z[:, :0], v)
    with pytest.raises(ob.OnebitError, match="grad_loss"):
        ob.onebit_distill_grad(x, t_ids, z, None, x)
    with pytest.raises(TypeError, match="loss must"):
        ob.onebit_distill_forward(x, t_ids, z, "loss")
    with pytest.raises(ob.OnebitError, match="loss is NULL"):
        ob.onebit_distill_forward(x, t_ids, z, None)


@pytest.mark.parametrize("vocab", [600, 9000, 30522, 40000, 70000])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_nan_in_the_first_column_among_many_candidates(dev, vocab, kind):
    """NaN is above all and the lowest index first, also where more logits than LDS has
    room for reach the bound: rows of NaN only, and NaN in column 0 of rows that are
    otherwise equal, masked or NaN but for one."""
    import paper_2102_02888_amd as ob
    nan = float("nan")
    x = torch.full((5, vocab), nan, device=dev)
    x[1] = 1.25
    x[2] = -INF
    x[3] = 0.5
    x[4, 5] = 2.0
    x[1:4, 0] = nan
    x[2:4, -1] = -nan
    x = x.to(TYPES[kind])
    best = torch.sort(x.float().cpu(), dim=1, descending=True, stable=True).indices.to(dev)
    assert best[0, :3].tolist() == [0, 1, 2] and best[2, :3].tolist() == [0, vocab - 1, 1]
    for k in (1, 6, 64):
        top = torch.full((5, k), 99, dtype=torch.int64, device=dev)
        logp = torch.zeros(5, k, device=dev)
        ob.onebit_logprobs_forward(x, None, None, top_ids=top, top_logprobs=logp)
        assert torch.equal(top, best[:, :k]), k
        assert bool(logp.isnan().all())


@pytest.mark.parametrize("vocab", [9, 300, 3000, 30522, 40000, 70000])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_nan_takes_the_whole_row_of_a_gradient(dev, vocab, kind):
    """A NaN or +infinity among a row's logits, or a NaN in what its values are weighted
    with, makes all of its gradient NaN, with the entropy as without, also where p is 0
    (masked or far below the largest).  Other rows with such places have numbers."""
    import paper_2102_02888_amd as ob
    nan = float("nan")
    x = torch.randn(6, vocab, device=dev, generator=_gen(dev, 1))
    x[:, 4], x[:, vocab - 2] = -INF, -500.0
    x[0, 2], x[1, 3] = nan, INF
    x = x.to(TYPES[kind])
    ids = torch.full((6,), 1, device=dev)
    g, h = torch.ones(6, device=dev), torch.ones(6, device=dev)
    g[2], h[3] = nan, nan
    d = torch.empty_like(x)
    ob.onebit_logprobs_grad(x, ids, g, d)
    assert d.isnan().all(1).tolist() == [True] * 3 + [False] * 3
    assert not bool(d[3:].isnan().any())
    for value in (None, torch.empty(6, device=dev)):
        ob.onebit_logprobs_grad(x, ids, g, d, grad_entropy=h, entropy=value)
        assert d.isnan().all(1).tolist() == [True] * 4 + [False] * 2
        assert not bool(d[4:].isnan().any()) and not bool(d[4:, [4, vocab - 2]].any())
