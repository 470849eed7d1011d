"""Layer norm (onebit_layer_norm_forward, onebit_layer_norm_grad) against plain
64-bit formulas, at sizes and rows where it can go wrong, and its refusals.

Tolerances.  A sum over a row adds at most 16 numbers of a thread, then 6 levels of
a wave and 16 waves: 38 additions deep, so that it is off by at most 40 * 2^-24 =
2.4e-6 of the sum of magnitudes.  A centred value is then off by 2.4e-6 of the row's
deviation and z = d r by 2.4e-6 + 2.4e-6 |z| + a few roundings: 6e-6 (|z| + 1).  The
means of g and g z in the gradient are off by 2.4e-6 of the means of their magnitudes
beside what z is off by: 1e-5 of all terms' magnitudes covers them.  The sums over n
rows add n 2^-24 of their magnitudes in any order.  Then one rounding to the type."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = 2.0 ** -25  # half of fp16's least number

SHAPES = [(1, 1, 0), (3, 2, 1), (1, 1024, 0), (70, 7, 2), (33, 8, 0), (65, 64, 0), (300, 65, 0),
          (9, 256, 0), (50, 257, 3), (17, 512, 0), (4, 513, 0), (1001, 771, 1), (5000, 1024, 0),
          (6, 1025, 0), (11, 2048, 0), (8, 2049, 1), (5, 4096, 0), (5, 4097, 0), (7, 8192, 0),
          (700, 8200, 0), (3, 16384, 0), (20011, 48, 0), (5, 16383, 1)]


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _strided(rows, cols, dtype, dev, extra, seed, std=1.0, mean=0.0):
    """[rows, cols] with `extra` elements between rows, from an odd element on."""
    flat = torch.empty(rows * (cols + extra) + 1, dtype=torch.float32, device=dev)
    flat.normal_(mean, std, generator=_gen(dev, seed))
    return flat.to(dtype)[1:].view(rows, cols + extra)[:, :cols]


def _vector(width, dtype, dev, seed, mean):
    return (torch.randn(width + 1, device=dev, generator=_gen(dev, seed)) * 0.5 + mean).to(dtype)[1:]


def _z(x, eps):
    x = x.double()
    d = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt(d.square().mean(1, keepdim=True) + eps)
    return d * r, r


def _between(t, extra):
    """What lies between the rows of a strided tensor (the last row's is another's)."""
    return t.as_strided((t.shape[0], t.shape[1] + extra), t.stride())[:-1, t.shape[1]:]


@pytest.mark.parametrize("rows,width,extra", SHAPES)
@pytest.mark.parametrize("src,dst,params", [("f32", "bf16", "f32"), ("bf16", "bf16", "f32"),
                                            ("f16", "f16", "f16"), ("bf16", "f32", "bf16"),
                                            ("f32", "f32", None)])
def test_forward(dev, rows, width, extra, src, dst, params):
    import paper_2102_02888_amd as ob
    eps = 1e-5
    x = _strided(rows, width, TYPES[src], dev, extra, 1, 2.0, 0.7)
    y = _strided(rows, width, TYPES[dst], dev, extra, 2)
    rest = _between(y, extra).clone()
    w = b = None
    if params:
        w = _vector(width, TYPES[params], dev, 3, 1.0)
        b = _vector(width, TYPES[params], dev, 4, 0.0)
    ob.onebit_layer_norm_forward(x, y, w, b, eps=eps)
    z, _ = _z(x, eps)
    w64 = 1.0 if w is None else w.double()
    b64 = torch.zeros(width, device=dev, dtype=torch.float64) if b is None else b.double()
    want = z * w64 + b64
    tol = abs(w64) * (z.abs() + 1) * 6e-6 + want.abs() * (ULP[dst] + 2.0 ** -23) + b64.abs() * 2.0 ** -23
    assert bool(((y.double() - want).abs() <= tol + LEAST).all())
    assert torch.equal(_between(y, extra), rest)


def test_rows_far_off_zero_and_constant_rows(dev):
    """A mean 2^20 times the deviation: differences of the given numbers are exact, so
    that the tolerance is that of any row.  A constant row is its bias."""
    import paper_2102_02888_amd as ob
    for width in (100, 1024, 3001):
        x = torch.randn(12, width, device=dev, generator=_gen(dev, 1)) + 2.0 ** 20
        x[5] = 3.25
        x[6] = 0
        y = torch.empty_like(x)
        b = _vector(width, torch.float32, dev, 2, 0.0)
        ob.onebit_layer_norm_forward(x, y, None, b)
        z, _ = _z(x, 1e-5)
        tol = (z.abs() + 1) * 6e-6 + (z + b).abs() * 2.0 ** -23 + b.abs() * 2.0 ** -23
        assert bool(((y.double() - (z + b)).abs() <= tol).all()), width
        assert torch.equal(y[5], b) and torch.equal(y[6], b)


@pytest.mark.parametrize("rows,width,extra", SHAPES)
@pytest.mark.parametrize("dt,src,params,accumulate", [
    ("bf16", "bf16", "f32", False), ("f32", "f32", "f32", True), ("bf16", "f32", "bf16", False),
    ("f16", "f16", "f16", True), ("f32", "bf16", None, False)])
def test_gradient(dev, rows, width, extra, dt, src, params, accumulate):
    import paper_2102_02888_amd as ob
    eps = 1e-5
    x = _strided(rows, width, TYPES[src], dev, extra, 1, 2.0, 0.7)
    dy = _strided(rows, width, TYPES[dt], dev, extra, 2, 0.5)
    dx = _strided(rows, width, TYPES[src], dev, extra, 3)
    rest = _between(dx, extra).clone()
    w = _vector(width, TYPES[params], dev, 4, 1.0) if params else None
    kind = params or "f32"
    dw, db = (_vector(width, TYPES[kind], dev, s, 0.0) for s in (5, 6))
    old = dw.clone(), db.clone()
    # the workspace has what the call needs, and what is behind it stays
    n = ctypes.c_size_t()
    assert ob.lib().onebit_layer_norm_grad_workspace(rows, width, ctypes.byref(n)) == 0
    whole = torch.full((n.value + 4096,), 0xA5, dtype=torch.uint8, device=dev)
    ob.onebit_layer_norm_grad(dy, x, dx, whole[:n.value], w, dw, db, eps=eps,
                              accumulate=accumulate)
    assert bool((whole[n.value:] == 0xA5).all())
    z, r = _z(x, eps)
    d64 = dy.double()
    g = d64 * (1.0 if w is None else w.double())
    mg, mgz = g.mean(1, keepdim=True), (g * z).mean(1, keepdim=True)
    want = r * (g - mg - z * mgz)
    a, b = g.abs().mean(1, keepdim=True), (g * z).abs().mean(1, keepdim=True)
    tol = 1e-5 * r * (g.abs() + a + (z.abs() + 1) * (a + b)) + want.abs() * ULP[src]
    assert bool(((dx.double() - want).abs() <= tol + LEAST).all())
    assert torch.equal(_between(dx, extra), rest)
    for got, was, terms, off in ((dw, old[0], d64 * z, 6e-6 * (d64.abs() * (z.abs() + 1)).sum(0)),
                                 (db, old[1], d64, 0.0)):
        want = terms.sum(0) + (was.double() if accumulate else 0.0)
        tol = terms.abs().sum(0) * (rows + 40) * 2.0 ** -24 + off
        tol = tol + want.abs() * (ULP[kind] + 2.0 ** -24) + was.double().abs() * 2.0 ** -24 + LEAST
        assert bool(((got.double() - want).abs() <= tol).all())
    again = [t.clone() for t in old]
    dx2 = torch.empty_like(dx)
    ob.onebit_layer_norm_grad(dy, x, dx2, whole[:n.value], w, *again, eps=eps,
                              accumulate=accumulate)
    assert torch.equal(dx2, dx) and torch.equal(again[0], dw) and torch.equal(again[1], db)


def test_gradient_parts_left_out_and_no_rows(dev):
    """Any of the three results alone is the same as with the others; without rows the
    sums are zeros, or what they were."""
    import paper_2102_02888_amd as ob
    for width in (40, 1000, 5000):
        x, dy = (torch.randn(37, width, device=dev, generator=_gen(dev, s)) for s in (1, 2))
        w = _vector(width, torch.float32, dev, 3, 1.0)
        work = ob.layer_norm_workspace(37, width, dev)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
        ob.onebit_layer_norm_grad(dy, x, dx, work, w, dw, db)
        one, two, three = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
        ob.onebit_layer_norm_grad(dy, x, one, None, w)
        ob.onebit_layer_norm_grad(dy, x, None, work, w, two)
        ob.onebit_layer_norm_grad(dy, x, None, work, w, None, three)
        assert torch.equal(dx, one) and torch.equal(dw, two) and torch.equal(db, three)
        ob.onebit_layer_norm_grad(dy[:0], x[:0], one[:0], work, w, two, three, accumulate=True)
        assert torch.equal(dw, two) and torch.equal(db, three)
        ob.onebit_layer_norm_grad(dy[:0], x[:0], one[:0], work, w, two, three)
        assert not bool(two.any()) and not bool(three.any())


def test_nan_and_infinity_stay_in_their_rows(dev):
    import paper_2102_02888_amd as ob
    for width in (50, 1024, 6000):
        x, dy = (torch.randn(9, width, device=dev, generator=_gen(dev, s)) for s in (1, 2))
        y, dx = torch.empty_like(x), torch.empty_like(x)
        work = ob.layer_norm_workspace(9, width, dev)
        x[2, 1], x[4, 3], dy[6, 5] = float("nan"), float("inf"), float("nan")
        ob.onebit_layer_norm_forward(x, y)
        assert y.isnan().all(1).tolist() == [k in (2, 4) for k in range(9)]
        assert y.isnan().any(1).tolist() == [k in (2, 4) for k in range(9)]
        ob.onebit_layer_norm_grad(dy, x, dx, work)
        assert dx.isnan().any(1).tolist() == [k in (2, 4, 6) for k in range(9)]


def test_gradient_against_differences(dev):
    """sum(dy y) moved along random directions of x, w and b, central differences of
    the 64-bit formula, h = 1e-6: 1e-5 of |gradient| |direction|, the gradient's own
    tolerance."""
    import paper_2102_02888_amd as ob
    x, dy, w, b = (torch.randn(s, device=dev, generator=_gen(dev, k))
                   for k, s in enumerate(((13, 90), (13, 90), (90,), (90,))))
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ob.onebit_layer_norm_grad(dy, x, dx, ob.layer_norm_workspace(13, 90, dev), w, dw, db)

    def value(x, w, b):
        return float(((_z(x, 1e-5)[0] * w + b) * dy.double()).sum())
    at = [t.double() for t in (x, w, b)]
    for k, grad in enumerate((dx, dw, db)):
        d = torch.randn(grad.shape, dtype=torch.float64, device=dev, generator=_gen(dev, 9 + k))
        got = [value(*at[:k], at[k] + h * d, *at[k + 1:]) for h in (1e-6, -1e-6)]
        along = float((grad.double() * d).sum())
        assert abs(along - (got[0] - got[1]) / 2e-6) < 1e-5 * float(grad.norm()) * float(d.norm())


def test_views_into_the_flat_buffers_streams_and_graph(dev):
    """Weight, bias and their gradients inside State's buffers; another stream; a graph
    replayed on new numbers against the eager result."""
    import paper_2102_02888_amd as ob
    width, rows = 96, 3000
    plan = ob.Plan([7, width, width], 1)
    st = ob.State(plan, dev)
    st.x.normal_(0, 1, generator=_gen(dev, 1))
    at = [int(o) for o in plan.tensor_off[1:3]]
    w, b = (st.x[o:o + width] for o in at)
    dw, db = (st.grads[0][o:o + width] for o in at)
    st.grads.fill_(7.0)
    x, dy = (torch.randn(3, rows // 3, width, device=dev, generator=_gen(dev, s)) for s in (2, 3))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    work = ob.layer_norm_workspace(rows, width, dev)

    def calls(stream=None):
        ob.onebit_layer_norm_forward(x, y, w, b, stream=stream)
        ob.onebit_layer_norm_grad(dy, x, dx, work, w, dw, db, stream=stream)
    calls()
    want = [t.clone() for t in (y, dx, dw, db)]
    assert float(st.grads[0][0]) == 7.0
    side = torch.cuda.Stream()
    for t in (y, dx, dw, db):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(want, (y, dx, dw, db)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (4, 5, 6):
        x.copy_(torch.randn(x.shape, device=dev, generator=_gen(dev, seed)))
        calls()
        want = [t.clone() for t in (y, dx, dw, db)]
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, c) for a, c in zip(want, (y, dx, dw, db))), seed
    plan.close()


def test_rows_past_32_bits(dev):
    """2^31 and more elements: the last rows at their places."""
    import paper_2102_02888_amd as ob
    rows, width = 140000, 16384
    x = torch.empty(rows, width, dtype=torch.bfloat16, device=dev)
    x[:] = torch.randn(width, device=dev, generator=_gen(dev, 1)).bfloat16()
    y = torch.empty_like(x)
    ob.onebit_layer_norm_forward(x, y)
    one = torch.empty_like(x[:1])
    ob.onebit_layer_norm_forward(x[:1], one)
    assert bool((y == one).all())
    dw = torch.empty(width, device=dev)
    work = ob.layer_norm_workspace(rows, width, dev)
    ob.onebit_layer_norm_grad(y, x, y, work, None, dw)  # dx over dy: a row is read before
    ob.onebit_layer_norm_grad(one, x[:1], one, work, None, None)
    assert bool((y == one).all())


def test_refusals(dev):
    import paper_2102_02888_amd as ob
    x, w = torch.zeros(5, 8, device=dev), torch.zeros(8, device=dev)
    work = ob.layer_norm_workspace(5, 8, dev)
    fwd, bwd = ob.onebit_layer_norm_forward, ob.onebit_layer_norm_grad
    with pytest.raises(TypeError, match="x must"):
        fwd(x.double(), x)
    with pytest.raises(ValueError, match="y is"):
        fwd(x, x[:4])
    with pytest.raises(ValueError, match="weight must be 1-D"):
        fwd(x, x, w[:7])
    with pytest.raises(ValueError, match="bias must be 1-D"):
        fwd(x, x, w, torch.zeros(16, device=dev)[::2])
    with pytest.raises(TypeError, match="one type"):
        fwd(x, x, w, w.bfloat16())
    with pytest.raises(ValueError, match="GPU tensor"):
        fwd(x, x, w.cpu())
    with pytest.raises(ValueError, match="unit stride"):
        fwd(torch.zeros(8, 5, device=dev).t(), x)
    with pytest.raises(ob.OnebitError, match="eps"):
        fwd(x, x, eps=-1.0)
    with pytest.raises(ob.OnebitError, match="eps"):
        fwd(x, x, eps=float("nan"))
    with pytest.raises(ob.OnebitError, match="width"):
        fwd(torch.zeros(1, 16385, device=dev), torch.zeros(1, 16385, device=dev))
    with pytest.raises(TypeError, match="grad_x must be of x's type"):
        bwd(x, x, x.bfloat16(), work)
    with pytest.raises(ValueError, match="workspace has"):
        bwd(x, x, x, work[:64], w, w)
    with pytest.raises(TypeError, match="workspace"):
        bwd(x, x, x, None, w, w)


@pytest.mark.parametrize("width", [40, 100, 400, 1000, 3001, 8000, 16384])
def test_deviations_whose_squares_leave_fp32(dev, width):
    """Rows of numbers up to 1e30 have squares past fp32's range, and a norm like any
    other: the tolerance is that of any row.  One far off zero beside them, and an
    ordinary one.  A row whose sum leaves fp32's range is NaN."""
    import paper_2102_02888_amd as ob
    x, dy = (torch.randn(6, width, device=dev, generator=_gen(dev, s)) for s in (1, 2))
    x *= torch.tensor([1e17, 3e19, 1e25, 1e30, 1.0, 1.0], device=dev)[:, None]
    x[2] += 1e30
    x[5] = 3e38
    y, dx, w = torch.empty_like(x), torch.empty_like(x), _vector(width, torch.float32, dev, 3, 1.0)
    ob.onebit_layer_norm_forward(x, y, w)
    z, r = _z(x[:5], 1e-5)
    w64 = w.double()
    tol = w64.abs() * (z.abs() + 1) * 6e-6 + (z * w64).abs() * 2.0 ** -22
    assert bool(((y[:5].double() - z * w64).abs() <= tol).all())
    assert bool(y[5].isnan().all())
    dw = torch.empty_like(w)
    ob.onebit_layer_norm_grad(dy[:5], x[:5], dx[:5], ob.layer_norm_workspace(5, width, dev), w, dw)
    g = dy[:5].double() * w64
    mg, mgz = g.mean(1, keepdim=True), (g * z).mean(1, keepdim=True)
    want = r * (g - mg - z * mgz)
    a, b = g.abs().mean(1, keepdim=True), (g * z).abs().mean(1, keepdim=True)
    tol = 1e-5 * r * (g.abs() + a + (z.abs() + 1) * (a + b)) + want.abs() * 2.0 ** -24
    assert bool(((dx[:5].double() - want).abs() <= tol + 2.0 ** -148).all())
    terms = dy[:5].double() * z
    tol = terms.abs().sum(0) * 45 * 2.0 ** -24 + 6e-6 * (dy[:5].double().abs() * (z.abs() + 1)).sum(0)
    assert bool(((dw.double() - terms.sum(0)).abs() <= tol).all())
