"""Orthogonalised updates (onebit_orthogonalize, onebit_muon_step) against the
formulas in 64 bits, at shapes, strides and values where they can go wrong,
and their refusals.

Tolerances (2-norm of the difference over the 2-norm of the result).
PRODUCTS_F32: operands and sums carry 2^-24 each; five steps raise a small
singular value up to 480 times, and with it the noise of every rounding before,
which an ill-conditioned matrix shows most: 1e-5 for matrices of ordinary noise,
1e-4 for a rank-16 matrix with 1e-3 of noise (an fp32 computation's own figure
there is 2e-5).  PRODUCTS_F16: operands carry 2^-12 (3e-4 as a whole over three
products and five steps, the last of which count): 3e-3.  An output type adds
its unit roundoff, 2^-8 or 2^-11 of every element."""
import ctypes
import math

import pytest
import torch

from matrix_lists import KERNEL_LISTS

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
ABC = (3.4445, -4.7750, 2.0315)


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _values(dev, r, c, kind, seed):
    g = _gen(dev, seed)
    u = torch.randn(r, c, device=dev, generator=g) * 1e-3
    if kind == "rank16":
        k = min(16, r, c)
        u = torch.randn(r, k, device=dev, generator=g) @ torch.randn(k, c, device=dev, generator=g)
        u = u * 1e-3 + torch.randn(r, c, device=dev, generator=g) * 1e-6 * 4
    elif kind == "sparse":
        u *= torch.rand(r, c, device=dev, generator=g) < 0.02
    elif kind == "one":
        u.zero_()
        u[r // 2, c // 2] = -3.0
    elif kind == "huge":
        u *= 1e33
    elif kind == "tiny":
        u *= 1e-30
    return u


def _ortho64(u, steps=5, eps=1e-7, abc=ABC):
    a, b, c = abc
    x = u.double()
    flip = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if flip else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if flip else x


def _rel(got, want):
    d = float((got.double() - want).norm())
    n = float(want.norm())
    return d / n if n else d


def _fill(mats, flat, values):
    for k, v in enumerate(values):
        mats.view(flat, k).copy_(v)


SHAPES = [(1, 1), (1, 64), (64, 1), (3, 500), (500, 3), (17, 17), (63, 65), (128, 128), (129, 127),
          (130, 384), (300, 1000), (1000, 257), (512, 512)]


@pytest.mark.parametrize("products,out", [("f32", "f32"), ("f32", "f16"), ("f32", "bf16"),
                                          ("f16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("src", ["f32", "bf16", "f16"])
def test_orthogonalize_shapes(dev, products, out, src):
    """One call over matrices of every shape; what lies between them stays."""
    import paper_2102_02888_amd as ob
    mats = ob.Matrices(SHAPES)
    prod = ob.PRODUCTS_F32 if products == "f32" else ob.PRODUCTS_F16
    grad = torch.full((mats.extent + 5,), float("nan"), dtype=TYPES[src], device=dev)
    _fill(mats, grad, [_values(dev, r, c, "noise", 10 + k) for k, (r, c) in enumerate(SHAPES)])
    res = torch.full((mats.extent + 5,), 7.0, dtype=TYPES[out], device=dev)
    work = mats.workspace(dev, prod)
    work.fill_(255)  # NaN in every type: nothing may be read before it is written
    ob.onebit_orthogonalize(mats, grad, res, work, products=prod)
    tol = (1e-5 if products == "f32" else 3e-3) + ROUND[out]
    between = torch.ones_like(res, dtype=torch.bool)
    for k in range(len(SHAPES)):
        got, want = mats.view(res, k), _ortho64(mats.view(grad, k))
        assert _rel(got, want) < tol, (SHAPES[k], _rel(got, want))
        mats.view(between, k).fill_(False)
    assert bool((res[between] == 7.0).all())
    again = torch.full_like(res, 7.0)
    ob.onebit_orthogonalize(mats, grad, again, work, products=prod)
    assert torch.equal(again, res)  # bit for bit
    mats.close()


@pytest.mark.parametrize("kind,tol32,tol16", [("noise", 1e-5, 3e-3), ("rank16", 1e-4, 5e-3),
                                              ("sparse", 1e-5, 3e-3), ("one", 1e-5, 3e-3),
                                              ("huge", 1e-5, 3e-3), ("tiny", 1e-5, 3e-3)])
def test_orthogonalize_values(dev, kind, tol32, tol16):
    import paper_2102_02888_amd as ob
    shapes = [(256, 256), (200, 700), (700, 200)]
    mats = ob.Matrices(shapes)
    grad, res = torch.zeros(mats.extent, device=dev), torch.zeros(mats.extent, device=dev)
    _fill(mats, grad, [_values(dev, r, c, kind, 50 + k) for k, (r, c) in enumerate(shapes)])
    for prod, tol in ((ob.PRODUCTS_F32, tol32), (ob.PRODUCTS_F16, tol16)):
        ob.onebit_orthogonalize(mats, grad, res, mats.workspace(dev, prod), products=prod)
        for k in range(3):
            eps = 1e-7
            assert _rel(mats.view(res, k), _ortho64(mats.view(grad, k), eps=eps)) < tol, k
    mats.close()


@pytest.mark.parametrize("steps,abc", [(1, None), (2, (1.5, -0.5, 0.0)), (10, (1.5, -0.5, 0.0)),
                                       (6, (2.0, -1.5, 0.5))])
def test_steps_and_coefficients(dev, steps, abc):
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(100, 160)])
    grad, res = torch.zeros(mats.extent, device=dev), torch.zeros(mats.extent, device=dev)
    _fill(mats, grad, [_values(dev, 100, 160, "noise", 1)])
    ob.onebit_orthogonalize(mats, grad, res, mats.workspace(dev), steps=steps, coefficients=abc)
    assert _rel(mats.view(res, 0), _ortho64(mats.view(grad, 0), steps, abc=abc or ABC)) < 1e-5
    mats.close()


def test_result_is_nearly_orthogonal(dev):
    """Five default steps put singular values of ordinary noise near 1."""
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(200, 600)])
    grad, res = torch.zeros(mats.extent, device=dev), torch.zeros(mats.extent, device=dev)
    _fill(mats, grad, [_values(dev, 200, 600, "noise", 1)])
    ob.onebit_orthogonalize(mats, grad, res, mats.workspace(dev))
    s = torch.linalg.svdvals(mats.view(res, 0).double().cpu())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25
    mats.close()


def test_zero_nan_and_infinite_matrices_stay_apart(dev):
    """A zero matrix gives zeros, one NaN or infinity makes its own matrix NaN,
    and its neighbours are as without it."""
    import paper_2102_02888_amd as ob
    shapes = [(100, 140), (100, 140), (100, 140), (140, 100), (0, 5), (100, 140)]
    mats = ob.Matrices(shapes)
    grad, res = torch.zeros(mats.extent, device=dev), torch.zeros(mats.extent, device=dev)
    for k in (0, 2, 3, 5):
        mats.view(grad, k).copy_(_values(dev, *shapes[k], "noise", k))
    mats.view(grad, 2)[3, 4] = float("nan")
    mats.view(grad, 3)[5, 6] = float("inf")
    for prod in (ob.PRODUCTS_F32, ob.PRODUCTS_F16):
        ob.onebit_orthogonalize(mats, grad, res, mats.workspace(dev, prod), products=prod)
        assert not bool(mats.view(res, 1).any())
        assert bool(mats.view(res, 2).isnan().all()) and bool(mats.view(res, 3).isnan().all())
        for k in (0, 5):
            assert _rel(mats.view(res, k), _ortho64(mats.view(grad, k))) < 3e-3
    mats.close()


def test_strided_matrices_in_place(dev):
    """Matrices that are column ranges of wider ones, in an order of their own,
    orthogonalised in place; the columns beside them stay."""
    import paper_2102_02888_amd as ob
    wide = torch.randn(150, 333, device=dev, generator=_gen(dev, 1))
    kept = wide.clone()
    mats = ob.Matrices([(150, 100), (150, 33), (150, 200)], offsets=[233, 0, 33], lds=[333] * 3)
    assert mats.extent == 150 * 333
    flat = wide.view(-1)
    ob.onebit_orthogonalize(mats, flat, flat, mats.workspace(dev))
    for a, b in ((233, 333), (0, 33), (33, 233)):
        assert _rel(wide[:, a:b], _ortho64(kept[:, a:b])) < 1e-5
    half = kept[:, :233].bfloat16().contiguous()
    mats2 = ob.Matrices([(150, 100)], offsets=[7], lds=[233])
    out = torch.zeros_like(half)
    ob.onebit_orthogonalize(mats2, half, out, mats2.workspace(dev, ob.PRODUCTS_F16))
    assert _rel(out[:, 7:107], _ortho64(half[:, 7:107])) < 5e-3
    assert not bool(out[:, :7].any()) and not bool(out[:, 107:].any())
    mats.close()
    mats2.close()


def _muon64(x, m, grads, lr, mu, nesterov, wd, scale):
    g = torch.zeros_like(x, dtype=torch.float64)
    for row in grads:
        g += row.double()
    g /= len(grads)
    m = mu * m.double() + g
    u = g + mu * m if nesterov else m
    r, c = x.shape
    s = {0: 1.0, 1: math.sqrt(max(1.0, r / c)), 2: 0.2 * math.sqrt(max(r, c))}[scale]
    return (1 - lr * wd) * x.double() - lr * s * _ortho64(u), m


@pytest.mark.parametrize("n,grad,nesterov,wd,scale", [
    (1, "f32", True, 0.0, 0), (1, "bf16", True, 0.1, 1), (4, "f32", False, 0.0, 2),
    (3, "f16", True, 0.01, 2), (8, "bf16", False, 0.0, 1)])
def test_muon_step(dev, n, grad, nesterov, wd, scale):
    """Two steps; m to fp32 rounding, x to the update's 1e-5."""
    import paper_2102_02888_amd as ob
    shapes = [(65, 63), (100, 300), (300, 100), (1, 20), (256, 128)]
    mats = ob.Matrices(shapes)
    opt = ob.Muon(mats, dev, lr=0.02, momentum=0.9, nesterov=nesterov, weight_decay=wd, scale=scale,
                  n_workers=n, grad_dtype=TYPES[grad])
    opt.x.normal_(0, 0.02, generator=_gen(dev, 1))
    x = [mats.view(opt.x, k).double() for k in range(len(shapes))]
    m = [torch.zeros_like(v) for v in x]
    for step in range(2):
        for i in range(n):
            for k, (r, c) in enumerate(shapes):
                mats.view(opt.grads[i], k).copy_(_values(dev, r, c, "noise", 100 * step + 10 * i + k))
        opt.step()
        for k in range(len(shapes)):
            rows = [mats.view(opt.grads[i], k) for i in range(n)]
            old = x[k]
            x[k], m[k] = _muon64(x[k], m[k], rows, 0.02, 0.9, nesterov, wd, scale)
            assert _rel(mats.view(opt.m, k), m[k]) < 3 * 2.0 ** -23
            move = float((x[k] - old).norm())
            far = float((mats.view(opt.x, k).double() - x[k]).norm())
            assert far < (step + 1) * (1e-5 * move + 2.0 ** -22 * float(x[k].norm())), (k, far, move)
    mats.close()


def test_muon_state_dict_and_streams(dev):
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(70, 90), (90, 70)])
    one, two = (ob.Muon(mats, dev, lr=0.01) for _ in range(2))
    one.x.normal_(0, 0.02, generator=_gen(dev, 1))
    one.grads.normal_(0, 1e-3, generator=_gen(dev, 2))
    one.step()
    two.load_state_dict(one.state_dict())
    two.grads.copy_(one.grads)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    one.step()
    two.step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(one.x, two.x) and torch.equal(one.m, two.m)
    mats.close()


def test_muon_step_in_a_graph(dev):
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(70, 290), (290, 70), (130, 130)])
    eager, replayed = (ob.Muon(mats, dev, lr=0.01) for _ in range(2))
    eager.x.normal_(0, 0.02, generator=_gen(dev, 1))
    replayed.x.copy_(eager.x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.step()
    for seed in range(4):
        eager.grads.normal_(0, 1e-3, generator=_gen(dev, 10 + seed))
        replayed.grads.copy_(eager.grads)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(eager.x, replayed.x) and torch.equal(eager.m, replayed.m), seed
    mats.close()


def test_refusals(dev):
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(10, 20)])
    f = dict(device=dev)
    g, o, w = torch.zeros(200, **f), torch.zeros(200, **f), mats.workspace(dev)
    with pytest.raises(TypeError, match="grad"):
        ob.onebit_orthogonalize(mats, g.double(), o, w)
    with pytest.raises(ValueError, match="grad has 199"):
        ob.onebit_orthogonalize(mats, g[:199], o, w)
    with pytest.raises(ValueError, match="GPU"):
        ob.onebit_orthogonalize(mats, g.cpu(), o, w)
    with pytest.raises(ValueError, match="contiguous"):
        ob.onebit_orthogonalize(mats, torch.zeros(400, **f)[::2], o, w)
    with pytest.raises(ValueError, match="workspace has"):
        ob.onebit_orthogonalize(mats, g, o, w[:64])
    with pytest.raises(ValueError, match="products"):
        ob.onebit_orthogonalize(mats, g, o, w, products=2)
    for bad in (dict(steps=0), dict(steps=65), dict(eps=0.0), dict(eps=float("nan")),
                dict(coefficients=(3.4445, -4.7750, 9.0)), dict(coefficients=(9.0, 0.0, 0.0)),
                dict(coefficients=(float("nan"), 0.0, 0.0))):
        with pytest.raises(ob.OnebitError):
            ob.onebit_orthogonalize(mats, g, o, w, **bad)
    with pytest.raises(ob.OnebitError, match="different types"):
        b = g.bfloat16()
        L = ob.lib()
        st = L.onebit_orthogonalize(mats.handle, b.data_ptr(), 1, b.data_ptr(), 0, 0, 5, None, 1e-7,
                                    w.data_ptr(), None)
        raise ob.OnebitError("onebit_orthogonalize", st)
    with pytest.raises(TypeError, match="x must be"):
        ob.onebit_muon_step(mats, g.bfloat16(), o, g, 0.1, 0.9, w)
    with pytest.raises(ValueError, match="grads is"):
        ob.onebit_muon_step(mats, g, o, torch.zeros(2, 150, **f), 0.1, 0.9, w)
    with pytest.raises(ob.OnebitError, match="scale"):
        ob.onebit_muon_step(mats, g, o, g.clone(), 0.1, 0.9, w, scale=3)
    mats.close()
    with pytest.raises(ValueError, match="closed"):
        ob.onebit_orthogonalize(mats, g, o, w)


@pytest.mark.parametrize("shapes", [
    [(17, 9000)],                                  # one tile row, the Gram sum in many parts
    [(5, 4000), (64, 2100), (130, 2000)] * 2,      # parts of several tiles
    [(700, 900), (900, 650)] * 8,                  # tiles of 128
    [(1025, 1100)] * 30 + [(1500, 520)] * 30,      # tiles of 256
    [(90, 200)] * 300,                             # tiles of 64 by two groups of waves
])
def test_every_kernel_shape(dev, shapes):
    """Lists that take each of the products' kernels, twice on one workspace
    (the parts' counters are left as a call finds them); some matrices against
    the formula."""
    import paper_2102_02888_amd as ob
    mats = ob.Matrices(shapes)
    grad, res = torch.empty(mats.extent, device=dev), torch.zeros(mats.extent, device=dev)
    grad.normal_(0, 1e-3, generator=_gen(dev, 1))
    for prod, tol in ((ob.PRODUCTS_F32, 1e-5), (ob.PRODUCTS_F16, 3e-3)):
        work = mats.workspace(dev, prod)
        work.fill_(255)
        ob.onebit_orthogonalize(mats, grad, res, work, products=prod)
        first = res.clone()
        for _ in range(3):
            ob.onebit_orthogonalize(mats, grad, res, work, products=prod)
            assert torch.equal(first, res)  # bit for bit, whichever part ends last
        for k in sorted({0, 1 % len(shapes), len(shapes) // 2, len(shapes) - 1}):
            assert _rel(mats.view(res, k), _ortho64(mats.view(grad, k))) < tol, (k, shapes[k])
    mats.close()


def test_parts_in_a_graph(dev):
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(17, 6000), (40, 3000)])
    grad = torch.empty(mats.extent, device=dev)
    res, want = torch.zeros_like(grad), torch.zeros_like(grad)
    work = mats.workspace(dev)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.onebit_orthogonalize(mats, grad, res, work)
    for seed in range(4):
        grad.normal_(0, 1e-3, generator=_gen(dev, seed))
        ob.onebit_orthogonalize(mats, grad, want, work)
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(res, want), seed
    mats.close()


def test_offsets_past_32_bits(dev):
    """A matrix that begins beyond 2^31 elements and 2^32 bytes of its buffers."""
    import paper_2102_02888_amd as ob
    at = (1 << 31) + 192
    mats = ob.Matrices([(70, 100), (100, 70)], offsets=[at, 5])
    grad = torch.zeros(mats.extent, dtype=torch.bfloat16, device=dev)
    res = torch.zeros(mats.extent, dtype=torch.bfloat16, device=dev)
    for k in range(2):
        mats.view(grad, k).copy_(_values(dev, *mats.shapes[k], "noise", k))
    ob.onebit_orthogonalize(mats, grad, res, mats.workspace(dev, ob.PRODUCTS_F16))
    for k in range(2):
        assert _rel(mats.view(res, k), _ortho64(mats.view(grad, k))) < 3e-3 + ROUND["bf16"]
    assert not bool(res[5 + 7000:at].any())
    mats.close()


def test_creation_refusals(dev):
    import paper_2102_02888_amd as ob
    for bad, text in ((dict(shapes=[(3, -1)]), "side"), (dict(shapes=[(1 << 21, 1)]), "side"),
                      (dict(shapes=[(1 << 16, 1 << 16)]), "2\\^31"),
                      (dict(shapes=[(4, 5)], lds=[4]), "ld"),
                      (dict(shapes=[(4, 5)], offsets=[-1]), "offset"),
                      (dict(shapes=[(4, 5)], offsets=[1 << 41]), "offset"),
                      (dict(shapes=[(1 << 20, 1)], lds=[1 << 40]), "ends above")):
        with pytest.raises(ob.OnebitError, match=text):
            ob.Matrices(**bad)
    with pytest.raises(ValueError, match="one entry per matrix"):
        ob.Matrices([(4, 5)], offsets=[0, 1])
    mats = ob.Matrices([(0, 4), (7, 0)])  # nothing to do, nothing needed
    x = torch.zeros(0, device=dev)
    ob.onebit_orthogonalize(mats, x, x, mats.workspace(dev))
    mats.close()


@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_default_products_are_those_of_fp32(dev, out):
    """A call that names no products takes PRODUCTS_F32 for every output type: it is
    off by that type's rounding alone.  One workspace serves both kinds."""
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(200, 300), (70, 64)])
    grad = torch.empty(mats.extent, device=dev).normal_(0, 1e-3, generator=_gen(dev, 3))
    work = mats.workspace(dev, ob.PRODUCTS_F16)
    got = {}
    for products in (None, ob.PRODUCTS_F32, ob.PRODUCTS_F16):
        got[products] = torch.zeros(mats.extent, dtype=TYPES[out], device=dev)
        ob.onebit_orthogonalize(mats, grad, got[products], work, products=products)
    assert torch.equal(got[None], got[ob.PRODUCTS_F32])
    assert not torch.equal(got[None], got[ob.PRODUCTS_F16])
    mats.close()


@pytest.mark.parametrize("name", list(KERNEL_LISTS))
@pytest.mark.parametrize("products,tol", [("f32", 1e-5), ("f16", 3e-3)])
def test_orthogonalize_by_every_kernel(dev, name, products, tol):
    """The kernels that the list is meant for are those that its call takes; every
    matrix against the formula; bit for bit the same in every call; nothing between
    the matrices is written."""
    import paper_2102_02888_amd as ob
    shapes, pairs, halves = KERNEL_LISTS[name]
    prod = ob.PRODUCTS_F32 if products == "f32" else ob.PRODUCTS_F16
    assert ob.matrices_kernels(shapes, prod) == (pairs if products == "f32" else halves)
    mats = ob.Matrices(shapes)
    grad = torch.empty(mats.extent, device=dev).normal_(0, 1e-3, generator=_gen(dev, 1))
    res = torch.full((mats.extent,), 7.0, device=dev)
    work = mats.workspace(dev, prod)
    work.fill_(255)
    ob.onebit_orthogonalize(mats, grad, res, work, products=prod)
    for k in range(len(shapes)):
        assert _rel(mats.view(res, k), _ortho64(mats.view(grad, k))) < tol, (k, shapes[k])
    between = torch.ones_like(res, dtype=torch.bool)
    for k in range(len(shapes)):
        mats.view(between, k).fill_(False)
    assert bool((res[between] == 7.0).all())
    again = torch.full_like(res, 7.0)
    for _ in range(4):
        ob.onebit_orthogonalize(mats, grad, again, work, products=prod)
        assert torch.equal(again, res)
    mats.close()


@pytest.mark.parametrize("name", list(KERNEL_LISTS))
@pytest.mark.parametrize("products,tol,n,grad", [("f32", 1e-5, 1, "bf16"), ("f32", 1e-5, 3, "f32"),
                                                 ("f16", 3e-3, 2, "bf16")])
def test_muon_step_by_every_kernel(dev, name, products, tol, n, grad):
    """One step from a momentum that is not zero; tolerances as for one step of
    test_muon_step, with the products' own."""
    import paper_2102_02888_amd as ob
    shapes = KERNEL_LISTS[name][0]
    mats = ob.Matrices(shapes)
    opt = ob.Muon(mats, dev, lr=0.02, momentum=0.9, weight_decay=0.1, scale=ob.MUON_SCALE_RMS,
                  n_workers=n, grad_dtype=TYPES[grad],
                  products=ob.PRODUCTS_F32 if products == "f32" else ob.PRODUCTS_F16)
    opt.x.normal_(0, 0.02, generator=_gen(dev, 1))
    opt.m.normal_(0, 2e-3, generator=_gen(dev, 2))
    for i in range(n):
        opt.grads[i].normal_(0, 1e-3, generator=_gen(dev, 3 + i))
    x, m = opt.x.clone(), opt.m.clone()
    opt.step()
    for k in range(len(shapes)):
        old = mats.view(x, k).double()
        want_x, want_m = _muon64(old, mats.view(m, k), [mats.view(g, k) for g in opt.grads], 0.02,
                                 0.9, True, 0.1, ob.MUON_SCALE_RMS)
        assert _rel(mats.view(opt.m, k), want_m) < 3 * 2.0 ** -23
        move = float((want_x - old).norm())
        far = float((mats.view(opt.x, k).double() - want_x).norm())
        assert far < tol * move + 2.0 ** -22 * float(want_x.norm()), (k, far, move)
    mats.close()


@pytest.mark.parametrize("kind", ["noise", "tiny"])
def test_coefficients_up_to_the_stated_bound(dev, kind):
    """|b| + 0.75 |c| is 7.4 in one call and 7.6 in the other, which is refused; all
    other bounds hold.  A singular value grows up to 4^5 = 1,024 times instead of
    480: twice the tolerance of the default's."""
    import paper_2102_02888_amd as ob
    mats = ob.Matrices([(100, 160)])
    grad, res = torch.zeros(mats.extent, device=dev), torch.zeros(mats.extent, device=dev)
    _fill(mats, grad, [_values(dev, 100, 160, kind, 1)])
    work = mats.workspace(dev)
    abc = (4.0, -5.9, 2.0)
    ob.onebit_orthogonalize(mats, grad, res, work, coefficients=abc)
    assert _rel(mats.view(res, 0), _ortho64(mats.view(grad, 0), abc=abc)) < 2e-5
    with pytest.raises(ob.OnebitError, match="leave the range"):
        ob.onebit_orthogonalize(mats, grad, res, work, coefficients=(4.0, -6.1, 2.0))
    mats.close()
