"""The small language model: its worker's gradients against the formula and
differences of its loss, and that both optimizers together learn its tokens."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _loss(model, ids, target, table, mats):
    """The model's loss in 64 bits, plain torch."""
    h = table[ids] * model.scale
    for a, b in zip(mats[::2], mats[1::2]):
        h = h + torch.relu(h @ a) @ b
    h = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6)
    bias = model._bias(model.adam.x).double()
    return torch.nn.functional.cross_entropy(h @ table.t() + bias, target)


def test_worker_gradients(dev):
    """The tied table's gradient is the sum of the output's and the lookup's, in
    the worker's row; the matrices' are in Muon's.  Against the formula in 64
    bits: a few chained fp32 products of up to 128 terms, 1e-5.  Against
    central differences in 64 bits along a direction d (h = 1e-6: no relu
    changes side): the gradient's rounding, 1e-5 of |gradient| |d|."""
    from paper_2102_02888_amd.lm_example import Model
    model = Model(dev, vocab=50, width=32, n_workers=1, tokens=60)
    ids, target = model.batch()
    model.batch = lambda: (ids, target)
    model.worker(0)
    have = [model.adam.grads[0][:50 * 32].view(50, 32)]
    have += [model.mats.view(model.muon.grads[0], k) for k in range(4)]
    x = [model.table.double()] + [m.double() for m in model.matrices]
    leaves = [v.clone().requires_grad_() for v in x]
    want = torch.autograd.grad(_loss(model, ids, target, leaves[0], leaves[1:]), leaves)
    g = torch.Generator(device=dev).manual_seed(5)
    for k in range(5):
        assert float((have[k].double() - want[k]).norm()) < 1e-5 * float(want[k].norm()), k
        d = torch.randn(x[k].shape, dtype=torch.float64, device=dev, generator=g)
        got = []
        for h in (1e-6, -1e-6):
            moved = x[:k] + [x[k] + h * d] + x[k + 1:]
            got.append(float(_loss(model, ids, target, moved[0], moved[1:])))
        along = float((have[k].double() * d).sum())
        bound = 1e-5 * float(have[k].norm()) * float(d.norm())
        assert abs(along - (got[0] - got[1]) / 2e-6) < bound, k


def test_model_learns_its_tokens(dev):
    """A token is followed by one of four: the loss goes from ln 1000 towards ln 4."""
    from paper_2102_02888_amd.lm_example import Model
    model = Model(dev)
    first = float(model.step())
    for _ in range(149):
        last = model.step()
    assert abs(first - math.log(1000)) < 1.0
    assert not model.adam.in_warmup
    assert float(last) < 3.5


def test_updates_do_not_depend_on_which_side_the_rows_are(dev):
    """The layers' matrices, width x 4 width and back, are used as h @ a, with inputs as
    rows.  Orthogonalised updates of both have the same number of singular values
    near 1; the scale must not make the one that leads back the larger."""
    from paper_2102_02888_amd.lm_example import Model
    model = Model(dev)
    old = [m.clone() for m in model.matrices]
    model.step()
    for a, b in zip(range(0, len(old), 2), range(1, len(old), 2)):
        one, two = (float((model.matrices[k] - old[k]).norm()) for k in (a, b))
        assert 0.75 < one / two < 1.33, (one, two)
