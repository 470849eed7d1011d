"""The small language model with attention layers and with a teacher: all its
operators together, its gradients against differences of the same formulas in 64 bits,
and that a step of both runs and changes every parameter."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _attention(qkv, at, heads):
    """Causal attention of packed sequences in plain torch; q, k and v side by side."""
    q, k, v = (t.unflatten(1, (heads, -1)) for t in qkv.split(qkv.shape[1] // 3, 1))
    out = []
    for a, b in zip(at, at[1:]):
        s = (q[a:b].transpose(0, 1) @ k[a:b].permute(1, 2, 0).contiguous()) * q.shape[2] ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, device=s.device).triu(1).bool(), -torch.inf)
        out.append((torch.softmax(s, 2) @ v[a:b].transpose(0, 1).contiguous()).transpose(0, 1))
    return torch.cat(out).flatten(1)


def _logits64(model, ids, table, bias, mats, vectors):
    """model.logits in plain 64-bit torch."""
    h, mats, vectors = table[ids] * model.scale, iter(mats), iter(vectors)

    def norm(h):
        w, b = next(vectors), next(vectors)
        d = h - h.mean(1, keepdim=True)
        return d / torch.sqrt(d.square().mean(1, keepdim=True) + 1e-5) * w + b
    at = model.starts.tolist()
    for qkv in mats:
        h = h + _attention(norm(h) @ qkv, at, model.heads) @ next(mats)
        h = h + torch.relu(norm(h) @ next(mats)) @ next(mats)
    h = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6)
    return h @ table.t() + bias


def _parameters64(model):
    table, bias, mats, vectors = model.parameters()
    return [t.detach().double().clone() for t in (table, bias, *mats, *vectors)]


def _split(model, flat):
    n = len(model.matrices)
    return flat[0], flat[1], flat[2:2 + n], flat[2 + n:]


class _Plain:
    """Attention without bf16, in the operator's place: its roundings move numbers by 2^-8,
    over a relu's corner here and there, where a gradient jumps."""

    @staticmethod
    def apply(qkv, starts, heads, workspace):
        return _attention(qkv, starts.tolist(), heads)


@pytest.mark.parametrize("taught", [False, True])
def test_gradients_of_a_model_with_attention(dev, taught, monkeypatch):
    """Layer norms, losses, vectors and matrices of a whole worker against the formulas in
    64 bits: a chain of some ten fp32 products of up to 128 terms, each off by at most
    128 * 2^-24 = 8e-6 of its terms' magnitudes: 1e-4 of each gradient as a whole."""
    from paper_2102_02888_amd import lm_example
    monkeypatch.setattr(lm_example, "_Attention", _Plain)
    make = lm_example.Model
    teacher = make(dev, vocab=50, width=32, n_workers=1, tokens=60, seed=7) if taught else None
    model = make(dev, vocab=50, width=32, n_workers=1, tokens=60, heads=4, teacher=teacher)
    for k, v in enumerate(model._vectors(model.adam.x)):
        v.add_(torch.randn(32, device=dev, generator=torch.Generator(device=dev).manual_seed(k)) * 0.1)
    ids, target = model.batch()
    model.batch = lambda: (ids, target)
    loss = model.worker(0)
    row = model.adam.grads[0]
    have = [model._table(row), model._bias(row)]
    have += [model.mats.view(model.muon.grads[0], k) for k in range(len(model.matrices))]
    have += model._vectors(row)
    leaves = [t.requires_grad_() for t in _parameters64(model)]
    table, bias, mats, vectors = _split(model, leaves)
    logp = torch.log_softmax(_logits64(model, ids, table, bias, mats, vectors), 1)
    if taught:
        q = torch.softmax(model.best_logprobs.double(), 1)
        want = (q * (q.log() - logp.gather(1, model.best.long()))).sum(1).mean()
    else:
        want = -logp.gather(1, target[:, None]).mean()
    assert abs(float(loss) - float(want.detach())) < 1e-4 * float(want.detach())
    for k, (a, b) in enumerate(zip(have, torch.autograd.grad(want, leaves))):
        assert float((a.double() - b).norm()) < 1e-4 * float(b.norm()), k


def test_attention_of_the_model(dev):
    """The autograd function around the operator, one product's rows in and out.  Operands
    and results are rounded to bf16, a step of 2^-8 at most half of which is lost: q, k,
    v and dout (2^-9 each of themselves), P or dS, and the result, in a sum where q and k
    count twice through the scores (about 1): 8 * 2^-9 = 1.6e-2 of the whole (2-norm)."""
    from paper_2102_02888_amd.attention import attention_workspace
    from paper_2102_02888_amd.lm_example import _Attention
    g = torch.Generator(device=dev).manual_seed(3)
    qkv = torch.randn(90, 3 * 64, device=dev, generator=g).requires_grad_()
    starts = torch.tensor([0, 11, 45, 90], dtype=torch.int32, device=dev)
    dout = torch.randn(90, 64, device=dev, generator=g)
    out = _Attention.apply(qkv, starts, 4, attention_workspace(90, 4, dev))
    have = torch.autograd.grad(out, qkv, dout)[0]
    x = qkv.detach().double().requires_grad_()
    want = _attention(x, starts.tolist(), 4)
    grad = torch.autograd.grad(want, x, dout.double())[0]
    out, want = out.detach(), want.detach()
    assert float((out - want).norm()) < 1.6e-2 * float(want.norm())
    assert float((have - grad).norm()) < 1.6e-2 * float(grad.norm())


@pytest.mark.parametrize("taught", [False, True])
def test_a_step_runs_and_moves_every_parameter(dev, taught):
    from paper_2102_02888_amd.lm_example import Model
    teacher = Model(dev, vocab=300, width=64, n_workers=1, tokens=200, seed=7) if taught else None
    model = Model(dev, vocab=300, width=64, layers=2, n_workers=2, tokens=200, heads=2, teacher=teacher)
    old = [t.clone() for t in _parameters64(model)]
    losses = [float(model.step()) for _ in range(3)]
    assert all(0 < l < 20 for l in losses)
    for a, b in zip(old, _parameters64(model)):
        assert bool(torch.isfinite(b).all()) and not torch.equal(a, b)


def test_second_derivatives_are_refused(dev):
    """The operators' gradients are not differentiated further: what a second derivative
    would need of them is not there, and leaving it out would pass for zero."""
    from paper_2102_02888_amd.attention import attention_workspace
    from paper_2102_02888_amd.lm_example import _Attention, _LayerNorm
    from paper_2102_02888_amd.norm import layer_norm_workspace
    g = torch.Generator(device=dev).manual_seed(3)
    x = torch.randn(20, 3 * 32, device=dev, generator=g).requires_grad_()
    w, b = torch.ones(96, device=dev), torch.zeros(96, device=dev)
    starts = torch.tensor([0, 5, 20], dtype=torch.int32, device=dev)
    for y in (_LayerNorm.apply(x, w, b, layer_norm_workspace(20, 96, dev)),
              _Attention.apply(x, starts, 2, attention_workspace(20, 2, dev)).repeat(1, 3)):
        with pytest.raises(RuntimeError, match="not differentiable twice"):
            first = torch.autograd.grad((x * y).sum(), x, create_graph=True)[0]
            torch.autograd.grad(first.square().sum(), x)
