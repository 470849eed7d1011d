"""Token embedding (onebit_embedding_forward, onebit_embedding_grad) against
plain 64-bit formulas, at sizes and ids where it can go wrong, and its
refusals.

Tolerances.  Forward: one fp32 product and one rounding, compared exactly with
the same two roundings.  Gradient: n products' fp32 sum is off by at most
n 2^-24 of the sum of magnitudes in any order; then one product with the scale,
one addition and one rounding to the type."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _ids(dev, kind, tokens, vocab, seed, dtype=torch.int64):
    g = _gen(dev, seed)
    if kind == "one":
        ids = torch.full((tokens,), vocab // 2, device=dev)
    elif kind == "distinct":
        ids = torch.randperm(max(tokens, vocab), device=dev, generator=g)[:tokens] % max(vocab, 1)
    elif kind == "masked":
        ids = torch.full((tokens,), -1, device=dev)
    else:
        u = torch.rand(tokens, dtype=torch.float64, device=dev, generator=g)
        ids = (torch.exp(u * torch.log(torch.tensor(vocab + 1.0, dtype=torch.float64))) - 1).long()
        ids.clamp_(0, vocab - 1)
        if kind == "mixed":  # masked places and ids outside the table on both sides
            r = torch.rand(tokens, device=dev, generator=g)
            ids[r < 0.2] = -1
            ids[(r >= 0.2) & (r < 0.25)] = vocab
            ids[(r >= 0.25) & (r < 0.3)] = -(1 << 31)
            if dtype == torch.int64:
                ids[(r >= 0.3) & (r < 0.35)] = (1 << 32) + 1
    return ids.to(dtype)


def _strided(rows, cols, dtype, dev, extra, seed, std=1.0):
    """[rows, cols] with `extra` elements between rows, from an odd element on."""
    flat = torch.empty(rows * (cols + extra) + 1, dtype=dtype, device=dev)
    flat.normal_(0.0, std, generator=_gen(dev, seed))
    return flat[1:].view(rows, cols + extra)[:, :cols]


@pytest.mark.parametrize("tokens,vocab,width,extra,kind", [
    (1, 1, 1, 0, "zipf"), (1, 100, 64, 0, "zipf"), (7, 5, 3, 2, "mixed"), (513, 300, 8, 0, "zipf"),
    (1000, 30522, 771, 1, "mixed"), (4097, 17, 1024, 0, "mixed"), (33, 40, 2049, 7, "distinct"),
    (50, 10, 16, 0, "masked"),
])
@pytest.mark.parametrize("src,dst", [("f32", "bf16"), ("bf16", "f32"), ("f16", "f16"),
                                     ("f32", "f32"), ("bf16", "f16")])
def test_forward(dev, tokens, vocab, width, extra, kind, src, dst):
    import paper_2102_02888_amd as ob
    table = _strided(vocab, width, TYPES[src], dev, extra, 1)
    for idt in (torch.int32, torch.int64):
        ids = _ids(dev, kind, tokens, vocab, 2, idt)
        out = _strided(tokens, width, TYPES[dst], dev, extra, 3)
        whole = out.as_strided((tokens, width + extra), (width + extra, 1))
        rest = whole[:, width:].clone() if extra else None
        ob.onebit_embedding_forward(table, ids, out, scale=1.7)
        on = (ids >= 0) & (ids < vocab)
        want = table[torch.where(on, ids, 0).long()].float() * torch.tensor(1.7, device=dev)
        want = torch.where(on[:, None], want, 0.0).to(TYPES[dst])
        assert torch.equal(out, want)
        if extra:  # what lies between the rows is not touched (the last row's is another's)
            assert torch.equal(whole[:-1, width:], rest[:-1])


def test_forward_of_a_batch_and_of_a_table_inside_the_parameters(dev):
    """ids of two dimensions; the table is a view into State's flat x."""
    import paper_2102_02888_amd as ob
    plan = ob.Plan([100 * 48, 77], 2)
    st = ob.State(plan, dev)
    st.x.normal_(0, 1, generator=_gen(dev, 1))
    table = st.x[:4800].view(100, 48)
    ids = _ids(dev, "zipf", 60, 100, 2).view(4, 15)
    out = torch.empty(4, 15, 48, dtype=torch.bfloat16, device=dev)
    ob.onebit_embedding_forward(table, ids, out)
    assert torch.equal(out, table[ids].bfloat16())
    plan.close()


def _grad64(dout, ids, vocab, padding, scale):
    on = (ids >= 0) & (ids < vocab) & (ids != padding)
    ids = torch.where(on, ids.long(), vocab)
    total = torch.zeros((vocab + 1, dout.shape[1]), dtype=torch.float64, device=dout.device)
    size = torch.zeros_like(total)
    d = torch.where(on[:, None], dout.double(), 0.0)
    total.index_put_((ids,), d * scale, accumulate=True)
    size.index_put_((ids,), d.abs() * scale, accumulate=True)
    count = torch.bincount(ids, minlength=vocab + 1)[:-1].double()
    return total[:-1], size[:-1], count


@pytest.mark.parametrize("tokens,vocab,width,extra,kind,padding", [
    (0, 5, 8, 0, "zipf", -1), (1, 1, 1, 0, "zipf", -1), (1, 300, 64, 0, "zipf", -1),
    (7, 5, 3, 2, "mixed", -1), (9, 4, 16, 0, "one", -1), (512, 3000, 1024, 0, "zipf", 0),
    (4095, 255, 20, 1, "mixed", 3), (4096, 256, 20, 0, "zipf", -1), (4097, 257, 20, 0, "zipf", -1),
    (5000, 70000, 9, 0, "mixed", 0), (20001, 30522, 771, 1, "mixed", 0), (70000, 3, 33, 0, "zipf", -1),
    (66000, 66000, 8, 0, "distinct", -1), (30000, 10, 40, 0, "one", -1), (6000, 50, 8, 0, "one", 25),
    (6000, 50, 8, 0, "masked", -1), (200000, 1000, 16, 3, "mixed", 1),
])
@pytest.mark.parametrize("src,dst,accumulate", [("bf16", "f32", False), ("f32", "f32", True),
                                                ("f16", "bf16", True), ("f32", "f16", False)])
def test_gradient(dev, tokens, vocab, width, extra, kind, padding, src, dst, accumulate):
    import paper_2102_02888_amd as ob
    scale = 1.5
    dout = _strided(tokens, width, TYPES[src], dev, extra, 4)
    idt = torch.int32 if tokens % 2 else torch.int64
    ids = _ids(dev, kind, tokens, vocab, 5, idt)
    dout[ids < 0] = float("nan")  # masked places are not read
    grad = _strided(vocab, width, TYPES[dst], dev, extra, 6)
    whole = grad.as_strided((vocab, width + extra), (width + extra, 1))
    old, rest = grad.clone(), whole[:, width:].clone()
    work = ob.embedding_workspace(tokens, vocab, width, dev)
    ob.onebit_embedding_grad(dout, ids, grad, work, scale=scale, padding_idx=padding,
                             accumulate=accumulate)
    total, size, count = _grad64(dout, ids, vocab, padding, scale)
    want = total + old.double() if accumulate else total
    # sum: n 2^-24; product, addition: 2^-24 each of what they form; the type's rounding
    tol = size * ((count + 4) * 2.0 ** -24)[:, None] + want.abs() * (ULP[dst] + 2.0 ** -22)
    tol += old.double().abs() * 2.0 ** -24 + 2.0 ** -25  # 2^-25: half of fp16's least value
    assert bool(((grad.double() - want).abs() <= tol).all())
    if accumulate:
        assert torch.equal(grad[count == 0], old[count == 0])
    else:
        assert not bool(grad[count == 0].any())
    if extra:
        assert torch.equal(whole[:-1, width:], rest[:-1])
    again = old.clone() if accumulate else torch.empty_like(old)
    ob.onebit_embedding_grad(dout, ids, again, work, scale=scale, padding_idx=padding,
                             accumulate=accumulate)
    assert torch.equal(again, grad)  # bit for bit


def test_gradient_keeps_nan_and_infinity_in_their_rows(dev):
    import paper_2102_02888_amd as ob
    ids = torch.arange(300, device=dev) % 30
    dout = torch.ones(300, 40, device=dev)
    dout[7, 3] = float("nan")
    dout[11, 5] = float("inf")
    grad = torch.full((31, 40), 9.0, device=dev)
    ob.onebit_embedding_grad(dout, ids, grad, ob.embedding_workspace(300, 31, 40, dev))
    want = torch.full((31, 40), 10.0, device=dev)
    want[30] = 0
    want[7, 3] = float("nan")
    want[11, 5] = float("inf")
    assert torch.equal(grad.isnan(), want.isnan())
    assert torch.equal(grad[~grad.isnan()], want[~want.isnan()])


def test_gradient_is_the_forwards_derivative(dev):
    """<dout, forward(table + h e)> - <dout, forward(table - h e)> over 2 h,
    exact here: the forward is linear and the values are small integers."""
    import paper_2102_02888_amd as ob
    g = _gen(dev, 1)
    table = torch.randint(-8, 8, (12, 10), device=dev, generator=g).float()
    ids = torch.randint(-1, 13, (50,), device=dev, generator=g)
    dout = torch.randint(-8, 8, (50, 10), device=dev, generator=g).float()
    grad = torch.empty_like(table)
    ob.onebit_embedding_grad(dout, ids, grad, ob.embedding_workspace(50, 12, 10, dev), scale=2.0)
    out = torch.empty(50, 10, device=dev)
    for v, c in ((0, 0), (3, 9), (11, 4), (5, 5)):
        got = []
        for h in (1.0, -1.0):
            t = table.clone()
            t[v, c] += h
            ob.onebit_embedding_forward(t, ids, out, scale=2.0)
            got.append((out.double() * dout.double()).sum())
        assert float(got[0] - got[1]) / 2 == float(grad[v, c])


def test_streams_and_graph(dev):
    """On another stream than the tensors' own, after an event; and replayed
    from a graph against the eager result, with new ids in the same buffer."""
    import paper_2102_02888_amd as ob
    tokens, vocab, width = 6000, 500, 96
    ids = _ids(dev, "zipf", tokens, vocab, 1)
    dout = torch.randn(tokens, width, device=dev, generator=_gen(dev, 2))
    grad, want = torch.empty(vocab, width, device=dev), torch.empty(vocab, width, device=dev)
    work = ob.embedding_workspace(tokens, vocab, width, dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ob.onebit_embedding_grad(dout, ids, grad, work, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    ob.onebit_embedding_grad(dout, ids, want, work)
    assert torch.equal(grad, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ob.onebit_embedding_grad(dout, ids, grad, work)
    for seed in range(3, 7):
        ids.copy_(_ids(dev, "zipf", tokens, vocab, seed))
        ob.onebit_embedding_grad(dout, ids, want, work)
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(grad, want), seed


def test_refusals(dev):
    import paper_2102_02888_amd as ob
    f = dict(device=dev)
    table, ids = torch.zeros(10, 8, **f), torch.zeros(5, dtype=torch.int64, **f)
    out, work = torch.zeros(5, 8, **f), ob.embedding_workspace(5, 10, 8, dev)
    fwd, bwd = ob.onebit_embedding_forward, ob.onebit_embedding_grad
    with pytest.raises(TypeError, match="ids"):
        fwd(table, ids.float(), out)
    with pytest.raises(TypeError, match="table"):
        fwd(table.double(), ids, out)
    with pytest.raises(ValueError, match="out is"):
        fwd(table, ids, torch.zeros(4, 8, **f))
    with pytest.raises(ValueError, match="out is"):
        fwd(table, ids, torch.zeros(5, 9, **f))
    with pytest.raises(ValueError, match="GPU tensor"):
        fwd(table.cpu(), ids, out)
    with pytest.raises(ValueError, match="GPU tensor"):
        fwd(table, ids.cpu(), out)
    with pytest.raises(ValueError, match="contiguous"):
        fwd(table, torch.zeros(10, dtype=torch.int64, **f)[::2], out)
    with pytest.raises(ValueError, match="unit stride"):
        fwd(torch.zeros(8, 10, **f).t(), ids, out)
    with pytest.raises(ValueError, match="overlapping"):
        fwd(table, ids, torch.zeros(1, 8, **f).expand(5, 8))
    with pytest.raises(ValueError, match="workspace has"):
        bwd(out, ids, table, work[:16])
    with pytest.raises(ValueError, match="grad_out is"):
        bwd(out[:3], ids, table, work)
    with pytest.raises(TypeError, match="workspace"):
        bwd(out, ids, table, None)
    L = ob.lib()
    n = ctypes.c_size_t()
    assert L.onebit_embedding_grad_workspace(-1, 4, 4, ctypes.byref(n)) == -1
    assert L.onebit_embedding_grad_workspace(4, 1 << 31, 4, ctypes.byref(n)) == -1
    assert L.onebit_embedding_grad_workspace(4, 4, 4, None) == -1
    p = table.data_ptr()
    for bad, status in (((p, 3, 8, 10, 8, ids.data_ptr(), 8, 5, 1.0, p, 0, 8, None), -1),
                        ((p, 0, 7, 10, 8, ids.data_ptr(), 8, 5, 1.0, p, 0, 8, None), -1),
                        ((p, 0, 8, 10, 8, ids.data_ptr(), 2, 5, 1.0, p, 0, 8, None), -1),
                        ((p + 2, 0, 8, 10, 8, ids.data_ptr(), 8, 5, 1.0, p, 0, 8, None), -2),
                        ((p, 0, 8, 10, 8, ids.data_ptr() + 4, 8, 5, 1.0, p, 0, 8, None), -2),
                        ((None, 0, 8, 10, 8, ids.data_ptr(), 8, 5, 1.0, p, 0, 8, None), -1)):
        assert L.onebit_embedding_forward(*bad) == status


def test_tables_past_32_bits(dev):
    """A table of 70,000 rows of 32,768 (2^31 and more elements): its last rows
    are read, written and zeroed at their places."""
    import paper_2102_02888_amd as ob
    vocab, width = 70000, 32768
    table = torch.zeros(vocab, width, dtype=torch.bfloat16, device=dev)
    last = torch.randn(16, width, device=dev, generator=_gen(dev, 1)).bfloat16()
    table[-16:] = last
    ids = torch.arange(vocab - 16, vocab, device=dev)
    out = torch.empty(16, width, dtype=torch.bfloat16, device=dev)
    ob.onebit_embedding_forward(table, ids, out)
    assert torch.equal(out, last)
    table.fill_(3.0)
    work = ob.embedding_workspace(16, vocab, width, dev)
    ob.onebit_embedding_grad(out, ids, table, work, scale=2.0)
    assert torch.equal(table[-16:], (last.float() * 2).bfloat16())
    assert not bool(table[:-16].any())
    many = ids.repeat(300)  # 4,800 places: the long lists' kernels
    dout = out.repeat(300, 1)
    work = ob.embedding_workspace(4800, vocab, width, dev)
    table.fill_(3.0)
    ob.onebit_embedding_grad(dout, many, table, work)
    assert torch.equal(table[-16:], (last.float() * 300).bfloat16())
    assert not bool(table[:-16].any())


@pytest.mark.parametrize("tokens", [100, 4096, 9000])
@pytest.mark.parametrize("vocab", [40, 262144, 262145, 300001])
def test_gradient_of_many_rows(dev, tokens, vocab):
    """Both sides of the sorting workgroup's rows and places; rows of 2 bytes."""
    import paper_2102_02888_amd as ob
    ids = torch.randint(-1, vocab + 1, (tokens,), device=dev, generator=_gen(dev, 1))
    dout = torch.ones(tokens, 1, device=dev, dtype=torch.bfloat16)
    grad = torch.full((vocab, 1), 5.0, device=dev, dtype=torch.float16)
    ob.onebit_embedding_grad(dout, ids, grad, ob.embedding_workspace(tokens, vocab, 1, dev))
    on = (ids >= 0) & (ids < vocab)
    want = torch.bincount(ids[on], minlength=vocab).to(torch.float16)
    assert torch.equal(grad[:, 0], want)


@pytest.mark.parametrize("src", ["bf16", "f32"])
def test_one_workspace_for_shorter_and_narrower_calls(dev, src):
    """A workspace of exactly the size for the largest call serves the others, and
    nothing behind it is touched: calls on both sides of where the pieces of the
    list get longer (32,768 places of 1,024 bf16 columns, 16,384 of fp32)."""
    import paper_2102_02888_amd as ob
    vocab, most, wide = 500, 32768, 1024
    n = ctypes.c_size_t()
    assert ob.lib().onebit_embedding_grad_workspace(most, vocab, wide, ctypes.byref(n)) == 0
    # as much again behind it as the largest need of any of these calls
    whole = torch.full((n.value + (64 << 20),), 0xA5, dtype=torch.uint8, device=dev)
    work, behind = whole[:n.value], whole[n.value:]
    for tokens, width in ((most, wide), (most - 1, wide), (most, 1016), (16384, wide),
                          (16383, wide), (16384, 1020), (4097, 1000), (4096, wide), (100, 7)):
        dout = torch.randint(-4, 5, (tokens, width), device=dev, generator=_gen(dev, 1))
        dout = dout.to(TYPES[src])
        ids = torch.randint(-1, vocab, (tokens,), device=dev, generator=_gen(dev, 2))
        grad = torch.full((vocab, width), 3.0, device=dev)
        ob.onebit_embedding_grad(dout, ids, grad, work)
        want = torch.zeros(vocab + 1, width, device=dev)  # small integers: exact in any order
        want.index_add_(0, torch.where(ids < 0, vocab, ids), dout.float())
        assert torch.equal(grad, want[:-1]), (tokens, width)
        assert bool((behind == 0xA5).all()), (tokens, width)


@pytest.mark.parametrize("src,width", [("f32", 523776), ("f32", 524292), ("bf16", 1048584)])
def test_gradient_of_short_lists_of_very_wide_rows(dev, src, width):
    """Up to 4,096 places on both sides of where a workgroup for every row and group
    of columns would be 2^32 threads and more."""
    import paper_2102_02888_amd as ob
    tokens, vocab = 4096, 3
    dout = torch.randint(-4, 5, (tokens, width), device=dev, dtype=TYPES[src],
                         generator=_gen(dev, 1))
    ids = torch.randint(-1, vocab - 1, (tokens,), device=dev, generator=_gen(dev, 2))
    grad = torch.full((vocab, width), 3.0, device=dev)
    ob.onebit_embedding_grad(dout, ids, grad, ob.embedding_workspace(tokens, vocab, width, dev))
    for v in range(vocab):  # small integers: exact in any order
        want = torch.zeros(width, device=dev)
        for part in torch.nonzero(ids == v)[:, 0].split(256):
            want += dout[part].float().sum(0)
        assert torch.equal(grad[v], want), v
