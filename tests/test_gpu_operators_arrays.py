"""The operators on arrays that lie in other arrays (results beside their inputs, in
place, and what may not be), on very many rows, and on rows that nothing is left of."""

import pytest

from .gpu_run import note, torch_cuda

pytestmark = pytest.mark.gpu


def _nf():
    from paper_1902_06714_amd import nf
    return nf


def _rand(*shape, seed=1):
    torch = torch_cuda()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda")


@pytest.mark.parametrize("rows,cols", [(40, 70), (300, 41), (70, 130)])
def test_orthogonalize_beside_its_matrices(rows, cols):
    torch, nf = torch_cuda(), _nf()
    note(f"orthogonalize beside its matrices, {rows}x{cols}")
    src = _rand(3, rows, cols)
    want = torch.empty_like(src)
    nf.nf_orthogonalize(src, want)
    wide = torch.full((3, rows, 2 * cols + 3), 7.0, device="cuda")          # in the same rows
    x, out = wide[:, :, :cols], wide[:, :, cols + 1:2 * cols + 1]
    x.copy_(src)
    nf.nf_orthogonalize(x, out)
    turns = torch.full((3, 2, rows, cols), 7.0, device="cuda")              # by turns in one stack
    turns[:, 1].copy_(src)
    nf.nf_orthogonalize(turns[:, 1], turns[:, 0])
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(x, src)
    assert (wide[:, :, cols] == 7.0).all() and (wide[:, :, 2 * cols + 1:] == 7.0).all()
    assert torch.equal(turns[:, 0], want) and torch.equal(turns[:, 1], src)


@pytest.mark.parametrize("rows,cols", [(90, 33), (30, 50), (70, 130)])
def test_orthogonalize_matrices_side_by_side(rows, cols):
    """A stack whose matrices are blocks of columns of one, as a layer's heads are."""
    torch, nf = torch_cuda(), _nf()
    note(f"orthogonalize side by side, {rows}x{cols}")
    heads = _rand(rows, 4 * cols + 1)
    x = heads[:, :4 * cols].view(rows, 4, cols).permute(1, 0, 2)
    want = torch.empty(4, rows, cols, device="cuda")
    nf.nf_orthogonalize(x, want)
    out = torch.full((rows, 4, cols + 2), 7.0, device="cuda")
    nf.nf_orthogonalize(x, out[:, :, :cols].permute(1, 0, 2))
    last = heads[:, 4 * cols].clone()
    nf.nf_orthogonalize(x, x)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :, :cols].permute(1, 0, 2), want) and (out[:, :, cols:] == 7.0).all()
    assert torch.equal(x, want) and torch.equal(heads[:, 4 * cols], last)


@pytest.mark.parametrize("rows,cols", [(40, 70), (70, 130)])
def test_orthogonalize_refuses_a_result_over_its_matrices(rows, cols):
    torch, nf = torch_cuda(), _nf()
    buf = _rand(rows + 1, cols + 7)
    flat = buf.view(-1)[:rows * cols].view(rows, cols)
    before = buf.clone()
    note(f"orthogonalize over its matrices, {rows}x{cols}")
    for x, out in ((buf[:rows, :cols], flat), (buf[:rows, :cols], buf[1:, :cols]), (buf[:rows, 1:cols + 1], buf[:rows, :cols]),
                   (buf[:rows, :cols].expand(1, rows, cols), flat[None])):
        with pytest.raises(nf.NfError):
            nf.nf_orthogonalize(x, out)
    torch.cuda.synchronize()
    assert torch.equal(buf, before)


@pytest.mark.parametrize("rows,cols", [(40, 70), (70, 130)])
def test_muon_step_in_the_gradients_place(rows, cols):
    torch, nf = torch_cuda(), _nf()
    note(f"muon in the gradient's place, {rows}x{cols}")
    w, m, g = (_rand(rows, cols, seed=k) for k in range(3))
    w_out, m_out = torch.empty_like(w), torch.empty_like(m)
    nf.nf_muon_step(w, m, g, w_out, m_out, 0.1)
    with pytest.raises(nf.NfError):
        nf.nf_muon_step(w, m, g.view(torch.bfloat16).view(-1)[:rows * cols].view(rows, cols), g, m, 0.1)
    nf.nf_muon_step(w, m, g, g, m, 0.1)
    torch.cuda.synchronize()
    assert torch.equal(g, w_out) and torch.equal(m, m_out)


@pytest.mark.parametrize("rows,classes", [(9, 50), (300, 1000), (5, 9000)])
def test_gradient_beside_the_logits(rows, classes):
    torch, nf = torch_cuda(), _nf()
    note(f"gradient beside the logits, {rows}x{classes}")
    wide = torch.full((rows, 2 * classes + 3), 7.0, device="cuda")
    x, dx = wide[:, :classes], wide[:, classes + 1:2 * classes + 1]
    x.copy_(_rand(rows, classes))
    t, g, want = torch.arange(rows, device="cuda") % classes, _rand(rows), torch.empty(rows, classes, device="cuda")
    stat = torch.empty(rows, 2, device="cuda")
    nf.nf_logprobs(x, t, stat=stat)
    nf.nf_logprobs_train(x, t, g, None, want)
    nf.nf_logprobs_train(x, t, g, None, dx)
    torch.cuda.synchronize()
    assert torch.equal(dx, want)
    nf.nf_logprobs_grad(x, t, stat, None, g, None, want)
    nf.nf_logprobs_grad(x, t, stat, None, g, None, dx)
    torch.cuda.synchronize()
    assert torch.equal(dx, want)
    assert (wide[:, classes] == 7.0).all() and (wide[:, 2 * classes + 1:] == 7.0).all()


@pytest.mark.parametrize("rows,inputs,outputs", [(1, 100, 20), (3, 64, 30), (12, 130, 40), (100, 77, 90)])
def test_linear_layer_beside_its_inputs(rows, inputs, outputs):
    """A layer's outputs appended to its inputs' rows, as where later layers read both."""
    torch, nf = torch_cuda(), _nf()
    note(f"linear beside its inputs, {rows}x{inputs}->{outputs}")
    wide = torch.full((rows, inputs + outputs), 7.0, device="cuda")
    x, y = wide[:, :inputs], wide[:, inputs:]
    x.copy_(_rand(rows, inputs))
    wq = torch.zeros((outputs, (inputs + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    ws = torch.empty(outputs, device="cuda")
    nf.nf_quantize_rows(_rand(outputs, inputs, seed=2), wq, ws)
    want = torch.empty(rows, outputs, device="cuda")
    nf.nf_linear_i8_dynamic(x.clone(), wq, ws, want, act="tanh")
    nf.nf_linear_i8_dynamic(x, wq, ws, y, act="tanh")
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    with pytest.raises(nf.NfError):
        nf.nf_linear_i8_dynamic(x, wq, ws, wide[:, inputs - 1:-1])
    q = torch.full((rows, 256), 9, dtype=torch.int8, device="cuda")       # quantised rows beside the rows
    q4 = q.view(torch.float32)
    n = min(inputs, 32)
    q4[:, :n].copy_(x[:, :n])
    scale, want_q = torch.empty(rows, device="cuda"), torch.empty((rows, 32), dtype=torch.int8, device="cuda")
    nf.nf_quantize_rows(q4[:, :n], q[:, 128:160], scale)
    nf.nf_quantize_rows(x[:, :n], want_q, scale)
    torch.cuda.synchronize()
    assert torch.equal(q[:, 128:160], want_q) and (q[:, 160:] == 9).all()


# more rows than one grid holds threads for: up to 128 classes four rows share a
# workgroup of 256, longer ones have a wave each
@pytest.mark.parametrize("classes", [65, 129])
def test_log_probabilities_of_more_rows_than_a_grid_holds(classes):
    torch, nf = torch_cuda(), _nf()
    rows = (1 << 26) + 9
    note(f"log probabilities of {rows} rows of {classes}")
    x = _rand_rows(rows, classes)
    t = torch.randint(0, classes, (rows,), device="cuda")
    g = torch.full((rows,), 0.5, device="cuda")
    logp, ids = torch.full((rows,), 1.0, device="cuda"), torch.full((rows, 1), -1, dtype=torch.int32, device="cuda")
    stat = torch.empty((rows, 2), device="cuda")
    nf.nf_logprobs(x, t, logp=logp, stat=stat, top_ids=ids)
    assert (logp <= 0).all() and (ids >= 0).all()
    parts = [slice(0, 100), slice((1 << 26) - 40, (1 << 26) - 10), slice(rows - 50, rows)]
    held = [x[p].clone() for p in parts]
    for p, a in zip(parts, held):
        l2, i2 = torch.empty_like(logp[p]), torch.empty_like(ids[p])
        nf.nf_logprobs(a, t[p], logp=l2, top_ids=i2)
        assert torch.equal(l2, logp[p]) and torch.equal(i2, ids[p])
    nf.nf_logprobs_train(x, t, g, None, x)
    for p, a in zip(parts, held):
        nf.nf_logprobs_train(a, t[p], g[p], None, a)
        assert torch.equal(a, x[p])


def test_gradient_of_more_rows_than_a_grid_holds():
    torch, nf = torch_cuda(), _nf()
    rows, classes = (1 << 24) + 9, 1025                  # 256 threads a row
    note(f"gradient of {rows} rows of {classes}")
    x = _rand_rows(rows, classes)
    t, g = torch.randint(0, classes, (rows,), device="cuda"), torch.full((rows,), 0.5, device="cuda")
    stat = torch.empty((rows, 2), device="cuda")
    nf.nf_logprobs(x, stat=stat)
    parts = [slice(0, 100), slice((1 << 24) - 40, (1 << 24) + 1), slice(rows - 5, rows)]
    held = [x[p].clone() for p in parts]
    nf.nf_logprobs_grad(x, t, stat, None, g, None, x)
    for p, a in zip(parts, held):
        nf.nf_logprobs_grad(a, t[p], stat[p], None, g[p], None, a)
        assert torch.equal(a, x[p])


def _rand_rows(rows, classes):
    """bf16 rows that differ from one another, few of them drawn."""
    torch = torch_cuda()
    x = torch.empty((rows, classes), dtype=torch.bfloat16, device="cuda")
    some = _rand(4099, classes).to(torch.bfloat16)
    for r in range(0, rows, 4099 * 1024):
        n = min(rows - r, 4099 * 1024)
        x[r:r + n].copy_(some.repeat((n + 4098) // 4099, 1)[:n])
    return x


def test_overwritten_values_are_not_differentiated():
    """Backpropagation through values that an operator has overwritten is refused."""
    torch, nf = torch_cuda(), _nf()
    note("versions")
    x = _rand(6, 9).requires_grad_()
    z = x.exp()                                           # keeps its result
    t, g = torch.zeros(6, dtype=torch.int64, device="cuda"), _rand(6)
    nf.nf_logprobs_train(z.detach(), t, g, None, z.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()
    q, scale, y = torch.zeros((6, 16), dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda"), torch.empty(3, 6, device="cuda")
    nf.nf_quantize_rows(x.detach(), q, scale)
    nf.nf_linear_i8_dynamic(_rand(3, 9), q, scale, y)
    nf.nf_linear_i8(q, scale, q, scale, torch.empty(6, 6, device="cuda"), 9)
    assert (q._version, scale._version, y._version) == (1, 1, 1)
    with torch.inference_mode():
        y = torch.empty(3, 6, device="cuda")
        nf.nf_linear_i8_dynamic(_rand(3, 9), q, scale, y)
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,classes", [(5, 10), (5, 300), (300, 5000), (3, 40000), (2, 131072)])
def test_rows_without_probabilities_have_no_gradient(rows, classes):
    """... whatever their weights are: exp of the difference of two log probabilities of
    minus infinity is NaN."""
    torch, nf = torch_cuda(), _nf()
    note(f"rows without probabilities, {rows}x{classes}")
    inf, nan = float("inf"), float("nan")
    x = _rand(rows, classes)
    x[0] = -inf
    x[-1] = -inf
    t = torch.arange(rows, device="cuda")
    logp, stat, entropy = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), torch.empty(rows, device="cuda")
    nf.nf_logprobs(x, t, logp=logp, stat=stat, entropy=entropy)
    g = torch.exp(logp - logp.clone())                     # 1, and NaN where nothing is left
    assert torch.isnan(g[0]) and torch.isnan(g[-1]) and (g[1:-1] == 1).all()
    for h in (None, torch.ones(rows, device="cuda"), torch.full((rows,), nan, device="cuda"), torch.full((rows,), inf, device="cuda")):
        both = []
        for way in range(2):
            dx = torch.full_like(x, 7.0)
            if way:
                nf.nf_logprobs_train(x, t, g, h, dx)
            else:
                nf.nf_logprobs_grad(x, t, stat, entropy, g, h, dx)
            assert (dx[0] == 0).all() and (dx[-1] == 0).all()
            both.append(dx)
        if h is None:
            assert all(torch.isfinite(dx).all() for dx in both)
    t[0] = classes                                         # a target past the classes is told all the same
    nf.nf_logprobs_train(x, t, g, None, dx)
    assert torch.isnan(dx[0]).all() and (dx[-1] == 0).all()
