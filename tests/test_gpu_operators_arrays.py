"""The operators on arrays that lie in other arrays: results beside their inputs, in
place, and what may not be."""

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
