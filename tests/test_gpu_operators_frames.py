"""What lies between and around the rows of the operators' results is not written, at
widths that are no whole number of vectors and in every kernel that writes rows."""

import pytest

from .frames import Framed
from .gpu_run import note, torch_cuda

pytestmark = pytest.mark.gpu


def _nf():
    from paper_1902_06714_amd import nf
    return nf


def _types():
    torch = torch_cuda()
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rand(shape, seed=1):
    torch = torch_cuda()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda")


# rows by lanes, by a wave, by workgroups with the row in registers or not, and cut
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,classes", [(9, 1), (9, 10), (9, 17), (9, 65), (9, 127), (9, 129), (9, 515), (9, 1031), (9, 2051),
                                          (9, 4099), (9, 8197), (300, 16411), (300, 33001), (9, 35003), (3, 140003)])
@pytest.mark.parametrize("pad,ahead", [(1, 1), (5, 3)])
def test_gradients(rows, classes, dtype, pad, ahead):
    torch, nf = torch_cuda(), _nf()
    note(f"frames of gradients {rows}x{classes} {dtype} pad={pad}")
    x = _rand((rows, classes)).to(_types()[dtype])
    t, g, h = torch.arange(rows, device="cuda") % classes, _rand((rows,), 2), _rand((rows,), 3)
    stat, entropy = torch.empty(rows, 2, device="cuda"), torch.empty(rows, device="cuda")
    nf.nf_logprobs(x, t, stat=stat, entropy=entropy)
    for way in range(2):
        dx = Framed((rows, classes), x.dtype, pad, ahead)
        if way:
            nf.nf_logprobs_train(x, t, g, h, dx.view)
        else:
            nf.nf_logprobs_grad(x, t, stat, entropy, g, h, dx.view)
        torch.cuda.synchronize()
        dx.check()
        assert not (dx.view == 7.0).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,cols", [(1, 1, 7), (1, 7, 1), (3, 30, 77), (3, 77, 30), (2, 64, 5), (2, 5, 64), (3, 49, 1001),
                                             (2, 67, 131), (2, 131, 67)])
@pytest.mark.parametrize("pad,ahead", [(1, 1), (3, 2)])
def test_orthogonalised(count, rows, cols, dtype, pad, ahead):
    torch, nf = torch_cuda(), _nf()
    note(f"frames of orthogonalised {count}x{rows}x{cols} {dtype} pad={pad}")
    out = Framed((count, rows, cols), _types()[dtype], pad, ahead)
    nf.nf_orthogonalize(_rand((count, rows, cols)).to(_types()[dtype]), out.view)
    torch.cuda.synchronize()
    out.check()
    assert not (out.view == 7.0).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 3, 9, 16, 40, 301])
@pytest.mark.parametrize("outputs", [1, 2, 3, 5, 17, 34, 91])
def test_layers(rows, outputs, dtype):
    torch, nf = torch_cuda(), _nf()
    note(f"frames of layers {rows}->{outputs} {dtype}")
    wq = torch.randint(-127, 128, (outputs, 112), device="cuda").to(torch.int8)
    wq[:, 100:] = 0
    scale = torch.full((outputs,), 1e-3, device="cuda")
    for pad, ahead in ((1, 1), (6, 2)):
        y = Framed((rows, outputs), _types()[dtype], pad, ahead)
        nf.nf_linear_i8_dynamic(_rand((rows, 100)), wq, scale, y.view, act="sigmoid")
        torch.cuda.synchronize()
        y.check()
        assert ((y.view >= 0) & (y.view <= 1)).all()
