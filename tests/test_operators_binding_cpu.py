"""The binding of the operators with tensors that have a type, a shape and a GPU but no
memory: what it refuses on its own, and what it leaves behind, without a GPU."""

import importlib.machinery
import importlib.util
import os
import shutil

import pytest
import torch

from paper_1902_06714_amd import nf

I8, I32, I64, F32 = torch.int8, torch.int32, torch.int64, torch.float32


class NoMemory(torch.Tensor):
    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} called")


def gpu(shape, dtype=F32, device=0):
    return torch.Tensor._make_wrapper_subclass(NoMemory, shape, dtype=dtype, device=f"cuda:{device}", storage_size=0)


@pytest.fixture(scope="module")
def bind(tmp_path_factory):
    """The module once more, which takes GPU 0 for the current one."""
    d = tmp_path_factory.mktemp("bind")
    here = os.path.dirname(nf.LIB_PATH)
    shutil.copy(os.path.join(here, "_nfbind.so"), d / "_nfbind.so")
    os.symlink(nf.LIB_PATH, d / "libnf.so")
    kept = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream = lambda: 0, lambda device: 0
    try:
        loader = importlib.machinery.ExtensionFileLoader("_nfbind", str(d / "_nfbind.so"))
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_nfbind", loader))
        loader.exec_module(module)
    finally:
        torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream = kept
    return module


# Calls without rows or matrices: nothing is launched.  Tensors by name, written ones marked.
CALLS = {
    "logprobs": ["logits", ("targets", I64), ("logp!",), ("entropy!",), ("stat!", F32, 2), ("top_ids!", I32, 3),
                 ("top_logp!", F32, 3), 1.0, "work", -1],
    "logprobs_train": ["logits", ("targets", I64), ("g_logp",), ("g_entropy",), "dlogits!", ("logp!",), ("entropy!",),
                       ("stat!", F32, 2), 1.0, "work", -1],
    "logprobs_grad": ["logits", ("targets", I64), ("stat", F32, 2), ("entropy",), ("g_logp",), ("g_entropy",), "dlogits!", 1.0,
                      -1],
    "orthogonalize": ["x", "out!", "work", -1],
    "muon_step": ["w", "m", "g", "w_out!", "m_out!", 0.1, 0.9, 1, 0.0, "work", -1],
    "quantize_rows": ["x", "q!", ("scale!",), -1],
    "linear_i8": ["xq", ("x_scale",), "wq", "w_scale", "y!", 7, "bias", -1, -1],
    "linear_i8_dynamic": ["x", "wq", "w_scale", "y!", "bias", -1, "work", -1],
}


def _args(call, away=None):
    """The call's arguments, one of its tensors on another GPU; and the written ones."""
    shapes = {"logits": (0, 7), "dlogits": (0, 7), "x": (0, 7), "xq": (0, 16), "q": (0, 16), "y": (0, 5), "wq": (5, 16),
              "w_scale": (5,), "bias": (5,), "work": (64,)}
    if call in ("orthogonalize", "muon_step"):
        shapes.update({k: (0, 4, 7) for k in ("x", "out", "w", "m", "g", "w_out", "m_out")})
    types = {"xq": I8, "q": I8, "wq": I8, "work": torch.uint8}
    args, written = [], []
    for a in CALLS[call]:
        if isinstance(a, str) or isinstance(a, tuple):
            name, dtype, *more = (a, None) if isinstance(a, str) else (*a, F32)[:2] + a[2:]
            plain = name.rstrip("!")
            shape = shapes.get(plain, (0, *more)) if isinstance(a, str) else (0, *more)
            t = gpu(shape, dtype or types.get(plain, F32), int(plain == away))
            if name != plain:
                written.append(t)
            a = t
        args.append(a)
    return args, written


NAMES = [(c, (a if isinstance(a, str) else a[0]).rstrip("!")) for c, args in CALLS.items() for a in args
         if isinstance(a, (str, tuple))]


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_the_current_gpu_pass(bind, call):
    st = getattr(bind, call)(*_args(call)[0])
    # (the missing memory of weights and of places for alternatives is the library's to refuse)
    assert st == (nf.NF_EINVAL if call in ("logprobs", "linear_i8", "linear_i8_dynamic") else nf.NF_OK), nf.nf_last_error()


@pytest.mark.parametrize("call,name", NAMES)
def test_tensors_of_another_gpu_are_refused(bind, call, name):
    with pytest.raises(ValueError, match=f"{name} is not on the current device"):
        getattr(bind, call)(*_args(call, name)[0])


@pytest.mark.parametrize("call", [c for c in CALLS if not c.startswith("linear")])
def test_written_tensors_have_a_new_version(bind, call):
    args, written = _args(call)
    if call == "logprobs":                                # without alternatives
        args[5] = args[6] = None
        written = written[:3]
    before = [t._version for t in args if isinstance(t, torch.Tensor)]
    assert getattr(bind, call)(*args) == nf.NF_OK
    after = [t._version for t in args if isinstance(t, torch.Tensor)]
    raised = [any(t is w for w in written) for t in args if isinstance(t, torch.Tensor)]
    assert [b - a for a, b in zip(before, after)] == [int(r) for r in raised]


def test_refused_calls_leave_versions(bind):
    args, written = _args("linear_i8_dynamic")
    assert bind.linear_i8_dynamic(*args) == nf.NF_EINVAL and written[0]._version == 0


@pytest.mark.parametrize("call,shape,dtype,status,says", [
    ("orthogonalize", (0, 4, 7), torch.float16, nf.NF_EINVAL, "fp32 or bf16"),
    ("orthogonalize", (0, 7), F32, nf.NF_EINVAL, "at least 1"), ("orthogonalize", (0, 4, 65537), F32, nf.NF_ESHAPE, "at most"),
    ("muon_step", (0, 4, 7), torch.float16, nf.NF_EINVAL, "fp32 or bf16"),
    ("muon_step", (2, 0, 7), F32, nf.NF_EINVAL, "at least 1"),
    ("linear_i8_dynamic", (0, 0), F32, nf.NF_EINVAL, "at least"),
    ("linear_i8_dynamic", (0, 131072), F32, nf.NF_ESHAPE, "at most")])
def test_sizes_are_refused_with_the_librarys_own_status(bind, call, shape, dtype, status, says):
    t = [gpu(shape, dtype) for _ in range(5)]
    if call == "orthogonalize":
        st = bind.orthogonalize(t[0], t[1], None, -1)
    elif call == "muon_step":
        st = bind.muon_step(t[0], gpu(shape), t[1], t[2], gpu(shape), 0.1, 0.9, 1, 0.0, None, -1)
    else:
        st = bind.linear_i8_dynamic(t[0], gpu((5, shape[1]), I8), gpu((5,)), gpu((0, 5)), None, -1, None, -1)
    assert st == status and says in nf.nf_last_error(), (st, nf.nf_last_error())
