"""The operators' CPU reference against worked cases and differences, and the
entry points' refusals, which need no GPU."""

import ctypes
import re

import numpy as np
import pytest

from oracle import operators as ref
from paper_1902_06714_amd import nf


def test_reference_logprobs_worked():
    ln = np.log
    x = np.array([[ln(1.0), ln(2.0), ln(5.0)], [0.0, 0.0, 0.0], [-np.inf, 0.0, -np.inf], [-np.inf] * 3])
    logp, ent, stat, ids, alt = ref.logprobs(x, 1.0, [1, 2, 1, 0], 3)
    assert np.allclose(logp[:3], [ln(2 / 8), ln(1 / 3), 0.0], atol=1e-7) and np.isneginf(logp[3])
    want = -(ln(1 / 8) / 8 + ln(2 / 8) * 2 / 8 + ln(5 / 8) * 5 / 8)
    assert np.allclose(ent, [want, ln(3), 0.0, 0.0], atol=1e-6)
    assert ids.tolist() == [[2, 1, 0], [0, 1, 2], [1, 0, 2], [0, 1, 2]]
    assert np.allclose(alt[0], ln(np.array([5, 2, 1]) / 8), atol=1e-7)
    logp, ent, _, ids, _ = ref.logprobs(np.array([[1.0, np.nan, 2.0]]), 1.0, [0], 2)
    assert np.isnan(logp[0]) and np.isnan(ent[0]) and ids.tolist() == [[1, 2]]
    assert ref.logprobs(np.zeros((1, 4)), 1.0, [-1])[0][0] == 0.0
    assert np.isnan(ref.logprobs(np.zeros((1, 4)), 1.0, [4])[0][0])


def test_reference_gradient_by_differences():
    rng = np.random.default_rng(3)
    # multiples of 2^-8 and a scale of 0.5: the fp32 step of the definition is exact
    x = np.round(rng.normal(0, 2, (3, 7)) * 256) / 256
    x[1, 2] = -np.inf
    t, g, h = [4, -1, 0], rng.normal(0, 1, 3), rng.normal(0, 1, 3)
    dx = ref.logprobs_grad(x, 0.5, t, g, h)

    def f(y):
        logp, ent = ref.logprobs(y, 0.5, t)[:2]
        return float((g * logp).sum() + (h * ent).sum())
    step = 2.0 ** -6
    for i in range(3):
        for j in range(7):
            if np.isneginf(x[i, j]):
                assert dx[i, j] == 0.0
                continue
            y = [x.copy() for _ in range(4)]
            for a, k in zip(y, (-2, -1, 1, 2)):
                a[i, j] += k * step
            d = (f(y[0]) - 8 * f(y[1]) + 8 * f(y[2]) - f(y[3])) / (12 * step)
            assert abs(d - dx[i, j]) < 1e-7, (i, j, d, dx[i, j])


def test_reference_orthogonalize():
    rng = np.random.default_rng(4)
    u = rng.normal(0, 1, (5, 9))
    left, s, right = np.linalg.svd(u, full_matrices=False)
    s = s / np.sqrt((s * s).sum())
    for _ in range(ref.STEPS):
        s = ref.QUINTIC[0] * s + ref.QUINTIC[1] * s ** 3 + ref.QUINTIC[2] * s ** 5
    assert np.allclose(ref.orthogonalize(u), (left * s) @ right, atol=1e-12)
    assert np.allclose(ref.orthogonalize(u.T), ref.orthogonalize(u).T, atol=1e-12)
    assert not ref.orthogonalize(np.zeros((3, 4))).any()


def test_reference_quantize_worked():
    q, s = ref.quantize_rows(np.array([[1.0, -2.0, 0.5, 127.0], [0.0] * 4, [np.inf, 1, 2, 3], [np.nan, 1, 2, 3]]))
    assert q[0].tolist() == [1, -2, 0, 127] and s[0] == 1.0      # 0.5 goes to the even 0
    assert not q[1:].any() and s[1] == 0.0 and np.isnan(s[2]) and np.isnan(s[3])
    y = ref.linear_i8(q[:1], s[:1], np.array([[1, 2, 3, 4]], np.int8), np.array([0.5], np.float32),
                      np.array([1.0], np.float32))
    assert y[0, 0] == 0.5 * (1 - 4 + 508) + 1


def test_every_operator_is_declared_and_exported():
    with open(nf.HEADER) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(nf_\w+)\s*\(", text))
    want = {"nf_logprobs_work", "nf_logprobs", "nf_logprobs_train", "nf_logprobs_grad", "nf_orthogonalize_work", "nf_orthogonalize",
            "nf_muon_step", "nf_quantize_rows", "nf_linear_i8", "nf_linear_i8_work", "nf_linear_i8_dynamic"}
    assert want <= names
    for n in want:
        assert hasattr(nf.raw(), n) and callable(getattr(nf, n))


# Addresses that no refused call may touch: the arguments are checked first.
P = 1 << 20
BIG = 1 << 62
E, S = nf.NF_EINVAL, nf.NF_ESHAPE
INF, NAN = float("inf"), float("nan")


def _call(name, base, change):
    args = dict(base)
    assert set(change) <= set(args), change
    args.update(change)
    return getattr(nf.raw(), name)(*args.values())


LOGP = dict(x=P, dtype=nf.NF_BF16, rows=4, classes=10, ld=10, scale=1.0, t=P, n_top=2, logp=P, ent=P, stat=P, ids=P,
            alt=P, work=None, bytes=0, stream=None)
TRAIN = dict(x=P, dtype=nf.NF_F32, rows=4, classes=10, ld=10, scale=1.0, t=P, g=P, h=P, logp=P, ent=P, stat=P,
             dx=2 * P, ldd=10, work=None, bytes=0, stream=None)
GRAD = dict(x=P, dtype=nf.NF_F32, rows=4, classes=10, ld=10, scale=1.0, t=P, stat=P, ent=P, g=P, h=P, dx=2 * P, ldd=10,
            stream=None)
ORTH = dict(x=P, dtype=nf.NF_F32, count=2, rows=6, cols=8, ld=8, stride=48, out=2 * P, ldo=8, so=48, work=4 * P,
            bytes=BIG, stream=None)
MUON = dict(w=P, wd=nf.NF_F32, m=2 * P, g=3 * P, gd=nf.NF_F32, count=1, rows=6, cols=8, eta=0.1, momentum=0.9,
            nesterov=1, decay=0.0, wo=4 * P, mo=5 * P, work=6 * P, bytes=BIG, stream=None)
QUANT = dict(x=P, dtype=nf.NF_F16, rows=4, cols=17, ld=17, q=2 * P, ldq=32, scale=P, stream=None)
LIN = dict(xq=P, ldx=32, xs=P, wq=2 * P, ldw=32, ws=P, bias=P, act=1, rows=3, inputs=17, outputs=5, y=3 * P,
           yd=nf.NF_F32, ldy=5, stream=None)
DYN = dict(x=P, xd=nf.NF_F32, ldx=17, wq=2 * P, ldw=32, ws=P, bias=P, act=1, rows=3, inputs=17, outputs=5, y=3 * P,
           yd=nf.NF_F32, ldy=5, work=4 * P, bytes=BIG, stream=None)


@pytest.mark.parametrize("name,base,change,status", [
    ("nf_logprobs", LOGP, {"dtype": nf.NF_F64}, E), ("nf_logprobs", LOGP, {"dtype": 9}, E),
    ("nf_logprobs", LOGP, {"x": None}, E), ("nf_logprobs", LOGP, {"x": P + 1}, E),
    ("nf_logprobs", LOGP, {"rows": -1}, E), ("nf_logprobs", LOGP, {"classes": 0}, E),
    ("nf_logprobs", LOGP, {"rows": 1 << 31}, S), ("nf_logprobs", LOGP, {"classes": (1 << 30) + 1, "ld": BIG}, S),
    ("nf_logprobs", LOGP, {"ld": 9}, S), ("nf_logprobs", LOGP, {"ld": BIG}, S),
    ("nf_logprobs", LOGP, {"scale": 0.0}, E), ("nf_logprobs", LOGP, {"scale": -1.0}, E),
    ("nf_logprobs", LOGP, {"scale": INF}, E), ("nf_logprobs", LOGP, {"scale": NAN}, E),
    ("nf_logprobs", LOGP, {"n_top": -1}, E), ("nf_logprobs", LOGP, {"n_top": 65, "classes": 100, "ld": 100}, E),
    ("nf_logprobs", LOGP, {"n_top": 11}, S), ("nf_logprobs", LOGP, {"ids": None, "alt": None}, E),
    ("nf_logprobs", LOGP, {"classes": 131072, "ld": 131072, "work": P, "bytes": 10}, S),
    ("nf_logprobs", LOGP, {"classes": 131072, "ld": 131072, "work": P + 8, "bytes": BIG}, E),
    ("nf_logprobs_train", TRAIN, {"classes": 131072, "ld": 131072, "ldd": 131072, "dx": 99 * P, "work": P, "bytes": 10}, S),
    ("nf_logprobs_train", TRAIN, {"dx": None}, E), ("nf_logprobs_train", TRAIN, {"ldd": 9}, S),
    ("nf_logprobs_train", TRAIN, {"dx": P + 8}, E), ("nf_logprobs_train", TRAIN, {"dx": P, "ldd": 12}, E),
    ("nf_logprobs_train", TRAIN, {"dx": 2 * P + 2}, E), ("nf_logprobs_train", TRAIN, {"t": None}, E),
    ("nf_logprobs_grad", GRAD, {"stat": None}, E), ("nf_logprobs_grad", GRAD, {"ent": None}, E),
    ("nf_logprobs_grad", GRAD, {"t": None}, E), ("nf_logprobs_grad", GRAD, {"dx": P + 4}, E),
    ("nf_logprobs_grad", GRAD, {"classes": 0}, E),
    ("nf_orthogonalize", ORTH, {"dtype": nf.NF_F16}, E), ("nf_orthogonalize", ORTH, {"dtype": nf.NF_F64}, E),
    ("nf_orthogonalize", ORTH, {"count": -1}, E), ("nf_orthogonalize", ORTH, {"rows": 0}, E),
    ("nf_orthogonalize", ORTH, {"cols": 65537, "ld": 70000, "ldo": 70000}, S),
    ("nf_orthogonalize", ORTH, {"count": 65536}, S), ("nf_orthogonalize", ORTH, {"x": None}, E),
    ("nf_orthogonalize", ORTH, {"out": None}, E), ("nf_orthogonalize", ORTH, {"ld": 7}, S),
    ("nf_orthogonalize", ORTH, {"ldo": 7}, S), ("nf_orthogonalize", ORTH, {"so": 47}, S),
    ("nf_orthogonalize", ORTH, {"x": P + 2}, E), ("nf_orthogonalize", ORTH, {"work": None}, E),
    ("nf_orthogonalize", ORTH, {"work": P + 16}, E), ("nf_orthogonalize", ORTH, {"bytes": 100}, S),
    ("nf_muon_step", MUON, {"wd": nf.NF_BF16}, E), ("nf_muon_step", MUON, {"gd": nf.NF_F16}, E),
    ("nf_muon_step", MUON, {"eta": -1.0}, E), ("nf_muon_step", MUON, {"eta": NAN}, E),
    ("nf_muon_step", MUON, {"momentum": 1.0}, E), ("nf_muon_step", MUON, {"momentum": NAN}, E),
    ("nf_muon_step", MUON, {"decay": -0.1}, E), ("nf_muon_step", MUON, {"nesterov": 2}, E),
    ("nf_muon_step", MUON, {"m": None}, E), ("nf_muon_step", MUON, {"g": None}, E),
    ("nf_muon_step", MUON, {"wo": P + 4}, E), ("nf_muon_step", MUON, {"mo": 2 * P + 4}, E),
    ("nf_muon_step", MUON, {"mo": 3 * P}, E), ("nf_muon_step", MUON, {"mo": P}, E),
    ("nf_muon_step", MUON, {"bytes": 0}, S), ("nf_muon_step", MUON, {"rows": 0}, E),
    ("nf_quantize_rows", QUANT, {"dtype": nf.NF_F64}, E), ("nf_quantize_rows", QUANT, {"ldq": 24}, S),
    ("nf_quantize_rows", QUANT, {"ldq": 16}, S), ("nf_quantize_rows", QUANT, {"ld": 16}, S),
    ("nf_quantize_rows", QUANT, {"cols": 131072, "ld": BIG, "ldq": 131072}, S),
    ("nf_quantize_rows", QUANT, {"q": None}, E), ("nf_quantize_rows", QUANT, {"scale": None}, E),
    ("nf_quantize_rows", QUANT, {"q": 2 * P + 8}, E), ("nf_quantize_rows", QUANT, {"q": P}, E),
    ("nf_linear_i8", LIN, {"act": 5}, E), ("nf_linear_i8", LIN, {"act": -2}, E),
    ("nf_linear_i8", LIN, {"inputs": 0}, E), ("nf_linear_i8", LIN, {"inputs": 131072, "ldx": 131072, "ldw": 131072}, S),
    ("nf_linear_i8", LIN, {"ldx": 16}, S), ("nf_linear_i8", LIN, {"ldw": 40}, S), ("nf_linear_i8", LIN, {"ldy": 4}, S),
    ("nf_linear_i8", LIN, {"wq": 2 * P + 4}, E), ("nf_linear_i8", LIN, {"xq": P + 4}, E),
    ("nf_linear_i8", LIN, {"xs": None}, E), ("nf_linear_i8", LIN, {"ws": None}, E), ("nf_linear_i8", LIN, {"y": None}, E),
    ("nf_linear_i8", LIN, {"yd": nf.NF_F64}, E), ("nf_linear_i8", LIN, {"y": P}, E),
    ("nf_linear_i8_dynamic", DYN, {"xd": nf.NF_F64}, E), ("nf_linear_i8_dynamic", DYN, {"ldx": 16}, S),
    ("nf_linear_i8_dynamic", DYN, {"x": None}, E), ("nf_linear_i8_dynamic", DYN, {"work": None}, E),
    ("nf_linear_i8_dynamic", DYN, {"bytes": 10}, S), ("nf_linear_i8_dynamic", DYN, {"y": P}, E),
    ("nf_linear_i8_dynamic", DYN, {"rows": -1}, E),
])
def test_refusals(name, base, change, status):
    assert _call(name, base, change) == status, nf.nf_last_error()
    assert nf.nf_last_error() != ""


@pytest.mark.parametrize("name,base", [
    ("nf_logprobs", {**LOGP, "rows": 0}), ("nf_logprobs_train", {**TRAIN, "rows": 0}),
    ("nf_logprobs_grad", {**GRAD, "rows": 0}), ("nf_orthogonalize", {**ORTH, "count": 0}),
    ("nf_muon_step", {**MUON, "count": 0}), ("nf_quantize_rows", {**QUANT, "rows": 0}),
    ("nf_linear_i8", {**LIN, "rows": 0}), ("nf_linear_i8_dynamic", {**DYN, "rows": 0})])
def test_nothing_to_do_is_no_error(name, base):
    assert _call(name, base, {}) == nf.NF_OK, nf.nf_last_error()


def test_workspace_sizes():
    lib = nf.raw()
    assert lib.nf_orthogonalize_work(nf.NF_F16, 1, 4, 4) == -1 and nf.nf_last_error() != ""
    assert lib.nf_orthogonalize_work(nf.NF_F32, 1, 0, 4) == -1
    assert lib.nf_orthogonalize_work(nf.NF_F32, 0, 4, 4) == 0
    assert lib.nf_logprobs_work(nf.NF_F64, 1, 10, 0, 0) == -1 and lib.nf_logprobs_work(nf.NF_F32, 1, 10, 65, 0) == -1
    assert lib.nf_logprobs_work(nf.NF_F32, 1000, 131072, 5, 0) == 0 and lib.nf_logprobs_work(nf.NF_F32, 1, 1000, 5, 0) == 0
    assert lib.nf_logprobs_work(nf.NF_F32, 1, 131072, 5, 0) > 0 and lib.nf_logprobs_work(nf.NF_F32, 0, 131072, 5, 1) == 0
    one = lib.nf_orthogonalize_work(nf.NF_F32, 1, 30, 784)
    assert one > 0 and lib.nf_orthogonalize_work(nf.NF_F32, 5, 30, 784) == 5 * one
    assert lib.nf_orthogonalize_work(nf.NF_F32, 1, 784, 30) == one
    assert lib.nf_linear_i8_work(0, 1) == 0 and lib.nf_linear_i8_work(1, 131072) == -1
    assert lib.nf_linear_i8_work(3, 17) >= 3 * 32 + 12


def test_tensors_must_be_on_the_gpu():
    import torch
    x = torch.zeros(2, 3)
    with pytest.raises(ValueError):
        nf.nf_logprobs(x)
    with pytest.raises(ValueError):
        nf.nf_orthogonalize(x, x)
    with pytest.raises(TypeError):
        nf.nf_logprobs([1.0])


def test_tensors_for_another_stream_must_be_on_the_gpu():
    import torch
    with pytest.raises(ValueError):
        nf.nf_orthogonalize(torch.zeros(70, 80), torch.zeros(70, 80), stream=0)
    with pytest.raises(ValueError):
        nf.nf_orthogonalize(torch.zeros(70), torch.zeros(70), stream=0)
    for bad in ([1.0], None):
        with pytest.raises(TypeError):
            nf.nf_logprobs(bad, stream=0)
