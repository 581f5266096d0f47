"""The operators on the GPU against their fp64 reference (oracle.operators), at the
sizes, masks, pitches and values where they can go wrong.

Tolerances (u = 2^-24, one fp32 rounding; ut, the output type's):

* log probabilities and entropies: exp(d) is formed with |d| + 2 roundings' relative
  error and the sum of V terms with at most 150, so log s is within
  (E|d| + 152) 2 u, and z - m and the last difference are rounded once each:
  TOL_LOGP = 1e-5 + 2.4e-7 (|z_t - m| + log s); the entropy, a sum of p d with the
  same errors, within three times that on its own size.
* gradient: p within 2e-5 of itself (the above, once more through exp), so
  |scale| p (|g| + |h| (|log p| + H + 1)) 2e-5, the rounding of g (1 - p), 4 u |scale g|
  at the target, and ut of the result (fp16: at least half a subnormal step).
* orthogonalisation in fp32: 15 roundings of 2^-22 (pairs of parts), grown by up to
  4: 2e-5 of the norm; where singular values are missing they grow by 485 over a
  norm of at least 1: 1.5e-4.  bf16: 2^-9 of the result and 15 roundings of
  2^-12 grown by up to 1.5: 6e-3.
* weights: bf16 2^-8 of themselves; fp32 1e-6 and eta times the orthogonalisation's.
* quantised rows and scales: equal.  Linear layers: 4 roundings of u on each
  term's size, 4 u for the activation, whose slope is at most 1, and ut.
"""

import numpy as np
import pytest

from oracle import operators as ref

from .gpu_run import note, torch_cuda

pytestmark = pytest.mark.gpu

U_OF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _dt(name):
    torch = torch_cuda()
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _nf():
    from paper_1902_06714_amd import nf
    return nf


def _dev(a, dtype=None, pad=0, shift=0):
    """A GPU tensor whose rows lie pad elements apart, beginning `shift` elements
    into its allocation; the gaps hold NaN (int8: 77)."""
    torch = torch_cuda()
    t = torch.as_tensor(np.ascontiguousarray(a))
    if dtype is not None:
        t = t.to(dtype)
    if not pad and not shift:
        return t.cuda()
    rows, cols = t.shape
    fill = float("nan") if t.is_floating_point() else 77
    buf = torch.full((rows * (cols + pad) + shift,), fill, dtype=t.dtype, device="cuda")
    v = buf[shift:].view(rows, cols + pad)[:, :cols]
    v.copy_(t)
    return v


def _empty(shape, dtype, fill=None):
    torch = torch_cuda()
    return torch.full(shape, 12345 if fill is None else fill, dtype=dtype, device="cuda")


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _same(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], want[inf]), f"{what}: infinities"
    ok = np.isfinite(want)
    if ok.any():
        off = np.abs(got - want)[ok] / np.broadcast_to(tol, want.shape)[ok]
        assert off.max() <= 1.0, f"{what}: {off.max():.3g} of the tolerance"


# -- log probabilities ----------------------------------------------------------
def _logits(rng, rows, classes, kind):
    x = rng.normal(0, 3, (rows, classes))
    if kind == "masked":
        x[rng.random((rows, classes)) < 0.3] = -np.inf
        if rows > 2:
            x[1] = -np.inf                        # a row that nothing is left of
            x[2] = -np.inf
            x[2, classes // 2] = 0.5              # and one with a single class
    elif kind == "lowest":
        x[rng.random((rows, classes)) < 0.5] = -65504.0
        if rows > 1:
            x[1] = -65504.0
    elif kind == "ties":
        x = np.round(x)
        x[0] = 1.0                                # more equal values than any list holds
    elif kind == "signs":
        x = np.where(rng.random((rows, classes)) < 0.5, 0.0, -0.0)
    elif kind == "bad":
        x[0, classes // 3] = np.nan
        if rows > 1:
            x[1, classes - 1] = np.inf
        if rows > 2:
            x[2] = np.nan
        if rows > 3:
            x[3] = -np.inf
            x[3, 0] = np.nan
    elif kind == "large":
        x *= 50.0
    return x


def _logp_tol(z, stat):
    d = np.abs(z - np.where(np.isfinite(stat[:, :1]), stat[:, :1], 0.0))
    ln = np.abs(np.where(np.isfinite(stat[:, 1:]), stat[:, 1:], 0.0))
    return 1e-5 + 2.4e-7 * (np.where(np.isfinite(d), d, 0.0) + ln)


def _check_logprobs(dtype, rows, classes, kind, n_top, pad, shift, scale, targets="some", grad=True):
    torch = torch_cuda()
    nf = _nf()
    rng = np.random.default_rng(rows * 7919 + classes * 31 + n_top)
    note(f"logprobs {dtype} {rows}x{classes} {kind} top={n_top} pad={pad} shift={shift} scale={scale}")
    x = _dev(_logits(rng, rows, classes, kind), _dt(dtype), pad, shift)
    xh = _np(x)
    t = rng.integers(0, classes, rows)
    if targets == "some" and rows > 4:
        t[3], t[4] = -1, classes
    td = _dev(t)
    out = {k: _empty(s, torch.float32) for k, s in (("logp", (rows,)), ("entropy", (rows,)), ("stat", (rows, 2)))}
    ids = _empty((rows, n_top), torch.int32) if n_top else None
    alt = _empty((rows, n_top), torch.float32) if n_top else None
    nf.nf_logprobs(x, td, out["logp"], out["entropy"], out["stat"], ids, alt, scale=scale)
    torch.cuda.synchronize()
    logp, ent, stat, rid, ralt = ref.logprobs(xh, scale, t, n_top)
    z = ref.scaled(xh, scale)
    zt = np.where((t >= 0) & (t < classes), z[np.arange(rows), np.clip(t, 0, classes - 1)], 0.0)
    logp_tol = _logp_tol(zt[:, None], stat)[:, 0]
    _same(_np(out["logp"]), logp, logp_tol, "logp")
    ent_tol = 3 * (1e-5 + 2.4e-7 * np.nan_to_num(np.abs(stat[:, 1]), posinf=0.0)) * (1 + np.nan_to_num(ent))
    _same(_np(out["entropy"]), ent, ent_tol, "entropy")
    bad = np.isnan(stat[:, 1])                    # of a NaN row only log s is told
    got = _np(out["stat"])
    _same(got[~bad], stat[~bad], 1e-5 + 1.2e-7 * np.abs(np.nan_to_num(stat[~bad], neginf=0.0)), "stat")
    assert np.isnan(got[bad, 1]).all()
    if n_top:
        assert np.array_equal(ids.cpu().numpy(), rid), "alternatives"
        _same(_np(alt), ralt, _logp_tol(np.take_along_axis(z, rid.astype(np.int64), 1), stat), "their logp")
    if not grad:
        return
    g, h = rng.normal(0, 1, rows).astype(np.float32), rng.normal(0, 1, rows).astype(np.float32)
    gd, hd = _dev(g), _dev(h)
    m, ln, p, lp, _ = ref._rows(z)
    for use_h in (False, True):
        want = ref.logprobs_grad(xh, scale, t, g, h if use_h else None)
        with np.errstate(all="ignore"):
            slope = np.abs(g)[:, None] + (np.abs(h)[:, None] * (np.abs(np.where(p > 0, lp, 0)) + np.nan_to_num(ent)[:, None] + 1)
                                          if use_h else 0)
            tol = 2e-5 * scale * np.nan_to_num(p) * slope + U_OF[dtype] * np.abs(np.nan_to_num(want)) + 2.0 ** -25
        tol[np.arange(rows), np.clip(t, 0, classes - 1)] += 4 * 2.0 ** -24 * scale * np.abs(g)
        for how in ("train", "grad", "over"):
            dx = x if how == "over" else _dev(np.zeros((rows, classes)), _dt(dtype), pad + 1)
            if how == "over":
                dx = _dev(xh, _dt(dtype), pad, shift)
            if how == "grad":
                nf.nf_logprobs_grad(x, td, out["stat"], out["entropy"] if use_h else None, gd, hd if use_h else None,
                                    dx, scale=scale)
            else:
                l2, e2 = _empty((rows,), torch.float32), _empty((rows,), torch.float32)
                nf.nf_logprobs_train(dx if how == "over" else x, td, gd, hd if use_h else None, dx, l2, e2,
                                     scale=scale)
                torch.cuda.synchronize()
                _same(_np(l2), logp, logp_tol, f"logp ({how})")
                _same(_np(e2), ent, ent_tol, f"entropy ({how})")
            torch.cuda.synchronize()
            _same(_np(dx), want, tol, f"gradient ({how}, entropies {use_h})")


KINDS = ["plain", "masked", "lowest", "ties", "signs", "bad", "large"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("classes,n_top", [(1, 1), (2, 2), (10, 3), (17, 17), (33, 8), (65, 64), (128, 5), (129, 64),
                                           (300, 7), (1031, 20), (5003, 5)])
def test_logprobs_small(classes, n_top, kind):
    dtype = ["f32", "bf16", "f16"][(classes + len(kind)) % 3]
    _check_logprobs(dtype, 7, classes, kind, n_top, classes % 3, classes % 2, 0.7 if classes % 2 else 1.0)


# the sizes at which a row's vectors, threads and registers change, and past the last
@pytest.mark.parametrize("dtype,classes", [
    ("f32", 256), ("f32", 257), ("f32", 1024), ("f32", 2048), ("f32", 4097), ("f32", 8192), ("f32", 8193),
    ("f32", 16384), ("f32", 16385), ("f32", 32769), ("f32", 65537),
    ("bf16", 512), ("bf16", 2049), ("bf16", 8191), ("bf16", 16385), ("bf16", 32768), ("bf16", 65539), ("bf16", 140001),
    ("f16", 513), ("f16", 4095), ("f16", 32771), ("f16", 131073)])
@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "bad"])
def test_logprobs_long_rows(dtype, classes, kind):
    _check_logprobs(dtype, 5, classes, kind, 9, 1, classes % 2, 1.25, grad=kind in ("plain", "masked", "bad"))


# more rows than compute units, or too many to be cut: other numbers of threads
@pytest.mark.parametrize("rows,dtype,classes,kind", [
    (300, "bf16", 2500, "plain"), (300, "f32", 3000, "masked"), (300, "bf16", 5003, "bad"), (300, "f16", 12000, "plain"),
    (300, "bf16", 32767, "masked"), (300, "f32", 16500, "plain"), (70, "f32", 66001, "plain"), (70, "bf16", 30000, "ties"),
    (300, "f32", 4097, "ties")])
def test_logprobs_many_rows(rows, dtype, classes, kind):
    _check_logprobs(dtype, rows, classes, kind, 0 if classes > 20000 and kind != "ties" else 6, 2, 1, 1.0)


# few rows that are cut, the last slice shorter than the alternatives, and the same rows whole
@pytest.mark.parametrize("rows,dtype,classes,n_top", [
    (1, "bf16", 49152, 1), (1, "bf16", 131072, 64), (2, "f32", 24581, 20), (64, "bf16", 65600, 3), (33, "f16", 131071, 7),
    (1, "f32", 300001, 64), (17, "f32", 65536, 5)])
@pytest.mark.parametrize("kind", ["plain", "ties", "bad"])
def test_logprobs_few_long_rows(rows, dtype, classes, n_top, kind):
    torch, nf = torch_cuda(), _nf()
    if rows * classes <= 1 << 20:
        _check_logprobs(dtype, rows, classes, kind, n_top, 1, 1, 0.7, grad=kind != "ties")
    rng = np.random.default_rng(classes)
    note(f"few long rows {dtype} {rows}x{classes} {kind} top={n_top}")
    x = _dev(_logits(rng, rows, classes, kind), _dt(dtype))
    t = _dev(rng.integers(0, classes, rows))
    code = {"f32": nf.NF_F32, "bf16": nf.NF_BF16, "f16": nf.NF_F16}[dtype]
    assert nf.nf_logprobs_work(code, rows, classes, n_top) > 0
    outs = []
    for whole in (False, True):
        logp, ent, stat = (_empty(s, torch.float32) for s in ((rows,), (rows,), (rows, 2)))
        ids, alt = _empty((rows, n_top), torch.int32), _empty((rows, n_top), torch.float32)
        if whole:
            st = nf.raw().nf_logprobs(x.data_ptr(), code, rows, classes, classes, 1.0, t.data_ptr(), n_top, logp.data_ptr(),
                                      ent.data_ptr(), stat.data_ptr(), ids.data_ptr(), alt.data_ptr(), None, 0,
                                      torch.cuda.current_stream().cuda_stream)
            assert st == nf.NF_OK
        else:
            nf.nf_logprobs(x, t, logp, ent, stat, ids, alt)
        torch.cuda.synchronize()
        outs.append((logp, ent, stat[:, 1], alt, ids))
    assert torch.equal(outs[0][4], outs[1][4])
    for a, b in zip(outs[0][:4], outs[1][:4]):
        _same(_np(a), _np(b), 3e-5, "cut and whole")


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 1001])
@pytest.mark.parametrize("classes", [3, 10, 30, 100])
def test_logprobs_many_short_rows(rows, classes):
    _check_logprobs("f32", rows, classes, "plain", min(3, classes), 0, 0, 1.0)


def test_logprobs_outputs_left_out():
    torch, nf = torch_cuda(), _nf()
    x = _dev(np.random.default_rng(1).normal(0, 1, (5, 400)), torch.float32)
    alt = _empty((5, 4), torch.float32)
    ids = _empty((5, 4), torch.int32)
    note("logprobs without targets or sums")
    nf.nf_logprobs(x, top_logp=alt)
    nf.nf_logprobs(x, top_ids=ids)
    want = ref.logprobs(_np(x), 1.0, None, 4)
    torch.cuda.synchronize()
    assert np.array_equal(ids.cpu().numpy(), want[3])
    _same(_np(alt), want[4], 1e-4, "alternatives")
    dx = torch.empty_like(x)
    h = _dev(np.ones(5, np.float32))
    nf.nf_logprobs_train(x, None, None, h, dx)         # the entropies alone
    torch.cuda.synchronize()
    _same(_np(dx), ref.logprobs_grad(_np(x), 1.0, None, None, np.ones(5)), 1e-4, "gradient of entropies")


def test_logprobs_past_32_bit_offsets():
    torch, nf = torch_cuda(), _nf()
    rows, cols, ld = 40000, 40, 65000                   # 2.6e9 elements
    note("logprobs past 2^31 elements")
    buf = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")
    x = buf[:, 7:7 + cols]
    x.copy_(torch.randn((rows, cols), device="cuda"))
    t = torch.randint(0, cols, (rows,), device="cuda")
    res = []
    for a in (x, x.contiguous()):
        logp, g = _empty((rows,), torch.float32), _empty((rows,), torch.float32, 0.5)
        dx = torch.empty_like(x.contiguous())
        nf.nf_logprobs_train(a, t, g, None, dx, logp)
        stat = _empty((rows, 2), torch.float32)
        nf.nf_logprobs(a, t, stat=stat)
        dx2 = torch.empty_like(dx)
        nf.nf_logprobs_grad(a, t, stat, None, g, None, dx2)
        res.append((logp, dx, dx2))
    torch.cuda.synchronize()
    for p, q in zip(*res):
        assert torch.equal(p, q)


# -- orthogonalised updates --------------------------------------------------------
def _rel(got, want):
    n = np.linalg.norm(want)
    return np.linalg.norm(got - want) / (n if n else 1.0)


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 200), (30, 784), (64, 64), (65, 63), (100, 1), (129, 257), (200, 96),
          (300, 300), (517, 259), (259, 1001), (16, 65), (17, 130), (33, 32), (32, 4100), (48, 49), (49, 1200), (2100, 64),
          (65, 65), (65, 3000), (96, 97)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols, dtype):
    torch, nf = torch_cuda(), _nf()
    rng = np.random.default_rng(rows * 1000 + cols)
    note(f"orthogonalize {dtype} {rows}x{cols}")
    x = _dev(rng.normal(0, 1, (rows, cols)), _dt(dtype), 0 if rows % 2 else 3)
    out = _dev(np.zeros((rows, cols)), _dt(dtype), 5 if cols % 2 else 0)
    nf.nf_orthogonalize(x, out)
    torch.cuda.synchronize()
    got, want = _np(out), ref.orthogonalize(_np(x))
    assert np.isfinite(got).all()
    assert _rel(got, want) <= (2e-5 if dtype == "f32" else 6e-3), _rel(got, want)
    if min(rows, cols) == 1:
        return
    # in place, and the same bits
    nf.nf_orthogonalize(x, x)
    torch.cuda.synchronize()
    assert torch.equal(x, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1100, 1300), (2050, 2100), (4100, 600)])
def test_orthogonalize_larger_tiles(rows, cols, dtype):
    torch, nf = torch_cuda(), _nf()
    note(f"orthogonalize {dtype} {rows}x{cols}")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    x = torch.randn((rows, cols), generator=gen, device="cuda").to(_dt(dtype))
    out = torch.empty_like(x)
    nf.nf_orthogonalize(x, out)
    u = x.double()
    u = u / u.norm()
    u = u if rows <= cols else u.t().contiguous()
    a, b, c = ref.QUINTIC
    for _ in range(ref.STEPS):
        gram = u @ u.t().contiguous()
        u = a * u + (b * gram + c * gram @ gram) @ u
    u = u if rows <= cols else u.t()
    off = ((out.double() - u).norm() / u.norm()).item()
    assert off <= (2e-5 if dtype == "f32" else 6e-3), off


# products of one call in tiles of 32 and of 64, the shorter side no whole tile of either
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(593, 641), (577, 800), (70, 4000), (225, 2100)])
def test_orthogonalize_mixed_tiles(rows, cols, dtype):
    test_orthogonalize(rows, cols, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_orthogonalize_stacks_and_values(dtype):
    """Matrices of a stack do not see one another: one of zeros, one with a NaN, one
    with an infinity, sizes from 1e-30 to 1e30, few singular values, zero rows."""
    torch, nf = torch_cuda(), _nf()
    rng = np.random.default_rng(8)
    u = rng.normal(0, 1, (9, 40, 70))
    u[1] = 0.0
    u[2, 3, 4] = np.nan
    u[3, 39, 69] = np.inf
    u[4] *= 1e-30
    u[5] *= 1e30
    u[6] = rng.normal(0, 1, (40, 2)) @ rng.normal(0, 1, (2, 70))
    u[7, 5:] = 0.0
    note(f"orthogonalize a stack, {dtype}")
    wide = torch.full((9, 43, 77), float("nan"), dtype=_dt(dtype), device="cuda")
    x = wide[:, :40, :70]
    x.copy_(torch.as_tensor(u))
    out = torch.empty((9, 40, 70), dtype=_dt(dtype), device="cuda")
    nf.nf_orthogonalize(x, out)
    torch.cuda.synchronize()
    got, xs = _np(out), _np(x)
    assert not got[1].any() and np.isnan(got[2]).all() and np.isnan(got[3]).all()
    for k in (0, 4, 5, 6, 7, 8):
        tol = (2e-5 if k not in (6, 7) else 1.5e-4) if dtype == "f32" else 6e-3
        if dtype == "bf16" and k in (6, 7):
            tol = 1e-2                            # 485 x 2^-12 x the gap's share of the noise, over a norm above 1
        assert _rel(got[k], ref.orthogonalize(xs[k])) <= tol, (k, _rel(got[k], ref.orthogonalize(xs[k])))
    # a stack's result is the matrices' own
    one = torch.empty((40, 70), dtype=_dt(dtype), device="cuda")
    nf.nf_orthogonalize(x[8], one)
    assert torch.equal(one, out[8])
    turned = torch.empty((70, 40), dtype=_dt(dtype), device="cuda")
    nf.nf_orthogonalize(x[0].t().contiguous(), turned)
    assert _rel(_np(turned).T, got[0]) <= (4e-5 if dtype == "f32" else 8e-3)


@pytest.mark.parametrize("w_dtype,g_dtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("shape", [(30, 784), (2, 257, 129), (1, 33), (70, 20)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step(w_dtype, g_dtype, shape, nesterov):
    torch, nf = torch_cuda(), _nf()
    rng = np.random.default_rng(sum(shape))
    note(f"muon {w_dtype} {g_dtype} {shape} nesterov={nesterov}")
    w, g = _dev(rng.normal(0, 0.1, shape), _dt(w_dtype)), _dev(rng.normal(0, 1, shape), _dt(g_dtype))
    m = _dev(rng.normal(0, 1, shape), torch.float32)
    wo, mo = torch.empty_like(w), torch.empty_like(m)
    eta, mu, decay = 0.05, 0.9, 0.2
    nf.nf_muon_step(w, m, g, wo, mo, eta, mu, nesterov, decay)
    torch.cuda.synchronize()
    three = lambda t: _np(t).reshape((-1,) + tuple(shape[-2:]))  # noqa: E731
    for k in range(three(w).shape[0]):
        f32 = np.float32
        want_w, want_m = ref.muon_step(three(w)[k], three(m)[k], three(g)[k], float(f32(eta)), float(f32(mu)),
                                       nesterov, float(f32(decay)))
        _same(three(mo)[k], want_m, 4 * 2.0 ** -24 * (np.abs(want_m) + np.abs(three(g)[k])), "momentum")
        size = np.sqrt(max(1.0, shape[-2] / shape[-1]))
        if w_dtype == "f32":
            assert np.linalg.norm(three(wo)[k] - want_w) <= 1e-6 * np.linalg.norm(want_w) + 2e-5 * eta * size * \
                np.sqrt(min(shape[-2:]))
        else:
            assert np.linalg.norm(three(wo)[k] - want_w) <= 2.0 ** -8 * np.linalg.norm(want_w) + 6e-3 * eta * size * \
                np.sqrt(min(shape[-2:]))
    # in place, the same bits
    nf.nf_muon_step(w, m, g, w, m, eta, mu, nesterov, decay)
    torch.cuda.synchronize()
    assert torch.equal(w, wo) and torch.equal(m, mo)


# -- linear layers in 8-bit integers ---------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 15), (5, 16), (4, 17), (2, 255), (7, 784), (3, 1001), (2, 2049),
                                       (2, 5003), (1, 16400), (2, 40000), (1, 131071)])
def test_quantize_rows(rows, cols, dtype):
    torch, nf = torch_cuda(), _nf()
    rng = np.random.default_rng(cols)
    note(f"quantize {dtype} {rows}x{cols}")
    xs = rng.normal(0, 2, (rows + 5, cols))
    xs[rows] = 0.0
    xs[rows + 1] *= 1e-41 if dtype == "f32" else 1e-6
    xs[rows + 2, cols // 2] = np.nan
    xs[rows + 3, cols // 2] = -np.inf
    xs[rows + 4] = 3e38 if dtype != "f16" else 65504.0
    x = _dev(xs, _dt(dtype), cols % 3, cols % 2)
    n, wide = rows + 5, (cols + 15) // 16 * 16
    q = torch.full((n, wide + 16), 99, dtype=torch.int8, device="cuda")
    scale = _empty((n,), torch.float32)
    nf.nf_quantize_rows(x, q, scale)
    torch.cuda.synchronize()
    xf = x.float().cpu().numpy()
    want, ws = ref.quantize_rows(xf)
    got, gs = q.cpu().numpy(), scale.cpu().numpy()
    small = np.abs(xf).max(axis=1) < 2.0 ** -100          # scaled up first: held to the value, not the bits
    keep = ~small | ~np.isfinite(np.abs(xf).max(axis=1))
    assert np.array_equal(got[:, :cols][keep], want[keep])
    assert np.array_equal(gs, ws, equal_nan=True)
    for i in np.nonzero(~keep)[0]:
        most = np.abs(xf[i].astype(np.float64)).max()
        r = xf[i].astype(np.float64) * (127.0 / most) if most else np.zeros(cols)
        assert np.abs(got[i, :cols] - r).max() <= 0.5 + 1e-4
    assert not got[:, cols:wide].any() and (got[:, wide:] == 99).all()


def _linear_case(rows, inputs, outputs, x_dtype, y_dtype, act, bias, pad=0, garbage=True):
    torch, nf = torch_cuda(), _nf()
    rng = np.random.default_rng(rows + 3 * inputs + 7 * outputs)
    note(f"linear {rows}x{inputs}->{outputs} {x_dtype} {y_dtype} {act} bias={bias} pad={pad}")
    x = _dev(rng.normal(0, 1, (rows, inputs)), _dt(x_dtype), pad, pad % 2)
    wide = (inputs + 15) // 16 * 16
    wq = np.zeros((outputs, wide), np.int8)
    wq[:, :inputs] = rng.integers(-128, 128, (outputs, inputs))
    ws = rng.uniform(0.5, 2, outputs).astype(np.float32) / (40 * np.sqrt(inputs)).astype(np.float32)
    b = rng.normal(0, 1, outputs).astype(np.float32) if bias else None
    wqd, wsd, bd = _dev(wq, None, 16 if pad else 0), _dev(ws), _dev(b) if bias else None
    y = _dev(np.zeros((rows, outputs)), _dt(y_dtype), pad)
    nf.nf_linear_i8_dynamic(x, wqd, wsd, y, bias=bd, act=act)
    xq, xs = ref.quantize_rows(x.float().cpu().numpy())
    # the same from rows quantised beforehand, whose padding holds anything
    full = rng.integers(-128, 128, (rows, wide)).astype(np.int8) if garbage else np.zeros((rows, wide), np.int8)
    full[:, :inputs] = xq
    y2 = _dev(np.zeros((rows, outputs)), _dt(y_dtype), pad + 1)
    nf.nf_linear_i8(_dev(full), _dev(xs), wqd, wsd, y2, inputs, bias=bd, act=act)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    want = ref.linear_i8(xq, xs, wq[:, :inputs], ws, b, act)
    size = np.abs(ref.linear_i8(xq, xs, wq[:, :inputs], ws)) + (np.abs(b)[None, :] if bias else 0.0)
    u = 2.0 ** -24
    if act == "step":
        ok = size > 1e-4                           # a step within rounding of 0 may fall on either side
        assert np.array_equal(_np(y)[ok], want[ok])
        return
    _same(_np(y), want, 4 * u * size + 4 * u * np.abs(want) + U_OF[y_dtype] * np.abs(want) + 2.0 ** -25, "y")


@pytest.mark.parametrize("rows,inputs,outputs", [
    (1, 1, 1), (1, 16, 10), (1, 784, 30), (1, 4097, 515), (2, 1001, 17), (3, 4096, 100), (4, 16320, 40), (4, 20000, 33),
    (5, 17, 259), (6, 784, 90), (15, 4100, 48), (16, 784, 1024), (17, 100, 64),
    (31, 2049, 33), (33, 1001, 517), (64, 64, 64), (65, 130, 100), (200, 784, 300), (257, 513, 129),
    (1000, 129, 77), (3, 30000, 20), (70, 9000, 70)])
@pytest.mark.parametrize("x_dtype,y_dtype", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
def test_linear(rows, inputs, outputs, x_dtype, y_dtype):
    acts = [None, "relu", "sigmoid", "tanh", "gaussian", "step"]
    k = rows + inputs + outputs
    _linear_case(rows, inputs, outputs, x_dtype, y_dtype, acts[k % 6], k % 3 > 0, k % 4)


@pytest.mark.parametrize("act", [None, "relu", "sigmoid", "tanh", "gaussian", "step"])
@pytest.mark.parametrize("rows", [1, 9, 80])
def test_linear_activations(act, rows):
    _linear_case(rows, 100, 90, "f32", "f32", act, True)


@pytest.mark.parametrize("rows,inputs,outputs", [(2100, 300, 2080), (4200, 129, 4100), (8200, 64, 2050)])
def test_linear_larger_tiles(rows, inputs, outputs):
    _linear_case(rows, inputs, outputs, "bf16", "f32", "relu", True, 3)


# tiles of 64 by two groups of waves, of 64, and of 128 x 192, each past its edges
@pytest.mark.parametrize("rows,inputs,outputs", [(700, 300, 901), (1501, 129, 1300), (4200, 250, 2101)])
@pytest.mark.parametrize("y_dtype", ["f32", "f16"])
def test_linear_middle_tiles(rows, inputs, outputs, y_dtype):
    _linear_case(rows, inputs, outputs, "f32", y_dtype, "tanh", True, 1)


@pytest.mark.parametrize("rows", [1, 3, 40, 300])
def test_linear_rows_that_cannot_be_quantised(rows):
    """A row with a NaN or an infinity is NaN throughout and leaves its neighbours
    alone; one of zeros gives act(b)."""
    torch, nf = torch_cuda(), _nf()
    rng = np.random.default_rng(rows)
    xs = rng.normal(0, 1, (rows, 50)).astype(np.float32)
    kinds = {0: "nan", rows // 2: "inf" if rows > 1 else "nan", rows - 1: "zero" if rows > 2 else "nan"}
    xs[0, 7] = np.nan
    if rows > 1:
        xs[rows // 2, 49] = np.inf
    if rows > 2:
        xs[rows - 1] = 0.0
    wq = np.zeros((20, 64), np.int8)
    wq[:, :50] = rng.integers(-127, 128, (20, 50))
    ws, b = np.full(20, 1e-3, np.float32), rng.normal(0, 1, 20).astype(np.float32)
    note(f"linear with rows that cannot be quantised, {rows}")
    for act in (None, "relu", "step"):
        y = _empty((rows, 20), torch.float32)
        nf.nf_linear_i8_dynamic(_dev(xs), _dev(wq), _dev(ws), y, bias=_dev(b), act=act)
        torch.cuda.synchronize()
        q, s = ref.quantize_rows(xs)
        want = ref.linear_i8(q, s, wq[:, :50], ws, b, act)
        got = _np(y)
        assert np.array_equal(np.isnan(got), np.isnan(want)), kinds
        ok = ~np.isnan(want)
        assert np.abs(got[ok] - want[ok]).max(initial=0.0) < 1e-5


def test_linear_largest_sums():
    """131071 products of -128 and -128: the sum is below 2^31."""
    torch, nf = torch_cuda(), _nf()
    n = 131071
    q = torch.zeros((2, n + 1), dtype=torch.int8, device="cuda")
    q[:, :n] = -128
    one = torch.ones(2, device="cuda")
    y = _empty((2, 2), torch.float32)
    note("largest sums")
    nf.nf_linear_i8(q, one, q, one, y, n)
    assert (y == float(np.float32(n * 16384))).all()


# -- streams, graphs, refusals ---------------------------------------------------------
def _all_calls(seed):
    """Inputs of one call of each operator, and the calls."""
    torch, nf = torch_cuda(), _nf()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, t = r(33, 1000), torch.randint(0, 1000, (33,), generator=gen, device="cuda")
    logp, ent, stat = torch.empty(33, device="cuda"), torch.empty(33, device="cuda"), torch.empty(33, 2, device="cuda")
    ids, alt = torch.empty(33, 6, dtype=torch.int32, device="cuda"), torch.empty(33, 6, device="cuda")
    g, dx, dx2 = r(33), torch.empty_like(x), torch.empty_like(x)
    w, m, gr = r(96, 130), r(96, 130), r(96, 130)
    wo, mo, o = torch.empty_like(w), torch.empty_like(m), torch.empty_like(w)
    q, qs = torch.empty((96, 144), dtype=torch.int8, device="cuda"), torch.empty(96, device="cuda")
    h, y, y1 = r(40, 130), torch.empty(40, 96, device="cuda"), torch.empty(1, 96, device="cuda")
    works = [torch.empty(1 << 20, dtype=torch.uint8, device="cuda") for _ in range(4)]

    def go(stream=None):
        nf.nf_logprobs(x, t, logp, ent, stat, ids, alt, stream=stream)
        nf.nf_logprobs_train(x, t, g, g, dx, stream=stream)
        nf.nf_logprobs_grad(x, t, stat, ent, g, g, dx2, stream=stream)
        nf.nf_orthogonalize(w, o, work=works[0], stream=stream)
        nf.nf_muon_step(w, m, gr, wo, mo, 0.02, work=works[1], stream=stream)
        nf.nf_quantize_rows(w, q, qs, stream=stream)
        nf.nf_linear_i8_dynamic(h, q, qs, y, act="tanh", work=works[2], stream=stream)
        nf.nf_linear_i8_dynamic(h[:1], q, qs, y1, work=works[3], stream=stream)
    return go, (x, w, m, gr, h), (logp, ent, stat, ids, alt, dx, dx2, o, wo, mo, q, qs, y, y1)


def test_a_stream_of_its_own():
    torch = torch_cuda()
    go, _, outs = _all_calls(5)
    note("operators on the current stream")
    go()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    for o in outs:
        o.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    note("operators on a stream of their own")
    go(side)
    side.synchronize()
    for o, e in zip(outs, want):
        assert torch.equal(o, e)


def test_workspace_belongs_to_the_stream(monkeypatch):
    """A workspace for another stream is that stream's memory from the beginning."""
    torch, nf = torch_cuda(), _nf()
    note("workspace of another stream")
    x, out = torch.randn(70, 90, device="cuda"), torch.empty(70, 90, device="cuda")
    torch.cuda.synchronize()
    side, seen, empty = torch.cuda.Stream(), [], torch.empty

    def watched(*a, **k):
        seen.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **k)

    monkeypatch.setattr(torch, "empty", watched)
    nf.nf_orthogonalize(x, out, stream=side)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert seen == [side.cuda_stream]
    want = ref.orthogonalize(_np(x))
    assert np.linalg.norm(_np(out) - want) <= 2e-5 * np.linalg.norm(want)


def test_captured_in_a_graph():
    torch = torch_cuda()
    go, ins, outs = _all_calls(6)
    note("operators in a graph")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for k in range(4):
        for a in ins:
            a.mul_(0.9).add_(0.01 * k)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        go()
        torch.cuda.synchronize()
        for o, e in zip(outs, got):
            assert torch.equal(o, e), k


def test_calls_do_not_depend_on_what_ran_before():
    """The same inputs give the same bits, whatever the workspaces held."""
    torch = torch_cuda()
    go, _, outs = _all_calls(7)
    note("operators twice")
    go()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    other, _, _ = _all_calls(8)
    other()
    go()
    torch.cuda.synchronize()
    for o, e in zip(outs, want):
        assert torch.equal(o, e)


def test_binding_refuses_tensors_that_do_not_fit():
    torch, nf = torch_cuda(), _nf()
    x = torch.zeros((4, 6), device="cuda")
    with pytest.raises(ValueError):
        nf.nf_logprobs(x.t())                             # columns first
    with pytest.raises(ValueError):
        nf.nf_logprobs(x, torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        nf.nf_logprobs(x, logp=torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError):
        nf.nf_logprobs_train(x, None, None, None, torch.zeros((4, 6), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        nf.nf_orthogonalize(x, torch.zeros((6, 4), device="cuda"))
    with pytest.raises(ValueError):
        nf.nf_muon_step(x.t(), x, x, x, x, 0.1)
    with pytest.raises(ValueError):
        nf.nf_linear_i8_dynamic(x, torch.zeros((5, 8), dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda"),
                                torch.zeros((4, 5), device="cuda"))
    with pytest.raises(nf.NfError):
        nf.nf_logprobs(x, top_logp=torch.zeros((4, 7), device="cuda"))
    with pytest.raises(nf.NfError):
        nf.nf_orthogonalize(x, torch.zeros_like(x), work=torch.zeros(16, device="cuda"))
    with pytest.raises(nf.NfError):
        nf.nf_linear_i8_dynamic(x, torch.zeros((5, 16), dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda"),
                                torch.zeros((4, 5), device="cuda"), work=torch.zeros(1, device="cuda"))
