"""Cases of the operators for the last layers of a language model or classifier:
log probabilities with their gradient, orthogonalised updates of weight
matrices, and linear layers in 8-bit integers.

A case names one call (``op``):

* ``score``: log probabilities of the targets, entropies and the largest
  alternatives of every row of logits (nf_logprobs);
* ``loss``: a training step's log probabilities and entropies with the gradient
  of a weighted sum of them, the weights known beforehand (nf_logprobs_train);
* ``grad``: the same gradient where the weights come from elsewhere, from the
  statistics that an earlier nf_logprobs kept (nf_logprobs_grad);
* ``orth``: a stack of matrices orthogonalised (nf_orthogonalize);
* ``muon``: a step of momentum, orthogonalisation and update of a stack of
  weight matrices (nf_muon_step);
* ``linear``: a linear layer on float rows, weights in 8 bits with a scale for
  each channel, the rows quantised with a scale for each (nf_linear_i8_dynamic).

``pad`` values lie between the rows of logits and outputs, as where a wider
buffer holds them.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
QUINTIC = (3.4445, -4.7750, 2.0315)
ACTS = ("none", "relu", "sigmoid", "tanh")


# -- the cases ---------------------------------------------------------------
def _logits(name, op, rows, classes, dtype, top=0, masked=False, entropy=False, scale=1.0, pad=0):
    c = {"op": op, "rows": rows, "classes": classes, "dtype": dtype, "top": top, "masked": masked,
         "entropy": entropy, "scale": scale, "pad": pad}
    return {"name": name, **c} if name else c


def _matrices(name, op, count, rows, cols, dtype, batch, weights="f32"):
    c = {"op": op, "count": count, "rows": rows, "cols": cols, "dtype": dtype, "batch": batch,
         "weights": weights}
    return {"name": name, **c} if name else c


def _linear(name, rows, inputs, outputs, dtype, act="none", bias=True):
    c = {"op": "linear", "rows": rows, "inputs": inputs, "outputs": outputs, "dtype": dtype,
         "act": act, "bias": bias}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one answered token: its log probability and five alternatives, pure latency
        _logits("score-1x32768-bf16", "score", 1, 32768, "bf16", top=5),
        # the held-out digits of the classifier workloads, three guesses each
        _logits("score-10000x10-f32", "score", 10000, 10, "f32", top=3),
        # scored text over an odd vocabulary, a part of which may not be answered
        _logits("score-2049x50021-bf16", "score", 2049, 50021, "bf16", top=8, masked=True, pad=3),
        # a training step's loss and gradient over a batch of tokens
        _logits("loss-4096x32768-bf16", "loss", 4096, 32768, "bf16"),
        # a gradient whose weights depend on the log probabilities, with an entropy term
        _logits("grad-1001x5003-f32", "grad", 1001, 5003, "f32", entropy=True, scale=0.7),
        # the hidden weights of the smallest workload
        _matrices("muon-30x784-f32", "muon", 1, 30, 784, "f32", 1000),
        # the first weights of the three-layer workload, more rows than columns
        _matrices("muon-1024x784-f32", "muon", 1, 1024, 784, "f32", 4096),
        # four odd-sized gradients in half the bits
        _matrices("orth-4x517x1001-bf16", "orth", 4, 517, 1001, "bf16", 3003),
        # the widest workload's square weights
        _matrices("muon-4096x4096-f32", "muon", 1, 4096, 4096, "f32", 8192),
        # one token through a wide layer, bound by the weights' bytes
        _linear("linear-1x4096x4096-bf16", 1, 4096, 4096, "bf16"),
        # the held-out samples through the first layer of the three-layer workload
        _linear("linear-10000x784x1024-f32", 10000, 784, 1024, "f32", act="relu"),
        # a batch through a hidden layer of the widest workload
        _linear("linear-8192x4096x4096-bf16", 8192, 4096, 4096, "bf16", act="relu"),
    ]


def _spread(rng, low, high):
    """A whole number of low .. high, uniform in its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    n = min(high, max(low, n))
    return n - 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(("score", "score", "loss", "grad", "orth", "muon", "muon", "linear", "linear", "linear"))
    if op in ("score", "loss", "grad"):
        dtype = rng.choice(("f32", "bf16", "f16"))
        classes = _spread(rng, 2, 131072)
        # at most the values of the largest listed loss in the same bytes
        most = (4096 * 32768 * 2) // (classes * (4 if dtype == "f32" else 2))
        rows = _spread(rng, 1, max(1, min(16384, most)))
        return _logits(None, op, rows, classes, dtype,
                       top=rng.choice((0, 1, 5, 8, 20)) if op == "score" and classes >= 20 else 0,
                       masked=rng.random() < 0.4 and classes >= 8,
                       entropy=op != "score" and rng.random() < 0.5,
                       scale=rng.choice((1.0, 0.7, 1.25)), pad=rng.choice((0, 0, 1, 8)))
    if op in ("orth", "muon"):
        rows, cols = _spread(rng, 8, 4096), _spread(rng, 8, 4096)
        small, large = min(rows, cols), max(rows, cols)
        count = max(1, min(rng.choice((1, 1, 1, 2, 4, 8)), 4096 ** 3 // (small * small * large)))
        dtype = rng.choice(("f32", "bf16"))
        weights = "f32" if dtype == "f32" or op == "orth" else rng.choice(("f32", "bf16"))
        return _matrices(None, op, count, rows, cols, dtype, min(8192, 2 * large), weights)
    inputs, outputs = _spread(rng, 16, 8192), _spread(rng, 10, 8192)
    rows = _spread(rng, 1, max(1, min(16384, 8192 * 4096 * 4096 // (inputs * outputs))))
    return _linear(None, rows, inputs, outputs, rng.choice(("f32", "bf16", "f16")),
                   act=rng.choice(ACTS), bias=rng.random() < 0.7)


# -- what a program has in hand ----------------------------------------------
def _prepare_logits(c, gen):
    rows, classes, dt = c["rows"], c["classes"], DTYPES[c["dtype"]]
    wide = torch.empty((rows, classes + c["pad"]), dtype=dt, device=DEV)
    wide.normal_(generator=gen).mul_(3.0)
    x = wide[:, :classes]
    targets = torch.randint(0, classes, (rows,), generator=gen, device=DEV)
    if c["masked"]:
        # classes that may not be answered (the same for all rows, but never a
        # target), and rows without a target
        out = torch.rand((classes,), generator=gen, device=DEV) < 0.25
        out[targets] = False
        x.masked_fill_(out, float("-inf"))
        targets[torch.rand((rows,), generator=gen, device=DEV) < 0.1] = -1
    s = {"x": x, "targets": targets, "top": c["top"], "scale": c["scale"],
         "logp": torch.empty((rows,), device=DEV), "entropy": torch.empty((rows,), device=DEV)}
    if c["op"] == "score":
        s["ids"] = torch.empty((rows, c["top"]), dtype=torch.int32, device=DEV)
        s["alt"] = torch.empty((rows, c["top"]), device=DEV)
    else:
        # a mean of negative log probabilities, some tokens weighing more
        s["g"] = (torch.rand((rows,), generator=gen, device=DEV) + 0.5).mul_(-1.0 / rows)
        s["h"] = torch.full((rows,), -0.01 / rows, device=DEV) if c["entropy"] else None
        s["dx"] = torch.empty((rows, classes + c["pad"]), dtype=dt, device=DEV)[:, :classes]
    if c["op"] == "grad":
        # the statistics of the earlier pass: maximum and logarithm of the sum
        z = x.float() * c["scale"]
        top = z.amax(1, keepdim=True)
        e = (z - top).exp()
        total = e.sum(1)
        s["stat"] = torch.stack((top[:, 0], total.log()), 1).contiguous()
        s["entropy"] = total.log() - (e * (z - top).clamp_min(-1e30)).sum(1) / total
    return s


def _gradient(c, gen):
    """Sums over a batch of the products of deltas and (positive) activations."""
    shape = (c["count"], c["batch"])
    delta = torch.randn(shape + (c["rows"],), generator=gen, device=DEV)
    act = torch.randn(shape + (c["cols"],), generator=gen, device=DEV).relu_()
    return torch.matmul(delta.transpose(1, 2).contiguous(), act) / c["batch"]


def _prepare_matrices(c, gen):
    g = _gradient(c, gen).to(DTYPES[c["dtype"]])
    s = {"g": g}
    if c["op"] == "muon":
        wt = DTYPES[c["weights"]]
        s["w"] = (torch.randn(g.shape, generator=gen, device=DEV) / math.sqrt(c["cols"])).to(wt)
        s["m"] = _gradient(c, gen) * 5.0
        s["w_out"], s["m_out"] = torch.empty_like(s["w"]), torch.empty_like(s["m"])
        s["rates"] = {"eta": 0.02, "momentum": 0.95, "decay": 0.1}
    else:
        s["out"] = torch.empty_like(g)
    return s


def _prepare_linear(c, gen):
    rows, n_in, n_out, dt = c["rows"], c["inputs"], c["outputs"], DTYPES[c["dtype"]]
    x = torch.randn((rows, n_in), generator=gen, device=DEV)
    if c["act"] == "relu":
        x.relu_()                      # a hidden layer's inputs
    w = torch.randn((n_out, n_in), generator=gen, device=DEV) / math.sqrt(n_in)
    scale = w.abs().amax(1) / 127.0
    wq = torch.zeros((n_out, (n_in + 15) // 16 * 16), dtype=torch.int8, device=DEV)
    wq[:, :n_in] = (w / scale[:, None]).round_().clamp_(-127, 127).to(torch.int8)
    return {"x": x.to(dt), "wq": wq, "scale": scale, "act": c["act"],
            "bias": torch.randn((n_out,), generator=gen, device=DEV) if c["bias"] else None,
            "y": torch.empty((rows, n_out), dtype=dt, device=DEV)}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    op = case["op"]
    make = _prepare_logits if op in ("score", "loss", "grad") else _prepare_linear if op == "linear" else _prepare_matrices
    return {"op": op, **make(case, gen)}


# -- one pass ----------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _own_score(s):
    from paper_1902_06714_amd import nf
    ids, alt = (s["ids"], s["alt"]) if s["top"] else (None, None)
    nf.nf_logprobs(s["x"], s["targets"], logp=s["logp"], entropy=s["entropy"], top_ids=ids, top_logp=alt,
                   scale=s["scale"])
    return (s["logp"], s["entropy"]) + ((ids, alt) if s["top"] else ())


def _own_loss(s):
    from paper_1902_06714_amd import nf
    nf.nf_logprobs_train(s["x"], s["targets"], s["g"], s["h"], s["dx"], logp=s["logp"], entropy=s["entropy"],
                         scale=s["scale"])
    return s["logp"], s["entropy"], s["dx"]


def _own_grad(s):
    from paper_1902_06714_amd import nf
    nf.nf_logprobs_grad(s["x"], s["targets"], s["stat"], s["entropy"], s["g"], s["h"], s["dx"],
                        scale=s["scale"])
    return s["dx"]


def _own_orth(s):
    from paper_1902_06714_amd import nf
    nf.nf_orthogonalize(s["g"], s["out"])
    return s["out"]


def _own_muon(s):
    from paper_1902_06714_amd import nf
    nf.nf_muon_step(s["w"], s["m"], s["g"], s["w_out"], s["m_out"], **s["rates"])
    return s["w_out"], s["m_out"]


def _own_linear(s):
    from paper_1902_06714_amd import nf
    nf.nf_linear_i8_dynamic(s["x"], s["wq"], s["scale"], s["y"], bias=s["bias"],
                            act=None if s["act"] == "none" else s["act"])
    return s["y"]


_own = {"score": _own_score, "loss": _own_loss, "grad": _own_grad, "orth": _own_orth, "muon": _own_muon,
        "linear": _own_linear}


def _softmax_parts(s):
    z = s["x"].float() * s["scale"]
    d = z - z.amax(1, keepdim=True)
    e = d.exp()
    total = e.sum(1, keepdim=True)
    ln = total.log()
    d = d.clamp_min(-1e30)             # a masked class adds 0 times it to the entropy
    entropy = ln - (e * d).sum(1, keepdim=True) / total
    t = s["targets"]
    logp = d.gather(1, t.clamp_min(0)[:, None]) - ln
    return z, d, e, total, ln, entropy, torch.where(t >= 0, logp[:, 0], 0.0)


def _plain_score(s):
    z, d, e, total, ln, entropy, logp = _softmax_parts(s)
    if not s["top"]:
        return logp, entropy[:, 0]
    # whole numbers in the order of the values, the lower index first among equals
    bits = (z + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64)
    last = z.shape[1] - 1
    order = order * (1 << 20) + torch.arange(last, -1, -1, device=z.device)
    ids = last - torch.topk(order, s["top"], dim=1, sorted=True).values % (1 << 20)
    return logp, entropy[:, 0], ids.to(torch.int32), (z - z.amax(1, keepdim=True)).gather(1, ids) - ln


def _gradient_of(s, d, p, ln, entropy):
    g = torch.where(s["targets"] >= 0, s["g"], 0.0)[:, None]
    dz = -g * p
    dz.scatter_add_(1, s["targets"].clamp_min(0)[:, None], g)
    if s["h"] is not None:
        dz = dz - s["h"][:, None] * p * (d - ln + entropy)
    return (dz * s["scale"]).to(s["x"].dtype)


def _plain_loss(s):
    z, d, e, total, ln, entropy, logp = _softmax_parts(s)
    return logp, entropy[:, 0], _gradient_of(s, d, e / total, ln, entropy)


def _plain_grad(s):
    d = (s["x"].float() * s["scale"] - s["stat"][:, :1]).clamp_min(-1e30)
    ln = s["stat"][:, 1:]
    return _gradient_of(s, d, (d - ln).exp(), ln, s["entropy"][:, None])


def _newton_schulz(x):
    a, b, c = QUINTIC
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / x.square().sum((1, 2), keepdim=True).sqrt().clamp_min(1e-30)
    for _ in range(5):
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _plain_orth(s):
    return _newton_schulz(s["g"].float()).to(s["g"].dtype)


def _plain_muon(s):
    r, g = s["rates"], s["g"].float()
    m = r["momentum"] * s["m"] + g
    o = _newton_schulz(g + r["momentum"] * m)
    size = math.sqrt(max(1.0, g.shape[1] / g.shape[2]))
    w = s["w"].float() * (1.0 - r["eta"] * r["decay"]) - (r["eta"] * size) * o
    return w.to(s["w"].dtype), m


def _activate(z, act):
    return z if act == "none" else z.relu() if act == "relu" else torch.tanh(z) if act == "tanh" else 1.0 / (1.0 + (-z).exp())


def _plain_linear(s):
    x = s["x"].float()
    most = x.abs().amax(1, keepdim=True)
    full = torch.full_like(most, 127.0)
    q = torch.round(x * (full / most.clamp_min(1e-30))).clamp(-127.0, 127.0)
    acc = torch.matmul(q, s["wq"][:, : x.shape[1]].float().t().contiguous())
    z = acc * (most / full) * s["scale"]
    if s["bias"] is not None:
        z = z + s["bias"]
    return _activate(z, s["act"]).to(s["x"].dtype)


_plain = {"score": _plain_score, "loss": _plain_loss, "grad": _plain_grad, "orth": _plain_orth, "muon": _plain_muon,
          "linear": _plain_linear}


# -- what a pass cannot do without --------------------------------------------
def work(case):
    c, op = case, case["op"]
    if op in ("score", "loss", "grad"):
        size = 4 if c["dtype"] == "f32" else 2
        values = c["rows"] * c["classes"]
        passes = 1 if op == "score" else 2
        return {"bytes": values * size * passes + c["rows"] * (16 + 8 * c["top"]), "flops": 8.0 * values}
    if op in ("orth", "muon"):
        m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        # the two symmetric products need half their entries
        flops = 5.0 * (3.0 * m * m * n + 1.0 * m * m * m)
        size, ws = (4 if c[k] == "f32" else 2 for k in ("dtype", "weights"))
        per = 2 * size if op == "orth" else size + 2 * ws + 8
        return {"bytes": c["count"] * m * n * per, "flops": c["count"] * flops}
    size = 4 if c["dtype"] == "f32" else 2
    return {"bytes": c["rows"] * (c["inputs"] + c["outputs"]) * size + c["outputs"] * (c["inputs"] + 8),
            "flops": 2.0 * c["rows"] * c["inputs"] * c["outputs"]}


# -- the definitions in 64 bits ----------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op in ("score", "loss", "grad"):
        return _exact_logits(s)
    if op == "linear":
        return _exact_linear(s)
    return _exact_matrices(s)


def _exact_logits(s):
    x = s["x"].double() * s["scale"]
    logp_all = torch.log_softmax(x, 1)
    p = logp_all.exp()
    entropy = -torch.where(p > 0, p * logp_all, 0.0).sum(1)
    has = s["targets"] >= 0
    t = torch.where(has, s["targets"], 0)
    rows = torch.arange(x.shape[0], device=x.device)
    logp = torch.where(has, logp_all[rows, t], 0.0)
    if s["op"] == "score":
        if not s["top"]:
            return logp, entropy
        best = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, : s["top"]]
        return logp, entropy, best.to(torch.int32), logp_all.gather(1, best)
    g = torch.where(has, s["g"].double(), 0.0)
    if s["op"] == "grad":                 # from the statistics as they were given
        logp_all = x - s["stat"].double().sum(1, keepdim=True)
        p, entropy = logp_all.exp(), s["entropy"].double()
    dz = -g[:, None] * p
    dz[rows, t] += g
    if s["h"] is not None:
        dz -= s["h"].double()[:, None] * torch.where(p > 0, p * (logp_all + entropy[:, None]), 0.0)
    dz *= s["scale"]
    return dz if s["op"] == "grad" else (logp, entropy, dz)


def _exact_matrices(s):
    u, muon = s["g"].double(), s["op"] == "muon"
    if muon:
        r = s["rates"]
        m = r["momentum"] * s["m"].double() + u
        u = u + r["momentum"] * m
    x = u / torch.linalg.matrix_norm(u, keepdim=True)
    for _ in range(5):
        # X (a + b X^T X + c (X^T X)^2), on the shorter side
        short = x.shape[1] <= x.shape[2]
        xt = x.transpose(1, 2).contiguous()
        gram = torch.matmul(x, xt) if short else torch.matmul(xt, x)
        poly = QUINTIC[1] * gram + QUINTIC[2] * torch.matmul(gram, gram)
        x = QUINTIC[0] * x + (torch.matmul(poly, x) if short else torch.matmul(x, poly))
    if not muon:
        return x
    rows, cols = x.shape[1:]
    w = s["w"].double() * (1.0 - r["eta"] * r["decay"]) - r["eta"] * math.sqrt(max(1.0, rows / cols)) * x
    return w, m


def _exact_linear(s):
    x = s["x"]
    most = x.abs().amax(1, keepdim=True).float()
    factor = torch.full_like(most, 127.0) / most.clamp_min(1e-30)
    q = torch.round(x.float() * factor).double()      # the operator's own rounding to 8 bits
    y = torch.matmul(q, s["wq"][:, : x.shape[1]].double().t().contiguous())
    y = y * (most.double() / 127.0) * s["scale"].double()
    if s["bias"] is not None:
        y = y + s["bias"].double()
    return torch.relu(y) if s["act"] == "relu" else torch.sigmoid(y) if s["act"] == "sigmoid" else torch.tanh(y) if s["act"] == "tanh" else y
