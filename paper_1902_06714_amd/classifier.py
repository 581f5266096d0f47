"""A classifier trained and served with the operators of include/nf.h.

    python -m paper_1902_06714_amd.classifier

A fully connected relu layer (a net of the library) gives features; a linear
layer on top of them is trained on negative log probabilities, its weights moved
by orthogonalised updates; then both layers answer in 8-bit integers, with the
log probability, the entropy and the likeliest alternatives of each answer.  The
data are synthetic: one prototype a class and noise.
"""

from __future__ import annotations

from typing import Dict

import numpy as np

from . import nf


def _data(rng, n: int, inputs: int, classes: int, prototypes: np.ndarray):
    labels = rng.integers(0, classes, n)
    x = 0.5 * prototypes[labels] + rng.normal(0, 1, (n, inputs))
    return x.astype(np.float32), labels


def run(steps: int = 60, batch: int = 1000, inputs: int = 784, hidden: int = 256, classes: int = 10, seed: int = 0,
        say=print) -> Dict[str, float]:
    import torch
    dev = torch.device("cuda", torch.cuda.current_device())
    rng = np.random.default_rng(seed)
    prototypes = rng.normal(0, 1, (classes, inputs))
    x, y = _data(rng, steps * batch, inputs, classes, prototypes)
    xt, yt = _data(rng, 2000, inputs, classes, prototypes)
    xd, yd = torch.from_numpy(x).to(dev), torch.from_numpy(y).to(dev)
    xtd, ytd = torch.from_numpy(xt).to(dev), torch.from_numpy(yt).to(dev)

    # the features: a relu layer with He-normal weights
    net = nf.nf_net_create((inputs, hidden), "relu")
    try:
        w1 = (rng.normal(0, 1, (hidden, inputs)) * np.sqrt(2.0 / inputs)).astype(np.float32)
        b1 = np.zeros(hidden, np.float32)
        nf.nf_set_params(net, np.concatenate([w1.ravel(), b1]))

        # the trained layer, its momentum, and what a step needs
        w = torch.zeros((classes, hidden), device=dev)
        b, m = torch.zeros(classes, device=dev), torch.zeros_like(w)
        h = torch.empty((batch, hidden), device=dev)
        logits, dlogits = (torch.empty((batch, classes), device=dev) for _ in range(2))
        logp, weight = torch.empty(batch, device=dev), torch.full((batch,), -1.0 / batch, device=dev)
        work = torch.empty(nf.nf_orthogonalize_work(nf.NF_F32, 1, classes, hidden), dtype=torch.uint8, device=dev)
        losses = []
        for k in range(steps):
            part = slice(k * batch, (k + 1) * batch)
            nf.nf_forward(net, xd[part], h)
            torch.addmm(b, h, w.t(), out=logits)
            # the mean of -log p, and its gradient with respect to the logits
            nf.nf_logprobs_train(logits, yd[part], weight, None, dlogits, logp=logp)
            g = torch.mm(dlogits.t(), h)
            nf.nf_muon_step(w, m, g, w, m, eta=0.05 * (1.0 - k / steps), work=work)
            b -= 0.5 * dlogits.sum(0)
            losses.append(-logp.mean())
        losses = torch.stack(losses).cpu().numpy()

        # answers in fp32
        ht = torch.empty((xt.shape[0], hidden), device=dev)
        nf.nf_forward(net, xtd, ht)
        full = torch.addmm(b, ht, w.t())
    finally:
        nf.nf_net_destroy(net)

    # and in 8 bits: the weights once, the rows of every call
    def quantised(a):
        rows, cols = a.shape
        q = torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=dev)
        scale = torch.empty(rows, device=dev)
        nf.nf_quantize_rows(a, q, scale)
        return q, scale
    w1q, s1 = quantised(torch.from_numpy(w1).to(dev))
    wq, s2 = quantised(w)
    out = torch.empty_like(full)
    nf.nf_linear_i8_dynamic(xtd, w1q, s1, ht, bias=torch.from_numpy(b1).to(dev), act="relu")
    nf.nf_linear_i8_dynamic(ht, wq, s2, out, bias=b)
    n = xt.shape[0]
    top, entropy, logp = min(3, classes), torch.empty(n, device=dev), torch.empty(n, device=dev)
    ids = torch.empty((n, top), dtype=torch.int32, device=dev)
    alt = torch.empty((n, top), device=dev)
    nf.nf_logprobs(out, ytd, logp=logp, entropy=entropy, top_ids=ids, top_logp=alt)
    result = {
        "first_loss": float(losses[0]), "last_loss": float(losses[-1]), "test_loss_8bit": float(-logp.mean()),
        "accuracy": float((full.argmax(1) == ytd).float().mean()),
        "accuracy_8bit": float((ids[:, 0] == ytd).float().mean()), "entropy": float(entropy.mean()),
    }
    say(f"loss {result['first_loss']:.4f} -> {result['last_loss']:.4f} in {steps} steps; held out: accuracy "
        f"{result['accuracy']:.4f} in fp32, {result['accuracy_8bit']:.4f} in 8 bits, loss {result['test_loss_8bit']:.4f}")
    say("first sample: class %d; alternatives %s" % (
        int(yt[0]), ", ".join(f"{i} ({np.exp(p):.3f})" for i, p in zip(ids[0].tolist(), alt[0].tolist()))))
    return result


if __name__ == "__main__":
    run()
