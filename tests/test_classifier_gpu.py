"""The block of classifier.py: one step against the float64 oracles of its parts, and whether it learns."""
import numpy as np
import pytest
import torch

import oracle
from oracle import dropout, embed, gnorm, kreg
from paper_2302_06646_amd import classifier

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().cpu().double().numpy()


def _rel(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


def test_a_step_against_the_oracles():
    B, N, H, G, classes, step = 3, 256, 24, 3, 4, 5
    m = classifier.Classifier(B, N, H, classes, G, dtype=torch.float32, seed=7)
    tokens, _ = classifier.batch(B, N, classes, torch.Generator(device="cuda").manual_seed(2))
    logits = m.forward(tokens, step)
    dlogits = torch.randn(B, classes, generator=torch.Generator().manual_seed(3)).cuda()
    m.backward(dlogits, tokens, step)
    p, ids, dl = {k: _np(v) for k, v in m.p.items()}, tokens.cpu().numpy(), _np(dlogits)
    mask = [dropout.mask((B, H, N), m.drop, 7, 3 * step), dropout.mask((H, N), m.kernel_drop, 7, 3 * step + 1),
            dropout.mask((B, H, N), m.tied_drop, 7, 3 * step + 2, N)]
    x0 = embed.embed_fwd(ids, p["E"], float(np.float32(m.scale)), True, mask[0])
    lam = float(np.float32(m.squash))
    kbar = kreg.kernel_reg_fwd(p["K"], mask[1], m.width, lam)
    x1 = x0 + mask[2] * oracle.longconv_fwd(x0, kbar, p["D"])
    t = x1.transpose(0, 2, 1)
    z, _, _ = gnorm.gnorm_fwd(t, p["gamma"], p["beta"], G, m.eps, "silu")
    there = (ids >= 0) / (ids >= 0).sum(1, keepdims=True)
    pooled = (z * there[..., None]).sum(1)
    assert _rel(_np(logits), pooled @ p["head"]) < 1e-5
    dz = (dl @ p["head"].T)[:, None, :] * there[..., None]
    dt, dgamma, dbeta = gnorm.gnorm_bwd(dz, t, p["gamma"], p["beta"], G, m.eps, "silu")
    dx1 = dt.transpose(0, 2, 1)
    du, dkbar, dD = oracle.longconv_bwd(dx1 * mask[2], x0, kbar, p["D"])
    want = {"E": embed.embed_bwd(dx1 + du, ids, 256, float(np.float32(m.scale)), True, mask[0]),
            "K": kreg.kernel_reg_bwd(p["K"], mask[1], m.width, lam, dkbar), "D": dD, "gamma": dgamma, "beta": dbeta,
            "head": pooled.T @ dl}
    for name, w in want.items():
        assert _rel(_np(m.p[name].grad), w) < 2e-5, name


def test_it_learns():
    assert classifier.main(["--steps", "60", "--batch", "16", "--length", "512", "--width", "32"]) < 0.7


def test_a_sequence_without_a_byte():
    B, N, H = 3, 256, 16
    runs = []
    for rows in (slice(0, 3), slice(0, 2)):                             # with the empty sequence, and without it
        m = classifier.Classifier(len(range(B)[rows]), N, H, 4, 2, dtype=torch.float32, seed=7, drop=0.0, kernel_drop=0.0, tied_drop=0.0)
        tokens, _ = classifier.batch(B, N, 4, torch.Generator(device="cuda").manual_seed(2))
        tokens[2] = -1
        tokens = tokens[rows].contiguous()
        logits = m.forward(tokens, 0)
        dlogits = torch.randn(B, 4, generator=torch.Generator().manual_seed(3)).cuda()[rows].contiguous()
        m.backward(dlogits, tokens, 0)
        runs.append((logits, {k: p.grad.clone() for k, p in m.p.items()}))
    (logits, grads), (logits2, grads2) = runs
    assert (logits[2] == 0).all() and _rel(_np(logits[:2]), _np(logits2)) < 1e-5      # nothing is pooled, and the others do not notice
    for name in grads:
        assert _rel(_np(grads[name]), _np(grads2[name])) < 1e-5, name
