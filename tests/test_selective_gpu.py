"""The block of selective.py, and with it short convolution, selective scan and dense product as they are used together."""
import numpy as np
import pytest
import torch

from oracle import dropout, embed, gnorm, selective
from paper_2302_06646_amd import classifier
from paper_2302_06646_amd.selective import Selective

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().cpu().double().numpy()


def _rel(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


def _block(B, N, H, dtype=torch.float32, seed=0, **more):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = Selective(B, N, H, dtype=dtype, generator=g, **more)
    m.p["taps_bias"].normal_(generator=g)
    m.refresh()
    return m, torch.randn(B, H, N, generator=g, device="cuda").to(dtype), torch.randn(B, H, N, generator=g, device="cuda").to(dtype)


# Sums of at most a few hundred terms, each rounded a few times, and the recurrence's hundreds of places, whose decays forget them: in norm some
# tens of 2^-24, 2e-5 at most.
@pytest.mark.parametrize("B,N,H,more", [(2, 70, 24, {}), (3, 530, 10, dict(states=5, taps=3, groups=2, inner=12)), (1, 1, 8, dict(states=1, taps=1)),
                                        (2, 1100, 16, dict(states=20, rank=3))])
@pytest.mark.parametrize("uneven", [False, True])
def test_forward_and_backward_against_the_oracles(B, N, H, more, uneven):
    m, x, dy = _block(B, N, H, **more)
    lengths = torch.tensor([N, N // 2, N // 3][:B], device="cuda") if uneven else None
    y, dx = torch.empty_like(x), torch.empty_like(x)
    m.forward(x, y, lengths)
    m.backward(dy, x, dx, lengths)
    p = {k: _np(v) for k, v in m.p.items()}
    n = None if lengths is None else lengths.cpu().numpy()
    want, kept, _ = selective.forward(_np(x), p, m.S, m.G, n)
    assert _rel(_np(y), want) < 2e-5
    want_dx, grads = selective.backward(_np(dy), p, kept, n)
    assert _rel(_np(dx), want_dx) < 2e-5
    for name, w in grads.items():
        assert _rel(_np(m.p[name].grad), w) < 2e-5 or np.abs(_np(m.p[name].grad) - w).max() < 1e-6, name


def test_steps_go_on_where_a_sequence_ended():
    B, N, H, cut = 3, 90, 16, 61
    m, x, _ = _block(B, N, H, states=6)
    want = torch.empty_like(x)
    m.forward(x, want, residual=x)
    first, _, _ = _block(B, cut, H, states=6, train=False)
    state, y = first.new_state(), torch.empty(B, H, cut, device="cuda")
    first.forward(x[:, :, :cut].contiguous(), y, residual=x[:, :, :cut].contiguous(), state=state)
    parts = [y]
    for t in range(cut, N):
        now = x[:, :, t].contiguous()
        out = torch.empty_like(now)
        first.step(now, out, state, residual=now)
        parts.append(out[:, :, None])
    assert _rel(_np(torch.cat(parts, 2)), _np(want)) < 2e-5


def test_onto_the_residual_and_padding_of_any_value():
    m, x, _ = _block(3, 200, 16, dtype=torch.bfloat16, seed=4)
    lengths = torch.tensor([200, 77, 0], device="cuda")
    want, y = torch.empty_like(x), x.clone()
    m.forward(x, want, lengths, residual=x)
    m.forward(x, y, lengths, residual=y)
    assert torch.equal(want, y)
    other = x.clone()
    for b, n in enumerate(lengths.tolist()):
        other[b, :, n:] = 100.0
    m.forward(other, y, lengths)
    m.forward(x, want, lengths)
    assert torch.equal(y, want) and not y[2].any() and not y[1, :, 77:].any()


def test_a_training_step_under_capture():
    m, x, dy = _block(2, 600, 32, dtype=torch.bfloat16, seed=5)
    y, dx = torch.empty_like(x), torch.empty_like(x)

    def run():
        m.refresh()
        m.forward(x, y)
        m.backward(dy, x, dx)

    run()
    kept = [y, dx, *(t.grad for t in m.p.values())]
    want = [t.clone() for t in kept]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.synchronize()
    for again in range(3):
        for t in kept:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, kept))


def test_the_classifier_with_it():
    B, N, H, G, classes, step = 3, 256, 24, 3, 4, 5
    m = classifier.Classifier(B, N, H, classes, G, dtype=torch.float32, seed=7, mixer="scan")
    tokens, _ = classifier.batch(B, N, classes, torch.Generator(device="cuda").manual_seed(2))
    tokens[2] = -1                                         # a sequence without a byte
    logits = m.forward(tokens, step)
    dlogits = torch.randn(B, classes, generator=torch.Generator().manual_seed(3)).cuda()
    m.backward(dlogits, tokens, step)
    p, ids, dl = {k: _np(v) for k, v in m.p.items()}, tokens.cpu().numpy(), _np(dlogits)
    lengths = (ids >= 0).sum(1)
    mask = [dropout.mask((B, H, N), m.drop, 7, 3 * step), dropout.mask((B, H, N), m.tied_drop, 7, 3 * step + 2, N)]
    scale = float(np.float32(m.scale))
    x0 = embed.embed_fwd(ids, p["E"], scale, True, mask[0])
    mixed, kept, _ = selective.forward(x0, p, m.block.S, m.block.G, lengths)
    t = (x0 + mask[1] * mixed).transpose(0, 2, 1)
    z, _, _ = gnorm.gnorm_fwd(t, p["gamma"], p["beta"], G, m.eps, "silu")
    there = (ids >= 0) / np.maximum(lengths, 1)[:, None]
    pooled = (z * there[..., None]).sum(1)
    assert _rel(_np(logits), pooled @ p["head"]) < 2e-5
    dz = (dl @ p["head"].T)[:, None, :] * there[..., None]
    dt, _, _ = gnorm.gnorm_bwd(dz, t, p["gamma"], p["beta"], G, m.eps, "silu")
    dx1 = dt.transpose(0, 2, 1)
    dx, grads = selective.backward(dx1 * mask[1], p, kept, lengths)
    grads["E"] = embed.embed_bwd(dx1 + dx, ids, 256, scale, True, mask[0])
    for name, w in grads.items():
        assert _rel(_np(m.p[name].grad), w) < 5e-5, name      # (behind the group norm's own 2e-5)


def test_the_command_runs_and_another_mixer_is_refused():
    assert np.isfinite(classifier.main(["--mixer", "scan", "--steps", "3", "--batch", "4", "--length", "256", "--width", "16"]))
    with pytest.raises(ValueError, match="mixer"):
        classifier.Classifier(2, 256, 16, mixer="other")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padding_that_is_not_finite_takes_no_part_in_gradients(dtype):
    B, N, H = 4, 200, 16
    m, x, dy = _block(B, N, H, dtype=dtype, seed=6)
    lengths = torch.tensor([200, 77, 0, 513], device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)

    def run():
        m.forward(x, y, lengths)
        m.backward(dy, x, dx, lengths)
        return [t.clone() for t in (y, dx, *(p.grad for p in m.p.values()))]

    def pad(to_x, to_dy):
        for b, n in enumerate(lengths.tolist()):
            x[b, :, n:], dy[b, :, n:] = to_x, to_dy

    pad(0.0, 0.0)
    want = run()
    assert all(t.isfinite().all() for t in want)
    for to_x, to_dy in ((float("nan"), float("inf")), (float("-inf"), float("nan")), (100.0, -50.0)):
        pad(to_x, to_dy)
        before = x.clone(), dy.clone()
        assert all(torch.equal(a, b) for a, b in zip(run(), want)), (to_x, to_dy)
        assert torch.equal(x.view(-1).view(torch.uint8), before[0].view(-1).view(torch.uint8))      # the caller's own, as they were
        assert torch.equal(dy.view(-1).view(torch.uint8), before[1].view(-1).view(torch.uint8))


# 16-bit: each stored tensor is off by half a step at most (2^-8, 2^-11 of a value), everything else by some 2^-24.  Forward, nine of them stand between x and
# y (u0, u, z, r, delta, B, C, the scan's y, y), and u, with what u0 brings to it, reaches the scan's y four ways (u itself, delta, B, C), each at most in
# proportion: 9 + 2 * 3 = 15 half steps.  A gradient takes what its forward values are off by, 15, and the gradients on its way down, at most twelve: of the scan's
# y, delta, B, C, z, u, r, three sums into u's, u0's, its own.  Both are sums of sizes, not of squares: norms stay well within.
@pytest.mark.parametrize("dtype,unit", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
@pytest.mark.parametrize("uneven", [False, True])
def test_sixteen_bits_against_the_oracles(dtype, unit, uneven):
    B, N, H = 3, 330, 48
    m, x, dy = _block(B, N, H, dtype=dtype, seed=8, states=6, groups=2)
    lengths = torch.tensor([N, 200, 31], device="cuda") if uneven else None
    y, dx = torch.empty_like(x), torch.empty_like(x)
    m.forward(x, y, lengths)
    m.backward(dy, x, dx, lengths)
    p = {k: _np(m.low.get(k, v)) for k, v in m.p.items()}      # the products' operands as they are
    n = None if lengths is None else lengths.cpu().numpy()
    want, kept, _ = selective.forward(_np(x), p, m.S, m.G, n)
    assert _rel(_np(y), want) < 15 * unit
    want_dx, grads = selective.backward(_np(dy), p, kept, n)
    assert _rel(_np(dx), want_dx) < 27 * unit
    for name, w in grads.items():
        assert _rel(_np(m.p[name].grad), w) < 27 * unit, name
