"""Dropout whose mask is never stored, alone and inside the kernel regularisers, against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2302_06646_amd as lc
from oracle import dropout, kreg

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}      # of one rounding
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}   # and of one below the normal range


def _np(t):
    return t.detach().cpu().double().numpy()


def _draw(shape, io, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(DT[io]).cuda()


def _close(got, want, size, io):
    # the factor's rounding, the multiply-add's and the result's
    assert (np.abs(_np(got) - want) <= (UNIT[io] + 2 * 2.0 ** -24) * size + TINY[io]).all()


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("n,p", [(1, 0.5), (7, 0.1), (8, 0.9), (9, 0.25), (2047, 0.0), (2048, 0.3), (2057, 1.0), (50001, 0.1)])
def test_dropout_against_oracle(io, n, p):
    seed, call = (n << 33) + 5, (7 << 32) + n
    x, r, dy = (_draw((n,), io, i) for i in range(3))
    m = dropout.mask((n,), p, seed, call)
    y, dx = torch.full_like(x, 9.0), torch.full_like(x, 9.0)
    lc.longconv_dropout_fwd(x, y, p, seed, call)
    lc.longconv_dropout_bwd(dy, dx, p, seed, call)
    for got, a in ((y, x), (dx, dy)):
        want = dropout.dropout(_np(a), m)
        assert ((_np(got) == 0) == (want == 0)).all()                  # which entries are kept is no matter of rounding
        _close(got, want, np.abs(want), io)
    lc.longconv_dropout_fwd(x, y, p, seed, call, residual=r)
    want = dropout.dropout(_np(x), m, _np(r))
    _close(y, want, np.abs(want) + np.abs(_np(x) * m), io)
    for buffer, more in ((x.clone(), r), (r.clone(), x)):              # in place of either input
        a, b = (buffer, more) if more is r else (more, buffer)
        lc.longconv_dropout_fwd(a, buffer, p, seed, call, residual=b)
        assert torch.equal(buffer, y)


@pytest.mark.parametrize("io", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,tie", [(5, 1), (100, 3), (33, 7), (65, 8), (9, 9), (20, 64), (7, 1001), (3, 4096), (1, 77)])
def test_entries_that_share_a_value(io, rows, tie):
    x, r = _draw((rows, tie), io, 1), _draw((rows, tie), io, 2)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    lc.longconv_dropout_fwd(x, y, 0.4, 11, 12, residual=r, tie=tie)
    lc.longconv_dropout_bwd(x, dx, 0.4, 11, 12, tie=tie)
    m = dropout.mask((rows, tie), 0.4, 11, 12, tie)
    want = dropout.dropout(_np(x), m, _np(r))
    _close(y, want, np.abs(want) + np.abs(_np(x) * m), io)
    want = dropout.dropout(_np(x), m)
    assert ((_np(dx) == 0) == (want == 0)).all()
    _close(dx, want, np.abs(want), io)


def test_what_is_dropped_counts_for_nothing():
    m = dropout.mask((4096,), 0.5, 3, 4)
    x = torch.where(torch.from_numpy(m).cuda() == 0, float("nan"), 1.0).float()
    x[torch.from_numpy(np.flatnonzero(m == 0)[::2]).cuda()] = float("inf")
    y = torch.empty_like(x)
    lc.longconv_dropout_fwd(x, y, 0.5, 3, 4)
    assert (_np(y) == m).all()
    x[int(np.flatnonzero(m)[0])] = float("nan")
    lc.longconv_dropout_fwd(x, y, 0.5, 3, 4)
    assert int(torch.isnan(y).sum()) == 1


@pytest.mark.parametrize("tie", [1, 1 << 30])
def test_entries_past_32_bits(tie):
    n = (1 << 32) + (1 << 30) + (0 if tie > 1 else 13)
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    lc.longconv_dropout_fwd(x, x, 0.5, 1, 2, tie=tie)
    for at in (0, (1 << 31) - 1000, (1 << 32) - 1000, n - 2000):
        e = np.arange(at, at + 2000)
        assert (_np(x[at:at + 2000]) == dropout.factors(e // tie, 0.5, 1, 2)).all()
    del x
    torch.cuda.empty_cache()


def test_step_on_the_device_and_graph_replays():
    x = _draw((3, 1000), "fp32", 1)
    y, step = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")
    k = _draw((2, 256), "fp32", 2)
    kbar = torch.empty_like(k)

    def both(call, step=None):
        lc.longconv_dropout_fwd(x, y, 0.3, 5, call, step=step)
        lc.longconv_kreg_fwd_seeded(k, kbar, 1, 0.01, 0.3, 5, call, step=step)
        return y.clone(), kbar.clone()

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(40, step)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lc.longconv_dropout_fwd(x, y, 0.3, 5, 40, step=step)
        lc.longconv_kreg_fwd_seeded(k, kbar, 1, 0.01, 0.3, 5, 40, step=step)
    seen = []
    for i in range(4):
        step.fill_(i)
        g.replay()
        got = y.clone(), kbar.clone()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, both(40 + i)))
        seen.append(got[0])
    assert not any(torch.equal(a, b) for i, a in enumerate(seen) for b in seen[:i])


def test_another_stream():
    s = torch.cuda.Stream()
    x = _draw((100003,), "bf16", 1)
    s.wait_stream(torch.cuda.current_stream())
    y, z = torch.empty_like(x), torch.empty_like(x)
    lc.longconv_dropout_fwd(x, y, 0.3, 5, 6, stream=s)
    s.synchronize()
    lc.longconv_dropout_fwd(x, z, 0.3, 5, 6)
    assert torch.equal(y, z)


@pytest.mark.parametrize("H,N,p,q", [(3, 256, 0, 0.5), (37, 1024, 1, 0.2), (2, 512, 32, 0.5), (5, 256, 31, 0.1), (4, 4096, 3, 0.0),
                                     (2, 131072, 2, 0.3)])
def test_seeded_regularisers_are_those_of_the_stored_mask(H, N, p, q):
    k, g = _draw((H, N), "fp32", 1) * 0.02, _draw((H, N), "fp32", 2)
    m = dropout.mask((H, N), q, 9, 10)
    stored = torch.from_numpy(m.astype(np.float32)).cuda()
    want, got = [torch.full_like(k, 5.0) for _ in range(2)], [torch.full_like(k, 6.0) for _ in range(2)]
    lc.longconv_kreg_fwd(k, stored, want[0], p, 0.002)
    lc.longconv_kreg_bwd(k, stored, g, want[1], p, 0.002)
    lc.longconv_kreg_fwd_seeded(k, got[0], p, 0.002, q, 9, 10)
    lc.longconv_kreg_bwd_seeded(k, g, got[1], p, 0.002, q, 9, 10)
    for a, b in zip(got, want):
        assert torch.equal(a, b)                                       # the same sums of the same products
    ref = kreg.kernel_reg_fwd(_np(k), m, p, float(np.float32(0.002)))
    scale = np.abs(_np(k)).max() * m.max()
    assert np.abs(_np(got[0]) - ref).max() <= 2e-6 * scale


def test_seeded_regularisers_drop_what_is_not_a_number():
    m = dropout.mask((2, 256), 0.5, 1, 2)
    k = torch.where(torch.from_numpy(m).cuda() == 0, float("nan"), 0.5).float()
    kbar, dk = torch.empty_like(k), torch.empty_like(k)
    lc.longconv_kreg_fwd_seeded(k, kbar, 1, 0.0, 0.5, 1, 2)
    lc.longconv_kreg_bwd_seeded(k, torch.ones_like(k), dk, 1, 0.0, 0.5, 1, 2)
    assert torch.isfinite(kbar).all() and torch.isfinite(dk).all()
    assert (_np(dk)[m == 0] == 0).all()


def test_every_way_through_the_binding_gives_the_same_bits():
    class Sub(torch.Tensor):
        pass

    x, k = _draw((3, 500), "fp16", 1), _draw((2, 256), "fp32", 1)
    outs = []
    for way in (lambda t: t, lambda t: t.as_subclass(Sub)):            # natively, and in Python
        y, dx, kbar, dk = (torch.empty_like(t) for t in (x, x, k, k))
        lc.longconv_dropout_fwd(way(x), y, 0.3, (1 << 63) + 5, 6, residual=x, tie=500)
        lc.longconv_dropout_bwd(way(x), dx, 0.3, 5, 6)
        lc.longconv_kreg_fwd_seeded(way(k), kbar, 1, 0.1, 0.3, 5, 6)
        lc.longconv_kreg_bwd_seeded(way(k), k, dk, 1, 0.1, 0.3, 5, 6)
        outs.append([y, dx, kbar, dk])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for bad in (x.t(), x[:, 1:], x.float(), x.cpu()):
        with pytest.raises(lc.LongconvError):
            lc.longconv_dropout_fwd(x, bad, 0.3, 1, 1)
    with pytest.raises(lc.LongconvError):
        lc.longconv_dropout_fwd(x, x, 0.3, 1, 1, step=torch.zeros(1, device="cuda"))
    with pytest.raises(KeyError):
        lc.longconv_dropout_fwd(x.double(), x, 0.3, 1, 1)
