"""Group norm with an activation against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2302_06646_amd as lc
from oracle import gnorm

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}
U = 2.0 ** -24
EPS = 1e-5


def _np(t):
    return t.detach().cpu().double().numpy()


class Run:
    def __init__(self, B, S, C, G, io, act, mean=0.5, params=True, seed=0):
        r = lambda *s, k=0: torch.randn(*s, generator=torch.Generator().manual_seed(seed * 10 + k))  # noqa: E731
        self.G, self.act, self.io = G, act, io
        self.x, self.dy = (r(B, S, C) + mean).to(DT[io]).cuda(), r(B, S, C, k=1).to(DT[io]).cuda()
        self.gamma, self.beta = ((1 + 0.3 * r(C, k=2)).cuda(), r(C, k=3).cuda()) if params else (None, None)
        self.y, self.dx = torch.full_like(self.x, 7.0), torch.full_like(self.x, 7.0)
        self.mean, self.rstd = (torch.full((B, G), 7.0, device="cuda") for _ in range(2))
        self.dgamma, self.dbeta = (torch.full((C,), 7.0, device="cuda") for _ in range(2))
        self.ws = lc.new_workspace_gnorm(B, S, C, G, lc.dtype_code(self.x), True)
        self.ws.fill_(0xA5)

    def fwd(self):
        lc.longconv_gnorm_fwd(self.x, self.gamma, self.beta, self.y, self.mean, self.rstd, EPS, self.act, self.ws)

    def bwd(self):
        lc.longconv_gnorm_bwd(self.dy, self.x, self.gamma, self.beta, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, self.act,
                              self.ws)

    def check(self):
        """Sums of n numbers in a few levels lose at most 64 roundings here (32 numbers one by one in a thread, and the levels above):
        the mean's error is 64 U (|mean| + deviation), which xhat has in units of the deviation.  An activation's slope is at most
        1.13, the slope's own at most 1.13 as well."""
        C = self.x.shape[2]
        x, dy = _np(self.x), _np(self.dy)
        gamma = np.ones(C) if self.gamma is None else _np(self.gamma)
        beta = np.zeros(C) if self.beta is None else _np(self.beta)
        y, mean, rstd = gnorm.gnorm_fwd(x, gamma, beta, self.G, EPS, self.act)
        dx, dgamma, dbeta = gnorm.gnorm_bwd(dy, x, gamma, beta, self.G, EPS, self.act)
        each = lambda a: np.repeat(a, C // self.G, 1)[:, None]  # noqa: E731
        off = 1 + np.abs(each(mean)) * each(rstd)                       # mean and deviation in units of the deviation
        xhat = (x - each(mean)) * each(rstd)
        K = 64 * U
        assert (np.abs(_np(self.mean) - mean) <= K * (np.abs(mean) + 1 / rstd)).all()
        assert (np.abs(_np(self.rstd) - rstd) <= K * rstd * off[:, 0, :: C // self.G]).all()
        dxhat = K * (off + np.abs(xhat))                                # error of xhat
        dz = 1.13 * np.abs(gamma) * dxhat
        unit, tiny = UNIT[self.io], TINY[self.io]
        assert (np.abs(_np(self.y) - y) <= dz + K * (1 + np.abs(y)) + unit * np.abs(y) + tiny).all()
        if self.act == "relu":                                          # its slope jumps where z is zero to rounding
            sure = np.abs(xhat * gamma + beta) > dz + K
            assert sure.mean() > 0.999
            if not sure.all():
                return
        slope = np.abs(gnorm.act(xhat * gamma + beta, self.act)[1])
        t = np.abs(gamma * dy)
        err = np.abs(dy) * 1.13 * (dz + K * (1 + slope))                # of dy act'(z)
        of = lambda a: each(a.reshape(*a.shape[:2], self.G, -1).mean(axis=(1, 3)))  # noqa: E731
        size = t + of(t) + np.abs(xhat) * of(t * np.abs(xhat))
        spread = np.abs(gamma) * err + of(np.abs(gamma) * err) + np.abs(xhat) * of(np.abs(gamma) * err * np.abs(xhat) + t * dxhat) \
            + dxhat * of(t * np.abs(xhat))
        bound = each(rstd) * (spread + K * off * size) + unit * np.abs(dx) + tiny
        assert (np.abs(_np(self.dx) - dx) <= bound).all()
        assert (np.abs(_np(self.dbeta) - dbeta) <= (err + K * np.abs(dy)).sum((0, 1))).all()
        assert (np.abs(_np(self.dgamma) - dgamma) <= (err * np.abs(xhat) + np.abs(dy) * 1.13 * dxhat + K * np.abs(dy * xhat)).sum((0, 1))).all()


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("B,S,C,G", [(1, 1, 8, 1), (2, 49, 24, 3), (3, 5, 195, 5), (1, 300, 1, 1), (2, 7, 64, 64), (1, 64, 520, 1), (5, 33, 1040, 8)])
def test_forward_and_backward_against_oracle(io, act, B, S, C, G):
    r = Run(B, S, C, G, io, act)
    r.fwd()
    r.bwd()
    r.check()


# one position to many, on both sides of the sizes where the way through the kernels changes
@pytest.mark.parametrize("B,S,C,G", [(1, 2048, 16, 2), (2, 1024, 256, 32), (1, 5000, 40, 5), (9, 700, 72, 9), (40, 3, 32, 4), (1, 20000, 8, 1),
                                     (300, 16, 16, 2), (3, 1, 4096, 1), (1, 513, 200, 25)])
@pytest.mark.parametrize("io", ["fp32", "bf16"])
def test_sizes(io, B, S, C, G):
    r = Run(B, S, C, G, io, "silu", seed=1)
    r.fwd()
    r.bwd()
    r.check()


# groups that just fit a workgroup's registers and just do not (pieces of eight channels: 16 of 512 threads forward, 8 backward), and
# partial results of a group that one wave puts together and that a workgroup does
@pytest.mark.parametrize("io,act,B,S,C,G", [("bf16", "silu", 1, 2048, 32, 4), ("fp16", "gelu", 2, 2049, 32, 1), ("fp32", "silu", 1, 1024, 16, 1),
                                            ("fp32", "gelu", 1, 1025, 24, 3), ("bf16", "gelu", 1, 8192, 8, 1), ("bf16", "none", 1, 8193, 8, 1),
                                            ("fp16", "silu", 1, 3000, 130, 1), ("fp32", "silu", 2, 1500, 104, 2), ("bf16", "silu", 3, 5000, 3, 1),
                                            ("fp32", "gelu", 1, 4097, 1, 1), ("fp16", "relu", 2, 700, 7, 7), ("bf16", "silu", 1, 2, 1030, 1),
                                            ("fp32", "none", 1, 1, 2056, 257)])
def test_where_the_way_through_changes(io, act, B, S, C, G):
    r = Run(B, S, C, G, io, act, seed=3)
    r.fwd()
    r.bwd()
    r.check()


def test_without_parameters():
    r = Run(2, 30, 48, 4, "fp32", "gelu", params=False)
    r.fwd()
    r.bwd()
    r.check()


@pytest.mark.parametrize("S", [30, 3000])
def test_a_mean_that_dwarfs_the_deviation(S):
    r = Run(2, S, 32, 4, "fp32", "none", mean=1000.0)
    r.fwd()
    r.bwd()
    r.check()


@pytest.mark.parametrize("S", [9, 4000])
def test_constant_groups(S):
    r = Run(1, S, 16, 2, "fp32", "none")
    r.x[..., :8] = 3.0
    r.fwd()
    assert torch.equal(r.mean[0, 0], torch.tensor(3.0, device="cuda")) and torch.isfinite(r.y).all()
    assert torch.equal(r.y[..., :8], r.beta[:8].expand(1, S, 8))
    r.bwd()
    r.check()


@pytest.mark.parametrize("S", [20, 2500])
def test_a_value_that_is_not_finite_stays_in_its_group(S):
    r, clean = Run(2, S, 24, 3, "fp32", "silu"), Run(2, S, 24, 3, "fp32", "silu")
    r.x[1, 5, 9] = float("inf")
    for q in (r, clean):
        q.fwd()
        q.bwd()
    for a, b in ((r.y, clean.y), (r.dx, clean.dx)):
        bad = torch.zeros_like(a, dtype=torch.bool)
        bad[1, :, 8:16] = True
        assert torch.equal(a[~bad], b[~bad]) and not torch.isfinite(a[bad]).any()
    assert torch.equal(r.dbeta[:8], clean.dbeta[:8]) and torch.equal(r.dgamma[16:], clean.dgamma[16:])


@pytest.mark.parametrize("S", [25, 2100])
def test_gradients_asked_for_alone_and_repeated(S):
    r = Run(3, S, 40, 5, "bf16", "gelu")
    r.fwd()
    r.bwd()
    want = [t.clone() for t in (r.dx, r.dgamma, r.dbeta)]
    for i in range(3):
        out = [torch.full_like(t, 5.0) if j == i else None for j, t in enumerate(want)]
        lc.longconv_gnorm_bwd(r.dy, r.x, r.gamma, r.beta, r.mean, r.rstd, *out, r.act, r.ws)
        assert torch.equal(out[i], want[i])
    r.fwd()
    r.bwd()
    assert all(torch.equal(a, b) for a, b in zip((r.dx, r.dgamma, r.dbeta), want))


def test_offsets_past_32_bits():
    B, S, C, G = 3, 1 << 20, 712, 8                                     # 2.2e9 elements
    x = torch.zeros(B, S, C, dtype=torch.bfloat16, device="cuda")
    x[B - 1] = torch.randn(S, C, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(B, G, device="cuda"), torch.empty(B, G, device="cuda")
    ws = lc.new_workspace_gnorm(B, S, C, G, lc.BF16, True)
    lc.longconv_gnorm_fwd(x, None, None, y, mean, rstd, EPS, "none", ws)
    assert (y[:2] == 0).all()
    g = x[B - 1].view(S, G, C // G).double()
    m = g.mean((0, 2))
    v = g.var((0, 2), unbiased=False)
    assert torch.allclose(mean[B - 1].double(), m, atol=1e-6) and torch.allclose(rstd[B - 1].double(), (v + EPS) ** -0.5, rtol=1e-5)
    want = ((g - m[:, None]) * ((v + EPS) ** -0.5)[:, None]).view(S, C)
    assert ((y[B - 1].double() - want).abs() <= 1.01 * UNIT["bf16"] * want.abs() + 1e-4).all()
    del g, want
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    lc.longconv_gnorm_bwd(y, x, None, None, mean, rstd, y.clone(), dgamma, dbeta, "none", ws)
    want = y[B - 1].double().square().sum(0)
    assert torch.allclose(dgamma.double(), want, rtol=1e-2)             # y is xhat to bf16's rounding
    torch.cuda.empty_cache()


def test_another_stream_and_graph_replays():
    r = Run(4, 256, 64, 8, "bf16", "silu")
    r.fwd()
    r.bwd()
    torch.cuda.synchronize()
    want = [t.clone() for t in (r.y, r.dx, r.dgamma, r.dbeta)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.fwd()
        r.bwd()
    for _ in range(4):
        for t in (r.y, r.dx, r.dgamma, r.dbeta):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((r.y, r.dx, r.dgamma, r.dbeta), want))
    s = torch.cuda.Stream()
    y = torch.empty_like(r.y)
    s.wait_stream(torch.cuda.current_stream())
    lc.longconv_gnorm_fwd(r.x, r.gamma, r.beta, y, r.mean, r.rstd, EPS, r.act, r.ws, stream=s)
    s.synchronize()
    assert torch.equal(y, want[0])


def test_every_way_through_the_binding_gives_the_same_bits():
    class Sub(torch.Tensor):
        pass

    a, b = Run(2, 20, 24, 3, "fp16", "silu"), Run(2, 20, 24, 3, "fp16", "silu")
    b.x = b.x.as_subclass(Sub)
    for r in (a, b):
        r.fwd()
        r.bwd()
    for name in ("y", "mean", "rstd", "dx", "dgamma", "dbeta"):
        assert torch.equal(getattr(a, name), getattr(b, name))
    for name, bad in (("y", a.y.float()), ("y", a.y[:, :10]), ("gamma", a.gamma[:5]), ("mean", a.mean[:, :2]), ("ws", a.ws[:8])):
        r = Run(2, 20, 24, 3, "fp16", "silu")
        setattr(r, name, bad)
        with pytest.raises(lc.LongconvError):
            r.fwd()


# groups of one value, however large: each entry is the mean, so xhat is zero and z is beta, to the last bit (sums of so few equal
# numbers of so few bits are exact); both ways through, and groups of a single entry
@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("value", [100.0, 300.0, -60000.0])
@pytest.mark.parametrize("B,S,C,G", [(2, 16, 32, 2), (1, 9000, 16, 2), (5, 1, 24, 24), (1, 16, 30, 5)])
def test_groups_of_one_value_give_beta(io, value, B, S, C, G):
    r = Run(B, S, C, G, io, "none")
    r.x.fill_(value)
    r.fwd()
    assert torch.equal(r.mean, r.x[:, 0, ::C // G].float())
    assert torch.equal(r.y, r.beta.to(r.x.dtype).expand(B, S, C))
    r = Run(B, S, C, G, io, "relu", params=False)
    r.x.fill_(value)
    r.fwd()
    r.bwd()
    for t in (r.y, r.dx, r.dgamma, r.dbeta):                            # z is zero, where the slope is zero
        assert (t == 0).all()


@pytest.mark.parametrize("S", [64, 20000])
def test_results_in_sixteen_bits_are_rounded_once(S):
    # Data of mean zero: z is good to a few roundings of fp32, and so is gelu(z).  A result with a relative error of 8 U before its one
    # rounding differs from the exact value's rounding if that lies within 8 U of a midpoint of fp16 (2^-11 apart at least): 16 U / 2^-11.
    half = torch.randn(1, S // 2, 64, generator=torch.Generator().manual_seed(5))
    r = Run(1, S, 64, 8, "fp16", "gelu", params=False)
    r.x = torch.cat([half, -half], 1).half().cuda()
    r.fwd()
    want = gnorm.gnorm_fwd(_np(r.x), np.ones(64), np.zeros(64), 8, EPS, "gelu")[0].astype(np.float16)
    assert (r.y.cpu().numpy() != want).mean() <= 16 * U * 2 ** 11


def test_as_many_sequences_as_a_launch_takes():
    B, S, C, G = (1 << 23) - 1, 2, 4, 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(B, S, C, generator=gen, device="cuda") for _ in range(2))

    def step(x, dy):
        out = [torch.full_like(x, 7.0) for _ in range(2)] + [torch.full((len(x), G), 7.0, device="cuda") for _ in range(2)]
        sums = [torch.empty(C, device="cuda") for _ in range(2)]
        ws = lc.new_workspace_gnorm(len(x), S, C, G, lc.F32, True)
        lc.longconv_gnorm_fwd(x, None, None, out[0], *out[2:], EPS, "silu", ws)
        lc.longconv_gnorm_bwd(dy, x, None, None, *out[2:], out[1], *sums, "silu", ws)
        return out, sums

    out, (dgamma, dbeta) = step(x, dy)
    for at in (slice(0, 1000), slice(B // 2, B // 2 + 1000), slice(B - 1000, B)):      # each of the B by itself
        few, _ = step(x[at].clone(), dy[at].clone())
        assert all(torch.equal(a[at], b) for a, b in zip(out, few))
    # a thread adds 2^17 numbers of both signs: as in test_gradients_past_32_bits, about one U of the sum of magnitudes; 64 are allowed
    each = lambda t: t.double().repeat_interleave(C // G, 1)[:, None]  # noqa: E731
    xhat = (x.double() - each(out[2])) * each(out[3])
    q = torch.sigmoid(xhat)
    dz = dy.double() * q * (1 + xhat * (1 - q))
    assert ((dbeta - dz.sum((0, 1))).abs() <= 64 * U * dy.abs().double().sum((0, 1)) * 1.13).all()
    assert ((dgamma - (dz * xhat).sum((0, 1))).abs() <= 64 * U * (dy.double() * (1 + xhat.abs())).abs().sum((0, 1)) * 1.13).all()


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("B,S,C,G", [(2, 64, 24, 3), (1, 9000, 16, 2), (3, 50, 195, 5)])
def test_relu_gradients_where_no_entry_is_near_zero(io, B, S, C, G):
    r = Run(B, S, C, G, io, "relu", seed=6)
    sign = torch.where(torch.rand(r.x.shape, generator=torch.Generator().manual_seed(7)) < 0.5, -1.0, 1.0)
    r.x = (sign * (1.5 + torch.rand(r.x.shape, generator=torch.Generator().manual_seed(8)))).to(r.x.dtype).cuda()
    r.gamma, r.beta = (torch.where(r.gamma < 1, -1.0, 1.0) * (0.5 + (r.gamma - 1).abs())).contiguous(), torch.zeros_like(r.beta)
    x = _np(r.x)
    mean, rstd = (np.repeat(a, C // G, 1)[:, None] for a in gnorm.statistics(x, G, EPS))
    assert np.abs((x - mean) * rstd * _np(r.gamma)).min() > 0.1         # (check() passes over gradients where one is near)
    r.fwd()
    r.bwd()
    r.check()


def test_gradients_past_32_bits():
    B, S, C, G = 3, 1 << 20, 1376, 8                                    # 4.3e9 elements
    D, tail = C // G, 4096
    x, dy = (torch.zeros(B, S, C, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t, seed in ((x, 1), (dy, 2)):
        t[B - 1].normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
    y, dx = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    mean, rstd, dgamma, dbeta = (torch.empty(*s, device="cuda") for s in ((B, G), (B, G), (C,), (C,)))
    ws = lc.new_workspace_gnorm(B, S, C, G, lc.BF16, True)
    lc.longconv_gnorm_fwd(x, None, None, y, mean, rstd, EPS, "none", ws)
    lc.longconv_gnorm_bwd(dy, x, None, None, mean, rstd, dx, dgamma, dbeta, "none", ws)
    assert all((t[:B - 1] == 0).all() for t in (y, dx))
    # Sums in 64 bits, a group at a time.  A thread adds about 1200 numbers one by one, of both signs: their sums stay near the root of
    # their number, so the roundings come to about one U of the sum of magnitudes; 64 are allowed, as in check().
    for g in range(G):
        c = slice(g * D, g * D + D)
        xg, dg = x[B - 1, :, c].double(), dy[B - 1, :, c].double()
        m, v = xg.mean(), xg.var(unbiased=False)
        xhat = (xg - m) * (v + EPS) ** -0.5
        K = 64 * U
        assert ((dbeta[c].double() - dg.sum(0)).abs() <= K * dg.abs().sum(0)).all()
        assert ((dgamma[c].double() - (dg * xhat).sum(0)).abs() <= K * (dg.abs() * (1 + xhat.abs())).sum(0)).all()
        want = (v + EPS) ** -0.5 * (dg - dg.mean() - xhat * (dg * xhat).mean())
        size = dg.abs() + dg.abs().mean() + xhat.abs() * (dg * xhat).abs().mean()
        for rows in (slice(0, tail), slice(S - tail, S)):
            for got, exact, slack in ((y, xhat, K * (1 + xhat.abs())), (dx, want, K * 2 * size)):
                off = (got[B - 1, rows, c].double() - exact[rows]).abs()
                assert (off <= slack[rows] + UNIT["bf16"] * exact[rows].abs()).all()
        del xg, dg, xhat, want, size
    del x, dy, y, dx
    torch.cuda.empty_cache()
