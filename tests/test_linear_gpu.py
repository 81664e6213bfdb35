"""Dense product between layers against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2302_06646_amd as lc
from oracle import gnorm, linear

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}
U = 2.0 ** -24
LAYOUT = {False: lc.CHANNELS_LAST, True: lc.CHANNELS_FIRST}


def _np(t):
    return None if t is None else t.detach().cpu().double().numpy()


class Run:
    def __init__(self, B, N, K, M, io, act="none", bias=True, residual=False, x_first=False, y_first=False, dW=None, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        dt = DT[io]
        self.io, self.act, self.x_first, self.y_first = io, act, x_first, y_first
        of_x, of_y = (B, K, N) if x_first else (B, N, K), (B, M, N) if y_first else (B, N, M)
        self.x, self.W, self.dy = r(*of_x).to(dt).cuda(), (r(M, K) / K ** 0.5).to(dt).cuda(), r(*of_y).to(dt).cuda()
        self.bias, self.residual = r(M).cuda() if bias else None, r(*of_y).to(dt).cuda() if residual else None
        new = lambda *s, dt=dt: torch.full(s, 7.0, dtype=dt, device="cuda")  # noqa: E731
        self.y, self.dx, self.dW, self.dbias = new(*of_y), new(*of_x), new(M, K, dt=DT[dW or "fp32"]), new(M, dt=torch.float32)
        self.ws = lc.new_workspace_linear(B, N, K, M, lc.dtype_code(self.x), True)
        self.ws.fill_(0xFF)

    def fwd(self):
        lc.longconv_linear_fwd(self.x, self.W, self.bias, self.y, self.act, self.ws, LAYOUT[self.x_first], LAYOUT[self.y_first], self.residual)
        return self

    def bwd(self, dx=True, dW=True, dbias=True):
        lc.longconv_linear_bwd(self.dy, self.x, self.W, self.bias, self.dx if dx else None, self.dW if dW else None,
                               self.dbias if dbias else None, self.act, self.ws, LAYOUT[self.x_first], LAYOUT[self.y_first])
        return self

    def check(self):
        """A sum of n products in fp32 is off by (n + 4) U of the sum of their sizes, however it is cut and added.  Activations and slopes as
        their kernels' comments say: (8 + |z|) U |z| and (8 + 2 |z|) U (1 + |z|), slopes and theirs at most 1.13.  Behind an activation dz
        is rounded to the I/O type in front of dx and dW: half a step of it."""
        x, W, dy = _np(self.x), _np(self.W), _np(self.dy)
        M, K = W.shape
        T = x.size // K
        bias = np.zeros(M) if self.bias is None else _np(self.bias)
        r = None if self.residual is None else _np(self.residual)
        y = linear.linear_fwd(x, W, bias, self.act, self.x_first, self.y_first, r)
        rows, g = linear.last(x, self.x_first), linear.last(dy, self.y_first)
        z = rows @ W.T + bias
        unit, tiny = UNIT[self.io], TINY[self.io]
        near = lambda got, want, bound: (np.abs(_np(got) - want) <= bound + tiny).all()  # noqa: E731
        err_z = (K + 4) * U * (np.abs(rows) @ np.abs(W).T + np.abs(bias))
        plain = self.act == "none"
        err_y = 1.13 * err_z + (0 if plain else U * (8 + np.abs(z)) * np.abs(z))
        back = lambda t: linear.last(t, self.y_first)  # noqa: E731  (its own inverse)
        assert near(self.y, y, back(err_y) + 2 * U * (np.abs(y) + (0 if r is None else np.abs(r))) + unit * np.abs(y))
        dx, dW, dbias, dz = linear.linear_bwd(dy, x, W, bias, self.act, self.x_first, self.y_first)
        err = 0 * dz if plain else np.abs(g) * (1.13 * err_z + U * (8 + 2 * np.abs(z)) * (1 + np.abs(z)))
        rounded = err if plain else err + unit * (np.abs(dz) + err) + tiny
        adz = np.abs(dz) + rounded
        bound = (rounded + (M + 4) * U * adz) @ np.abs(W)
        assert near(self.dx, dx, linear.last(bound, self.x_first) + unit * np.abs(dx))
        flat = lambda t: t.reshape(T, -1)  # noqa: E731
        bound = flat(rounded + (T + 4) * U * adz).T @ flat(np.abs(rows))
        assert near(self.dW, dW, bound + (UNIT[self.io] if self.dW.dtype != torch.float32 else U) * np.abs(dW))
        assert near(self.dbias, dbias, flat(err + (T + 4) * U * (np.abs(dz) + err)).sum(0))
        return self


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("x_first", [False, True])
@pytest.mark.parametrize("y_first", [False, True])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_layouts_and_activations_against_oracle(io, x_first, y_first, act):
    Run(2, 37, 40, 72, io, act, residual=True, x_first=x_first, y_first=y_first).fwd().bwd().check()


# one place, one column, around tiles of 128 and steps of 64 (16 in fp32), odd everything
@pytest.mark.parametrize("B,N,K,M", [(1, 1, 1, 1), (1, 1, 64, 128), (4, 1, 130, 33), (1, 128, 128, 128), (1, 129, 65, 127), (3, 5, 7, 300), (2, 200, 193, 9),
                                     (1, 257, 8, 257), (7, 3, 520, 5), (2, 130, 16, 260), (40, 2, 31, 31)])
@pytest.mark.parametrize("io", ["fp32", "bf16"])
@pytest.mark.parametrize("firsts", [(False, False), (True, True), (False, True)])
def test_sizes(B, N, K, M, io, firsts):
    Run(B, N, K, M, io, "none", x_first=firsts[0], y_first=firsts[1], seed=1).fwd().bwd().check()
    Run(B, N, K, M, io, "silu", bias=False, x_first=firsts[0], y_first=firsts[1], dW=io, seed=2).fwd().bwd().check()


# few places, as in decoding: on both sides of what goes by another kernel, if one does
@pytest.mark.parametrize("T", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65])
@pytest.mark.parametrize("K,M", [(768, 256), (100, 77), (4096, 40)])
@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
def test_few_places(T, K, M, io):
    Run(T, 1, K, M, io, "gelu", residual=True, seed=3).fwd().bwd().check()


@pytest.mark.parametrize("io,B,N,K,M,firsts", [("bf16", 3, 700, 256, 512, (False, True)), ("fp16", 2, 1030, 520, 264, (True, False)),
                                               ("fp32", 2, 600, 200, 150, (True, True)), ("bf16", 1, 4000, 96, 640, (False, False))])
def test_several_tiles_and_shares(io, B, N, K, M, firsts):
    Run(B, N, K, M, io, "silu", residual=True, x_first=firsts[0], y_first=firsts[1], dW=io, seed=4).fwd().bwd().check()
    Run(B, N, K, M, io, "none", x_first=firsts[0], y_first=firsts[1], seed=5).fwd().bwd().check()


def test_relu():
    r = Run(2, 20, 30, 40, "fp32", "relu", residual=True, seed=6)
    r.bias.copy_(torch.where(torch.arange(40, device="cuda") % 2 == 0, 30.0, -30.0))       # its slope jumps at zero: z stays away from it
    r.fwd().bwd().check()


def test_onto_the_residual_in_place():
    for first in (False, True):
        r = Run(3, 70, 40, 136, "bf16", "gelu", residual=True, y_first=first, seed=7).fwd()
        want = r.y.clone()
        r.y = r.residual
        r.fwd()
        assert torch.equal(r.y, want)


def test_optional_results_and_repeatability():
    for act in ("none", "silu"):
        r = Run(3, 300, 70, 90, "fp16", act, seed=8).fwd().bwd()
        want = [t.clone() for t in (r.dx, r.dW, r.dbias)]
        for i in range(3):
            for t in (r.dx, r.dW, r.dbias):
                t.fill_(5.0)
            r.bwd(*(j == i for j in range(3)))
            assert torch.equal((r.dx, r.dW, r.dbias)[i], want[i])
            assert all((t == 5).all() for j, t in enumerate((r.dx, r.dW, r.dbias)) if j != i)


@pytest.mark.parametrize("firsts", [(False, False), (True, True), (False, True), (True, False)])
def test_a_value_that_is_not_finite_stays_in_its_place(firsts):
    r, clean = (Run(2, 150, 70, 140, "bf16", "none", x_first=firsts[0], y_first=firsts[1], seed=9) for _ in range(2))
    place = 77
    (r.x[1, 3] if firsts[0] else r.x[1, :, 3])[place] = float("nan")
    for q in (r, clean):
        q.fwd()
    bad = torch.zeros_like(r.y, dtype=torch.bool)
    (bad[1].t() if firsts[1] else bad[1])[place] = True
    assert torch.equal(r.y[~bad], clean.y[~bad]) and r.y[bad].isnan().all()


def test_refusals():
    r = Run(2, 3, 16, 8, "fp32")
    with pytest.raises(lc.LongconvError, match="W"):
        lc.longconv_linear_fwd(r.x, r.W.half(), None, r.y, "none", r.ws)
    with pytest.raises(lc.LongconvError, match="y:"):
        lc.longconv_linear_fwd(r.x, r.W, None, r.y, "none", r.ws, lc.CHANNELS_LAST, lc.CHANNELS_FIRST)
    with pytest.raises(lc.LongconvError, match="layout"):
        lc.longconv_linear_fwd(r.x, r.W, None, r.y, "none", r.ws, 2)
    with pytest.raises(lc.LongconvError, match="dW"):
        lc.longconv_linear_bwd(r.dy, r.x, r.W, None, r.dx, r.dW.half(), None, "none", r.ws)
    with pytest.raises(lc.LongconvError, match="workspace"):
        lc.longconv_linear_bwd(r.dy, r.x, r.W, None, r.dx, r.dW, None, "none", r.ws[:4])


def test_under_graph_capture_on_a_side_stream():
    r = Run(3, 600, 96, 264, "bf16", "silu", residual=True, y_first=True, seed=10).fwd().bwd()
    kept = [r.y, r.dx, r.dW, r.dbias]
    want = [t.clone() for t in kept]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.fwd().bwd()
        with torch.cuda.graph(graph, stream=side):
            r.fwd().bwd()
    torch.cuda.synchronize()
    for again in range(3):
        for t in kept:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, kept))


# one sequence, or one place of each: what is few places in one layout is columns in another
@pytest.mark.parametrize("B,N", [(1, 1), (1, 2), (1, 17), (1, 64), (5, 1), (64, 1)])
@pytest.mark.parametrize("firsts", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("io", ["fp32", "bf16"])
def test_few_places_in_other_layouts(B, N, firsts, io):
    Run(B, N, 72, 136, io, "silu", residual=True, x_first=firsts[0], y_first=firsts[1], seed=11).fwd().bwd().check()


# the sums' shares where places are few and tiles many, and where tiles are the largest; a workspace of just the size asked for
@pytest.mark.parametrize("io,B,N,K,M,firsts", [("bf16", 200, 32, 64, 256, (False, True)), ("fp16", 260, 24, 256, 64, (True, True)), ("bf16", 1, 1, 16, 65528, (False, False)),
                                               ("fp16", 1, 3300, 64, 4096, (False, False)), ("bf16", 2, 1600, 64, 4096, (False, True)),
                                               ("fp32", 120, 8, 8, 72, (True, True)), ("bf16", 3, 200, 1024, 1032, (False, False))])
def test_writes_stay_within_the_workspace(io, B, N, K, M, firsts):
    for act in ("silu", "none"):
        r = Run(B, N, K, M, io, act, x_first=firsts[0], y_first=firsts[1], seed=12)
        room = torch.full((r.ws.numel() + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        r.ws = room[:-65536]
        r.fwd().bwd().check()
        assert (room[-65536:] == 0x5A).all()


# long sums, whose tiles are the largest where they fill the card: with a remainder on each side, in each layout, and short sums beside
@pytest.mark.parametrize("firsts", [(False, False), (True, True), (False, True), (True, False)])
@pytest.mark.parametrize("K", [1016, 1032])
def test_the_largest_tiles(K, firsts):
    Run(1, 3400, K, 3544, "bf16", "silu", residual=True, x_first=firsts[0], y_first=firsts[1], dW="bf16", seed=13).fwd().bwd().check()


# few tiles and a long sum, which is cut into shares: forward, behind an activation and in dx; workspaces of just the size asked for, the forward call's its own
@pytest.mark.parametrize("B,N,K,M", [(1, 130, 4096, 40), (3, 70, 2056, 136), (2, 65, 2113, 77), (1, 200, 72, 3000), (2, 100, 2054, 2100), (1, 70, 515, 33)])
@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("firsts", [(False, False), (True, True), (False, True), (True, False)])
def test_long_sums_of_few_tiles(B, N, K, M, io, firsts):
    for act, residual in (("silu", True), ("none", False)):
        r = Run(B, N, K, M, io, act, residual=residual, x_first=firsts[0], y_first=firsts[1], seed=14)
        code, back = lc.dtype_code(r.x), r.ws
        small = lc.longconv_linear_workspace_bytes(B, N, K, M, code, False)
        assert small <= back.numel()
        room = torch.full((back.numel() + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        r.ws = room[:small]
        r.fwd()
        assert (room[small:] == 0x5A).all()
        r.ws = room[:back.numel()]
        r.bwd().check()
        assert (room[back.numel():] == 0x5A).all()


# sums of dbias by tiles of 256 that are filled least, by other tiles, by cut sums and by dW's shares; each within a workspace of just the size asked for
@pytest.mark.parametrize("io,B,N,K,M,firsts", [("bf16", 13, 200, 1024, 4096, (False, True)), ("fp16", 13, 200, 1024, 4096, (True, False)), ("bf16", 200, 1, 1024, 49432, (False, False)),
                                               ("bf16", 193, 1, 72, 136, (True, True)), ("fp32", 100, 1, 520, 72, (False, True)), ("bf16", 130, 1, 2056, 40, (False, False)),
                                               ("fp16", 300, 2, 64, 72, (True, True)), ("fp32", 90, 3, 70, 33, (False, True)), ("bf16", 1, 1, 8, 8, (False, False))])
def test_sums_of_dbias_stay_within_the_workspace(io, B, N, K, M, firsts):
    for act in ("silu", "none"):
        r = Run(B, N, K, M, io, act, x_first=firsts[0], y_first=firsts[1], seed=16)
        room = torch.full((r.ws.numel() + 65536,), 0x5A, dtype=torch.uint8, device="cuda")
        r.ws = room[:-65536]
        r.bwd()
        assert (room[-65536:] == 0x5A).all()
        r.bwd(dx=False, dW=False)
        assert (room[-65536:] == 0x5A).all()
        if M < 10000:
            r.fwd().bwd().check()
            continue
        z = r.x.double().view(-1, K) @ r.W.double().t() + r.bias        # (as check() bounds it, on the GPU)
        q, dy = torch.sigmoid(z), r.dy.double().view(-1, M)
        dz = dy * (q * (1 + z * (1 - q))) if act == "silu" else dy
        size = r.x.double().abs().view(-1, K) @ r.W.double().abs().t() + r.bias.abs()
        err = 0 * dz if act == "none" else dy.abs() * (1.13 * (K + 4) * U * size + U * (8 + 2 * z.abs()) * (1 + z.abs()))
        assert ((r.dbias - dz.sum(0)).abs() <= (err + (B * N + 4) * U * (dz.abs() + err)).sum(0)).all()


# dbias has the same bits whichever results are asked for beside it: rows of whole pieces, where it comes of dW's products, tiles of 128 and of 256, and others
@pytest.mark.parametrize("io,B,N,K,M", [("bf16", 3, 400, 128, 264), ("fp16", 1, 72, 8, 8), ("bf16", 2, 520, 1024, 1032), ("bf16", 2, 51, 40, 136),
                                        ("fp16", 5, 1, 64, 4096), ("fp32", 2, 90, 40, 72), ("bf16", 2, 2600, 64, 8)])
@pytest.mark.parametrize("firsts", [(False, False), (True, True), (False, True), (True, False)])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_dbias_is_the_same_beside_any_results(io, B, N, K, M, firsts, act):
    r = Run(B, N, K, M, io, act, x_first=firsts[0], y_first=firsts[1], seed=15).fwd().bwd().check()
    want = r.dbias.clone()
    for dx, dW in ((False, False), (True, False), (False, True)):
        r.dbias.fill_(5.0)
        r.bwd(dx=dx, dW=dW)
        assert torch.equal(r.dbias, want), (dx, dW)


# fp32, a sum that makes two shares, on both sides of the length from which it is cut: forward, behind an activation, and in dx
@pytest.mark.parametrize("K", [513, 864, 865, 900, 1009])
@pytest.mark.parametrize("T,M", [(700, 1400), (2695, 193), (65 * 16, 11 * 64 - 3)])
def test_sums_of_two_shares(K, T, M):
    Run(1, T, K, M, "fp32", "silu", residual=True, y_first=True, seed=17).fwd().bwd().check()
    Run(5, T // 5, M, K, "fp32", "none", seed=18).fwd().bwd().check()
