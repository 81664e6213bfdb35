"""Short causal convolution against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2302_06646_amd as lc
from oracle import gnorm, short

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}
U = 2.0 ** -24


def _np(t):
    return None if t is None else t.detach().cpu().double().numpy()


class Run:
    def __init__(self, B, H, N, taps, io, act, bias=True, carry=False, lengths=None, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        dt = DT[io]
        self.io, self.act, self.taps = io, act, taps
        self.x, self.dy = r(B, H, N).to(dt).cuda(), r(B, H, N).to(dt).cuda()
        self.k, self.bias = r(H, taps).cuda(), r(H).cuda() if bias else None
        self.state, self.dlast = (r(B, H, taps - 1).to(dt).cuda() if carry else None for _ in range(2))
        self.lengths = None if lengths is None else torch.tensor(lengths, device="cuda")
        new = lambda *s, dt=dt: torch.full(s, 7.0, dtype=dt, device="cuda")  # noqa: E731
        self.y, self.dx, self.last, self.dstate = new(B, H, N), new(B, H, N), new(B, H, taps - 1), new(B, H, taps - 1)
        self.dk, self.dbias = new(H, taps, dt=torch.float32), new(H, dt=torch.float32)
        self.ws = lc.new_workspace_short(B, H, N, taps, lc.dtype_code(self.x))
        self.ws.fill_(0xA5)

    def run(self):
        lc.longconv_short_fwd(self.x, self.k, self.bias, self.y, self.act, state=self.state, last=self.last, lengths=self.lengths)
        lc.longconv_short_bwd(self.dy, self.x, self.k, self.bias, self.dx, self.dk, self.dbias, self.act, self.ws, state=self.state,
                              dlast=self.dlast, dstate=self.dstate, lengths=self.lengths)
        return self

    def check(self):
        """Sums of at most nine terms: ten roundings of the sum of their sizes.  An activation is off by (8 + |z|) U |z| (its exponential's
        argument is rounded: |z| U; gelu's distribution function by 4 U of one), its slope by (8 + 2 |z|) U (1 + |z|); slopes are at most 1.13
        and so are theirs.  dk and dbias: 40 terms one by one in a thread and a tree above, 64 roundings at most."""
        H, N = self.x.shape[1:]
        x, dy, k = _np(self.x), _np(self.dy), _np(self.k)
        bias = np.zeros(H) if self.bias is None else _np(self.bias)
        lengths = _np(self.lengths)
        there = np.arange(N) < (np.full(len(x), N) if lengths is None else np.clip(lengths, 0, N))[:, None]
        x, dy = np.where(there[:, None], x, 0), np.where(there[:, None], dy, 0)
        y, last = short.short_fwd(x, k, bias, self.act, _np(self.state), lengths)
        dx, dk, dbias, dstate = short.short_bwd(dy, x, k, bias, self.act, _np(self.state), lengths, _np(self.dlast))
        unit, tiny = UNIT[self.io], TINY[self.io]
        absolute = lambda a: None if a is None else np.abs(a)  # noqa: E731
        z, _ = short.short_fwd(x, k, bias, "none", _np(self.state), lengths)
        size, _ = short.short_fwd(np.abs(x), np.abs(k), np.abs(bias), "none", absolute(_np(self.state)), lengths)
        err_z = 10 * U * size
        near = lambda got, want, bound: (np.abs(_np(got) - want) <= bound + tiny).all()  # noqa: E731
        assert near(self.y, y, 1.13 * err_z + (U * (8 + np.abs(z)) * np.abs(z) if self.act != "none" else 0) + unit * np.abs(y))
        assert torch.equal(self.last.cpu(), torch.from_numpy(last).to(DT[self.io]))
        slope = np.abs(gnorm.act(z, self.act)[1])
        err = np.abs(dy) * (1.13 * err_z + U * (8 + 2 * np.abs(z)) * (1 + np.abs(z))) if self.act != "none" else 0 * dy
        adj = lambda e: short.short_bwd(e, np.abs(x), np.abs(k), 0 * bias, "none", absolute(_np(self.state)), lengths,  # noqa: E731
                                        absolute(_np(self.dlast)))
        e_dx, e_dk, e_db, e_ds = adj(err)
        s_dx, s_dk, s_db, s_ds = adj(np.abs(dy) * slope)
        assert near(self.dx, dx, e_dx + 10 * U * s_dx + unit * np.abs(dx))
        assert near(self.dstate, dstate, e_ds + 10 * U * s_ds + unit * np.abs(dstate))
        assert near(self.dk, dk, e_dk + 64 * U * (s_dk + e_dk)) and near(self.dbias, dbias, e_db + 64 * U * (s_db + e_db))
        return self


@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("taps", [1, 2, 4, 5, 8])
def test_forward_and_backward_against_oracle(io, act, taps):
    if act == "relu":      # its slope jumps where z is zero to rounding: heads whose z stay away from it
        r = Run(2, 3, 45, taps, io, act, seed=3)
        r.k.abs_(), r.bias.abs_()
        r.x.abs_().add_(0.5)
        r.run().check()
        return
    Run(2, 3, 45, taps, io, act).run().check()


# one place to several workgroups, around pieces of eight and around the taps
@pytest.mark.parametrize("B,H,N", [(1, 1, 1), (5, 2, 2), (3, 4, 3), (2, 3, 7), (2, 2, 8), (1, 3, 9), (2, 1, 17), (3, 2, 1000), (1, 1, 20000), (70, 5, 33), (2, 193, 10)])
@pytest.mark.parametrize("taps,io", [(4, "bf16"), (8, "fp32"), (3, "fp16")])
def test_sizes_with_states(B, H, N, taps, io):
    Run(B, H, N, taps, io, "silu", carry=True, seed=1).run().check()


@pytest.mark.parametrize("taps", [1, 4, 8])
@pytest.mark.parametrize("carry", [False, True])
def test_uneven_lengths(taps, carry):
    # none, one, fewer than the taps, around pieces, all, and what is outside counts as none or all
    lengths = [0, 1, 2, 7, 8, 9, 15, 16, 17, 30, 31, 99, -3]
    r = Run(len(lengths), 3, 31, taps, "fp32", "silu", carry=carry, lengths=lengths, seed=2)
    for b, n in enumerate(np.clip(lengths, 0, 31)):
        r.x[b, :, n:] = float("nan")
        r.dy[b, :, n:] = float("inf")
    r.run().check()
    for b, n in enumerate(np.clip(lengths, 0, 31)):
        assert not r.y[b, :, n:].any() and not r.dx[b, :, n:].any()


def test_parts_of_a_sequence_make_the_whole_and_steps_do():
    B, H, N, taps = 3, 20, 50, 4
    r = Run(B, H, N, taps, "fp16", "silu").run()
    state, y = torch.zeros(B, H, taps - 1, dtype=torch.float16, device="cuda"), torch.empty_like(r.y)
    for a, b in ((0, 1), (1, 2), (2, 30), (30, 50)):
        x, part = r.x[:, :, a:b].contiguous(), torch.empty(B, H, b - a, dtype=torch.float16, device="cuda")
        lc.longconv_short_fwd(x, r.k, r.bias, part, "silu", state=state, last=state)         # in place
        y[:, :, a:b] = part
    assert torch.equal(y, r.y) and torch.equal(state, r.last)
    state.zero_()
    for t in range(N):
        out = torch.empty(B, H, dtype=torch.float16, device="cuda")
        lc.longconv_short_step(r.x[:, :, t].contiguous(), r.k, r.bias, state, out, "silu")
        y[:, :, t] = out
    assert torch.equal(y, r.y) and torch.equal(state, r.last)


@pytest.mark.parametrize("taps", [1, 2, 8])
@pytest.mark.parametrize("io", ["fp32", "bf16"])
def test_step_against_oracle(taps, io):
    r = Run(5, 67, 1, taps, io, "gelu", carry=True, seed=4)
    r.run().check()
    state, y = r.state.clone(), torch.empty(5, 67, dtype=DT[io], device="cuda")
    lc.longconv_short_step(r.x[..., 0].contiguous(), r.k, r.bias, None if taps == 1 else state, y, "gelu")
    assert torch.equal(y, r.y[..., 0]) and torch.equal(state, r.last)


def test_gradients_through_parts():
    # two parts, the second one's dstate the first one's dlast, as one sequence
    B, H, N, taps, a = 2, 3, 40, 4, 13
    r = Run(B, H, N, taps, "fp32", "silu", carry=True, seed=5).run()
    def part(s, state, dlast):
        q = Run(B, H, s.stop - s.start, taps, "fp32", "silu", carry=True)
        q.x, q.dy, q.k, q.bias, q.state, q.dlast = r.x[:, :, s].contiguous(), r.dy[:, :, s].contiguous(), r.k, r.bias, state, dlast
        return q.run()
    middle = r.x[:, :, a - taps + 1:a].contiguous()
    second = part(slice(a, N), middle, r.dlast)
    first = part(slice(0, a), r.state, second.dstate)
    # dx of the last places before the cut gets its second part rounded once more
    assert torch.allclose(torch.cat([first.dx, second.dx], 2), r.dx, rtol=1e-5, atol=1e-5) and torch.allclose(first.dstate, r.dstate, atol=1e-5)
    assert torch.allclose(first.dk + second.dk, r.dk, rtol=1e-4, atol=1e-4) and torch.allclose(first.dbias + second.dbias, r.dbias, rtol=1e-4, atol=1e-4)


def test_optional_results_and_repeatability():
    r = Run(4, 6, 300, 4, "bf16", "silu", carry=True, seed=6).run()
    want = [t.clone() for t in (r.dx, r.dk, r.dbias, r.dstate)]
    r.run()
    assert all(torch.equal(a, b) for a, b in zip(want, (r.dx, r.dk, r.dbias, r.dstate)))
    for i in range(4):
        out = [torch.zeros_like(t) if j == i else None for j, t in enumerate(want)]
        lc.longconv_short_bwd(r.dy, r.x, r.k, r.bias, out[0], out[1], out[2], "silu", r.ws, state=r.state, dlast=r.dlast, dstate=out[3])
        assert torch.equal(out[i], want[i])


def test_a_value_that_is_not_finite_reaches_its_taps_alone():
    r, clean = (Run(2, 3, 60, 3, "fp32", "silu", seed=7) for _ in range(2))
    r.x[1, 2, 20] = float("nan")
    for q in (r, clean):
        q.run()
    bad = torch.zeros_like(r.y, dtype=torch.bool)
    bad[1, 2, 20:23] = True
    assert torch.equal(r.y[~bad], clean.y[~bad]) and r.y[bad].isnan().all()
    bad[1, 2, 18:20] = True                       # dx: places whose taps reach a z that is NaN
    assert torch.equal(r.dx[~bad], clean.dx[~bad])


def test_refusals():
    r = Run(2, 3, 16, 4, "fp32", "silu", carry=True)
    with pytest.raises(lc.LongconvError, match="contiguous"):
        lc.longconv_short_fwd(r.x.transpose(0, 1).contiguous().transpose(0, 1), r.k, r.bias, r.y, "silu")
    with pytest.raises(lc.LongconvError, match="state"):
        lc.longconv_short_fwd(r.x, r.k, r.bias, r.y, "silu", state=r.state[..., :2].contiguous())
    with pytest.raises(lc.LongconvError, match="lengths"):
        lc.longconv_short_fwd(r.x, r.k, r.bias, r.y, "silu", lengths=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(lc.LongconvError, match="workspace"):
        lc.longconv_short_bwd(r.dy, r.x, r.k, r.bias, r.dx, r.dk, r.dbias, "silu", r.ws[:8])
    with pytest.raises(lc.LongconvError, match="bad shape|unsupported|shape"):
        lc.longconv_short_fwd(r.x, torch.zeros(3, 9, device="cuda"), None, r.y, "silu")


def test_under_graph_capture_on_a_side_stream():
    r = Run(3, 40, 600, 4, "bf16", "silu", carry=True, lengths=[600, 10, 333], seed=8).run()
    want = [t.clone() for t in (r.y, r.last, r.dx, r.dk, r.dbias, r.dstate)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.run()
        with torch.cuda.graph(graph, stream=side):
            r.run()
    torch.cuda.synchronize()
    for again in range(3):
        for t in (r.y, r.last, r.dx, r.dk, r.dbias, r.dstate):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (r.y, r.last, r.dx, r.dk, r.dbias, r.dstate)))


# rows that go by whole waves in the backward pass: around 64 pieces of eight, units of 128, and several units.  Few rows: a thread adds up one unit,
# sixteen terms
@pytest.mark.parametrize("N", [504, 505, 512, 513, 900, 1023, 1024, 1025, 1031, 1536, 2048, 2051, 4000])
@pytest.mark.parametrize("taps,io,act", [(4, "bf16", "silu"), (8, "fp32", "gelu"), (2, "fp16", "none")])
def test_long_rows(N, taps, io, act):
    Run(3, 2, N, taps, io, act, carry=True, seed=6).run().check()


@pytest.mark.parametrize("taps", [1, 4, 8])
@pytest.mark.parametrize("carry", [False, True])
def test_uneven_lengths_of_long_rows(taps, carry):
    N, lengths = 2060, [0, 1, 3, 511, 512, 513, 1023, 1024, 1025, 1027, 1031, 1032, 2047, 2048, 2052, 2060]
    r = Run(len(lengths), 2, N, taps, "fp32", "silu", carry=carry, lengths=lengths, seed=7)
    for b, n in enumerate(lengths):
        r.x[b, :, n:] = float("nan")
        r.dy[b, :, n:] = float("inf")
    r.run().check()
    for b, n in enumerate(lengths):
        assert not r.y[b, :, n:].any() and not r.dx[b, :, n:].any()
