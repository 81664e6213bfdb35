"""A block that mixes places by a selective scan, in the convolution's layout [B, H, N]: every step of it a call of this library.

    u    = silu(short convolution of W_u x)                 longconv_linear_fwd, longconv_short_fwd, [B, E, N]
    z    = W_z x                                            the gate
    B, C = W_B u, W_C u                                     [B, groups, states, N]
    y    = W_y scan(u, W_d W_r u, A, B, C, z) + residual    longconv_scan_fwd with A = -exp(rate), longconv_linear_fwd

Its backward pass gives the gradients of all parameters, and `step` one new place of each sequence from the state that the sequence left.
`classifier.py` runs it in the long convolution's place (`--mixer scan`).
"""
from __future__ import annotations

import math

import torch

import paper_2302_06646_amd as lc

FIRST = lc.CHANNELS_FIRST


class Selective:
    """Parameters (fp32, float32 gradients in `.grad`), workspaces and activations for batches of B sequences of N places of H values."""

    def __init__(self, B, N, H, inner=None, states=16, taps=4, rank=None, groups=1, dtype=torch.bfloat16, train=True, generator=None):
        E, R = inner or 2 * H, rank or max(1, H // 16)
        randn = lambda *s: torch.randn(*s, generator=generator, device="cuda")  # noqa: E731
        self.B, self.N, self.H, self.E, self.S, self.G, self.taps, self.dtype, self.train = B, N, H, E, states, groups, taps, dtype, train
        dt = torch.exp(torch.rand(E, generator=generator, device="cuda") * math.log(100.0) + math.log(1e-3))      # 0.001 to 0.1
        shapes = {"W_u": (E, H), "W_z": (E, H), "W_r": (R, E), "W_d": (E, R), "W_B": (groups * states, E), "W_C": (groups * states, E), "W_y": (H, E)}
        self.p = {k: randn(*s) / math.sqrt(s[1]) for k, s in shapes.items()}
        self.p.update(taps=randn(E, taps) / math.sqrt(taps), taps_bias=torch.zeros(E, device="cuda"),
                      rate=torch.log(torch.arange(1.0, states + 1, device="cuda")).repeat(E, 1), D=torch.ones(E, device="cuda"),
                      dt_bias=dt + torch.log(-torch.expm1(-dt)))      # softplus of it is dt
        self.low = {k: torch.empty_like(self.p[k], dtype=dtype) for k in shapes}      # the products' operands, in the I/O type
        self.A = torch.empty(E, states, device="cuda")
        new = lambda *s: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        wide, of_states = (B, E, N), (B, groups, states, N)
        self.u0, self.u, self.z, self.delta, self.y = (new(*wide) for _ in range(5))
        self.r, self.Bm, self.Cm = new(B, R, N), new(*of_states), new(*of_states)
        io = lc.dtype_code(self.u)
        room = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.ws_scan = lc.new_workspace_scan(B, E, N, states, groups, io, train)
        self.ws_linear = room(max(lc.longconv_linear_workspace_bytes(B, n, k, m, io, train) for m, k in shapes.values() for n in (N, 1)))
        self.marks = None
        if train:
            for t in self.p.values():
                t.grad = torch.zeros_like(t)
            self.marks = lc.new_scan_marks(B, E, N, states)
            self.ws_short = lc.new_workspace_short(B, E, N, taps, io)
            self.du0, self.du, self.dz, self.ddelta, self.dy, self.more = (new(*wide) for _ in range(6))
            self.dr, self.dB, self.dC, self.dx, self.x = new(B, R, N), new(*of_states), new(*of_states), new(B, H, N), new(B, H, N)
            self.one = torch.ones(H, 1, device="cuda")
            self.dA = torch.empty_like(self.A)
        self.refresh()

    def refresh(self):
        """The operands of the kernels from the parameters: once behind each change of these."""
        for k, t in self.low.items():
            t.copy_(self.p[k])
        torch.exp(self.p["rate"], out=self.A).neg_()

    def _linear(self, name, x, y, residual=None):
        lc.longconv_linear_fwd(x, self.low[name], None, y, "none", self.ws_linear, FIRST, FIRST, residual)

    def _linear_back(self, name, dy, x, dx):
        lc.longconv_linear_bwd(dy, x, self.low[name], None, dx, self.p[name].grad, None, "none", self.ws_linear, FIRST, FIRST)

    def _inside(self, t, to, lengths):
        """`to` <- t up to each sequence's end and zeros behind it: the short convolution whose one tap is 1."""
        lc.longconv_short_fwd(t, self.one, None, to, "none", lengths=lengths)
        return to

    def _rows(self, t):
        return t.view(self.B, self.G * self.S, self.N)

    def new_state(self):
        """For a sequence's beginning: the short convolution's last inputs and the scan's states."""
        return (torch.zeros(self.B, self.E, self.taps - 1, dtype=self.dtype, device="cuda"), torch.zeros(self.B, self.E, self.S, device="cuda"))

    def forward(self, x, y, lengths=None, residual=None, state=None):
        """y [B, H, N] of x [B, H, N] (y may be `residual`).  lengths [B] int64: what lies behind a sequence's end takes no part.  state: of
        new_state(), moved on in place (a backward pass follows only a call without one)."""
        p, (short, scan) = self.p, state or (None, None)
        self._linear("W_u", x, self.u0)
        self._linear("W_z", x, self.z)
        lc.longconv_short_fwd(self.u0, p["taps"], p["taps_bias"], self.u, "silu", state=short, last=short, lengths=lengths)
        self._linear("W_r", self.u, self.r)
        self._linear("W_d", self.r, self.delta)
        self._linear("W_B", self.u, self._rows(self.Bm))
        self._linear("W_C", self.u, self._rows(self.Cm))
        lc.longconv_scan_fwd(self.u, self.delta, self.A, self.Bm, self.Cm, self.y, self.ws_scan, D=p["D"], z=self.z, bias=p["dt_bias"], state=scan,
                             last=scan, marks=None if state else self.marks, lengths=lengths)
        self._linear("W_y", self.y, y, residual)

    def backward(self, dy, x, dx, lengths=None):
        """dx and the parameters' gradients from dy, behind forward() of the same x and lengths (the residual's gradient is dy).  Where several
        gradients of a tensor meet they are added in the I/O type, as they are kept."""
        p = self.p
        if lengths is not None:      # (products over places take all of them: zeros of the other operand do not take NaN or infinity out)
            x, dy = self._inside(x, self.x, lengths), self._inside(dy, self.dx, lengths)
        self._linear_back("W_y", dy, self.y, self.dy)
        lc.longconv_scan_bwd(self.dy, self.u, self.delta, self.A, self.Bm, self.Cm, self.marks, self.du, self.ddelta, self.dA, self.dB, self.dC,
                             self.ws_scan, D=p["D"], z=self.z, bias=p["dt_bias"], dD=p["D"].grad, dz=self.dz, dbias=p["dt_bias"].grad,
                             lengths=lengths)
        torch.mul(self.dA, self.A, out=p["rate"].grad)
        self._linear_back("W_d", self.ddelta, self.r, self.dr)
        for name, d in (("W_r", self.dr), ("W_B", self._rows(self.dB)), ("W_C", self._rows(self.dC))):
            self._linear_back(name, d, self.u, self.more)
            self.du.add_(self.more)
        lc.longconv_short_bwd(self.du, self.u0, p["taps"], p["taps_bias"], self.du0, p["taps"].grad, p["taps_bias"].grad, "silu", self.ws_short,
                              lengths=lengths)
        self._linear_back("W_u", self.du0, x, dx)
        self._linear_back("W_z", self.dz, x, self.dx)
        dx.add_(self.dx)

    def step(self, x, y, state, residual=None):
        """One new place of each sequence, x, y [B, H] (y may be `residual`); state, of new_state() or as forward() left it, is moved on."""
        p, (short, scan), B = self.p, state, self.B
        new = lambda n: torch.empty(B, n, dtype=self.dtype, device="cuda")  # noqa: E731
        def linear(name, x, n, y=None, residual=None):
            y = new(n) if y is None else y
            lc.longconv_linear_fwd(x[:, None], self.low[name], None, y[:, None], "none", self.ws_linear,
                                   residual=None if residual is None else residual[:, None])
            return y
        u, out = new(self.E), new(self.E)
        lc.longconv_short_step(linear("W_u", x, self.E), p["taps"], p["taps_bias"], short, u, "silu")
        delta = linear("W_d", linear("W_r", u, self.low["W_r"].shape[0]), self.E)
        Bm, Cm = (linear(k, u, self.G * self.S).view(B, self.G, self.S) for k in ("W_B", "W_C"))
        lc.longconv_scan_step(u, delta, self.A, Bm, Cm, scan, out, D=p["D"], z=linear("W_z", x, self.E), bias=p["dt_bias"])
        linear("W_y", out, self.H, y, residual)
