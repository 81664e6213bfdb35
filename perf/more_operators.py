"""Operators of layers beside the long convolution, as cases to be timed and compared: a short causal convolution, a selective state
space scan, and the dense product between layers, for training, for prompts and for single tokens.

A case names one of five paths:

  short       y = act(k * x + bias), a causal convolution of a few taps per head, [B,H,N]; alone or with its backward pass
  short_step  the same for one new token of each sequence, with the last inputs kept as its state
  scan        h_t = exp(dt_t A) h_{t-1} + dt_t B_t u_t,  y_t = (C_t h_t + D u_t) silu(z_t),  dt = softplus(delta + bias), [B,H,N]
  scan_step   the same for one new token, with h as its state
  linear      y = act(x W^T + bias) + residual, from and to [B,N,.] ("last") or [B,.,N] ("first")

`run` computes them in their plain form, elementary operations in 32 bits, or, where `own` is true, by the library's calls.

Sequences of uneven lengths: places behind a sequence's end count for nothing, are zero in what is written, and the last state is that
of the end.  States that go in (`carry`) are those of the sequence's part before, and their gradients come back.
"""
import math

import torch

own = False

_DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}


def listed():
    return [
        # 64 sequences being decoded: their next tokens through a layer's short convolution, nothing but latency
        dict(name="short_token_bf16", path="short_step", B=64, H=1024, taps=4, act="silu", bias=True, io="bf16"),
        # language-model block, training step
        dict(name="short_lm_bf16", path="short", B=16, H=1024, N=1024, taps=4, act="silu", bias=True, io="bf16", train=True, carry=False,
             ragged=False),
        # prompts of uneven lengths, whose last inputs start the decoding
        dict(name="short_prompt_fp16", path="short", B=8, H=256, N=16384, taps=4, act="silu", bias=True, io="fp16", train=False,
             carry=False, ragged=True),
        # odd counts everywhere, full precision, a sequence trained part by part
        dict(name="short_odd_fp32", path="short", B=7, H=193, N=385, taps=3, act="none", bias=False, io="fp32", train=True, carry=True,
             ragged=False),
        # the next tokens of 64 sequences through the scan: 4 MB of state in and out
        dict(name="scan_token_bf16", path="scan_step", B=64, H=1024, S=16, G=1, gated=True, softplus=True, io="bf16"),
        # language-model block, training step, the largest there is
        dict(name="scan_lm_bf16", path="scan", B=16, H=1024, N=1024, S=16, G=1, gated=True, softplus=True, io="bf16", train=True,
             carry=False, ragged=False),
        # prompts of uneven lengths
        dict(name="scan_prompt_fp16", path="scan", B=8, H=256, N=16384, S=16, G=1, gated=False, softplus=True, io="fp16", train=False,
             carry=False, ragged=True),
        # odd counts everywhere, full precision, a sequence trained part by part
        dict(name="scan_odd_fp32", path="scan", B=7, H=193, N=385, S=5, G=1, gated=True, softplus=False, io="fp32", train=True,
             carry=True, ragged=False),
        # the next tokens of four sequences into a wider layer: the weights are what is read
        dict(name="linear_token_bf16", path="linear", B=4, N=1, K=768, M=2048, act="gelu", bias=True, residual=False, x="last", y="last",
             io="bf16", train=False),
        # language-model block: from the layout of dense layers into the convolution's, training step
        dict(name="linear_lm_bf16", path="linear", B=16, N=1024, K=768, M=2048, act="none", bias=True, residual=False, x="last",
             y="first", io="bf16", train=True),
        # feed-forward layer on long sequences, activation recomputed in the backward pass
        dict(name="linear_wide_fp16", path="linear", B=8, N=16384, K=256, M=1024, act="gelu", bias=True, residual=False, x="last",
             y="last", io="fp16", train=True),
        # odd counts everywhere, full precision, out of the convolution's layout onto a residual
        dict(name="linear_odd_fp32", path="linear", B=7, N=385, K=193, M=1009, act="silu", bias=True, residual=True, x="first", y="last",
             io="fp32", train=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the same paths: 1 to 64 sequences, any length up to 16384, 1 to 1024 heads, 1 to 8 taps, 1 to 64 states in 1 to 4
    groups of heads, dense layers of 8 to 4096 columns."""
    path = rng.choice(["short", "short", "short_step", "scan", "scan", "scan", "scan_step", "linear", "linear", "linear"])
    io = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if path == "linear":
        c = dict(path=path, B=_log_int(rng, 1, 64), K=_log_int(rng, 8, 4096), M=_log_int(rng, 8, 4096))
        if rng.random() < 0.6:
            c["K"], c["M"] = max(8, c["K"] // 8 * 8), max(8, c["M"] // 8 * 8)
        c["N"] = _log_int(rng, 1, max(1, min(16384, (1 << (33 if io == "fp32" else 35)) // (c["B"] * c["K"] * c["M"]))))
        c.update(act=rng.choice(["none", "silu", "gelu", "relu"]), bias=rng.random() < 0.7, residual=rng.random() < 0.4,
                 x=rng.choice(["last", "first"]), y=rng.choice(["last", "first"]), io=io, train=rng.random() < 0.6)
        if c["train"] and c["act"] == "relu":  # its slope jumps: 32 bits do not say on which side an entry is
            c["act"] = "silu"
        return c
    c = dict(path=path, B=_log_int(rng, 1, 64), H=_log_int(rng, 1, 1024))
    if path in ("short", "short_step"):
        c.update(taps=rng.randint(1, 8), act=rng.choice(["silu", "silu", "none"]), bias=rng.random() < 0.7, io=io)
        if path == "short":
            c["N"] = _log_int(rng, 1, min(16384, (1 << 25) // (c["B"] * c["H"])))
    else:
        c.update(S=rng.choice([1, 4, 8, 16, 16, 16, _log_int(rng, 1, 64)]), gated=rng.random() < 0.5, softplus=rng.random() < 0.8, io=io)
        c["G"] = rng.choice([g for g in (1, 1, 2, 4) if c["H"] % g == 0])
        if path == "scan":
            c["N"] = _log_int(rng, 1, max(1, min(16384, (1 << 28) // (c["B"] * c["H"] * c["S"]))))
    if path in ("short", "scan"):
        c.update(train=rng.random() < 0.6, carry=rng.random() < 0.4, ragged=rng.random() < 0.4)
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device="cuda")  # noqa: E731
    io, B, train = _DT[c["io"]], c["B"], c.get("train")
    new = lambda *s: torch.empty(*s, dtype=io, device="cuda")  # noqa: E731
    new32 = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    s = dict(case=c)
    if c.get("ragged"):
        s["lengths"] = ((0.2 + 0.8 * rand(B)) * c["N"]).ceil().long()
    if c["path"] == "linear":
        N, K, M = c["N"], c["K"], c["M"]
        s["x"] = randn(*((B, N, K) if c["x"] == "last" else (B, K, N))).to(io)
        s["W"] = (randn(M, K) / math.sqrt(K)).to(io)
        s["bias"] = 0.1 * randn(M) if c["bias"] else None
        of_y = (B, N, M) if c["y"] == "last" else (B, M, N)
        s["residual"] = randn(*of_y).to(io) if c["residual"] else None
        s["y"] = new(*of_y)
        if train:
            s["dy"], s["dx"] = randn(*of_y).to(io), torch.empty_like(s["x"])
            # behind an activation the gradient of W has W's type, otherwise 32 bits
            s["dW"] = new(M, K) if c["act"] != "none" else new32(M, K)
            s["dbias"] = new32(M) if c["bias"] else None
    elif c["path"] in ("short", "short_step"):
        H, taps = c["H"], c["taps"]
        s["k"] = randn(H, taps) / math.sqrt(taps)
        s["bias"] = 0.1 * randn(H) if c["bias"] else None
        shape = (B, H, c["N"]) if c["path"] == "short" else (B, H)
        s["x"], s["y"] = randn(*shape).to(io), new(*shape)
        if c["path"] == "short_step" or c["carry"]:
            s["state"] = randn(B, H, taps - 1).to(io)
        if c["path"] == "short":
            s["last"] = new(B, H, taps - 1)
        if train:
            s["dy"], s["dx"], s["dk"] = randn(*shape).to(io), new(*shape), new32(H, taps)
            s["dbias"] = new32(H) if c["bias"] else None
            if c["carry"]:
                s["dlast"], s["dstate"] = randn(B, H, taps - 1).to(io), new(B, H, taps - 1)
    else:
        H, S, G = c["H"], c["S"], c["G"]
        dt = torch.exp(math.log(1e-3) + (math.log(1e-1) - math.log(1e-3)) * rand(H))  # time steps of 0.001 to 0.1
        s["A"] = -(1.0 + torch.arange(S, device="cuda")) * (0.8 + 0.4 * rand(H, S))
        s["D"] = 1 + 0.1 * randn(H)
        shape = (B, H, c["N"]) if c["path"] == "scan" else (B, H)
        each = dt.view(H, 1) if c["path"] == "scan" else dt
        if c["softplus"]:
            s["bias"] = torch.log(torch.expm1(dt))
            s["delta"] = (0.5 * randn(*shape)).to(io)
        else:
            s["bias"] = None
            s["delta"] = (each * torch.exp(0.5 * randn(*shape))).to(io)
        s["u"], s["y"] = randn(*shape).to(io), new(*shape)
        s["z"] = randn(*shape).to(io) if c["gated"] else None
        of_b = (B, G, S, c["N"]) if c["path"] == "scan" else (B, G, S)
        s["Bm"], s["Cm"] = randn(*of_b).to(io), randn(*of_b).to(io)
        if c["path"] == "scan_step" or c["carry"]:
            s["state"] = 0.3 * randn(B, H, S)
        if c["path"] == "scan":
            s["last"] = new32(B, H, S)
        if train:
            s["dy"], s["du"], s["ddelta"] = randn(*shape).to(io), new(*shape), new(*shape)
            s["dz"] = new(*shape) if c["gated"] else None
            s["dA"], s["dD"] = new32(H, S), new32(H)
            s["dbias"] = new32(H) if c["softplus"] else None
            s["dB"], s["dC"] = new(*of_b), new(*of_b)
            if c["carry"]:
                s["dlast"], s["dstate"] = randn(B, H, S), new32(B, H, S)
    if own:  # the scratch memory that a program keeps for the library's calls
        import paper_2302_06646_amd as lc
        code = lc.dtype_code(s["y"])
        if c["path"] == "linear":
            s["ws"] = lc.new_workspace_linear(B, c["N"], c["K"], c["M"], code, train)
        elif c["path"] == "short" and train:
            s["ws"] = lc.new_workspace_short(B, c["H"], c["N"], c["taps"], code)
        elif c["path"] == "scan":
            s["ws"] = lc.new_workspace_scan(B, c["H"], c["N"], c["S"], c["G"], code, train)
            s["marks"] = lc.new_scan_marks(B, c["H"], c["N"], c["S"]) if train else None
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------


def run(s):
    return (_own if own else _plain)[s["case"]["path"]](s)


def _given(s, *names):
    return {n: s[n] for n in names if s.get(n) is not None}


def _own_short(s):
    import paper_2302_06646_amd as lc
    c, some = s["case"], _given(s, "state", "lengths")
    lc.longconv_short_fwd(s["x"], s["k"], s["bias"], s["y"], c["act"], last=s["last"], **some)
    if not c["train"]:
        return _given(s, "y", "last")
    lc.longconv_short_bwd(s["dy"], s["x"], s["k"], s["bias"], s["dx"], s["dk"], s["dbias"], c["act"], s["ws"], **some,
                          **_given(s, "dlast", "dstate"))
    return _given(s, "y", "last", "dx", "dk", "dbias", "dstate")


def _own_short_step(s):
    import paper_2302_06646_amd as lc
    lc.longconv_short_step(s["x"], s["k"], s["bias"], s["state"], s["y"], s["case"]["act"])
    return _given(s, "y", "state")


def _own_scan(s):
    import paper_2302_06646_amd as lc
    c, some = s["case"], _given(s, "D", "z", "bias", "lengths")
    lc.longconv_scan_fwd(s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["y"], s["ws"], softplus=c["softplus"], last=s["last"], **some,
                         **_given(s, "state", "marks"))
    if not c["train"]:
        return _given(s, "y", "last")
    lc.longconv_scan_bwd(s["dy"], s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["marks"], s["du"], s["ddelta"], s["dA"], s["dB"], s["dC"],
                         s["ws"], softplus=c["softplus"], **some, **_given(s, "dD", "dz", "dbias", "dlast", "dstate"))
    return _given(s, "y", "last", "du", "ddelta", "dA", "dB", "dC", "dD", "dz", "dbias", "dstate")


def _own_scan_step(s):
    import paper_2302_06646_amd as lc
    lc.longconv_scan_step(s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["state"], s["y"], softplus=s["case"]["softplus"],
                          **_given(s, "D", "z", "bias"))
    return _given(s, "y", "state")


def _own_linear(s):
    import paper_2302_06646_amd as lc
    c = s["case"]
    layout = {"last": lc.CHANNELS_LAST, "first": lc.CHANNELS_FIRST}
    lc.longconv_linear_fwd(s["x"], s["W"], s["bias"], s["y"], c["act"], s["ws"], layout[c["x"]], layout[c["y"]], s["residual"])
    if not c["train"]:
        return _given(s, "y")
    lc.longconv_linear_bwd(s["dy"], s["x"], s["W"], s["bias"], s["dx"], s["dW"], s["dbias"], c["act"], s["ws"], layout[c["x"]],
                           layout[c["y"]])
    return _given(s, "y", "dx", "dW", "dbias")


def _act(z, act):
    """act(z) and its derivative."""
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return z * q, q * (1 + z * (1 - q))
    if act == "gelu":
        q = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * q, q + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    return z, torch.ones_like(z)


def _there(s):
    """Which places belong to their sequence, [B,1,N], or None if all do."""
    return None if s.get("lengths") is None else (torch.arange(s["case"]["N"], device="cuda") < s["lengths"][:, None])[:, None]


def _plain_short(s):
    c, k, io = s["case"], s["k"], s["x"].dtype
    B, H, N, W = c["B"], c["H"], c["N"], c["taps"]
    there = _there(s)
    x = s["x"].float() if there is None else s["x"].float() * there
    x = torch.cat([s["state"].float() if "state" in s else x.new_zeros(B, H, W - 1), x], 2)
    z = sum(k[:, j, None] * x[:, :, W - 1 - j:W - 1 - j + N] for j in range(W))
    if s["bias"] is not None:
        z = z + s["bias"][:, None]
    y, slope = _act(z, c["act"])
    y = y if there is None else y * there
    ends = torch.full((B,), N, device="cuda") if there is None else s["lengths"]
    at = (ends[:, None, None] + torch.arange(W - 1, device="cuda")).expand(B, H, W - 1)
    out = {"y": y.to(io), "last": x.gather(2, at).to(io)}
    if c["train"]:
        dz = s["dy"].float() * slope
        dz = dz if there is None else dz * there
        dx = x.new_zeros(B, H, N + W - 1)
        for j in range(W):
            dx[:, :, W - 1 - j:W - 1 - j + N] += k[:, j, None] * dz
        if "dlast" in s:
            dx.scatter_add_(2, at, s["dlast"].float())
        out["dk"] = torch.stack([(dz * x[:, :, W - 1 - j:W - 1 - j + N]).sum((0, 2)) for j in range(W)], 1)
        out["dx"] = dx[:, :, W - 1:].to(io)
        if s["bias"] is not None:
            out["dbias"] = dz.sum((0, 2))
        if "dstate" in s:
            out["dstate"] = dx[:, :, :W - 1].to(io)
    return out


def _plain_short_step(s):
    c = s["case"]
    x = torch.cat([s["state"].float(), s["x"].float()[..., None]], 2)
    z = (x * s["k"].flip(1)).sum(2)
    if s["bias"] is not None:
        z = z + s["bias"]
    s["state"].copy_(x[..., 1:])
    return {"y": _act(z, c["act"])[0].to(s["x"].dtype), "state": s["state"]}


def _recurrence(a, x):
    """h_t = a_t h_{t-1} + x_t along the last axis, by doubling; both arguments are written over."""
    d = 1
    while d < x.shape[-1]:
        x[..., d:] += a[..., d:] * x[..., :-d]
        a[..., d:] *= a[..., :-d].clone()
        d *= 2
    return x


def _plain_scan(s):
    c, io = s["case"], s["u"].dtype
    B, H, N, S, G = (c[k] for k in "BHNSG")
    there = _there(s)
    u, w, A = s["u"].float(), s["delta"].float(), s["A"][:, :, None]
    if s["bias"] is not None:
        w = w + s["bias"][:, None]
    dt = w.clamp(min=0) + torch.log1p(torch.exp(-w.abs())) if c["softplus"] else w
    if there is not None:
        dt, u = dt * there, u * there
    per_head = lambda t: t.float().view(B, G, 1, S, N).expand(B, G, H // G, S, N).reshape(B, H, S, N)  # noqa: E731
    a = torch.exp(dt[:, :, None] * A)
    Bm, Cm = per_head(s["Bm"]), per_head(s["Cm"])
    x = (dt * u)[:, :, None] * Bm
    if "state" in s:
        x[..., 0] += a[..., 0] * s["state"]
    h = _recurrence(a.clone(), x)
    y = (Cm * h).sum(2) + s["D"][:, None] * u
    gate, slope = _act(s["z"].float(), "silu") if c["gated"] else (None, None)
    out = {"y": (y if gate is None else y * gate), "last": h[..., -1].clone()}
    if there is not None:
        out["y"] = out["y"] * there
    out["y"] = out["y"].to(io)
    if c["train"]:
        dy = s["dy"].float() if there is None else s["dy"].float() * there
        if gate is not None:
            out["dz"] = (dy * y * slope).to(io)
            dy = dy * gate
        g = dy[:, :, None] * Cm
        if "dlast" in s:
            g[..., -1] += s["dlast"]
        later = torch.cat([a[..., 1:], torch.ones_like(a[..., :1])], 3)
        g = _recurrence(later.flip(3), g.flip(3)).flip(3)
        before = torch.cat([s["state"][..., None] if "state" in s else torch.zeros_like(h[..., :1]), h[..., :-1]], 3)
        kept = g * a * before
        if "dstate" in s:
            out["dstate"] = g[..., 0] * a[..., 0]
        out["dA"] = (kept * dt[:, :, None]).sum((0, 3))
        gb = (g * Bm).sum(2)
        ddt = (kept * A).sum(2) + gb * u
        out["du"] = (gb * dt + dy * s["D"][:, None]).to(io)
        out["dD"] = (dy * u).sum((0, 2))
        dw = ddt / (1 + torch.exp(-w)) if c["softplus"] else ddt
        dw = dw if there is None else dw * there
        out["ddelta"] = dw.to(io)
        if s["bias"] is not None:
            out["dbias"] = dw.sum((0, 2))
        out["dB"] = (g * (dt * u)[:, :, None]).view(B, G, H // G, S, N).sum(2).to(io)
        out["dC"] = (h * dy[:, :, None]).view(B, G, H // G, S, N).sum(2).to(io)
    return out


def _plain_scan_step(s):
    c, io = s["case"], s["u"].dtype
    B, H, S, G = (c[k] for k in "BHSG")
    u, w = s["u"].float(), s["delta"].float()
    if s["bias"] is not None:
        w = w + s["bias"]
    dt = w.clamp(min=0) + torch.log1p(torch.exp(-w.abs())) if c["softplus"] else w
    per_head = lambda t: t.float().view(B, G, 1, S).expand(B, G, H // G, S).reshape(B, H, S)  # noqa: E731
    s["state"].copy_(torch.exp(dt[..., None] * s["A"]) * s["state"] + (dt * u)[..., None] * per_head(s["Bm"]))
    y = (s["state"] * per_head(s["Cm"])).sum(2) + s["D"] * u
    if c["gated"]:
        y = y * _act(s["z"].float(), "silu")[0]
    return {"y": y.to(io), "state": s["state"]}


def _plain_linear(s):
    c, io = s["case"], s["x"].dtype
    W = s["W"].float()
    last = lambda t, layout: (t if layout == "last" else t.transpose(1, 2)).float().contiguous()  # noqa: E731
    back = lambda t, layout: t if layout == "last" else t.transpose(1, 2).contiguous()  # noqa: E731
    x = last(s["x"], c["x"])
    z = x @ W.t()
    if s["bias"] is not None:
        z = z + s["bias"]
    y, slope = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + last(s["residual"], c["y"])
    out = {"y": back(y.to(io), c["y"])}
    if c["train"]:
        dz = last(s["dy"], c["y"]) * slope
        out["dx"] = back((dz @ W).to(io), c["x"])
        flat = dz.view(-1, c["M"])
        out["dW"] = (flat.t() @ x.view(-1, c["K"])).to(s["dW"].dtype)
        if s["bias"] is not None:
            out["dbias"] = flat.sum(0)
    return out


_own = dict(short=_own_short, short_step=_own_short_step, scan=_own_scan, scan_step=_own_scan_step, linear=_own_linear)
_plain = dict(short=_plain_short, short_step=_plain_short_step, scan=_plain_scan, scan_step=_plain_scan_step, linear=_plain_linear)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------


def work(case):
    c = case
    e, B = _SIZE[c["io"]], c["B"]
    if c["path"] == "linear":
        T, K, M = B * c["N"], c["K"], c["M"]
        if c["train"]:
            dw = e if c["act"] != "none" else 4
            return {"bytes": (2 * T * K + (2 + c["residual"]) * T * M + M * K) * e + M * K * dw + 8 * M, "flops": 6 * T * K * M}
        return {"bytes": (T * K + (1 + c["residual"]) * T * M + M * K) * e + 4 * M, "flops": 2 * T * K * M}
    share = 0.6 if c.get("ragged") else 1.0  # of the places that belong to a sequence
    if c["path"] in ("short", "short_step"):
        n, H, W = B * c["H"], c["H"], c["taps"]
        ends = n * (W - 1) * e
        if c["path"] == "short_step":
            return {"bytes": 2 * n * e + 2 * ends + 4 * H * (W + 1), "flops": n * (2 * W + 8)}
        n *= c["N"]
        if c["train"]:
            return {"bytes": (2 * share + 2) * n * e + ends * (1 + 3 * c["carry"]) + 8 * H * (W + 1), "flops": share * n * (8 * W + 24)}
        return {"bytes": (share + 1) * n * e + ends * (1 + c["carry"]) + 4 * H * (W + 1), "flops": share * n * (2 * W + 8)}
    n, H, S, G = B * c["H"], c["H"], c["S"], c["G"]
    rows, states, small = 3 + c["gated"], 4 * n * S, 4 * (H * S + 2 * H)
    if c["path"] == "scan_step":
        return {"bytes": rows * n * e + 2 * B * G * S * e + 2 * states + small, "flops": n * (7 * S + 30)}
    n *= c["N"]
    of_b = 2 * B * G * S * c["N"] * e
    if c["train"]:
        read = 3 + c["gated"]  # u, delta, dy, z; written: y, du, ddelta, dz
        return {"bytes": (share * read + read) * n * e + (share + 1) * of_b + states * (1 + 3 * c["carry"]) + 2 * small,
                "flops": share * n * (25 * S + 60)}
    return {"bytes": (share * (rows - 1) + 1) * n * e + share * of_b + states * (1 + c["carry"]) + small, "flops": share * n * (7 * S + 30)}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------


def _slopes(z, act):
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * torch.sigmoid(-z)
    if act == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
    if act == "relu":
        return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
    return z, torch.ones_like(z)


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    return {"short": _exact_short, "short_step": _exact_short, "scan": _exact_scan, "scan_step": _exact_scan,
            "linear": _exact_linear}[c["path"]](c, f, s.get("lengths"))


def _exact_short(c, f, lengths):
    B, H, W = c["B"], c["H"], c["taps"]
    step = c["path"] == "short_step"
    x = f["x"][..., None] if step else f["x"]
    N = x.shape[2]
    ends = torch.full((B,), N, device="cuda") if lengths is None else lengths
    inside = torch.arange(N, device="cuda")[None, None] < ends[:, None, None]
    x = torch.where(inside, x, 0.0)
    if "state" not in f:
        f["state"] = torch.zeros(B, H, W - 1, dtype=torch.float64, device="cuda")
    whole = torch.cat([f["state"], x], 2)
    z = torch.nn.functional.conv1d(whole, f["k"].flip(1)[:, None], f.get("bias"), groups=H)
    y, slope = _slopes(z, c["act"])
    last = torch.stack([whole[b, :, e:e + W - 1] for b, e in enumerate(ends.tolist())])
    if step:
        return {"y": y[..., 0], "state": last}
    out = {"y": torch.where(inside, y, 0.0), "last": last}
    if c["train"]:
        dz = torch.where(inside, f["dy"] * slope, 0.0)
        dwhole = torch.nn.functional.conv_transpose1d(dz, f["k"].flip(1)[:, None], groups=H)
        if "dlast" in f:
            for b, e in enumerate(ends.tolist()):
                dwhole[b, :, e:e + W - 1] += f["dlast"][b]
        windows = whole.unfold(2, W, 1)  # [B,H,N,W], oldest first
        out["dk"] = torch.stack([(windows[..., W - 1 - j] * dz).sum(2).sum(0) for j in range(W)], 1)
        out["dx"] = dwhole[:, :, W - 1:]
        if "bias" in f:
            out["dbias"] = dz.sum(2).sum(0)
        if "dlast" in f:
            out["dstate"] = dwhole[:, :, :W - 1]
    return out


def _exact_scan(c, f, lengths):
    """Place by place, forwards and then backwards."""
    B, H, S, G = (c[k] for k in "BHSG")
    step = c["path"] == "scan_step"
    line = lambda t: t[..., None] if step else t  # noqa: E731
    u, w, Bm, Cm = line(f["u"]), line(f["delta"]), line(f["Bm"]), line(f["Cm"])
    N = u.shape[2]
    if "bias" in f:
        w = w + f["bias"][None, :, None]
    dt = torch.logaddexp(w, torch.zeros_like(w)) if c["softplus"] else w
    ends = torch.full((B,), N, device="cuda") if lengths is None else lengths
    inside = torch.arange(N, device="cuda")[None, None] < ends[:, None, None]
    dt = torch.where(inside, dt, 0.0)
    # places first, so that each is one piece of memory
    u, dt, Bm, Cm = u.permute(2, 0, 1).contiguous(), dt.permute(2, 0, 1).contiguous(), Bm.permute(3, 0, 1, 2).contiguous(), Cm.permute(3, 0, 1, 2).contiguous()
    wide = lambda t: t.repeat_interleave(H // G, 1)  # noqa: E731  [B,G,S] -> [B,H,S]
    h = f["state"] if "state" in f else torch.zeros(B, H, S, dtype=torch.float64, device="cuda")
    train = c.get("train")
    seen = torch.empty(N + 1, B, H, S, dtype=torch.float64, device="cuda") if train else None
    if train:
        seen[0] = h
    plain = torch.empty(N, B, H, dtype=torch.float64, device="cuda")
    for t in range(N):
        h = torch.exp(dt[t][..., None] * f["A"]) * h + (dt[t] * u[t])[..., None] * wide(Bm[t])
        plain[t] = (h * wide(Cm[t])).sum(2)
        if train:
            seen[t + 1] = h
    plain = plain + f["D"] * u
    z = line(f["z"]).permute(2, 0, 1) if "z" in f else None
    gate, slope = _slopes(z, "silu") if z is not None else (1.0, None)
    back = lambda t: t.permute(1, 2, 0)  # noqa: E731
    y = torch.where(inside, back(plain * gate), 0.0)
    if step:
        return {"y": y[..., 0], "state": h}
    out = {"y": y, "last": h}
    if train:
        dy = torch.where(inside, f["dy"], 0.0).permute(2, 0, 1)
        if z is not None:
            out["dz"] = back(dy * plain * slope)
            dy = dy * gate
        g = f["dlast"] if "dlast" in f else torch.zeros(B, H, S, dtype=torch.float64, device="cuda")
        dA, du, ddt = torch.zeros_like(f["A"]), torch.empty_like(plain), torch.empty_like(plain)
        dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
        for t in range(N - 1, -1, -1):
            g = g + dy[t][..., None] * wide(Cm[t])
            decay = torch.exp(dt[t][..., None] * f["A"])
            dC[t] = (dy[t][..., None] * seen[t + 1]).view(B, G, H // G, S).sum(2)
            dB[t] = (g * (dt[t] * u[t])[..., None]).view(B, G, H // G, S).sum(2)
            through = (g * wide(Bm[t])).sum(2)
            g = g * decay  # the gradient of the state before
            kept = g * seen[t]
            dA += (kept * dt[t][..., None]).sum(0)
            ddt[t] = (kept * f["A"]).sum(2) + through * u[t]
            du[t] = through * dt[t] + dy[t] * f["D"]
        dw = torch.where(inside, back(ddt), 0.0)
        dw = dw * torch.sigmoid(w) if c["softplus"] else dw
        out.update(du=torch.where(inside, back(du), 0.0), ddelta=dw, dA=dA, dB=dB.permute(1, 2, 3, 0), dC=dC.permute(1, 2, 3, 0),
                   dD=(dy * u).sum((0, 1)))
        if "bias" in f:
            out["dbias"] = dw.sum(2).sum(0)
        if "dlast" in f:
            out["dstate"] = g
    return out


def _exact_linear(c, f, lengths):
    first = lambda t: t.permute(0, 2, 1)  # noqa: E731
    x = f["x"] if c["x"] == "last" else first(f["x"])
    x = x.reshape(-1, c["K"])
    shape = (c["B"], c["N"], c["M"])
    z = torch.mm(x, f["W"].t())
    if "bias" in f:
        z += f["bias"][None]
    y, slope = _slopes(z, c["act"])
    y = y.view(shape) if c["y"] == "last" else first(y.view(shape))
    out = {"y": y + f["residual"] if "residual" in f else y}
    if c["train"]:
        dy = f["dy"] if c["y"] == "last" else first(f["dy"])
        dz = dy.reshape(-1, c["M"]) * slope
        dx = torch.mm(dz, f["W"]).view(c["B"], c["N"], c["K"])
        out["dx"] = dx if c["x"] == "last" else first(dx)
        out["dW"] = torch.mm(dz.t(), x)
        if "bias" in f:
            out["dbias"] = torch.ones(1, dz.shape[0], dtype=torch.float64, device="cuda").mm(dz)[0]
    return out
