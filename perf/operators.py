"""Operators around the long convolution, as cases to be timed and compared: embedding lookup and its gradient, dropout whose
mask is never stored, group norm with an activation.

A case names one of five paths:

  embed       tokens -> rows of a table, scaled, dropped out: [B,N,H] (layout "last") or the convolution's [B,H,N] ("first")
  embed_grad  the gradient of the table for a gradient of those rows
  dropout     forward (with the residual sum where asked for) and backward of one training step
  kreg        dropout, smoothing and squashing of a convolution kernel, and the chain rule back
  gnorm       group norm and activation of [B,S,C], alone (train False) or with its backward

`run` computes them in their plain form, elementary operations in 32 bits, or, where `own` is true, by the library's calls.

Random numbers: entry e of a tensor in memory order is dropped if its 16 random bits are below T = round(65536 p), and multiplied
by 65536 / (65536 - T) otherwise.  The bits are half e mod 8 (the low half of a word first) of the four words that Philox4x32 with
seven rounds makes of the counter (e div 8, number of the call) and the key `seed`.
"""
import math

import numpy as np
import torch

own = False

_DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
_EPS = 1e-5
_SQUASH = 0.003


def listed():
    return [
        # one token of each of four sequences that are being decoded: nothing but latency
        dict(name="embed_token_bf16", path="embed", B=4, N=1, V=32768, H=768, table="bf16", io="bf16", ids="i64", layout="last",
             drop=0.0, text="zipf"),
        # language-model batch: master table in fp32, scaled by sqrt(H), embedding dropout
        dict(name="embed_lm_bf16", path="embed", B=16, N=1024, V=32768, H=768, table="fp32", io="bf16", ids="i64", layout="last",
             drop=0.1, text="zipf"),
        # long-range task on bytes, of uneven lengths, straight into the convolution's layout
        dict(name="embed_bytes_fp16", path="embed", B=8, N=16384, V=256, H=256, table="fp32", io="fp16", ids="i64",
             layout="first", drop=0.0, text="padded"),
        # the gradients of the two
        dict(name="embed_grad_lm_bf16", path="embed_grad", B=16, N=1024, V=32768, H=768, table="fp32", io="bf16", ids="i64",
             layout="last", drop=0.1, text="zipf"),
        dict(name="embed_grad_bytes_fp16", path="embed_grad", B=8, N=16384, V=256, H=256, table="fp32", io="fp16", ids="i64",
             layout="first", drop=0.1, text="padded"),
        # odd counts everywhere, full precision
        dict(name="embed_grad_odd_fp32", path="embed_grad", B=7, N=385, V=1009, H=193, table="fp32", io="fp32", ids="i32",
             layout="last", drop=0.0, text="zipf"),
        # residual branch of the widest configuration, the largest tensors there are
        dict(name="dropout_wide_bf16", path="dropout", B=64, H=1024, N=4096, io="bf16", residual=True, tied=False, drop=0.1),
        # language-model block, one mask value for a whole sequence of a head
        dict(name="dropout_tied_bf16", path="dropout", B=16, H=768, N=1024, io="bf16", residual=True, tied=True, drop=0.2),
        # Algorithm 1 lines 1-3 of the same block
        dict(name="kreg_lm_fp32", path="kreg", H=768, N=1024, width=1, drop=0.2),
        # one small odd feature map, inference
        dict(name="gnorm_odd_fp32", path="gnorm", B=3, S=49, C=195, G=5, io="fp32", act="silu", train=False),
        # image layer on 32 x 32 images, training step
        dict(name="gnorm_image_bf16", path="gnorm", B=64, S=1024, C=256, G=32, io="bf16", act="silu", train=True),
        # image layer on 128 x 128 images, training step
        dict(name="gnorm_large_fp16", path="gnorm", B=16, S=16384, C=256, G=32, io="fp16", act="gelu", train=True),
    ]


def _log_int(rng, lo, hi):
    v = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return v + 1 if v == 3072 else v


def draw(rng):
    """A case of the same paths: 1 to 64 sequences, any length up to 16384, any vocabulary up to 65536, any width up to 1024."""
    path = rng.choice(["embed", "embed", "embed_grad", "embed_grad", "dropout", "dropout", "kreg", "gnorm", "gnorm", "gnorm"])
    io = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if path in ("embed", "embed_grad"):
        c = dict(path=path, B=_log_int(rng, 1, 64), V=_log_int(rng, 200, 65536), H=_log_int(rng, 16, 1024))
        if rng.random() < 0.6:
            c["H"] = max(16, c["H"] // 16 * 16)
        c["N"] = _log_int(rng, 1, min(16384, (1 << 27) // c["B"] // c["H"]))
        c.update(io=io, table=rng.choice(["fp32", io]), ids=rng.choice(["i64", "i64", "i32"]),
                 layout=rng.choice(["last", "last", "first"]), drop=rng.choice([0.0, 0.1, 0.25]),
                 text=rng.choice(["zipf", "zipf", "padded"]))
        return c
    if path == "dropout":
        c = dict(path=path, B=_log_int(rng, 1, 64), H=_log_int(rng, 1, 1024))
        c["N"] = _log_int(rng, 1, min(16384, (1 << 27) // c["B"] // c["H"]))
        c.update(io=io, residual=rng.random() < 0.5, tied=rng.random() < 0.3, drop=rng.choice([0.05, 0.1, 0.2, 0.5]))
        return c
    if path == "kreg":
        return dict(path=path, H=_log_int(rng, 4, 1024), N=1 << rng.randint(8, 14), width=rng.randint(0, 3),
                    drop=rng.choice([0.1, 0.2, 0.5]))
    G = rng.choice([1, 4, 8, 16, 32])
    c = dict(path=path, B=_log_int(rng, 1, 64), C=G * _log_int(rng, 1, max(1, 1024 // G)), G=G)
    least = -(-16 * G // c["C"])  # a group of very few entries has a gradient of x that cancels to nothing
    c["S"] = _log_int(rng, max(1, least), max(least, min(16384, (1 << 26) // c["B"] // c["C"])))
    c.update(io=io, act=rng.choice(["silu", "silu", "gelu", "relu", "none"]), train=rng.random() < 0.6)
    if io == "fp32" and c["train"] and c["act"] == "relu":  # its slope jumps: 32 bits do not say on which side an entry is
        c["act"] = "silu"
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------------------


def _shares(V):
    """How often each of V tokens comes up: the long-tailed law of text."""
    p = 1.0 / (np.arange(V) + 2.7)
    return p / p.sum()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device="cuda")  # noqa: E731
    io = _DT[c.get("io", "fp32")]
    s = dict(case=c, seed=seed * 0x9E3779B1 % (1 << 63), call=seed % 1000)
    if c["path"] in ("embed", "embed_grad"):
        B, N, V, H = c["B"], c["N"], c["V"], c["H"]
        cdf = torch.from_numpy(np.cumsum(_shares(V))).float().cuda()
        order = torch.randperm(V, generator=gen, device="cuda")
        ids = order[torch.searchsorted(cdf, rand(B, N)).clamp_(max=V - 1)]
        if c["text"] == "padded":  # sequences of uneven lengths; -1 is no token
            ids = torch.where(torch.arange(N, device="cuda") < (0.2 + 0.8 * rand(B, 1)) * N, ids, -1)
        s["ids"] = ids.to(torch.int64 if c["ids"] == "i64" else torch.int32).contiguous()
        s["scale"] = math.sqrt(H)
        shape = (B, N, H) if c["layout"] == "last" else (B, H, N)
        if c["path"] == "embed":
            s["E"] = (0.02 * randn(V, H)).to(_DT[c["table"]])
            s["y"] = torch.empty(shape, dtype=io, device="cuda")
        else:
            s["dy"] = randn(*shape).to(io)
            s["dE"] = torch.empty(V, H, device="cuda")
    elif c["path"] == "dropout":
        shape = (c["B"], c["H"], c["N"])
        s["x"], s["dy"] = randn(*shape).to(io), randn(*shape).to(io)
        s["r"] = randn(*shape).to(io) if c["residual"] else None
        s["y"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["tie"] = c["N"] if c["tied"] else 1
    elif c["path"] == "kreg":
        s["k"], s["dkbar"] = 0.02 * randn(c["H"], c["N"]), randn(c["H"], c["N"])
        s["kbar"], s["dk"] = torch.empty_like(s["k"]), torch.empty_like(s["k"])
    else:
        B, S, C, G = c["B"], c["S"], c["C"], c["G"]
        s["x"] = (randn(B, S, C) * (0.5 + rand(C)) + randn(C)).to(io)
        s["gamma"], s["beta"] = 1 + 0.1 * randn(C), 0.1 * randn(C)
        s["y"] = torch.empty_like(s["x"])
        s["mean"], s["rstd"] = torch.empty(B, G, device="cuda"), torch.empty(B, G, device="cuda")
        if c["train"]:
            s["dy"] = randn(B, S, C).to(io)
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    if own:  # the scratch memory that a program keeps for the library's calls
        import paper_2302_06646_amd as lc
        if c["path"] == "embed_grad":
            s["ws"] = lc.new_workspace_embed(c["B"], c["N"], c["V"], c["H"], lc.dtype_code(s["dy"]),
                                             lc.CHANNELS_LAST if c["layout"] == "last" else lc.CHANNELS_FIRST)
        elif c["path"] == "gnorm":
            s["ws"] = lc.new_workspace_gnorm(c["B"], c["S"], c["C"], c["G"], lc.dtype_code(s["x"]), c["train"])
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------------


def run(s):
    return (_own if own else _plain)[s["case"]["path"]](s)


def _own_embed(s):
    import paper_2302_06646_amd as lc
    c = s["case"]
    lc.longconv_embed_fwd(s["ids"], s["E"], s["y"], s["scale"], lc.CHANNELS_LAST if c["layout"] == "last" else lc.CHANNELS_FIRST,
                          c["drop"], s["seed"], s["call"])
    return {"y": s["y"]}


def _own_embed_grad(s):
    import paper_2302_06646_amd as lc
    c = s["case"]
    lc.longconv_embed_bwd(s["dy"], s["ids"], s["dE"], s["scale"], lc.CHANNELS_LAST if c["layout"] == "last" else lc.CHANNELS_FIRST,
                          s["ws"], c["drop"], s["seed"], s["call"])
    return {"dE": s["dE"]}


def _own_dropout(s):
    import paper_2302_06646_amd as lc
    p = s["case"]["drop"]
    lc.longconv_dropout_fwd(s["x"], s["y"], p, s["seed"], s["call"], s["r"], s["tie"])
    lc.longconv_dropout_bwd(s["dy"], s["dx"], p, s["seed"], s["call"], s["tie"])
    return {"y": s["y"], "dx": s["dx"]}


def _own_kreg(s):
    import paper_2302_06646_amd as lc
    c = s["case"]
    lc.longconv_kreg_fwd_seeded(s["k"], s["kbar"], c["width"], _SQUASH, c["drop"], s["seed"], s["call"])
    lc.longconv_kreg_bwd_seeded(s["k"], s["dkbar"], s["dk"], c["width"], _SQUASH, c["drop"], s["seed"], s["call"])
    return {"kbar": s["kbar"], "dk": s["dk"]}


def _own_gnorm(s):
    import paper_2302_06646_amd as lc
    c = s["case"]
    lc.longconv_gnorm_fwd(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], _EPS, c["act"], s["ws"])
    if not c["train"]:
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    lc.longconv_gnorm_bwd(s["dy"], s["x"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], c["act"],
                          s["ws"])
    return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}


_LOW = 0xFFFFFFFF


def _factors(n, p, seed, call):
    """m of the entries 0 .. n - 1: 0 where dropped, else 65536 / (65536 - T)."""
    T = round(p * 65536)
    i = torch.arange((n + 7) // 8, device="cuda")
    c0, c1, c2, c3 = i & _LOW, i >> 32, call & _LOW, call >> 32
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(7):  # products of 32 bits each, kept modulo 2^64
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & _LOW) ^ c1 ^ k0, b & _LOW, (a >> 32 & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    halves = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 1)
    return (halves.view(-1)[:n] >= T) * torch.tensor(65536 / (65536 - T), dtype=torch.float32, device="cuda")


def _plain_embed(s):
    c, E, ids = s["case"], s["E"], s["ids"].long()
    y = E[ids.clamp(0, c["V"] - 1)].float() * s["scale"] * ((ids >= 0) & (ids < c["V"]))[..., None]
    if c["layout"] == "first":
        y = y.transpose(1, 2).contiguous()
    if c["drop"]:
        y = y * _factors(y.numel(), c["drop"], s["seed"], s["call"]).view(y.shape)
    return {"y": y.to(s["y"].dtype)}


def _plain_embed_grad(s):
    c, g, ids = s["case"], s["dy"].float(), s["ids"].long().view(-1)
    if c["drop"]:
        g = g * _factors(g.numel(), c["drop"], s["seed"], s["call"]).view(g.shape)
    if c["layout"] == "first":
        g = g.transpose(1, 2)
    valid = (ids >= 0) & (ids < c["V"])
    dE = torch.zeros(c["V"], c["H"], device="cuda")
    dE.index_add_(0, ids.clamp(0, c["V"] - 1), g.reshape(-1, c["H"]) * valid[:, None])
    return {"dE": dE * s["scale"]}


def _plain_dropout(s):
    x, dy, tie = s["x"], s["dy"], s["tie"]
    m = _factors(x.numel() // tie, s["case"]["drop"], s["seed"], s["call"])
    m = m.view(*x.shape[:2], 1) if tie > 1 else m.view(x.shape)
    y = x.float() * m
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(x.dtype), "dx": (dy.float() * m).to(x.dtype)}


def _windows(a, w):
    """Sums of 2 w + 1 neighbours, entries outside a row zero, from left to right."""
    N = a.shape[1]
    a = torch.nn.functional.pad(a, (w, w))
    t = a[:, :N]
    for d in range(1, 2 * w + 1):
        t = t + a[:, d:d + N]
    return t


def _plain_kreg(s):
    c, k = s["case"], s["k"]
    m = _factors(k.numel(), c["drop"], s["seed"], s["call"]).view(k.shape)
    inv = torch.tensor(1 / (2 * c["width"] + 1), dtype=torch.float32, device="cuda")
    lam = torch.tensor(_SQUASH, dtype=torch.float32, device="cuda")
    k2 = _windows(k * m, c["width"]) * inv
    kbar = k2.sign() * (k2.abs() - lam).clamp(min=0)
    dk = _windows(s["dkbar"] * (k2.abs() > lam), c["width"]) * inv * m
    return {"kbar": kbar, "dk": dk}


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


def _plain_gnorm(s):
    c = s["case"]
    B, S, C, G = c["B"], c["S"], c["C"], c["G"]
    x = s["x"].float().view(B, S, G, C // G)
    gamma, beta = s["gamma"].view(G, C // G), s["beta"].view(G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + _EPS)
    xhat = d * rstd
    y, slope = _act(xhat * gamma + beta, c["act"])
    out = {"y": y.view(B, S, C).to(s["x"].dtype), "mean": mean.view(B, G), "rstd": rstd.view(B, G)}
    if c["train"]:
        dz = s["dy"].float().view(B, S, G, C // G) * slope
        out["dgamma"], out["dbeta"] = (dz * xhat).sum((0, 1)).view(C), dz.sum((0, 1)).view(C)
        t = dz * gamma
        dx = rstd * (t - t.mean((1, 3), keepdim=True) - xhat * (t * xhat).mean((1, 3), keepdim=True))
        out["dx"] = dx.view(B, S, C).to(s["x"].dtype)
    return out


_own = dict(embed=_own_embed, embed_grad=_own_embed_grad, dropout=_own_dropout, kreg=_own_kreg, gnorm=_own_gnorm)
_plain = dict(embed=_plain_embed, embed_grad=_plain_embed_grad, dropout=_plain_dropout, kreg=_plain_kreg, gnorm=_plain_gnorm)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------


def work(case):
    c = case
    e = _SIZE[c.get("io", "fp32")]
    if c["path"] in ("embed", "embed_grad"):
        M, V, H = c["B"] * c["N"], c["V"], c["H"]
        ids = M * (8 if c["ids"] == "i64" else 4)
        if c["path"] == "embed_grad":
            return {"bytes": ids + M * H * e + V * H * 4, "flops": M * H}
        drawn = M * (0.6 if c["text"] == "padded" else 1.0)  # tokens that name a row, and how many rows they are expected to name
        rows = float((1 - np.exp(drawn * np.log1p(-_shares(V)))).sum())
        return {"bytes": ids + rows * H * _SIZE[c["table"]] + M * H * e, "flops": M * H}
    if c["path"] == "dropout":
        n = c["B"] * c["H"] * c["N"]
        return {"bytes": n * e * (5 if c["residual"] else 4), "flops": 3 * n}
    if c["path"] == "kreg":
        n = c["H"] * c["N"]
        return {"bytes": n * 4 * 5, "flops": n * (4 * c["width"] + 8)}
    n, small = c["B"] * c["S"] * c["C"], (2 * c["B"] * c["G"] + 2 * c["C"]) * 4
    if c["train"]:
        return {"bytes": n * e * 5 + 2 * small, "flops": 30 * n}
    return {"bytes": n * e * 2 + small, "flops": 10 * n}


# ---- the definition, in 64 bits --------------------------------------------------------------------------------------------


def _kept(e, T, seed, call):
    """Whether the entries numbered `e` are kept; products in halves of 16 bits, so that nothing passes 2^63."""
    def mul(c, f):
        lo, hi = c * (f & 0xFFFF), c * (f >> 16)
        low = lo + ((hi & 0xFFFF) << 16)
        return (hi >> 16) + (low >> 32), low & _LOW

    block, at = e // 8, e % 8
    x, key = [block % (1 << 32), block // (1 << 32), torch.full_like(e, call % (1 << 32)), torch.full_like(e, call // (1 << 32))], seed
    for _ in range(7):
        (h0, l0), (h1, l1) = mul(x[0], 0xD2511F53), mul(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ (key % (1 << 32)), l1, h0 ^ x[3] ^ (key // (1 << 32)), l0]
        key = (key + 0x9E3779B9) % (1 << 32) + (key // (1 << 32) + 0xBB67AE85) % (1 << 32) * (1 << 32)
    word = torch.where(at < 2, x[0], torch.where(at < 4, x[1], torch.where(at < 6, x[2], x[3])))
    return torch.where(at % 2 == 0, word % 65536, word // 65536) >= T


def _exact_factors(n, c, s):
    T = math.floor(c["drop"] * 65536 + 0.5)
    kept = torch.cat([_kept(torch.arange(a, min(n, a + (1 << 24)), device="cuda"), T, s["seed"], s["call"])
                      for a in range(0, n, 1 << 24)])
    return kept.double() * (65536.0 / (65536 - T))


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    if c["path"] in ("embed", "embed_grad"):
        B, N, V, H = c["B"], c["N"], c["V"], c["H"]
        first = c["layout"] == "first"
        ids = s["ids"].to(torch.int64)
        named = torch.where((ids < 0) | (ids >= V), V, ids)  # row V: no token
        m = _exact_factors(B * N * H, c, s).view((B, H, N) if first else (B, N, H))
        if c["path"] == "embed":
            table = torch.cat([s["E"].double(), torch.zeros(1, H, dtype=torch.float64, device="cuda")])
            y = torch.index_select(table, 0, named.view(-1)).view(B, N, H) * s["scale"]
            return {"y": (y.permute(0, 2, 1) if first else y) * m}
        g = s["dy"].double() * m
        g = (g.permute(0, 2, 1) if first else g).reshape(B * N, H)
        order = torch.argsort(named.view(-1), stable=True)
        ends = torch.searchsorted(named.view(-1)[order], torch.arange(V, device="cuda"), right=True)
        sums = torch.cat([torch.zeros(1, H, dtype=torch.float64, device="cuda"), torch.cumsum(g[order], 0)])
        starts = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), ends[:-1]])
        return {"dE": (sums[ends] - sums[starts]) * s["scale"]}
    if c["path"] == "dropout":
        n = s["x"].numel()
        if c["tied"]:
            m = _exact_factors(c["B"] * c["H"], c, s).repeat_interleave(c["N"]).view(s["x"].shape)
        else:
            m = _exact_factors(n, c, s).view(s["x"].shape)
        y = m * s["x"].double()
        return {"y": y if s["r"] is None else y.add_(s["r"].double()), "dx": m * s["dy"].double()}
    if c["path"] == "kreg":
        H, N, w = c["H"], c["N"], c["width"]
        lam = float(np.float32(_SQUASH))
        m = _exact_factors(H * N, c, s).view(H, N)
        pool = lambda a: torch.nn.functional.conv1d(a[:, None], torch.full((1, 1, 2 * w + 1), 1.0 / (2 * w + 1), dtype=torch.float64),  # noqa: E731
                                                    padding=w)[:, 0]
        k2 = pool((s["k"].double() * m).cpu())
        dk = pool(torch.where(k2.abs() > lam, s["dkbar"].double().cpu(), 0.0)).cuda() * m
        return {"kbar": torch.where(k2 > lam, k2 - lam, torch.where(k2 < -lam, k2 + lam, 0.0)).cuda(), "dk": dk}
    B, S, C, G = c["B"], c["S"], c["C"], c["G"]
    each = lambda v: v.repeat_interleave(C // G, 1)[:, None, :]  # noqa: E731  [B,G] -> [B,1,C]
    of = lambda a: a.sum(1).view(B, G, C // G).sum(2) / (S * (C // G))  # noqa: E731  mean over a group
    x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
    mean = of(x)
    var = of((x - each(mean)) ** 2)
    rstd = (var + _EPS) ** -0.5
    xhat = (x - each(mean)) * each(rstd)
    z = gamma * xhat + beta
    if c["act"] == "silu":
        y, slope = z * torch.sigmoid(z), torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    elif c["act"] == "gelu":
        cdf = torch.special.ndtr(z)
        y, slope = z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
    elif c["act"] == "relu":
        y, slope = torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
    else:
        y, slope = z, torch.ones_like(z)
    out = {"y": y, "mean": mean, "rstd": rstd}
    if c["train"]:
        dz = s["dy"].double() * slope
        out["dgamma"], out["dbeta"] = (dz * xhat).sum((0, 1)), dz.sum((0, 1))
        out["dx"] = each(rstd) * (gamma * dz - each(of(gamma * dz)) - xhat * each(of(gamma * dz * xhat)))
    return out
