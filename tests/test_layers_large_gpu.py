"""Short convolution, selective scan and dense product on tensors of more than 2^32 elements, and of one workspace that two captured graphs share."""
import pytest
import torch

import paper_2302_06646_amd as lc

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _near(a, b):
    """Both are of the same fp32 sums, added in another order at most: half a step of bf16 each, and one more where that moves a rounding."""
    return ((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-3).all()


@pytest.fixture(autouse=True)
def _release():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("B,H,N", [(1, 65535, 65544), (2, 33000, 65541), (17200, 1000, 250)])      # by rows and by pieces, and rows of odd lengths
def test_short_convolution_past_2_32_elements(B, H, N):
    assert B * H * N > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.zeros(B, H, N, dtype=BF16, device="cuda")
    k, bias = torch.randn(H, 4, generator=g, device="cuda"), torch.randn(H, generator=g, device="cuda")
    x[-1, -3:].normal_(generator=g)
    x[0, :2].normal_(generator=g)
    y, state = torch.empty_like(x), torch.randn(B, H, 3, generator=g, device="cuda").to(BF16)
    lc.longconv_short_fwd(x, k, bias, y, "silu", state=state)
    dx, dk, dbias = torch.empty_like(x), torch.empty_like(k), torch.empty_like(bias)
    lc.longconv_short_bwd(x, x, k, bias, dx, dk, dbias, "silu", lc.new_workspace_short(B, H, N, 4, lc.BF16), state=state)
    for b, h in ((0, slice(0, 2)), (B - 1, slice(H - 3, H))):
        part = x[b:b + 1, h].clone()
        few, want, want_dx = k[h].clone(), torch.empty_like(part), torch.empty_like(part)
        some = state[b:b + 1, h].clone()
        lc.longconv_short_fwd(part, few, bias[h].clone(), want, "silu", state=some)
        lc.longconv_short_bwd(part, part, few, bias[h].clone(), want_dx, None, None, "silu", lc.new_workspace_short(1, part.shape[1], N, 4, lc.BF16),
                              state=some)
        assert torch.equal(y[b, h], want[0]) and torch.equal(dx[b, h], want_dx[0])
    # places of zeros have gradients of zero in dk, and in dbias as dy is zero: what is left is the last rows'
    if B == 1:
        part = x[:, -3:].clone()
        want_dk, want_db = torch.empty(3, 4, device="cuda"), torch.empty(3, device="cuda")
        lc.longconv_short_bwd(part, part, k[-3:].clone(), bias[-3:].clone(), None, want_dk, want_db, "silu",
                              lc.new_workspace_short(1, 3, N, 4, lc.BF16), state=state[:, -3:].clone())
        assert torch.allclose(dk[-3:], want_dk, rtol=1e-3, atol=1e-2) and torch.allclose(dbias[-3:], want_db, rtol=1e-3, atol=1e-2)


def test_scan_past_2_32_elements():
    B, H, N, S = 2, 33000, 65541, 1
    assert B * H * N > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.zeros(B, H, N, dtype=BF16, device="cuda")
    delta = torch.zeros_like(u)
    for t in (u, delta):
        t[-1, -3:].normal_(generator=g)
        t[0, :2].normal_(generator=g)
    A = -torch.rand(H, S, generator=g, device="cuda") - 0.1
    Bm, Cm = (torch.randn(B, 1, S, N, generator=g, device="cuda").to(BF16) for _ in range(2))
    y, marks, ws = torch.empty_like(u), lc.new_scan_marks(B, H, N, S), lc.new_workspace_scan(B, H, N, S, 1, lc.BF16, True)
    lc.longconv_scan_fwd(u, delta, A, Bm, Cm, y, ws, marks=marks)
    du, ddelta = torch.empty_like(u), torch.empty_like(u)
    lc.longconv_scan_bwd(u, u, delta, A, Bm, Cm, marks, du, ddelta, None, None, None, ws)
    for b, h in ((0, slice(0, 2)), (B - 1, slice(H - 3, H))):
        part, steps = u[b:b + 1, h].clone(), delta[b:b + 1, h].clone()
        heads = part.shape[1]
        want, some, few = torch.empty_like(part), lc.new_scan_marks(1, heads, N, S), lc.new_workspace_scan(1, heads, N, S, 1, lc.BF16, True)
        args = (part, steps, A[h].clone(), Bm[b:b + 1].clone(), Cm[b:b + 1].clone())
        lc.longconv_scan_fwd(*args, want, few, marks=some)
        want_du, want_dd = torch.empty_like(part), torch.empty_like(part)
        lc.longconv_scan_bwd(part, *args, some, want_du, want_dd, None, None, None, few)
        assert _near(y[b, h], want[0]) and _near(du[b, h], want_du[0]) and _near(ddelta[b, h], want_dd[0])


@pytest.mark.parametrize("first", [False, True])
def test_dense_product_past_2_32_elements(first):
    B, N, K, M = (2, 33000, 64, 65528) if first else (1, 66000, 64, 65528)
    layout = lc.CHANNELS_FIRST if first else lc.CHANNELS_LAST
    assert B * N * M > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(2)
    x, W, bias = torch.randn(B, N, K, generator=g, device="cuda").to(BF16), torch.randn(M, K, generator=g, device="cuda").to(BF16), torch.randn(M, device="cuda")
    y = torch.empty((B, M, N) if first else (B, N, M), dtype=BF16, device="cuda")
    ws = lc.new_workspace_linear(B, N, K, M, lc.BF16, True)
    lc.longconv_linear_fwd(x, W, bias, y, "none", ws, lc.CHANNELS_LAST, layout)
    rows = x[-1, -37:].float() @ W.float().t() + bias
    assert _near(y[-1, :, -37:].t() if first else y[-1, -37:], rows)
    y.zero_()                                              # now a gradient, of the last places
    dy = y[-1, :, -37:] if first else y[-1, -37:]
    dy.normal_(generator=g)
    dx, dW, dbias = torch.empty_like(x), torch.empty(M, K, device="cuda"), torch.empty(M, device="cuda")
    lc.longconv_linear_bwd(y, x, W, bias, dx, dW, dbias, "none", ws, lc.CHANNELS_LAST, layout)
    rows = (dy.t() if first else dy).float()
    want = rows @ W.float()
    assert ((dx[-1, -37:].float() - want).abs() <= 2.0 ** -8 * want.abs() + 0.05).all() and not dx[-1, :-37].any()      # sums of 65528 products of size one
    assert torch.allclose(dW, rows.t() @ x[-1, -37:].float(), rtol=1e-4, atol=1e-4) and torch.allclose(dbias, rows.sum(0), rtol=1e-4, atol=1e-4)


def test_one_workspace_of_two_captured_graphs():
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)  # noqa: E731
    B, H, N, S = 2, 40, 3000, 9                            # several segments
    sizes = (lc.longconv_scan_workspace_bytes(B, H, N, S, 1, lc.BF16, True), lc.longconv_short_workspace_bytes(B, H, N, 4, lc.BF16),
             lc.longconv_linear_workspace_bytes(B, N, H, H, lc.BF16, True))
    ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")
    A, k, W = -torch.rand(H, S, generator=g, device="cuda") - 0.1, torch.randn(H, 4, generator=g, device="cuda"), r(H, H)

    def work():
        x, delta, Bm, Cm, dy, u, y, out, du, dx = (r(B, *s) for s in ((H, N), (H, N), (1, S, N), (1, S, N), (H, N), (H, N), (H, N), (H, N), (H, N), (H, N)))
        marks, dk, dW = lc.new_scan_marks(B, H, N, S), torch.empty_like(k), torch.empty_like(W)
        dd, dA, dB, dC, dz = torch.empty_like(x), torch.empty_like(A), torch.empty_like(Bm), torch.empty_like(Cm), torch.empty_like(x)

        def run():
            lc.longconv_short_fwd(x, k, None, u, "silu")
            lc.longconv_scan_fwd(u, delta, A, Bm, Cm, y, ws, marks=marks)
            lc.longconv_linear_fwd(y, W, None, out, "gelu", ws, lc.CHANNELS_FIRST, lc.CHANNELS_FIRST)
            lc.longconv_linear_bwd(dy, y, W, None, dz, dW, None, "gelu", ws, lc.CHANNELS_FIRST, lc.CHANNELS_FIRST)
            lc.longconv_scan_bwd(dz, u, delta, A, Bm, Cm, marks, du, dd, dA, dB, dC, ws)
            lc.longconv_short_bwd(du, x, k, None, dx, dk, None, "silu", ws)

        return run, [out, dW, dd, dA, dB, dC, dx, dk]

    pairs, graphs = [work() for _ in range(2)], []
    want = []
    for run, kept in pairs:
        run()
        want.append([t.clone() for t in kept])
    torch.cuda.synchronize()
    for run, _ in pairs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        graphs.append(graph)
    for which in (0, 1, 1, 0, 0, 1):
        ws.fill_(0xFF)
        for t in pairs[which][1]:
            t.fill_(3.0)
        graphs[which].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[which], pairs[which][1]))


def test_scan_backward_where_B_and_C_have_2_31_elements():
    # two blocks of heads, whose sums dB and dC are joined; more states than a workgroup's waves hold
    B, H, N, S = 512, 33, 65536, 64
    assert B * N * S == 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(4)
    u, delta, dy = (torch.zeros(B, H, N, dtype=BF16, device="cuda") for _ in range(3))
    Bm, Cm = (torch.zeros(B, 1, S, N, dtype=BF16, device="cuda") for _ in range(2))
    for t in (u, delta, dy, Bm, Cm):
        t[0].normal_(generator=g)
        t[-1].normal_(generator=g)
    A = -torch.rand(H, S, generator=g, device="cuda") - 0.1
    new = lambda like: torch.full_like(like, 7.0)  # noqa: E731
    y, marks, ws = torch.empty_like(u), lc.new_scan_marks(B, H, N, S), lc.new_workspace_scan(B, H, N, S, 1, lc.BF16, True)
    lc.longconv_scan_fwd(u, delta, A, Bm, Cm, y, ws, marks=marks)
    du, ddelta, dA, dB, dC = (new(t) for t in (u, u, A, Bm, Cm))
    lc.longconv_scan_bwd(dy, u, delta, A, Bm, Cm, marks, du, ddelta, dA, dB, dC, ws)
    sums = torch.zeros_like(dA)
    for b in (0, B - 1):
        one = [t[b:b + 1].clone() for t in (dy, u, delta, Bm, Cm)]
        args = (one[1], one[2], A, one[3], one[4])
        some, few = lc.new_scan_marks(1, H, N, S), lc.new_workspace_scan(1, H, N, S, 1, lc.BF16, True)
        lc.longconv_scan_fwd(*args, torch.empty_like(one[1]), few, marks=some)
        want = [new(t) for t in (one[1], one[1], A, one[3], one[4])]
        lc.longconv_scan_bwd(one[0], *args, some, *want, few)
        assert all(_near(got[b], w[0]) for got, w in zip((du, ddelta, dB, dC), (want[0], want[1], want[3], want[4])))
        sums += want[2]
    assert torch.allclose(dA, sums, rtol=1e-4, atol=1e-3 * sums.abs().max().item())
    assert not any(t[b].any() for t in (dB, dC, du) for b in (1, B // 2, B - 2))      # all of their inputs are zero
