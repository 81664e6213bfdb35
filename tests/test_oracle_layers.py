"""The oracles of the short convolution, the selective scan and the dense product: closed forms, parts of sequences, differences."""
import numpy as np
import pytest

import oracle
from oracle import linear, scan, selective, short


def _differences(f, args, grads, names, eps=1e-6):
    for name in names:
        a = args[name]
        for i in np.ndindex(a.shape):
            up, down = ({k: (v.copy() if isinstance(v, np.ndarray) else v) for k, v in args.items()} for _ in range(2))
            up[name][i] += eps
            down[name][i] -= eps
            assert np.isclose((f(**up) - f(**down)) / (2 * eps), grads[name][i], rtol=2e-5, atol=1e-7), (name, i)


def test_short_convolution_is_the_long_one_with_few_taps():
    r = np.random.default_rng(0)
    x, k = r.standard_normal((2, 3, 16)), np.zeros((3, 16))
    k[:, :4] = r.standard_normal((3, 4))
    y, last = short.short_fwd(x, k[:, :4], np.zeros(3), "none")
    assert np.allclose(y, oracle.longconv_fwd(x, k, np.zeros(3)), atol=1e-12) and (last == x[:, :, -3:]).all()


@pytest.mark.parametrize("taps", [1, 3])
@pytest.mark.parametrize("name", ["none", "silu"])
def test_short_gradients_against_differences(taps, name):
    r = np.random.default_rng(1)
    B, H, N = 3, 2, 5
    lengths = np.array([5, 1, 0])
    args = dict(x=r.standard_normal((B, H, N)), k=r.standard_normal((H, taps)), bias=r.standard_normal(H),
                state=r.standard_normal((B, H, taps - 1)))
    dy, dlast = r.standard_normal((B, H, N)), r.standard_normal((B, H, taps - 1))

    def loss(x, k, bias, state):
        y, last = short.short_fwd(x, k, bias, name, state, lengths)
        return (y * dy).sum() + (last * dlast).sum()

    got = short.short_bwd(dy, args["x"], args["k"], args["bias"], name, args["state"], lengths, dlast)
    _differences(loss, args, dict(zip(("x", "k", "bias", "state"), got)), args)


def test_short_parts_make_the_whole():
    r = np.random.default_rng(2)
    x, k, bias = r.standard_normal((2, 3, 11)), r.standard_normal((3, 4)), r.standard_normal(3)
    y, last = short.short_fwd(x, k, bias, "gelu")
    a, mid = short.short_fwd(x[:, :, :2], k, bias, "gelu")
    b, end = short.short_fwd(x[:, :, 2:], k, bias, "gelu", mid)
    assert np.allclose(np.concatenate([a, b], 2), y) and np.allclose(end, last)


def test_scan_of_constant_coefficients_is_a_convolution():
    # dt, B, C fixed: y = k * u with k[j] = sum_s C exp(j dt A) dt B, and D
    r = np.random.default_rng(3)
    B, H, N, S = 2, 3, 16, 4
    u, A, D, dt = r.standard_normal((B, H, N)), -r.random((H, S)), r.standard_normal(H), 0.3
    b, c = r.standard_normal(S), r.standard_normal(S)
    wide = lambda v: np.broadcast_to(v[None, None, :, None], (B, 1, S, N)).copy()  # noqa: E731
    y, last, _ = scan.scan_fwd(u, np.full((B, H, N), dt), A, wide(b), wide(c), D, softplus=False)
    k = np.einsum("s,hsj,s->hj", c, np.exp(dt * A[:, :, None] * np.arange(N)), dt * b)
    assert np.allclose(y, oracle.longconv_fwd(u, k, D), atol=1e-12)
    assert np.allclose(last, np.einsum("hsj,s,bhj->bhs", np.exp(dt * A[:, :, None] * np.arange(N)[::-1]), dt * b, u))


@pytest.mark.parametrize("softplus", [False, True])
@pytest.mark.parametrize("G", [1, 2])
def test_scan_gradients_against_differences(softplus, G):
    r = np.random.default_rng(4)
    B, H, N, S = 3, 2, 4, 3
    lengths = np.array([4, 1, 0])
    args = dict(u=r.standard_normal((B, H, N)), delta=0.5 + 0.1 * r.standard_normal((B, H, N)), A=-r.random((H, S)),
                Bm=r.standard_normal((B, G, S, N)), Cm=r.standard_normal((B, G, S, N)), D=r.standard_normal(H),
                z=r.standard_normal((B, H, N)), bias=0.1 * r.standard_normal(H), state=r.standard_normal((B, H, S)))
    dy, dlast = r.standard_normal((B, H, N)), r.standard_normal((B, H, S))

    def loss(**a):
        y, last, _ = scan.scan_fwd(**a, softplus=softplus, lengths=lengths)
        return (y * dy).sum() + (last * dlast).sum()

    g = scan.scan_bwd(dy, **args, softplus=softplus, lengths=lengths, dlast=dlast)
    _differences(loss, args, {n: g["d" + {"Bm": "B", "Cm": "C"}.get(n, n)] for n in args}, args)


def test_scan_parts_make_the_whole():
    r = np.random.default_rng(5)
    B, H, N, S = 2, 4, 9, 3
    a = dict(u=r.standard_normal((B, H, N)), delta=r.standard_normal((B, H, N)), Bm=r.standard_normal((B, 2, S, N)),
             Cm=r.standard_normal((B, 2, S, N)), z=r.standard_normal((B, H, N)))
    A = -r.random((H, S))
    y, last, _ = scan.scan_fwd(A=A, **a)
    part = lambda s: {k: v[..., s] for k, v in a.items()}  # noqa: E731
    y1, mid, _ = scan.scan_fwd(A=A, **part(slice(0, 4)))
    y2, end, _ = scan.scan_fwd(A=A, state=mid, **part(slice(4, N)))
    assert np.allclose(np.concatenate([y1, y2], 2), y) and np.allclose(end, last)


@pytest.mark.parametrize("x_first", [False, True])
@pytest.mark.parametrize("y_first", [False, True])
def test_linear_gradients_against_differences(x_first, y_first):
    r = np.random.default_rng(6)
    B, N, K, M = 2, 3, 4, 2
    args = dict(x=r.standard_normal((B, K, N) if x_first else (B, N, K)), W=r.standard_normal((M, K)), bias=r.standard_normal(M))
    dy = r.standard_normal((B, M, N) if y_first else (B, N, M))
    loss = lambda x, W, bias: (linear.linear_fwd(x, W, bias, "gelu", x_first, y_first) * dy).sum()  # noqa: E731
    _differences(loss, args, dict(zip(("x", "W", "bias"), linear.linear_bwd(dy, **args, name="gelu", x_first=x_first, y_first=y_first))), args)


def test_linear_by_hand():
    y = linear.linear_fwd(np.array([[[1.0, 2.0]]]), np.array([[1.0, 1.0], [-1.0, -1.0], [0.0, 2.0]]), np.array([0.5, 0.0, 0.0]), "relu",
                          residual=np.full((1, 1, 3), 10.0))
    assert (y == [[[13.5, 10.0, 14.0]]]).all()


def test_the_selective_blocks_gradients_against_differences():
    rng = np.random.default_rng(11)
    B, N, H, E, R, S, G, taps = 2, 9, 3, 4, 2, 3, 2, 3
    shapes = dict(W_u=(E, H), W_z=(E, H), W_r=(R, E), W_d=(E, R), W_B=(G * S, E), W_C=(G * S, E), W_y=(H, E), taps=(E, taps), taps_bias=(E,),
                  rate=(E, S), D=(E,), dt_bias=(E,))
    p = {k: rng.standard_normal(s) * 0.7 for k, s in shapes.items()}
    x, dy, lengths = rng.standard_normal((B, H, N)), rng.standard_normal((B, H, N)), np.array([N, 6])
    dx, grads = selective.backward(dy, p, selective.forward(x, p, S, G, lengths)[1], lengths)
    value = lambda x, p: (dy * selective.forward(x, p, S, G, lengths)[0]).sum()  # noqa: E731
    eps = 1e-5      # differences: eps^2 of third derivatives and 2^-53 / eps of values of some tens
    for name in (*shapes, None):
        d = rng.standard_normal(x.shape if name is None else shapes[name])
        side = lambda s: value(x + s * d, p) if name is None else value(x, {**p, name: p[name] + s * d})  # noqa: E731
        want = (d * (dx if name is None else grads[name])).sum()
        assert abs((side(eps) - side(-eps)) / (2 * eps) - want) < 1e-6 * max(1.0, abs(want)), name
