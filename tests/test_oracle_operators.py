"""The oracles of dropout, embedding and group norm: published values, closed forms, differences."""
import numpy as np
import pytest

from oracle import dropout, embed, gnorm


def test_generator_against_published_values():
    # the known answers that the generator's authors publish: counter and key zero, then all ones
    f = 0xFFFFFFFF
    assert [int(w) for w in dropout.philox((0, 0, 0, 0), (0, 0), 7)] == [0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48]
    assert [int(w) for w in dropout.philox((0, 0, 0, 0), (0, 0), 10)] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert [int(w) for w in dropout.philox((f, f, f, f), (f, f), 10)] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_mask_drops_the_share_it_says_and_does_not_repeat():
    n = 1 << 18
    for p in (0.0, 0.1, 0.5, 1.0):
        m = dropout.mask((n,), p, seed=3 << 40, call=7)
        assert abs((m == 0).mean() - p) <= 5 * np.sqrt(p * (1 - p) / n) + 2.0 ** -16
        assert p == 1.0 or np.isclose(m.max(), 1 / (1 - p), rtol=1e-4)
    a, b, c = (dropout.mask((n,), 0.5, seed, call) for seed, call in ((1, 1), (1, 2), (2, 1)))
    for x, y in ((a, b), (a, c), (a[8:], a[:-8])):
        assert abs(np.corrcoef(x, y)[0, 1]) < 5 / np.sqrt(n)
    tied = dropout.mask((6, 100), 0.5, 1, 1, tie=100)
    assert (tied == tied[:, :1]).all() and (tied[:, 0] == dropout.mask((6,), 0.5, 1, 1)).all()
    x = np.array([np.nan, np.inf, 2.0])
    assert (dropout.dropout(x, np.array([0.0, 0.0, 2.0]), np.ones(3)) == [1, 1, 5]).all()


@pytest.mark.parametrize("first", [False, True])
def test_embedding_gradient_is_the_adjoint(first):
    rng = np.random.default_rng(1)
    B, N, V, H = 2, 7, 5, 3
    ids = rng.integers(-1, V + 1, (B, N))
    shape = (B, H, N) if first else (B, N, H)
    m = dropout.mask(shape, 0.3, 5, 6)
    E, dy = rng.standard_normal((V, H)), rng.standard_normal(shape)
    y = embed.embed_fwd(ids, E, 1.5, first, m)
    dE = embed.embed_bwd(dy, ids, V, 1.5, first, m)
    assert np.isclose((y * dy).sum(), (E * dE).sum(), rtol=1e-12)       # linear in E
    t = tuple(np.argwhere(ids == -1)[0])
    assert (y[t[0], :, t[1]] if first else y[t]).any() == False         # noqa: E712


@pytest.mark.parametrize("name", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("C,G", [(6, 1), (6, 3), (4, 4)])
def test_group_norm_gradients_against_differences(name, C, G):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 5, C)) + 3, rng.standard_normal((2, 5, C))
    gamma, beta = rng.standard_normal(C), rng.standard_normal(C)
    f = lambda x, gamma, beta: (gnorm.gnorm_fwd(x, gamma, beta, G, 1e-5, name)[0] * dy).sum()  # noqa: E731
    for got, at in zip(gnorm.gnorm_bwd(dy, x, gamma, beta, G, 1e-5, name), range(3)):
        args, h = [x, gamma, beta], 1e-6
        for i in np.ndindex(args[at].shape):
            up, down = [[a.copy() for a in args] for _ in range(2)]
            up[at][i] += h
            down[at][i] -= h
            assert np.isclose((f(*up) - f(*down)) / (2 * h), got[i], rtol=1e-5, atol=1e-6)


def test_group_norm_of_constants_and_known_numbers():
    y, mean, rstd = gnorm.gnorm_fwd(np.full((1, 3, 4), 7.0), np.ones(4), np.full(4, 0.5), 2, 1e-2, "none")
    assert (y == 0.5).all() and (mean == 7).all() and np.allclose(rstd, 10)
    y, _, _ = gnorm.gnorm_fwd(np.array([[[-1.0, 1.0]]]), np.ones(2), np.zeros(2), 1, 0.0, "relu")
    assert np.allclose(y, [[[0, 1]]])
