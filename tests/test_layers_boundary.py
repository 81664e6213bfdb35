"""Refusals and sizes of the short convolution, the selective scan and the dense product.  No kernel is launched: arguments are checked first."""
import ctypes

import pytest
import torch

import paper_2302_06646_amd as lc

A, ODD, HALF, BIG = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), ctypes.c_void_p(0x1004), 1 << 50
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


def _refuses(f, good, changes):
    for at, value, want in changes:
        args = list(good)
        for i, v in zip(at, value) if isinstance(at, tuple) else ((at, value),):
            args[i] = v
        assert f(*args) == want, (f.__name__, at, value)


def test_short_refusals_and_workspace():
    L = lc.lib()
    #       x  k  bias state y last lengths B H  N   taps act io stream
    good = (A, A, A, A, A, A, A, 2, 3, 50, 4, 1, 2, None)
    shapes = [(7, 0, SHAPE), (8, 0, SHAPE), (9, 0, SHAPE), (8, 65536, SHAPE), (9, 1 << 35, SHAPE), ((7, 9), (1 << 20, 1 << 20), SHAPE),
              (7, 1 << 62, SHAPE), (10, 0, SHAPE), (10, 9, SHAPE), (11, 4, SHAPE), (11, -1, SHAPE), (12, 3, DTYPE), (12, -1, DTYPE)]
    _refuses(L.longconv_short_fwd, good, shapes + [(0, None, NULL), (1, None, NULL), (4, None, NULL)] +
             [(i, ODD, ALIGN) for i in range(6)] + [(6, HALF, ALIGN)])
    #       dy x k bias state dlast dx dk dbias dstate lengths B H  N  taps act io ws bytes stream
    good = (A, A, A, A, A, A, A, A, A, A, A, 2, 3, 50, 4, 1, 2, A, BIG, None)
    _refuses(L.longconv_short_bwd, good, [(0, None, NULL), (1, None, NULL), (2, None, NULL), (13, 0, SHAPE), (14, 9, SHAPE), (15, 7, SHAPE),
                                          (16, 5, DTYPE), (17, None, WORKSPACE),
                                          (18, lc.longconv_short_workspace_bytes(2, 3, 50, 4, 2) - 1, WORKSPACE), (10, HALF, ALIGN)] +
             [(i, ODD, ALIGN) for i in (*range(10), 17)])
    args = list(good)
    args[6:10] = [None] * 4
    assert L.longconv_short_bwd(*args) == 0                              # nothing asked for
    #       x  k bias state y B  H taps act io stream
    good = (A, A, A, A, A, 2, 3, 4, 1, 2, None)
    _refuses(L.longconv_short_step, good, [(0, None, NULL), (1, None, NULL), (3, None, NULL), (4, None, NULL), (5, 0, SHAPE), (6, 65536, SHAPE),
                                           (7, 9, SHAPE), (8, 4, SHAPE), (9, 3, DTYPE), (3, ODD, ALIGN)])
    for H, N in ((1, 1), (3, 100), (193, 385), (1024, 4096), (2, 70000)):
        sizes = [lc.longconv_short_workspace_bytes(B, H, N, 4, lc.BF16) for B in (*range(1, 300), 500, 1000)]
        assert min(sizes) > 0 and sizes == sorted(sizes)
    assert lc.longconv_short_workspace_bytes(1, 1, 1, 9, lc.F32) == 0
    with pytest.raises(lc.LongconvError):
        lc.new_workspace_short(1, 1, 0, 4, lc.F32)


def test_scan_refusals_and_workspace():
    L = lc.lib()
    #       u  delta A B C D z bias state y last marks lengths B H  N   S  G softplus io ws bytes stream
    good = (A, A, A, A, A, A, A, A, A, A, A, A, A, 2, 6, 50, 16, 2, 1, 2, A, BIG, None)
    shapes = [(13, 0, SHAPE), (14, 0, SHAPE), (15, 0, SHAPE), (16, 0, SHAPE), (17, 0, SHAPE), (16, 65, SHAPE), (17, 4, SHAPE), (17, 7, SHAPE),
              (14, 65536, SHAPE), (15, 1 << 34, SHAPE), (13, 1 << 60, SHAPE), ((13, 14, 15, 16), (1 << 24, 60, 1, 64), SHAPE), (19, 3, DTYPE)]
    _refuses(L.longconv_scan_fwd, good, shapes + [(i, None, NULL) for i in (0, 1, 2, 3, 4, 9)] + [(i, ODD, ALIGN) for i in (*range(12), 20)] +
             [(12, HALF, ALIGN), (20, None, WORKSPACE), (21, lc.longconv_scan_workspace_bytes(2, 6, 50, 16, 2, 2, False) - 1, WORKSPACE)])
    #       dy u delta A B C D z bias marks dlast du ddelta dA dB dC dD dz dbias dstate lengths B H  N   S  G softplus io ws bytes stream
    good = (A,) * 21 + (2, 6, 50, 16, 2, 1, 2, A, BIG, None)
    _refuses(L.longconv_scan_bwd, good, [(i, None, NULL) for i in (0, 1, 2, 3, 4, 5, 9)] + [(i, ODD, ALIGN) for i in (*range(20), 28)] + [
        (7, None, NULL), (20, HALF, ALIGN), (21, 0, SHAPE), (24, 65, SHAPE), (25, 5, SHAPE), (27, 9, DTYPE), (28, None, WORKSPACE),
        (29, lc.longconv_scan_workspace_bytes(2, 6, 50, 16, 2, 2, True) - 1, WORKSPACE)])
    args = list(good)
    args[11:20] = [None] * 9
    assert L.longconv_scan_bwd(*args) == 0
    #       u  delta A B C D z bias state y B H S  G softplus io stream
    good = (A,) * 10 + (2, 6, 16, 2, 1, 2, None)
    _refuses(L.longconv_scan_step, good, [(i, None, NULL) for i in (0, 1, 2, 3, 4, 8, 9)] + [(10, 0, SHAPE), (12, 65, SHAPE), (13, 4, SHAPE),
                                                                                            (15, 3, DTYPE), (8, ODD, ALIGN)])
    for H, N, S, G in ((1, 1, 1, 1), (193, 385, 5, 1), (1024, 1024, 16, 1), (256, 16384, 16, 4), (64, 131072, 16, 1), (40, 3000, 64, 2), (12, 600, 3, 12)):
        for bwd in (False, True):
            sizes = [lc.longconv_scan_workspace_bytes(B, H, N, S, G, lc.F16, bwd) for B in (*range(1, 300), 500, 511, 512, 513, 600, 1000, 2000)]
            assert min(sizes) > 0 and sizes == sorted(sizes)
        assert lc.longconv_scan_workspace_bytes(3, H, N, S, G, 1, True) >= lc.longconv_scan_workspace_bytes(3, H, N, S, G, 1, False)
    with pytest.raises(lc.LongconvError):
        lc.new_workspace_scan(1, 6, 10, 4, 4, lc.F32, True)


def test_linear_refusals_and_workspace():
    L = lc.lib()
    #       x  W bias residual y B N  K   M  act xl yl io ws bytes stream
    good = (A, A, A, A, A, 2, 9, 64, 32, 1, 0, 1, 2, A, BIG, None)
    shapes = [(5, 0, SHAPE), (6, 0, SHAPE), (7, 0, SHAPE), (8, 0, SHAPE), (7, 65536, SHAPE), (8, 65536, SHAPE), (6, 1 << 26, SHAPE),
              (5, 1 << 40, SHAPE), ((5, 6, 8), (1 << 24, 2, 129), SHAPE), (9, 4, SHAPE), (9, -1, SHAPE), (10, 2, SHAPE), (11, -1, SHAPE),
              (12, 3, DTYPE)]
    _refuses(L.longconv_linear_fwd, good, shapes + [(0, None, NULL), (1, None, NULL), (4, None, NULL), (13, None, WORKSPACE), (14, 0, WORKSPACE)] +
             [(i, ODD, ALIGN) for i in (0, 1, 2, 3, 4, 13)])
    #       dy x W bias dx dW dW_type dbias B N K   M  act xl yl io ws bytes stream
    good = (A, A, A, A, A, A, 0, A, 2, 9, 64, 32, 1, 0, 1, 2, A, BIG, None)
    _refuses(L.longconv_linear_bwd, good, [(0, None, NULL), (1, None, NULL), (2, None, NULL), (6, 1, DTYPE), (6, 7, DTYPE), (9, 0, SHAPE),
                                           (12, 9, SHAPE), (13, 3, SHAPE), (15, 4, DTYPE), (16, None, WORKSPACE),
                                           (17, lc.longconv_linear_workspace_bytes(2, 9, 64, 32, 2, True) - 1, WORKSPACE)] +
             [(i, ODD, ALIGN) for i in (0, 1, 2, 3, 4, 5, 7, 16)])
    args = list(good)
    args[4] = args[5] = args[7] = None
    assert L.longconv_linear_bwd(*args) == 0
    for N, K, M in ((1, 1, 1), (385, 193, 1009), (1024, 768, 2048), (7, 4096, 8), (16384, 256, 1024)):
        for io in (lc.F32, lc.BF16):
            for bwd in (False, True):
                sizes = [lc.longconv_linear_workspace_bytes(B, N, K, M, io, bwd) for B in (*range(1, 200), 300, 1000)]
                assert min(sizes) > 0 and sizes == sorted(sizes)
    assert lc.longconv_linear_workspace_bytes(1, 0, 5, 5, 0, True) == 0
    with pytest.raises(lc.LongconvError):
        lc.new_workspace_linear(1, 1, 0, 5, lc.F32, False)


def test_the_binding_refuses_host_tensors_and_unknown_names():
    x, k = torch.zeros(2, 3, 4), torch.zeros(3, 2)
    with pytest.raises(lc.LongconvError, match="x must be a contiguous device tensor"):
        lc.longconv_short_fwd(x, k, None, x, "silu")
    with pytest.raises(lc.LongconvError, match="x must be"):
        lc.longconv_short_bwd(x, x, k, None, x, k, None, "silu", k)
    with pytest.raises(lc.LongconvError, match="x must be"):
        lc.longconv_short_step(x[..., 0], k, None, x, x[..., 0], "none")
    with pytest.raises(lc.LongconvError, match="u must be"):
        lc.longconv_scan_fwd(x, x, k, x[:, None], x[:, None], x, k)
    with pytest.raises(lc.LongconvError, match="u must be"):
        lc.longconv_scan_bwd(x, x, x, k, x[:, None], x[:, None], k, x, x, k, x, x, k)
    with pytest.raises(lc.LongconvError, match="u must be"):
        lc.longconv_scan_step(x[0], x[0], k, x, x, x, x[0])
    with pytest.raises(lc.LongconvError, match="x must be"):
        lc.longconv_linear_fwd(x, k, None, x, "none", k)
    with pytest.raises(lc.LongconvError, match="x must be"):
        lc.longconv_linear_bwd(x, x, k, None, x, k, None, "none", k)
    with pytest.raises(KeyError):
        lc.longconv_linear_fwd(x, k, None, x, "tanh", k)


@pytest.mark.parametrize("io", [lc.F32, lc.F16, lc.BF16])
@pytest.mark.parametrize("K,M", [(768, 2048), (64, 4096), (100, 77), (4096, 40)])
def test_scratch_of_many_short_sequences_is_that_of_their_places(io, K, M):
    size = lambda B, N: lc.longconv_linear_workspace_bytes(B, N, K, M, io, True)  # noqa: E731
    for B in (1, 3, 15, 64, 1000, 65536):
        assert size(B, 1) == size(1, B)                    # the same product, whichever way its places are counted
    # of two places each: beside what all places as one need, two rows of sums for each sequence, as [B,.,N] is cut
    assert size(65536, 2) <= size(1, 131072) + 65536 * 2 * M * 4
