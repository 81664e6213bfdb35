"""Refusals and sizes of the operators around the convolution.  No kernel is launched: arguments are checked first."""
import ctypes

import pytest
import torch

import paper_2302_06646_amd as lc

A, ODD, BIG = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), 1 << 50
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
NAN = float("nan")


def _refuses(f, good, changes):
    for at, value, want in changes:
        args = list(good)
        for i, v in zip(at, value) if isinstance(at, tuple) else ((at, value),):
            args[i] = v
        assert f(*args) == want, (f.__name__, at, value)


def test_dropout_refusals():
    L = lc.lib()
    #       x  r  y  n    tie io p    seed call step stream
    good = (A, A, A, 100, 1, 0, 0.1, 1, 1, A, None)
    _refuses(L.longconv_dropout_fwd, good, [
        (0, None, NULL), (2, None, NULL), (3, 0, SHAPE), (3, -5, SHAPE), (3, (1 << 34) + 1, SHAPE), (4, 0, SHAPE), (4, 3, SHAPE),
        (4, 200, SHAPE), (5, 3, DTYPE), (6, -0.1, SHAPE), (6, 1.1, SHAPE), (6, NAN, SHAPE), (0, ODD, ALIGN), (1, ODD, ALIGN),
        (2, ODD, ALIGN), (9, ctypes.c_void_p(0x1004), ALIGN)])
    good = (A, A, 100, 1, 0, 0.1, 1, 1, A, None)
    _refuses(L.longconv_dropout_bwd, good, [(0, None, NULL), (1, None, NULL), (2, 0, SHAPE), (3, 7, SHAPE), (4, -1, DTYPE),
                                            (5, 2.0, SHAPE), (1, ODD, ALIGN)])


def test_seeded_regulariser_refusals():
    L = lc.lib()
    #       k  kbar H  N     p  lambda q    seed call step stream
    good = (A, A, 4, 1024, 1, 0.01, 0.1, 1, 1, None, None)
    _refuses(L.longconv_kreg_fwd_seeded, good, [(0, None, NULL), (1, None, NULL), (2, 0, SHAPE), (3, 1000, SHAPE), (4, 33, SHAPE),
                                                (5, -1.0, SHAPE), (6, 1.5, SHAPE), (6, NAN, SHAPE), (9, ctypes.c_void_p(0x1004), ALIGN)])
    good = (A, A, A, 4, 1024, 1, 0.01, 0.1, 1, 1, None, None)
    _refuses(L.longconv_kreg_bwd_seeded, good, [(0, None, NULL), (1, None, NULL), (2, None, NULL), (4, 128, SHAPE), (7, -0.5, SHAPE)])


def test_embedding_refusals_and_workspace():
    L = lc.lib()
    #       ids bytes E table y  B  N    V    H   io layout scale p    seed call step stream
    good = (A, 8, A, 0, A, 2, 100, 500, 64, 2, 0, 1.0, 0.1, 1, 1, A, None)
    shapes = [(5, 0, SHAPE), (6, 0, SHAPE), (7, 0, SHAPE), (8, 0, SHAPE), (7, (1 << 24) + 1, SHAPE), (8, 65536, SHAPE),
              (5, 1 << 27, SHAPE), (6, 1 << 26, SHAPE), ((5, 6, 8), (1 << 10, 1 << 10, 1 << 15), SHAPE), (10, 2, SHAPE), (9, 5, DTYPE),
              (12, -1.0, SHAPE), (12, NAN, SHAPE), (1, 2, DTYPE)]
    _refuses(L.longconv_embed_fwd, good, shapes + [
        (0, None, NULL), (2, None, NULL), (4, None, NULL), (3, 1, DTYPE), (3, 9, DTYPE), (0, ODD, ALIGN), (2, ODD, ALIGN), (4, ODD, ALIGN),
        ((5, 6, 10), (1 << 24, 1, 1), SHAPE)])
    #       dy ids bytes dE B  N    V    H   io layout scale p    seed call step ws bytes stream
    good = (A, A, 4, A, 2, 100, 500, 64, 1, 1, 1.0, 0.0, 1, 1, None, A, BIG, None)
    need = lc.longconv_embed_workspace_bytes(2, 100, 500, 64, 1, 1)
    _refuses(L.longconv_embed_bwd, good, [
        (0, None, NULL), (1, None, NULL), (3, None, NULL), (2, 1, DTYPE), (4, -1, SHAPE), (8, 7, DTYPE), (9, 3, SHAPE), (11, 2.0, SHAPE),
        (3, ODD, ALIGN), (15, ODD, ALIGN), (15, None, WORKSPACE), (16, need - 1, WORKSPACE)])
    assert lc.longconv_embed_workspace_bytes(0, 1, 1, 1, 0, 0) == 0 and lc.longconv_embed_workspace_bytes(1, 1, 1, 1, 3, 0) == 0
    with pytest.raises(lc.LongconvError):
        lc.new_workspace_embed(1, 0, 5, 5, lc.F32)
    for layout in (lc.CHANNELS_LAST, lc.CHANNELS_FIRST):
        for V, H in ((1, 1), (300, 33), (65536, 768)):
            for N in (1, 300, 5000):
                sizes = [lc.longconv_embed_workspace_bytes(B, N, V, H, lc.BF16, layout) for B in (*range(1, 150), 200, 500, 1000)]
                assert min(sizes) > 0 and sizes == sorted(sizes)


def test_group_norm_refusals_and_workspace():
    L = lc.lib()
    #       x  gamma beta y mean rstd B  S  C   G  eps  act io ws bytes stream
    good = (A, A, A, A, A, A, 2, 9, 64, 8, 1e-5, 1, 0, A, BIG, None)
    shapes = [(6, 0, SHAPE), (7, 0, SHAPE), (8, 0, SHAPE), (9, 0, SHAPE), (9, 7, SHAPE), (9, 65, SHAPE), (8, 1 << 16, SHAPE),
              (6, 1 << 20, SHAPE), (7, 1 << 30, SHAPE)]
    _refuses(L.longconv_gnorm_fwd, good, shapes + [
        (0, None, NULL), (3, None, NULL), (4, None, NULL), (5, None, NULL), (10, -1.0, SHAPE), (10, NAN, SHAPE), (10, float("inf"), SHAPE),
        (11, 4, SHAPE), (11, -1, SHAPE), (12, 3, DTYPE), (0, ODD, ALIGN), (2, ODD, ALIGN), (13, ODD, ALIGN), (13, None, WORKSPACE),
        (14, lc.longconv_gnorm_workspace_bytes(2, 9, 64, 8, 0, False) - 1, WORKSPACE)])
    #       dy x gamma beta mean rstd dx dgamma dbeta B S C G act io ws bytes stream
    good = (A, A, A, A, A, A, A, A, A, 2, 9, 64, 8, 1, 0, A, BIG, None)
    _refuses(L.longconv_gnorm_bwd, good, [
        (0, None, NULL), (1, None, NULL), (4, None, NULL), (5, None, NULL), (9, 0, SHAPE), (12, 5, SHAPE), (13, 9, SHAPE), (14, 4, DTYPE),
        (6, ODD, ALIGN), (8, ODD, ALIGN), (15, None, WORKSPACE),
        (16, lc.longconv_gnorm_workspace_bytes(2, 9, 64, 8, 0, True) - 1, WORKSPACE)])
    args = list(good)
    args[6] = args[7] = args[8] = None
    assert L.longconv_gnorm_bwd(*args) == 0                              # nothing asked for
    with pytest.raises(lc.LongconvError):
        lc.new_workspace_gnorm(1, 1, 6, 4, lc.F32, True)
    for S, C, G in ((1, 1, 1), (50, 195, 5), (16384, 256, 32), (7, 5000, 50)):
        for bwd in (False, True):
            sizes = [lc.longconv_gnorm_workspace_bytes(B, S, C, G, lc.F16, bwd) for B in (*range(1, 100), 300, 512, 1000, 3000)]
            assert min(sizes) > 0 and sizes == sorted(sizes)
        assert lc.longconv_gnorm_workspace_bytes(4, S, C, G, lc.F16, True) >= lc.longconv_gnorm_workspace_bytes(4, S, C, G, lc.F16, False)


def test_the_binding_refuses_host_tensors_and_unknown_names():
    x = torch.zeros(2, 3, 4)
    s = torch.zeros(2, 2)
    with pytest.raises(lc.LongconvError, match="x must be a contiguous device tensor"):
        lc.longconv_dropout_fwd(x, x, 0.5, 1, 1)
    with pytest.raises(lc.LongconvError, match="dy must be"):
        lc.longconv_dropout_bwd(x, x, 0.5, 1, 1)
    with pytest.raises(lc.LongconvError, match="ids"):
        lc.longconv_embed_fwd(s, torch.zeros(5, 4), torch.zeros(2, 2, 4), 1.0)
    with pytest.raises(lc.LongconvError, match="x must be"):
        lc.longconv_gnorm_fwd(x, None, None, x, s, s, 1e-5, "silu", s)
    with pytest.raises(KeyError):
        lc.longconv_gnorm_fwd(x, None, None, x, s, s, 1e-5, "tanh", s)


def test_group_norm_takes_as_many_sequences_as_a_launch_does():
    # a launch has fewer than 2^32 threads, and rows of fewer than eight channels take a workgroup of 512 for each of the B
    L = lc.lib()
    for C, G in ((1, 1), (3, 1), (4, 2)):
        assert lc.longconv_gnorm_workspace_bytes((1 << 23) - 1, 2, C, G, lc.F32, True) > 0
        for B in (1 << 23, 1 << 24):
            assert lc.longconv_gnorm_workspace_bytes(B, 2, C, G, lc.F32, True) == 0
            assert L.longconv_gnorm_fwd(A, A, A, A, A, A, B, 2, C, G, 1e-5, 1, 0, A, BIG, None) == SHAPE
            assert L.longconv_gnorm_bwd(A, A, A, A, A, A, A, A, A, B, 2, C, G, 1, 0, A, BIG, None) == SHAPE
