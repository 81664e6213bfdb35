"""Embedding and its gradient against the float64 oracle."""
import numpy as np
import pytest
import torch

import paper_2302_06646_amd as lc
from oracle import dropout, embed

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}
U = 2.0 ** -24


def _np(t):
    return t.detach().cpu().double().numpy()


def _layout(first):
    return lc.CHANNELS_FIRST if first else lc.CHANNELS_LAST


def _ids(B, N, V, kind, seed, dtype=torch.int64):
    """Tokens: any ("all"), one ("one"), half of them one and some none ("heavy"), none ("none")."""
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, V, (B, N))
    if kind == "one":
        ids[:] = V - 1
    elif kind == "heavy":
        ids[rng.random((B, N)) < 0.5] = V // 2
        ids[rng.random((B, N)) < 0.1] = -1
        ids[rng.random((B, N)) < 0.05] = V
    elif kind == "none":
        ids = np.where(rng.random((B, N)) < 0.5, -1, np.iinfo(np.int32).max)
    return torch.from_numpy(ids).to(dtype).cuda()


def _randn(shape, dtype, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("io,table", [("fp32", "fp32"), ("fp16", "fp32"), ("fp16", "fp16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("B,N,V,H,p", [(1, 1, 1, 1, 0.0), (2, 3, 5, 7, 0.5), (1, 65, 300, 64, 0.1), (3, 64, 17, 193, 0.3), (4, 1, 1000, 768, 0.0),
                                       (2, 129, 40, 65, 1.0), (5, 7, 9, 3, 0.4)])
def test_forward_against_oracle(first, io, table, B, N, V, H, p):
    ids = _ids(B, N, V, "heavy", B + N, torch.int32 if N % 2 else torch.int64)
    E = _randn((V, H), DT[table], 1)
    shape = (B, H, N) if first else (B, N, H)
    y = torch.full(shape, 7.0, dtype=DT[io], device="cuda")
    lc.longconv_embed_fwd(ids, E, y, 1.7, _layout(first), p, 5, 6)
    m = dropout.mask(shape, p, 5, 6)
    want = embed.embed_fwd(_np(ids).astype(np.int64), _np(E), float(np.float32(1.7)), first, m)
    # the factor (two roundings), its product with the entry, the result
    assert (np.abs(_np(y) - want) <= (UNIT[io] + 3 * U) * np.abs(want) + TINY[io]).all()
    assert ((_np(y) == 0) == (want == 0)).all()


@pytest.mark.parametrize("first", [False, True])
def test_fused_dropout_is_dropout_of_the_rows(first):
    ids, E = _ids(3, 50, 20, "all", 1), _randn((20, 72), torch.bfloat16, 2)
    shape = (3, 72, 50) if first else (3, 50, 72)
    y, want = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lc.longconv_embed_fwd(ids, E, want, 1.0, _layout(first))
    lc.longconv_dropout_fwd(want, want, 0.3, 8, 9)
    lc.longconv_embed_fwd(ids, E, y, 1.0, _layout(first), 0.3, 8, 9)
    assert torch.equal(y, want)


def _backward(ids, V, H, first, io, p, seed, scale=0.7):
    B, N = ids.shape
    shape = (B, H, N) if first else (B, N, H)
    dy = _randn(shape, DT[io], seed)
    dE = torch.full((V, H), float("nan"), device="cuda")
    ws = lc.new_workspace_embed(B, N, V, H, lc.dtype_code(dy), _layout(first))
    ws.fill_(0xA5)                                                     # what was there before is no matter
    lc.longconv_embed_bwd(dy, ids, dE, scale, _layout(first), ws, p, 5, 6)
    again = torch.full((V, H), float("nan"), device="cuda")
    lc.longconv_embed_bwd(dy, ids, again, scale, _layout(first), ws, p, 5, 6)
    assert torch.equal(dE, again)                                      # a fixed order
    ids64, m = _np(ids).astype(np.int64), dropout.mask(shape, p, 5, 6)
    s = float(np.float32(scale))
    want = embed.embed_bwd(_np(dy), ids64, V, s, first, m)
    size = embed.embed_bwd(np.abs(_np(dy)), ids64, V, s, first, m)
    most = np.bincount(ids64[(ids64 >= 0) & (ids64 < V)], minlength=V).max()
    # n - 1 additions of sums no larger than the sum of magnitudes, the factor (two roundings) and its product
    assert (np.abs(_np(dE) - want) <= (most + 3) * U * size).all()
    assert (_np(dE)[size.sum(1) == 0] == 0).all()


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("io", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("kind", ["all", "heavy", "one", "none"])
@pytest.mark.parametrize("B,N,V,H,p", [(1, 1, 1, 1, 0.0), (1, 31, 4, 8, 0.2), (2, 16, 3, 9, 0.0), (1, 33, 700, 17, 0.1), (3, 700, 50, 40, 0.3)])
def test_gradient_against_oracle(first, io, kind, B, N, V, H, p):
    _backward(_ids(B, N, V, kind, N, torch.int32 if H % 2 else torch.int64), V, H, first, io, p, N + V)


# vocabularies around the digits of one, two and three sorting passes; tokens around a tile, several tiles, larger tiles
@pytest.mark.parametrize("V", [255, 256, 257, 511, 512, 513, 65536, 262143, 262144, 1 << 24])
def test_vocabularies(V):
    _backward(_ids(2, 1100, V, "heavy", V), V, 2, False, "fp32", 0.0, 1)


@pytest.mark.parametrize("M", [32, 64, 2047, 2048, 2049, 5000, 530000])
@pytest.mark.parametrize("kind", ["all", "heavy", "one"])
def test_token_counts(M, kind):
    _backward(_ids(1, M, 300, kind, M), 300, 1, False, "fp16", 0.0, 2)


@pytest.mark.parametrize("io", ["fp16", "bf16"])
@pytest.mark.parametrize("kind", ["all", "heavy", "one"])
@pytest.mark.parametrize("B,N,V,H,p", [(1, 4096, 256, 64, 0.1), (2, 1500, 256, 70, 0.0), (3, 1001, 40, 33, 0.2), (1, 8192, 5, 16, 0.0),
                                       (7, 257, 255, 130, 0.1)])
def test_small_vocabularies_in_the_convolutions_layout(io, kind, B, N, V, H, p):
    _backward(_ids(B, N, V, kind, N), V, H, True, io, p, 3)


# what one workgroup sorts and what tiles do; runs of few chunks and of many, in rows of one column to rows of several waves
@pytest.mark.parametrize("M,V,H,io", [(8191, 2000, 9, "fp32"), (8192, 40, 1, "fp32"), (8193, 600, 20, "bf16"), (16384, 3, 70, "fp16"),
                                      (12000, 5000, 300, "bf16"), (20000, 2, 33, "fp32"), (3000, 2, 515, "bf16")])
@pytest.mark.parametrize("kind", ["all", "heavy", "one"])
def test_sorts_and_joins(M, V, H, io, kind):
    _backward(_ids(1, M, V, kind, M), V, H, False, io, 0.1, 4)


def test_wide_rows():
    _backward(_ids(2, 40, 6, "heavy", 1), 6, 5000, False, "bf16", 0.1, 1)
    _backward(_ids(2, 40, 6, "heavy", 1), 6, 5000, True, "bf16", 0.1, 1)


def test_a_gradient_that_is_not_finite_stays_with_its_token():
    ids = torch.tensor([[0, 1, 2, 1, -1]], device="cuda")
    dy = torch.ones(1, 5, 4, device="cuda")
    dy[0, 1, 2], dy[0, 4, 0] = float("nan"), float("inf")
    dE = torch.empty(3, 4, device="cuda")
    lc.longconv_embed_bwd(dy, ids, dE, 1.0, lc.CHANNELS_LAST, lc.new_workspace_embed(1, 5, 3, 4, lc.F32))
    want = torch.tensor([[1, 1, 1, 1], [2, 2, float("nan"), 2], [1, 1, 1, 1.0]])
    assert torch.equal(torch.nan_to_num(dE.cpu(), 99.0), torch.nan_to_num(want, 99.0))


@pytest.mark.parametrize("io", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_columns_that_are_not_finite_stay_with_their_tokens(io, p):
    # what is not finite at a place without a token, or dropped, reaches nothing; elsewhere its own token and channel
    B, N, V, H = 2, 700, 90, 40
    ids = _ids(B, N, V, "heavy", 3)
    dy = _randn((B, H, N), DT[io], 4)
    m = dropout.mask((B, H, N), p, 5, 6)
    gone = (ids < 0) | (ids >= V)
    dy.masked_fill_(gone[:, None, :], float("nan"))
    dy.masked_fill_(torch.from_numpy(m).cuda() == 0, float("inf"))
    kept = np.argwhere((m[1, 7] != 0) & ~gone[1].cpu().numpy())[:, 0]
    dy[1, 7, int(kept[11])] = float("inf")
    dy[1, 7, int(kept[30])] = float("nan")
    dE = torch.full((V, H), 3.0, device="cuda")
    ws = lc.new_workspace_embed(B, N, V, H, lc.dtype_code(dy), lc.CHANNELS_FIRST)
    lc.longconv_embed_bwd(dy, ids, dE, 1.0, lc.CHANNELS_FIRST, ws, p, 5, 6)
    ids64 = _np(ids).astype(np.int64)
    clean = np.nan_to_num(_np(dy), nan=0.0, posinf=0.0)
    want, size = (embed.embed_bwd(a, ids64, V, 1.0, True, m) for a in (clean, np.abs(clean)))
    bad = {int(ids64[1, int(kept[i])]) for i in (11, 30)}
    got = _np(dE)
    for v in range(V):
        for h in range(H):
            if v in bad and h == 7:
                assert not np.isfinite(got[v, h])
    ok = np.ones((V, H), bool)
    ok[list(bad), 7] = False
    most = np.bincount(ids64[(ids64 >= 0) & (ids64 < V)], minlength=V).max()
    assert (np.abs(got - want)[ok] <= ((most + 3) * U * size)[ok]).all()


@pytest.mark.parametrize("first", [False, True])
def test_offsets_past_32_bits(first):
    B, N, V, H = 3, 1 << 20, 8, 1030                                   # 3.2e9 elements
    ids = torch.full((B, N), -1, device="cuda")
    ids[B - 1, N - 70:] = torch.arange(70, device="cuda") % V
    E = _randn((V, H), torch.bfloat16, 1)
    y = torch.empty((B, H, N) if first else (B, N, H), dtype=torch.bfloat16, device="cuda")
    lc.longconv_embed_fwd(ids, E, y, 2.0, _layout(first), 0.25, 3, 4)
    tail = y[B - 1, :, N - 70:].t() if first else y[B - 1, N - 70:]
    t, h = np.meshgrid(np.arange(N - 70, N, dtype=np.int64), np.arange(H, dtype=np.int64), indexing="ij")
    m = dropout.factors(((B - 1) * H + h) * N + t if first else ((B - 1) * N + t) * H + h, 0.25, 3, 4)
    rows = _np(E)[np.arange(70) % V]
    want = 2 * rows * m
    assert (np.abs(_np(tail) - want) <= 1.01 * UNIT["bf16"] * np.abs(want)).all()
    dE = torch.empty(V, H, device="cuda")
    ws = lc.new_workspace_embed(B, N, V, H, lc.BF16, _layout(first))
    lc.longconv_embed_bwd(y, ids, dE, 1.0, _layout(first), ws, 0.25, 3, 4)
    g = _np(tail) * m
    want = np.stack([g[v::V].sum(0) for v in range(V)])
    assert (np.abs(_np(dE) - want) <= 12 * U * np.stack([np.abs(g[v::V]).sum(0) for v in range(V)])).all()
    del y, ws
    torch.cuda.empty_cache()


def test_graph_replays_with_new_masks():
    B, N, V, H = 2, 300, 1000, 64
    ids, E, dy = _ids(B, N, V, "heavy", 1), _randn((V, H), torch.float32, 1), _randn((B, N, H), torch.bfloat16, 2)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    ws, y, dE = lc.new_workspace_embed(B, N, V, H, lc.BF16), torch.empty_like(dy), torch.empty(V, H, device="cuda")

    def both(call, step=None):
        lc.longconv_embed_fwd(ids, E, y, 1.0, lc.CHANNELS_LAST, 0.2, 1, call, step)
        lc.longconv_embed_bwd(dy, ids, dE, 1.0, lc.CHANNELS_LAST, ws, 0.2, 1, call, step)

    both(5, step)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(5, step)
    for i in range(3):
        step.fill_(i)
        g.replay()
        got = y.clone(), dE.clone()
        torch.cuda.synchronize()
        both(5 + i)
        assert torch.equal(got[0], y) and torch.equal(got[1], dE)


def test_every_way_through_the_binding_gives_the_same_bits():
    class Sub(torch.Tensor):
        pass

    ids, E, dy = _ids(2, 30, 50, "all", 1), _randn((50, 24), torch.float32, 1), _randn((2, 30, 24), torch.bfloat16, 2)
    ws = lc.new_workspace_embed(2, 30, 50, 24, lc.BF16)
    outs = []
    for way in (lambda t: t, lambda t: t.as_subclass(Sub)):
        y, dE = torch.empty_like(dy), torch.empty(50, 24, device="cuda")
        lc.longconv_embed_fwd(way(ids), E, y, 2.0, p=0.5, seed=1, call=2)
        lc.longconv_embed_bwd(way(dy), ids, dE, 2.0, lc.CHANNELS_LAST, ws, 0.5, 1, 2)
        outs.append((y, dE))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    with pytest.raises(lc.LongconvError):
        lc.longconv_embed_fwd(ids, E, dy.transpose(1, 2), 1.0)          # not contiguous
    with pytest.raises(lc.LongconvError):
        lc.longconv_embed_fwd(ids, E, dy, 1.0, lc.CHANNELS_FIRST)       # the other layout's shape
    with pytest.raises(lc.LongconvError):
        lc.longconv_embed_fwd(ids.short(), E, dy, 1.0)
    with pytest.raises(lc.LongconvError):
        lc.longconv_embed_fwd(ids, E.half(), dy, 1.0)                   # neither fp32 nor the rows' type
    with pytest.raises(lc.LongconvError):
        lc.longconv_embed_bwd(dy, ids, E, 1.0, lc.CHANNELS_LAST, ws[:100])


def test_more_long_runs_than_a_workgroup_notes_down():
    # 288 tokens of 640 places each (20 chunks of 32 and the ends of one), in rows of 255 pieces of 256 columns: about 287 long runs for
    # each workgroup that joins them.  The order of a sum is that of its run's length alone, whatever else is joined: that of the first
    # 256 columns by themselves, where no workgroup has more than two.
    V, each, H = 288, 640, 255 * 256
    ids = (torch.randperm(V * each, generator=torch.Generator().manual_seed(1)) % V)[None].cuda()
    dy = torch.empty(1, V * each, H, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    dE = torch.empty(V, H, device="cuda")
    ws = lc.new_workspace_embed(1, V * each, V, H, lc.BF16)
    lc.longconv_embed_bwd(dy, ids, dE, 1.0, lc.CHANNELS_LAST, ws)
    for at in (0, 256 * 100, H - 256):
        narrow = torch.empty(V, 256, device="cuda")
        lc.longconv_embed_bwd(dy[:, :, at:at + 256].contiguous(), ids, narrow, 1.0, lc.CHANNELS_LAST, ws)
        assert torch.equal(dE[:, at:at + 256], narrow)
    del dy, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("V", [40, 300])
@pytest.mark.parametrize("size", [1.1e38, 3e-39])
def test_gradients_at_the_ends_of_the_range(first, V, size):
    # sums of two that fit fp32, though twice as much would not; and of two below the normal range
    ids = torch.arange(16, device="cuda").remainder_(8)[None]
    shape = (1, 24, 16) if first else (1, 16, 24)
    dy = (size * (0.5 + torch.rand(*shape, generator=torch.Generator().manual_seed(1)))).to(torch.bfloat16).cuda()
    dE = torch.empty(V, 24, device="cuda")
    lc.longconv_embed_bwd(dy, ids, dE, 1.0, _layout(first), lc.new_workspace_embed(1, 16, V, 24, lc.BF16, _layout(first)))
    want = embed.embed_bwd(_np(dy), _np(ids).astype(np.int64), V, 1.0, first)
    assert (np.abs(_np(dE) - want) <= 2 * U * np.abs(want) + 2.0 ** -149).all()


@pytest.mark.parametrize("bad", ["one for each channel", "all"])
def test_columns_that_are_not_finite_cost_a_few_times_as_much(bad):
    # An overflow under loss scaling is an ordinary step.  Places taken one by one from memory, a workgroup's waves in turn, would wait
    # for it two thousand times here, about a hundred times the product's time.
    B, N, V, H = 8, 16384, 256, 256
    ids = torch.randint(0, V, (B, N), generator=torch.Generator().manual_seed(1)).cuda()
    clean = _randn((B, H, N), torch.float16, 2)
    dy = clean.clone()
    if bad == "all":
        dy.fill_(float("nan"))
    else:
        dy[:, :, 5::512] = float("inf")                                 # in every wave's share of every channel
    dE = torch.empty(V, H, device="cuda")
    ws = lc.new_workspace_embed(B, N, V, H, lc.F16, lc.CHANNELS_FIRST)

    def time(t):
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(5):
            lc.longconv_embed_bwd(t, ids, dE, 1.0, lc.CHANNELS_FIRST, ws, 0.1, 1, 2)
        end.record()
        end.synchronize()
        return start.elapsed_time(end) / 5

    times = [(time(clean), time(dy)) for _ in range(6)][1:]
    assert min(t[1] for t in times) < 8 * min(t[0] for t in times), times
