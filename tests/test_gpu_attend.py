"""GPU parity of the attention of new tokens over a cache, and over chosen pages, with the float64 oracle."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as C
import cache_testlib as TL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2503_00022_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def _status():
    import torch
    return torch.zeros(4, dtype=torch.int32, device="cuda:0")


class Case:
    """Tensors of one call and their float64 values."""

    def __init__(self, B, dtype, fmt, D, Hq, Hkv, lens, counts, layers=1, own=False, layout=None, seed=0, gain=1.0):
        self.B, self.dtype, self.D, self.Hq, self.Hkv, self.lens, self.counts, self.layers = B, dtype, D, Hq, Hkv, lens, counts, layers
        T, N = sum(lens), sum(counts)
        layout = layout or (lambda t: t)
        k, v = (TL.normal(seed + i, (layers, T, Hkv, D), dtype) * gain for i in (1, 2))
        self.k_dense = layout(k)
        self.q = layout(TL.normal(seed + 3, (layers, N, Hq, D), dtype))
        if fmt is None:
            self.k, self.v, self.k64, self.v64 = layout(k), layout(v), TL.numpy64(k), TL.numpy64(v)
        else:
            (self.k, self.k64), (self.v, self.v64) = (TL.quantise(B, x, fmt) for x in (k, v))
        self.q64 = TL.numpy64(self.q)
        self.kn = self.vn = None
        if own:
            self.kn, self.vn = (layout(TL.normal(seed + i, (layers, N, Hkv, D), dtype)) for i in (4, 5))
        self.cu, self.cn = np.concatenate([[0], np.cumsum(lens)]), np.concatenate([[0], np.cumsum(counts)])
        self.prob = B.Problem(layers, Hq, Hkv, D, lens, device="cuda:0")
        self.out, self.lse = layout(self.q.clone().fill_(7.0)), None
        import torch
        self.lse = torch.full((layers, Hq, N), 7.0, dtype=torch.float32, device="cuda:0")
        self.status = _status()

    def run(self, new, **more):
        self.B.kvcrush_attend(self.prob, new, self.q, self.k, self.v, self.out, k_new=self.kn, v_new=self.vn, lse=self.lse,
                              status=self.status, **more)

    def check(self, visible):
        """visible(layer, s, i, kv head): (row numbers of the cache, numbers of the sequence's new tokens) that token i sees."""
        G, scale = self.Hq // self.Hkv, 1.0 / math.sqrt(self.D)
        out, lse = TL.numpy64(self.out), self.lse.double().cpu().numpy()
        kn, vn = (TL.numpy64(self.kn), TL.numpy64(self.vn)) if self.kn is not None else (None, None)
        for l in range(self.layers):
            for s, n in enumerate(self.counts):
                for i in range(n):
                    t = self.cn[s] + i
                    for h in range(self.Hkv):
                        rows, new = visible(l, s, i, h)
                        k, v = self.k64[l, rows, h], self.v64[l, rows, h]
                        if len(new):
                            new = np.asarray(new) + self.cn[s]
                            k, v = np.concatenate([k, kn[l, new, h]]), np.concatenate([v, vn[l, new, h]])
                        heads = range(h * G, h * G + G)
                        TL.check_rows([out[l, t, x] for x in heads], [lse[l, x, t] for x in heads],
                                      [(self.q64[l, t, x], k, v, scale) for x in heads], self.dtype, self.D)
        assert self.status.cpu().tolist()[0] == 0


SHAPES = [
    # type, cache, D, query heads, KV heads, cached rows, new tokens
    ("bf16", None, 128, 8, 2, (300, 1, 17, 2000), (1, 1, 1, 1)),
    ("bf16", None, 64, 4, 4, (129,), (5,)),
    ("fp16", None, 96, 6, 2, (33, 0, 250), (3, 2, 0)),
    ("fp16", None, 40, 9, 1, (100,), (2,)),
    ("bf16", None, 256, 2, 1, (70, 515), (4, 1)),
    ("bf16", None, 200, 24, 2, (31,), (6,)),
    ("fp32", None, 64, 8, 8, (257, 40), (3, 1)),
    ("fp32", None, 136, 3, 1, (90,), (11,)),
    ("bf16", C.INT8, 128, 8, 2, (300, 1, 17, 2000), (1, 1, 1, 1)),
    ("fp16", C.INT8, 64, 12, 1, (100, 9), (4, 7)),
    ("bf16", C.INT8, 80, 4, 2, (65,), (9,)),
    ("bf16", C.INT8, 256, 4, 2, (200,), (1,)),
    ("bf16", C.E4M3, 128, 4, 1, (513, 16), (1, 2)),
    ("fp16", C.E4M3, 48, 2, 2, (77,), (17,)),
    ("bf16", C.INT4, 128, 8, 2, (400, 3, 1000), (1, 1, 1)),
    ("fp16", C.INT4, 96, 6, 3, (150,), (8,)),
    ("bf16", C.INT4, 64, 5, 1, (60, 48), (3, 20)),
    ("bf16", C.INT4, 256, 2, 2, (130,), (2,)),
    ("fp32", C.INT8, 64, 4, 2, (120,), (2,)),
    ("fp32", C.INT4, 32, 4, 2, (120,), (3,)),
    ("fp32", C.E4M3, 128, 4, 2, (50,), (3,)),
]


@pytest.mark.parametrize("dtype,fmt,D,Hq,Hkv,lens,counts", SHAPES)
def test_tokens_at_the_end_of_the_cache(B, dtype, fmt, D, Hq, Hkv, lens, counts):
    c = Case(B, dtype, fmt, D, Hq, Hkv, lens, counts, layers=2, seed=D + Hq)
    c.run(B.NewTokens(counts))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s] + max(0, lens[s] - counts[s] + 1 + i)), []))


@pytest.mark.parametrize("dtype,fmt,D,Hq,Hkv,lens,counts", SHAPES)
def test_trees_of_drafted_tokens(B, dtype, fmt, D, Hq, Hkv, lens, counts):
    """Every token sees the whole cache and its ancestors; one token of every larger tree sees no drafted token at all, which
    leaves it nothing where the cache is empty."""
    words = max(counts) // 32 + 2                       # more than are needed
    bits, sees = TL.tree_bits(D, counts, words, empty_row=True)
    c = Case(B, dtype, fmt, D, Hq, Hkv, lens, counts, own=True, seed=D + Hq)
    c.run(B.NewTokens(counts, mask=_dev(bits)))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.flatnonzero(sees[s][i])))


@pytest.mark.parametrize("dtype,fmt,Hq,Hkv,n", [("bf16", None, 8, 2, 63), ("fp16", C.INT8, 32, 4, 33), ("bf16", C.INT4, 4, 4, 100),
                                               ("fp16", None, 128, 1, 3), ("fp32", None, 4, 2, 40), ("bf16", C.E4M3, 16, 1, 64)])
def test_many_query_rows(B, dtype, fmt, Hq, Hkv, n):
    """Trees and groups of more rows than one block of rows holds, chains without a mask."""
    lens, counts = (700, 45), (n, n // 2)
    bits, sees = TL.tree_bits(n, counts, (n + 31) // 32)
    c = Case(B, dtype, fmt, 128, Hq, Hkv, lens, counts, own=True, seed=n)
    c.run(B.NewTokens(counts, mask=_dev(bits)))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.flatnonzero(sees[s][i])))
    c.run(B.NewTokens(counts))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.arange(i + 1)))
    c.kn = c.vn = None
    c.run(B.NewTokens(counts))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s] + max(0, lens[s] - counts[s] + 1 + i)), []))


@pytest.mark.parametrize("layout", [TL.strided, TL.by_head])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides(B, layout, dtype):
    lens, counts = (50, 131), (3, 1)
    c = Case(B, dtype, None, 64, 6, 3, lens, counts, layers=2, own=True, layout=layout, seed=5)
    c.run(B.NewTokens(counts))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.arange(i + 1)))


@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("fp16", C.INT4), ("fp32", None), ("bf16", C.INT8)])
def test_growing_caches_with_counts_on_the_device(B, dtype, fmt):
    """Rows of each layer and sequence start where the arrays say; counts beyond the longest sequence or the layer's end are
    taken up to there, negative ones as none; rows behind the count may hold anything."""
    import torch
    lens, counts, layers = (64, 64, 64), (1, 2, 1), 2
    c = Case(B, dtype, fmt, 128, 4, 2, lens, counts, layers=layers, seed=9)
    begin = np.asarray([[0, 70, 150], [100, 3, 180]], dtype=np.int32)
    count = np.asarray([[60, 64, 1], [-3, 37, 64]], dtype=np.int32)
    if fmt is None:
        for x in (c.k, c.v):
            x[0, 60:70] = float("nan")
            x[0, 151:] = float("nan")
            x[1, 40:100] = float("nan")
    c.run(B.NewTokens(counts), row_begin=_dev(begin), row_count=_dev(count))
    held = np.minimum(np.clip(count, 0, 64), 192 - begin)
    c.check(lambda l, s, i, h: (begin[l, s] + np.arange(max(0, held[l, s] - counts[s] + 1 + i)), []))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_unseen_rows_have_no_influence(B, dtype):
    """Infinities and NaN in the keys and values of tokens that a row does not see stay out of it, and reach those that see
    them."""
    lens, counts, n = (20, 37), (6, 9), 15
    bits, sees = TL.tree_bits(77, counts, 1, empty_row=True)
    c = Case(B, dtype, None, 64, 4, 2, lens, counts, own=True, seed=21)
    c.vn[0, 2, :, 3] = float("nan")                      # seen by token 2 of the first tree and those below it
    c.vn[0, 9, 0, 60] = float("inf")
    c.kn[0, 12, :, 0] = float("nan")
    c.kn[0, 4] = float("-inf")
    c.vn[0, 14] = float("inf")
    c.run(B.NewTokens(counts, mask=_dev(bits)))
    with np.errstate(invalid="ignore"):
        c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.flatnonzero(sees[s][i])))
    # the same for rows of the cache that come after a token's own
    c = Case(B, dtype, None, 64, 4, 2, lens, (4, 4), seed=22)
    c.v[0, 19], c.k[0, 18, 0], c.v[0, 56, 1, 5] = float("nan"), float("nan"), float("inf")
    c.k64, c.v64 = TL.numpy64(c.k), TL.numpy64(c.v)
    c.run(B.NewTokens((4, 4)))
    with np.errstate(invalid="ignore"):
        c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s] + lens[s] - 3 + i), []))


def test_rows_without_weight(B):
    """Logits of -inf throughout give zeros; weights far below the largest vanish; a value row's scale far below the others' still
    counts where it alone has weight."""
    import torch
    lens, counts = (40, 40), (1, 1)
    c = Case(B, "bf16", None, 64, 2, 1, lens, counts, seed=31)
    c.q[0, 0] = 1.0
    c.k[0, :40] = 0.0
    c.k[0, :40, :, 0] = float("-inf")
    c.q64, c.k64 = TL.numpy64(c.q), TL.numpy64(c.k)
    c.run(B.NewTokens(counts))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), []))
    assert (TL.numpy64(c.out)[0, 0] == 0).all() and (c.lse[0, :, 0] == float("-inf")).all()
    c = Case(B, "bf16", C.INT8, 64, 2, 1, (50,), (1,), seed=32)
    k = TL.normal(33, (1, 50, 1, 64), "bf16")
    v = TL.normal(34, (1, 50, 1, 64), "bf16")
    k[0, 7] = c.q[0, 0, 0] * 12                          # row 7 has all the weight of the first head, and tiny values
    v[0, 7] *= 2.0 ** -40
    (c.k, c.k64), (c.v, c.v64) = TL.quantise(B, k, C.INT8), TL.quantise(B, v, C.INT8)
    c.run(B.NewTokens((1,)))
    c.check(lambda l, s, i, h: (np.arange(50), []))


def test_wide_range_of_queries_and_scales(B):
    """Queries and caches of very large and very small values."""
    for qs, ks, fmt in ((2.0 ** 60, 2.0 ** -60, C.INT8), (2.0 ** -60, 2.0 ** 58, C.E4M3), (2.0 ** 40, 2.0 ** -41, C.INT4), (2.0 ** 50, 2.0 ** -50, None)):
        c = Case(B, "bf16", fmt, 64, 4, 2, (70,), (2,), seed=41, gain=ks)
        c.q *= qs
        c.q64 = TL.numpy64(c.q)
        c.run(B.NewTokens((2,)))
        c.check(lambda l, s, i, h: (np.arange(69 + i), []))


PAGED = [
    # type, cache, D, query heads, KV heads, cached rows, new tokens, page, budget, initial, recent
    ("bf16", None, 128, 8, 2, (1000, 31, 1), (1, 1, 1), 32, 6, 1, 2),
    ("fp16", None, 64, 4, 4, (515, 0), (2, 1), 8, 11, 0, 0),
    ("bf16", C.INT8, 128, 16, 2, (700,), (3,), 24, 5, 1, 1),
    ("fp16", C.INT4, 96, 3, 1, (400, 90), (1, 4), 16, 300, 1, 1),
    ("bf16", C.E4M3, 256, 2, 2, (333,), (1,), 40, 3, 3, 3),
    ("fp32", None, 64, 4, 2, (260, 17), (1, 2), 8, 4, 0, 1),
    ("fp32", C.INT8, 32, 2, 1, (100,), (1,), 8, 1, 0, 0),
    ("bf16", None, 40, 40, 1, (200,), (2,), 64, 2, 0, 0),
    ("fp16", None, 256, 20, 1, (210, 9), (1, 1), 8, 9, 1, 1),
    ("bf16", None, 192, 2, 2, (300,), (1,), 16, 4, 0, 2),
    ("bf16", C.INT4, 256, 4, 1, (260,), (2,), 16, 5, 0, 1),
    ("fp32", C.E4M3, 256, 2, 1, (90,), (1,), 8, 3, 0, 0),
]


@pytest.mark.parametrize("dtype,fmt,D,Hq,Hkv,lens,counts,page,budget,initial,recent", PAGED)
def test_chosen_pages(B, dtype, fmt, D, Hq, Hkv, lens, counts, page, budget, initial, recent):
    import torch
    layers, G = 2, Hq // Hkv
    c = Case(B, dtype, fmt, D, Hq, Hkv, lens, counts, layers=layers, seed=D + page)
    most = -(-max(lens) // page)
    shape = (layers, len(lens) * most, Hkv, D)
    lo, hi = (torch.full(shape, 5.0, dtype=c.q.dtype, device="cuda:0") for _ in range(2))
    B.kvcrush_page_bounds(c.prob, c.k_dense, page, lo, hi, status=c.status)
    k_dense, want_lo, want_hi = TL.numpy64(c.k_dense), np.full(shape, 5.0), np.full(shape, 5.0)
    for l in range(layers):
        for s, n in enumerate(lens):
            for h in range(Hkv):
                if n:
                    a, b = C.page_bounds(k_dense[l, c.cu[s]:c.cu[s + 1], h], page)
                    want_lo[l, s * most:s * most + len(a), h], want_hi[l, s * most:s * most + len(a), h] = a, b
    assert np.array_equal(TL.numpy64(lo), want_lo) and np.array_equal(TL.numpy64(hi), want_hi)
    N = sum(counts)
    idx = torch.full((layers, N, Hkv, budget), -7, dtype=torch.int32, device="cuda:0")
    num = torch.full((layers, N, Hkv), -7, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend_pages(c.prob, B.NewTokens(counts), c.q, c.k, c.v, page, lo, hi, budget, c.out, keep_initial=initial,
                           keep_recent=recent, page_idx=idx, n_pages=num, lse=c.lse, status=c.status)
    idx, num = idx.cpu().numpy(), num.cpu().numpy()

    def visible(l, s, i, h):
        seen = max(0, lens[s] - counts[s] + 1 + i)
        pages, t = -(-seen // page), c.cn[s] + i
        scores = C.page_scores(c.q64[l, t, h * G:h * G + G], want_lo[l, s * most:s * most + pages, h], want_hi[l, s * most:s * most + pages, h])
        chosen = C.choose_pages(scores, budget, initial, recent)
        assert num[l, t, h] == len(chosen) and idx[l, t, h, :len(chosen)].tolist() == chosen.tolist(), (l, s, i, h)
        assert (idx[l, t, h, len(chosen):] == -1).all()
        rows = (chosen[:, None] * page + np.arange(page)).reshape(-1)
        return c.cu[s] + rows[rows < seen], []

    c.check(visible)


def test_ties_nan_and_zero_queries_in_the_choice(B):
    """Equal scores go to the lower page, a NaN bound counts as the largest, channels that no head asks for are left out."""
    import torch
    page, L, D = 8, 96, 32
    c = Case(B, "bf16", None, D, 1, 1, (L,), (1,), seed=51)
    c.k.copy_(torch.arange(L, device="cuda:0").div(8, rounding_mode="floor").remainder(3).view(1, L, 1, 1).expand_as(c.k))
    c.q.fill_(1.0)
    c.q[..., 4] = 0.0
    c.k[0, 17, 0, 4] = float("inf")                      # not asked for
    c.k[0, 90, 0, 5] = float("nan")
    lo, hi = (torch.zeros((1, 12, 1, D), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
    B.kvcrush_page_bounds(c.prob, c.k, page, lo, hi, status=c.status)
    assert torch.isnan(lo[0, 11, 0, 5]) and torch.isnan(hi[0, 11, 0, 5])
    for budget, want in ((1, [11]), (3, [2, 5, 11]), (4, [2, 5, 8, 11]), (6, [1, 2, 4, 5, 8, 11]), (12, list(range(12)))):
        idx = torch.zeros((1, 1, 1, budget), dtype=torch.int32, device="cuda:0")
        B.kvcrush_attend_pages(c.prob, B.NewTokens((1,)), c.q, c.k, c.v, page, lo, hi, budget, c.out, page_idx=idx, status=c.status)
        assert idx.cpu().numpy().reshape(-1).tolist() == want


def test_bounds_of_the_last_pages_only(B):
    import torch
    page, lens = 16, (100, 7, 0, 64)
    c = Case(B, "fp16", None, 64, 2, 2, lens, (1, 1, 1, 1), seed=61)
    full, part = (torch.full((2, 1, 4 * 7, 2, 64), 3.0, dtype=torch.float16, device="cuda:0") for _ in range(2))
    B.kvcrush_page_bounds(c.prob, c.k, page, full[0], full[1], status=c.status)
    for recent in (1, 2, 50):
        part.fill_(3.0)
        B.kvcrush_page_bounds(c.prob, c.k, page, part[0], part[1], recent_pages=recent, status=c.status)
        for s, n in enumerate(lens):
            P = -(-n // page)
            for p in range(7):
                here = part[:, 0, s * 7 + p]
                assert torch.equal(here, full[:, 0, s * 7 + p]) if max(0, P - recent) <= p < P else (here == 3).all()


def test_every_page_is_the_whole_cache(B):
    """A budget of all pages gives what kvcrush_attend gives."""
    import torch
    lens = (200, 333)
    c = Case(B, "bf16", None, 128, 8, 2, lens, (1, 1), seed=71)
    lo, hi = (torch.zeros((1, 2 * 11, 2, 128), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
    B.kvcrush_page_bounds(c.prob, c.k, 32, lo, hi, status=c.status)
    B.kvcrush_attend_pages(c.prob, B.NewTokens((1, 1)), c.q, c.k, c.v, 32, lo, hi, 11, c.out, lse=c.lse, status=c.status)
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), []))


def test_the_same_call_gives_the_same_bits_and_replays(B):
    """Two calls, and a captured one replayed on new contents, on a stream of its own."""
    import torch
    c = Case(B, "bf16", C.INT8, 128, 8, 2, (3000, 500), (4, 4), own=True, seed=81)
    new = B.NewTokens((4, 4))
    c.run(new)
    first, first_lse = c.out.clone(), c.lse.clone()
    c.out.zero_()
    c.run(new)
    assert torch.equal(first, c.out) and torch.equal(first_lse, c.lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.run(new)
    c.q.copy_(c.q.flip(1))
    c.q64 = TL.numpy64(c.q)
    g.replay()
    torch.cuda.synchronize()
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.arange(i + 1)))


def test_no_new_tokens_and_empty_caches(B):
    c = Case(B, "bf16", None, 64, 2, 1, (0, 0), (2, 0), own=True, seed=91)
    c.run(B.NewTokens((2, 0)))
    c.check(lambda l, s, i, h: ([], np.arange(i + 1)))
    c.kn = c.vn = None
    c.run(B.NewTokens((2, 0)))
    c.check(lambda l, s, i, h: ([], []))
    B.kvcrush_attend(c.prob, B.NewTokens((0, 0)), c.q, c.k, c.v, c.out, status=c.status)


TREES = [
    # type, D, query heads, KV heads, cached rows, new tokens, layers
    ("bf16", 128, 8, 2, (700, 130, 64, 5), (20, 33, 63, 9), 1),
    ("fp16", 64, 16, 2, (1000, 0, 333), (5, 40, 7), 2),
    ("bf16", 96, 4, 1, (257,), (100,), 1),
    ("fp16", 40, 33, 1, (128, 127), (1, 4), 1),
    ("bf16", 128, 64, 1, (5000,), (3,), 1),
    ("bf16", 64, 2, 2, (640,), (300,), 1),
]


@pytest.mark.parametrize("dtype,D,Hq,Hkv,lens,counts,layers", TREES)
@pytest.mark.parametrize("layout", [None, TL.strided, TL.by_head])
def test_tiles_of_query_rows(B, dtype, D, Hq, Hkv, lens, counts, layers, layout):
    """Rows that fill tiles of 128: trees, chains, tokens at the end of the cache; tails, short sequences, several tiles of rows."""
    bits, sees = TL.tree_bits(D, counts, (max(counts) + 31) // 32, empty_row=True)
    c = Case(B, dtype, None, D, Hq, Hkv, lens, counts, own=True, seed=D + Hq, layers=layers, layout=layout)
    c.run(B.NewTokens(counts, mask=_dev(bits)))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.flatnonzero(sees[s][i])))
    c.kn = c.vn = None
    c.run(B.NewTokens(counts))
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s] + max(0, lens[s] - counts[s] + 1 + i)), []))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_unseen_rows_have_no_influence_on_tiles(B, dtype):
    lens, counts = (300, 170), (40, 36)
    bits, sees = TL.tree_bits(78, counts, 2, empty_row=True)
    c = Case(B, dtype, None, 64, 4, 2, lens, counts, own=True, seed=23)
    c.vn[0, 20, :, 3] = float("nan")
    c.kn[0, 30, 0, 0] = float("nan")
    c.vn[0, 60, 1] = float("inf")
    c.run(B.NewTokens(counts, mask=_dev(bits)))
    with np.errstate(invalid="ignore"):
        c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.flatnonzero(sees[s][i])))
    c = Case(B, dtype, None, 64, 4, 2, lens, counts, seed=24)
    c.v[0, 290], c.k[0, 280, 0], c.v[0, 465, 1, 5] = float("nan"), float("nan"), float("inf")
    c.k64, c.v64 = TL.numpy64(c.k), TL.numpy64(c.v)
    c.run(B.NewTokens(counts))
    with np.errstate(invalid="ignore"):
        c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s] + lens[s] - counts[s] + 1 + i), []))
    # rows behind the counts, and what one sequence's rows hold, stay out of the others
    c = Case(B, dtype, None, 64, 4, 2, (320, 320), (20, 20), own=True, seed=25)
    c.k[0, 300:320], c.v[0, 300:320] = float("nan"), float("inf")
    c.run(B.NewTokens((20, 20)), row_begin=_dev(np.asarray([[0, 320]], dtype=np.int32)), row_count=_dev(np.asarray([[300, 200]], dtype=np.int32)))
    c.check(lambda l, s, i, h: (np.arange((0, 320)[s], (300, 520)[s]), np.arange(i + 1)))


def test_growing_maxima_on_tiles(B):
    """Keys whose logits grow along the cache, so that the reference of the weights has to move often."""
    import torch
    c = Case(B, "bf16", None, 128, 8, 1, (2000,), (10,), own=True, seed=26)
    c.k *= torch.linspace(0.1, 12.0, 2000, device="cuda:0").view(1, -1, 1, 1).to(c.k.dtype)
    c.k64 = TL.numpy64(c.k)
    c.run(B.NewTokens((10,)))
    c.check(lambda l, s, i, h: (np.arange(2000), np.arange(i + 1)))


def test_negative_scale(B):
    c = Case(B, "bf16", None, 64, 16, 2, (500,), (9,), seed=27)
    c.prob.struct.softmax_scale = -0.1
    c.run(B.NewTokens((9,)))
    import torch
    out = TL.numpy64(c.out)
    for i in (0, 8):
        for x in (0, 15):
            n = 500 - 9 + 1 + i
            o, lse, _, _ = C.attend_row(c.q64[0, i, x], c.k64[0, :n, x // 8], c.v64[0, :n, x // 8], -0.1)
            assert np.abs(out[0, i, x] - o).max() < 0.01 and abs(float(c.lse[0, x, i]) - lse) < 1e-3


@pytest.mark.parametrize("dtype,n", [("bf16", 2), ("fp16", 30), ("fp32", 3)])
def test_heads_that_share_memory(B, dtype, n):
    """A stride of 0 along the heads of the cache and of the new tokens (the TMA unit cannot take it)."""
    c = Case(B, dtype, None, 64, 8, 4, (300,), (n,), own=True, seed=28)
    c.k, c.v, c.kn, c.vn = (x[:, :, :1].expand(-1, -1, 4, -1) for x in (c.k, c.v, c.kn, c.vn))
    c.k64, c.v64 = TL.numpy64(c.k), TL.numpy64(c.v)
    c.run(B.NewTokens((n,)))
    c.check(lambda l, s, i, h: (np.arange(300), np.arange(i + 1)))


@pytest.mark.parametrize("pages,page", [(8192, 8), (3000, 16)])
@pytest.mark.parametrize("dtype,fmt,D,Hq,Hkv", [("bf16", None, 64, 2, 1), ("fp16", C.INT4, 32, 1, 1), ("fp32", None, 8, 2, 1), ("bf16", None, 136, 1, 1)])
def test_many_pages(B, dtype, fmt, D, Hq, Hkv, pages, page):
    """As many pages as a sequence may have, budgets from one page to nearly all of them."""
    import torch
    L = pages * page - 3
    c = Case(B, dtype, fmt, D, Hq, Hkv, (L,), (1,), seed=29)
    lo, hi = (torch.zeros((1, pages, Hkv, D), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
    B.kvcrush_page_bounds(c.prob, c.k_dense, page, lo, hi, status=c.status)
    lo64, hi64 = TL.numpy64(lo), TL.numpy64(hi)
    for budget in (1, 100, pages - 1):
        idx = torch.zeros((1, 1, Hkv, budget), dtype=torch.int32, device="cuda:0")
        B.kvcrush_attend_pages(c.prob, B.NewTokens((1,)), c.q, c.k, c.v, page, lo, hi, budget, c.out, keep_recent=1, page_idx=idx,
                               lse=c.lse, status=c.status)

        def visible(l, s, i, h):
            q = c.q64[0, 0]
            up, down = np.where(q > 0, q, 0).sum(0), np.where(q < 0, q, 0).sum(0)
            scores = hi64[0, :, h] @ up + lo64[0, :, h] @ down
            chosen = C.choose_pages(scores, budget, 0, 1)
            assert idx.cpu().numpy().reshape(-1).tolist() == chosen.tolist()
            rows = (chosen[:, None] * page + np.arange(page)).reshape(-1)
            return rows[rows < L], []

        c.check(visible)


def test_scores_at_the_ends_of_the_range(B):
    """Scores beyond float32 and far below 1 are ordered as float64 orders them."""
    import torch
    for qs, ks in ((2.0 ** 100, 2.0 ** 60), (2.0 ** -60, 2.0 ** -50), (2.0 ** -100, 2.0 ** 60)):
        c = Case(B, "bf16", None, 64, 4, 2, (400,), (1,), seed=30, gain=ks)
        c.q *= qs
        c.q64 = TL.numpy64(c.q)
        lo, hi = (torch.zeros((1, 50, 2, 64), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
        B.kvcrush_page_bounds(c.prob, c.k, 8, lo, hi, status=c.status)
        idx = torch.zeros((1, 1, 2, 7), dtype=torch.int32, device="cuda:0")
        B.kvcrush_attend_pages(c.prob, B.NewTokens((1,)), c.q, c.k, c.v, 8, lo, hi, 7, c.out, page_idx=idx, status=c.status)
        for h in range(2):
            scores = C.page_scores(c.q64[0, 0, 2 * h:2 * h + 2], TL.numpy64(lo)[0, :, h], TL.numpy64(hi)[0, :, h])
            assert idx[0, 0, h].cpu().numpy().tolist() == C.choose_pages(scores, 7, 0, 0).tolist()


@pytest.mark.parametrize("dtype,fmt,n", [("bf16", None, 1), ("fp16", None, 40), ("bf16", C.INT8, 2), ("fp16", C.INT4, 1), ("fp32", None, 1)])
def test_rows_beyond_four_gigabytes(B, dtype, fmt, n):
    """A token stride of a mebibyte: the last rows of the cache lie more than 2^32 bytes from its start."""
    import torch
    L, D, page = 4400, 64, 8
    c = Case(B, dtype, fmt, D, 2, 1, (L,), (n,), own=True, seed=33)

    def spread(t):
        step = (1 << 20) // t.element_size()
        big = torch.zeros(L * step, dtype=t.dtype, device="cuda:0")
        view = big.as_strided((1, L, 1, t.shape[3]), (L * step, step, t.shape[3], 1))
        view.copy_(t)
        return view

    if fmt is None:
        c.k, c.v = spread(c.k), spread(c.v)
    else:
        c.k, c.v = (B.QuantTensor(spread(x.codes), x.scales, fmt) for x in (c.k, c.v))
    c.run(B.NewTokens((n,)))
    c.check(lambda l, s, i, h: (np.arange(L), np.arange(i + 1)))
    if fmt is None:
        lo, hi = (torch.zeros((1, L // page, 1, D), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
        B.kvcrush_page_bounds(c.prob, c.k, page, lo, hi, status=c.status)
        a, b = C.page_bounds(c.k64[0, :, 0], page)
        assert np.array_equal(TL.numpy64(lo)[0, :, 0], a) and np.array_equal(TL.numpy64(hi)[0, :, 0], b)
    else:
        back = torch.zeros((1, L, 1, D), dtype=torch.float32, device="cuda:0")
        B.kvcrush_dequantize(c.prob, c.k, None, back, None, status=c.status)
        assert np.allclose(TL.numpy64(back), c.k64, rtol=2.0 ** -22, atol=2.0 ** -21)


@pytest.mark.parametrize("lens", [(700,), (40, 300)])
def test_a_bounded_wait_that_runs_out_is_reported(B, lens):
    """The producer of the kernel for many query rows stops before its first copy: nothing is in flight, every role's first wait
    gives up, the kernel returns and says so, and the same call succeeds once the status word is cleared."""
    import ctypes
    import torch
    counts = (12,) * len(lens)
    c = Case(B, "bf16", None, 128, 8, 2, lens, counts, own=True, seed=34)
    new = B.NewTokens(counts)
    fn = B.lib().kvcrush_diag_attend
    fn.argtypes, fn.restype = [ctypes.c_void_p] * 10 + [ctypes.c_int] * 2, ctypes.c_int
    call = lambda withhold: fn(c.prob.address, new.ref, *(B._packed(t) for t in (c.q, c.k, c.v, c.kn, c.vn, c.out)),   # noqa: E731
                               c.status.data_ptr(), B._stream(), 1, withhold)
    assert call(1) == 0
    torch.cuda.synchronize()
    st = c.status.cpu().tolist()
    assert st[0] == B.DEV_TIMEOUT and st[1] == 5
    c.status.zero_()
    c.run(new)
    c.check(lambda l, s, i, h: (np.arange(c.cu[s], c.cu[s + 1]), np.arange(i + 1)))


@pytest.mark.parametrize("dtype,fmt", (("bf16", None), ("fp16", C.INT4), ("fp32", None)))
def test_pages_of_an_empty_cache(B, dtype, fmt):
    """No row at all: no page is chosen, the output is zero, and tensors without rows need no memory."""
    import torch
    c = Case(B, dtype, fmt, 64, 4, 2, (0, 0), (1, 2), layers=2, seed=81)
    lo, hi = (torch.empty((2, 0, 2, 64), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
    B.kvcrush_page_bounds(c.prob, c.k_dense, 16, lo, hi, status=c.status)
    idx = torch.full((2, 3, 2, 4), -7, dtype=torch.int32, device="cuda:0")
    num = torch.full((2, 3, 2), -7, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend_pages(c.prob, B.NewTokens((1, 2)), c.q, c.k, c.v, 16, lo, hi, 4, c.out, page_idx=idx, n_pages=num, lse=c.lse,
                           status=c.status)
    assert (idx == -1).all() and (num == 0).all() and (c.out == 0).all() and torch.isneginf(c.lse).all()
    assert c.status.cpu().tolist()[0] == 0


@pytest.mark.parametrize("dtype,fmt,n,page", (("bf16", C.INT8, 1, 0), ("bf16", None, 40, 0), ("fp32", None, 3, 0), ("fp16", C.INT4, 1, 16)))
def test_calls_at_once_on_two_streams(B, dtype, fmt, n, page):
    """Two calls over different caches, in turn on two streams that are not the current one, give the bits of calls alone."""
    import torch
    cases = [Case(B, dtype, fmt, 64, 8, 2, (900, 300), (n, 1), own=not page, seed=101 + i) for i in (0, 10)]
    new = B.NewTokens((n, 1))
    bounds = []
    for c in cases:
        lo, hi = (torch.zeros((1, 2 * 57, 2, 64), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
        if page:
            B.kvcrush_page_bounds(c.prob, c.k_dense, page, lo, hi, status=c.status)
        bounds.append((lo, hi))

    def call(i, **more):
        c = cases[i]
        if page:
            B.kvcrush_attend_pages(c.prob, new, c.q, c.k, c.v, page, *bounds[i], 7, c.out, lse=c.lse, status=c.status, **more)
        else:
            c.run(new, **more)

    alone = []
    for i, c in enumerate(cases):
        call(i)
        alone.append((c.out.clone(), c.lse.clone()))
        c.out.fill_(7.0)
        c.lse.fill_(7.0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        for i, s in enumerate(streams):
            call(i, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for c, (out, lse) in zip(cases, alone):
        assert torch.equal(c.out, out) and torch.equal(c.lse, lse) and c.status.cpu().tolist()[0] == 0
