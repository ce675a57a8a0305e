"""The choice of pages when scores lie closer than their last bits: all blocks of a cluster read the same pages, the ones that are
reported.  And the choice in caches whose rows start where the device arrays say."""
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


@pytest.mark.parametrize("dtype,fmt,G,spread", [("fp32", None, 1, 8), ("fp32", C.INT8, 4, 0), ("fp32", None, 8, 16), ("fp16", None, 8, 16),
                                                ("fp16", C.INT4, 8, 16), ("bf16", None, 4, 24), ("bf16", C.INT8, 8, 24)])
def test_pages_of_equal_scores_are_chosen_alike_by_all_blocks(B, dtype, fmt, G, spread):
    """The bounds of every page are those of the first with the channels in another order and a query asks for all channels
    alike: the scores are one number, summed in 512 orders, and differ in the last bits of their sums."""
    import torch
    D, page, pages, budget = 128, 32, 512, 100
    L = page * pages
    g = np.random.Generator(np.random.Philox(400 + G + spread))
    dt = TL.torch_dtype(dtype)
    first = g.standard_normal(D) * np.exp2(-g.uniform(0, spread, D))
    hi = torch.from_numpy(np.stack([first[g.permutation(D)] for _ in range(pages)])[None, :, None].astype(np.float32)).to("cuda:0").to(dt)
    lo = hi.clone()
    q = torch.from_numpy(np.abs(g.standard_normal(G)) * np.exp2(-g.uniform(0, 12, G))).to("cuda:0").to(dt)
    q = q.view(1, 1, G, 1).expand(1, 1, G, D).contiguous()
    k, v = (TL.normal(410 + i, (1, L, 1, D), dtype) for i in range(2))
    k64, v64 = TL.numpy64(k), TL.numpy64(v)
    if fmt is not None:
        (k, k64), (v, v64) = TL.quantise(B, k, fmt), TL.quantise(B, v, fmt)
    out, lse = torch.empty_like(q), torch.empty((1, G, 1), dtype=torch.float32, device="cuda:0")
    idx = torch.full((1, 1, 1, budget), -7, dtype=torch.int32, device="cuda:0")
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend_pages(B.Problem(1, G, 1, D, [L]), B.NewTokens([1]), q, k, v, page, lo, hi, budget, out, page_idx=idx, lse=lse,
                           status=status)
    chosen = idx.cpu().numpy().reshape(-1)
    assert (np.diff(chosen) > 0).all() and chosen[0] >= 0 and chosen[-1] < pages
    rows = (chosen[:, None] * page + np.arange(page)).reshape(-1)
    q64, out, lse = TL.numpy64(q), TL.numpy64(out), lse.cpu().numpy()
    TL.check_rows([out[0, 0, x] for x in range(G)], [lse[0, x, 0] for x in range(G)],
                  [(q64[0, 0, x], k64[0, rows, 0], v64[0, rows, 0], 1.0 / math.sqrt(D)) for x in range(G)], dtype, D)
    assert status.cpu().tolist()[0] == 0


@pytest.mark.parametrize("dtype,fmt", [("bf16", None), ("fp16", C.INT8), ("bf16", C.E4M3), ("fp16", C.INT4), ("fp32", None)])
def test_pages_of_rows_that_start_where_the_arrays_say(B, dtype, fmt):
    """Several sequences, layers and new tokens; every layer holds its sequences at other places and in other lengths."""
    import torch
    layers, Hq, Hkv, D, page, budget, total = 2, 4, 2, 64, 16, 4, 500
    counts, initial, recent = [2, 1, 3], 1, 1
    begin = np.asarray([[0, 210, 300], [260, 3, 100]], dtype=np.int32)
    count = np.asarray([[197, 64, 200], [150, 96, 1]], dtype=np.int32)
    k, v = (TL.normal(420 + i, (layers, total, Hkv, D), dtype) for i in range(2))
    dense = k
    k64, v64, dense64 = TL.numpy64(k), TL.numpy64(v), TL.numpy64(k)
    if fmt is not None:
        (k, k64), (v, v64) = TL.quantise(B, k, fmt), TL.quantise(B, v, fmt)
    prob = B.Problem(layers, Hq, Hkv, D, [total, 0, 0])
    most, n = -(-total // page), sum(counts)
    lo, hi = (torch.zeros((layers, 3 * most, Hkv, D), dtype=dense.dtype, device="cuda:0") for _ in range(2))
    q = TL.normal(430, (layers, n, Hq, D), dtype)
    out, lse = torch.empty_like(q), torch.empty((layers, Hq, n), dtype=torch.float32, device="cuda:0")
    idx = torch.full((layers, n, Hkv, budget), -7, dtype=torch.int32, device="cuda:0")
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    where = dict(row_begin=_dev(begin), row_count=_dev(count), status=status)
    B.kvcrush_page_bounds(prob, dense, page, lo, hi, **where)
    B.kvcrush_attend_pages(prob, B.NewTokens(counts), q, k, v, page, lo, hi, budget, out, keep_initial=initial, keep_recent=recent,
                           page_idx=idx, lse=lse, **where)
    q64, out, lse, idx = TL.numpy64(q), TL.numpy64(out), lse.cpu().numpy(), idx.cpu().numpy()
    cn = np.concatenate([[0], np.cumsum(counts)])
    for l in range(layers):
        for s, c in enumerate(counts):
            for i in range(c):
                seen, t = max(0, count[l, s] - c + 1 + i), cn[s] + i
                for h in range(Hkv):
                    # bounds are those of all the sequence's rows, also where a token does not see the last ones
                    a, b = C.page_bounds(dense64[l, begin[l, s]:begin[l, s] + count[l, s], h], page)
                    pages = -(-seen // page)
                    heads = range(2 * h, 2 * h + 2)
                    chosen = C.choose_pages(C.page_scores(q64[l, t, 2 * h:2 * h + 2], a[:pages], b[:pages]), budget, initial, recent)
                    assert idx[l, t, h].tolist() == chosen.tolist() + [-1] * (budget - len(chosen))
                    rows = (chosen[:, None] * page + np.arange(page)).reshape(-1)
                    rows = begin[l, s] + rows[rows < seen]
                    TL.check_rows([out[l, t, x] for x in heads], [lse[l, x, t] for x in heads],
                                  [(q64[l, t, x], k64[l, rows, h], v64[l, rows, h], 1.0 / math.sqrt(D)) for x in heads], dtype, D)
    assert status.cpu().tolist()[0] == 0
