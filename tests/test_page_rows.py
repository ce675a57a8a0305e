"""Rows of a cache that was reduced by pages: a short last page has slots that hold no token, and whether it was kept only the
selection knows."""
import math

import numpy as np
import pytest

import cache_testlib as TL
from paper_2503_00022_b200 import binding as B
from paper_2503_00022_b200 import build as kbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


def _pass(lens, kept, device, layers=1, page=8, **more):
    prob = B.Problem(layers, 2, 1, 64, lens, device=device)
    kept = np.broadcast_to(np.asarray(kept, dtype=np.int32), (layers, len(lens)))
    return B.CompressionPass(prob, kept - kept // 2, kept // 2, page_size=page, **more)


def test_rows_follow_the_chosen_pages():
    """On the host: lists of pages with and without the sequence's last one."""
    import torch
    lens, kept = [100, 96, 3, 0, 20, 61], [[4, 4, 1, 2, 2, 0], [5, 12, 0, 1, 3, 3]]
    cp = _pass(lens, kept, "cpu", layers=2, with_cache=False)
    assert cp.row_begin.tolist() == [[0, 32, 64, 72, 72, 88], [0, 40, 136, 136, 136, 160]]
    pages = [[0, 3, 5, 12], [0, 1, 2, 3], [0], [0, 2], [0, 1, 2, 5, 11], list(range(12)), [0, 1, 2], [4, 6, 7]]
    cp.idx.copy_(torch.tensor(sum(pages, []), dtype=torch.int32))
    cp._count_rows()
    assert cp.row_count.tolist() == [[28, 32, 3, 0, 12, 0], [40, 96, 0, 0, 20, 21]]
    # another selection of the same pass
    pages[0], pages[3], pages[7] = [0, 1, 2, 11], [0, 1], [0, 1, 2]
    cp.idx.copy_(torch.tensor(sum(pages, []), dtype=torch.int32))
    cp._count_rows()
    assert cp.row_count.tolist() == [[32, 32, 3, 0, 16, 0], [40, 96, 0, 0, 20, 24]]


def test_rows_that_the_budgets_decide():
    """Whole pages, whole sequences and nothing at all: no selection changes them."""
    assert _pass([96, 33, 8], [4, 5, 0], "cpu", with_cache=False).row_count.tolist() == [[32, 33, 0]]
    assert _pass([7, 5], [3, 1], "cpu", page=1, with_cache=False).row_count.tolist() == [[3, 1]]


def _attend(cp, layers, heads, D, q):
    import torch
    out, lse = torch.empty_like(q), torch.empty((layers, heads, q.shape[1]), dtype=torch.float32, device="cuda:0")
    cache = B.Problem(layers, heads, 1, D, [cp.k_out.shape[1]] + [0] * (cp.problem.n_seqs - 1))
    B.kvcrush_attend(cache, B.NewTokens([1] * cp.problem.n_seqs), q, cp.k_out, cp.v_out, out, lse=lse, row_begin=cp.row_begin,
                     row_count=cp.row_count, status=cp.status)
    return TL.numpy64(out), lse.cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("keep_recent", [0, 1])
def test_attention_over_a_cache_reduced_by_pages(keep_recent):
    """100 tokens (a last page of four), 96, 3 and 61: attention reads the kept tokens and no slot without one; a captured pass
    and attention follow what is selected."""
    import torch
    layers, heads, D, page, lens = 2, 2, 64, 8, [100, 96, 3, 61]
    n, S = sum(lens), len(lens)
    cp = _pass(lens, [4, 4, 1, 5], "cuda:0", layers=layers, cache_dtype=torch.bfloat16, keep_recent=keep_recent)
    qk = [TL.normal(720 + i, (layers, n, h, D), "bf16") for i, h in enumerate((heads, 1))]
    kc, vc = (TL.normal(730 + i, (layers, n, 1, D), "bf16") for i in range(2))
    q = TL.normal(740, (layers, S, heads, D), "bf16")
    cu = np.concatenate([[0], np.cumsum(lens)])

    def check(out, lse):
        cp.check_status()
        short = 0
        for l in range(layers):
            for s, L in enumerate(lens):
                rows = (cp.kept(l, s)[:, None] * page + np.arange(page)).reshape(-1)
                rows = rows[rows < L]
                short += len(rows) % page != 0
                assert int(cp.row_count[l, s]) == len(rows)
                k, v = TL.numpy64(kc)[l, cu[s] + rows, 0], TL.numpy64(vc)[l, cu[s] + rows, 0]
                TL.check_rows([out[l, s, x] for x in range(heads)], [lse[l, x, s] for x in range(heads)],
                              [(TL.numpy64(q)[l, s, x], k, v, 1.0 / math.sqrt(D)) for x in range(heads)], "bf16", D)
        if keep_recent:
            assert short == 3 * layers

    cp.run(*qk, kc, vc)
    check(*_attend(cp, layers, heads, D, q))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cp.run(*qk, kc, vc)
    for seed in range(3):
        qk[0].copy_(TL.normal(750 + seed, tuple(qk[0].shape), "bf16"))
        qk[1].copy_(TL.normal(760 + seed, tuple(qk[1].shape), "bf16"))
        g.replay()
        check(*_attend(cp, layers, heads, D, q))
