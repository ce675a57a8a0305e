"""The operators together, as a decoding loop uses them: a prompt is compressed into a quantised cache, drafted tokens attend to
it, the accepted ones are appended, the next token attends to all; and the same prompt read by pages."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as C
from paper_2503_00022_b200 import inputs
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


def _check(out, lse, q64, layers, cn, counts, Hq, Hkv, D, rows_of):
    G = Hq // Hkv
    out, lse = TL.numpy64(out), lse.double().cpu().numpy()
    for l in range(layers):
        for s, n in enumerate(counts):
            for i in range(n):
                for h in range(Hkv):
                    k, v = rows_of(l, s, i, h)
                    heads = range(h * G, h * G + G)
                    TL.check_rows([out[l, cn[s] + i, x] for x in heads], [lse[l, x, cn[s] + i] for x in heads],
                                  [(q64[l, cn[s] + i, x], k, v, 1.0 / math.sqrt(D)) for x in heads], "bf16", D)


@pytest.mark.parametrize("fmt", [C.INT8, C.E4M3, C.INT4])
def test_compress_draft_append_and_go_on(B, fmt):
    import torch
    layers, Hq, Hkv, D, lens, draft = 2, 8, 2, 128, [900, 331], [5, 4]
    S, spare = len(lens), 8
    w = inputs.Workload("loop", layers, Hq, Hkv, D, tuple(lens), inputs.BF16, inputs.BF16, 0.25, base_seed=300)
    import kvc_testlib as T
    _, q, k, kc, vc = T.stack_layers(w, range(layers))
    q, k, kc, vc = (T.torch_storage(x, inputs.BF16, "cuda:0") for x in (q, k, kc, vc))
    budget = np.asarray([[200, 61], [150, 90]], dtype=np.int32)          # layers keep different numbers of rows
    prob = B.Problem(layers, Hq, Hkv, D, lens)
    cp = B.CompressionPass(prob, budget - budget // 2, budget // 2, cache_format=fmt, spare_rows=spare)
    cp.run(q, k, kc, vc)
    cp.check_status()
    # the reduced cache holds the kept rows, quantised
    k64, v64 = TL.numpy64(kc), TL.numpy64(vc)
    cu = np.concatenate([[0], np.cumsum(lens)])
    begin = cp.row_begin.cpu().numpy()

    def cached():
        return tuple(C.decode(x.codes.cpu().numpy(), x.scales.cpu().numpy(), fmt) for x in (cp.k_out, cp.v_out))

    got = cached()
    for l in range(layers):
        for s in range(S):
            kept = cp.kept(l, s) + cu[s]
            assert len(kept) == budget[l, s]
            at = begin[l, s] + np.arange(len(kept))
            for g, x in zip(got, (k64, v64)):
                y, scale, _ = C.quotients(x[l, kept], fmt)
                assert (np.abs(g[l, at] - x[l, kept]) <= (0.51 if fmt != C.E4M3 else 16.5) * scale + 1e-6).all()
    # a tree of drafted tokens for each sequence
    bits, sees = TL.tree_bits(5, draft, 1)
    n = sum(draft)
    cn = np.concatenate([[0], np.cumsum(draft)])
    qn, kn, vn = (TL.normal(310 + i, (layers, n, h, D), "bf16") for i, h in enumerate((Hq, Hkv, Hkv)))
    # the problem gives the rows of a layer and the longest sequence; who owns which rows the arrays say
    cache_prob = B.Problem(layers, Hq, Hkv, D, [cp.k_out.codes.shape[1]] + [0] * (S - 1))
    out = torch.empty_like(qn)
    lse = torch.empty((layers, Hq, n), dtype=torch.float32, device="cuda:0")
    B.kvcrush_attend(cache_prob, B.NewTokens(draft, mask=_dev(bits)), qn, cp.k_out, cp.v_out, out, k_new=kn, v_new=vn, lse=lse,
                     row_begin=cp.row_begin, row_count=cp.row_count, status=cp.status)
    kn64, vn64 = TL.numpy64(kn), TL.numpy64(vn)

    def rows_of(l, s, i, h):
        at, new = begin[l, s] + np.arange(budget[l, s]), cn[s] + np.flatnonzero(sees[s][i])
        return np.concatenate([got[0][l, at, h], kn64[l, new, h]]), np.concatenate([got[1][l, at, h], vn64[l, new, h]])

    _check(out, lse, TL.numpy64(qn), layers, cn, draft, Hq, Hkv, D, rows_of)
    # the accepted path of each tree is appended, and a next token attends to everything, itself included
    path = [np.flatnonzero(m[-1]) for m in sees]
    accepted = [len(p) for p in path]
    new_prob = B.Problem(layers, Hq, Hkv, D, draft)
    cu_acc = np.concatenate([[0], np.cumsum(np.tile(accepted, layers))]).astype(np.int32)
    idx = np.tile(np.concatenate(path), layers).astype(np.int32)
    ends = cp.row_begin + cp.row_count
    B.kvcrush_quantize(new_prob, kn, vn, cp.k_out, cp.v_out, cu_kept=_dev(cu_acc), idx=_dev(idx), total_kept=int(cu_acc[-1]),
                       out_begin=ends, status=cp.status)
    count = cp.row_count + _dev(np.asarray([accepted] * layers, dtype=np.int32))
    q1 = TL.normal(320, (layers, S, Hq, D), "bf16")
    out1, lse1 = torch.empty_like(q1), torch.empty((layers, Hq, S), dtype=torch.float32, device="cuda:0")
    B.kvcrush_attend(cache_prob, B.NewTokens([1] * S), q1, cp.k_out, cp.v_out, out1, lse=lse1, row_begin=cp.row_begin,
                     row_count=count, status=cp.status)
    now = cached()
    c1 = count.cpu().numpy()
    _check(out1, lse1, TL.numpy64(q1), layers, np.arange(S + 1), [1] * S, Hq, Hkv, D,
           lambda l, s, i, h: tuple(x[l, begin[l, s] + np.arange(c1[l, s]), h] for x in now))
    # and the kept rows read back
    back = torch.empty((layers, 4, Hkv, D), dtype=torch.float32, device="cuda:0")
    B.kvcrush_dequantize(B.Problem(layers, Hq, Hkv, D, [2, 2]), cp.k_out, None, back, None, in_begin=cp.row_begin, status=cp.status)
    want = np.stack([now[0][l, [begin[l, 0], begin[l, 0] + 1, begin[l, 1], begin[l, 1] + 1]] for l in range(layers)])
    assert np.allclose(TL.numpy64(back), want, rtol=2.0 ** -22, atol=2.0 ** -22 * np.abs(want).max())
    cp.check_status()


def test_pages_of_a_growing_cache(B):
    """Token after token: the last page's bounds follow the cache, and a token reads the pages that look best to it."""
    import torch
    Hq, Hkv, D, page, budget, room = 8, 2, 64, 16, 5, 300
    k, v = TL.normal(330, (1, room, Hkv, D), "bf16"), TL.normal(331, (1, room, Hkv, D), "bf16")
    prob = B.Problem(1, Hq, Hkv, D, [room])
    lo, hi = (torch.zeros((1, -(-room // page), Hkv, D), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    begin = _dev(np.zeros((1, 1), dtype=np.int32))
    L0 = 190
    B.kvcrush_page_bounds(prob, k, page, lo, hi, row_begin=begin, row_count=_dev(np.asarray([[L0]], dtype=np.int32)), status=status)
    k64, v64 = TL.numpy64(k), TL.numpy64(v)
    for L in range(L0 + 1, L0 + 20):
        count = _dev(np.asarray([[L]], dtype=np.int32))
        q = TL.normal(332 + L, (1, 1, Hq, D), "bf16")
        out, lse = torch.empty_like(q), torch.empty((1, Hq, 1), dtype=torch.float32, device="cuda:0")
        idx = torch.empty((1, 1, Hkv, budget), dtype=torch.int32, device="cuda:0")
        B.kvcrush_page_bounds(prob, k, page, lo, hi, recent_pages=1, row_begin=begin, row_count=count, status=status)
        B.kvcrush_attend_pages(prob, B.NewTokens([1]), q, k, v, page, lo, hi, budget, out, keep_initial=1, keep_recent=1,
                               page_idx=idx, lse=lse, row_begin=begin, row_count=count, status=status)
        q64, idx = TL.numpy64(q), idx.cpu().numpy()

        def rows_of(l, s, i, h):
            a, b = C.page_bounds(k64[0, :L, h], page)
            chosen = C.choose_pages(C.page_scores(q64[0, 0, h * 4:h * 4 + 4], a, b), budget, 1, 1)
            assert idx[0, 0, h].tolist() == chosen.tolist()
            rows = (chosen[:, None] * page + np.arange(page)).reshape(-1)
            return k64[0, rows[rows < L], h], v64[0, rows[rows < L], h]

        _check(out, lse, q64, 1, [0], [1], Hq, Hkv, D, rows_of)
    assert status.cpu().tolist()[0] == 0


def test_captured_loop_step_follows_the_counts(B):
    """One step (append, attend) captured once and replayed while the counts on the device grow."""
    import torch
    layers, Hq, Hkv, D, room, L0 = 2, 4, 2, 64, 64, 20
    kq, vq = (B.QuantTensor.empty(layers, room, Hkv, D, C.INT8) for _ in range(2))
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    k, v = TL.normal(340, (layers, L0, Hkv, D), "bf16"), TL.normal(341, (layers, L0, Hkv, D), "bf16")
    B.kvcrush_quantize(B.Problem(layers, Hq, Hkv, D, [L0]), k, v, kq, vq, status=status)
    prob, one, new = B.Problem(layers, Hq, Hkv, D, [room]), B.Problem(layers, Hq, Hkv, D, [1]), B.NewTokens([1])
    kn, vn, q = (TL.normal(342 + i, (layers, 1, h, D), "bf16") for i, h in enumerate((Hkv, Hkv, Hq)))
    begin = torch.zeros((layers, 1), dtype=torch.int32, device="cuda:0")
    count = torch.full((layers, 1), L0, dtype=torch.int32, device="cuda:0")
    out, lse = torch.empty_like(q), torch.empty((layers, Hq, 1), dtype=torch.float32, device="cuda:0")

    def step():
        B.kvcrush_quantize(one, kn, vn, kq, vq, out_begin=count, status=status)
        count.add_(1)
        B.kvcrush_attend(prob, new, q, kq, vq, out, lse=lse, row_begin=begin, row_count=count, status=status)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        for j, (t, h) in enumerate(((kn, Hkv), (vn, Hkv), (q, Hq))):
            t.copy_(TL.normal(350 + 3 * i + j, (layers, 1, h, D), "bf16"))
        g.replay()
        torch.cuda.synchronize()
        n = L0 + 2 + i
        assert count.cpu().tolist() == [[n]] * layers
        now = [C.decode(x.codes.cpu().numpy(), x.scales.cpu().numpy(), C.INT8) for x in (kq, vq)]
        _check(out, lse, TL.numpy64(q), layers, [0], [1], Hq, Hkv, D, lambda l, s, i, h: tuple(x[l, :n, h] for x in now))
    assert status.cpu().tolist()[0] == 0


def test_a_quantised_cache_is_refused_where_it_cannot_be(B):
    prob = B.Problem(1, 2, 2, 32, [40])
    with pytest.raises(ValueError):
        B.CompressionPass(prob, np.asarray([[2]]), np.asarray([[2]]), cache_format=B.INT8, page_size=8)
    with pytest.raises(ValueError):
        B.CompressionPass(prob, np.asarray([[8]]), np.asarray([[8]]), spare_rows=4)
