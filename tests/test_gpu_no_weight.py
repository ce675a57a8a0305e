"""Tokens all of whose logits are -inf: zeros and a log-sum-exp of -inf, whatever the values hold."""
import math

import numpy as np
import pytest

import cache_testlib as TL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2503_00022_b200 import binding, build
    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype,G,n", [("bf16", 1, 1), ("fp16", 8, 2), ("bf16", 8, 16), ("fp16", 4, 40), ("fp32", 2, 2)])
def test_no_weight_at_all(B, dtype, G, n):
    """The first sequence's logits are -inf throughout and its values hold an infinity and a NaN; the second is an ordinary one."""
    import torch
    D, lens = 64, (300, 200)
    k, v = (TL.normal(600 + i, (1, sum(lens), 1, D), dtype) for i in range(2))
    q = TL.normal(602, (1, 2 * n, G, D), dtype)
    q[0, :n] = 1.0
    k[0, :300] = 0.0
    k[0, :300, :, 0] = float("-inf")
    v[0, 20, 0, 5], v[0, 290, 0, 9] = float("inf"), float("nan")
    out, lse = torch.full_like(q, 7.0), torch.full((1, G, 2 * n), 7.0, dtype=torch.float32, device="cuda:0")
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend(B.Problem(1, G, 1, D, lens), B.NewTokens((n, n)), q, k, v, out, lse=lse, status=status)
    assert (out[0, :n] == 0).all() and torch.isneginf(lse[0, :, :n]).all()
    q64, k64, v64, out, lse = TL.numpy64(q), TL.numpy64(k), TL.numpy64(v), TL.numpy64(out), lse.cpu().numpy()
    for i in range(n):
        rows = 300 + np.arange(200 - n + 1 + i)
        TL.check_rows([out[0, n + i, x] for x in range(G)], [lse[0, x, n + i] for x in range(G)],
                      [(q64[0, n + i, x], k64[0, rows, 0], v64[0, rows, 0], 1.0 / math.sqrt(D)) for x in range(G)], dtype, D)
    assert status.cpu().tolist()[0] == 0
