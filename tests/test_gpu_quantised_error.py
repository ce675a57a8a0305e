"""The error of attention over integer codes, channel by channel: where one key has nearly all the weight and a code that stands for
0, an output is far below the row's scale, and what the arithmetic of the codes leaves behind is counted against that scale."""
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


def _bound(q, k, v, scale, scales, fmt, dtype, D):
    """(output, log-sum-exp, bound of the output's error [D], bound of the log-sum-exp's).

    Weights p (of the softmax), codes c taken less an offset (INT8: 0, INT4: 8, so that a value is its middle plus scale * (c - 8)):
      - p times the row's scale is rounded to half precision: half a step of scale * |c|, or of 2^-24 of the largest such product;
      - codes are multiplied with 128 (INT4: 8) on top, which the sum of the weights takes off again: n / 8 + 16 sums (tiles of 16 keys in two
        halves, warps, blocks) of at most 2 * 128 (8) times the weights and scales, each a step of float32; the same for the INT4 rows' middles;
      - the same for a logit: D + 4 products and sums of |q| times twice the largest |code| (INT4: the middle and the code) times the
        scale, each half a step, then the exponential (2^-20 with the rest);
      - the output is rounded to its type."""
    o, lse, size, dot = C.attend_row(q, k, v, scale)
    x = k @ q * scale
    p = np.exp(x - lse)
    s, top, n = scales["v"][:, 0], 128.0 if fmt == C.INT8 else 8.0, len(k)
    ks = scales["k"]
    # largest sum of |q| |operand| of a logit: codes below 256 and the offset's 128, or codes below 8 and the row's middle
    reach = ks[:, 0] * 384 if fmt == C.INT8 else np.abs(ks[:, 1]) + 24 * ks[:, 0]
    logit = (D + 4) * 2.0 ** -24 * float(reach.max() * np.abs(q).sum() * scale)
    middle = scales["v"][:, 1] + 8 * s if fmt == C.INT4 else 0 * s
    code = np.abs(v - middle[:, None])                                 # times the scale
    total = (p * s).sum()
    err = 2.0 ** -11 * (p @ code) + n * 2.0 ** -25 * top * (p * s).max() + (n / 8 + 16) * 2.0 ** -23 * (2 * top * total + (p * np.abs(middle)).sum())
    err = err + (2 * logit + 2.0 ** -20 + (n + 16) * 2.0 ** -24) * (p @ (code + np.abs(middle)[:, None]))
    return o, lse, err + TL.UNIT[dtype] * (np.abs(o) + err) + (2.0 ** -25 if dtype == "fp16" else 0.0), logit + (n + 16) * 2.0 ** -24 + 2.0 ** -20 + abs(lse) * 2.0 ** -22


@pytest.mark.parametrize("fmt", [C.INT8, C.INT4])
@pytest.mark.parametrize("dtype,D,G,L,n", [("bf16", 128, 4, 60, 1), ("fp16", 64, 2, 300, 1), ("bf16", 96, 1, 33, 12), ("fp16", 256, 3, 130, 5), ("fp16", 128, 7, 2000, 2)])
@pytest.mark.parametrize("gain", [0.5, 3.0])
def test_errors_stay_in_proportion_to_the_scales(B, fmt, dtype, D, G, L, n, gain):
    import torch
    Hkv = 2
    k, v = (TL.normal(950 + i, (1, L, Hkv, D), dtype) for i in range(2))
    v[0, ::3] = torch.where(v[0, ::3].abs() < 0.5, 0.0, v[0, ::3].float()).to(v.dtype)     # many values that are 0
    q = (TL.normal(952, (1, n, Hkv * G, D), dtype) * gain).to(k.dtype)
    (kq, k64), (vq, v64) = TL.quantise(B, k, fmt), TL.quantise(B, v, fmt)
    out, lse = torch.empty_like(q), torch.empty((1, Hkv * G, n), dtype=torch.float32, device="cuda:0")
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend(B.Problem(1, Hkv * G, Hkv, D, [L]), B.NewTokens([n]), q, kq, vq, out, lse=lse, status=status)
    q64, out, lse = TL.numpy64(q), TL.numpy64(out), lse.double().cpu().numpy()
    sc = {name: x.scales.double().cpu().numpy()[0] for name, x in (("k", kq), ("v", vq))}
    for i in range(n):
        rows = np.arange(L - n + 1 + i)
        for h in range(Hkv * G):
            rs = {name: s[rows, h // G].reshape(len(rows), -1) for name, s in sc.items()}
            o, want, tol, tol_lse = _bound(q64[0, i, h], k64[0, rows, h // G], v64[0, rows, h // G], 1.0 / math.sqrt(D), rs, fmt, dtype, D)
            off = np.abs(out[0, i, h] - o)
            assert (off <= tol).all(), (i, h, float((off / tol).max()))
            assert abs(lse[0, h, i] - want) <= tol_lse, (i, h)
    assert status.cpu().tolist()[0] == 0
