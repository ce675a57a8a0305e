"""GPU parity of the quantised cache: codes, scales and read-back values against the float64 definition, gathers and appends,
rows that cannot be quantised, and what is left alone."""
import numpy as np
import pytest

from oracle import cache_oracle as C
import cache_testlib as TL

pytestmark = pytest.mark.gpu

FORMATS = (C.INT8, C.E4M3, C.INT4)


@pytest.fixture(scope="module")
def B():
    from paper_2503_00022_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _status(dev="cuda:0"):
    import torch
    return torch.zeros(4, dtype=torch.int32, device=dev)


def _check_codes(codes, scales, x, fmt, dtype):
    """codes and scales of rows x (float64): the scale is off by two roundings at most, a code by half a step of the format;
    rows of 16-bit values, whose quotients are exact to float32, get exactly the rounded quotient."""
    y, scale, zero = C.quotients(x, fmt)
    s = scales[..., 0] if fmt == C.INT4 else scales
    assert (np.abs(s - scale[..., 0]) <= 2.0 ** -22 * scale[..., 0]).all()
    if fmt == C.INT4:
        assert np.array_equal(scales[..., 1], zero[..., 0].astype(np.float32))
    got = C.decode(codes, np.stack([np.ones_like(s), np.zeros_like(s)], -1) if fmt == C.INT4 else np.ones_like(s), fmt)
    want = C.round_e4m3(y) if fmt == C.E4M3 else np.rint(y)
    if dtype != "fp32":
        assert np.array_equal(got, want)
    else:                                               # quotients that lie within 2^-20 of a border may fall on either side
        near = np.abs(np.abs(y - got) - np.abs(y - want)) <= 2.0 ** -20 * (1 + np.abs(y))
        assert ((got == want) | near).all()
    return got * scale + zero


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,heads,rows", [(128, 8, 37), (64, 3, 5), (96, 1, 1), (32, 33, 9), (256, 2, 20), (160, 5, 11)])
def test_codes_scales_and_values_match_the_definition(B, dtype, fmt, D, heads, rows):
    import torch
    x = TL.normal(7 + D, (2, rows, heads, D), dtype)
    x[0, 0, 0] = 0
    v = TL.strided(TL.normal(8 + D, (2, rows, heads, D), dtype) * 40)
    prob = B.Problem(2, heads, heads, D, [rows], device="cuda:0")
    kq, vq = (B.QuantTensor.empty(2, rows, heads, D, fmt) for _ in range(2))
    st = _status()
    B.kvcrush_quantize(prob, x, v, kq, vq, status=st)
    back = torch.full((2, 2, rows + 1, heads, D), 9.0, dtype=x.dtype, device="cuda:0")
    B.kvcrush_dequantize(prob, kq, vq, back[0], back[1], status=st)
    assert st.cpu().tolist()[0] == 0
    for given, q, b in ((x, kq, back[0]), (v, vq, back[1])):
        codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
        _check_codes(codes, scales, TL.numpy64(given), fmt, dtype)
        want = C.decode(codes, scales, fmt)
        # float32 product (and sum) and the rounding to the type
        big = np.abs(want) + (np.abs(scales[..., 1:].astype(np.float64)) if fmt == C.INT4 else 0)
        tol = TL.UNIT[dtype] * np.abs(want) * (1 + 2.0 ** -20) + 2.0 ** -23 * big + (2.0 ** -25 if dtype == "fp16" else 0)
        assert (np.abs(TL.numpy64(b)[:, :rows] - want) <= tol).all()
        assert (TL.numpy64(b)[:, rows:] == 9).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_at_the_ends_of_the_range(B, fmt, dtype):
    """Infinities and NaN make a row NaN and leave the others alone; the largest and the smallest numbers quantise; scales below
    the smallest normal number count as zero."""
    import torch
    D, big = 64, 3.0e38
    x = TL.normal(3, (1, 8, 1, D), dtype)
    x[0, 0, 0, 5] = float("inf")
    x[0, 1, 0, 9] = float("nan")
    x[0, 2, 0, 63] = -float("inf")
    x[0, 3] *= 1e37
    x[0, 4] *= 1e-30
    x[0, 5] = 1e-38
    x[0, 6] *= 0
    x[0, 7] = torch.where(x[0, 7] > 0, big, -big)       # INT4: the span overflows
    prob = B.Problem(1, 1, 1, D, [8], device="cuda:0")
    q = B.QuantTensor.empty(1, 8, 1, D, fmt)
    st = _status()
    B.kvcrush_quantize(prob, x, None, q, None, status=st)
    back = torch.zeros((1, 8, 1, D), dtype=torch.float32, device="cuda:0")
    B.kvcrush_dequantize(prob, q, None, back, None, status=st)
    codes, scales, got = q.codes.cpu().numpy()[0, :, 0], q.scales.cpu().numpy()[0, :, 0], TL.numpy64(back)[0, :, 0]
    lost = [0, 1, 2] + ([7] if fmt == C.INT4 else [])
    for r in range(8):
        assert np.isnan(got[r]).all() == (r in lost), r
        if r in lost:
            assert np.isnan(scales[r]).all() and (codes[r] == 0).all()
    x64 = TL.numpy64(x)[0, :, 0]
    for r in (3, 4):
        _check_codes(codes[r:r + 1], scales[r:r + 1], x64[r:r + 1], fmt, "fp32")
    assert (codes[5:7] == 0).all() and (scales[5:7, 0] == 0).all() if fmt == C.INT4 else (codes[5:7] == 0).all() and (scales[5:7] == 0).all()
    if fmt != C.INT4:
        assert np.abs(got[7] - x64[7]).max() <= 2.0 ** -20 * big
        assert (got[5] == 0).all()
    else:
        assert (got[5] == x64[5]).all()                 # the row's zero is the value itself


@pytest.mark.parametrize("fmt", FORMATS)
def test_kept_rows_appends_and_rows_left_alone(B, fmt):
    """Kept rows land behind each other like kvcrush_compact's, appended rows at given places; total_kept may be larger than the
    list; no other row of the cache changes; any part is read back."""
    import torch
    layers, heads, D, lens = 3, 4, 64, [50, 0, 33]
    S, T = len(lens), sum(lens)
    g = np.random.Generator(np.random.Philox(11))
    k, v = TL.normal(1, (layers, T, heads, D), "bf16"), TL.normal(2, (layers, T, heads, D), "bf16")
    kept = [[np.sort(g.permutation(n)[:g.integers(0, n + 1)]) for n in lens] for _ in range(layers)]
    counts = np.asarray([[len(x) for x in row] for row in kept])
    cu = np.concatenate([[0], np.cumsum(counts.reshape(-1))]).astype(np.int32)
    idx = np.concatenate([x for row in kept for x in row]).astype(np.int32)
    prob = B.Problem(layers, heads, heads, D, lens, device="cuda:0")
    rows = int(counts.sum(1).max()) + 4
    kq, vq = (B.QuantTensor.empty(layers, rows, heads, D, fmt) for _ in range(2))
    for q in (kq, vq):
        q.codes.fill_(77)
        q.scales.fill_(-5.0)
    st = _status()
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")   # noqa: E731
    B.kvcrush_quantize(prob, k, v, kq, vq, cu_kept=d(cu), idx=d(idx), total_kept=int(cu[-1]) + 100, status=st)
    for x, q in ((k, kq), (v, vq)):
        codes, scales, x64 = q.codes.cpu().numpy(), q.scales.cpu().numpy(), TL.numpy64(x)
        for l in range(layers):
            source = np.concatenate([np.asarray(kept[l][s]) + sum(lens[:s]) for s in range(S)]).astype(int)
            n = len(source)
            _check_codes(codes[l, :n], scales[l, :n], x64[l, source], fmt, "bf16")
            assert (codes[l, n:] == 77).all() and (scales[l, n:] == -5).all()
    # two new tokens of the first sequence and one of the third go behind row 2 of their layer's part
    new = TL.normal(3, (layers, 3, heads, D), "bf16")
    begin = np.asarray([[rows - 4, 0, rows - 1]] * layers, dtype=np.int32)
    before = kq.codes.clone()
    pn = B.Problem(layers, heads, heads, D, [2, 0, 1], device="cuda:0")
    B.kvcrush_quantize(pn, new, None, kq, None, out_begin=d(begin), status=st)
    at = [rows - 4, rows - 3, rows - 1]
    codes, scales = kq.codes.cpu().numpy(), kq.scales.cpu().numpy()
    _check_codes(codes[:, at], scales[:, at], TL.numpy64(new), fmt, "bf16")
    others = [r for r in range(rows) if r not in at]
    assert np.array_equal(codes[:, others], before.cpu().numpy()[:, others])
    # read back: rows by number, and the appended ones
    back = torch.full((layers, 5, heads, D), 3.0, dtype=torch.float32, device="cuda:0")
    pick, cu2 = np.asarray([rows - 4, 0, rows - 1] * layers, dtype=np.int32), np.asarray([0, 2, 2, 3, 5, 5, 6, 8, 8, 9], dtype=np.int32)
    zero = d(np.zeros((layers, S), dtype=np.int32))
    B.kvcrush_dequantize(prob, kq, None, back, None, cu_kept=d(cu2), idx=d(pick), total_kept=9, in_begin=zero, status=st)
    want = C.decode(codes, scales, fmt)[:, [rows - 4, 0, rows - 1]]
    assert np.allclose(TL.numpy64(back)[:, :3], want, rtol=2.0 ** -22, atol=2.0 ** -22 * np.abs(want).max())
    assert (TL.numpy64(back)[:, 3:] == 3).all()
    back.fill_(3.0)
    B.kvcrush_dequantize(pn, kq, None, back, None, in_begin=d(begin), status=st)
    want = C.decode(codes, scales, fmt)[:, at]
    assert np.allclose(TL.numpy64(back)[:, :3], want, rtol=2.0 ** -22, atol=2.0 ** -22 * np.abs(want).max())
    assert st.cpu().tolist()[0] == 0


def test_an_empty_list_is_a_call(B):
    import torch
    prob = B.Problem(1, 2, 2, 32, [0], device="cuda:0")
    x = torch.zeros((1, 1, 2, 32), dtype=torch.bfloat16, device="cuda:0")
    q = B.QuantTensor.empty(1, 1, 2, 32, C.INT8)
    q.codes.fill_(5)
    B.kvcrush_quantize(prob, x, None, q, None, status=_status())
    cu = torch.zeros(2, dtype=torch.int32, device="cuda:0")
    B.kvcrush_quantize(prob, x, None, q, None, cu_kept=cu, idx=cu, total_kept=0, status=_status())
    B.kvcrush_quantize(prob, x, None, q, None, cu_kept=cu, idx=cu, total_kept=64, status=_status())
    assert (q.codes == 5).all()
