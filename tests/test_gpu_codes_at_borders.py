"""Quotients that lie on the border between two codes, and as close beside it as the type allows: the nearest code, ties to even."""
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


def _borders(fmt):
    """Quotients halfway between two codes."""
    if fmt == C.INT8:
        return np.arange(-127, 127) + 0.5
    if fmt == C.INT4:
        return np.arange(0, 15) + 0.5
    v = np.asarray([C.e4m3_value(i) for i in range(127)])
    b = (v[1:] + v[:-1]) / 2
    return np.concatenate([-b, b])


def _rows(dtype, fmt, D):
    """Rows [n, D] of the type: their ends, and values on and next to the borders for several spans and zeros."""
    import torch
    g = np.random.Generator(np.random.Philox(700 + fmt))
    dt = TL.torch_dtype(dtype)
    rows = []
    step = 2.0 * TL.UNIT[dtype]
    for top in [C.TOP[fmt], 1.0, 3.0, 0.7, 1.9990234375, 96.0, 2.0 ** -9] + list(np.exp2(g.uniform(-6, 6, 9))):
        for zero in ([0.0, -1.0, -0.5, 0.25, -3.0] if fmt == C.INT4 else [0.0]):
            ends = torch.tensor([zero * top, zero * top + top], dtype=torch.float64).to(dt).double().numpy()
            span = ends[1] - ends[0] if fmt == C.INT4 else ends[1]
            x = _borders(fmt) * span / C.TOP[fmt] + (ends[0] if fmt == C.INT4 else 0.0)
            x = np.concatenate([x * (1 + s * step) for s in (-2, -1, 0, 1, 2)])
            x = torch.from_numpy(x).to(dt).double().numpy()
            x = x[(x > ends[0]) & (x < ends[1])] if fmt == C.INT4 else x[np.abs(x) < ends[1]]
            n = D - 2
            for i in range(0, len(x), n):
                r = np.full(D, ends[1])
                r[0] = ends[0] if fmt == C.INT4 else -ends[1]
                part = x[i:i + n]
                r[1:1 + len(part)] = part
                rows.append(r)
    if fmt == C.INT4:                                    # a value far below the ends takes the quotient off the border
        for top in (1.0, 15.0, 0.875):
            tiny = [s * 2.0 ** -e for e in range(8, 23 if dtype == "fp16" else 45) for s in (1, -1)]
            for i in range(0, len(tiny), D - 2):
                r = np.full(D, top)
                r[0] = -top
                part = tiny[i:i + D - 2]
                r[1:1 + len(part)] = part
                rows.append(r)
        # an end far below the other: the span itself is not a float32
        for e in range(20, 24 if dtype == "fp16" else 40, 3):
            for s in (1, -1):
                r = np.full(D, 15.0)
                r[0] = s * 2.0 ** -e
                r[1:16] = np.arange(15) + 0.5
                rows.append(r)
    return np.asarray(rows)


@pytest.mark.parametrize("fmt", [C.INT8, C.E4M3, C.INT4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", [32, 96, 128])
def test_the_nearest_code_on_and_beside_borders(B, dtype, fmt, D):
    import torch
    rows = _rows(dtype, fmt, D)
    x = torch.from_numpy(rows).to("cuda:0").to(TL.torch_dtype(dtype)).view(1, -1, 1, D)
    q, _ = TL.quantise(B, x, fmt)
    x64 = TL.numpy64(x)
    assert np.array_equal(x64[0, :, 0], rows)
    y, _, _ = C.quotients(x64, fmt)
    scales = q.scales.cpu().numpy()
    plain = np.stack([np.ones(scales.shape[:3]), np.zeros(scales.shape[:3])], -1) if fmt == C.INT4 else np.ones_like(scales)
    got = C.decode(q.codes.cpu().numpy(), plain, fmt)
    want = C.round_e4m3(y) if fmt == C.E4M3 else np.rint(y)
    # Where the header gives either code: in INT4, rows of 16 bits with an end that is small but not zero, whose quotients are decided to
    # 44.5 half steps of float32 of the span (constants of the border 14.5 + 15, the border itself 15; 2^-18.5); float32 rows, with
    # quotients of four roundings (difference, product and span half a step each, the quotient a step: 2.5 * 2^-23 of their size)
    slack = np.zeros_like(y)
    if dtype == "fp32":
        slack = 2.0 ** -21 * np.abs(y)
    elif fmt == C.INT4:
        ends = np.abs(np.stack([x64.min(-1), x64.max(-1)], -1))
        small = ((ends > 0) & (ends < 2.0 ** -7 * (x64.max(-1) - x64.min(-1))[..., None])).any(-1)
        assert 0 < small.sum() < small.size / 2
        slack = np.where(small[..., None], 2.0 ** -18, 0.0)
    bad = np.argwhere((got != want) & (np.abs(y - (got + want) / 2) > slack))
    assert len(bad) == 0, [(x64[tuple(b)], y[tuple(b)], got[tuple(b)]) for b in bad[:5]]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_four_bit_rows_whose_middle_is_not_quite_the_middle(B, dtype):
    """x - min is not a float32 here: -2^-30 lies just below the border 7.5 of the row from -1 to 1, 2^-30 just above, 0 on it."""
    import torch
    x = torch.zeros((1, 1, 1, 32), dtype=torch.float32, device="cuda:0")
    x[0, 0, 0, :5] = torch.tensor([-1.0, 1.0, -2.0 ** -30, 2.0 ** -30, 0.0])
    q, _ = TL.quantise(B, x.to(TL.torch_dtype(dtype)), C.INT4)
    codes = q.codes.cpu().numpy()[0, 0, 0, :3].tolist()
    if dtype == "fp32":                                  # either code, 2^-30 from the border
        assert codes[0] == 0 | 15 << 4 and codes[1] & 15 in (7, 8) and codes[1] >> 4 in (7, 8) and codes[2] == 8 | 8 << 4
    else:
        assert codes == [0 | 15 << 4, 7 | 8 << 4, 8 | 8 << 4]


@pytest.mark.parametrize("power", [-80, 118])
@pytest.mark.parametrize("fmt", [C.INT8, C.E4M3, C.INT4])
def test_the_same_codes_near_the_ends_of_the_range(B, fmt, power):
    """The rows of the test above in bf16 times a power of two: the quotients, and so the codes, are the same numbers."""
    import torch
    D = 64
    rows = _rows("bf16", fmt, D)
    x = torch.from_numpy(rows * 2.0 ** power).to("cuda:0").to(torch.bfloat16).view(1, -1, 1, D)
    assert np.array_equal(TL.numpy64(x)[0, :, 0], rows * 2.0 ** power)
    got, plain = (TL.quantise(B, t, fmt)[0] for t in (x, torch.from_numpy(rows).to("cuda:0").to(torch.bfloat16).view(1, -1, 1, D)))
    assert torch.equal(got.codes, plain.codes)
    assert np.array_equal(got.scales.double().cpu().numpy(), plain.scales.double().cpu().numpy() * 2.0 ** power)


@pytest.mark.parametrize("fmt", [C.INT8, C.E4M3, C.INT4])
@pytest.mark.parametrize("dtype,most", [("bf16", 255), ("fp16", 2047)])
def test_rows_of_whole_numbers(B, dtype, fmt, most):
    """Whole numbers around a middle, near 0 and far from it: spans of a few units to most of the type's whole numbers, many ties."""
    import torch
    g = np.random.Generator(np.random.Philox(790 + fmt))
    n, D = 4000, 64
    width = np.exp2(g.uniform(0.5, np.log2(most), (n, 1))).astype(int)
    middle = g.integers(-most, most + 1, (n, 1)) * g.integers(0, 2, (n, 1))
    rows = np.clip(middle + g.integers(-width, width + 1, (n, D)), -most, most).astype(np.float64)
    x = torch.from_numpy(rows).to("cuda:0").to(TL.torch_dtype(dtype)).view(1, n, 1, D)
    assert np.array_equal(TL.numpy64(x)[0, :, 0], rows)
    q, _ = TL.quantise(B, x, fmt)
    y = C.quotients(rows, fmt)[0]
    scales = q.scales.cpu().numpy()
    plain = np.stack([np.ones(scales.shape[:3]), np.zeros(scales.shape[:3])], -1) if fmt == C.INT4 else np.ones_like(scales)
    got = C.decode(q.codes.cpu().numpy(), plain, fmt)[0, :, 0]
    want = C.round_e4m3(y) if fmt == C.E4M3 else np.rint(y)
    # ends that are not zero are 2^-7 of the span or more but for the longest rows of float16 (1 beside 4094)
    near = np.zeros((n, 1))
    if fmt == C.INT4:
        ends, span = np.abs(np.stack([rows.min(-1), rows.max(-1)], -1)), rows.max(-1) - rows.min(-1)
        near = np.where(((ends > 0) & (ends < 2.0 ** -7 * span[:, None])).any(-1), 2.0 ** -18, 0.0)[:, None]
        assert (near == 0).mean() > 0.9
    bad = np.argwhere((got != want) & (np.abs(y - (got + want) / 2) > near))
    assert len(bad) == 0, [(rows[b[0]].min(), rows[b[0]].max(), rows[tuple(b)], y[tuple(b)], got[tuple(b)]) for b in bad[:5]]
    if fmt != C.E4M3:
        assert (np.abs(y - np.trunc(y)) == 0.5).sum() > 100
