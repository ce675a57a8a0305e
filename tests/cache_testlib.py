"""Shared helpers of the tests of quantised caches and of the attention over them: inputs, the oracle row by row, and the
bound that a float32 computation keeps to."""
import numpy as np

from oracle import cache_oracle as C

UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}      # half a step, relative


def torch_dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


def normal(seed, shape, dtype, device="cuda:0"):
    """Normal values of the given type on the device."""
    import torch
    g = np.random.Generator(np.random.Philox(seed))
    return torch.from_numpy(g.standard_normal(shape).astype(np.float32)).to(device).to(torch_dtype(dtype))


def numpy64(t):
    return t.double().cpu().numpy()


def strided(t, pad_heads=1, pad_tokens=3):
    """The same values [layers, tokens, heads, D] in a larger allocation: other strides, rows around them hold NaN."""
    import torch
    l, n, h, d = t.shape
    fill = float("nan") if t.is_floating_point() else 0xFF
    big = torch.full((l, n + pad_tokens, h + pad_heads, d), fill, dtype=t.dtype, device=t.device)
    big[:, :n, :h] = t
    return big[:, :n, :h]


def by_head(t):
    """The same values with the rows of a head side by side: [layers][heads][tokens][D] in memory."""
    return t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)


def quantise(B, x, fmt):
    """(QuantTensor, float64 values) of x [layers, rows, heads, D] by the library."""
    import torch
    layers, rows, heads, D = x.shape
    q = B.QuantTensor.empty(layers, rows, heads, D, fmt, device=x.device)
    prob = B.Problem(layers, heads, heads, D, [rows], device=x.device)
    st = torch.zeros(4, dtype=torch.int32, device=x.device)
    B.kvcrush_quantize(prob, x, None, q, None, status=st)
    return q, C.decode(q.codes.cpu().numpy(), q.scales.cpu().numpy(), fmt)


def check_rows(got, got_lse, rows, dtype, D):
    """got [n, D], got_lse [n] against oracle rows (q, k, v, scale) of float64 arrays.

    Error of a float32 evaluation, relative to sum p |v|: a weight rounded to the 16-bit type (half a step; once more for the
    types whose weights are scaled first), twice the error of a logit (D products and sums, each half a step of float32,
    of at most sum |q k|, and its product with the scale), a half step for every key added; an exponential is good to a few
    2^-23.  The output is rounded once more.  A log-sum-exp takes the logit's error and the sum's."""
    for i, (q, k, v, scale) in enumerate(rows):
        o, lse, size, dot = C.attend_row(q, k, v, scale)
        weight = UNIT[dtype] if dtype != "fp32" else 0.0
        if not np.isfinite(dot):                        # a key that is not finite: the whole row follows the definition
            assert np.array_equal(np.isnan(got[i]), np.isnan(o)) and (np.isnan(got_lse[i]) == np.isnan(lse)), i
            continue
        logit = (D + 4) * 2.0 ** -24 * dot
        rel = weight + 2 * logit + (len(k) + 16) * 2.0 ** -24 + 2.0 ** -20
        fine = np.isfinite(o)                           # a value that is not finite reaches its own channel only
        assert np.array_equal(np.isnan(got[i]), np.isnan(o)) and np.array_equal(got[i][np.isinf(o)], o[np.isinf(o)]), i
        tol = (rel * size + UNIT[dtype] * (np.abs(o) + rel * size) + (2.0 ** -25 if dtype == "fp16" else 1e-37))[fine]
        off = np.abs(got[i][fine] - o[fine])
        assert (off <= tol).all(), (i, float(np.max(off / tol)))
        if lse == -np.inf:
            assert got_lse[i] == lse, i
        else:
            assert abs(got_lse[i] - lse) <= logit + (len(k) + 16) * 2.0 ** -24 + 2.0 ** -20 + abs(lse) * 2.0 ** -22, (i, got_lse[i], lse)


def tree_bits(seed, counts, words, empty_row=False):
    """Random trees: mask words [total, words] (int32) and the list of bool matrices [n, n]."""
    g = np.random.Generator(np.random.Philox(seed))
    sees, bits = [], []
    for n in counts:
        m = np.zeros((n, n), dtype=bool)
        for i in range(n):
            if i:
                m[i] = m[g.integers(0, i)]
            m[i, i] = True
        if empty_row and n > 2:
            m[n // 2] = False
        b = np.zeros((n, words * 32), dtype=np.uint64)
        b[:, :n] = m
        b[:, n:] = 1                                   # bits behind the sequence's tokens are ignored
        bits.append((b.reshape(n, words, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32))
        sees.append(m)
    return np.concatenate(bits) if bits else np.zeros((0, words), np.int32), sees
