"""Quantised caches: codes, scales and zeros that are not numbers, in rows that a token does not see, stay out of its output and
reach the tokens that see them."""
import numpy as np
import pytest

from oracle import cache_oracle as C
import cache_testlib as TL

pytestmark = pytest.mark.gpu

FORMATS = [C.INT8, C.E4M3, C.INT4]


@pytest.fixture(scope="module")
def B():
    from paper_2503_00022_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


class Call:
    def __init__(self, B, dtype, fmt, D, Hq, Hkv, rows, counts, layers=1, own=False, seed=0):
        import torch
        self.dtype, self.fmt, self.D, self.G, self.counts, self.layers = dtype, fmt, D, Hq // Hkv, counts, layers
        n = sum(counts)
        self.k, self.v = (TL.quantise(B, TL.normal(seed + i, (layers, rows, Hkv, D), dtype), fmt)[0] for i in (1, 2))
        self.q = TL.normal(seed + 3, (layers, n, Hq, D), dtype)
        self.kn, self.vn = (TL.normal(seed + i, (layers, n, Hkv, D), dtype) if own else None for i in (4, 5))
        self.out, self.lse = torch.full_like(self.q, 7.0), torch.full((layers, Hq, n), 7.0, dtype=torch.float32, device="cuda:0")
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda:0")

    def run(self, B, prob, new, **more):
        B.kvcrush_attend(prob, new, self.q, self.k, self.v, self.out, k_new=self.kn, v_new=self.vn, lse=self.lse, status=self.status,
                         **more)

    def check(self, visible):
        """visible(layer, s, i): rows of the cache and new tokens (packed numbers) that token i of sequence s sees."""
        k64, v64 = (C.decode(x.codes.cpu().numpy(), x.scales.cpu().numpy(), self.fmt) for x in (self.k, self.v))
        q64, out, lse = TL.numpy64(self.q), TL.numpy64(self.out), self.lse.double().cpu().numpy()
        kn, vn = (TL.numpy64(x) if x is not None else None for x in (self.kn, self.vn))
        for l in range(self.layers):
            t = 0
            for s, n in enumerate(self.counts):
                for i in range(n):
                    rows, new = visible(l, s, i)
                    for h in range(k64.shape[2]):
                        k, v = k64[l, rows, h], v64[l, rows, h]
                        if len(new):
                            k, v = np.concatenate([k, kn[l, new, h]]), np.concatenate([v, vn[l, new, h]])
                        heads = range(h * self.G, (h + 1) * self.G)
                        TL.check_rows([out[l, t, x] for x in heads], [lse[l, x, t] for x in heads],
                                      [(q64[l, t, x], k, v, 1.0 / np.sqrt(self.D)) for x in heads], self.dtype, self.D)
                    t += 1
        assert self.status.cpu().tolist()[0] == 0


def _spoil(cache, fmt, layer, rows, value):
    """Rows whose scale (INT4: and zero) is `value`, with codes of all ones: NaN for E4M3."""
    cache.codes[layer, rows] = 0xFF
    cache.scales[layer, rows] = value


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,G,n", [("bf16", 2, 3), ("fp16", 4, 9), ("fp32", 2, 4)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_rows_of_later_tokens(B, fmt, dtype, G, n, value):
    """The last rows of the cache are the new tokens' own: the last one's is spoiled, in keys or in values, and so are the rows
    behind the sequence.  Only the last token sees it; with a NaN there its output is NaN, so that it is left out where the
    value is infinite (0 times infinity among its products)."""
    L = 70
    for spoil in "kv":
        c = Call(B, dtype, fmt, 64, 2 * G, 2, L + 40, (n,), seed=500 + n)
        for x in (c.k, c.v):
            _spoil(x, fmt, 0, slice(L, L + 40), value)
        _spoil(getattr(c, spoil), fmt, 0, L - 1, value)
        prob = B.Problem(1, 2 * G, 2, 64, [L, 40])
        new = B.NewTokens((n, 0))
        c.run(B, prob, new)
        if value != value:
            with np.errstate(invalid="ignore"):
                c.check(lambda l, s, i: (np.arange(L - n + 1 + i), []))
        else:
            c.counts, c.q, c.out, c.lse = (n - 1,), c.q[:, :n - 1], c.out[:, :n - 1], c.lse[:, :, :n - 1]
            c.check(lambda l, s, i: (np.arange(L - n + 1 + i), []))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,own", [("bf16", False), ("fp16", True), ("fp32", True)])
def test_rows_behind_the_counts(B, fmt, dtype, own):
    """Caches with room behind their sequences, whose codes and scales are what the memory held."""
    layers, total, counts = 2, 300, (1, 2)
    begin = np.asarray([[0, 130], [200, 5]], dtype=np.int32)
    count = np.asarray([[101, 20], [0, 64]], dtype=np.int32)
    c = Call(B, dtype, fmt, 128, 4, 2, total, counts, layers=layers, own=own, seed=520)
    for l in range(layers):
        held = np.zeros(total, dtype=bool)
        for s in range(2):
            held[begin[l, s]:begin[l, s] + count[l, s]] = True
        for j, r in enumerate(np.flatnonzero(~held)):
            for x in (c.k, c.v):
                _spoil(x, fmt, l, int(r), (float("nan"), float("inf"), -float("inf"))[j % 3])
    prob = B.Problem(layers, 4, 2, 128, [total, 0])
    c.run(B, prob, B.NewTokens(counts), row_begin=_dev(begin), row_count=_dev(count))
    base = (0, 1)
    c.check(lambda l, s, i: (begin[l, s] + np.arange(count[l, s] if own else max(0, count[l, s] - counts[s] + 1 + i)),
                             base[s] + np.arange(i + 1) if own else []))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,n", [("bf16", 11), ("fp16", 40), ("fp32", 6)])
def test_drafted_tokens_beside_a_quantised_cache(B, fmt, dtype, n):
    """NaN and infinities in keys and values of drafted tokens that a token does not see."""
    L = 37
    bits, sees = TL.tree_bits(79, (n,), (n + 31) // 32, empty_row=True)
    c = Call(B, dtype, fmt, 96, 4, 2, L, (n,), own=True, seed=540)
    c.vn[0, 2, :, 3] = float("nan")
    c.kn[0, n - 2, 0, 0] = float("nan")
    c.vn[0, n - 1, 1] = float("inf")
    c.run(B, B.Problem(1, 4, 2, 96, [L]), B.NewTokens((n,), mask=_dev(bits)))
    with np.errstate(invalid="ignore"):
        c.check(lambda l, s, i: (np.arange(L), np.flatnonzero(sees[0][i])))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages_that_are_not_read(B, fmt, dtype):
    """Chosen pages of a quantised cache: codes and scales of the others, and of the rows behind the sequence, may be anything."""
    import torch
    L, page, D = 83, 8, 64
    c = Call(B, dtype, fmt, D, 4, 2, L + 30, (1,), seed=560)
    for x in (c.k, c.v):
        _spoil(x, fmt, 0, slice(L, L + 30), float("nan"))
        _spoil(x, fmt, 0, slice(16, 40), float("inf"))
    prob = B.Problem(1, 4, 2, D, [L, 30])
    lo, hi = (torch.zeros((1, 2 * 11, 2, D), dtype=c.q.dtype, device="cuda:0") for _ in range(2))
    lo[0, 2:5], hi[0, 2:5] = -9.0, -9.0                  # pages 2, 3, 4 promise nothing to positive queries
    c.q.abs_()
    idx = torch.full((1, 1, 2, 8), -7, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend_pages(prob, B.NewTokens((1, 0)), c.q, c.k, c.v, page, lo, hi, 8, c.out, page_idx=idx, lse=c.lse, status=c.status)
    assert idx[0, 0].cpu().tolist() == [[0, 1, 5, 6, 7, 8, 9, 10]] * 2
    c.check(lambda l, s, i: (np.concatenate([np.arange(16), np.arange(40, L)]), []))
