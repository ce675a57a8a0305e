"""The largest steps from one token of a cache to the next: less than 2^31 bytes are taken, in bytes of the cache's own type."""
import ctypes
import math

import numpy as np
import pytest

from oracle import cache_oracle as C
import cache_testlib as TL
from paper_2503_00022_b200 import binding as B
from paper_2503_00022_b200 import build as kbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


@pytest.mark.parametrize("dtype,code,limit", [(B.BF16, None, 1 << 30), (B.FP32, None, 1 << 29), (B.BF16, B.INT8, 1 << 31), (B.FP32, B.E4M3, 1 << 31),
                                              (B.FP16, B.INT4, 1 << 32)])
@pytest.mark.parametrize("far", [0, 64, 1 << 40, 1 << 61])
def test_longer_steps_are_refused(dtype, code, limit, far):
    """On the host: steps of 2^31 bytes and more, also those whose bytes do not fit 64 bits."""
    cu, cn = np.asarray([0, 100], dtype=np.int32), np.asarray([0, 2], dtype=np.int32)
    p = B.ProblemStruct(1, 1, 8, 4, 64, 100, 100, 1, 0.0, 0, cu.ctypes.data, 0x1000)
    n = B.NewTokensStruct(2, 2, 0, 0, cn.ctypes.data, 0x1000, None)
    r = ctypes.byref
    near = lambda t: B.TensorStruct(0x10000, t, 0, 1 << 40, 256, 64)             # noqa: E731
    long_ = lambda t: B.TensorStruct(0x10000, t, 0, 1 << 40, limit + far, 64)    # noqa: E731
    s = B.ScalesStruct(0x20000, 800, 2, 200)
    sc = None if code is None else r(s)
    kt = dtype if code is None else code

    def attend(k, v, k_scales=sc, kn=None, vn=None):
        return B.lib().kvcrush_attend(r(p), r(n), r(near(dtype)), r(k), k_scales, r(v), sc, kn, vn, None, None, r(near(dtype)), None, 0x100, None)

    assert attend(long_(kt), near(kt)) == B.ERR_UNSUPPORTED and attend(near(kt), long_(kt)) == B.ERR_UNSUPPORTED
    if code is not None:
        assert attend(near(kt), near(kt), k_scales=r(B.ScalesStruct(0x20000, 800, (1 << 29) + far, 200))) == B.ERR_UNSUPPORTED
    else:
        assert attend(near(kt), near(kt), kn=r(long_(dtype)), vn=r(near(dtype))) == B.ERR_UNSUPPORTED
        assert attend(near(kt), near(kt), kn=r(near(dtype)), vn=r(long_(dtype))) == B.ERR_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fmt,step", [("bf16", C.INT8, (1 << 31) - 64), ("fp32", C.E4M3, 5 << 28), ("fp16", C.INT4, 5 << 28), ("bf16", None, (1 << 31) - 128)])
def test_the_longest_steps_that_are_taken(dtype, fmt, step):
    """Two rows of a cache `step` bytes apart."""
    import torch
    D = 64
    k, v = (TL.normal(900 + i, (1, 2, 1, D), dtype) for i in range(2))
    k64, v64 = TL.numpy64(k), TL.numpy64(v)
    if fmt is not None:
        (k, k64), (v, v64) = TL.quantise(B, k, fmt), TL.quantise(B, v, fmt)

    def spread(t):
        n, width = step // t.element_size(), t.shape[3]
        view = torch.empty(n + width, dtype=t.dtype, device="cuda:0").as_strided((1, 2, 1, width), (n, n, width, 1))
        view.copy_(t)
        return view

    k, v = (B.QuantTensor(spread(x.codes), x.scales, fmt) if fmt is not None else spread(x) for x in (k, v))
    q = TL.normal(910, (1, 1, 2, D), dtype)
    out, lse = torch.empty_like(q), torch.empty((1, 2, 1), dtype=torch.float32, device="cuda:0")
    status = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    B.kvcrush_attend(B.Problem(1, 2, 1, D, [2]), B.NewTokens([1]), q, k, v, out, lse=lse, status=status)
    q64, out, lse = TL.numpy64(q), TL.numpy64(out), lse.cpu().numpy()
    TL.check_rows(out[0, 0], lse[0, :, 0], [(q64[0, 0, x], k64[0, :, 0], v64[0, :, 0], 1.0 / math.sqrt(D)) for x in range(2)], dtype, D)
    assert status.cpu().tolist()[0] == 0
