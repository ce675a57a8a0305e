"""Refusals of the quantised cache's and the attention's entry points: every bad argument is found on the host before anything
is launched (none of these calls touches a GPU)."""
import ctypes

import numpy as np
import pytest

from paper_2503_00022_b200 import binding as B
from paper_2503_00022_b200 import build as kbuild

r = ctypes.byref
INV, UNS, MIS = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_MISALIGNED


@pytest.fixture(scope="module")
def lib():
    kbuild.build()
    return B.lib()


def _problem(cu=(0, 100), D=64, Hq=8, Hkv=4, **over):
    c = np.asarray(cu, dtype=np.int32)
    kw = dict(n_layers=1, n_seqs=len(c) - 1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, total_tokens=int(c[-1]),
              max_seqlen=int(np.diff(c).max()), causal=1, softmax_scale=0.0, query_window=0, cu_seqlens_host=c.ctypes.data,
              cu_seqlens_dev=0x1000)
    kw.update(over)
    p = B.ProblemStruct(**kw)
    p._keep = c
    return p


def _new(cu=(0, 2), mask=None, words=0, **over):
    c = np.asarray(cu, dtype=np.int32)
    kw = dict(total_new=int(c[-1]), max_new=int(np.diff(c).max()), mask_words=words, reserved=0, cu_new_host=c.ctypes.data,
              cu_new_dev=0x1000, mask_dev=mask)
    kw.update(over)
    n = B.NewTokensStruct(**kw)
    n._keep = c
    return n


def _t(dtype=B.BF16, ptr=0x10000, token=4 * 64, head=64, layer=100 * 4 * 64):
    return B.TensorStruct(ptr, dtype, 0, layer, token, head)


def _s(ptr=0x20000, layer=800, token=2, head=200):
    return B.ScalesStruct(ptr, layer, token, head)


def test_quantise_and_back_refuse_bad_arguments(lib):
    p, t = _problem(), _t()

    def both(code, want, prob=p, val=t, codes=None, scales=None, v=True, cu=None, idx=None, total=0, status=0x100, v_codes=True):
        c = codes or _t(code)
        s = scales or _s()
        vv = r(val) if v else None
        vc, vs = (r(c), r(s)) if v_codes else (None, None)
        assert lib.kvcrush_quantize(r(prob), r(val), vv, cu, idx, total, None, None, r(c), r(s), vc, vs, status, None) == want
        assert lib.kvcrush_dequantize(r(prob), r(c), r(s), vc, vs, cu, idx, total, None, None, r(val), vv, status, None) == want

    for code in (B.INT8, B.E4M3, B.INT4):
        both(code, INV, status=None)
        both(code, INV, v_codes=False)
        both(code, INV, v=False)
        both(code, INV, idx=0x100)                          # rows by number without a list
        both(code, INV, cu=0x100, idx=0x100, total=-1)
        both(code, MIS, codes=_t(code, ptr=0x10008))
        both(code, MIS, codes=_t(code, token=4 * 64 + 8))
        both(code, INV, codes=_t(code, token=-64))
        both(code, INV, codes=_t(code, ptr=None))
        both(code, INV, scales=_s(ptr=None))
        both(code, MIS, scales=_s(ptr=0x20002))
        both(code, INV, scales=_s(token=-1))
        both(code, MIS, val=_t(ptr=0x10002))
        both(code, INV, val=_t(code))                       # codes where values belong
        both(code, UNS, prob=_problem(D=264))
        both(code, INV, prob=_problem(total_tokens=99))
    both(B.BF16, INV)                                       # values where codes belong
    both(7, INV)
    both(B.INT4, MIS, scales=_s(ptr=0x20004))
    both(B.INT4, MIS, scales=_s(token=1))
    both(B.INT4, MIS, codes=_t(B.INT4, head=48))
    both(B.INT4, UNS, prob=_problem(D=48))
    both(B.INT8, UNS, prob=_problem(D=24))
    c, s = _t(B.INT8), _s()
    c2 = _t(B.E4M3)
    f = _t(B.FP16)
    assert lib.kvcrush_quantize(r(p), r(t), r(f), None, None, 0, None, None, r(c), r(s), r(c), r(s), 0x100, None) == INV
    assert lib.kvcrush_quantize(r(p), r(t), r(t), None, None, 0, None, None, r(c), r(s), r(c2), r(s), 0x100, None) == INV
    assert lib.kvcrush_quantize(r(p), r(t), None, None, None, 0, None, None, r(c), None, None, None, 0x100, None) == INV
    assert lib.kvcrush_quantize(None, r(t), None, None, None, 0, None, None, r(c), r(s), None, None, 0x100, None) == INV


def _attend(lib, p=None, n=None, q=None, k=None, ks=None, v=None, vs=None, kn=None, vn=None, begin=None, count=None, o=None,
            status=0x100):
    t = _t()
    ref = lambda x: None if x is None else r(x)   # noqa: E731
    return lib.kvcrush_attend(r(p or _problem()), r(n or _new()), r(q or t), r(k or t), ref(ks), r(v or t), ref(vs), ref(kn), ref(vn),
                              begin, count, r(o or t), None, status, None)


def test_attention_refuses_bad_arguments(lib):
    f, c, s = _t(B.FP16), _t(B.INT8), _s()
    assert _attend(lib, status=None) == INV
    assert _attend(lib, q=f) == INV                         # another type than the cache
    assert _attend(lib, o=f) == INV
    assert _attend(lib, v=f) == INV
    assert _attend(lib, k=c, ks=s, v=c) == INV              # only one side quantised
    assert _attend(lib, k=c, ks=s, v=_t(B.E4M3), vs=s) == INV
    assert _attend(lib, k=c, v=c) == INV                    # codes without scales
    assert _attend(lib, ks=s, vs=s) == INV                  # scales of values
    assert _attend(lib, kn=_t()) == INV
    assert _attend(lib, kn=f, vn=f) == INV
    assert _attend(lib, begin=0x100) == INV and _attend(lib, count=0x100) == INV
    assert _attend(lib, n=_new(mask=0x100, words=1)) == INV                       # a mask without new keys
    assert _attend(lib, n=_new(cu=(0, 33), mask=0x100, words=1), kn=_t(), vn=_t()) == INV
    assert _attend(lib, n=_new(cu=(0, 1025)), kn=_t(), vn=_t()) == UNS
    assert _attend(lib, n=_new(max_new=1)) == INV
    assert _attend(lib, n=_new(total_new=3)) == INV
    assert _attend(lib, n=_new(cu_new_dev=None)) == INV
    assert _attend(lib, n=_new(cu=(0, 3, 1)), p=_problem(cu=(0, 50, 100))) == INV
    assert _attend(lib, p=_problem(D=264)) == UNS and _attend(lib, p=_problem(D=12)) == UNS
    assert _attend(lib, p=_problem(Hq=7)) == INV and _attend(lib, p=_problem(Hq=256)) == UNS
    assert _attend(lib, q=_t(ptr=0x10002)) == MIS and _attend(lib, o=_t(head=68)) == MIS and _attend(lib, k=_t(token=-64)) == INV
    assert _attend(lib, k=_t(ptr=None)) == INV
    assert _attend(lib, n=_new(cu=(0, 0)), q=_t(ptr=None), o=_t(ptr=None)) == 0   # nothing to do


def test_pages_refuse_bad_arguments(lib):
    t, f, p = _t(), _t(B.FP16), _problem()

    def bounds(page=32, recent=0, k=t, lo=t, hi=t, prob=p, begin=None, count=None, status=0x100):
        return lib.kvcrush_page_bounds(r(prob), r(k), page, recent, begin, count, r(lo), r(hi), status, None)

    assert bounds(page=0) == INV and bounds(page=12) == UNS and bounds(page=2048) == UNS and bounds(recent=-1) == INV
    assert bounds(lo=f) == INV and bounds(hi=f) == INV and bounds(k=_t(B.INT8)) == INV and bounds(status=None) == INV
    assert bounds(begin=0x100) == INV and bounds(hi=_t(ptr=0x10004)) == MIS and bounds(prob=_problem(D=272)) == UNS

    def pages(page=32, budget=4, initial=0, recent=0, lo=t, hi=t, n=None, prob=p, q=t):
        return lib.kvcrush_attend_pages(r(prob), r(n or _new()), r(q), r(t), None, r(t), None, page, r(lo), r(hi), budget, initial,
                                        recent, None, None, None, None, r(t), None, 0x100, None)

    assert pages(page=0) == INV and pages(page=20) == UNS and pages(page=4096) == UNS and pages(budget=0) == INV
    assert pages(initial=-1) == INV and pages(recent=-1) == INV and pages(lo=f) == INV and pages(hi=_t(ptr=None)) == INV
    assert pages(n=_new(mask=0x100, words=1)) == INV and pages(q=f) == INV
    assert pages(page=8, prob=_problem(cu=(0, 70000))) == UNS                     # more than 8192 pages
    assert pages(n=_new(cu=(0, 0)), q=_t(ptr=None)) == 0


def test_pages_of_an_empty_cache_need_no_memory(lib):
    """A cache without rows, whose tensors have no memory: no bounds to write, and the checks of the arguments stay."""
    none, t, p = _t(ptr=None), _t(), _problem(cu=(0, 0))

    def bounds(prob=p, k=none, lo=none, hi=none, page=32, status=0x100):
        return lib.kvcrush_page_bounds(r(prob), r(k), page, 0, None, None, r(lo), r(hi), status, None)

    assert bounds() == 0
    assert bounds(page=0) == INV and bounds(page=12) == UNS and bounds(status=None) == INV
    assert bounds(lo=_t(B.FP16, ptr=None)) == INV and bounds(k=_t(B.INT8, ptr=None)) == INV
    assert bounds(prob=_problem(cu=(0, 50))) == INV and bounds(prob=_problem(cu=(0, 50)), k=t) == INV

    def pages(prob, lo, hi):
        return lib.kvcrush_attend_pages(r(prob), r(_new()), r(t), r(none), None, r(none), None, 32, r(lo), r(hi), 4, 0, 0, None, None, None,
                                        None, r(t), None, None, None)

    assert pages(p, none, none) == INV                                            # no status word


def test_rows_of_an_empty_list_need_no_memory(lib):
    """Quantising no rows, from and into tensors without memory, is a call like any other; the types are checked all the same."""
    t, c, s = _t(ptr=None), _t(B.INT8, ptr=None), _s(ptr=None)

    def both(want, prob=_problem(cu=(0, 0)), val=t, cu=None, total=0):
        assert lib.kvcrush_quantize(r(prob), r(val), r(val), cu, None, total, None, None, r(c), r(s), r(c), r(s), 0x100, None) == want
        assert lib.kvcrush_dequantize(r(prob), r(c), r(s), r(c), r(s), cu, None, total, None, None, r(val), r(val), 0x100, None) == want

    both(0)
    both(0, prob=_problem(), cu=0x100)
    both(INV, prob=_problem())
    both(INV, prob=_problem(), cu=0x100, total=1)
    both(INV, val=c)
