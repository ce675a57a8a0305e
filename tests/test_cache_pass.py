"""What a compression pass into a quantised cache refuses, before anything is enqueued."""
import numpy as np
import pytest

from paper_2503_00022_b200 import binding as B
from paper_2503_00022_b200 import build as kbuild


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


def _pass(D=64, **more):
    return B.CompressionPass(B.Problem(1, 2, 2, D, [40], device="cpu"), np.asarray([[4]]), np.asarray([[4]]), **more)


@pytest.mark.parametrize("fmt,D", [(B.INT8, 40), (B.E4M3, 24), (B.INT4, 48), (B.INT4, 16), (B.INT8, 272), (B.BF16, 64), (7, 64)])
def test_formats_and_head_sizes_that_do_not_go_together(fmt, D):
    with pytest.raises(ValueError):
        _pass(D, cache_format=fmt)


def test_less_than_no_room():
    with pytest.raises(ValueError):
        _pass(cache_format=B.INT8, spare_rows=-1)


@pytest.mark.parametrize("more", [dict(cache_format=B.INT8, with_cache=False), dict(cache_format=B.INT4, with_cache=False), dict(),
                                  dict(page_size=8)])
def test_a_pass_without_a_reduced_cache_takes_no_cache(monkeypatch, more):
    """The error comes before the first stage is enqueued, and from compact alone too."""
    import torch
    cp = _pass(**more)
    called = []
    for name in B.EXPORTS:
        if hasattr(B, name) and name not in ("kvcrush_strerror", "kvcrush_version", "kvcrush_workspace_size"):
            monkeypatch.setattr(B, name, lambda *a, _n=name, **k: called.append(_n))
    x = torch.zeros((1, 40, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        cp.run(x, x, x, x)
    with pytest.raises(ValueError):
        cp.compact(x, x)
    assert not called
    cp.run(x, x)                                         # without a cache the pass selects
    assert "kvcrush_score" in called and not any("compact" in n or "quantize" in n for n in called)


def test_an_int8_pass_of_an_allowed_size():
    cp = _pass(80, cache_format=B.INT8, spare_rows=2)
    assert cp.k_out.codes.shape == (1, 10, 2, 80) and cp.row_count.tolist() == [[8]]
