"""The serving operators' later arguments: checks that answer before any GPU call."""
import ctypes

import pytest

import paper_1909_09927_amd as sconv

torch = pytest.importorskip("torch")
from paper_1909_09927_amd import serving as S  # noqa: E402

P = ctypes.c_void_p(4096)      # never read


def test_linear8_exact_is_0_or_1():
    def call(exact, M=3, y_type=1):
        d = S.Linear8Desc(M=M, N=5, K=200, y_type=y_type, x_m=200, w_n=200, y_m=5, exact=exact)
        return S._serving_lib().sconv_linear8(ctypes.byref(d), P, P, P, P, P, None)

    for bad in (-1, 2, 1 << 30):
        assert call(bad) == call(bad, M=0) == sconv.SCONV_EINVAL
    assert call(0, M=0) == call(1, M=0) == call(1, M=0, y_type=0) == 0
