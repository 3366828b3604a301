"""Refusals of the operators of a layer of experts at the edges of what they take, without a GPU."""
import ctypes as C

import pytest

from paper_1505_04956_b200 import binding, experts

from .test_experts_host import _p, _q

EINVAL, EUNSUPPORTED, ECUDA, OK = binding.ASGD_EINVAL, binding.ASGD_EUNSUPPORTED, binding.ASGD_ECUDA, binding.ASGD_OK


@pytest.mark.parametrize("bad", [dict(M=(1 << 31) - 255), dict(M=(1 << 31) - 1), dict(N=(1 << 31) - 255, ldc=1 << 31), dict(N=(1 << 31) - 1, ldc=1 << 31),
                                 dict(K=(1 << 31) - 255, lda=1 << 31, ldb=1 << 31)])
@pytest.mark.parametrize("grouped", [dict(), dict(groups=3, offsets=1 << 20)])
def test_product_refuses_sizes_whose_tiles_pass_32_bits(bad, grouped):
    assert experts._load().asgd_product(C.byref(_p(**bad, **grouped)), None) == EUNSUPPORTED


def test_quantize_refuses_rows_whose_blocks_pass_32_bits():
    wide = 1 << 31
    assert experts._load().asgd_quantize(C.byref(_q(M=1, rows_x=1, K=wide - 65535, ldx=wide, ldq=wide, square=1)), None) == EUNSUPPORTED
