"""Coefficients of the policy loss that 64 bits hold and 32 do not: refused before any CUDA work."""
import pytest

from paper_1911_08020_gb300 import build as darb_build
from paper_1911_08020_gb300 import darb
from tests.test_policy_abi import call


@pytest.fixture(scope="module")
def L():
    darb_build.build()
    return darb.lib()


@pytest.mark.parametrize("kw", [dict(kl=1e39), dict(kl=-1e300), dict(bonus=3.5e38), dict(bonus=-1e39)])
def test_refused(L, kw):
    assert call(L, **kw) == darb.ERR_INVALID_ARG
