"""Host-only checks of the 8-bit product's limits (the pointers are never
dereferenced: every call here is refused)."""
import pytest

from paper_2606_28516_amd import clearmoe as cm
from tests.test_serving_host import A, INVALID, _product

TOP = (1 << 31) - 1


@pytest.mark.parametrize("kw", [
    dict(M=TOP, N=1, out=cm.F32), dict(M=TOP - 2000, N=128, out=cm.F32), dict(M=1 << 30, N=257, out=cm.F32),
    dict(M=TOP, N=129), dict(M=1 << 30, N=513), dict(M=1 << 23, N=65536), dict(M=TOP, N=129, out=2, sc=A),
    dict(M=(1 << 28) + 1, N=65536), dict(M=TOP - 2047, N=128, out=cm.F32, groups=1, offsets=A)])
def test_more_threads_than_a_launch_holds(kw):
    assert _product(**kw) == INVALID
