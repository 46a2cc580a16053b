"""Host-side bounds of the serving entry points that test_abi_serve does not reach (no GPU
needed).  Every rejected call carries a second defect that is checked last, as there."""

from tests.test_abi_host import L  # noqa: F401  (the library fixture)
from tests.test_abi_serve import Plan, Store, _expect


def test_rows_of_a_call(L):
    """2^30 rows at most: a wave's row numbers step past the last one by up to a page."""
    near = dict(ks=(0, 0, 0), vs=(0, 0, 0), k=1 << 50, v=1 << 51, slots=1 << 52, codes=1 << 53, scales=1 << 54)
    for T in ((1 << 30) + 1, (1 << 31) - 1):
        _expect(L, 5, Store, T=T, **{**near, "scales": near["slots"]})
        _expect(L, 5, Plan, T=T)
    _expect(L, 6, Store, T=1 << 30, **{**near, "scales": near["slots"]})   # comes to the last check
