"""Host-side bounds of the serving entry points that test_abi_serve does not reach (no GPU
needed).  Every rejected call carries a second defect that is checked last, as there."""

import pytest
import torch

from paper_2608_03893_amd import kvx
from tests.test_abi_host import L  # noqa: F401  (the library fixture)
from tests.test_abi_serve import Attend, Plan, Store, _expect


def test_rows_of_a_call(L):
    """2^30 rows at most: a wave's row numbers step past the last one by up to a page."""
    near = dict(ks=(0, 0, 0), vs=(0, 0, 0), k=1 << 50, v=1 << 51, slots=1 << 52, codes=1 << 53, scales=1 << 54)
    for T in ((1 << 30) + 1, (1 << 31) - 1):
        _expect(L, 5, Store, T=T, **{**near, "scales": near["slots"]})
        _expect(L, 5, Plan, T=T)
    _expect(L, 6, Store, T=1 << 30, **{**near, "scales": near["slots"]})   # comes to the last check


# (B, T, dtype): below 96 query rows a request and KV head, at it, and fp32 queries
@pytest.mark.parametrize("B,T,dtype", [(3, 71, 0), (3, 72, 0), (3, 72, 1), (1, 1, 0), (4096, 1 << 17, 0)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_workspace(L, B, T, dtype, d):
    dims = kvx.AttendDims(B, 2, 4, T, d, 0)
    need = kvx.attend_workspace_bytes(dims, "f32" if dtype else "bf16")
    assert need > kvx.ATTEND_COUNTER_BYTES
    call = dict(dims=dims, dtype=dtype, qs=(8 * d, d))
    _expect(L, 7, Attend, **call, ws=None, wsb=need)
    _expect(L, 7, Attend, **call, wsb=need - 1)
    _expect(L, 7, Attend, **call, wsb=0)
    at = 1 << 40
    for off in (16, 128):
        _expect(L, 7, Attend, **call, ws=at + off, wsb=need)
    _expect(L, 6, Attend, **call, ws=at, wsb=need)                # comes to the last check
    base = Attend()
    for name in ("q", "codes", "scales", "tables", "lens", "cu", "out", "lse"):
        for ws in (getattr(base, name), getattr(base, name) - need // 256 * 256 + 256):   # its last bytes
            if ws > 0:
                assert Attend(**call, ws=ws, wsb=1 << 40).run(L) == 6, (name, L.kvx_last_error())


def test_a_workspace_of_few_rows_is_too_small_for_chunks(L):
    """The bytes change where the kernel by rows may be chosen, and never fall as rows grow."""
    for d in (64, 128):
        few, many = (kvx.attend_workspace_bytes(kvx.AttendDims(3, 2, 4, T, d, 0)) for T in (71, 72))
        assert few < many
        _expect(L, 7, Attend, dims=kvx.AttendDims(3, 2, 4, 72, d, 0), qs=(8 * d, d), wsb=few)
        assert kvx.attend_workspace_bytes(kvx.AttendDims(3, 2, 4, 1 << 20, d, 0)) == many


def test_attention_bound_of_the_longest(L):
    for longest in (-1, -2 ** 31):
        dims = kvx.AttendDims(3, 2, 4, 10, 128, longest)
        _expect(L, 2, Attend, dims=dims)
        assert L.kvx_attend_workspace_bytes(dims, 0) == 0


def test_binding_refuses_sizes_outside_32_bits():
    """Neither cut to 32 bits nor allocated for first."""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    for T, page in ((4, 2 ** 32 + 16), (4, -2 ** 32 + 16), (2 ** 32 + 4, 16), (2 ** 31, 16), (-2 ** 32 + 4, 16)):
        with pytest.raises(ValueError, match="32 bits"):
            kvx.plan_pages(i(3), i(3), i(3, 2), i(9), i(2), T, page)
    q, pool = torch.zeros((5, 6, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 64, 64), dtype=torch.float8_e4m3fn)
    for longest in (2 ** 31, -2 ** 32 + 5):
        with pytest.raises(ValueError, match="32 bits"):
            kvx.attend_cache8(q, pool, torch.ones((2, 2, 4)), i(2, 4), i(2), i(3), longest=longest)
