"""kvx_prefix_workspace_bytes over sizes that grow (no GPU needed)."""

import pytest

from paper_2608_03893_amd import kvx

SIZES = [(1, 1, 1, 1, 64), (3, 2, 2, 4, 128), (8, 1, 8, 8, 128), (64, 1, 8, 8, 64), (5, 5, 2, 3, 64), (300, 70, 1, 16, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S,H,G,d", SIZES)
def test_more_rows_never_need_less(B, S, H, G, d, dtype):
    """A workspace for the longest step of a program is enough for its shorter ones."""
    need = [kvx.prefix_workspace_bytes(kvx.AttendDims(B, H, G, T, d, 0), kvx.PrefixDims(S, 9, 0), dtype)
            for T in list(range(1, 2100)) + [4096, 20000, 65535, 65536, 65537, 70000]]
    drop = [(a, b) for a, b in zip(need, need[1:]) if b < a]
    assert not drop, drop[:3]


def test_calls_that_cannot_go_in_one_launch_hold_no_room_for_it():
    """What is asked for beyond the sums of a part's rows stays the same once a launch of its own
    is certain for either part."""
    def rest(T):
        dims = kvx.AttendDims(8, 8, 8, T, 128, 0)
        return kvx.prefix_workspace_bytes(dims, kvx.PrefixDims(1, 9, 0)) - T * 64 * (128 + 4) * 4
    one = kvx.prefix_kernel_names(kvx.AttendDims(8, 8, 8, 700, 128, 0), kvx.PrefixDims(1, 1, 0), kvx.Pool(100, 16, 1))
    assert one[0] != one[1]
    assert abs(rest(700) - rest(1400)) <= 1024
