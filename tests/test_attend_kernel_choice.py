"""Host-only: which kernel an attention call takes, at the edges of the rules on rows, requests
and the length of the tables, and what the arguments may be."""

import pytest

from paper_2608_03893_amd import kvx


def _name(B, rows, keys, H=8, G=8, d=128, dtype="bf16", longest=0, page=16):
    """B requests of `rows` query rows a KV head each on average, tables of `keys` tokens."""
    return kvx.attend_kernel_name(kvx.AttendDims(B, H, G, B * rows // G, d, longest),
                                  kvx.Pool(1000, page, keys // page), dtype)


SPLIT, ROWS = "attend8_split_kernel<%d, %d, %d, %d>", "attend8_rows_kernel<%d, 2>"


@pytest.mark.parametrize("args,kernel", [
    # chunks: 96 rows a request and blocks of 256 rows for the CUs, or work enough
    (dict(B=32, rows=96, keys=304), ROWS % 128),
    (dict(B=32, rows=88, keys=304), SPLIT % (0, 128, 4, 2)),
    (dict(B=24, rows=96, keys=16), ROWS % 128),                     # 192 units
    (dict(B=23, rows=96, keys=16), SPLIT % (0, 128, 4, 1)),
    (dict(B=1, rows=2048, keys=8192), ROWS % 128),                  # 2^34
    (dict(B=1, rows=2048, keys=8176), SPLIT % (0, 128, 4, 2)),
    (dict(B=16, rows=128, keys=4096), ROWS % 128),                  # 2^33 in 128 units
    (dict(B=1, rows=4096, keys=8192, d=64), ROWS % 64),
    (dict(B=1, rows=4096, keys=8192, dtype="f32"), SPLIT % (1, 128, 4, 1)),
    # blocks of 32 rows
    (dict(B=64, rows=24, keys=256), SPLIT % (0, 128, 4, 2)),
    (dict(B=64, rows=24, keys=240), SPLIT % (0, 128, 4, 1)),        # too few keys
    (dict(B=64, rows=16, keys=4096), SPLIT % (0, 128, 12, 1)),      # one tile a request
    (dict(B=32, rows=24, keys=1024), SPLIT % (0, 128, 8, 2)),       # few units of 1024 keys
    (dict(B=32, rows=24, keys=1008), SPLIT % (0, 128, 4, 2)),
    (dict(B=64, rows=24, keys=1024), SPLIT % (0, 128, 4, 2)),       # 512 units
    (dict(B=32, rows=24, keys=1024, d=64), SPLIT % (0, 64, 12, 2)),
    # blocks of 16
    (dict(B=8, rows=8, keys=1024), SPLIT % (0, 128, 12, 1)),
    (dict(B=8, rows=8, keys=1008), SPLIT % (0, 128, 4, 1)),
    (dict(B=1, rows=4, keys=8192, G=4), SPLIT % (0, 128, 12, 1)),
    (dict(B=1, rows=3, keys=8192, G=3), SPLIT % (0, 128, 4, 1)),    # few units of few rows
    (dict(B=1, rows=3, keys=65536, G=3), SPLIT % (0, 128, 12, 1)),
    (dict(B=64, rows=8, keys=1024), SPLIT % (0, 128, 4, 1)),        # many short units
    (dict(B=64, rows=8, keys=1040), SPLIT % (0, 128, 12, 1)),
    (dict(B=64, rows=8, keys=1040, d=64), SPLIT % (0, 64, 12, 1)),
    (dict(B=8, rows=32, keys=1024, dtype="f32"), SPLIT % (1, 128, 8, 1)),
    (dict(B=8, rows=120, keys=1024, dtype="f32"), SPLIT % (1, 128, 8, 1)),
    (dict(B=8, rows=128, keys=4096, dtype="f32"), SPLIT % (1, 128, 4, 1)),         # 512 units
    (dict(B=8, rows=128, keys=4096, d=64, dtype="f32"), SPLIT % (1, 64, 4, 1)),
    (dict(B=2, rows=64, keys=1024), SPLIT % (0, 128, 12, 1)),       # too few keys for 32 rows a block
    (dict(B=64, rows=8, keys=4096, dtype="f32"), SPLIT % (1, 128, 4, 1)),
    (dict(B=64, rows=8, keys=4096, d=64, dtype="f32"), SPLIT % (1, 64, 12, 1)),
    # a stated bound counts where it is below the tables' length
    (dict(B=8, rows=8, keys=131072, longest=1023), SPLIT % (0, 128, 4, 1)),
    (dict(B=8, rows=8, keys=1008, longest=1 << 30), SPLIT % (0, 128, 4, 1)),
])
def test_choice(args, kernel):
    for page in (16, 128):
        if args["keys"] % page == 0:
            assert _name(**args, page=page) == kernel


def test_extreme_sizes():
    """Products of sizes at their bounds do not wrap."""
    big = kvx.Pool(1 << 26, 16, 2 ** 31 - 1)
    assert kvx.attend_kernel_name(kvx.AttendDims(4096, 32767, 2, 1 << 28, 128, 0), big) == ROWS % 128
    assert kvx.attend_kernel_name(kvx.AttendDims(4096, 65535, 1, 4096, 64, 0), big) == SPLIT % (0, 64, 12, 1)


def test_refusals():
    good = dict(B=3, H=2, G=4, T=10, d=128, longest=0)
    for bad in (dict(B=-1), dict(B=4097), dict(B=0), dict(T=0), dict(H=0), dict(G=0), dict(d=96), dict(longest=-1)):
        with pytest.raises(ValueError):
            kvx.attend_kernel_name(kvx.AttendDims(**{**good, **bad}), kvx.Pool(100, 16, 8))
    for pool in ((0, 16, 8), (100, 17, 8), (100, 16, 0)):
        with pytest.raises(ValueError):
            kvx.attend_kernel_name(kvx.AttendDims(**good), kvx.Pool(*pool))
    with pytest.raises(ValueError):
        kvx.attend_kernel_name(kvx.AttendDims(**good), kvx.Pool(100, 16, 8), "f16")
    lib = kvx.load()
    assert lib.kvx_attend_kernel_name(None, None, 0) is None
