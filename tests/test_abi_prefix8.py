"""Host-side checks of kvx_attend_prefix8 (no GPU needed); see test_abi_serve for the scheme."""

import ctypes

import pytest

from paper_2608_03893_amd import kvx
from tests.test_abi_host import L  # noqa: F401  (the library fixture)
from tests.test_abi_serve import A, Call, _expect


class Prefix(Call):
    entry = "kvx_attend_prefix8"

    def __init__(self, **kw):
        self.dims, self.pool, self.prefix = kvx.AttendDims(3, 2, 4, 10, 128), kvx.Pool(100, 16, 8), kvx.PrefixDims(2, 9, 0)
        self.dtype, self.qs, self.scale = 0, (8 * 128, 128), 0.1
        (self.q, self.codes, self.scales, self.ptables, self.plens, self.pcu, self.tables, self.lens, self.cu, self.out,
         self.lse, self.ws) = (n * A for n in range(1, 13))
        self.wsb = 1 << 29
        self.__dict__.update(kw)

    def args(self):
        return (self.dims, self.prefix, self.pool, self.dtype, self.q,
                None if self.qs is None else (ctypes.c_int64 * 2)(*self.qs), self.codes, self.scales, self.ptables,
                self.plens, self.pcu, self.tables, self.lens, self.cu, self.scale, self.out, self.lse, self.ws, self.wsb,
                None)

    spoil = dict(lse=9 * A)               # on top of cu


def test_sizes_and_types(L):
    _expect(L, 1, Prefix, pool=None)
    _expect(L, 1, Prefix, dims=None)
    _expect(L, 1, Prefix, prefix=None)
    _expect(L, 4, Prefix, dtype=3)
    for p in ((-1, 9, 0), (2, 0, 0), (2, -3, 0), (2, 9, -1)):
        _expect(L, 2, Prefix, prefix=kvx.PrefixDims(*p))
    _expect(L, 5, Prefix, prefix=kvx.PrefixDims(4097, 9, 0))
    for d in ((-1, 2, 4, 10, 128), (3, 0, 4, 10, 128), (3, 2, 0, 10, 128), (3, 2, 4, -1, 128), (3, 2, 4, 10, 128, -1)):
        _expect(L, 2, Prefix, dims=kvx.AttendDims(*d))
    for d in ((4097, 2, 4, 10, 128), (3, 2, 4, 10, 96), (3, 2, 4, 1 << 28, 128)):
        _expect(L, 5, Prefix, dims=kvx.AttendDims(*d))
    for bad in (float("nan"), float("inf")):
        _expect(L, 2, Prefix, scale=bad)


def test_operands(L):
    for name in ("q", "codes", "out"):
        _expect(L, 1, Prefix, **{name: None})
        _expect(L, 5, Prefix, **{name: 20 * A + 8})
    for name in ("scales", "ptables", "plens", "pcu", "tables", "lens", "cu"):
        _expect(L, 1, Prefix, **{name: None})
        _expect(L, 5, Prefix, **{name: 20 * A + 2})
    _expect(L, 5, Prefix, lse=20 * A + 2)
    _expect(L, 1, Prefix, qs=None)
    _expect(L, 2, Prefix, qs=(-8, 128))
    _expect(L, 5, Prefix, qs=(1028, 128))
    # without prefixes nothing of theirs is looked at
    _expect(L, 6, Prefix, prefix=kvx.PrefixDims(0, 9, 0), ptables=None, plens=None, pcu=None)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,S,T", [(3, 2, 10), (1, 1, 1), (3, 1, 72), (4096, 4096, 1 << 12), (3, 0, 10)])
def test_workspace(L, dtype, B, S, T):
    dims, prefix = kvx.AttendDims(B, 2, 4, T, 64, 0), kvx.PrefixDims(S, 9, 0)
    need = kvx.prefix_workspace_bytes(dims, prefix, "f32" if dtype else "bf16")
    plain = max(kvx.attend_workspace_bytes(kvx.AttendDims(n, 2, 4, T, 64, 0), "f32" if dtype else "bf16")
                for n in (B, max(S, 1)))
    assert need >= plain if S == 0 else need >= plain + T * 8 * (64 + 2) * 4
    call = dict(dims=dims, prefix=prefix, dtype=dtype, qs=(8 * 64, 64))
    _expect(L, 7, Prefix, **call, ws=None, wsb=need)
    _expect(L, 7, Prefix, **call, wsb=need - 1)
    _expect(L, 7, Prefix, **call, ws=20 * A + 128, wsb=need)
    _expect(L, 6, Prefix, **call, wsb=need)


@pytest.mark.parametrize("out", ["out", "lse", "ws"])
@pytest.mark.parametrize("name", ["q", "codes", "scales", "ptables", "plens", "pcu", "tables", "lens", "cu"])
def test_outputs_overlap_nothing(L, out, name):
    assert Prefix(**{out: getattr(Prefix(), name)}).run(L) == 6
    assert b"overlaps" in L.kvx_last_error()


def test_empty_calls_launch_nothing(L):
    for dims in ((0, 2, 4, 10, 128), (3, 2, 4, 0, 128)):
        none = dict.fromkeys(("q", "codes", "scales", "ptables", "plens", "pcu", "tables", "lens", "cu", "out", "lse", "ws"))
        assert Prefix(dims=kvx.AttendDims(*dims), **none).run(L) == 0
        assert kvx.prefix_workspace_bytes(kvx.AttendDims(*dims), kvx.PrefixDims(1, 1, 0)) == 0


def test_kernel_names():
    dims, pool = (lambda B, T, d=128, G=8: kvx.AttendDims(B, 8, G, T, d, 0)), (lambda M: kvx.Pool(1000, 16, M))
    names = kvx.prefix_kernel_names
    assert names(dims(4, 4), kvx.PrefixDims(1, 100, 0), pool(5)) == ("prefix8_split_kernel<0, 128, 4, 1>",) * 2
    assert names(dims(4, 4), kvx.PrefixDims(0, 100, 0), pool(5))[0] is None
    assert names(dims(4, 4), kvx.PrefixDims(0, 100, 0), pool(5))[1] == kvx.attend_kernel_name(dims(4, 4), pool(5))
    common, own = names(dims(64, 64), kvx.PrefixDims(1, 512, 0), pool(70))
    assert common == "prefix8_common_split_kernel<0, 128, 8, 2>" and own == "prefix8_own_split_kernel<0, 128, 4, 1>"
    common, own = names(dims(8, 2048), kvx.PrefixDims(1, 512, 0), pool(70))
    assert common == "prefix8_common_rows_kernel<128, 2>" and own.startswith("prefix8_own_")
    assert names(dims(0, 0), kvx.PrefixDims(1, 512, 0), pool(70)) == (None, None)
    for bad in ((dims(4, 4, d=96), kvx.PrefixDims(1, 9, 0), pool(5)), (dims(4, 4), kvx.PrefixDims(-1, 9, 0), pool(5)),
                (dims(4, 4), kvx.PrefixDims(1, 9, 0), pool(0))):
        with pytest.raises(kvx.KvxError):
            names(*bad)
