"""Host-side checks of the serving entry points (no GPU needed): page plan, 8-bit store,
attention over the 8-bit pool.

Calls pass placeholder addresses 1 GiB apart.  Each rejected call also carries a second
defect that is checked last, an output on top of an input, so that a missed check still
cannot reach a launch."""

import ctypes

import pytest
import torch

from paper_2608_03893_amd import kvx
from tests.test_abi_host import L  # noqa: F401  (the library fixture)

A = 1 << 30


class Call:
    def run(self, L):
        return getattr(L, self.entry)(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a
                                        for a in self.args()])


class Plan(Call):
    entry = "kvx_plan_pages"

    def __init__(self, **kw):
        self.pool = kvx.Pool(100, 16, 8)
        self.B, self.T = 4, 64
        for n, name in enumerate(("lens", "add", "tables", "ring", "free", "lens_out", "cu", "pos", "slots",
                                  "free_out")):
            setattr(self, name, (n + 1) * A)
        self.__dict__.update(kw)

    def args(self):
        return (self.pool, self.B, self.T, self.lens, self.add, self.tables, self.ring, self.free,
                self.lens_out, self.cu, self.pos, self.slots, self.free_out, None)

    spoil = dict(free_out=5 * A)          # on top of free


class Store(Call):
    entry = "kvx_store_cache8"

    def __init__(self, **kw):
        self.pool = kvx.Pool(100, 16, 0)
        self.dtype, self.L, self.H, self.T, self.d = 0, 2, 4, 64, 128
        self.ks = self.vs = (2 * 4 * 64 * 128, 64 * 128, 128)
        self.k, self.v, self.slots, self.codes, self.scales = (n * A for n in range(1, 6))
        self.__dict__.update(kw)

    def args(self):
        st = [None if s is None else (ctypes.c_int64 * 3)(*s) for s in (self.ks, self.vs)]
        return (self.pool, self.dtype, self.L, self.H, self.T, self.d, self.k, st[0], self.v, st[1],
                self.slots, self.codes, self.scales, None)

    spoil = dict(scales=3 * A)            # on top of slots


class Attend(Call):
    entry = "kvx_attend_cache8"

    def __init__(self, **kw):
        self.dims, self.pool = kvx.AttendDims(3, 2, 4, 10, 128), kvx.Pool(100, 16, 8)
        self.dtype, self.qs, self.scale = 0, (8 * 128, 128), 0.1
        (self.q, self.codes, self.scales, self.tables, self.lens, self.cu, self.out, self.lse,
         self.ws) = (n * A for n in range(1, 10))
        self.wsb = 1 << 29
        self.__dict__.update(kw)

    def args(self):
        return (self.dims, self.pool, self.dtype, self.q,
                None if self.qs is None else (ctypes.c_int64 * 2)(*self.qs), self.codes, self.scales,
                self.tables, self.lens, self.cu, self.scale, self.out, self.lse, self.ws, self.wsb, None)

    spoil = dict(lse=6 * A)               # on top of cu


def _expect(lib, status, call, /, **kw):
    st = call(**{**call.spoil, **kw}).run(lib)
    assert st == status, (kvx.STATUS.get(st), lib.kvx_last_error())
    assert lib.kvx_last_error() != b""


@pytest.mark.parametrize("call", [Plan, Store, Attend])
def test_pools(L, call):
    m = 1 if call is not Store else 0
    _expect(L, 1, call, pool=None)
    for pool in ((0, 16, 8), (-1, 16, 8), (10, 0, 8), (10, -16, 8)) + (((10, 16, 0),) if m else ()):
        _expect(L, 2, call, pool=kvx.Pool(*pool))
    for size in (1, 8, 17, 48, 256):
        _expect(L, 5, call, pool=kvx.Pool(10, size, 8))
    _expect(L, 2, call, pool=kvx.Pool(1 << 27, 16, 8))                   # 2^31 slots


def test_plan_rejections(L):
    _expect(L, 2, Plan, B=-1)
    _expect(L, 2, Plan, T=-1)
    _expect(L, 5, Plan, B=4097)
    _expect(L, 5, Plan, T=(1 << 30) + 1)
    for name in ("lens", "add", "tables", "ring", "free", "lens_out", "cu", "pos", "slots"):
        _expect(L, 1, Plan, **{name: None})
        _expect(L, 5, Plan, **{name: 20 * A + 2})
    _expect(L, 5, Plan, pos=20 * A + 4)
    _expect(L, 1, Plan, free_out=None)
    # every output against inputs and outputs
    for a, b in (("lens_out", "lens"), ("cu", "add"), ("tables", "free"), ("slots", "pos"),
                 ("free_out", "ring"), ("lens_out", "cu"), ("tables", "ring")):
        p = Plan()
        assert Plan(**{a: getattr(p, b)}).run(L) == 6
    assert Plan(ring=3 * A + 4 * 4 * 8 - 4).run(L) == 6                  # the table's last entry


def test_store_rejections(L):
    _expect(L, 3 + 1, Store, dtype=7)
    for kw in (dict(L=0), dict(H=0), dict(T=-1), dict(d=0)):
        _expect(L, 2, Store, **kw)
    for kw in (dict(d=96), dict(d=256), dict(L=4096, H=16)):
        _expect(L, 5, Store, **kw)
    for name in ("k", "v", "slots", "codes", "scales"):
        _expect(L, 1, Store, **{name: None})
        _expect(L, 5, Store, **{name: 20 * A + 2})
    for name in ("k", "v", "codes"):
        _expect(L, 5, Store, **{name: 20 * A + 8})
    for name in ("ks", "vs"):
        _expect(L, 1, Store, **{name: None})
        _expect(L, 2, Store, **{name: (-128, 128, 128)})
        _expect(L, 2, Store, **{name: (1 << 62, 128, 128)})
        _expect(L, 5, Store, **{name: (1024, 128, 132)})                 # 264 bytes
    _expect(L, 5, Store, dtype=1, ks=(1024, 130, 128))
    for a, b in (("codes", "k"), ("codes", "v"), ("scales", "slots"), ("codes", "scales")):
        assert Store(**{a: getattr(Store(), b)}).run(L) == 6
    assert Store(codes=1 * A + 2 * 2 * 4 * 64 * 128 * 2 - 128 * 2 - 64 * 128 * 2 * 4).run(L) == 6   # k's last row
    assert Store(T=0, k=None, v=None, slots=None, codes=None, scales=None).run(L) == 0


def test_attend_rejections(L):
    _expect(L, 1, Attend, dims=None)
    _expect(L, 4, Attend, dtype=2)
    for kw in (dict(B=-1), dict(T=-1), dict(H=0), dict(G=0), dict(d=0)):
        _expect(L, 2, Attend, dims=kvx.AttendDims(**{**dict(B=3, H=2, G=4, T=10, d=128), **kw}))
    for kw in (dict(B=4097), dict(d=80), dict(H=1 << 15, G=2), dict(T=1 << 29, G=2)):
        _expect(L, 5, Attend, dims=kvx.AttendDims(**{**dict(B=3, H=2, G=4, T=10, d=128), **kw}))
    for name in ("q", "codes", "scales", "tables", "lens", "cu", "out"):
        _expect(L, 1, Attend, **{name: None})
        _expect(L, 5, Attend, **{name: 20 * A + 2})
    _expect(L, 5, Attend, lse=20 * A + 2, out=1 * A)
    for name in ("q", "codes", "out"):
        _expect(L, 5, Attend, **{name: 20 * A + 8})
    _expect(L, 1, Attend, qs=None)
    _expect(L, 2, Attend, qs=(-1024, 128))
    _expect(L, 5, Attend, qs=(1024, 132))
    for bad in (float("nan"), float("inf")):
        _expect(L, 2, Attend, scale=bad)
    for a, b in (("out", "q"), ("out", "codes"), ("lse", "lens"), ("out", "tables"), ("lse", "out"), ("out", "cu")):
        assert Attend(**{a: getattr(Attend(), b)}).run(L) == 6
    for kw in (dict(B=0), dict(T=0)):
        d = kvx.AttendDims(**{**dict(B=3, H=2, G=4, T=10, d=128), **kw})
        assert Attend(dims=d, q=None, codes=None, ws=None, wsb=0).run(L) == 0
        assert kvx.attend_workspace_bytes(d) == 0
    assert L.kvx_attend_workspace_bytes(None, 0) == 0


def test_binding_rejects_bad_tensors():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        kvx.plan_pages(i(3), i(4), i(3, 2), i(9), i(2), 4, 16)            # add's length
    with pytest.raises(ValueError):
        kvx.plan_pages(i(3), i(3), i(3), i(9), i(2), 4, 16)               # tables' rank
    with pytest.raises(ValueError):
        kvx.plan_pages(i(3), i(3), i(3, 2), i(9), i(1), 4, 16)            # free's length
    with pytest.raises(ValueError):
        kvx.plan_pages(i(3), i(3), i(3, 2), i(9), i(2), 4, 16)            # not on the GPU
    k = torch.zeros((1, 2, 5, 64), dtype=torch.bfloat16)
    pool, scales = torch.zeros((1, 2, 2, 64, 64), dtype=torch.float8_e4m3fn), torch.ones((1, 2, 2, 4))
    with pytest.raises(ValueError):
        kvx.store_cache8(k, k[:, :, :4], i(5), pool, scales)
    with pytest.raises(ValueError):
        kvx.store_cache8(k, k.float(), i(5), pool, scales)
    with pytest.raises(ValueError):
        kvx.store_cache8(k, k, i(5), pool.view(torch.uint8), scales)
    with pytest.raises(ValueError):
        kvx.store_cache8(k, k, i(5), pool, scales[..., :3])               # 64 slots on 3 pages
    with pytest.raises(ValueError):
        kvx.store_cache8(torch.zeros((1, 2, 5, 128)), torch.zeros((1, 2, 5, 128)), i(5), pool, scales)
    with pytest.raises(ValueError):
        kvx.store_cache8(k, k, i(5), pool, scales)                        # not on the GPU
    q = torch.zeros((5, 6, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kvx.attend_cache8(q[:, :5], pool[0], scales[0], i(2, 4), i(2), i(3))     # 5 heads on 2
    with pytest.raises(TypeError):
        kvx.attend_cache8(q.half(), pool[0], scales[0], i(2, 4), i(2), i(3))
    with pytest.raises(ValueError):
        kvx.attend_cache8(q, pool, scales, i(2, 4), i(2), i(3))           # all layers
    with pytest.raises(ValueError):
        kvx.attend_cache8(q, pool[0], scales[0], i(2, 4), i(2), i(2))     # cu's length
    with pytest.raises(ValueError):
        kvx.attend_cache8(q, pool[0], scales[0], i(2, 4), i(2), i(3), out=q.float())
