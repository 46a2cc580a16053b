"""Host-side checks of kvx_norm_rope (no GPU needed); see test_abi_serve for the scheme."""

import ctypes

import pytest

from paper_2608_03893_amd import kvx
from tests.test_abi_host import L  # noqa: F401  (the library fixture)
from tests.test_abi_serve import A, Call, _expect


class NormRope(Call):
    entry = "kvx_norm_rope"

    def __init__(self, **kw):
        self.dtype, self.T, self.Hq, self.Hk, self.d, self.eps = 0, 10, 8, 2, 128, 1e-6
        self.qs, self.ks = (12 * 128, 128), (12 * 128, 128)
        self.q, self.k, self.qw, self.kw, self.pos, self.qo, self.ko = (n * A for n in range(1, 8))
        self.rope = kvx.make_rope(dict(theta=1e4))
        self.__dict__.update(kw)

    def args(self):
        s = [None if x is None else (ctypes.c_int64 * 2)(*x) for x in (self.qs, self.ks)]
        return (self.dtype, self.T, self.Hq, self.Hk, self.d, self.q, s[0], self.k, s[1], self.qw, self.kw, self.eps,
                self.rope, self.pos, self.qo, self.ko, None)

    spoil = dict(ko=5 * A)               # on top of the positions


def test_sizes_and_types(L):
    _expect(L, 4, NormRope, dtype=2)
    for kw in (dict(T=-1), dict(Hq=0), dict(Hk=-1), dict(d=0), dict(eps=-1e-6), dict(eps=float("nan")),
               dict(eps=float("inf"))):
        _expect(L, 2, NormRope, **kw)
    for kw in (dict(d=96), dict(d=256), dict(T=(1 << 30) + 1), dict(Hq=65535, Hk=1)):
        _expect(L, 5, NormRope, **kw)
    _expect(L, 1, NormRope, rope=None)
    for bad in (dict(theta=1.0), dict(theta=float("inf")), dict(theta=1e4, style=2), dict(theta=1e4, factor=0.5),
                dict(theta=1e4, factor=8.0, low_freq_factor=4.0, high_freq_factor=4.0)):
        _expect(L, 9, NormRope, rope=kvx.make_rope(bad))


def test_operands(L):
    for name in ("q", "k", "pos", "qo"):
        _expect(L, 1, NormRope, **{name: None})
        _expect(L, 5, NormRope, **{name: 20 * A + 2})
    for name in ("qw", "kw"):
        _expect(L, 5, NormRope, **{name: 20 * A + 8})
        _expect(L, 6, NormRope, **{name: None})            # no norm: comes to the last check
    _expect(L, 1, NormRope, ko=None, qo=5 * A)
    for name in ("qs", "ks"):
        _expect(L, 1, NormRope, **{name: None})
        _expect(L, 2, NormRope, **{name: (-128, 128)})
        _expect(L, 5, NormRope, **{name: (1024 + 4, 128)})
        _expect(L, 2, NormRope, **{name: (1 << 60, 128)})
    # without keys nothing of theirs is looked at
    _expect(L, 6, NormRope, Hk=0, k=None, ks=None, kw=6, ko=None, qo=5 * A)


@pytest.mark.parametrize("a,b", [("qo", "k"), ("qo", "qw"), ("qo", "kw"), ("qo", "pos"), ("ko", "q"), ("ko", "qw"),
                                 ("qo", "ko"), ("qo", "q"), ("ko", "k")])
def test_outputs_overlap_nothing(L, a, b):
    """An output on top of its own input is refused too, where that is not dense."""
    assert NormRope(**{a: getattr(NormRope(), b)}).run(L) == 6
    assert NormRope(**{b: getattr(NormRope(), a) + 10 * 2 * 128 * 2 - 16}).run(L) == 6


def test_in_place_is_the_same_address_and_dense(L):
    dense = dict(qs=(8 * 128, 128), ks=(2 * 128, 128))
    for kw in (dict(qo=A), dict(ko=2 * A)):
        # comes to the last check with it
        other = dict(ko=5 * A) if "qo" in kw else dict(qo=5 * A)
        _expect(L, 6, NormRope, **dense, **kw, **other)
        assert b"positions" in L.kvx_last_error()
    assert NormRope(**dense, qo=A + 256).run(L) == 6
    assert b"q_out overlaps q" in L.kvx_last_error()


def test_an_empty_call_is_checked_and_launches_nothing(L):
    assert NormRope(T=0, q=None, k=None, pos=None, qo=None, ko=None).run(L) == 0
    assert NormRope(T=0, d=96).run(L) == 5
