"""Host-side checks of kvx_sample_tokens (no GPU needed); see test_abi_serve for the scheme."""

import pytest

from tests.test_abi_host import L  # noqa: F401  (the library fixture)
from tests.test_abi_serve import A, Call, _expect


class Sample(Call):
    entry = "kvx_sample_tokens"

    def __init__(self, **kw):
        self.dtype, self.B, self.V, self.stride = 1, 8, 1000, 1000
        (self.logits, self.u, self.temperature, self.top_k, self.top_p, self.min_p, self.tokens, self.logprob,
         self.ws) = (n * A for n in range(1, 10))
        self.wsb = 1 << 29
        self.__dict__.update(kw)

    def args(self):
        return (self.dtype, self.B, self.V, self.logits, self.stride, self.u, self.temperature, self.top_k, self.top_p,
                self.min_p, self.tokens, self.logprob, self.ws, self.wsb, None)

    spoil = dict(logprob=6 * A)           # on top of min_p


def test_sizes_and_types(L):
    _expect(L, 4, Sample, dtype=2)
    for kw in (dict(B=-1), dict(V=0), dict(V=-5), dict(stride=-1), dict(stride=1 << 60)):
        _expect(L, 2, Sample, **kw)
    for kw in (dict(B=65536), dict(V=(1 << 20) + 1)):
        _expect(L, 5, Sample, **kw)
    _expect(L, 6, Sample, B=1, stride=-1)          # never stepped: comes to the last check
    _expect(L, 6, Sample, stride=0)


def test_operands(L):
    for name in ("logits", "u", "tokens"):
        _expect(L, 1, Sample, **{name: None})
        _expect(L, 5, Sample, **{name: 20 * A + 2})
    for name in ("temperature", "top_k", "top_p"):
        _expect(L, 5, Sample, **{name: 20 * A + 2})
        _expect(L, 6, Sample, **{name: None})
    _expect(L, 5, Sample, min_p=20 * A + 2)
    assert Sample(logprob=20 * A + 1).run(L) == 5
    _expect(L, 5, Sample, dtype=0, logits=20 * A + 1)
    _expect(L, 6, Sample, dtype=0, logits=20 * A + 2)    # bf16 rows begin anywhere


@pytest.mark.parametrize("dtype,B,V", [(0, 1, 1), (1, 8, 1000), (0, 512, 1 << 20), (1, 65535, 7)])
def test_workspace(L, dtype, B, V):
    need = L.kvx_sample_workspace_bytes(dtype, B, V)
    call = dict(dtype=dtype, B=B, V=V, stride=V, logits=100 * A, ws=2000 * A)
    assert need > 0
    _expect(L, 7, Sample, **{**call, "ws": None}, wsb=need)
    _expect(L, 7, Sample, **call, wsb=need - 1)
    _expect(L, 7, Sample, **{**call, "ws": 2000 * A + 64}, wsb=need)
    _expect(L, 6, Sample, **call, wsb=need)


@pytest.mark.parametrize("out", ["tokens", "logprob", "ws"])
@pytest.mark.parametrize("name", ["logits", "u", "temperature", "top_k", "top_p", "min_p"])
def test_outputs_overlap_nothing(L, out, name):
    assert Sample(**{out: getattr(Sample(), name)}).run(L) == 6
    assert Sample(**{name: getattr(Sample(), out) - 28}).run(L) == 6


def test_empty_calls_launch_nothing(L):
    none = dict.fromkeys(("logits", "u", "temperature", "top_k", "top_p", "min_p", "tokens", "logprob", "ws"))
    assert Sample(B=0, **none).run(L) == 0
    assert L.kvx_sample_workspace_bytes(1, 0, 1000) == 0
    for bad in ((2, 8, 1000), (1, -1, 1000), (1, 8, 0), (1, 8, (1 << 20) + 1), (1, 65536, 10)):
        assert L.kvx_sample_workspace_bytes(*bad) == 0
