"""Norm and rotation, attention over shared prefixes and sampling on a GPU that is not the current
one."""

import pytest
import torch

from paper_2608_03893_amd import synth

pytestmark = pytest.mark.gpu


def _operands(dev):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    g = torch.Generator().manual_seed(810)
    r = lambda *s: torch.randn(s, generator=g).to(dev)  # noqa: E731
    pool = torch.randint(0, 96, (2, 2, 8 * 16, 64), generator=g, dtype=torch.uint8).to(dev).view(torch.float8_e4m3fn)
    rope = [r(3, 4, 64), r(3, 2, 64), r(64), r(64), i32(20, 21, 22)]
    prefix = [r(3, 4, 64), pool, torch.ones((2, 2, 8), device=dev), i32(0, 1).view(1, 2), i32(20), i32(0, 2),
              i32(2, 3, 4, 5).view(2, 2), i32(17, 1), i32(0, 2, 3)]
    sample = [r(3, 1000), torch.tensor([0.1, 0.5, 0.9], device=dev), torch.ones(3, device=dev), i32(0, 5, 200),
              torch.tensor([0.9, 1.0, 0.8], device=dev)]
    return rope, prefix, sample


def _norm_rope(kvx, q, k, qw, kw, pos):
    return kvx.norm_rope(q, k, qw, kw, synth.rope_dict(1e6), pos)


def _calls(kvx):
    return (lambda *a: _norm_rope(kvx, *a), lambda *a: (kvx.attend_prefix8(*a),), lambda *a: (kvx.sample_tokens(*a),))


def test_they_run_where_their_tensors_live(gpu_kvx):
    results = []
    with torch.cuda.device(0):
        for dev in ("cuda:0", "cuda:1") if torch.cuda.device_count() > 1 else ("cuda:0", "cuda"):
            got = [y for f, a in zip(_calls(gpu_kvx), _operands(dev)) for y in f(*a)]
            torch.cuda.synchronize(dev)
            results.append([y.cpu() for y in got])
        assert torch.cuda.current_device() == 0
    for a, b in zip(*results):
        assert torch.equal(a, b)
        assert not a.is_floating_point() or torch.isfinite(a).all()


def test_operands_share_a_device(gpu_kvx):
    """Another GPU's tensors are refused, as the host's are."""
    other = "cuda:1" if torch.cuda.device_count() > 1 else "cpu"
    for f, a in zip(_calls(gpu_kvx), _operands("cuda:0")):
        for n in range(len(a)):
            with pytest.raises(ValueError):
                f(*[t.to(other) if i == n else t for i, t in enumerate(a)])
