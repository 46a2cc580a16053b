"""Which way a row of token sampling goes, from what the call leaves in the row's workspace (its
layout is the kernels' own: entries of the list and three counters, whether the first launch's list
did not hold, what the third launch did), and that hardly any draw of the example's steps is so near
a border that its test lets it pass."""

import numpy as np
import pytest
import torch

from oracle import serve_oracle as S
from tests.test_gpu_sample import DEV, _check

pytestmark = pytest.mark.gpu
MARK = 0x55555555
LIST, OVER = 0, 1                        # the first launch's list held, or not
UNTOUCHED, DONE, CUT, NARROW = MARK, 0, 1, 2


def _ways(kvx, x, settings, u):
    ws = kvx.sample_workspace(x)
    words = ws.view(torch.int32).view(len(settings), -1)
    words[:, kvx.SAMPLE_COUNTER_BYTES // 4:] = MARK
    _check(kvx, x, settings, u, workspace=ws, exact=lambda b: len(torch.unique(x[b])) == 1)
    return [tuple(r) for r in words[:, [kvx.SAMPLE_COUNTER_BYTES // 4, kvx.SAMPLE_COUNTER_BYTES // 4 + 2]].tolist()]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,V", [(1, 131072), (7, 60013), (300, 20011), (1100, 9001)])
def test_every_way_is_taken(gpu_kvx, B, V, dtype):
    g = np.random.default_rng(B)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    peaked, flat, none = g.standard_normal(V) * 3, np.ones(V), np.full(V, -np.inf)
    rows = [   # logits, setting, what is in the workspace then
        (peaked, (0.8, 50, 0.9, 0.0), (LIST, UNTOUCHED)),
        (peaked, (0.8, 128, 1.0, 0.0), (LIST, UNTOUCHED)),
        (peaked, (0.8, 129, 0.9, 0.0), (MARK, CUT)),
        (peaked, (1.0, 0, 0.9, 0.0), (MARK, CUT)),
        (peaked, (1.0, 0, 1.0, 0.1), (MARK, UNTOUCHED)),
        (peaked, (0.0, 50, 0.9, 0.0), (MARK, UNTOUCHED)),
        (flat, (1.0, 100, 1.0, 0.0), (OVER, NARROW)),
        (flat, (1.0, 0, 0.5, 0.0), (MARK, NARROW)),
        (none, (1.0, 0, 0.5, 0.0), (MARK, DONE)),
        (none, (1.0, 20, 0.5, 0.0), (LIST, UNTOUCHED)),
    ]
    for first in range(0, len(rows), B):
        some = [rows[(first + b) % len(rows)] for b in range(B)]
        x = torch.tensor(np.stack([r[0] for r in some])).to(dt).to(DEV)
        got = _ways(gpu_kvx, x, [r[1] for r in some], g.random(B))
        for (over, mode), (_, setting, want) in zip(got, some):
            assert (over, mode) == want, (setting, over, mode, want)


@pytest.mark.parametrize("name", ["tiny", "qwen3_14b_32b"])
def test_the_examples_draws_are_clear(gpu_kvx, monkeypatch, name):
    from tests import test_gpu_continue as example
    near, draw = [], S.sample_token

    def counted(*a):
        r = draw(*a)
        near.append(r[2])
        return r
    monkeypatch.setattr(S, "sample_token", counted)
    example.test_continuations(gpu_kvx, name)
    assert len(near) == 21 * example.B
    assert sum(n <= example.V * (2.0 ** -44 + 2.0 ** -52) for n in near) <= 1
