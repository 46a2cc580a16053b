"""Serving calls on a GPU that is not the current one."""

import numpy as np
import pytest
import torch

from tests.test_gpu_attend8 import _case, _gpu

pytestmark = pytest.mark.gpu


def _steps(kvx, dev):
    """A plan, a store and an attention call on a device; their results on the host."""
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    tables, ring = torch.zeros((2, 4), dtype=torch.int32, device=dev), torch.arange(8, dtype=torch.int32, device=dev)
    plan = kvx.plan_pages(i32(0, 0), i32(20, 5), tables, ring, i32(0, 8), 25, 16)
    g = torch.Generator().manual_seed(800)
    k, v, q = (torch.randn(s, generator=g).to(dev) for s in ((1, 2, 25, 64), (1, 2, 25, 64), (25, 4, 64)))
    pool = torch.zeros((1, 2, 2, 128, 64), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
    scales = torch.ones((1, 2, 2, 8), device=dev)
    kvx.store_cache8(k, v, plan.slots, pool, scales)
    out, lse = kvx.attend_cache8(q, pool[0], scales[0], tables, plan.lens, plan.cu, with_lse=True)
    torch.cuda.synchronize(dev)
    return [t.cpu() for t in (*plan, tables, ring, pool.view(torch.uint8), scales, out, lse)]


def test_calls_run_where_their_tensors_live(gpu_kvx):
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    with torch.cuda.device(0):
        here, there = _steps(gpu_kvx, "cuda:0"), _steps(gpu_kvx, "cuda:1")
        assert torch.cuda.current_device() == 0
    for a, b in zip(here, there):
        assert torch.equal(a, b)


def test_operands_share_a_device(gpu_kvx):
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    a = list(_gpu(_case(np.random.default_rng(801), [40], [3], 2, 4, 64, 16, "bf16")))
    for n in range(6):
        with pytest.raises(ValueError):
            gpu_kvx.attend_cache8(*[t.to("cuda:1") if i == n else t for i, t in enumerate(a)])
