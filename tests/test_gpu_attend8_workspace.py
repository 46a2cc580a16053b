"""What attention calls clear of their workspace: the counters, and nothing else."""

import numpy as np
import pytest
import torch

from tests.test_gpu_attend8 import DEV, _case, _compare, _gpu
from tests.test_gpu_attend8_kernels import _wide

pytestmark = pytest.mark.gpu


def _cases():
    rng = np.random.default_rng(700)
    for lens, news, dtype, d, M in (([9000, 700, 33], [1, 1, 2], "bf16", 128, None),
                                    ([9000, 700, 33], [1, 1, 2], "f32", 64, None),
                                    ([9000, 700], [7, 9], "bf16", 128, 2 ** 14),
                                    ([3000, 700], [130, 97], "bf16", 128, 2 ** 17)):
        c = _case(rng, lens, news, 2, 4, d, 16, dtype)
        yield c if M is None else _wide(c, M)


def test_counters_alone_are_cleared(gpu_kvx):
    """A call without a workspace makes one; what lies behind its counters stays as it was."""
    for c in _cases():
        a = _gpu(c)
        need = gpu_kvx.attend_workspace(a[0], a[1], a[3]).numel()
        torch.cuda.synchronize()
        marks = torch.full((need,), 0x5A, dtype=torch.uint8, device=DEV)
        at = marks.data_ptr()
        del marks
        out, lse = gpu_kvx.attend_cache8(*a, with_lse=True)
        left = torch.empty(need, dtype=torch.uint8, device=DEV)   # the allocator gives the same bytes again
        assert left.data_ptr() == at
        head = gpu_kvx.ATTEND_COUNTER_BYTES
        assert not left[:head].any()
        assert (left[head:] == 0x5A).float().mean() > 0.5     # but for partial sums
        _compare(c, out, lse, c["q"].shape[2] ** -0.5, "workspace made by the call")


def test_what_lies_behind_the_counters_does_not_matter(gpu_kvx):
    for c in _cases():
        a = _gpu(c)
        clean = gpu_kvx.attend_cache8(*a, with_lse=True)
        for fill in (0xFF, 0x7F):       # NaN as fp32, and a large number
            ws = gpu_kvx.attend_workspace(a[0], a[1], a[3])
            ws[gpu_kvx.ATTEND_COUNTER_BYTES:] = fill
            for _ in range(2):
                out = gpu_kvx.attend_cache8(*a, with_lse=True, workspace=ws)
                assert torch.equal(out[0], clean[0]) and torch.equal(out[1], clean[1])
            assert not ws[:gpu_kvx.ATTEND_COUNTER_BYTES].any()


def test_a_call_without_a_workspace_in_a_graph(gpu_kvx):
    for c in _cases():
        a = _gpu(c)
        eager = gpu_kvx.attend_cache8(*a, with_lse=True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = gpu_kvx.attend_cache8(*a, with_lse=True)
        for _ in range(3):
            out.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
            gpu_kvx.attend_cache8(*a)
