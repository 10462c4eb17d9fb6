"""A decode step after psv_cache_slots refused a request: with a length of 0 in its place the step leaves that request's cache alone."""
import numpy as np
import pytest
import torch

from paper_2501_08192_amd import binding as psv
from paper_2501_08192_amd import synth
from paper_2501_08192_amd.harness import Session
from test_gpu_cache_rows import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["bf16", "int8"])
def test_a_refused_request_keeps_its_cache(kv):
    batch, mb = 3, 4
    w = synth.Workload("refused", 1, 512, 4, 2, 128, 512, batch, mb * 16, True, (0.0, 0.0), kv_format=kv)
    with Session(w, seed=22) as s:
        lens, new = dev([20, 32, 15]), dev([1, 1, 1])      # the second one needs a block, and there is none
        table = torch.full((batch, mb), -1, dtype=torch.int32, device="cuda")
        table[0, :2], table[1, :2], table[2, :1] = dev([5, 1]), dev([0, 7]), dev([3])
        free, ranges, seq_lens, starts, refused = dev([9]), [dev([1, 1]), dev([0, 0])], dev([0] * batch), dev([0] * 4), dev([0])
        slots, positions, requests = torch.empty(batch, dtype=torch.int64, device="cuda"), dev([0] * batch), dev([0] * batch)
        torch.cuda.synchronize()
        psv.psv_cache_slots(lens, new, table, free, ranges[0], s.pool_blocks, seq_lens, starts, slots, positions, requests, ranges[1], refused, s.main)
        s.main.synchronize()
        assert slots.tolist() == [1 * 16 + 4, -1, 3 * 16 + 15] and seq_lens.tolist() == [21, 32, 16] and refused.item() == 1
        step_lens = torch.where(slots >= 0, seq_lens, 0)
        assert step_lens.dtype == torch.int32
        psv.psv_set_kv(s.ctx, [s.k_pools[0]], [s.v_pools[0]], table, mb, s.pool_blocks, step_lens)
        torch.cuda.synchronize()
        before = [p.clone() for p in (s.k_pools[0], s.v_pools[0])]
        assert torch.isfinite(s.run()).all()
        for a, b in zip(before, (s.k_pools[0], s.v_pools[0])):
            same = [torch.equal(a[i], b[i]) for i in range(s.pool_blocks)]
            assert [i for i, eq in enumerate(same) if not eq] == [1, 3]
