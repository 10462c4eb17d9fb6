"""Calls of as many rows as are allowed, in the shapes whose workgroups take the fewest rows."""
import numpy as np
import pytest
import torch

from paper_2501_08192_amd import binding as psv
from test_gpu_cache_rows import Pools, dev
from test_gpu_rotate import bound, rotated

pytestmark = pytest.mark.gpu
MOST_ROWS, MOST_HEADS = 1 << 24, 1 << 28


def some(n, seed):
    rng = np.random.default_rng(seed)
    return torch.as_tensor(np.unique(np.concatenate([np.arange(600), n - 1 - np.arange(600), rng.integers(0, n, size=2000)])))


def test_rotation_of_the_most_rows():
    heads, dim = 3, 130      # 129 pieces a head: a workgroup has one in hand
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("less than 24 GiB free")
    rope = psv.psv_rope_plan(dims=2, theta=10000.0)
    x = torch.randn(1, heads, dim, generator=torch.Generator().manual_seed(1)).half().cuda()
    p = torch.arange(MOST_ROWS, dtype=torch.int32, device="cuda")
    y = torch.full((MOST_ROWS, heads, dim), float("nan"), dtype=torch.float16, device="cuda")
    psv.psv_rotate(x.expand(MOST_ROWS, heads, dim), y, p, rope, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for part in y.split(1 << 20):
        assert torch.equal(part[..., 2:], x[..., 2:].expand(len(part), heads, dim - 2)) and not part[..., :2].isnan().any()
    at = some(MOST_ROWS, 1)
    want, size = rotated(x.cpu().expand(len(at), heads, dim), at, rope)
    assert ((y[at.cuda()].cpu().double() - want).abs() <= bound(want, size, torch.float16)).all()


@pytest.mark.parametrize("rows,nkv,layout", [(MOST_HEADS // 25, 25, "head"), (MOST_ROWS, 13, "token")])
def test_append_of_the_most_rows(rows, nkv, layout):
    """Nearly all rows without a place; those that have one spread over the call."""
    blocks = 8
    pools = Pools(blocks, nkv, "bf16", layout, 2)
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn(1, nkv, 128, generator=gen).cuda() for _ in range(2))
    at = some(rows, 2)
    at = at[torch.as_tensor(np.random.default_rng(3).permutation(len(at))[:blocks * 16 - 1])].sort().values
    at[-1] = rows - 1
    slots = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    places = dev(np.random.default_rng(4).permutation(blocks * 16)[:len(at)], torch.int64)
    slots[at.cuda()] = places
    p = torch.arange(rows, dtype=torch.int32, device="cuda")
    rope = psv.psv_rope_plan(theta=10000.0)
    psv.psv_cache_append(None, k.expand(rows, nkv, 128), v.expand(rows, nkv, 128), None, p, slots, pools.cache, rope, torch.cuda.current_stream())
    torch.cuda.synchronize()
    (kc, _), (vc, _) = pools.rows(pools.gpu, places.cpu())
    want, size = rotated(k.cpu().expand(len(at), nkv, 128), at, rope)
    assert ((kc - want).abs() <= bound(want, size, torch.bfloat16)).all()
    assert torch.equal(vc, v.cpu().bfloat16().double().expand(len(at), nkv, 128))
    rest = np.setdiff1d(np.arange(blocks * 16), places.cpu())
    for (a, _), (b, _) in zip(pools.rows(pools.gpu, rest), pools.rows(pools.before, rest)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("widths,records", [([40] * 256, 1), ([9] * 128 + [33] * 128, 1), ([700] * 2, 128), ([3000] * 16, 16)])
def test_log_probabilities_joined_from_the_most_records(widths, records):
    """256 records of 32 alternatives: ordinary rows, rows of equal logits, steps of equal ones, rows that one record has all the largest of."""
    from test_gpu_logprobs import check, given, logits
    v = sum(widths)
    x = logits(8, v, "bf16", seed=14)
    x[1] = 0.0
    x[2] = (torch.arange(v) // 50 % 7).bfloat16().cuda()
    x[3] = (torch.arange(v) % 31 == 0).bfloat16().cuda()
    x[4, v - 40:] = 20.0
    x[5] = -float("inf")
    x[5, ::max(1, v // 20)] = 1.0
    x[6] = torch.arange(v, 0, -1).bfloat16().cuda() / 64
    x[7, widths[0]:] = -1e10
    check(x, given(8, v, 2, 14), top=32, shards=widths, records=records)
    check(x, given(8, v, 2, 14), top=3, shards=widths, records=records)
