"""psv_cache_append of rows that hold NaN and infinities into an int8 cache: codes and scales by the rule of the decode step, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2501_08192_amd import binding as psv
from test_gpu_cache_rows import Pools, dev
from test_gpu_rotate import TYPES

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def by_the_rule(rows):
    """In single precision; maxima and the clamp pass over what is not a number, which leaves a quotient of it at the lower end."""
    x = rows.float().numpy()
    most = np.where(np.isnan(x), 0.0, np.abs(x)).max(-1)
    scale = np.where(most > 0, most / np.float32(127.0), np.float32(1.0)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        q = x / scale[..., None]
    return np.where(np.isnan(q), -127.0, np.clip(np.rint(q), -127, 127)), scale


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("scattered", [False, True])
def test_codes_of_rows_that_are_not_numbers(dtype, scattered):
    gen = torch.Generator().manual_seed(6)
    n, nkv = 40, 3
    v = torch.randn(n, nkv, 128, generator=gen)
    v[1, :, 3] = NAN
    v[2, :, ::7] = NAN
    v[3] = NAN
    v[4, :, 127] = INF
    v[5, :, 0] = -INF
    v[6, :, 64:] = INF
    v[7, 0, 5], v[7, 0, 6], v[7, 1, 5] = INF, NAN, -NAN
    v[8] = 0.0
    v[8, :, 9] = NAN
    v[9:20:2, 1, 40] = NAN
    v[20:, :, 100] = torch.where(torch.arange(20) % 3 == 0, NAN, 1.5)[:, None]
    v = v.to(TYPES[dtype])
    k = v.flip(0).contiguous()
    pools = Pools(4, nkv, "int8", "head", 6)
    at = np.random.default_rng(6).permutation(64)[:n] if scattered else np.arange(5, 5 + n)
    psv.psv_cache_append(None, k.cuda(), v.cuda(), None, None, dev(at, torch.int64), pools.cache, None, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for rows, (codes, scales) in zip((k, v), pools.rows(pools.gpu, at)):
        want, scale = by_the_rule(rows)
        assert np.array_equal(scales.numpy(), scale)
        assert np.array_equal(codes.numpy(), want)
