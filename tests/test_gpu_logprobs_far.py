"""psv_logprobs and its parts where logit times scale is large: logits far from zero, pieces and shards that a mask filled with a finite
value, and the whole documented range of scales."""
import math

import numpy as np
import pytest
import torch

from test_gpu_logprobs import TYPES, check_values, given, logits, reference, run

pytestmark = pytest.mark.gpu
F32_MAX = float(np.finfo(np.float32).max)


def in_range(a):
    """What 32 bits cannot hold is infinite there."""
    return np.where(np.asarray(a) < -F32_MAX, -math.inf, a)


def check(x, tokens, scale, top=5, **kw):
    """The tolerances of check_values hold as they stand: a column's exponent is a difference, a product with a rounded constant and one more
    rounding, whatever the largest logit is."""
    out = run(x, tokens, scale, top, **kw)
    lp, ent, best, ids, spread = reference(x.cpu(), tokens, scale, top)
    check_values(out[0], in_range(lp), spread)
    check_values(out[1], ent, spread, entropy=True)
    assert np.array_equal(out[3].cpu().numpy(), ids)
    check_values(out[2], in_range(best), spread)


SCALES = [2.0 ** k for k in range(-32, 33, 8)] + [0.75, 300007424.0, 1000013824.0, 3999989760.0]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_rows_far_from_zero(dtype, scale):
    """Largest logits of 1.37 times every power of two that the type holds, of both signs, and others up to 40 of its steps below; a
    row of equal ones beside each.  Some of the rows of every scale have differences that count."""
    t, v = TYPES[dtype], 3001
    step = torch.finfo(t).eps
    gen = torch.Generator().manual_seed(31)
    rows = []
    for k in range(2, 16 if dtype == "f16" else 127, 3):
        for sign in (1.0, -1.0):
            m = torch.tensor(sign * 1.37 * 2.0 ** k, dtype=t).double()
            below = torch.randint(0, 41, (v,), generator=gen).double() * step * 2.0 ** k
            rows += [(m - below).to(t), m.expand(v).to(t)]
    x = torch.stack(rows).cuda()
    assert torch.isfinite(x).all()
    tokens = given(len(rows), v, 2, 5)
    check(x, tokens, scale)
    check(x, tokens, scale, shards=[1000, 2001])
    check(x, tokens, scale, shards=[v], records=3)


def fills(dtype):
    return [-65504.0, 60000.0] if dtype == "f16" else [-1e9, -9.9992e9, -1e10, -1e12, -1e15, -1e20, -1e26, -3e38, 1e10, 1e20]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("scale", [1.0, 0.625, 100000.0])
def test_a_piece_or_a_shard_that_is_filled_with_a_finite_value(dtype, scale):
    """Ordinary logits beside one piece, one shard, or all but one column, that hold a far value."""
    values, v = fills(dtype), 40000
    x = logits(3 * len(values), v, dtype, seed=11)
    for i, value in enumerate(values):
        x[3 * i, 4000:8000] = value
        x[3 * i + 1, 16000:24000] = value
        x[3 * i + 2] = value
        x[3 * i + 2, 17] = 3.0
    tokens = given(len(x), v, 4, 11)
    tokens[:, 1], tokens[:, 2] = 4001, 17
    check(x, tokens, scale, top=20)
    check(x, tokens, scale, top=20, shards=[16000, 8000, 16000])
    check(x, tokens, scale, top=0, shards=[4000, 4000, 8000, 8000, 16000])


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("v", [1000, 9000, 33000])
def test_ordinary_logits_at_every_scale(dtype, v):
    x, tokens = logits(24, v, dtype, seed=v, size=10.0), given(24, v, 2, v)
    x[3] = 7.0
    for scale in SCALES:
        check(x, tokens, scale)
        check(x, tokens, scale, top=9, shards=[v - v // 3, v // 3])


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_far_rows_in_the_largest_pieces(dtype):
    """128 columns a lane, by the rule and by asking for one record."""
    x, tokens = logits(2100, 17003, dtype, seed=12), given(2100, 17003, 1, 12)
    far = 60000.0 if dtype == "f16" else 1e11
    x[:50] -= far
    x[50:60] = -far
    x[60:70] += far
    check(x[:90], tokens[:90], 400.0, top=9, shards=[17003], records=1)
    out = run(x, tokens, 400.0, 9)
    some = torch.arange(0, 2100, 7)
    some[:12] = torch.arange(48, 72, 2)
    lp, ent, best, ids, spread = reference(x.cpu()[some], tokens[some], 400.0, 9)
    out = [o.cpu()[some] for o in out]
    check_values(out[0], lp, spread)
    check_values(out[1], ent, spread, entropy=True)
    assert np.array_equal(out[3].numpy(), ids)
    check_values(out[2], best, spread)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, 0.25, 2.0 ** -20, 2.0 ** -32])
def test_logits_whose_difference_passes_32_bits(dtype, scale):
    """A finite logit has a finite log probability wherever 32 bits hold it."""
    x = logits(4, 5000, dtype, seed=13)
    x[0, 10], x[0, 4000] = 3e38, -3e38
    x[1, ::2], x[1, 1::2] = 3.3e38, -3.3e38
    x[2, 4900] = -3.3e38
    x[3] = torch.finfo(TYPES[dtype]).min
    x[3, 1] = 2e38
    tokens = torch.tensor([[10, 4000, 0, 4999]] * 4)
    for kw in (dict(), dict(shards=[2500, 2500]), dict(shards=[1, 4999])):
        check(x, tokens, scale, top=8, **kw)
