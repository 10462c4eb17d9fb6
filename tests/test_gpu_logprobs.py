"""psv_logprobs (whole and in shards) against log probabilities, entropy and alternatives in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2501_08192_amd import binding as psv
from test_gpu_rotate import TYPES

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


def reference(x, tokens, scale, top):
    """On the host, in 64 bits; alternatives by (largest, lowest id)."""
    z = x.double().numpy()
    n, v = z.shape
    lp, ent = np.zeros((n, tokens.shape[1])), np.zeros(n)
    ids, best = np.full((n, top), -1, np.int64), np.full((n, top), -INF)
    spread = np.zeros(n)
    for r in range(n):
        row = z[r]
        bad = np.isnan(row).any() or (row == INF).any()
        none = not bad and (row == -INF).all()
        if bad:
            logp = np.full(v, NAN)
        elif none:
            logp = np.full(v, -INF)
        else:
            d = (row - row.max()) * scale
            with np.errstate(divide="ignore"):
                logp = d - math.log(np.exp(d).sum())
        with np.errstate(invalid="ignore"):
            p = np.exp(logp)
            ent[r] = NAN if bad else -np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0).sum()
        for k, t in enumerate(tokens[r].tolist()):
            lp[r, k] = 0.0 if t < 0 else NAN if t >= v else logp[t]
        if bad:
            best[r] = NAN
        else:
            order = np.argsort(-row, kind="stable")[:top]
            order = order[row[order] > -INF]
            ids[r, :len(order)], best[r, :len(order)] = order, logp[order]
        spread[r] = math.log(v) + 1.0
    return lp, ent, best, ids, spread


def check_values(got, want, spread, entropy=False):
    """ln S: an exponent is off by 3 half steps of 2^-24 of its size, on average at most ln n of the row; a lane adds up to 64 terms, a
    workgroup 256 lanes in a tree and a row up to 256 records the same way: (3 ln n + 64 + 8 + 8) 2^-24 of S, and so of ln S absolutely.
    The hardware's exponential and logarithm are good to 2 steps of 2^-23.  The differences from the largest: three more half steps of
    their size.  The entropy's second sum carries the same relative error, times its size, at most ln n."""
    got, want = got.cpu().double().numpy(), np.asarray(want)
    rel = (3 * spread + 64 + 8 + 8 + 8) * 2.0 ** -24
    tol = rel * (1 + spread) if entropy else rel[:, None] + np.abs(np.where(np.isfinite(want), want, 0.0)) * 2.0 ** -21
    off = np.abs(np.where(np.isfinite(got), got, 0.0) - np.where(np.isfinite(want), want, 0.0))
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert (same | (np.isfinite(want) & np.isfinite(got) & (off <= tol))).all(), (got, want)


def outputs(n, given, top):
    f = dict(dtype=torch.float32, device="cuda")
    return (torch.full((n, given), 9.0, **f), torch.full((n,), 9.0, **f), torch.full((n, top), 9.0, **f), torch.full((n, top), 9, dtype=torch.int32, device="cuda"))


def run(x, tokens, scale, top, shards=None, records=0):
    """x on the device; shards: widths of the vocabulary's slices, or None for the call that has it whole."""
    n, v = x.shape
    given = tokens.shape[1]
    t, stream = tokens.to(torch.int32).cuda(), torch.cuda.current_stream()
    out = outputs(n, given, top)
    if shards is None:
        ws = torch.full((psv.psv_logprobs_bytes(n, psv.psv_logprobs_records(n, v), given, top),), 255, dtype=torch.uint8, device="cuda")
        psv.psv_logprobs(x, t, scale, *out, ws, stream)
    else:
        records = records or psv.psv_logprobs_records(n, max(shards))
        size = psv.psv_logprobs_bytes(n, records, given, top)
        parts, at = torch.full((len(shards), size // 4), NAN, device="cuda"), 0
        for part, width in zip(parts, shards):
            psv.psv_logprobs_part(x[:, at:at + width], t, scale, top, part, stream, first_token=at, vocab=v, records=records)
            at += width
        assert at == v
        psv.psv_logprobs_join(n, t, scale, v, records, len(shards), *out, parts, stream, top=top)
    torch.cuda.synchronize()
    return out


def check(x, tokens, scale=1.0, top=5, **kw):
    out = run(x, tokens, scale, top, **kw)
    lp, ent, best, ids, spread = reference(x.cpu(), tokens, scale, top)
    check_values(out[0], lp, spread)
    check_values(out[1], ent, spread, entropy=True)
    assert np.array_equal(out[3].cpu().numpy(), ids)
    check_values(out[2], best, spread)
    return out


def logits(n, v, dtype, seed=0, masked=0.0, size=2.5):
    gen = torch.Generator().manual_seed(seed)
    x = size * torch.randn(n, v, generator=gen)
    if masked:
        x[torch.rand(n, v, generator=gen) < masked] = -INF
    return x.to(TYPES[dtype]).cuda()


def given(n, v, k, seed=0):
    return torch.randint(0, v, (n, k), generator=torch.Generator().manual_seed(seed + 1000))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,v", [(1, 1), (1, 2), (3, 7), (2, 8), (2, 9), (5, 255), (4, 1000), (1, 2047), (3, 2048), (2, 2049), (7, 4099), (1, 16384), (2, 16385), (61, 32003),
                                 (1, 128256), (3, 151936)])
def test_against_64_bits(n, v, dtype):
    check(logits(n, v, dtype, seed=v), given(n, v, 2, v), top=min(20, 32))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,v", [(600, 3000), (300, 16000), (130, 33000), (1100, 130)])
def test_pieces_of_every_size(n, v, dtype):
    """Rows enough for pieces of 8 to 64 columns a lane."""
    check(logits(n, v, dtype, seed=n), given(n, v, 1, n), top=3, scale=0.7)


@pytest.mark.parametrize("top", [0, 1, 2, 31, 32])
@pytest.mark.parametrize("k", [0, 1, 32])
def test_numbers_of_given_tokens_and_alternatives(top, k):
    for n, v in ((2, 5), (3, 5000), (2, 40000)):
        check(logits(n, v, "f32", seed=top), given(n, v, k, top), top=top)
        check(logits(n, v, "bf16", seed=top), given(n, v, k, top), top=top, shards=[v - v // 2, v // 2])


def test_outputs_that_are_not_wanted():
    x, t = logits(4, 3000, "f32"), given(4, 3000, 1)
    lp, ent, top_lp, top = run(x, t, 1.0, 4)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    a, b = torch.zeros_like(lp), torch.zeros_like(ent)
    psv.psv_logprobs(x, t.int().cuda(), 1.0, a, None, None, None, ws, torch.cuda.current_stream())
    psv.psv_logprobs(x, None, 1.0, None, b, None, None, ws, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(a, lp) and torch.equal(b, ent)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("masked", [0.5, 0.99, 0.9999])
def test_masked_logits(dtype, masked):
    check(logits(9, 20000, dtype, seed=3, masked=masked), given(9, 20000, 8, 3), top=20)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_rows_that_leave_nothing_or_are_not_numbers(dtype):
    x = logits(10, 5000, dtype, seed=4)
    x[0] = -INF
    x[1] = -INF
    x[1, 4999] = 3.0
    x[2, 77] = NAN
    x[3, 4000] = INF
    x[4] = NAN
    x[5] = torch.finfo(x.dtype).min
    x[6] = torch.finfo(x.dtype).min
    x[6, 2500] = 1.0
    x[7] = torch.finfo(x.dtype).max
    x[8, :2048] = -INF
    x[9, 3], x[9, 4] = INF, -INF
    t = torch.tensor([[0, 4999, -1, 5000, 77]] * 10)
    for kw in (dict(), dict(shards=[2500, 2500]), dict(shards=[1, 4999]), dict(shards=[4096, 904])):
        check(x, t, top=7, **kw)
    check(x[:, :1], torch.zeros(10, 1).long(), top=3)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_equal_logits_go_to_the_lowest_id(dtype):
    n, v = 8, 40000
    x = torch.zeros(n, v)
    x[1] = -3.0
    x[2, ::2] = -0.0                                       # zeros of both signs are equal
    x[3] = torch.arange(v) % 2
    x[4] = torch.arange(v).flip(0) // 7000                  # long steps, descending
    x[5] = torch.arange(v) // 7000
    x[6] = (torch.arange(v) % 999 == 0).float()
    x[7] = torch.where(torch.arange(v) < 39990, -INF, 5.0)  # ten equal ones at the end
    for top in (1, 20, 32):
        check(x.to(TYPES[dtype]).cuda(), given(n, v, 1), top=top)
        check(x.to(TYPES[dtype]).cuda(), given(n, v, 1), top=top, shards=[16000, 16000, 8000])


def test_a_lane_that_holds_all_the_largest():
    """Columns that one lane of a piece has: the list of candidates is as long as it gets."""
    for dtype, vec in (("f32", 4), ("bf16", 8)):
        x = logits(2000, 16384, dtype, size=0.5)[:8]
        cols = (torch.arange(64 // vec)[:, None] * 256 * vec + torch.arange(vec)[None]).reshape(-1)
        for lanes in (1, 31, 32):
            for lane in range(lanes):
                x[:, (cols + lane * vec).cuda()] = (20.0 + torch.arange(64.0) / 8).to(x.dtype).cuda()
            check(x, given(8, 16384, 1), top=32, shards=[16384], records=1)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_the_largest_pieces(dtype):
    """128 columns a lane: by the rule (thousands of pieces), and by asking for one record; ties, lanes that hold all the largest, few left."""
    n, v = 2100, 17003
    x = logits(n, v, dtype, seed=9)
    x[0], x[1, :] = 0.0, -INF
    x[1, v - 1] = 1.0
    x[2, ::7] = 30.0
    t = given(n, v, 1, 9)
    check(x, t, top=20)
    y = logits(6, 32768, dtype, seed=10, size=0.5)
    y[0], y[1, 5:], y[2, 100] = -2.0, -INF, NAN
    vec = 4 if dtype == "f32" else 8
    cols = (torch.arange(128 // vec)[:, None] * 256 * vec + torch.arange(vec)[None]).reshape(-1)
    for lane in range(32):
        y[3:, (cols + lane * vec).cuda()] = (20.0 + torch.arange(128.0) / 8).to(y.dtype).cuda()
    for top in (1, 32):
        check(y, given(6, 32768, 2), top=top, shards=[32768], records=1)
        check(y[:, :30001], given(6, 30001, 2), top=top, shards=[30001], records=1)


def test_ascending_and_far_offset_logits():
    v = 30000
    x = torch.stack([torch.linspace(-20, 20, v), torch.linspace(20, -20, v), 1.0e4 + 3 * torch.randn(v, generator=torch.Generator().manual_seed(2)),
                     -1.0e6 + torch.arange(v) % 100, 1e30 * torch.randn(v, generator=torch.Generator().manual_seed(3))]).cuda()
    check(x, given(5, v, 3), top=11)
    check(x, given(5, v, 3), top=11, scale=1e-3)
    check(x[:3], given(3, v, 3), top=11, scale=50.0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_row_strides_and_alignment(dtype):
    base = logits(6, 3100, dtype, seed=8)
    for x in (base[:, 1:3000], base[:, 3:2052], base[::2, 5:6], base[:, 7:], base[1:2, 2:1500], base[:1].expand(4, 3100)):
        check(x, given(x.shape[0], x.shape[1], 2), top=6)


@pytest.mark.parametrize("widths,records", [([16032] * 8, 0), ([501, 500, 1, 3000], 0), ([1000, 3], 5), ([4096], 2), ([40] * 100, 1), ([9, 9], 128)])
def test_shards_agree_with_the_whole(widths, records):
    v, n = sum(widths), 6
    x, t = logits(n, v, "bf16", seed=6, masked=0.1), given(n, v, 3, 6)
    t[0, 0], t[1, 1], t[2, 2], t[3, 0] = -1, v, 2**31 - 1, v - 1
    check(x, t, scale=0.9, top=9, shards=widths, records=records)


def test_no_rows_the_same_bits_again_other_streams_and_a_captured_graph():
    x, t = logits(33, 9000, "f16", seed=7), given(33, 9000, 1, 7)
    run(x[:0], t[:0], 1.0, 3)
    want = run(x, t, 1.0, 20)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(x, t, 1.0, 20), want))
    tokens = t.int().cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    size = psv.psv_logprobs_bytes(33, psv.psv_logprobs_records(33, 9000), 1, 20)
    outs, spaces = [outputs(33, 1, 20) for _ in streams], [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, o, w in zip(streams, outs, spaces):
            psv.psv_logprobs(x, tokens, 1.0, *o, w, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, want))
    # two graphs that share a workspace, replayed one after the other
    graphs, y, space = [], [x.clone(), x.flip(1).contiguous()], spaces[0]
    for src, o in zip(y, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            psv.psv_logprobs(src, tokens, 1.0, *o, space, torch.cuda.current_stream())
        graphs.append(g)
    for k in range(3):
        for src, g, o in zip(y, graphs, outs):
            src.copy_(logits(33, 9000, "f16", seed=50 + k))
            g.replay()
        torch.cuda.synchronize()
        for src, o in zip(y, outs):
            assert all(torch.equal(a, b) for a, b in zip(run(src, t, 1.0, 20), o))
