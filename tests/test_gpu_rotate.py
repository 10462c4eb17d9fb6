"""psv_rotate against the rotation in 64 bits, and psv_set_rope against the keys that a decode step appends."""
import numpy as np
import pytest
import torch

from paper_2501_08192_amd import binding as psv
from paper_2501_08192_amd import synth
from paper_2501_08192_amd.harness import Session

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rotated(x, positions, rope, transpose=False):
    """[rows, heads, dim] in 64 bits, and the sum of the magnitudes that every element is made of."""
    n = rope.dims // 2
    freq = torch.tensor(list(rope.freq)[:n], dtype=torch.float64)
    angle = positions.double()[:, None, None] * freq
    c, s = torch.cos(angle) * rope.magnitude, torch.sin(angle) * rope.magnitude * (-1.0 if transpose else 1.0)
    x = x.double()
    y, size = x.clone(), x.abs().clone()
    lo, hi = (slice(0, n), slice(n, 2 * n)) if rope.pairing == 0 else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    size[..., lo] = size[..., hi] = (a.abs() + b.abs()) * abs(rope.magnitude)
    return y, size


def bound(want, size, dtype):
    """Sine and cosine are rounded to 32 bits, then one product, one multiply-add: three half steps of 2^-24 of each of the two terms;
    the result's own rounding is half a step of its type (and half the smallest step of f16, 2^-25)."""
    b = 3 * 2.0 ** -24 * size
    return b if dtype == torch.float32 else b + want.abs() * torch.finfo(dtype).eps / 2 * (1 + 2.0 ** -20) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def check(y, x, positions, rope, transpose=False):
    want, size = rotated(x.cpu(), positions.cpu(), rope, transpose)
    err = (y.cpu().double() - want).abs()
    assert (err <= bound(want, size, y.dtype)).all(), (err.max().item(), (err / bound(want, size, y.dtype)).max().item())
    n = rope.dims
    assert torch.equal(y[..., n:].cpu(), x[..., n:].cpu())


def rows(seed, n, heads, dim, dtype):
    return torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(seed)).to(TYPES[dtype]).cuda()


def run(x, y, positions, rope, **kw):
    psv.psv_rotate(x, y, positions, rope, torch.cuda.current_stream(), **kw)
    torch.cuda.synchronize()
    return y


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("n,heads,dim,dims", [(1, 1, 128, 128), (1, 40, 128, 128), (3, 1, 64, 32), (17, 5, 128, 64), (257, 3, 96, 96), (64, 8, 128, 128),
                                              (2049, 2, 80, 80), (8195, 1, 128, 128), (33, 2, 256, 256), (5, 3, 26, 26), (9, 2, 7, 2),
                                              (4, 1, 1024, 256), (2, 3, 1023, 254), (31, 7, 72, 24), (2050, 1, 40, 24)])
def test_against_64_bits(n, heads, dim, dims, pairing, dtype):
    x = rows(n + dim, n, heads, dim, dtype)
    rope = psv.psv_rope_plan(dims=dims, pairing=pairing, theta=10000.0)
    p = torch.arange(100, 100 + n, dtype=torch.int32, device="cuda")
    check(run(x, torch.full_like(x, float("nan")), p, rope), x, p, rope)


@pytest.mark.parametrize("scaling,kw", [("linear", dict(factor=4.0)), ("turns", dict(factor=8.0)),
                                        ("channel", dict(factor=16.0, high_turns=32.0, trained_context=4096.0, magnitude=1.27))])
@pytest.mark.parametrize("transpose", [False, True])
def test_scaled_frequencies_and_far_positions(scaling, kw, transpose):
    x = rows(5, 12, 4, 128, "f32")
    p = torch.tensor([0, 1, 2, 4095, 4096, 131071, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -1, -70000, -(1 << 31)], dtype=torch.int64).int().cuda()
    rope = psv.psv_rope_plan(scaling=scaling, **kw)
    check(run(x, torch.empty_like(x), p, rope, transpose=transpose), x, p, rope, transpose)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_strides_alignment_and_what_lies_between(pairing, dtype):
    rope = psv.psv_rope_plan(dims=64, pairing=pairing)
    n, heads, dim = 37, 6, 128
    p = torch.arange(n, dtype=torch.int32, device="cuda") * 3
    base = rows(9, n, heads + 3, dim + 8, dtype)
    for x in (base[:, 1:1 + heads, :dim], base[:, 2:2 + heads, 1:1 + dim], base[:, :heads, 8:], base.transpose(0, 1).contiguous().transpose(0, 1)[:, :heads, :dim]):
        out = torch.full((n, heads + 1, dim + 16), 7.0, dtype=x.dtype, device="cuda")
        for y in (out[:, 1:, 8:8 + dim], out[:, :heads, 3:3 + dim]):
            out.fill_(7.0)
            check(run(x, y, p, rope), x, p, rope)
            keep = torch.ones_like(out, dtype=torch.bool)
            keep.as_strided(y.shape, y.stride(), y.storage_offset())[:] = False
            assert (out[keep] == 7.0).all()
    by_head = torch.empty(heads, n, dim, dtype=base.dtype, device="cuda").transpose(0, 1)      # rows within heads
    check(run(base[:, :heads, :dim], by_head, p, rope), base[:, :heads, :dim], p, rope)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_in_place_and_broadcast_inputs(dtype):
    rope = psv.psv_rope_plan()
    p = torch.arange(50, dtype=torch.int32, device="cuda")
    x = rows(3, 50, 9, 128, dtype)
    part = x.clone()
    check(run(part[:, 2:7], part[:, 2:7], p, rope), x[:, 2:7], p, rope)
    assert torch.equal(part[:, :2], x[:, :2]) and torch.equal(part[:, 7:], x[:, 7:])
    one = x[:1, :1].expand(50, 9, 128)
    check(run(one, torch.empty_like(x), p, rope), one, p, rope)


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_the_transposed_rotation_is_the_gradient(pairing):
    """Of L = sum(g * rotate(x)): against differences of the forward pass, which is linear, so that a step of 1 is exact but for rounding;
    and for magnitude 1 it undoes the rotation."""
    rope = psv.psv_rope_plan(dims=64, pairing=pairing, scaling="channel", factor=8.0, high_turns=32.0, magnitude=1.3)
    x, g = rows(1, 6, 2, 128, "f32"), rows(2, 6, 2, 128, "f32")
    p = torch.tensor([0, 1, 77, 5000, 100000, 9], dtype=torch.int32, device="cuda")
    dx = run(g, torch.empty_like(g), p, rope, transpose=True)
    check(dx, g, p, rope, transpose=True)
    for at in [(0, 0, 0), (1, 1, 3), (2, 0, 32), (3, 1, 63), (4, 0, 5), (5, 1, 100), (2, 1, 127)]:
        step = torch.zeros_like(x)
        step[at] = 1.0
        far, near = (run(x + s * step, torch.empty_like(x), p, rope).double() for s in (1.0, -1.0))
        diff = ((far - near) / 2 * g.double()).sum().item()
        # each of two elements is off by 3 * 2^-24 * 1.3 * (|a| + |b|), |a|, |b| <= 6 here
        assert abs(diff - dx[at].item()) <= 2 * 2.0 ** -20 * 1.3 * 12 * g.abs().max().item()
    plain = psv.psv_rope_plan(dims=64, pairing=pairing)
    back = run(run(x, torch.empty_like(x), p, plain), torch.empty_like(x), p, plain, transpose=True)
    assert ((back - x).abs() <= 6 * 2.0 ** -24 * 4 * 6.0).all()


def test_no_rows_another_stream_and_a_captured_graph():
    rope = psv.psv_rope_plan()
    x = rows(4, 65, 3, 128, "bf16")
    p = torch.arange(65, dtype=torch.int32, device="cuda")
    run(x[:0], x[:0], p[:0], rope)
    want = run(x, torch.empty_like(x), p, rope)
    side, y = torch.cuda.Stream(), torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    psv.psv_rotate(x, y, p, rope, side)
    side.synchronize()
    assert torch.equal(y, want)
    graph, z = torch.cuda.CUDAGraph(), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        psv.psv_rotate(x, z, p, rope, torch.cuda.current_stream())
    for k in range(3):
        x.copy_(rows(40 + k, 65, 3, 128, "bf16"))
        p.add_(1000)
        want = run(x, torch.empty_like(x), p, rope)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want)


# ---- psv_set_rope --------------------------------------------------------------------------------------------------------------

def small(batch, context=200, hidden=512, nq=4, nkv=2, **kw):
    return synth.Workload("rope", 1, hidden, nq, nkv, 128, 512, batch, context, False, (0.0, 0.0), **kw)


@pytest.mark.parametrize("batch,kw", [(1, {}), (2, {}), (5, {}), (33, {}), (4, dict(kv_layout="token")), (1, dict(hidden=4096, nkv=1))])
def test_a_step_rotates_with_the_frequencies_that_were_set(batch, kw):
    w = small(batch, **kw)
    with Session(w, seed=11) as s:
        plain = s.run().clone()
        k_plain = s.k_pools[0].clone()
        psv.psv_set_rope(s.ctx, psv.psv_rope_plan(theta=w.rope_theta))
        assert torch.equal(s.run(), plain) and torch.equal(s.k_pools[0], k_plain)      # the descriptor's frequencies, by the other way
        rope = psv.psv_rope_plan(theta=w.rope_theta, scaling="channel", factor=8.0, high_turns=32.0, trained_context=64.0, magnitude=1.2)
        psv.psv_set_rope(s.ctx, rope)
        out = s.run().clone()
        assert not torch.equal(out, plain)
        qkv = psv.psv_debug_read(s.ctx, psv.PSV_DBG_QKV, np.zeros((batch, (w.n_q_heads + 2 * w.n_kv_heads) * 128), dtype=np.float32))
        keys = torch.from_numpy(qkv).view(batch, -1, 128)[:, w.n_q_heads:w.n_q_heads + w.n_kv_heads]
        t = w.context - 1
        pool = s.k_pools[0]
        blocks = torch.arange(batch, device="cuda") * w.blocks_per_seq + t // 16
        got = pool[blocks, t % 16] if w.kv_layout == "token" else pool[blocks, :, t % 16]
        want, size = rotated(keys, torch.full((batch,), t), rope)
        assert ((got.cpu().double() - want).abs() <= bound(want, size, torch.bfloat16)).all()
        psv.psv_set_rope(s.ctx, None)
        assert torch.equal(s.run(), plain)
        with pytest.raises(psv.PsvError) as e:
            psv.psv_set_rope(s.ctx, psv.psv_rope_plan(pairing="interleaved"))
        assert e.value.status == psv.PSV_ERR_UNSUPPORTED
        with pytest.raises(psv.PsvError):
            psv.psv_set_rope(s.ctx, psv.psv_rope_plan(dims=64))
        assert torch.equal(s.run(), plain)      # a refusal changes nothing


def test_set_rope_on_a_context_without_rotation():
    w = small(3, rope_theta=0.0)
    with Session(w, seed=12) as s:
        plain = s.run().clone()
        psv.psv_set_rope(s.ctx, psv.psv_rope_plan(theta=10000.0))
        assert not torch.equal(s.run(), plain)
        psv.psv_set_rope(s.ctx, None)
        assert torch.equal(s.run(), plain)


@pytest.mark.parametrize("fused", [0, 1, 2])
def test_every_kind_of_step_rotates_with_them(fused):
    """Kernels of an operator, of a block, of the whole step: the same output and keys to rounding."""
    w = synth.Workload("rope_fused", 2, 4096, 4, 1, 128, 1792, 1, 300, False, (0.0, 0.0))
    rope = psv.psv_rope_plan(theta=w.rope_theta, scaling="turns", factor=8.0, trained_context=100.0, magnitude=1.1)
    got = {}
    for kind in {0, fused}:
        with Session(w, seed=13, fused=kind) as s:
            psv.psv_set_rope(s.ctx, rope)
            got[kind] = (s.run().clone().cpu(), s.k_pools[0].cpu().float())
            assert psv.psv_debug_last_step_path(s.ctx) == kind
    (a, ka), (b, kb) = got[fused], got[0]
    assert ((a - b).abs() <= 2e-2 + 1e-2 * b.abs()).all()
    assert ((ka - kb).abs() <= kb.abs() * 2.0 ** -7).all()      # a key on either side of a rounding: one step


@pytest.mark.parametrize("batch", [1, 8])
def test_the_policies_agree_bit_for_bit_with_frequencies_set(batch):
    w = synth.Workload("rope_windows", 3, 4096, 4, 1, 128, 1792, batch, 200, True, (15.0, 15.0))
    from paper_2501_08192_amd.harness import default_policy
    with Session(w, seed=14) as s:
        psv.psv_set_rope(s.ctx, psv.psv_rope_plan(theta=w.rope_theta, scaling="linear", factor=4.0))
        off = s.run().clone()
        for kw in (dict(), dict(prelaunch=0)):
            s.set_policy(default_policy(w, **kw))
            assert torch.equal(s.run(), off)
