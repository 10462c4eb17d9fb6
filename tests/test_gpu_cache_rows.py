"""psv_cache_slots against a request-by-request walk, psv_cache_append and psv_cache_gather against rows in 64 bits, and all of them in
a run with decode steps and log probabilities."""
import numpy as np
import pytest
import torch

import oracle
from paper_2501_08192_amd import binding as psv
from paper_2501_08192_amd import synth
from paper_2501_08192_amd.harness import Session
from helpers import to_bits
from test_gpu_rotate import TYPES, bound, rotated

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype).cuda()


# ---- slots ------------------------------------------------------------------------------------------------------------------------

def walked(lens, new, table, free, free_range, max_blocks, pool_blocks, n_rows):
    """The definition, one request after the other."""
    batch = len(lens)
    table = None if table is None else table.copy()
    lo, hi = free_range if table is not None else (0, 0)
    left = hi - lo if table is not None and 0 <= lo <= hi <= len(free) else 0
    out = dict(seq_lens=list(lens), row_starts=[], slots=np.full(n_rows, -1, np.int64), positions=np.zeros(n_rows, np.int32),
               requests=np.full(n_rows, -1, np.int32), refused=0)
    row = want = used = 0
    for b in range(batch):
        t, n = int(lens[b]), int(new[b])
        out["row_starts"].append(min(row, n_rows))
        good = t >= 0 and n >= 0 and t + n <= max_blocks * 16 and row + n <= n_rows
        need = -(-(t + n) // 16) - -(-t // 16) if good else 0
        first = lo + want
        want += need
        if table is not None and need and want > left:
            good = False
        if good:
            used += need
            out["seq_lens"][b] = t + n
            if table is not None:
                for i in range(need):
                    table[b, -(-t // 16) + i] = free[first + i]
        else:
            out["refused"] += 1
        for i in range(max(0, min(n, n_rows - row))):
            p = t + i
            out["positions"][row + i], out["requests"][row + i] = np.int64(p).astype(np.int32), b      # a refused one's may not fit 32 bits
            if good:
                blk = b * max_blocks + p // 16 if table is None else table[b, p // 16]
                if 0 <= blk < pool_blocks:
                    out["slots"][row + i] = int(blk) * 16 + p % 16
        row += max(n, 0)
    out["row_starts"].append(min(row, n_rows))
    out["table"], out["free_range"] = table, (lo + used, hi)
    return out


def check_slots(lens, new, max_blocks=40, n_rows=None, n_free=None, contiguous=False, pool_blocks=None, seed=0, free_range=None, spoil=None):
    rng = np.random.default_rng(seed)
    batch = len(lens)
    held = [max(0, -(-int(t) // 16)) for t in lens]
    n_rows = sum(max(0, int(n)) for n in new) if n_rows is None else n_rows
    total = sum(min(h, max_blocks) for h in held) + (500 if n_free is None else n_free)
    ids = rng.permutation(total).astype(np.int32)
    table = None
    at = 0
    if not contiguous:
        table = rng.integers(-5, 0, size=(batch, max_blocks)).astype(np.int32)
        for b, h in enumerate(held):
            h = min(h, max_blocks)
            table[b, :h] = ids[at:at + h]
            at += h
        if spoil:
            spoil(table)
    free = ids[at:].copy()
    pool_blocks = (batch * max_blocks if contiguous else total) if pool_blocks is None else pool_blocks
    free_range = (0, len(free)) if free_range is None else free_range
    want = walked(lens, new, table, free, free_range, max_blocks, pool_blocks, n_rows)
    seq_lens, starts = torch.full((batch,), -9, dtype=torch.int32).cuda(), torch.full((batch + 1,), -9, dtype=torch.int32).cuda()
    slots, positions = torch.full((n_rows,), -9).cuda(), torch.full((n_rows,), -9, dtype=torch.int32).cuda()
    requests, refused = positions.clone(), dev([-9])
    t_dev = None if contiguous else dev(table)
    args = (dev(lens), dev(new), t_dev, None if contiguous else dev(free), None if contiguous else dev(free_range), pool_blocks)
    out_range = None if contiguous else dev([-9, -9])
    for _ in range(2):      # a second call gives the same
        psv.psv_cache_slots(*args, seq_lens, starts, slots, positions, requests, out_range, refused, torch.cuda.current_stream(),
                            max_blocks=max_blocks)
        torch.cuda.synchronize()
        assert seq_lens.tolist() == want["seq_lens"] and starts.tolist() == want["row_starts"]
        assert np.array_equal(requests.cpu(), want["requests"]) and np.array_equal(positions.cpu(), want["positions"])
        assert np.array_equal(slots.cpu(), want["slots"]) and refused.item() == want["refused"]
        if not contiguous:
            assert np.array_equal(t_dev.cpu(), want["table"]) and tuple(out_range.tolist()) == tuple(want["free_range"])
    return want


@pytest.mark.parametrize("contiguous", [False, True])
@pytest.mark.parametrize("batch,longest,most", [(1, 0, 1), (1, 600, 1), (64, 600, 1), (5, 300, 200), (63, 100, 20), (257, 500, 3), (300, 15, 40), (4096, 40, 2)])
def test_slots_of_mixed_lengths(batch, longest, most, contiguous):
    rng = np.random.default_rng(batch + most)
    lens, new = rng.integers(0, longest + 1, size=batch), rng.integers(0, most + 1, size=batch)
    new[-1] = max(1, new[-1])
    check_slots(lens, new, contiguous=contiguous, n_free=batch * (most // 16 + 2), seed=batch)
    check_slots(lens, new, contiguous=contiguous, n_free=batch * (most // 16 + 2), n_rows=int(new.sum()) + 77, seed=batch)      # padded


@pytest.mark.parametrize("contiguous", [False, True])
@pytest.mark.parametrize("batch", [120, 700, 2500])
def test_slots_of_many_rows(batch, contiguous):
    """More rows than compute units times threads, for each number of requests a lane: four rows a lane, and a last few behind them."""
    rng = np.random.default_rng(batch)
    most = 2 * 70000 // batch
    lens, new = rng.integers(0, 640 - min(most, 600), size=batch), rng.integers(0, min(most, 600) + 1, size=batch)
    new[rng.integers(0, batch, size=batch // 9)] = 0
    n = max(int(new.sum()), 1 << 16) + 3
    check_slots(lens, new, contiguous=contiguous, n_free=int((new // 16 + 2).sum()), n_rows=n, seed=batch)
    check_slots(lens, new, contiguous=contiguous, n_free=int((new // 16 + 2).sum()) // 3, n_rows=n - 1000, seed=batch)      # some refused


def test_slots_at_block_edges_and_without_rows():
    check_slots([0, 15, 16, 17, 31, 32, 0, 16], [16, 1, 16, 15, 1, 0, 0, 1])
    check_slots([0, 0, 0], [0, 0, 0], n_rows=0)
    check_slots([5, 16, 0], [0, 0, 0], n_rows=9)
    check_slots([0], [40 * 16])
    check_slots([40 * 16], [0], n_rows=3)


def test_slots_refuses_requests_one_by_one():
    assert check_slots([-1, 10, 630, 5, 640, 3], [4, -2, 20, 7, 1, 2])["refused"] == 4
    assert check_slots([2**31 - 1, 5], [2**31 - 1, 3], n_rows=50)["refused"] == 2      # sums beyond 32 bits; the second's rows do not fit either
    assert check_slots([3, 3, 3], [10, 10, 1], n_rows=15)["refused"] == 2              # the row arrays are full after the first
    # too few free blocks: the first needs 2, the second 3 (refused), the third none, the fourth one (refused: those before it come first)
    assert check_slots([10, 16, 20, 32], [30, 40, 5, 1], n_free=4)["refused"] == 2
    assert check_slots([0, 0], [1, 1], n_free=1)["refused"] == 1
    assert check_slots([0, 7], [1, 1], n_free=0)["refused"] == 1


@pytest.mark.parametrize("free_range", [(3, 9), (9, 3), (-1, 4), (0, 1000), (5, 5)])
def test_slots_of_a_partial_or_impossible_free_list(free_range):
    check_slots([0, 5, 16], [20, 20, 1], n_free=12, free_range=free_range)


def test_slots_never_name_a_block_outside_the_pool():
    def spoil(table):
        table[0, 1], table[2, 0] = 10000, -3
    want = check_slots([40, 5, 20], [9, 9, 9], spoil=spoil, pool_blocks=506)
    assert (want["slots"] >= 0).any()
    spans = check_slots([20, 16], [4, 1], spoil=lambda t: t.__setitem__((0, 1), 99999))
    assert (spans["slots"][:4] == -1).all() and spans["slots"][4] >= 0


def test_slots_of_steps_that_follow_one_another_in_a_captured_graph():
    """Two sets of lengths and ranges taken in turn: a prompt, then steps of one token, replayed."""
    batch, mb = 7, 6
    lens = [dev(np.zeros(batch)), dev(np.zeros(batch))]
    ranges = [dev([0, 60]), dev([0, 0])]
    table, free = dev(np.full((batch, mb), -1)), dev(np.random.default_rng(1).permutation(60))
    new, refused = dev([3, 16, 17, 0, 30, 1, 15]), dev([0])
    starts, slots = dev(np.zeros(batch + 1)), torch.empty(90, dtype=torch.int64, device="cuda")
    positions, requests = dev(np.zeros(90)), dev(np.zeros(90))

    def both():
        for k in (0, 1):
            psv.psv_cache_slots(lens[k], new, table, free, ranges[k], 60, lens[1 - k], starts, slots, positions, requests, ranges[1 - k], refused,
                                torch.cuda.current_stream())
    host_len, host_table, host_range = np.zeros(batch, int), np.full((batch, mb), -1, np.int32), (0, 60)

    def host():
        nonlocal host_len, host_table, host_range
        w = walked(host_len, new.cpu().numpy(), host_table, free.cpu().numpy(), host_range, mb, 60, 90)
        host_len, host_table, host_range = np.array(w["seq_lens"]), w["table"], w["free_range"]
        return w
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for step in range(6):
        graph.replay()
        torch.cuda.synchronize()
        host()
        w = host()
        assert lens[0].tolist() == w["seq_lens"] and np.array_equal(table.cpu(), w["table"]) and tuple(ranges[0].tolist()) == tuple(w["free_range"])
        assert np.array_equal(slots.cpu(), w["slots"]) and refused.item() == w["refused"]
        new.fill_(1)
        torch.cuda.synchronize()


# ---- rows into and out of the cache --------------------------------------------------------------------------------------------------

class Pools:
    """A layer's pools with known contents, on the host and on the device."""

    def __init__(self, blocks, nkv, kv, layout, seed=0):
        self.blocks, self.nkv, self.kv, self.layout = blocks, nkv, kv, layout
        w = synth.Workload("pools", 1, 512, nkv, nkv, 128, 256, 1, 16 * blocks, False, (0.0, 0.0), kv_format=kv, kv_layout=layout)
        self.before = [t.cpu() for t in synth.kv_pools(w, 0, seed, "cpu", n_blocks=blocks)]
        self.gpu = [t.cuda() for t in self.before]
        self.cache = psv.kv_cache(self.gpu[0], self.gpu[1], nkv, kv, layout, blocks)

    def rows(self, pools, slots):
        """(values [n, nkv, 128] in 64 bits, scales [n, nkv] or None) for K and V."""
        blk, off = torch.as_tensor(slots) // 16, torch.as_tensor(slots) % 16
        out = []
        for which, pool in enumerate(pools):
            pool = pool.cpu()
            if self.kv == "int8":
                codes = pool[..., :2048].contiguous().view(torch.int8)
                scales = pool[..., 2048:].contiguous().view(torch.float32)
                c = codes.view(-1, self.nkv, 16, 128)[blk, :, off] if which == 0 else codes.view(-1, self.nkv, 128, 16)[blk, :, :, off]
                s = scales[blk, :, off]
                out.append((c.double(), s))
            elif self.layout == "token":
                out.append((pool[blk, off].double(), None))
            else:
                out.append(((pool[blk, :, off] if which == 0 else pool[blk, :, :, off]).double(), None))
        return out


def check_cached(pools, which, slots, want, size):
    """A cached row against its value in 64 bits: bf16 by the rounding, int8 by half a code step (and what 32 bits lose of it)."""
    got, scale = pools.rows(pools.gpu, slots)[which]
    if pools.kv == "int8":
        most = want.abs().amax(-1)
        # the largest magnitude is off by 3 * 2^-24 of the two terms that it is made of, together at most twice itself; one division
        assert ((scale.double() - torch.where(most > 0, most / 127.0, 1.0)).abs() <= 2.0 ** -21 * torch.where(most > 0, most / 127.0, 1.0)).all()
        assert (got.abs() <= 127).all()
        # half a step; the value's 3 * 2^-24 of its terms (twice 127 steps at most) and the division's 2^-24 stay under 1e-4 steps, the clamp's
        # edge and the scale's own 2^-21 of 127 steps too
        assert ((got * scale.double()[..., None] - want).abs() <= 0.5003 * scale.double()[..., None]).all()
    else:
        assert ((got - want).abs() <= bound(want, size, torch.bfloat16)).all()


def append_case(n, nq, nkv, kv="bf16", layout="head", dtype="bf16", pairing="half", dims=128, start=0, seed=1, rope=True, skip=(), packed=True, blocks=None,
                scattered=False):
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    blocks = -(-(start + n) // 16) + 3 if blocks is None else blocks
    pools = Pools(blocks, nkv, kv, layout, seed)
    table = rng.permutation(blocks)
    p = np.arange(start, start + n)
    slots = rng.permutation(blocks * 16)[:n].astype(np.int64) if scattered else (table[p // 16] * 16 + p % 16).astype(np.int64)
    for i, bad in skip:
        slots[i] = bad
    q, k, v = (torch.randn(n, h, 128, generator=gen).to(TYPES[dtype]) for h in (nq, nkv, nkv))
    if packed:
        all_rows = torch.cat([q, k, v], dim=1).cuda()
        dq, dk, dv = all_rows[:, :nq], all_rows[:, nq:nq + nkv], all_rows[:, nq + nkv:]
    else:
        dq, dk, dv = q.cuda(), k.cuda(), v.cuda()
    plan = psv.psv_rope_plan(dims=dims, pairing=pairing, theta=10000.0) if rope else None
    q_out = torch.full((n, nq, 128), float("nan"), dtype=TYPES[dtype], device="cuda") if nq else None
    psv.psv_cache_append(dq if nq else None, dk, dv, q_out, dev(p) if rope else None, dev(slots, torch.int64), pools.cache, plan, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for rows, want_rows, got in ((q, dq, q_out),):
        if nq:
            want, size = rotated(rows, torch.as_tensor(p), plan) if rope else (rows.double(), rows.double().abs())
            assert ((got.cpu().double() - want).abs() <= bound(want, size, rows.dtype)).all()
    ok = (slots >= 0) & (slots < blocks * 16)
    want, size = rotated(k, torch.as_tensor(p), plan) if rope else (k.double(), k.double().abs())
    check_cached(pools, 0, slots[ok], want[torch.as_tensor(ok)], size[torch.as_tensor(ok)])
    check_cached(pools, 1, slots[ok], v.double()[torch.as_tensor(ok)], 0.0 * v.double().abs()[torch.as_tensor(ok)])
    rest = np.setdiff1d(np.arange(blocks * 16), slots[ok])
    for (a, sa), (b, sb) in zip(pools.rows(pools.gpu, rest), pools.rows(pools.before, rest)):
        assert torch.equal(a, b) and (sa is None or torch.equal(sa, sb))
    return pools, slots, (q, k, v)


LAYOUTS = [("bf16", "head"), ("bf16", "token"), ("int8", "head")]


@pytest.mark.parametrize("kv,layout", LAYOUTS)
@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("pairing,dims", [("half", 128), ("interleaved", 128), ("half", 32), ("interleaved", 96)])
def test_append_types_layouts_and_parts_of_a_head(kv, layout, dtype, pairing, dims):
    append_case(53, 5, 2, kv, layout, dtype, pairing, dims, start=7)


@pytest.mark.parametrize("kv,layout", LAYOUTS)
@pytest.mark.parametrize("n,start", [(1, 0), (1, 31), (2, 15), (15, 1), (16, 0), (16, 16), (17, 3), (33, 0), (64, 0), (64, 8), (129, 13), (1000, 5)])
def test_append_lengths_and_starts(n, start, kv, layout):
    append_case(n, 4, 1, kv, layout, start=start, seed=n)


@pytest.mark.parametrize("kv,layout", LAYOUTS)
@pytest.mark.parametrize("nq,nkv", [(0, 1), (1, 1), (8, 8), (16, 2), (3, 5), (128, 128)])
def test_append_heads(nq, nkv, kv, layout):
    append_case(21, nq, nkv, kv, layout, start=4, packed=nq != 3)


@pytest.mark.parametrize("kv,layout", LAYOUTS)
def test_append_without_rotation_skipped_and_scattered_rows(kv, layout):
    append_case(40, 2, 2, kv, layout, rope=False)
    append_case(40, 2, 2, kv, layout, start=9, skip=[(0, -1), (5, -2**62), (17, 10**15), (38, -1), (39, -1)])
    pools, _, _ = append_case(40, 2, 2, kv, layout, skip=[(i, -1 - i) for i in range(40)])
    assert all(torch.equal(a.cpu(), b) for a, b in zip(pools.gpu, pools.before))
    append_case(100, 2, 3, kv, layout, scattered=True, blocks=30)
    append_case(70, 1, 1, kv, layout, scattered=True, blocks=70, dtype="f32", pairing="interleaved")


@pytest.mark.parametrize("kv,layout", LAYOUTS)
@pytest.mark.parametrize("n,nq,nkv,dtype,start", [(9001, 1, 1, "bf16", 3), (4099, 3, 3, "f32", 21), (2500, 0, 4, "f16", 0)])
def test_append_and_gather_of_whole_tiles(n, nq, nkv, dtype, start, kv, layout):
    """Rows enough for the largest tiles of both kinds of workgroups, some of them skipped, so that octets end inside tiles and across them."""
    rng = np.random.default_rng(n)
    skip = [(int(i), -1) for i in rng.integers(0, n, size=n // 40)]
    pools, slots, (q, k, v) = append_case(n, nq, nkv, kv, layout, dtype, start=start, skip=skip)
    out = torch.full((2, n, nkv, 128), 5.0, device="cuda")
    psv.psv_cache_gather(dev(slots, torch.int64), out[0], out[1], pools.cache, torch.cuda.current_stream())
    torch.cuda.synchronize()
    ok = torch.as_tensor(slots >= 0)
    for got, (value, scale) in zip(out, pools.rows(pools.gpu, slots[slots >= 0])):
        assert torch.equal(got.cpu()[ok], value.float() if scale is None else value.float() * scale[..., None]) and (got.cpu()[~ok] == 5.0).all()


def test_append_int8_rows_of_zeros_and_of_one_size():
    pools = Pools(4, 1, "int8", "head")
    k = torch.zeros(3, 1, 128, device="cuda")
    v = torch.stack([torch.zeros(128), torch.full((128,), -2.0), torch.linspace(-1, 1, 128)]).view(3, 1, 128).cuda()
    k[1, 0, 5] = 1e-30
    psv.psv_cache_append(None, k, v, None, None, dev([0, 17, 34], torch.int64), pools.cache, None, torch.cuda.current_stream())
    torch.cuda.synchronize()
    (kc, ks), (vc, vs) = pools.rows(pools.gpu, [0, 17, 34])
    assert (kc[0] == 0).all() and ks[0] == 1.0 and kc[1, 0, 5] == 127 and (kc[1, 0].abs().sum() == 127)
    assert (vc[0] == 0).all() and vs[0] == 1.0 and (vc[1] == -127).all() and vc[2, 0, 0] == -127 and vc[2, 0, 127] == 127


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_append_int8_codes_are_the_rule_in_single_precision(dtype):
    """Without rotation nothing but the rule is computed: scale = max|v| / 127 and code = rint(v / scale), bit for bit; among the values many
    that lie on, or one rounding beside, the middle between two codes, and rows whose scale is tiny or has an infinite reciprocal."""
    gen = torch.Generator().manual_seed(8)
    n, nkv = 48, 2
    v = torch.randn(n, nkv, 128, generator=gen)
    half = torch.randint(-126, 126, (n, nkv, 128), generator=gen) + 0.5
    near = half * (1.0 + torch.randint(-2, 3, half.shape, generator=gen) * 2.0 ** -23)
    v[8:24] = near[8:24] * torch.rand(16, nkv, 1, generator=gen)
    v[8:24, :, 0] = 127.0 * v[8:24, :, 0].sign()
    v[24:32] = near[24:32]
    v[24:32, :, 5] = -127.0
    v[32] *= 1e-30
    v[33] *= 1e-38
    v[34] *= 1e-41
    v[35] *= 1e30
    v = v.to(TYPES[dtype])
    k = v.flip(0).contiguous()
    pools = Pools(4, nkv, "int8", "head", 8)
    slots = dev(np.arange(5, 5 + n), torch.int64)
    psv.psv_cache_append(None, k.cuda(), v.cuda(), None, None, slots, pools.cache, None, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for rows, (codes, scales) in zip((k, v), pools.rows(pools.gpu, slots.cpu())):
        x = rows.float()
        most = x.abs().amax(-1)
        want = torch.where(most > 0, most / 127.0, torch.ones_like(most))
        assert torch.equal(scales, want)
        fine = (want > 0) & torch.isfinite(want)      # 1e30 is infinite in f16: inf / inf is no number, and has no code
        assert torch.equal(codes[fine], torch.round(x / want[..., None]).clamp(-127, 127).double()[fine])


@pytest.mark.parametrize("kv,layout", LAYOUTS)
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_gather_returns_what_is_cached(kv, layout, dtype):
    for nkv, blocks, n, seed in ((1, 5, 80, 1), (2, 9, 37, 2), (5, 40, 640, 3), (128, 2, 3, 4)):
        pools = Pools(blocks, nkv, kv, layout, seed)
        rng = np.random.default_rng(seed)
        for slots in (np.arange(n), rng.integers(0, blocks * 16, size=n), np.arange(n)[::-1].copy(), np.arange(3, 3 + min(n, 16 * blocks - 3))):
            slots = slots.astype(np.int64)
            slots[len(slots) // 2], skipped = (-1 if seed % 2 else 16 * blocks), len(slots) // 2
            out = torch.full((2, len(slots), nkv + 1, 128), 5.0, dtype=TYPES[dtype], device="cuda")
            k, v = out[0, :, :nkv], out[1, :, 1:]
            psv.psv_cache_gather(dev(slots, torch.int64), k, v, pools.cache, torch.cuda.current_stream())
            torch.cuda.synchronize()
            keep = np.delete(np.arange(len(slots)), skipped)
            for got, (value, scale) in zip((k, v), pools.rows(pools.gpu, slots[keep])):
                want = value if scale is None else (value.float() * scale[..., None]).double()      # code times scale in 32 bits: exact but for one rounding
                assert torch.equal(got.cpu()[keep], want.float().to(TYPES[dtype]))
                assert (got[skipped] == 5.0).all()
            assert (out[0, :, nkv] == 5.0).all() and (out[1, :, 0] == 5.0).all()


def test_slots_beyond_32_bits_of_an_element():
    """A pool of more than 4 GiB: its last blocks."""
    blocks = (1 << 32) // 4096 + 64
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("less than 12 GiB free")
    pools = [torch.zeros(blocks, 1, 16, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(blocks, 1, 128, 16, dtype=torch.bfloat16, device="cuda")]
    cache = psv.kv_cache(pools[0], pools[1], 1, "bf16", "head", blocks)
    slots = dev([blocks * 16 - 1, 5, blocks * 16 - 18], torch.int64)
    k, v = torch.randn(3, 1, 128).bfloat16().cuda(), torch.randn(3, 1, 128).bfloat16().cuda()
    psv.psv_cache_append(None, k, v, None, None, slots, cache, None, torch.cuda.current_stream())
    a, b = torch.empty_like(k), torch.empty_like(v)
    psv.psv_cache_gather(slots, a, b, cache, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(a, k) and torch.equal(b, v) and torch.equal(pools[0][-1, 0, 15], k[0, 0]) and torch.equal(pools[1][-2, 0, :, 14], v[2, 0])


def test_append_and_gather_in_place_on_another_stream_and_captured():
    pools = Pools(8, 2, "bf16", "head")
    rows = torch.randn(30, 6, 128).bfloat16().cuda()
    first = rows.clone()
    p, slots = torch.arange(30, dtype=torch.int32, device="cuda"), torch.arange(20, 50, device="cuda")
    rope = psv.psv_rope_plan()
    q_out, k, v = torch.empty(30, 2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(30, 2, 128).cuda(), torch.zeros(30, 2, 128).cuda()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    psv.psv_cache_append(rows[:, :2], rows[:, 2:4], rows[:, 4:], q_out, p, slots, pools.cache, rope, stream)
    psv.psv_cache_append(rows[:, :2], rows[:, 2:4], rows[:, 4:], rows[:, :2], p, slots, pools.cache, rope, stream)
    psv.psv_cache_gather(slots, k, v, pools.cache, stream)
    stream.synchronize()
    assert torch.equal(rows[:, :2], q_out) and torch.equal(rows[:, 2:], first[:, 2:]) and torch.equal(v, first[:, 4:].float())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        psv.psv_cache_append(first[:, :2], first[:, 2:4], first[:, 4:], q_out, p, slots, pools.cache, rope, torch.cuda.current_stream())
        psv.psv_cache_gather(slots, k, v, pools.cache, torch.cuda.current_stream())
    for step in range(3):
        first.normal_()
        p.add_(5)
        graph.replay()
        torch.cuda.synchronize()
        want, size = rotated(first[:, 2:4].cpu(), p.cpu(), rope)
        assert torch.equal(v, first[:, 4:].float()) and ((k.cpu().double() - want).abs() <= bound(want, size, torch.bfloat16)).all()


# ---- a run of all of them, as a program serves -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kv", ["bf16", "int8"])
def test_prompts_then_a_decode_step_then_answers(kv):
    """Lengths -> places, prompt rows -> cache, decode step over it against the oracle, logits of its result -> log probabilities."""
    nq, nkv, hidden, batch, mb = 4, 2, 512, 5, 8
    w = synth.Workload("serve", 1, hidden, nq, nkv, 128, 512, batch, mb * 16, True, (0.0, 0.0), kv_format=kv)
    prompts = [1, 37, 64, 100, 16]
    gen = torch.Generator().manual_seed(5)
    with Session(w, seed=21) as s:
        stream = s.main
        lens, spans = dev(np.zeros(batch)), dev(np.zeros(batch))
        ranges = [dev([0, s.pool_blocks]), dev([0, 0])]
        free = dev(np.random.default_rng(3).permutation(s.pool_blocks))
        table = torch.full((batch, mb), -1, dtype=torch.int32, device="cuda")
        n = sum(prompts) + 6                  # padded rows behind the last prompt
        starts, refused = dev(np.zeros(batch + 1)), dev([0])
        slots, positions, requests = torch.empty(n, dtype=torch.int64, device="cuda"), dev(np.zeros(n)), dev(np.zeros(n))
        qkv = torch.randn(n, nq + 2 * nkv, 128, generator=gen).cuda()
        q_out = torch.empty(n, nq, 128, device="cuda")
        cache = psv.kv_cache(s.k_pools[0], s.v_pools[0], nkv, kv, "head", s.pool_blocks)
        rope = psv.psv_rope_plan(theta=w.rope_theta)
        new = dev(prompts)
        torch.cuda.synchronize()
        psv.psv_cache_slots(lens, new, table, free, ranges[0], s.pool_blocks, spans, starts, slots, positions, requests, ranges[1], refused, stream)
        psv.psv_cache_append(qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:], q_out, positions, slots, cache, rope, stream)
        one = dev([1] * batch)
        step_lens, row_starts = dev(np.zeros(batch)), dev(np.zeros(batch + 1))
        step_slots, step_pos, step_req = torch.empty(batch, dtype=torch.int64, device="cuda"), dev(np.zeros(batch)), dev(np.zeros(batch))
        torch.cuda.synchronize()
        psv.psv_cache_slots(spans, one, table, free, ranges[1], s.pool_blocks, step_lens, row_starts, step_slots, step_pos, step_req, ranges[0], refused, stream)
        psv.psv_set_kv(s.ctx, [s.k_pools[0]], [s.v_pools[0]], table, mb, s.pool_blocks, step_lens)
        stream.synchronize()
        before = s.host_pools(0)
        before = [p.copy() for p in before]
        out = s.run().clone()
        assert step_lens.tolist() == [p + 1 for p in prompts] and refused.item() == 0 and step_pos.tolist() == prompts
        m = oracle.model(hidden, nq, nkv, 128, 512, 16, w.rms_eps, w.rope_theta)
        x = s.x_in.cpu().numpy().astype(np.float64)
        if kv == "bf16":
            # the prompts' rows, rotated in 64 bits and rounded to bf16, in pools of the oracle's own
            kp, vp = (np.zeros_like(p) for p in before)
            want, size = rotated(qkv[:, nq:nq + nkv].cpu(), positions.cpu(), rope)
            for r, slot in enumerate(slots.tolist()):
                if slot >= 0:
                    kp[slot // 16, :, slot % 16] = to_bits(want[r])
                    vp[slot // 16, :, :, slot % 16] = to_bits(qkv[r, nq + nkv:].cpu())
            ref = oracle.decode_layer(m, s.host_layer(0), kp, vp, table.cpu().numpy(), mb, step_lens.cpu().numpy(), x)
        else:
            ref = oracle.decode_layer_x(m, s.host_layer(0), before[0], before[1], table.cpu().numpy(), mb, step_lens.cpu().numpy(), x)
        assert (np.abs(out.cpu().numpy() - ref) <= 2e-2 + 1e-2 * np.abs(ref)).all()
        assert (slots[-6:] == -1).all() and (requests[-6:] == -1).all()
        # the step's own keys lie at the slots that were computed for it
        gk, gv = torch.empty(batch, nkv, 128, device="cuda"), torch.empty(batch, nkv, 128, device="cuda")
        psv.psv_cache_gather(step_slots, gk, gv, cache, stream)
        stream.synchronize()
        step = torch.from_numpy(psv.psv_debug_read(s.ctx, psv.PSV_DBG_QKV, np.zeros((batch, (nq + 2 * nkv) * 128), dtype=np.float32))).view(batch, -1, 128)
        values = step[:, nq + nkv:].double()
        tol = 0.5003 * values.abs().amax(-1, keepdim=True) / 127 * (1 + 2.0 ** -20) if kv == "int8" else bound(values, 0.0, torch.bfloat16)
        assert ((gv.cpu().double() - values).abs() <= tol).all()
        # answers
        head = (torch.randn(1000, hidden, generator=gen) / 16).cuda()
        logits = out @ head.T
        lp, ent, top_lp, top = torch.empty(batch, 1).cuda(), torch.empty(batch).cuda(), torch.empty(batch, 4).cuda(), dev(np.zeros((batch, 4)))
        ws = torch.empty(psv.psv_logprobs_bytes(batch, psv.psv_logprobs_records(batch, 1000), 1, 4), dtype=torch.uint8, device="cuda")
        tokens = dev([[3], [999], [0], [500], [77]])
        torch.cuda.synchronize()
        psv.psv_logprobs(logits, tokens, 1.0, lp, ent, top_lp, top, ws, stream)
        stream.synchronize()
        want = torch.log_softmax(logits.double().cpu(), dim=1)
        assert (lp.cpu().double() - want.gather(1, tokens.cpu().long())).abs().max() <= 1e-5 * want.abs().max()
        assert torch.equal(top.cpu().long(), want.topk(4, dim=1).indices)
