"""The operators around the decode step (include/preserve_ops.h) as far as no GPU is needed: exports, struct layouts, the rotary
frequencies, and everything that is refused before a launch."""
import ctypes as C
import math

import pytest
import torch

from paper_2501_08192_amd import binding as psv
from test_library_abi import header_symbols

BAD, UNSUPPORTED = psv.PSV_ERR_INVALID_ARG, psv.PSV_ERR_UNSUPPORTED
P = 1 << 20      # an address that is never followed


def test_every_operator_is_exported_and_bound():
    assert sorted(psv.OPERATOR_EXPORTS) == header_symbols(("preserve_ops.h",))
    for n in psv.OPERATOR_EXPORTS:
        assert hasattr(psv.lib(), n) and callable(getattr(psv, n))


def test_struct_layouts():
    # restated from the header: pointers and 64-bit fields of 8 bytes, the others of 4
    sizes = dict(psv_rope_desc=4 * 4 + 6 * 8, psv_rope=2 * 4 + 8 + 128 * 8, psv_rotate_args=3 * 8 + 6 * 4 + 4 * 8, psv_slots_args=5 * 8 + 6 * 4 + 7 * 8,
                 psv_cache=2 * 8 + 4 * 4, psv_append_args=6 * 8 + 4 * 4 + 4 * 8, psv_gather_args=3 * 8 + 2 * 4 + 2 * 8,
                 psv_logprobs_args=2 * 8 + 10 * 4 + 8, psv_logprobs_out=4 * 8)
    for name, size in sizes.items():
        assert C.sizeof(getattr(psv, name)) == size, name


# ---- frequencies ----------------------------------------------------------------------------------------------------------

def freq(**kw):
    r = psv.psv_rope_plan(**kw)
    n = kw.get("dims", 128) // 2
    assert all(f == 0.0 for f in list(r.freq)[n:])
    return list(r.freq)[:n], r


@pytest.mark.parametrize("dims,theta", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (256, 1e6)])
def test_plain_and_linear_frequencies(dims, theta):
    want = [theta ** (-2.0 * i / dims) for i in range(dims // 2)]
    got, r = freq(dims=dims, theta=theta)
    assert got == pytest.approx(want, rel=1e-14) and r.dims == dims and r.magnitude == 1.0
    got, _ = freq(dims=dims, theta=theta, scaling="linear", factor=4.0)
    assert got == pytest.approx([f / 4.0 for f in want], rel=1e-14)


def test_frequencies_between_the_two_turn_counts_are_mixed():
    kw = dict(theta=500000.0, factor=8.0, low_turns=1.0, high_turns=4.0, trained_context=8192.0)
    plain, _ = freq(theta=500000.0)
    got, _ = freq(scaling="turns", **kw)
    seen = set()
    for f, g in zip(plain, got):
        turns = 8192.0 * f / (2 * math.pi)
        if turns >= 4.0:
            assert g == pytest.approx(f, rel=1e-14)
            seen.add("kept")
        elif turns <= 1.0:
            assert g == pytest.approx(f / 8.0, rel=1e-14)
            seen.add("stretched")
        else:
            w = (turns - 1.0) / 3.0
            assert g == pytest.approx(w * f + (1 - w) * f / 8.0, rel=1e-14)
            seen.add("mixed")
    assert seen == {"kept", "mixed", "stretched"}


def test_frequencies_mixed_by_channel():
    plain, _ = freq(theta=10000.0)
    got, r = freq(theta=10000.0, scaling="channel", factor=16.0, low_turns=1.0, high_turns=32.0, trained_context=4096.0, magnitude=1.25)
    assert r.magnitude == 1.25
    at = [128 * math.log(4096.0 / (2 * math.pi * n)) / (2 * math.log(10000.0)) for n in (32.0, 1.0)]
    lo, hi = math.floor(at[0]), math.ceil(at[1])
    for i, (f, g) in enumerate(zip(plain, got)):
        w = 1.0 - min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert g == pytest.approx(w * f + (1 - w) * f / 16.0, rel=1e-13)
    assert got[lo] == pytest.approx(plain[lo]) and got[hi] == pytest.approx(plain[hi] / 16.0)
    # a factor of 1 changes nothing, whatever the ramp
    for scaling in ("linear", "turns", "channel"):
        assert freq(scaling=scaling, factor=1.0)[0] == pytest.approx(freq()[0], rel=1e-14)


@pytest.mark.parametrize("kw", [dict(dims=0), dict(dims=3), dict(dims=258), dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")),
                                dict(magnitude=float("inf")), dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")),
                                dict(scaling="turns", low_turns=0.0), dict(scaling="turns", low_turns=4.0, high_turns=4.0),
                                dict(scaling="channel", trained_context=0.0), dict(scaling="channel", high_turns=float("inf"))])
def test_rope_descriptions_are_checked(kw):
    with pytest.raises(psv.PsvError) as e:
        psv.psv_rope_plan(**kw)
    assert e.value.status == BAD


def test_rope_plan_null_and_unknown_forms():
    d, out = psv.psv_rope_desc(128, 0, 0, 0, 0.0, 10000.0), psv.psv_rope()
    L = psv.lib()
    assert L.psv_rope_plan(None, C.byref(out)) == BAD and L.psv_rope_plan(C.byref(d), None) == BAD
    assert L.psv_rope_plan(C.byref(d), C.byref(out)) == psv.PSV_OK and out.magnitude == 1.0
    for field, value in (("pairing", 2), ("scaling", 4)):
        d = psv.psv_rope_desc(128, 0, 0, 0, 0.0, 10000.0)
        setattr(d, field, value)
        assert L.psv_rope_plan(C.byref(d), C.byref(out)) == BAD
    assert L.psv_set_rope(None, C.byref(out)) == BAD


# ---- refusals ------------------------------------------------------------------------------------------------------------------

def rotate_status(rope_kw={}, rope=True, **kw):
    a = psv.psv_rotate_args(P, 2 * P, 3 * P, 4, 8, 128, psv.PSV_BF16, 0, 0, 1024, 128, 1024, 128)
    for k, v in kw.items():
        setattr(a, k, v)
    r = psv.psv_rope_plan(**rope_kw)
    return psv.lib().psv_rotate(C.byref(a), C.byref(r) if rope else None, None)


@pytest.mark.parametrize("kw", [dict(x=None), dict(y=None), dict(positions=None), dict(x=P + 1), dict(y=P + 1), dict(positions=P + 2),
                                dict(rows=(1 << 24) + 1), dict(heads=0), dict(heads=65536), dict(head_dim=64), dict(head_dim=1026),
                                dict(dtype=3), dict(transpose=2), dict(x_row=-1), dict(x_head=-128), dict(y_row=-1024), dict(x_row=1 << 33),
                                dict(y_row=0), dict(y_head=0), dict(y_head=64), dict(y_row=1023), dict(y_row=128, y_head=128),
                                dict(y=P, x_row=2048), dict(y=P, x_head=256), dict(rope=False)])
def test_rotate_refuses(kw):
    assert rotate_status(**kw) == BAD


def test_rotate_refuses_made_up_frequencies_and_takes_no_rows():
    r = psv.psv_rope_plan()
    a = psv.psv_rotate_args(P, 2 * P, 3 * P, 4, 8, 128, psv.PSV_BF16, 0, 0, 1024, 128, 1024, 128)
    for field, value in (("dims", 0), ("dims", 258), ("dims", 5), ("pairing", 2), ("magnitude", float("nan"))):
        q = psv.psv_rope.from_buffer_copy(r)
        setattr(q, field, value)
        assert psv.lib().psv_rotate(C.byref(a), C.byref(q), None) == BAD
    r.freq[63] = float("inf")
    assert psv.lib().psv_rotate(C.byref(a), C.byref(r), None) == BAD
    assert psv.lib().psv_rotate(None, C.byref(psv.psv_rope_plan()), None) == BAD
    assert rotate_status(rows=0, x=None, y=None, positions=None) == psv.PSV_OK


def slots_status(**kw):
    a = psv.psv_slots_args(P, 2 * P, 3 * P, 4 * P, 5 * P, 64, 4, 16, 100, 32, 0, 6 * P, 7 * P, 8 * P, 9 * P, 10 * P, 11 * P, 12 * P)
    for k, v in kw.items():
        setattr(a, k, v)
    return psv.lib().psv_cache_slots(C.byref(a), None)


@pytest.mark.parametrize("kw", [dict(lens=None), dict(new_lens=None), dict(seq_lens=None), dict(row_starts=None), dict(refused=None),
                                dict(slots=None), dict(positions=None), dict(requests=None), dict(free_blocks=None), dict(free_range=None),
                                dict(free_range_out=None), dict(batch=0), dict(batch=4097), dict(max_blocks=0), dict(max_blocks=1 << 30),
                                dict(num_pool_blocks=0), dict(num_pool_blocks=1 << 31), dict(rows=1 << 31), dict(free_capacity=1 << 31),
                                dict(lens=P + 2), dict(slots=P + 4), dict(seq_lens=P), dict(seq_lens=2 * P), dict(free_range_out=5 * P)])
def test_slots_refuses(kw):
    assert slots_status(**kw) == BAD
    assert psv.lib().psv_cache_slots(None, None) == BAD


def append_status(rope_kw={}, rope=True, cache_kw={}, cache=True, **kw):
    a = psv.psv_append_args(P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 4, 8, psv.PSV_BF16, 0, 1280, 1280, 1280, 1024)
    c = psv.psv_cache(7 * P, 8 * P, 1, 0, 0, 100)
    for k, v in kw.items():
        setattr(a, k, v)
    for k, v in cache_kw.items():
        setattr(c, k, v)
    r = psv.psv_rope_plan(**rope_kw)
    return psv.lib().psv_cache_append(C.byref(a), C.byref(c) if cache else None, C.byref(r) if rope else None, None)


CACHES = [dict(k_pool=None), dict(v_pool=None), dict(k_pool=P + 8), dict(v_pool=P + 8), dict(n_kv_heads=0), dict(n_kv_heads=129), dict(kv_format=2),
          dict(kv_layout=2), dict(kv_format=1, kv_layout=1), dict(num_pool_blocks=0), dict(num_pool_blocks=1 << 31)]


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(v=None), dict(q_out=None), dict(positions=None), dict(slots=None), dict(q=P + 8),
                                dict(k=P + 2), dict(v=P + 4), dict(q_out=P + 8), dict(positions=P + 2), dict(slots=P + 4), dict(rows=(1 << 24) + 1),
                                dict(n_q_heads=129), dict(dtype=3), dict(q_row=1284), dict(k_row=-1280), dict(v_row=4), dict(q_out_row=1016),
                                dict(q_out=P), dict(cache=False)] + [dict(cache_kw=c) for c in CACHES])
def test_append_refuses(kw):
    assert append_status(**kw) == BAD


def test_append_unsupported_rotations_and_no_rows():
    assert append_status(rope_kw=dict(dims=256)) == UNSUPPORTED and append_status(rope_kw=dict(dims=72)) == UNSUPPORTED
    assert append_status(rows=1 << 24, cache_kw=dict(n_kv_heads=17)) == UNSUPPORTED
    assert append_status(rows=0, k=None, v=None, slots=None) == psv.PSV_OK
    assert psv.lib().psv_cache_append(None, None, None, None) == BAD


@pytest.mark.parametrize("kw", [dict(slots=None), dict(k=None), dict(v=None), dict(slots=P + 4), dict(k=P + 2), dict(v=P + 8), dict(rows=(1 << 24) + 1),
                                dict(dtype=3), dict(k_row=64), dict(v_row=132), dict(cache=False)] + [dict(cache_kw=c) for c in CACHES])
def test_gather_refuses(kw):
    a = psv.psv_gather_args(P, 2 * P, 3 * P, 4, psv.PSV_BF16, 128, 128)
    c = psv.psv_cache(7 * P, 8 * P, 1, 0, 0, 100)
    kw = dict(kw)
    for k, v in kw.pop("cache_kw", {}).items():
        setattr(c, k, v)
    there = kw.pop("cache", True)
    for k, v in kw.items():
        setattr(a, k, v)
    assert psv.lib().psv_cache_gather(C.byref(a), C.byref(c) if there else None, None) == BAD
    a.rows = 0
    if there and a.dtype < 3 and c.n_kv_heads == 1 and c.k_pool and c.v_pool and c.k_pool % 16 == 0 and c.v_pool % 16 == 0 and c.kv_format + c.kv_layout < 2 \
            and 0 < c.num_pool_blocks < 1 << 31:
        assert psv.lib().psv_cache_gather(C.byref(a), C.byref(c), None) == psv.PSV_OK


def logprob_args(**kw):
    a = psv.psv_logprobs_args(P, 2 * P, 4, 1000, 0, 1000, psv.PSV_F32, 1, 5, 1.0, 0, 0, 1000)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


SHARED = [dict(tokens=None), dict(tokens=2 * P + 1), dict(rows=(1 << 20) + 1), dict(given=33), dict(top=33), dict(scale=0.0), dict(scale=-1.0),
          dict(scale=float("nan")), dict(scale=1e-10), dict(scale=5e9), dict(scale=float("inf")), dict(vocab=0), dict(vocab=(1 << 21) + 1)]


@pytest.mark.parametrize("kw", SHARED + [dict(logits=None), dict(logits=P + 2), dict(columns=0), dict(columns=(1 << 21) + 1), dict(first_token=1), dict(vocab=999),
                                         dict(first_token=0xffffffff), dict(dtype=3), dict(row=1 << 33), dict(row=-1000), dict(records=257),
                                         dict(columns=128256, vocab=128256, row=128256, records=3)])
def test_logprobs_part_refuses(kw):
    L, a = psv.lib(), logprob_args(**kw)
    assert L.psv_logprobs_part(C.byref(a), 3 * P, None) == BAD
    out = psv.psv_logprobs_out(4 * P, 5 * P, 6 * P, 7 * P)
    assert L.psv_logprobs(C.byref(a), C.byref(out), 3 * P, 1 << 30, None) == BAD


@pytest.mark.parametrize("kw", SHARED + [dict(records=0), dict(records=129)])
def test_logprobs_join_refuses(kw):
    a = logprob_args(**dict(dict(records=4), **kw))
    out = psv.psv_logprobs_out(4 * P, 5 * P, 6 * P, 7 * P)
    assert psv.lib().psv_logprobs_join(C.byref(a), 3 * P, 2, C.byref(out), None) == BAD


def test_logprobs_refuses_buffers_and_takes_no_rows():
    L, a = psv.lib(), logprob_args()
    out = psv.psv_logprobs_out(4 * P, 5 * P, 6 * P, 7 * P)
    need = psv.psv_logprobs_bytes(4, psv.psv_logprobs_records(4, 1000), 1, 5)
    assert L.psv_logprobs_part(C.byref(a), None, None) == BAD and L.psv_logprobs_part(C.byref(a), 3 * P + 2, None) == BAD
    assert L.psv_logprobs(C.byref(a), C.byref(out), 3 * P, need - 1, None) == BAD
    assert L.psv_logprobs(C.byref(a), None, 3 * P, need, None) == BAD and L.psv_logprobs(None, C.byref(out), 3 * P, need, None) == BAD
    for half in (psv.psv_logprobs_out(4 * P, 5 * P, None, 7 * P), psv.psv_logprobs_out(4 * P, 5 * P, 6 * P, None)):
        assert L.psv_logprobs(C.byref(a), C.byref(half), 3 * P, need, None) == BAD
        assert L.psv_logprobs_join(C.byref(logprob_args(records=1)), 3 * P, 1, C.byref(half), None) == BAD
    bad = psv.psv_logprobs_out(4 * P, 5 * P + 2, None, None)
    assert L.psv_logprobs_join(C.byref(logprob_args(records=1)), 3 * P, 1, C.byref(bad), None) == BAD
    assert L.psv_logprobs(C.byref(logprob_args(first_token=1, columns=999)), C.byref(out), 3 * P, need, None) == BAD      # a shard
    assert L.psv_logprobs_part(C.byref(logprob_args(rows=1 << 20, records=16)), 3 * P, None) == UNSUPPORTED
    assert L.psv_logprobs(C.byref(logprob_args(rows=0, logits=None)), C.byref(out), None, 0, None) == psv.PSV_OK
    for shards in (0, 257):
        assert L.psv_logprobs_join(C.byref(logprob_args(records=1)), 3 * P, shards, C.byref(out), None) == BAD


def test_logprobs_records():
    assert psv.psv_logprobs_records(1, 0) == 0 and psv.psv_logprobs_records(1, (1 << 21) + 1) == 0 and psv.psv_logprobs_records((1 << 20) + 1, 8) == 0
    for rows in (0, 1, 3, 64, 5000, 1 << 20):
        for columns in (1, 8, 2048, 2049, 16032, 32003, 128256, 1 << 21):
            n = psv.psv_logprobs_records(rows, columns)
            chunk = (-(-columns // n) + 7) // 8 * 8
            assert 1 <= n <= 256 and chunk <= 16384, (rows, columns)
    assert psv.psv_logprobs_bytes(3, 5, 2, 7) == 4 * 3 * 5 * (4 + 2 + 14)


def test_the_binding_checks_tensors():
    f, i = torch.zeros(2, 3, 128), torch.zeros(2, dtype=torch.int32)
    rope = psv.psv_rope_plan()
    for call in (lambda: psv.psv_rotate(f, f.double(), i, rope, None), lambda: psv.psv_rotate(f, f.clone(), i.long(), rope, None),
                 lambda: psv.psv_rotate(f.transpose(1, 2), f.transpose(1, 2), i, rope, None), lambda: psv.psv_rotate(f, f.clone(), i[:1], rope, None),
                 lambda: psv.psv_cache_gather(i, f, f, psv.kv_cache(P, P, 3, "bf16", "head", 4), None),
                 lambda: psv.psv_cache_gather(i.long(), f, f, psv.kv_cache(P, P, 2, "bf16", "head", 4), None),
                 lambda: psv.psv_cache_append(None, f, f[:, :2], None, i, i.long(), psv.kv_cache(P, P, 3, "bf16", "head", 4), rope, None),
                 lambda: psv.psv_cache_append(f, f, f, f[:1], i, i.long(), psv.kv_cache(P, P, 3, "bf16", "head", 4), rope, None),
                 lambda: psv.psv_logprobs(f[0].t(), None, 1.0, None, None, None, None, f, None),
                 lambda: psv.psv_logprobs(f[0], i, 1.0, None, None, None, None, f, None) if i.dim() == 2 else psv.psv_logprobs(
                     f[0], i.reshape(1, 2), 1.0, None, None, None, None, f, None)):
        with pytest.raises(ValueError):
            call()
