"""Where the tensors of the operators around the decode step lie: the binding hands no address to the library that its stream's GPU cannot
follow.  No GPU is used: tensors that say where they are, and a library that only counts its calls."""
import types

import pytest
import torch

from paper_2501_08192_amd import binding as psv


class On0(torch.Tensor):
    def get_device(self):
        return 0


class On1(torch.Tensor):
    def get_device(self):
        return 1


class Library:
    calls = 0

    def __getattr__(self, name):
        if name in ("psv_logprobs_records", "psv_logprobs_bytes"):
            return lambda *a: 1 if name == "psv_logprobs_records" else 4 * a[0] * a[1] * (4 + a[2] + 2 * a[3])

        def call(*args):
            Library.calls += 1
            return psv.PSV_OK
        return call


N, BATCH, V = 6, 3, 50
ROPE = psv.psv_rope_plan()


def rows(heads):
    return torch.zeros(N, heads, 128)


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def slots_call(t, stream):
    table = t.get("block_table")
    psv.psv_cache_slots(t["lens"], t["new_lens"], table, t["free_blocks"], t["free_range"], 64, t["seq_lens"], t["row_starts"], t["slots"], t["positions"],
                        t["requests"], t["free_range_out"], t["refused"], stream)


def cache(t):
    return psv.kv_cache(t["k_pool"], t["v_pool"], 2, "bf16", "head", 4)


POOLS = dict(k_pool=torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16), v_pool=torch.zeros(4, 2, 128, 16, dtype=torch.bfloat16))
ANSWERS = dict(tokens=ints(N, 1), logprobs=torch.zeros(N, 1), entropy=torch.zeros(N), top_logprobs=torch.zeros(N, 4), top_ids=ints(N, 4), records=torch.zeros(N * 13))
CALLS = {
    "rotate": (dict(x=rows(2), y=rows(2), positions=ints(N)), lambda t, s: psv.psv_rotate(t["x"], t["y"], t["positions"], ROPE, s)),
    "slots": (dict(lens=ints(BATCH), new_lens=ints(BATCH), block_table=ints(BATCH, 8), free_blocks=ints(20), free_range=ints(2), seq_lens=ints(BATCH),
                   row_starts=ints(BATCH + 1), slots=torch.zeros(N, dtype=torch.int64), positions=ints(N), requests=ints(N), free_range_out=ints(2),
                   refused=ints(1)), slots_call),
    "append": (dict(POOLS, q=rows(4), k=rows(2), v=rows(2), q_out=rows(4), positions=ints(N), slots=torch.zeros(N, dtype=torch.int64)),
               lambda t, s: psv.psv_cache_append(t["q"], t["k"], t["v"], t["q_out"], t["positions"], t["slots"], cache(t), ROPE, s)),
    "gather": (dict(POOLS, slots=torch.zeros(N, dtype=torch.int64), k=rows(2), v=rows(2)),
               lambda t, s: psv.psv_cache_gather(t["slots"], t["k"], t["v"], cache(t), s)),
    "part": (dict(logits=torch.zeros(N, V), **{k: ANSWERS[k] for k in ("tokens", "records")}),
             lambda t, s: psv.psv_logprobs_part(t["logits"], t["tokens"], 1.0, 4, t["records"], s)),
    "join": (dict(ANSWERS), lambda t, s: psv.psv_logprobs_join(N, t["tokens"], 1.0, V, 1, 1, t["logprobs"], t["entropy"], t["top_logprobs"], t["top_ids"],
                                                                t["records"], s)),
    "logprobs": (dict(ANSWERS, logits=torch.zeros(N, V)), lambda t, s: psv.psv_logprobs(t["logits"], t["tokens"], 1.0, t["logprobs"], t["entropy"],
                                                                                         t["top_logprobs"], t["top_ids"], t["records"], s)),
}


@pytest.fixture
def library(monkeypatch):
    monkeypatch.setattr(psv, "lib", lambda: Library())
    Library.calls = 0
    return Library


@pytest.mark.parametrize("stream", [None, 0, "stream"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_one_tensor_elsewhere_is_refused(name, stream, library):
    tensors, call = CALLS[name]
    if stream == "stream":
        stream = types.SimpleNamespace(device_index=0, cuda_stream=0)
    there = {k: t.as_subclass(On0) for k, t in tensors.items()}
    call(there, stream)
    assert library.calls == 1
    for k, t in tensors.items():
        for other in (t, t.as_subclass(On1)):      # on the host, on another GPU
            with pytest.raises(ValueError, match="GPU"):
                call(dict(there, **{k: other}), stream)
    with pytest.raises(ValueError, match="GPU"):
        call(tensors, stream)
    if getattr(stream, "device_index", None) == 0:      # all of them on another GPU than the stream
        with pytest.raises(ValueError, match="GPU"):
            call({k: t.as_subclass(On1) for k, t in tensors.items()}, stream)
    assert library.calls == 1


@pytest.mark.parametrize("name", ["part", "join", "logprobs"])
def test_records_whose_memory_is_smaller_than_their_size_are_refused(name, library):
    tensors, call = CALLS[name]
    there = {k: t.as_subclass(On0) for k, t in tensors.items()}
    for records in (torch.zeros(1).expand(N * 13), torch.zeros(N * 13, 2)[:, 0]):
        with pytest.raises(ValueError, match="contiguous"):
            call(dict(there, records=records.as_subclass(On0)), None)
    assert library.calls == 0


def test_no_rows_need_no_records(library):
    psv.psv_logprobs_part(torch.zeros(0, V).as_subclass(On0), None, 1.0, 4, None, None)
    assert library.calls == 1


@pytest.mark.parametrize("name", ["join", "logprobs"])
def test_alternatives_are_ids_and_log_probabilities_together(name, library):
    """The one without the other would be left as it was, without a word."""
    tensors, call = CALLS[name]
    there = {k: t.as_subclass(On0) for k, t in tensors.items()}
    for missing in ("top_ids", "top_logprobs"):
        with pytest.raises(ValueError, match="both or neither"):
            call(dict(there, **{missing: None}), None)
    call(dict(there, top_ids=None, top_logprobs=None), None)
    assert library.calls == 1


def test_shapes_types_and_strides_of_tensors_that_lie_right_are_checked_as_well(library):
    f, i, l = (t.as_subclass(On0) for t in (torch.zeros(2, 3, 128), torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)))
    three, two = (psv.kv_cache(1 << 20, 1 << 20, n, "bf16", "head", 4) for n in (3, 2))
    x, t12 = f[0], i.reshape(1, 2)
    calls = [
        (lambda: psv.psv_rotate(f, f.double(), i, ROPE, None), "one shape"),
        (lambda: psv.psv_rotate(f, f, l, ROPE, None), "positions"),
        (lambda: psv.psv_rotate(f.transpose(1, 2), f.transpose(1, 2), i, ROPE, None), "adjacent"),
        (lambda: psv.psv_rotate(f, f, i[:1], ROPE, None), "positions"),
        (lambda: psv.psv_cache_gather(i, f, f, three, None), "slots"),
        (lambda: psv.psv_cache_gather(l, f, f, two, None), "heads"),
        (lambda: psv.psv_cache_gather(l, f, f[:, :2], three, None), "heads"),
        (lambda: psv.psv_cache_gather(l, f, f.transpose(1, 2), three, None), "adjacent"),
        (lambda: psv.psv_cache_append(None, f, f[:, :2], None, i, l, three, ROPE, None), "heads"),
        (lambda: psv.psv_cache_append(f, f, f, f[:1], i, l, three, ROPE, None), "rows"),
        (lambda: psv.psv_cache_append(f, f, f, f.half(), i, l, three, ROPE, None), "type"),
        (lambda: psv.psv_cache_append(None, f, f, None, i, i, three, ROPE, None), "slots"),
        (lambda: psv.psv_cache_append(None, f.int(), f.int(), None, i, l, three, ROPE, None), "float32"),
        (lambda: psv.psv_logprobs(x.t(), None, 1.0, None, None, None, None, f, None), "adjacent"),
        (lambda: psv.psv_logprobs(x, t12, 1.0, None, None, None, None, f, None), "tokens"),
        (lambda: psv.psv_logprobs_part(x, None, 1.0, 4, i, None), "bytes"),
        (lambda: psv.psv_logprobs_join(3, None, 1.0, 128, 1, 2, None, None, None, None, i, None, top=4), "bytes"),
    ]
    for call, what in calls:
        with pytest.raises(ValueError, match=what):
            call()
    assert library.calls == 0
    for pools in ((1 << 20, f[0, 0]), (f[0, 0], 1 << 20)):
        psv.kv_cache(*pools, 1, "bf16", "head", 4)
        with pytest.raises(ValueError, match="GPU"):
            psv.kv_cache(*(p if isinstance(p, int) else torch.zeros(8) for p in pools), 1, "bf16", "head", 4)
