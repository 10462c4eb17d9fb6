"""The operators around a decode step, as a serving program calls them, and the cases that they are timed on.

A case names one operator ("op") and its sizes.  `prepare` makes what the program has in hand -- rows, pools, tables, output
buffers -- and `run` is one call of the operator: of this library's (`own`), or in its plain form, written with elementary torch
operations in 32 bits.  `exact` is the same in 64 bits from the operator's definition.
"""
import math
import random

import numpy as np
import torch

own = False

# Local query and kv heads of the benchmark's shards.
SHARDS = {"small": (8, 8), "8b-tp8": (4, 1), "8b-tp4": (8, 2), "70b-tp8": (8, 1), "70b-tp4": (16, 2)}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK, DIM = 16, 128
THETA = 500000.0


def listed():
    return [
        # one new token for each of 64 users: the queries of a 70B-shaped shard, as the decode step's rotation has them
        dict(name="rotate_b64_decode", op="rotate", rows=64, heads=8, dim=128, dims=128, pairing="half", scaling="plain", dtype="bf16",
             span=32768, transpose=False),
        # a prompt part of a model that rotates half of each head in neighbouring pairs, context stretched eight times; odd row count
        dict(name="rotate_6001_partial_interleaved", op="rotate", rows=6001, heads=16, dim=128, dims=64, pairing="interleaved",
             scaling="turns", dtype="f16", span=65536, transpose=False),
        # gradient of a long document's queries in 32 bits, far positions
        dict(name="rotate_16384_transposed_f32", op="rotate", rows=16384, heads=16, dim=128, dims=128, pairing="half",
             scaling="channel", dtype="f32", span=1048576, transpose=True),
        # the next decode step of a full batch: every user brings one token
        dict(name="slots_b64_decode", op="slots", batch=64, new=1, context=8192, spread=False, max_blocks=2048),
        # prompts of very different lengths admitted together
        dict(name="slots_b509_prompts", op="slots", batch=509, new=400, context=3000, spread=True, max_blocks=2048),
        # one new token a user: 8B-shaped shard, bf16 cache
        dict(name="append_b64_decode", op="append", shard="8b-tp8", requests=64, new=1, context=4096, kv="bf16", layout="head",
             dtype="bf16", pairing="half", scaling="plain"),
        # a few prompts at once, each from the middle of a block on: 8B-shaped shard with two kv heads
        dict(name="append_8b_prompts", op="append", shard="8b-tp4", requests=5, new=1900, context=3001, kv="bf16", layout="head",
             dtype="bf16", pairing="half", scaling="turns"),
        # a long prompt of the small multi-head decoder: as many kv heads as query heads, token-major cache, rows of 32 bits
        dict(name="append_small_long", op="append", shard="small", requests=1, new=16384, context=0, kv="bf16", layout="token",
             dtype="f32", pairing="interleaved", scaling="plain"),
        # a prompt part into an int8 cache, then the whole sequence's keys and values for the part's attention
        dict(name="prompt_part_int8", op="part", shard="70b-tp4", requests=3, new=1024, context=5000, kv="int8", layout="head",
             dtype="bf16", pairing="half", scaling="plain"),
        # one user of a large vocabulary: the sampler's five alternatives
        dict(name="logprobs_b1_v128256", op="logprobs", rows=1, columns=128256, dtype="f32", given=1, top=5, temperature=1.0, masked=0.0),
        # a batch with constrained answers: most tokens are masked, an odd vocabulary, a temperature
        dict(name="logprobs_b61_v32003_masked", op="logprobs", rows=61, columns=32003, dtype="f16", given=1, top=20, temperature=0.7,
             masked=0.9),
        # a prompt is scored: every position's next token, with alternatives
        dict(name="logprobs_prompt_2048", op="logprobs", rows=2048, columns=128256, dtype="bf16", given=1, top=8, temperature=1.0,
             masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(2.0 ** rng.uniform(math.log2(lo), math.log2(hi + 1)))))


def draw(rng):
    """Rows 1-16384 (to 200k for slots), every shard, layout, format, type, pairing and scaling, part of a head; vocabularies
    1000-200000."""
    op = rng.choice(["rotate", "slots", "append", "part", "logprobs"])
    pairing, scaling = rng.choice(["half", "interleaved"]), rng.choice(["plain", "linear", "turns", "channel"])
    dtype = rng.choice(sorted(DTYPES))
    if op == "rotate":
        dim = rng.choice([64, 80, 96, 128, 192, 256])
        heads = rng.choice([1, 2, 5, 8, 16])
        rows = _log_int(rng, 1, min(16384, (1 << 25) // (heads * dim)))
        return dict(op=op, rows=rows, heads=heads, dim=dim, dims=rng.choice([dim, dim, dim // 2, dim // 4 * 2 - 6]),
                    pairing=pairing, scaling=scaling, dtype=dtype, span=_log_int(rng, max(64, rows), 1 << 20), transpose=rng.random() < 0.3)
    if op == "slots":
        new = _log_int(rng, 1, 2000)
        return dict(op=op, batch=_log_int(rng, 1, min(1024, 200000 // new)), new=new, context=_log_int(rng, 1, 8192),
                    spread=rng.random() < 0.7, max_blocks=2048)
    if op in ("append", "part"):
        kv = "int8" if op == "part" and rng.random() < 0.7 else "bf16"
        requests = _log_int(rng, 1, 64)
        most = 16384 if op == "append" else 4096
        return dict(op=op, shard=rng.choice(sorted(SHARDS)), requests=requests, new=_log_int(rng, 1, max(1, most // requests)),
                    context=rng.choice([0, _log_int(rng, 1, max(2, 16384 // requests))]), kv=kv,
                    layout=rng.choice(["head", "head", "token"]) if kv == "bf16" else "head",
                    dtype=dtype, pairing=pairing, scaling=scaling)
    columns = _log_int(rng, 1000, 200000)
    top = rng.choice([0, 1, 5, 20, 32])
    return dict(op=op, rows=_log_int(rng, 1, min(4096, 500000000 // (DTYPES[dtype].itemsize * columns))), columns=columns, dtype=dtype, given=rng.choice([0, 1, 1, 3]) if top else 1,
                top=top, temperature=rng.choice([1.0, 1.0, 0.6, 1.3]), masked=rng.choice([0.0, 0.0, 0.5, 0.95]))


# ---- what a program has in hand ------------------------------------------------------------------------------------------


def _rope_desc(case, dims):
    """Keywords of psv_rope_plan."""
    kw = dict(dims=dims, pairing=case["pairing"], scaling=case["scaling"], theta=THETA)
    if case["scaling"] != "plain":
        kw.update(factor=8.0)
    if case["scaling"] in ("turns", "channel"):
        kw.update(low_turns=1.0, high_turns=4.0 if case["scaling"] == "turns" else 32.0, trained_context=8192.0)
    if case["scaling"] == "channel":
        kw.update(magnitude=0.1 * math.log(8.0) + 1.0)
    return kw


def _requests(case, seed):
    """(tokens cached, new tokens) of every request of a batch; the seed decides their order."""
    n = case.get("requests", case.get("batch"))
    rng = random.Random(n * 1009 + case["new"])
    if not case.get("spread", True) or n == 1:
        return [case["context"]] * n, [case["new"]] * n
    if case["op"] == "slots":
        pairs = [(int(case["context"] * 2.0 ** rng.uniform(-6.0, 0.0)) if rng.random() < 0.8 else 0, max(1, int(2 * case["new"] * rng.random())))
                 for _ in range(n)]
    else:
        pairs = [(max(0, case["context"] - rng.randrange(min(40, case["context"] + 1))), case["new"]) for _ in range(n)]
    random.Random(seed).shuffle(pairs)
    return [a for a, _ in pairs], [b for _, b in pairs]


class State:
    pass


def _prepare_rotate(s, case, gen):
    rows, heads, dim, dt = case["rows"], case["heads"], case["dim"], DTYPES[case["dtype"]]
    s.x = torch.randn(rows, heads, dim, generator=gen, device="cuda").to(dt)
    start = int(torch.randint(0, max(1, case["span"] - rows), (1,), generator=gen, device="cuda"))
    s.positions = torch.arange(start, start + rows, dtype=torch.int32, device="cuda")
    s.y = torch.empty_like(s.x)


def _prepare_slots(s, case, seed):
    lens, new = _requests(case, seed)
    n, mb = case["batch"], case["max_blocks"]
    rng = np.random.RandomState(seed % (1 << 31))
    held = [(t + BLOCK - 1) // BLOCK for t in lens]
    want = [(t + k + BLOCK - 1) // BLOCK for t, k in zip(lens, new)]
    s.pool_blocks = sum(want) + 64
    ids = rng.permutation(s.pool_blocks).astype(np.int32)
    table, at = np.full((n, mb), -1, dtype=np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    s.rows = sum(new)
    dev = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int32), device="cuda")      # noqa: E731
    s.lens, s.new_lens, s.table, s.free = dev(lens), dev(new), dev(table), dev(ids[at:].copy())
    s.free_range = dev([0, len(ids) - at])
    s.seq_lens, s.row_starts, s.requests = torch.empty_like(s.lens), dev([0] * (n + 1)), dev(np.zeros(s.rows))
    s.positions, s.slots = torch.empty_like(s.requests), torch.empty(s.rows, dtype=torch.int64, device="cuda")
    s.free_out, s.refused = dev([0, 0]), dev([0])


def _prepare_rows(s, case, seed, gen):
    """Rows of one projection output [rows][(nq + 2 nkv) * 128], the cache they go to, and their places in it."""
    nq, nkv = SHARDS[case["shard"]]
    lens, new = _requests(case, seed)
    rows = sum(new)
    s.nkv = nkv
    qkv = torch.randn(rows, nq + 2 * nkv, DIM, generator=gen, device="cuda").to(DTYPES[case["dtype"]])
    s.q, s.k, s.v = qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:]
    s.q_out = torch.empty(rows, nq, DIM, dtype=qkv.dtype, device="cuda")
    blocks = [(a + b + BLOCK - 1) // BLOCK for a, b in zip(lens, new)]
    s.pool_blocks = sum(blocks)
    ids = np.random.RandomState(seed % (1 << 31)).permutation(s.pool_blocks).astype(np.int64)
    pos, slots, every, at = [], [], [], 0
    for a, b, n in zip(lens, new, blocks):
        p = np.arange(a + b)
        sl = ids[at + p // BLOCK] * BLOCK + p % BLOCK
        pos.append(p[a:])
        slots.append(sl[a:])
        every.append(sl)
        at += n
    s.positions = torch.as_tensor(np.concatenate(pos).astype(np.int32), device="cuda")
    s.slots = torch.as_tensor(np.concatenate(slots), device="cuda")
    s.every = torch.as_tensor(np.concatenate(every), device="cuda")      # the whole sequences
    shape = (s.pool_blocks, nkv)
    if case["kv"] == "int8":
        s.pools = []
        for _ in range(2):
            p = torch.empty(shape + (2112,), dtype=torch.int8, device="cuda")
            p[..., :2048] = torch.randint(-127, 128, shape + (2048,), generator=gen, device="cuda", dtype=torch.int8)
            p.view(torch.float32)[..., 512:] = 0.02 + 0.01 * torch.rand(shape + (16,), generator=gen, device="cuda")
            s.pools.append(p)
    else:
        k_shape = (s.pool_blocks, BLOCK, nkv, DIM) if case["layout"] == "token" else shape + (BLOCK, DIM)
        v_shape = k_shape if case["layout"] == "token" else shape + (DIM, BLOCK)
        s.pools = [torch.randn(sh, generator=gen, device="cuda").to(torch.bfloat16) for sh in (k_shape, v_shape)]
    if case["op"] == "part":
        s.k_all = torch.empty(len(s.every), nkv, DIM, dtype=torch.bfloat16, device="cuda")
        s.v_all = torch.empty_like(s.k_all)


def _prepare_logprobs(s, case, gen):
    rows, columns = case["rows"], case["columns"]
    s.logits = torch.empty(rows, columns, dtype=DTYPES[case["dtype"]], device="cuda")
    for r in range(0, rows, 256):
        x = 2.5 * torch.randn(min(256, rows - r), columns, generator=gen, device="cuda")
        likely = torch.randint(0, columns, (x.shape[0], 12), generator=gen, device="cuda")      # what the model means to say
        x.scatter_add_(1, likely, 4.0 + 8.0 * torch.rand(likely.shape, generator=gen, device="cuda"))
        if case["masked"]:
            x.masked_fill_(torch.rand(x.shape, generator=gen, device="cuda") < case["masked"], -math.inf)
        s.logits[r:r + 256] = x
    s.tokens = torch.randint(0, columns, (rows, case["given"]), generator=gen, device="cuda", dtype=torch.int32)
    s.logprobs = torch.empty(rows, case["given"], device="cuda")
    s.entropy = torch.empty(rows, device="cuda")
    s.top_logprobs = torch.empty(rows, case["top"], device="cuda")
    s.top_ids = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
    s.workspace = None


def prepare(case, seed):
    s = State()
    s.case, s.rope = case, None
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "rotate":
        _prepare_rotate(s, case, gen)
    elif case["op"] == "slots":
        _prepare_slots(s, case, seed)
    elif case["op"] == "logprobs":
        _prepare_logprobs(s, case, gen)
    else:
        _prepare_rows(s, case, seed, gen)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------


def _frequencies(desc):
    """Radians per position of every pair, in 64 bits, on the host."""
    n = desc["dims"] // 2
    f = desc["theta"] ** (-2.0 * torch.arange(n, dtype=torch.float64) / desc["dims"])
    if desc["scaling"] == "linear":
        f = f / desc["factor"]
    elif desc["scaling"] != "plain":
        turns = desc["trained_context"] * f / (2.0 * math.pi)
        if desc["scaling"] == "turns":
            w = ((turns - desc["low_turns"]) / (desc["high_turns"] - desc["low_turns"])).clamp(0.0, 1.0)
        else:
            at = [desc["dims"] * math.log(desc["trained_context"] / (2.0 * math.pi * t)) / (2.0 * math.log(desc["theta"]))
                  for t in (desc["high_turns"], desc["low_turns"])]
            lo, hi = max(0, math.floor(at[0])), min(desc["dims"] - 1, math.ceil(at[1]))
            w = 1.0 - ((torch.arange(n, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        f = w * f + (1.0 - w) * f / desc["factor"]
    return f


def _rotated(x, positions, desc, freq, transpose=False):
    """[rows, heads, dim] in 32 bits."""
    n = desc["dims"]
    angle = positions.double()[:, None] * freq
    m = desc.get("magnitude", 1.0)
    c, sn = (torch.cos(angle) * m).float()[:, None], (torch.sin(angle) * (-m if transpose else m)).float()[:, None]
    y = x.float().clone()
    if desc["pairing"] == "half":
        a, b = x[..., :n // 2].float(), x[..., n // 2:n].float()
        y[..., :n // 2], y[..., n // 2:n] = a * c - b * sn, b * c + a * sn
    else:
        a, b = x[..., 0:n:2].float(), x[..., 1:n:2].float()
        y[..., 0:n:2], y[..., 1:n:2] = a * c - b * sn, b * c + a * sn
    return y


def _plain_freq(s, dims):
    if s.rope is None:      # a program keeps its frequencies
        s.rope = (_rope_desc(s.case, dims), _frequencies(_rope_desc(s.case, dims)).cuda())
    return s.rope


def _plain_rotate(s):
    desc, freq = _plain_freq(s, s.case["dims"])
    return {"y": _rotated(s.x, s.positions, desc, freq, s.case["transpose"]).to(s.x.dtype)}


def _plain_slots(s):
    n, mb = s.table.shape
    lens, new = s.lens.long(), s.new_lens.long()
    ends = torch.cumsum(new, 0)
    starts = ends - new
    held = (lens + BLOCK - 1) // BLOCK
    need = (lens + new + BLOCK - 1) // BLOCK - held
    good = (lens + new <= mb * BLOCK) & (ends <= s.rows)
    need = torch.where(good, need, 0)
    taken = torch.cumsum(need, 0)
    good = good & ((need == 0) | (taken <= s.free_range[1] - s.free_range[0]))
    first = s.free_range[0] + taken - need                     # the request's first block in the free list
    col = torch.arange(mb, device=s.table.device)[None]
    fresh = good[:, None] & (col >= held[:, None]) & (col < (held + need)[:, None])
    table = torch.where(fresh, s.free[(first[:, None] + col - held[:, None]).clamp(0, len(s.free) - 1)], s.table)
    row = torch.arange(s.rows, device=s.table.device)
    req = torch.searchsorted(ends, row, right=True).clamp(max=n - 1)
    used = row < ends[-1]
    pos = lens[req] + row - starts[req]
    block = table[req, (pos // BLOCK).clamp(0, mb - 1)].long()
    slot = torch.where(used & good[req] & (block >= 0) & (block < s.pool_blocks), block * BLOCK + pos % BLOCK, -1)
    return {"table": table, "seq_lens": torch.where(good, lens + new, lens).int(),
            "row_starts": torch.cat([starts, ends[-1:]]).clamp(max=s.rows).int(), "slots": slot,
            "positions": torch.where(used, pos, 0).int(), "requests": torch.where(used, req, -1).int(),
            "free": torch.stack([s.free_range[0] + torch.where(good, need, 0).sum(), s.free_range[1].long()]).int(),
            "refused": (~good).sum().reshape(1).int()}


def _codes(t):
    scale = t.abs().amax(-1, keepdim=True) / 127.0
    scale = torch.where(scale > 0, scale, 1.0)
    return torch.clamp(torch.round(t / scale), -127, 127).to(torch.int8), scale[..., 0]


def _plain_append(s):
    desc, freq = _plain_freq(s, DIM)
    q = _rotated(s.q, s.positions, desc, freq).to(s.q.dtype)
    k, v = _rotated(s.k, s.positions, desc, freq), s.v.float()
    blk, off = s.slots // BLOCK, s.slots % BLOCK
    kp, vp = s.pools
    if s.case["kv"] == "int8":
        heads = torch.arange(s.nkv, device=k.device)[None]
        for rows, pool, shape in ((k, kp, (BLOCK, DIM)), (v, vp, (DIM, BLOCK))):
            codes, scale = _codes(rows)
            view = pool[..., :2048].unflatten(-1, shape)
            if shape[0] == BLOCK:
                view[blk, :, off] = codes
            else:
                view[blk, :, :, off] = codes
            pool.view(torch.float32)[blk[:, None], heads, 512 + off[:, None]] = scale
    elif s.case["layout"] == "token":
        kp[blk, off], vp[blk, off] = k.bfloat16(), v.bfloat16()
    else:
        kp[blk, :, off], vp[blk, :, :, off] = k.bfloat16(), v.bfloat16()
    return q


def _plain_gather(s):
    blk, off = s.every // BLOCK, s.every % BLOCK
    kp, vp = s.pools
    if s.case["kv"] == "int8":
        heads = torch.arange(s.nkv, device=blk.device)[None]
        k = kp[..., :2048].unflatten(-1, (BLOCK, DIM))[blk, :, off].float()
        v = vp[..., :2048].unflatten(-1, (DIM, BLOCK))[blk, :, :, off].float()
        k = k * kp.view(torch.float32)[blk[:, None], heads, 512 + off[:, None]][..., None]
        v = v * vp.view(torch.float32)[blk[:, None], heads, 512 + off[:, None]][..., None]
    elif s.case["layout"] == "token":
        k, v = kp[blk, off], vp[blk, off]
    else:
        k, v = kp[blk, :, off], vp[blk, :, :, off]
    return k.to(torch.bfloat16), v.to(torch.bfloat16)


def _plain_logprobs(s):
    scale, top = 1.0 / s.case["temperature"], s.case["top"]
    x = s.logits.float()
    most = x.amax(1, keepdim=True)
    d = (x - most) * scale
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log_s = torch.log(total)
    entropy = log_s[:, 0] - torch.where(e > 0, e * d, 0.0).sum(1) / total[:, 0]
    out = {"logprobs": torch.gather(d, 1, s.tokens.long()) - log_s, "entropy": entropy}
    del d, e
    if top:
        # largest first, equal ones by lowest id: one whole number a token that orders so
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 21
        key += (1 << 21) - 1 - torch.arange(x.shape[1], device=x.device)
        ids = (1 << 21) - 1 - (torch.topk(key, top, dim=1).values & ((1 << 21) - 1))
        values = torch.gather(x, 1, ids)
        there = values > -math.inf
        out["top_ids"] = torch.where(there, ids, -1).int()
        out["top_logprobs"] = torch.where(there, (values - most) * scale - log_s, -math.inf)
    return out


# ---- the library's operators ----------------------------------------------------------------------------------------------


def _own(s):
    from paper_2501_08192_amd import binding as psv
    case, stream = s.case, torch.cuda.current_stream()
    if case["op"] in ("rotate", "append", "part") and s.rope is None:      # a program keeps its frequencies
        s.rope = psv.psv_rope_plan(**_rope_desc(case, case.get("dims", DIM)))
    if case["op"] == "rotate":
        psv.psv_rotate(s.x, s.y, s.positions, s.rope, stream, transpose=case["transpose"])
        return {"y": s.y}
    if case["op"] == "slots":
        psv.psv_cache_slots(s.lens, s.new_lens, s.table, s.free, s.free_range, s.pool_blocks, s.seq_lens, s.row_starts, s.slots,
                            s.positions, s.requests, s.free_out, s.refused, stream)
        return {"table": s.table, "seq_lens": s.seq_lens, "row_starts": s.row_starts, "slots": s.slots, "positions": s.positions,
                "requests": s.requests, "free": s.free_out, "refused": s.refused}
    if case["op"] == "logprobs":
        if s.workspace is None:
            s.workspace = torch.empty(psv.psv_logprobs_bytes(case["rows"], psv.psv_logprobs_records(case["rows"], case["columns"]),
                                                             case["given"], case["top"]), dtype=torch.uint8, device="cuda")
        psv.psv_logprobs(s.logits, s.tokens, 1.0 / case["temperature"], s.logprobs, s.entropy, s.top_logprobs, s.top_ids, s.workspace, stream)
        return dict({"logprobs": s.logprobs, "entropy": s.entropy},
                    **({"top_ids": s.top_ids, "top_logprobs": s.top_logprobs} if case["top"] else {}))
    cache = psv.kv_cache(s.pools[0], s.pools[1], s.nkv, case["kv"], case["layout"], s.pool_blocks)
    psv.psv_cache_append(s.q, s.k, s.v, s.q_out, s.positions, s.slots, cache, s.rope, stream)
    if case["op"] == "append":
        return {"q": s.q_out, "k_pool": s.pools[0], "v_pool": s.pools[1]}
    psv.psv_cache_gather(s.every, s.k_all, s.v_all, cache, stream)
    return {"q": s.q_out, "k": s.k_all, "v": s.v_all}


def run(state):
    if own:
        return _own(state)
    op = state.case["op"]
    if op == "rotate":
        return _plain_rotate(state)
    if op == "slots":
        return _plain_slots(state)
    if op == "logprobs":
        return _plain_logprobs(state)
    q = _plain_append(state)
    if op == "append":
        return {"q": q, "k_pool": state.pools[0], "v_pool": state.pools[1]}
    k, v = _plain_gather(state)
    return {"q": q, "k": k, "v": v}


# ---- what a pass cannot do without, and its results in 64 bits -----------------------------------------------------------


def work(case):
    size = DTYPES[case["dtype"]].itemsize if "dtype" in case else 0
    if case["op"] == "rotate":
        n = case["rows"] * case["heads"] * case["dim"]
        return {"bytes": 2.0 * n * size + 4.0 * case["rows"], "flops": 3.0 * case["rows"] * case["heads"] * case["dims"]}
    if case["op"] == "slots":
        lens, new = _requests(case, 1)
        blocks = sum((a + b + BLOCK - 1) // BLOCK - (a + BLOCK - 1) // BLOCK for a, b in zip(lens, new))
        return {"bytes": 16.0 * sum(new) + 16.0 * case["batch"] + 8.0 * blocks, "flops": 0.0}
    if case["op"] == "logprobs":
        n = float(case["rows"]) * case["columns"]
        return {"bytes": n * size + case["rows"] * (8.0 * case["given"] + 4.0 + 8.0 * case["top"]), "flops": 6.0 * n}
    nq, nkv = SHARDS[case["shard"]]
    rows = case["requests"] * case["new"]
    cached = 2.0 * nkv * (DIM + 4 if case["kv"] == "int8" else 2 * DIM)      # keys and values of one token in the cache
    moved = rows * ((2 * nq + 2 * nkv) * DIM * size + cached + 12.0)
    if case["op"] == "part":
        tokens = sum(_requests(case, 1)[0]) + rows
        moved += tokens * (cached + 2.0 * nkv * DIM * 2 + 8.0)
    return {"bytes": moved, "flops": 3.0 * rows * (nq + nkv) * DIM}


def _turned(x, positions, case, dims, transpose=False):
    """The rotation in 64 bits, a pair as a complex number."""
    d = _rope_desc(case, dims)
    i = torch.arange(dims // 2, dtype=torch.float64, device=x.device)
    f = torch.exp(i * (-2.0 / dims * math.log(d["theta"])))
    if d["scaling"] == "linear":
        f = f / d["factor"]
    elif d["scaling"] == "turns":
        n = d["trained_context"] * f / (2 * math.pi)
        w = torch.clamp((n - d["low_turns"]) / (d["high_turns"] - d["low_turns"]), 0, 1)
        f = f * w + f / d["factor"] * (1 - w)
    elif d["scaling"] == "channel":
        lo, hi = (dims * math.log(d["trained_context"] / (2 * math.pi * n)) / (2 * math.log(d["theta"]))
                  for n in (d["high_turns"], d["low_turns"]))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), dims - 1)
        w = 1 - torch.clamp((i - lo) / max(hi - lo, 0.001), 0, 1)
        f = f * w + f / d["factor"] * (1 - w)
    angle = positions.double()[:, None, None] * f
    turn = torch.polar(torch.full_like(angle, d.get("magnitude", 1.0)), -angle if transpose else angle)
    x = x.double()
    head, rest = x[..., :dims], x[..., dims:]
    pairs = head.unflatten(-1, (2, dims // 2)).transpose(-1, -2) if d["pairing"] == "half" else head.unflatten(-1, (dims // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = y.transpose(-1, -2) if d["pairing"] == "half" else y
    return torch.cat([y.flatten(-2), rest], dim=-1)


def _exact_logprobs(s):
    scale, top = 1.0 / s.case["temperature"], s.case["top"]
    lp, ent, best = [], [], []
    for r in range(0, s.case["rows"], 256):
        z = s.logits[r:r + 256].double() * scale
        logp = z - torch.logsumexp(z, dim=1, keepdim=True)
        lp.append(logp.gather(1, s.tokens[r:r + 256].long()))
        ent.append(-torch.nan_to_num(logp * torch.exp(logp), nan=0.0).sum(1))
        if top:
            best.append(torch.topk(logp, top, dim=1).values)
    out = {"logprobs": torch.cat(lp), "entropy": torch.cat(ent)}
    if top:
        out.update(top_ids=None, top_logprobs=torch.cat(best))
    return out


def exact(case, seed):
    if case["op"] == "slots":
        return None      # whole numbers
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return {"y": _turned(s.x, s.positions, case, case["dims"], case["transpose"])}
    if case["op"] == "logprobs":
        return _exact_logprobs(s)
    q, k, v = _turned(s.q, s.positions, case, DIM), _turned(s.k, s.positions, case, DIM), s.v.double()
    blk, off = s.slots // BLOCK, s.slots % BLOCK

    def dense(pool, channel_major):
        """[blocks, 16, kv heads, 128] in 64 bits."""
        if case["kv"] == "int8":
            scale = pool[..., 2048:].contiguous().view(torch.float32).double()
            codes = pool[..., :2048].double()
            codes = codes.unflatten(-1, (DIM, BLOCK)).transpose(2, 3) if channel_major else codes.unflatten(-1, (BLOCK, DIM))
            return (codes * scale[..., None]).transpose(1, 2).contiguous()
        p = pool.double()
        if case["layout"] == "token":
            return p
        return (p.permute(0, 3, 1, 2) if channel_major else p.transpose(1, 2)).contiguous()

    both = []
    for rows, pool, channel_major in ((k, s.pools[0], False), (v, s.pools[1], True)):
        p = dense(pool, channel_major)
        if case["kv"] == "int8":      # the stored code is a decision in single precision
            step = rows.abs().amax(-1, keepdim=True).float() / 127
            step = torch.where(step > 0, step, torch.ones_like(step))
            rows = torch.round(rows.float() / step).clamp(-127, 127).double() * step.double()
        p[blk, off] = rows
        both.append(p)
    if case["op"] == "part":
        at, o = s.every // BLOCK, s.every % BLOCK
        return {"q": q, "k": both[0][at, o], "v": both[1][at, o]}
    if case["layout"] == "head":
        both = [both[0].transpose(1, 2), both[1].permute(0, 2, 3, 1)]
    return {"q": q, "k_pool": both[0].contiguous(), "v_pool": both[1].contiguous()}
