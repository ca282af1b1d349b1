"""Cases that a pool of cache blocks, attention over a shared prefix and filtered sampling are measured on.

Several continuations of one source: the prompt's blocks are shared by all of them (`cache_fork`), each gets blocks of its own where it goes on
(`cache_reserve`), attention reads the shared positions once for all (`cache_attention_shared`), and the next tokens are drawn from what
temperature, top-k, top-p and min-p leave (`sample`).  Continuations that end make room for others; what is in use moves to the front of the pool
(`cache_compact`).  Head layouts, vocabularies and lengths are those of the model shapes and recipes in `paper_2205_10350_b200/synth.py` where the
library's own models use them, and grouped heads of 128 with long prefixes for what a user's decoder of another make brings along.

`run` computes the plain form from elementary torch operations, or, with `own`, makes the library's calls.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

DEV = "cuda:0"
own = False

GOLDEN = 0.6180339887498949


def listed():
    return [
        # hypotheses of one sentence change places: launch and latency
        dict(name="fork_b8", op="fork", batch=8, beams=8, len_lo=33, len_hi=57, block=32, row_blocks=16),
        # the same for a full batch of beams with long rows in small blocks
        dict(name="fork_b512", op="fork", batch=512, beams=8, len_lo=900, len_hi=32000, block=16, row_blocks=2050),
        # one sentence becomes eight samples, each of which goes on by a token: six layers of the base model
        dict(name="branch_n8", op="branch", prompts=1, samples=8, len_lo=40, len_hi=40, new_lo=1, new_hi=1, kv_heads=8, dim=64, block=32, fmt="e4m3", layers=6),
        # long prompts into eight samples each that go on by blocks of drafted tokens, grouped heads
        dict(name="branch_b32_n8", op="branch", prompts=32, samples=8, len_lo=500, len_hi=4000, new_lo=1, new_hi=64, kv_heads=8, dim=128, block=64, fmt="int8",
             layers=6),
        # half of a batch of sentences has ended, others come in
        dict(name="turnover_b8", op="turnover", batch=8, len_lo=100, len_hi=400, kv_heads=8, dim=64, block=32, fmt="int8", layers=6),
        # the same for long rows
        dict(name="turnover_b64", op="turnover", batch=64, len_lo=700, len_hi=2100, kv_heads=8, dim=128, block=64, fmt="e4m3", layers=6),
        # eight samples of one sentence, a token each
        dict(name="attend_n8", op="attend", prompts=1, samples_lo=8, samples_hi=8, new_lo=1, new_hi=1, shared_lo=40, shared_hi=40, tail_lo=0, tail_hi=20, heads=8,
             kv_heads=8, dim=64, block=32, fmt="e4m3", dtype="bf16", causal=True),
        # cross-attention of sixteen samples with blocks of up to 25 tokens over the encoder's keys of each of eight sources, FP32 activations
        dict(name="attend_source_b8_n16", op="attend", prompts=8, samples_lo=16, samples_hi=16, new_lo=5, new_hi=25, shared_lo=250, shared_hi=400, tail_lo=0,
             tail_hi=0, heads=8, kv_heads=8, dim=64, block=32, fmt="int8", dtype="fp32", causal=False),
        # a token of each of 64 samples behind one long prefix, grouped heads
        dict(name="attend_n64_long", op="attend", prompts=1, samples_lo=64, samples_hi=64, new_lo=1, new_hi=1, shared_lo=32000, shared_hi=32000, tail_lo=1,
             tail_hi=500, heads=32, kv_heads=8, dim=128, block=64, fmt="e4m3", dtype="bf16", causal=True),
        # drafts of samples of four prompts, grouped heads: many queries a prefix
        dict(name="attend_b4_n32_k8", op="attend", prompts=4, samples_lo=24, samples_hi=32, new_lo=3, new_hi=8, shared_lo=6000, shared_hi=16000, tail_lo=10,
             tail_hi=700, heads=32, kv_heads=8, dim=128, block=64, fmt="int8", dtype="bf16", causal=True),
        # the next token of one sentence
        dict(name="sample_b1", op="sample", rows=1, vocab=32000, dtype="fp32", filters="p", filtered=False),
        # next tokens of a full batch, each row with its own filters, and the scores that are left for a verification of drafts
        dict(name="sample_b256", op="sample", rows=256, vocab=128000, dtype="bf16", filters="mixed", filtered=True),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    op = rng.choice(["fork", "branch", "turnover", "attend", "attend", "attend", "sample", "sample"])
    if op == "sample":
        return dict(op=op, rows=_log_int(rng, 1, 512), vocab=rng.choice([1000, 32000, 50265, _log_int(rng, 500, 160000)]), dtype=rng.choice(["fp32", "bf16"]),
                    filters=rng.choice(["k", "p", "min", "mixed", "mixed"]), filtered=rng.random() < 0.4)
    block = rng.choice([16, 32, 64, 128])
    if op == "fork":
        beams, len_hi = rng.choice([2, 4, 5, 8, 16]), _log_int(rng, 20, 32000)
        return dict(op=op, batch=beams * _log_int(rng, 1, 64), beams=beams, len_lo=rng.randint(1, len_hi), len_hi=len_hi, block=block,
                    row_blocks=(len_hi + block - 1) // block + rng.randint(0, 20))
    layout = dict(kv_heads=rng.choice([4, 8, 8, 16]), dim=rng.choice([32, 64, 64, 128]), block=block, fmt=rng.choice(["e4m3", "int8"]))
    if op == "attend":
        samples_hi, new_hi, shared_hi = _log_int(rng, 1, 64), _log_int(rng, 1, 25), _log_int(rng, 20, 40000)
        causal, tail_hi = rng.random() < 0.75, _log_int(rng, 1, 1000)
        return dict(op=op, prompts=_log_int(rng, 1, 8), samples_lo=rng.randint(max(1, samples_hi // 2), samples_hi), samples_hi=samples_hi,
                    new_lo=rng.randint(1, new_hi), new_hi=new_hi, shared_lo=rng.randint(shared_hi // 3, shared_hi), shared_hi=shared_hi,
                    tail_lo=rng.randint(0, tail_hi) if causal else 0, tail_hi=tail_hi if causal else 0, heads=layout["kv_heads"] * rng.choice([1, 1, 2, 4]),
                    dtype=rng.choice(["fp32", "bf16", "bf16"]), causal=causal, **layout)
    layers, len_hi = rng.choice([1, 2, 6, 6, 12]), _log_int(rng, 20, 5000)
    if op == "turnover":
        return dict(op=op, batch=2 * _log_int(rng, 1, 64), len_lo=rng.randint(1, len_hi), len_hi=len_hi, layers=layers, **layout)
    new_hi = _log_int(rng, 1, 200)
    return dict(op=op, prompts=_log_int(rng, 1, 32), samples=rng.randint(2, 16), len_lo=rng.randint(1, len_hi), len_hi=len_hi, new_lo=rng.randint(1, new_hi),
                new_hi=new_hi, layers=layers, **layout)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


@functools.lru_cache(maxsize=None)
def _largest():
    return {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("fork", "branch", "turnover", "attend", "sample")}


def draw(rng):
    while True:
        case = _draw_once(rng)
        if _cost(case) <= _largest()[case["op"]] and _pool_bytes(case) <= 4 << 30:
            return case


# ------------------------------------------------------------------------------------------------------
# sizes of a case
# ------------------------------------------------------------------------------------------------------
def _spread(lo, hi, n, first):
    """n whole numbers between lo and hi, both ends among them where n > 1, the rest spread out."""
    if n == 1:
        return [hi]
    return [lo, hi][:n] + [lo + int((hi - lo) * ((first + (b + 1) * GOLDEN) % 1.0)) for b in range(n - 2)]


def _up(n, block):
    return (n + block - 1) // block


def _fork_lens(case):
    """Tokens that a row keeps."""
    return _spread(case["len_lo"], case["len_hi"], case["batch"], 0.2)


def _branch_rows(case):
    """(tokens of every prompt, new tokens of every row)."""
    return _spread(case["len_lo"], case["len_hi"], case["prompts"], 0.0), _spread(case["new_lo"], case["new_hi"], case["prompts"] * case["samples"], 0.37)


def _turnover_lens(case):
    """Tokens of the rows of either half of the batch."""
    return _spread(case["len_lo"], case["len_hi"], case["batch"] // 2, 0.1)


def _attend_rows(case):
    """(rows of every prompt, shared positions of every prompt, new tokens and tail of every row)."""
    samples = _spread(case["samples_lo"], case["samples_hi"], case["prompts"], 0.5)
    n = sum(samples)
    return (samples, _spread(case["shared_lo"], case["shared_hi"], case["prompts"], 0.1), _spread(case["new_lo"], case["new_hi"], n, 0.0),
            _spread(case["tail_lo"], case["tail_hi"], n, 0.37)[::-1])


def _block_bytes(case):
    """A block's codes and scales, keys and values, all layers."""
    return 2 * case["layers"] * case["kv_heads"] * (case["block"] * case["dim"] + 4)


def _pool_blocks(case):
    bl = case["block"]
    if case["op"] == "branch":
        lens, new = _branch_rows(case)
        return sum(_up(n, bl) for n in lens) + sum(_up(n, bl) + 1 for n in new) + 5
    lens = _turnover_lens(case)
    return 2 * sum(_up(n, bl) for n in lens) + case["batch"] + 5


def _pool_bytes(case):
    return _pool_blocks(case) * _block_bytes(case) if case["op"] in ("branch", "turnover") else 0


def _element(case):
    return 4 if case["dtype"] == "fp32" else 2


def work(case):
    """Bytes: every input read once, every output written once.  Operations: a multiplication and an addition of each product; a handful of
    operations per element where there are no products."""
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * _element(case) * (2 if case["filtered"] else 1) + case["rows"] * 28, "flops": 4 * n}
    bl = case["block"]
    if case["op"] == "fork":
        # entries that stay, read and written, and what is counted of their blocks
        held = sum(_up(n, bl) for n in _fork_lens(case))
        return {"bytes": 8 * held + 8 * held + 8 * case["batch"], "flops": 2 * held}
    if case["op"] == "branch":
        lens, new = _branch_rows(case)
        B, token = len(new), 2 * case["layers"] * case["kv_heads"] * case["dim"]
        held = sum(_up(n, bl) for n in lens) * case["samples"]
        fresh = sum(_up(n + new[g * case["samples"] + s], bl) - _up(n, bl) for g, n in enumerate(lens) for s in range(case["samples"]))
        copies = sum((n % bl) * (case["samples"] - 1) for n in lens)
        return {"bytes": 16 * (held + fresh) + 2 * copies * token + 12 * B, "flops": 2 * held}
    if case["op"] == "turnover":
        held = sum(_up(n, bl) for n in _turnover_lens(case))
        return {"bytes": 2 * held * _block_bytes(case) + 2 * 16 * held + 16 * case["batch"], "flops": 4 * held}
    samples, shared, new, tail = _attend_rows(case)
    rows = [g for g, n in enumerate(samples) for _ in range(n)]
    M, token, own_keys = sum(new), case["kv_heads"] * case["dim"] * 2, [t + n if case["causal"] else t for t, n in zip(tail, new)]
    pairs = sum(n * (shared[g] + t) + (n * (n + 1) // 2 if case["causal"] else 0) for g, n, t in zip(rows, new, tail))
    return {"bytes": (sum(shared) + sum(own_keys)) * token + 2 * M * case["heads"] * case["dim"] * _element(case),
            "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------
def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _offsets(n):
    return _int([0] + [int(x) for x in np.cumsum(n)])


def _code_type(fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.int8


def _any_codes(case, n_blocks, g):
    """Codes and scales of blocks that are only moved about."""
    shape = (n_blocks, case["kv_heads"], case["block"], case["dim"])
    codes = torch.randint(0, 120, shape, generator=g, device=DEV, dtype=torch.uint8).view(_code_type(case["fmt"]))
    return codes, torch.exp2(torch.randint(-9, 3, shape[:2], generator=g, device=DEV).float())


def _rows_of_blocks(needs, ids, row_blocks):
    """Table whose row b holds the next needs[b] of ids."""
    table = torch.full((len(needs), row_blocks), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(needs):
        table[b, :n] = ids[at: at + n]
        at += n
    return table


def _prepare_pool(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    bl = case["block"]
    state = dict(case=case)
    if case["op"] == "fork":
        B, beams = case["batch"], case["beams"]
        lens = _fork_lens(case)
        held = [min(case["row_blocks"], _up(case["len_hi"], bl))] * B
        n_blocks = sum(held) + 3
        table = _rows_of_blocks(held, torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32), case["row_blocks"])
        # every hypothesis goes on from one of its sentence's, good ones more than once
        chosen = (torch.rand(B, generator=g, device=DEV).pow(2) * beams).long().clamp_max(beams - 1)
        state["parent"] = (torch.arange(B, device=DEV) // beams * beams + chosen).to(torch.int32)
        state["keep"] = _int(lens)
    elif case["op"] == "branch":
        lens, new = _branch_rows(case)
        S = case["samples"]
        n_blocks = _pool_blocks(case)
        row_blocks = max(_up(n + new[i * S + s], bl) for i, n in enumerate(lens) for s in range(S)) + 1
        needs = [_up(lens[b // S], bl) if b % S == 0 else 0 for b in range(len(new))]
        table = _rows_of_blocks(needs, torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32), row_blocks)
        state["parent"], state["keep"] = _int([b // S * S for b in range(len(new))]), _int([lens[b // S] for b in range(len(new))])
        state["off"], state["len"] = _offsets(new), state["keep"]
    else:
        # rows of the front half have ended; the others move there, and new ones come in behind them
        lens = _turnover_lens(case)
        half = len(lens)
        n_blocks = _pool_blocks(case)
        needs = [_up(n, bl) for n in lens] * 2
        front = torch.randperm(sum(needs) // 2, generator=g, device=DEV)
        back = torch.randperm(sum(needs) // 2, generator=g, device=DEV) + sum(needs) // 2 + 2
        table = _rows_of_blocks(needs, torch.cat([front, back]).to(torch.int32), max(needs) + 1)
        state["parent"], state["keep"] = _int([b + half for b in range(half)] + [-1] * half), _int(lens + [0] * half)
        state["off"], state["len"] = _offsets([1] * half + lens), _int(lens + [0] * half)
    state["table"] = table
    state["refs"] = torch.bincount(table[table >= 0].long(), minlength=n_blocks).to(torch.int32)
    state["layers"] = []
    for _ in range(case.get("layers", 0)):
        (kc, ks), (vc, vs) = _any_codes(case, n_blocks, g), _any_codes(case, n_blocks, g)
        state["layers"].append((kc, vc, ks, vs))
    if own:
        from paper_2205_10350_b200 import binding
        state["pool"] = binding.KvPool(table.shape[0], table.shape[1], n_blocks, bl, device=DEV, tensors=(table, state["refs"]))
        for layer in state["layers"]:
            state["pool"].add_cache(case["kv_heads"], case["dim"], case["fmt"], tensors=layer)
    return state


def _scale_for(amax, fmt):
    """The smallest power of two s with amax / s within the format."""
    m, e = torch.frexp(amax)
    bits, edge = (9, 0.875) if fmt == "e4m3" else (7, 127.0 / 128.0)
    return torch.ldexp(torch.ones_like(m), (e - bits + (m > edge)).to(torch.float32))


def _filled(case, n_blocks, g):
    """Codes and scales of a cache whose blocks have been written: normal values, some channels and some blocks larger than others."""
    shape = (n_blocks, case["kv_heads"], case["block"], case["dim"])
    codes = torch.empty(shape, dtype=torch.uint8, device=DEV).view(_code_type(case["fmt"]))
    scale = torch.empty(shape[:2], device=DEV)
    channel = torch.exp(0.5 * torch.randn((1, case["kv_heads"], 1, case["dim"]), generator=g, device=DEV))
    step = max(1, (1 << 27) // (shape[1] * shape[2] * shape[3]))
    for b in range(0, n_blocks, step):
        n = min(step, n_blocks - b)
        x = torch.randn((n,) + shape[1:], generator=g, device=DEV)
        x *= channel
        x *= torch.exp(0.3 * torch.randn((n, shape[1], 1, 1), generator=g, device=DEV))
        s = _scale_for(x.abs().amax((2, 3)), case["fmt"])
        x /= s[:, :, None, None]
        codes[b: b + n] = x.to(torch.float8_e4m3fn) if case["fmt"] == "e4m3" else x.round().clamp(-127, 127).to(torch.int8)
        scale[b: b + n] = s
    return codes, scale


def _prepare_attend(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    samples, shared, new, tail = _attend_rows(case)
    group = [i for i, n in enumerate(samples) for _ in range(n)]
    B, M, bl = len(new), sum(new), case["block"]
    lens = [shared[i] + t for i, t in zip(group, tail)]
    ends = [o + n if case["causal"] else o for o, n in zip(lens, new)]
    row_blocks = max(_up(n, bl) for n in ends) + 1
    # the blocks that the shared positions fill stand in all rows of a prompt; from there on each row has its own, or, where that is all there is to
    # look at (an encoder's keys), the last one is shared like the others
    whole = [_up(n, bl) if not case["causal"] else n // bl for n in shared]
    n_blocks = sum(whole) + sum(_up(e, bl) - min(whole[i], _up(e, bl)) for i, e in zip(group, ends)) + 3
    order = torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, row_blocks), -1, dtype=torch.int32, device=DEV)
    at, first = 0, [0]
    k, v = _filled(case, n_blocks, g), _filled(case, n_blocks, g)
    b = 0
    for i, n in enumerate(samples):
        table[b: b + n, : whole[i]] = order[at: at + whole[i]]
        at += whole[i]
        for r in range(b, b + n):
            more = _up(ends[r], bl) - whole[i]
            if more > 0:
                table[r, whole[i]: whole[i] + more] = order[at: at + more]
                at += more
        if case["causal"] and shared[i] % bl:
            # rows that were forked inside a block hold the same tokens in copies of it
            ids = table[b: b + n, whole[i]].long()
            for codes, scale in (k, v):
                raw = codes.view(torch.uint8)
                raw[ids[1:], :, : shared[i] % bl] = raw[ids[:1], :, : shared[i] % bl]
                scale[ids[1:]] = scale[ids[:1]]
        b += n
        first.append(b)
    state = dict(case=case, q=(torch.randn((M, case["heads"], case["dim"]), generator=g, device=DEV) * 1.2).to(dt), off=_offsets(new), len=_int(lens),
                 groups=_int(first), shared=_int(shared), table=table, k=k, v=v, most=max(ends), most_shared=max(shared))
    if own:
        from paper_2205_10350_b200 import binding
        state["cache"] = binding.KvCache(n_blocks, case["kv_heads"], case["dim"], bl, case["fmt"], table=table, device=DEV, tensors=(k[0], v[0], k[1], v[1]))
    return state


def _prepare_sample(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    M, V = case["rows"], case["vocab"]
    scores = torch.randn((M, V), generator=g, device=DEV)
    scores *= 2.0
    likely = torch.randint(4, V, (M, 3), generator=g, device=DEV)         # a few tokens hold most of a row's probability
    scores.scatter_add_(1, likely, torch.tensor([[12.0, 10.0, 9.0]], device=DEV).expand(M, 3))
    row = torch.arange(M, device=DEV)
    pick = lambda values, shift: torch.tensor(values, device=DEV)[(row + shift) % len(values)]
    state = dict(case=case, scores=scores.to(torch.float32 if case["dtype"] == "fp32" else torch.bfloat16), r=torch.rand(M, generator=g, device=DEV),
                 temperature=pick([0.8, 1.0, 1.3, 0.6, 2.0], seed), top_k=None, top_p=None, min_p=None)
    mixed = case["filters"] == "mixed"
    if mixed or case["filters"] == "k":
        state["top_k"] = pick([50, 0, 40, 1, 1000, 20, 0], seed).to(torch.int32)
    if mixed or case["filters"] == "p":
        state["top_p"] = pick([0.9, 0.95, 1.0, 0.8, 0.99], 0)
    if mixed or case["filters"] == "min":
        state["min_p"] = pick([0.0, 0.05, 0.0, 0.01, 0.1, 0.0001], 1)
    return state


def prepare(case, seed):
    return {"attend": _prepare_attend, "sample": _prepare_sample}.get(case["op"], _prepare_pool)(case, seed)


# ------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------
def _plain_fork(state):
    """Row b becomes the first keep[b] tokens of row parent[b]; blocks are counted by the entries that name them."""
    table, refs = state["table"], state["refs"]
    held = (state["keep"].long() + state["case"]["block"] - 1) // state["case"]["block"]
    held = torch.where(state["parent"] < 0, 0, held)
    old = table[state["parent"].long().clamp_min(0)]
    table.copy_(torch.where(torch.arange(table.shape[1], device=DEV)[None, :] < held[:, None], old, -1))
    refs.copy_(torch.bincount(table[table >= 0].long(), minlength=refs.numel()))


def _plain_reserve(state):
    """Blocks for the new tokens: where there is none yet, and where others hold it too."""
    case, table, refs = state["case"], state["table"], state["refs"]
    bl, n_blocks = case["block"], refs.numel()
    start, n = state["len"].long(), (state["off"][1:] - state["off"][:-1]).long()
    place = torch.arange(table.shape[1], device=DEV)[None, :]
    written = (n > 0)[:, None] & (place >= (start // bl)[:, None]) & (place <= ((start + n - 1) // bl)[:, None])
    entry = table.long()
    others = written & (entry >= 0) & (refs[entry.clamp_min(0)] > 1)
    at = torch.arange(table.numel(), device=DEV).view_as(table)
    writers = torch.zeros(n_blocks, dtype=torch.int64, device=DEV).index_add_(0, entry[others], torch.ones_like(entry[others]))
    first = torch.full((n_blocks,), table.numel(), device=DEV).scatter_reduce_(0, entry[others], at[others], "amin")
    # the first of its writers keeps a block that nobody else holds
    keeps = others & (writers == refs)[entry.clamp_min(0)] & (first[entry.clamp_min(0)] == at)
    fresh = (written & (entry < 0)) | (others & ~keeps)
    ids = torch.nonzero(refs == 0)[:, 0][: int(fresh.sum())]
    left = entry[others & ~keeps]
    copied = (others & ~keeps)[fresh] & (place.expand_as(table)[fresh] == (start // bl).repeat_interleave(fresh.sum(1)))
    src, dst = entry[fresh][copied], ids[copied]
    live = (start % bl).repeat_interleave(fresh.sum(1))[copied]
    table[fresh] = ids.to(torch.int32)
    refs[ids] = 1
    refs.index_add_(0, left, torch.full_like(left, -1, dtype=torch.int32))
    token = torch.arange(bl, device=DEV)
    for layer in state["layers"]:
        for codes in layer[:2]:
            raw = codes.view(torch.uint8)
            raw[dst] = torch.where(token[None, None, :, None] < live[:, None, None, None], raw[src], raw[dst])
        for scale in layer[2:]:
            scale[dst] = torch.where((live > 0)[:, None], scale[src], scale[dst])


def _plain_compact(state):
    """Blocks in use behind their number move to the free ones in front of it, both in order."""
    table, refs = state["table"], state["refs"]
    used = int((refs > 0).sum())
    holes, movers = torch.nonzero(refs[:used] == 0)[:, 0], torch.nonzero(refs[used:] > 0)[:, 0] + used
    to = torch.arange(refs.numel(), device=DEV, dtype=torch.int32)
    to[movers] = holes.to(torch.int32)
    table.copy_(torch.where(table >= 0, to[table.long().clamp_min(0)], table))
    refs[holes] = refs[movers]
    refs[movers] = 0
    for layer in state["layers"]:
        for x in layer:
            raw = x if x.dtype == torch.float32 else x.view(torch.uint8)
            raw[holes] = raw[movers]
    return torch.tensor([used], dtype=torch.int32, device=DEV)


def _row_values(state, name, b, lo, hi, wide):
    """Values of positions lo..hi-1 of row b, [heads, tokens, dim]."""
    bl = state["case"]["block"]
    codes, scale = state[name]
    ids = state["table"][b, lo // bl: (hi - 1) // bl + 1].long()
    x = codes.view(torch.uint8)[ids].view(codes.dtype).to(wide) * scale[ids].to(wide)[:, :, None, None]
    return x.transpose(0, 1).flatten(1, 2)[:, lo - lo // bl * bl: hi - lo // bl * bl]


def _plain_attend(state):
    case, q = state["case"], state["q"]
    samples, shared, new, tail = _attend_rows(case)
    out = torch.zeros_like(q)
    per_kv, D = case["heads"] // case["kv_heads"], case["dim"]
    b = at = 0
    for i, rows in enumerate(samples):
        kp, vp = (_row_values(state, c, b, 0, shared[i], torch.float32) for c in ("k", "v")) if shared[i] else (None, None)
        for _ in range(rows):
            n, hi = new[b], shared[i] + tail[b] + (new[b] if case["causal"] else 0)
            if hi:
                parts = [(kp, vp)] if shared[i] else []
                if hi > shared[i]:
                    parts.append(tuple(_row_values(state, c, b, shared[i], hi, torch.float32) for c in ("k", "v")))
                k, v = (torch.cat([p[z] for p in parts], 1) for z in range(2))
                qb = q[at: at + n].float().view(n, case["kv_heads"], per_kv, D).permute(1, 0, 2, 3).flatten(1, 2)
                s = qb @ k.transpose(1, 2) * D ** -0.5                                          # [kv heads, n * per_kv, keys]
                if case["causal"]:
                    sees = shared[i] + tail[b] + 1 + torch.arange(n, device=DEV).repeat_interleave(per_kv)
                    s = s.masked_fill(torch.arange(hi, device=DEV)[None, :] >= sees[:, None], -math.inf)
                s = torch.exp(s - s.amax(2, keepdim=True))
                s = (s / s.sum(2, keepdim=True)) @ v
                out[at: at + n] = s.unflatten(1, (n, per_kv)).permute(1, 0, 2, 3).flatten(1, 2).to(out.dtype)
            at += n
            b += 1
    return out


def _plain_sample(state):
    case, scores = state["case"], state["scores"]
    M, V = scores.shape
    tokens, logp = torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(M, device=DEV)
    filtered = torch.empty_like(scores) if case["filtered"] else None
    step = max(1, (1 << 24) // V)
    for lo in range(0, M, step):
        sl = slice(lo, min(M, lo + step))
        # 64 bits: a random number or a threshold next to a border of the distribution decides on a token
        x, order = torch.sort(scores[sl].double(), dim=1, descending=True, stable=True)         # (ties: lowest id first)
        w = torch.exp((x - x[:, :1]) / state["temperature"][sl].double()[:, None])
        keep = torch.ones_like(w, dtype=torch.bool)
        if state["top_k"] is not None:
            k = state["top_k"][sl].long()[:, None]
            keep &= (k <= 0) | (torch.arange(V, device=DEV)[None, :] < k)
        if state["top_p"] is not None:
            p, inside = state["top_p"][sl].double()[:, None], torch.where(keep, w, torch.zeros_like(w))
            total = torch.cumsum(inside, 1)
            keep &= (p >= 1) | (total - inside < p * total[:, -1:])
        keep[:, 0] = True
        if state["min_p"] is not None:
            keep &= w >= state["min_p"][sl].double()[:, None]
        # back in the order of ids
        w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, torch.zeros_like(w)))
        total = torch.cumsum(w, 1)
        t = (total <= state["r"][sl].double()[:, None] * total[:, -1:]).sum(1).clamp_max(V - 1)
        tokens[sl] = t.to(torch.int32)
        logp[sl] = torch.log(w.gather(1, t[:, None])[:, 0] / total[:, -1]).float()
        if filtered is not None:
            kept = torch.zeros_like(keep).scatter_(1, order, keep)
            filtered[sl] = torch.where(kept, scores[sl], torch.full_like(scores[sl], -math.inf))
    return [tokens, logp] + ([filtered] if filtered is not None else [])


def _pool_state(state):
    return [state["table"], state["refs"]] + [x for layer in state["layers"] for x in layer]


def _own_run(state):
    from paper_2205_10350_b200 import binding
    case = state["case"]
    if case["op"] == "sample":
        filtered = torch.empty_like(state["scores"]) if case["filtered"] else None
        tokens, logp = binding.sample(state["scores"], state["r"], state["temperature"], state["top_k"], state["top_p"], state["min_p"], filtered=filtered)
        return [tokens, logp] + ([filtered] if filtered is not None else [])
    if case["op"] == "attend":
        return binding.cache_attention_shared(state["cache"], state["q"], state["off"], state["len"], state["groups"], state["shared"], max_new=case["new_hi"],
                                              max_keys=state["most"], max_shared=state["most_shared"], causal=case["causal"])
    pool, more = state["pool"], []
    binding.cache_fork(pool, state["parent"], state["keep"])
    if case["op"] == "turnover":
        more.append(binding.cache_compact(pool))
    if case["op"] != "fork":
        binding.cache_reserve(pool, state["off"], state["len"])
    return _pool_state(state) + more


def run(state):
    if own:
        return _own_run(state)
    op = state["case"]["op"]
    if op == "attend":
        return _plain_attend(state)
    if op == "sample":
        return _plain_sample(state)
    _plain_fork(state)
    more = [_plain_compact(state)] if op == "turnover" else []
    if op != "fork":
        _plain_reserve(state)
    return _pool_state(state) + more


# ------------------------------------------------------------------------------------------------------
# the operators' definitions, in 64 bits and on the host
# ------------------------------------------------------------------------------------------------------
def _exact_pool(state):
    """Row by row and block by block; contents of blocks have no other value than the one that is moved."""
    case = state["case"]
    bl = case["block"]
    rows = [[e for e in row if e >= 0] for row in state["table"].cpu().tolist()]
    width, n_blocks = state["table"].shape[1], state["refs"].numel()
    count = [0] * n_blocks
    rows = [list(rows[p][: _up(n, bl)]) if p >= 0 else [] for p, n in zip(state["parent"].tolist(), state["keep"].tolist())]
    for row in rows:
        for e in row:
            count[e] += 1
    more = []
    if case["op"] == "turnover":
        used = sum(1 for c in count if c)
        holes = iter([e for e in range(used) if not count[e]])
        to = {e: next(holes) for e in range(used, n_blocks) if count[e]}
        rows = [[to.get(e, e) for e in row] for row in rows]
        for e, h in to.items():
            count[h], count[e] = count[e], 0
        more = [torch.tensor([used], dtype=torch.int32)]
    if case["op"] != "fork":
        off, lens = state["off"].tolist(), state["len"].tolist()
        writers = {}
        for b, row in enumerate(rows):
            if off[b + 1] > off[b]:
                for i in range(lens[b] // bl, min(len(row), (lens[b] + off[b + 1] - off[b] - 1) // bl + 1)):
                    writers.setdefault(row[i], []).append((b, i))
        spare = iter([e for e in range(n_blocks) if not count[e]])
        before = list(count)
        for b, row in enumerate(rows):
            if off[b + 1] == off[b]:
                continue
            for i in range(lens[b] // bl, (lens[b] + off[b + 1] - off[b] - 1) // bl + 1):
                if i < len(row):
                    e = row[i]
                    if before[e] == 1 or (len(writers[e]) == before[e] and writers[e][0] == (b, i)):
                        continue
                    count[e] -= 1
                    row[i] = next(spare)
                else:
                    row.append(next(spare))
                count[row[i]] += 1
    table = torch.tensor([row + [-1] * (width - len(row)) for row in rows], dtype=torch.int32)
    return [table, torch.tensor(count, dtype=torch.int32)] + [None] * (4 * len(state["layers"])) + more


def _exact_attend(state):
    case = state["case"]
    samples, shared, new, tail = _attend_rows(case)
    per_kv = case["heads"] // case["kv_heads"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEV)
    off, lens = state["off"].tolist(), state["len"].tolist()
    for b in range(len(new)):
        hi = lens[b] + (new[b] if case["causal"] else 0)
        if not hi:
            continue
        k, v = (_row_values(state, c, b, 0, hi, torch.float64) for c in ("k", "v"))
        for j in range(case["heads"]):
            s = torch.einsum("id,td->it", state["q"][off[b]: off[b + 1], j].double(), k[j // per_kv]) / math.sqrt(case["dim"])
            if case["causal"]:
                s += torch.full_like(s, -math.inf).triu(lens[b] + 1)
            out[off[b]: off[b + 1], j] = torch.einsum("it,td->id", torch.exp(s - torch.logsumexp(s, 1, keepdim=True)), v[j // per_kv])
    return out


def _exact_sample(state):
    """Row by row: how many are in front of the first that goes, by a search in the sums."""
    case, scores = state["case"], state["scores"]
    at = lambda name, m, off: off if state[name] is None else float(state[name][m])
    tokens, logp, filtered = [], [], torch.full(scores.shape, -math.inf, dtype=torch.float64) if case["filtered"] else None
    for m in range(scores.shape[0]):
        x = scores[m].double().cpu().numpy()
        order = np.argsort(-x, kind="stable")
        w = np.exp((x[order] - x[order[0]]) / at("temperature", m, 1.0))
        n = len(w)
        if 0 < (k := int(at("top_k", m, 0))) < n:
            n = k
        if (p := at("top_p", m, 1.0)) < 1:
            c = np.cumsum(w[:n])
            n = max(1, min(n, 1 + int(np.searchsorted(c, p * c[-1], side="left"))))
        n = min(n, int(np.searchsorted(-w, -at("min_p", m, 0.0), side="right")))
        ids = np.sort(order[: max(n, 1)])
        c = np.cumsum(np.exp((x[ids] - x[order[0]]) / at("temperature", m, 1.0)))
        i = min(int(np.searchsorted(c, float(state["r"][m]) * c[-1], side="right")), len(ids) - 1)
        tokens.append(int(ids[i]))
        logp.append((x[ids[i]] - x[order[0]]) / at("temperature", m, 1.0) - math.log(c[-1]))
        if filtered is not None:
            filtered[m, ids] = torch.from_numpy(x[ids])
    return [torch.tensor(tokens, dtype=torch.int32), torch.tensor(logp, dtype=torch.float64)] + ([filtered] if filtered is not None else [])


def exact(case, seed):
    """What a pass returns, from the definitions."""
    if case["op"] == "attend":
        return None if work(case)["flops"] > 6e11 else _exact_attend(prepare(case, seed))
    return (_exact_sample if case["op"] == "sample" else _exact_pool)(prepare(case, seed))
