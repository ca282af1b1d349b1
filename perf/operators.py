"""Cases that the 8-bit key/value cache and the sampled verification are measured on.

One verification step writes the keys and values of a drafted block into the cache (`cache_append`), attends over it
(`cache_attention`), and decides which drafts stay, here from given random numbers (`accept_sampled`); `cache_read` brings cached tokens back
to FP32 or BF16.  A case is one such call over a ragged batch.  Head layouts, vocabularies and block lengths are those of the model shapes
and recipes in `paper_2205_10350_b200/synth.py` where the library's own models use them, and grouped heads of 128 with long prefixes for what
a user's decoder of another make brings along.

`run` computes the plain form from elementary torch operations, or, with `own`, makes the library's calls.
"""
from __future__ import annotations

import functools
import math

import torch

DEV = "cuda:0"
own = False

GOLDEN = 0.6180339887498949
TOP = {"e4m3": 448.0, "int8": 127.0}
TINY = 2.0 ** -126


def listed():
    return [
        # one token of one sentence: greedy decoding without drafts, launch and latency
        dict(name="append_b1_k1", op="append", batch=1, new_lo=1, new_hi=1, len_lo=57, len_hi=57, kv_heads=8, dim=64, block=32, fmt="e4m3",
             dtype="bf16", table=False),
        # blocks of drafted tokens of a batch of sentences, wide model
        dict(name="append_b32_k64", op="append", batch=32, new_lo=9, new_hi=64, len_lo=0, len_hi=400, kv_heads=16, dim=64, block=32, fmt="int8",
             dtype="bf16", table=True),
        # long prompts, written as the prefix of what is decoded next
        dict(name="append_prompts_b8", op="append", batch=8, new_lo=2500, new_hi=8190, len_lo=0, len_hi=70, kv_heads=8, dim=128, block=64,
             fmt="e4m3", dtype="bf16", table=True),
        # a sentence's prefix for a layer that runs in FP32
        dict(name="read_b1_n40", op="read", batch=1, new_lo=40, new_hi=40, len_lo=11, len_hi=11, kv_heads=8, dim=64, block=32, fmt="int8",
             dtype="fp32", table=False),
        # prefixes of a batch, read back whole
        dict(name="read_b8_long", op="read", batch=8, new_lo=2500, new_hi=8190, len_lo=0, len_hi=0, kv_heads=8, dim=128, block=64, fmt="e4m3",
             dtype="bf16", table=True),
        # grammatical error correction of one sentence: the whole source as a draft behind a short prefix
        dict(name="attend_b1_k40", op="attend", batch=1, new_lo=40, new_hi=40, len_lo=21, len_hi=21, heads=8, kv_heads=8, dim=64, block=32,
             fmt="e4m3", dtype="bf16", table=False, causal=True),
        # cross-attention of blocks of 25 over the encoder's keys of 400-token sources, FP32 activations
        dict(name="attend_source_b8_k25", op="attend", batch=8, new_lo=25, new_hi=25, len_lo=250, len_hi=400, heads=8, kv_heads=8, dim=64,
             block=32, fmt="int8", dtype="fp32", table=False, causal=False),
        # large blocks behind prefixes of the length of articles, wide model
        dict(name="attend_b32_k64", op="attend", batch=32, new_lo=17, new_hi=64, len_lo=200, len_hi=4000, heads=16, kv_heads=16, dim=64, block=32,
             fmt="int8", dtype="bf16", table=True, causal=True),
        # short drafts behind long prefixes, grouped heads
        dict(name="attend_b16_k8_long", op="attend", batch=16, new_lo=3, new_hi=8, len_lo=6000, len_hi=32000, heads=32, kv_heads=8, dim=128,
             block=64, fmt="e4m3", dtype="bf16", table=True, causal=True),
        # a single token behind one very long prefix
        dict(name="attend_b1_k1_long", op="attend", batch=1, new_lo=1, new_hi=1, len_lo=200001, len_hi=200001, heads=32, kv_heads=8, dim=128,
             block=64, fmt="int8", dtype="bf16", table=True, causal=True),
        # drafts copied from the source, one sentence: no drafter's distribution
        dict(name="accept_copied_b1_k25", op="accept", batch=1, new_lo=25, new_hi=25, vocab=32000, dtype="fp32", drafter=False, temperature=1.0),
        # drafts sampled from a drafter, a full batch of large blocks
        dict(name="accept_b32_k64", op="accept", batch=32, new_lo=40, new_hi=64, vocab=32000, dtype="bf16", drafter=True, temperature=0.8),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    op = rng.choice(["append", "read", "attend", "attend", "attend", "accept", "accept"])
    if op == "accept":
        new_hi = _log_int(rng, 1, 64)
        return dict(op=op, batch=_log_int(rng, 1, 32), new_lo=rng.randint(1, new_hi), new_hi=new_hi,
                    vocab=rng.choice([1000, 32000, 50265, _log_int(rng, 500, 60000)]), dtype=rng.choice(["fp32", "bf16"]),
                    drafter=rng.random() < 0.6, temperature=rng.choice([0.5, 0.8, 1.0, 1.3]))
    dim = rng.choice([32, 64, 64, 128])
    kv_heads = rng.choice([4, 8, 8, 16])
    case = dict(op=op, batch=_log_int(rng, 1, 32), kv_heads=kv_heads, dim=dim, block=rng.choice([16, 32, 64, 128]), fmt=rng.choice(["e4m3", "int8"]),
                dtype=rng.choice(["fp32", "bf16", "bf16"]), table=rng.random() < 0.6)
    if op == "attend":
        new_hi, len_hi = _log_int(rng, 1, 64), _log_int(rng, 1, 60000)
        case.update(heads=kv_heads * rng.choice([1, 1, 2, 4]), causal=rng.random() < 0.8)
    else:
        new_hi, len_hi = _log_int(rng, 1, 8190), _log_int(rng, 1, 500)
    case.update(new_lo=rng.randint(max(1, new_hi // 3), new_hi), new_hi=new_hi, len_lo=rng.randint(len_hi // 5, len_hi), len_hi=len_hi)
    return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


@functools.lru_cache(maxsize=None)
def _largest():
    return {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("append", "read", "attend", "accept")}


def draw(rng):
    while True:
        case = _draw_once(rng)
        if _cost(case) <= _largest()[case["op"]]:
            return case


# ------------------------------------------------------------------------------------------------------
# sizes of a case
# ------------------------------------------------------------------------------------------------------
def _spread(lo, hi, n, first):
    """n whole numbers between lo and hi, both ends among them where n > 1, the rest spread out."""
    if n == 1:
        return [hi]
    return [lo, hi][:n] + [lo + int((hi - lo) * ((first + (b + 1) * GOLDEN) % 1.0)) for b in range(n - 2)]


def _rows(case):
    """(new tokens, tokens in front of them) of every row."""
    new = _spread(case["new_lo"], case["new_hi"], case["batch"], 0.0)
    old = _spread(case["len_lo"], case["len_hi"], case["batch"], 0.37)[::-1] if "len_lo" in case else [0] * case["batch"]
    return new, old


def _element(case):
    return 4 if case["dtype"] == "fp32" else 2


def work(case):
    """Bytes: every input read once, every output written once.  Operations: a multiplication and an addition of each product; a handful of
    operations per element where there are no products."""
    new, old = _rows(case)
    M, t = sum(new), _element(case)
    if case["op"] == "accept":
        n = M * case["vocab"] * (2 if case["drafter"] else 1)
        return {"bytes": n * t + M * 12 + case["batch"] * 8, "flops": 4 * n}
    token = case["kv_heads"] * case["dim"] * 2                       # a token's keys and values
    if case["op"] == "append":
        live = sum(o % case["block"] for o in old)
        blocks = sum((o + n - 1) // case["block"] - o // case["block"] + 1 for n, o in zip(new, old))
        return {"bytes": M * token * (t + 1) + live * token + blocks * case["kv_heads"] * 8, "flops": 3 * M * token}
    if case["op"] == "read":
        return {"bytes": M * token * (t + 1), "flops": M * token}
    keys = sum(o + n if case["causal"] else o for n, o in zip(new, old))
    pairs = sum(n * o + (n * (n + 1) // 2 if case["causal"] else 0) for n, o in zip(new, old))
    return {"bytes": keys * token + 2 * M * case["heads"] * case["dim"] * t, "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------
def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _code_type(fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.int8


def _scale_for(amax, fmt):
    """The smallest power of two s with amax / s within the format (1 where there is nothing)."""
    m, e = torch.frexp(amax)
    bits, edge = (9, 0.875) if fmt == "e4m3" else (7, 127.0 / 128.0)
    s = torch.ldexp(torch.ones_like(m), (e - bits + (m > edge)).to(torch.float32))
    return torch.where(amax > 0, s.clamp_min(TINY), torch.ones_like(s))


def _encode(x, fmt):
    x = x.clamp(-TOP[fmt], TOP[fmt])
    return x.to(torch.float8_e4m3fn) if fmt == "e4m3" else x.round().to(torch.int8)


def _decode(codes, fmt):
    return codes.view(_code_type(fmt)).to(torch.float32)


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
        codes[b: b + n] = _encode(x, case["fmt"])
        scale[b: b + n] = s
    return codes, scale


def _prepare_cache(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    new, old = _rows(case)
    B, M, H, D, bl = case["batch"], sum(new), case["kv_heads"], case["dim"], case["block"]
    per_row = (max(o + n for n, o in zip(new, old)) + bl - 1) // bl
    if case["table"]:
        # blocks handed out in any order, each row as many as it needs; behind them nothing that may be looked at
        need = [(o + n + bl - 1) // bl for n, o in zip(new, old)]
        n_blocks = sum(need) + 3
        order = torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32)
        table = torch.full((B, per_row), -1, dtype=torch.int32, device=DEV)
        first = 0
        for b, n in enumerate(need):
            table[b, :n] = order[first: first + n]
            first += n
    else:
        n_blocks, table = B * per_row, None
    state = dict(case=case, off=_int([sum(new[:b]) for b in range(B + 1)]), len=_int(old), table=table, per_row=per_row, dtype=dt)
    state["k_codes"], state["k_scale"] = _filled(case, n_blocks, g)
    state["v_codes"], state["v_scale"] = _filled(case, n_blocks, g)
    if case["op"] == "append":
        # keys and values as a projection leaves them: next to each other, with the queries in front
        qkv = torch.randn((M, 3 * H * D), generator=g, device=DEV)
        qkv *= torch.exp(0.4 * torch.randn((M, 1), generator=g, device=DEV))
        qkv = qkv.to(dt)
        state["k"], state["v"] = qkv[:, H * D: 2 * H * D].view(M, H, D), qkv[:, 2 * H * D:].view(M, H, D)
    elif case["op"] == "attend":
        state["q"] = (torch.randn((M, case["heads"], D), generator=g, device=DEV) * 1.2).to(dt)
    if own:
        from paper_2205_10350_b200 import binding
        state["cache"] = binding.KvCache(n_blocks, H, D, bl, case["fmt"], table=table, row_blocks=per_row, device=DEV,
                                         tensors=(state["k_codes"], state["v_codes"], state["k_scale"], state["v_scale"]))
    return state


def _prepare_accept(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    new, _ = _rows(case)
    B, M, V, kmax = case["batch"], sum(new), case["vocab"], case["new_hi"]
    target = torch.randn((M, V), generator=g, device=DEV)
    target *= 2.0
    likely = torch.randint(4, V, (M, 3), generator=g, device=DEV)         # a few tokens hold most of a position's probability
    target.scatter_add_(1, likely, torch.tensor([[12.0, 10.0, 9.0]], device=DEV).expand(M, 3))
    draft = None
    if case["drafter"]:
        # a drafter that mostly agrees
        draft = torch.randn((M, V), generator=g, device=DEV)
        draft *= 0.6
        draft += target
        draft = draft.to(dt)
        drawn = torch.multinomial(torch.softmax(draft.float() / case["temperature"], 1), 1, generator=g)[:, 0]
    else:
        drawn = torch.where(torch.rand(M, generator=g, device=DEV) < 0.9, likely[:, 0], likely[:, 2])
    target = target.to(dt)
    drafts = torch.full((B, kmax), -1, dtype=torch.int32, device=DEV)
    off = 0
    for b, n in enumerate(new):
        drafts[b, :n] = drawn[off: off + n].to(torch.int32)
        if not case["drafter"]:
            drafts[b, n - 1] = -1                                       # a copied block ends in a slot that matches nothing
        off += n
    return dict(case=case, target=target, draft=draft, drafts=drafts, off=_int([sum(new[:b]) for b in range(B + 1)]),
                u=torch.rand((B, kmax), generator=g, device=DEV), r=torch.rand(B, generator=g, device=DEV))


def prepare(case, seed):
    return (_prepare_accept if case["op"] == "accept" else _prepare_cache)(case, seed)


# ------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------
def _blocks_of(state, b, first, last):
    """Ids of blocks first..last (inclusive) of row b."""
    if state["table"] is None:
        return torch.arange(b * state["per_row"] + first, b * state["per_row"] + last + 1, device=DEV)
    return state["table"][b, first: last + 1].long()


def _plain_append(state):
    case = state["case"]
    bl, fmt = case["block"], case["fmt"]
    new, old = _rows(case)
    at = 0
    for b, (n, o) in enumerate(zip(new, old)):
        ids = _blocks_of(state, b, o // bl, (o + n - 1) // bl)
        pos = torch.arange(o // bl * bl, (o // bl + len(ids)) * bl, device=DEV)
        live, fresh = pos < o, (pos >= o) & (pos < o + n)
        for name in ("k", "v"):
            codes, scale = state[name + "_codes"].view(torch.uint8), state[name + "_scale"]
            x = _decode(codes[ids], fmt) * scale[ids][:, :, None, None]     # [blocks, heads, block, dim]
            x = x.transpose(1, 2).flatten(0, 1)                              # [positions, heads, dim]
            x = torch.where(live[:, None, None], x, torch.zeros_like(x))
            x[fresh] = state[name][at: at + n].float()
            x = x.unflatten(0, (len(ids), bl)).transpose(1, 2)
            s = _scale_for(x.abs().amax((2, 3)), fmt)
            written = (live | fresh).view(len(ids), 1, bl, 1)
            codes[ids] = torch.where(written, _encode(x / s[:, :, None, None], fmt).view(torch.uint8), codes[ids])
            scale[ids] = s
        at += n
    return [state[n] for n in ("k_codes", "k_scale", "v_codes", "v_scale")]


def _row_values(state, name, b, lo, hi, wide=torch.float32):
    """Values of positions lo..hi-1 of row b, [tokens, heads, dim]."""
    bl = state["case"]["block"]
    ids = _blocks_of(state, b, lo // bl, (hi - 1) // bl)
    x = _decode(state[name + "_codes"].view(torch.uint8)[ids], state["case"]["fmt"]).to(wide) * state[name + "_scale"][ids].to(wide)[:, :, None, None]
    return x.transpose(1, 2).flatten(0, 1)[lo - lo // bl * bl: hi - lo // bl * bl]


def _plain_read(state):
    new, old = _rows(state["case"])
    return [torch.cat([_row_values(state, name, b, o, o + n).to(state["dtype"]) for b, (n, o) in enumerate(zip(new, old))]) for name in ("k", "v")]


def _plain_attend(state):
    case, q = state["case"], state["q"]
    new, old = _rows(case)
    out = torch.zeros_like(q)
    group = case["heads"] // case["kv_heads"]
    at = 0
    for b, (n, o) in enumerate(zip(new, old)):
        keys = o + n if case["causal"] else o
        if keys:
            k, v = (_row_values(state, name, b, 0, keys).transpose(0, 1) for name in ("k", "v"))        # [kv heads, keys, dim]
            qb = q[at: at + n].float().view(n, case["kv_heads"], group, case["dim"]).permute(1, 0, 2, 3).flatten(1, 2)
            s = qb @ k.transpose(1, 2) * case["dim"] ** -0.5                                        # [kv heads, n * group, keys]
            if case["causal"]:
                hidden = torch.arange(keys, device=DEV)[None, :] > o + torch.arange(n, device=DEV).repeat_interleave(group)[:, None]
                s = s.masked_fill(hidden, -math.inf)
            s = torch.exp(s - s.amax(2, keepdim=True))
            s = (s / s.sum(2, keepdim=True)) @ v
            out[at: at + n] = s.unflatten(1, (n, group)).permute(1, 0, 2, 3).flatten(1, 2).to(out.dtype)
        at += n
    return out


def _plain_accept(state):
    case = state["case"]
    new, _ = _rows(case)
    T, kmax, B = case["temperature"], case["new_hi"], case["batch"]
    tokens = torch.full((B, kmax), -1, dtype=torch.int32, device=DEV)
    count = torch.empty(B, dtype=torch.int32, device=DEV)
    place = torch.arange(kmax, device=DEV)
    at = 0
    for b, n in enumerate(new):
        # 64 bits: a random number next to a border of the distribution decides on a token
        d = state["drafts"][b, :n].long()
        there, d = d >= 0, d.clamp_min(0)[:, None]
        p = torch.softmax(state["target"][at: at + n].double() / T, 1)
        q = torch.softmax(state["draft"][at: at + n].double() / T, 1) if case["drafter"] else torch.zeros_like(p).scatter_(1, d, 1.0)
        stays = there & (state["u"][b, :n].double() * q.gather(1, d)[:, 0] < p.gather(1, d)[:, 0])
        first = torch.cummin(stays.int(), 0).values.sum()                  # drafts in front of the first that falls
        i = first.clamp_max(n - 1)
        left = torch.where(there[i], (p[i] - q[i]).clamp_min(0), p[i])
        total = torch.cumsum(left, 0)
        token = (total <= state["r"][b].double() * total[-1]).sum().clamp_max(case["vocab"] - 1)
        tokens[b] = torch.where(place < first, state["drafts"][b], torch.where((place == first) & (first < n), token.int(), tokens[b]))
        count[b] = torch.where(first < n, first + 1, first)
        at += n
    return tokens, count


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "accept": _plain_accept}[op](state)
    from paper_2205_10350_b200 import binding
    if op == "accept":
        return binding.accept_sampled(state["target"], state["draft"], state["drafts"], state["off"], state["u"], state["r"],
                                      temperature=case["temperature"])
    cache = state["cache"]
    if op == "append":
        binding.cache_append(cache, state["k"], state["v"], state["off"], state["len"], max_new=case["new_hi"])
        return [cache.k_codes, cache.k_scale, cache.v_codes, cache.v_scale]
    if op == "read":
        return binding.cache_read(cache, state["off"], state["len"], tokens=sum(_rows(case)[0]), max_tokens=case["new_hi"], dtype=state["dtype"])
    return binding.cache_attention(cache, state["q"], state["off"], state["len"], max_new=case["new_hi"],
                                   max_keys=case["len_hi"] + (case["new_hi"] if case["causal"] else 0), causal=case["causal"])


# ------------------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ------------------------------------------------------------------------------------------------------
def _exact_attend(state):
    case = state["case"]
    new, old = _rows(case)
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, o) in enumerate(zip(new, old)):
        keys = o + n if case["causal"] else o
        for h in range(case["kv_heads"] if keys else 0):
            bl = case["block"]
            ids = _blocks_of(state, b, 0, (keys - 1) // bl)
            k, v = ((_decode(state[c + "_codes"].view(torch.uint8)[ids, h], case["fmt"]).double() *
                     state[c + "_scale"][ids, h].double()[:, None, None]).reshape(-1, case["dim"])[:keys] for c in ("k", "v"))
            for j in range(h * group, (h + 1) * group):
                s = torch.einsum("id,td->it", state["q"][at: at + n, j].double(), k) / math.sqrt(case["dim"])
                if case["causal"]:
                    s += torch.full_like(s, -math.inf).triu(o + 1)
                out[at: at + n, j] = torch.einsum("it,td->id", torch.exp(s - torch.logsumexp(s, 1, keepdim=True)), v)
        at += n
    return out


def _nearest(x, fmt):
    """x in steps of the format: E4M3 has 3 bits behind the leading one, down to steps of 2^-9; ties to even."""
    if fmt == "int8":
        return torch.round(x)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(state):
    """Block by block: what the tokens in front stand for and the new ones, over the largest of them."""
    case = state["case"]
    bl, fmt = case["block"], case["fmt"]
    new, old = _rows(case)
    outs = []
    for name in ("k", "v"):
        codes, scale = state[name + "_codes"].float().double(), state[name + "_scale"].double()
        at = 0
        for b, (n, o) in enumerate(zip(new, old)):
            for i in range(o // bl, (o + n - 1) // bl + 1):
                block = int(_blocks_of(state, b, i, i))
                lo, hi = max(o - i * bl, 0), min(o + n - i * bl, bl)           # first new slot of the block, end of its tokens
                first = at + i * bl + lo - o
                x = torch.cat([codes[block, :, :lo] * scale[block, :, None, None],
                               state[name][first: first + hi - lo].double().transpose(0, 1)], 1)
                top = x.abs().amax((1, 2)) / TOP[fmt]
                exponent = torch.ceil(torch.log2(top)).clamp_min(-126)
                exponent -= (torch.exp2(exponent - 1) >= top).double()                     # (a logarithm may be rounded past a whole number)
                exponent += (torch.exp2(exponent) < top).double()
                s = torch.where(top > 0, torch.exp2(exponent.clamp_min(-126)), torch.ones_like(top))
                codes[block, :, :hi] = _nearest(x / s[:, None, None], fmt)
                scale[block] = s
            at += n
        outs += [codes, scale]
    return outs


def _exact_accept(state):
    """Position by position, on the host."""
    case = state["case"]
    new, _ = _rows(case)
    drafts, u, r = (state[n].cpu() for n in ("drafts", "u", "r"))
    tokens, counts, at = torch.full_like(drafts, -1), [], 0
    for b, n in enumerate(new):
        count = 0
        for i in range(n):
            d = int(drafts[b, i])
            p = torch.exp((z := state["target"][at + i].double() / case["temperature"]) - torch.logsumexp(z, 0))
            if case["drafter"]:
                q = torch.exp((z := state["draft"][at + i].double() / case["temperature"]) - torch.logsumexp(z, 0))
            else:
                q = torch.zeros_like(p)
                q[max(d, 0)] = 1.0
            count += 1
            if d >= 0 and float(u[b, i]) * float(q[d]) < float(p[d]):
                tokens[b, i] = d
                continue
            rest = torch.relu(p - q) if d >= 0 else p
            c = torch.cumsum(rest / rest.sum(), 0)
            tokens[b, i] = min(int(torch.searchsorted(c, float(r[b]), right=True)), case["vocab"] - 1)
            break
        counts.append(count)
        at += n
    return tokens, torch.tensor(counts, dtype=torch.int32)


def exact(case, seed):
    """What a pass returns, in 64 bits, from the definitions; codes of the cache and decided tokens as the whole steps they are."""
    if work(case)["flops"] > 3e12:
        return None
    state = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(state)
    if case["op"] == "accept":
        return _exact_accept(state)
    if case["op"] == "attend":
        return _exact_attend(state)
    new, old = _rows(case)
    return [torch.cat([_row_values(state, name, b, o, o + n, torch.float64) for b, (n, o) in enumerate(zip(new, old))]) for name in ("k", "v")]
