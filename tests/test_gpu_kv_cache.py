"""The 8-bit key/value cache against its definition in 64 bits: what is written, what is read back, and attention over it."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOP = {"e4m3": 448.0, "int8": 127.0}
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------
# the definition
# ---------------------------------------------------------------------------------------------------------
def scale_of(amax, fmt):
    """Smallest power of two that brings amax into the format, by trying them."""
    if amax == 0:
        return 1.0
    e = -126
    while amax > TOP[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def nearest(x, fmt):
    x = np.clip(x, -TOP[fmt], TOP[fmt])
    if fmt == "int8":
        return np.rint(x)
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)
    return np.rint(x / step) * step


class Model:
    """A cache in float64: codes as values, blocks found as the call finds them."""

    def __init__(self, n_blocks, heads, dim, block, fmt, table=None, row_blocks=None):
        self.block, self.fmt, self.table, self.row_blocks = block, fmt, table, row_blocks or n_blocks
        self.codes = [np.zeros((n_blocks, heads, block, dim)) for _ in range(2)]
        self.scale = [np.ones((n_blocks, heads)) for _ in range(2)]

    def block_id(self, b, i):
        return int(self.table[b, i]) if self.table is not None else b * self.row_blocks + i

    def append(self, k, v, off, lens):
        for z, x in enumerate((k, v)):
            for b, p in enumerate(lens):
                n = off[b + 1] - off[b]
                for i in range(p // self.block, (p + n - 1) // self.block + 1) if n else ():
                    g, lo, hi = self.block_id(b, i), max(p - i * self.block, 0), min(p + n - i * self.block, self.block)
                    first = off[b] + i * self.block + lo - p
                    for h in range(x.shape[1]):
                        vals = np.concatenate([self.codes[z][g, h, :lo] * self.scale[z][g, h], x[first: first + hi - lo, h]])
                        vals = np.where(np.isnan(vals), 0.0, vals)
                        finite = np.abs(vals[np.isfinite(vals)])
                        s = scale_of(finite.max() if finite.size else 0.0, self.fmt)
                        self.codes[z][g, h, :hi] = nearest(vals / s, self.fmt)
                        self.scale[z][g, h] = s

    def values(self, z, b, n):
        """First n positions of row b, [n, heads, dim]."""
        ids = [self.block_id(b, i) for i in range((n + self.block - 1) // self.block)]
        if not ids:
            return np.zeros((0,) + self.codes[z].shape[1:2] + self.codes[z].shape[3:])
        x = self.codes[z][ids] * self.scale[z][ids][:, :, None, None]
        return x.transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:n]

    def attend(self, q, off, lens, causal, scale):
        """(result, sum of |p v|, sum of |q k| at its largest, largest p * scale times the sum of |codes|) of every query and head."""
        out, weight, size, floor = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape)
        group = q.shape[1] // self.codes[0].shape[1]
        for b, p in enumerate(lens):
            n = off[b + 1] - off[b]
            k, v = (self.values(z, b, p + n if causal else p) for z in range(2))
            scales = np.repeat([self.scale[1][self.block_id(b, i)] for i in range((len(v) + self.block - 1) // self.block)], self.block, 0)[: len(v)]
            for i in range(n):
                keys = p + i + 1 if causal else p
                if not keys:
                    continue
                for h in range(q.shape[1]):
                    kk, vv, qq = k[:keys, h // group], v[:keys, h // group], q[off[b] + i, h]
                    s = kk @ qq * scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[off[b] + i, h], weight[off[b] + i, h] = w @ vv, w @ np.abs(vv)
                    size[off[b] + i, h] = (np.abs(kk) @ np.abs(qq)).max() * scale
                    sv = scales[:keys, h // group]
                    floor[off[b] + i, h] = (w * sv).max() * (np.abs(vv) / sv[:, None]).sum(0)
        return out, weight, size, floor


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def offsets(new):
    return [int(x) for x in np.concatenate([[0], np.cumsum(new)])]


def both(n_blocks, heads, dim, block, fmt, table=None, row_blocks=None):
    t = None if table is None else ints(table)
    return (binding.KvCache(n_blocks, heads, dim, block, fmt, table=t, row_blocks=row_blocks, device=DEV),
            Model(n_blocks, heads, dim, block, fmt, table, row_blocks))


def same(cache, model):
    for codes, scale, want, want_scale in ((cache.k_codes, cache.k_scale, model.codes[0], model.scale[0]),
                                           (cache.v_codes, cache.v_scale, model.codes[1], model.scale[1])):
        assert np.array_equal(scale.cpu().numpy(), want_scale)
        assert np.array_equal(codes.float().cpu().numpy(), want)


def numbers(shape, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(spread * torch.randn((shape[0],) + (1,) * (len(shape) - 1), generator=g))
    return x.to(TORCH[dtype])


def shuffled(rows, row_blocks, seed, spare=3):
    r = np.random.default_rng(seed)
    n = rows * row_blocks + spare
    return r.permutation(n)[: rows * row_blocks].reshape(rows, row_blocks).astype(np.int32), n


# ---------------------------------------------------------------------------------------------------------
# writing and reading
# ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,dim,block", [(1, 32, 16), (2, 64, 32), (3, 128, 64), (2, 128, 128), (5, 32, 128), (1, 64, 16)])
def test_written_blocks_hold_what_the_definition_says(fmt, dtype, heads, dim, block):
    """Several calls, rows of all lengths (none, one token, more than a block), blocks in any order, keys and values inside a wider array."""
    B, row_blocks = 4, 5
    table, n_blocks = shuffled(B, row_blocks, block + dim)
    cache, model = both(n_blocks, heads, dim, block, fmt, table, row_blocks)
    lens = [0, block - 1, 3, 2 * block]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    # what lies in front: written by the call itself
    for step, new in enumerate((lens, [1, 1, 1, 1], [block + 3, 0, 2, block], [0, 2 * block - 2, block + 1, 1])):
        M, off, at = sum(new), offsets(new), [0] * B if step == 0 else lens
        wide = numbers((M, 3 * heads * dim + 16), dtype, 7 * step + dim)
        d = wide.to(DEV)
        k, v = d[:, 8: 8 + heads * dim].view(M, heads, dim), d[:, 16 + heads * dim: 16 + 2 * heads * dim].view(M, heads, dim)
        binding.cache_append(cache, k, v, ints(off), ints(at), max_new=max(new), status_t=status)
        model.append(k.cpu().double().numpy(), v.cpu().double().numpy(), off, at)
        same(cache, model)
        if step:
            lens = [p + n for p, n in zip(lens, new)]
    assert int(status.item()) == 0
    # read back: a code times a power of two has no more than 8 bits, so neither type rounds
    start = [min(2, n) for n in lens]
    count = [n - s for n, s in zip(lens, start)]
    off = offsets(count)
    for dt in (torch.float32, torch.bfloat16):
        got = binding.cache_read(cache, ints(off), ints(start), tokens=sum(count), max_tokens=max(count), dtype=dt, status_t=status)
        for z in range(2):
            want = np.concatenate([model.values(z, b, lens[b])[start[b]:] for b in range(B)])
            assert got[z].dtype is dt and np.array_equal(got[z].double().cpu().numpy(), want)
    assert int(status.item()) == 0


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_drafts_that_were_given_up_leave_no_trace(fmt):
    """Ten tokens, then a block with a far larger one that is rolled back, then others: E4M3 as if it had never been there (its live codes only
    move by binary places, none here down to the subnormals), INT8 within a step of the larger scale."""
    k, v = numbers((10, 2, 64), "bf16", 1, 0.0).abs() + 0.25, numbers((10, 2, 64), "bf16", 2, 0.0).abs() + 0.25
    big, more = numbers((4, 2, 64), "bf16", 3, 0.0) * 4, numbers((3, 2, 64), "bf16", 4, 0.0)
    cache, _ = both(1, 2, 64, 32, fmt)
    other, _ = both(1, 2, 64, 32, fmt)
    for c, drafts in ((cache, True), (other, False)):
        binding.cache_append(c, k.to(DEV), v.to(DEV), ints([0, 10]), ints([0]), max_new=10)
        if drafts:
            binding.cache_append(c, big.to(DEV), big.to(DEV), ints([0, 4]), ints([10]), max_new=4)
            binding.cache_append(c, big[:1].to(DEV), big[:1].to(DEV), ints([0, 1]), ints([10]), max_new=1)
        binding.cache_append(c, more.to(DEV), more.to(DEV), ints([0, 3]), ints([10]), max_new=4)
    a, b = ([x.float() for x in binding.cache_read(c, ints([0, 13]), ints([0]), 13, 13, torch.float32)] for c in (cache, other))
    for z, (x, y) in enumerate(zip(a, b)):
        if fmt == "e4m3":
            assert torch.equal(x, y) and torch.equal((cache.k_scale, cache.v_scale)[z], (other.k_scale, other.v_scale)[z])
        else:
            largest = scale_of(float(big.abs().max()), fmt)
            assert float((x[:10] - y[:10]).abs().max()) <= largest


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_numbers_at_the_ends_of_their_types(fmt, dtype):
    """Zeros, subnormals, the largest numbers, ties between codes, numbers at the border of a scale; infinities take the largest code, a NaN none."""
    block, heads, dim = 16, 8, 32
    tiny, huge = (2.0 ** -149, 3.4e38) if dtype == "fp32" else (2.0 ** -133, 3.38e38)
    x = np.zeros((block, heads, dim), np.float32)
    x[:, 1] = tiny
    x[3, 2], x[4, 2, 5] = huge, -huge
    x[:, 3, 0] = np.arange(block) + 0.5                      # ties of INT8
    x[0, 3, 1] = 127.0
    x[:, 4, 0], x[0, 4, 1] = 16 + np.arange(block) + 0.0, 448.0     # ties of E4M3 (steps of 2 from 16 on)
    x[0, 5, 0], x[0, 6, 0] = TOP[fmt] * 8, np.nextafter(np.float32(TOP[fmt] * 8), np.float32(1e9)) if dtype == "fp32" else TOP[fmt] * 8 * (1 + 2.0 ** -7)
    x[1, 7, 0], x[2, 7, 1], x[3, 7, 2], x[4, 7, 3] = np.inf, -np.inf, np.nan, 5.0
    t = torch.tensor(x).to(TORCH[dtype])
    cache, model = both(2, heads, dim, block, fmt)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    clean = t.clone()
    clean[3, 7, 2] = 0
    binding.cache_append(cache, clean.to(DEV), clean.to(DEV), ints([0, block]), ints([0]), max_new=block, status_t=status)
    assert int(status.item()) == 0                           # infinities are no error
    model.append(clean.double().numpy(), clean.double().numpy(), [0, block], [0])
    same(cache, model)
    binding.cache_append(cache, t.to(DEV), t.to(DEV), ints([0, block]), ints([0]), max_new=block, status_t=status)
    assert int(status.item()) == binding.AD_ERR_ARG
    same(cache, model)
    assert float(cache.k_codes.float()[0, 7, 1, 0]) == TOP[fmt] and float(cache.v_codes.float()[0, 7, 2, 1]) == -TOP[fmt]


def test_slots_behind_the_last_token_stay_as_they_were():
    table, n_blocks = shuffled(2, 3, 5)
    cache, _ = both(n_blocks, 2, 64, 32, "int8", table, 3)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(77)
    new = [5, 33]
    x = numbers((38, 2, 64), "fp32", 3).to(DEV)
    binding.cache_append(cache, x, x, ints(offsets(new)), ints([3, 0]), max_new=33)
    used = torch.zeros((n_blocks, 32), dtype=torch.bool)
    used[table[0, 0], :8] = True                             # (the three in front are re-coded)
    used[table[1, 0], :32] = True
    used[table[1, 1], :1] = True
    for t in (cache.k_codes, cache.v_codes):
        assert bool((t.cpu().permute(0, 2, 1, 3)[~used] == 77).all())
        assert not bool((t.cpu().permute(0, 2, 1, 3)[used] == 77).all())


@pytest.mark.parametrize("what,code", [("table", binding.AD_ERR_ARG), ("capacity", binding.AD_ERR_CAPACITY), ("long", binding.AD_ERR_ARG), ("offset", binding.AD_ERR_ARG)])
def test_rows_that_cannot_be_done_are_latched_and_the_others_done(what, code):
    """What the device alone can see: a block that does not exist, a row beyond its capacity, more tokens than announced, offsets beyond the batch."""
    table = np.array([[0, 1], [2, 3], [4, 5]], np.int32)
    new, lens, max_new = [4, 4, 4], [10, 30, 0], 4
    off = offsets(new)
    if what == "table":
        table[1, 1] = 6                                       # row 1's tokens lie in its blocks 0 and 1
    elif what == "capacity":
        lens[1] = 61
    elif what == "long":
        off, max_new = [0, 4, 9, 12], 4
    else:
        off = [0, 4, 4, 13]
    cache, model = both(6, 2, 64, 32, "e4m3", table, 2)
    x = numbers((12, 2, 64), "bf16", 9).to(DEV)
    out = torch.full((12, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    for call in ("append", "read", "attend"):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        if call == "append":
            binding.cache_append(cache, x, x, ints(off), ints(lens), max_new=max_new, status_t=status)
        elif call == "read":
            k, _ = binding.cache_read(cache, ints(off), ints(lens), tokens=12, max_tokens=max_new, status_t=status)
        else:
            binding.cache_attention(cache, x, ints(off), ints(lens), max_new=max_new, max_keys=64, out=out, status_t=status)
        assert int(status.item()) == code, call
    good = {"table": [0, 2], "capacity": [0, 2], "long": [0, 2], "offset": [0]}[what]
    xs = x.cpu().double().numpy()
    for b in good:
        n = off[b + 1] - off[b]
        row = Model(6, 2, 64, 32, "e4m3", table, 2)
        at = [0] * (b + 1) + [n] * (3 - b)
        row.append(xs[off[b]: off[b + 1]], xs[off[b]: off[b + 1]], at, lens)
        got = binding.cache_read(cache, ints(at), ints(lens), tokens=n, max_tokens=max_new)[0].double().cpu().numpy()
        assert np.array_equal(got, row.values(0, b, lens[b] + n)[lens[b]:])
    if what in ("capacity", "long"):
        assert bool((out[off[1]: off[2]] == 7.0).all())       # the row's queries have no result


# ---------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------
def bound(dtype, want, weight, size, floor, keys, dim):
    """How far a result may be off.  A score: dim products and their sum, the scales and the query's 22 bits (2^-24 and 2^-22 of sum |q k|, as
    exponents); an exponential 2^-21; sums over keys 2^-24 each addition; both numerator and denominator.  BF16 besides: probabilities of 11 bits,
    and the result's own half step.  A probability times its block's scale goes into the product as an FP16 number that is 2^6
    to 2^15 for the largest so far in the row (whose reference is a whole exponent, up to 9 above it); FP16's steps are 2^-24 at the least, so one that
    is too small for 11 bits is off by at most 2^-25 there, 2^-31 of the largest, times its code."""
    e = (dim + 8) * 2.0 ** -24 + 2.0 ** -22
    rel = 2 * (e * size[..., None] + 2.0 ** -21 + keys * 2.0 ** -24) + 2.0 ** -22
    tol = rel * weight + 2.0 ** -31 * floor + 1e-37
    if dtype == "bf16":
        tol = (rel + 2.0 ** -11) * weight + 2.0 ** -31 * floor + 2.0 ** -8 * np.abs(want) * 1.01 + 1e-37
    return tol


def attend_and_check(cache, model, q, new, lens, causal, dtype, max_keys=None, scale=None):
    off = offsets(new)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    longest = max((p + n if causal else p) for p, n in zip(lens, new))
    got = binding.cache_attention(cache, q, ints(off), ints(lens), max_new=max(new), max_keys=longest if max_keys is None else max_keys, causal=causal,
                                  scale=scale, status_t=status)
    assert int(status.item()) == 0
    want, weight, size, floor = model.attend(q.cpu().double().numpy(), off, lens, causal, q.shape[2] ** -0.5 if scale is None else scale)
    err = np.abs(got.double().cpu().numpy() - want)
    tol = bound(dtype, want, weight, size, floor, longest, q.shape[2])
    assert got.dtype is q.dtype and (err <= tol).all(), (float(err.max()), float((err / tol).max()))
    return got


def filled(new_tokens, heads, dim, block, fmt, dtype, seed, row_blocks=None):
    """Cache and model that hold new_tokens[b] tokens of row b, blocks in any order."""
    B = len(new_tokens)
    rb = row_blocks or max(1, (max(new_tokens) + block - 1) // block)
    table, n_blocks = shuffled(B, rb, seed)
    cache, model = both(n_blocks, heads, dim, block, fmt, table, rb)
    # slots that hold no token: whatever is there, a NaN (E4M3) among it, must not be looked at
    for t in (cache.k_codes, cache.v_codes):
        t.view(torch.uint8).fill_(0x7F)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(float("nan"))
    M = sum(new_tokens)
    if M:
        k, v = numbers((M, heads, dim), dtype, seed, 0.5), numbers((M, heads, dim), dtype, seed + 1, 0.5)
        binding.cache_append(cache, k.to(DEV), v.to(DEV), ints(offsets(new_tokens)), ints([0] * B), max_new=max(new_tokens))
        model.append(k.double().numpy(), v.double().numpy(), offsets(new_tokens), [0] * B)
    return cache, model


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 1, 32, 16), (2, 1, 64, 32), (1, 4, 128, 64), (2, 2, 64, 128), (1, 8, 64, 16), (3, 3, 32, 128), (2, 1, 128, 16)])
def test_blocks_of_queries_over_ragged_rows(fmt, dtype, heads, group, dim, block):
    """Rows without a prefix, with one of a single token, at block borders and beyond; blocks of one query and of many; rows without queries."""
    new = [1, 7, 0, 33, 2, 1, 20, 64]
    lens = [0, 1, 9, block - 1, 2 * block, 3 * block + 5, 129, 70]
    total = [p + n for p, n in zip(lens, new)]
    cache, model = filled(total, heads, dim, block, fmt, dtype, dim + block)
    q = numbers((sum(new), heads * group, dim), dtype, 5, 0.3).to(DEV)
    attend_and_check(cache, model, q, new, lens, True, dtype)
    attend_and_check(cache, model, q, new, lens, False, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lens", [[0, 1, 2, 15], [16, 17, 31, 32], [33, 63, 64, 65], [127, 128, 129, 255], [256, 257, 511, 513], [1023, 1024, 1500, 2047]])
def test_single_queries_over_every_kind_of_length(dtype, lens):
    """One query a row, encoder keys: a row of none gives zeros."""
    for fmt, heads, group, dim, block in (("e4m3", 2, 1, 64, 32), ("int8", 1, 4, 128, 64)):
        cache, model = filled(lens, heads, dim, block, fmt, dtype, lens[1])
        q = numbers((4, heads * group, dim), dtype, 3, 0.3).to(DEV)
        got = attend_and_check(cache, model, q, [1] * 4, lens, False, dtype)
        if lens[0] == 0:
            assert bool((got[0] == 0).all())
        new = [1 if n else 0 for n in lens]
        attend_and_check(cache, model, q[: sum(new)], new, [max(n - 1, 0) for n in lens], True, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("max_keys", [0, 1, 300, 100000])
def test_the_announced_length_only_plans(dtype, max_keys):
    lens, new = [290, 3, 0, 120], [5, 40, 9, 1]
    cache, model = filled([p + n for p, n in zip(lens, new)], 2, 64, 32, "e4m3", dtype, 8)
    q = numbers((sum(new), 4, 64), dtype, 6, 0.3).to(DEV)
    attend_and_check(cache, model, q, new, lens, True, dtype, max_keys=max_keys)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_scales_far_apart(dtype, fmt):
    """Blocks whose keys and values differ by factors of up to 2^20 either way, scores that leave one key, and scores that are all alike."""
    block, n = 16, 16 * 9 + 3
    cache, model = both(10, 1, 64, block, fmt)
    g = np.random.default_rng(2)
    k, v = (torch.tensor(g.standard_normal((n, 1, 64)), dtype=torch.float32) for _ in range(2))
    for i, e in enumerate([0, 20, -20, 3, -7, 12, 0, -14, 6, 1]):
        v[i * block: (i + 1) * block] *= 2.0 ** e
        k[i * block: (i + 1) * block] *= 2.0 ** (-abs(e) / 4)
    k, v = (x.to(TORCH[dtype]) for x in (k, v))
    binding.cache_append(cache, k.to(DEV), v.to(DEV), ints([0, n]), ints([0]), max_new=n)
    model.append(k.double().numpy(), v.double().numpy(), [0, n], [0])
    for factor in (0.0, 1e-20, 0.2, 3.0, 60.0, 1e15):
        q = (torch.tensor(g.standard_normal((4, 1, 64)), dtype=torch.float32) * factor).to(TORCH[dtype]).to(DEV)
        if factor < 1e10:
            attend_and_check(cache, model, q, [4], [n - 4], True, dtype)
        else:                                                # one key has all of it
            got = binding.cache_attention(cache, q, ints([0, 4]), ints([n]), 4, n, causal=False).double().cpu().numpy()
            kk, vv = model.values(0, 0, n)[:, 0], model.values(1, 0, n)[:, 0]
            best = (q.cpu().double().numpy()[:, 0] @ kk.T).argmax(1)
            assert (np.abs(got[:, 0] - vv[best]) <= 2.0 ** -8 * np.abs(vv[best])).all()


def test_queries_that_are_not_finite_spoil_no_other():
    cache, model = filled([100], 2, 64, 32, "e4m3", "bf16", 4)
    q = numbers((9, 2, 64), "bf16", 6, 0.3).to(DEV)
    clean = binding.cache_attention(cache, q, ints([0, 9]), ints([91]), 9, 100)
    q[4, 1, 7], q[6, 0, 0] = float("nan"), float("inf")
    got = binding.cache_attention(cache, q, ints([0, 9]), ints([91]), 9, 100)
    spoiled = torch.zeros((9, 2), dtype=torch.bool, device=DEV)
    spoiled[4, 1] = spoiled[6, 0] = True
    assert torch.equal(got[~spoiled], clean[~spoiled])
    assert bool(torch.isnan(got[4, 1]).all()) and not bool(torch.isfinite(got[6, 0]).any())


def test_queries_inside_a_wider_array_and_results_of_other_rows():
    """Queries next to keys and values, a result whose rows behind the last sequence stay as they were, in any order of calls."""
    lens, new = [37, 64], [3, 5]
    cache, model = filled([p + n for p, n in zip(lens, new)], 2, 64, 32, "int8", "bf16", 4)
    wide = numbers((12, 3 * 256), "bf16", 6, 0.3).to(DEV)
    q = wide[:, 256: 512].view(12, 4, 64)
    out = torch.full((12, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    binding.cache_attention(cache, q, ints([0, 3, 8]), ints(lens), 5, 69, out=out)
    want = attend_and_check(cache, model, q[:8].contiguous(), new, lens, True, "bf16")
    assert torch.equal(out[:8], want) and bool((out[8:] == 9.0).all())
    again = binding.cache_attention(cache, q, ints([0, 3, 8]), ints(lens), 5, 69)
    assert torch.equal(again[:8], want)                       # nothing depends on the order in which CTAs run


def test_addresses_beyond_32_bits():
    """A cache of more than 2^31 bytes of keys: its last blocks."""
    heads, dim, block = 8, 128, 64
    n_blocks = (1 << 31) // (heads * dim * block) + 40
    table = np.array([[n_blocks - 1, n_blocks - 2, n_blocks - 3]], np.int32)
    cache = binding.KvCache(n_blocks, heads, dim, block, "int8", table=ints(table), device=DEV)
    small = Model(3, heads, dim, block, "int8", np.array([[2, 1, 0]]), 3)
    k, v = numbers((150, heads, dim), "bf16", 1), numbers((150, heads, dim), "bf16", 2)
    binding.cache_append(cache, k.to(DEV), v.to(DEV), ints([0, 150]), ints([0]), max_new=150)
    small.append(k.double().numpy(), v.double().numpy(), [0, 150], [0])
    got = binding.cache_read(cache, ints([0, 150]), ints([0]), 150, 150, torch.float32)
    assert np.array_equal(got[1].double().cpu().numpy(), small.values(1, 0, 150))
    assert not bool(cache.k_codes[: n_blocks - 3].view(torch.uint8).any())
    q = numbers((3, heads, dim), "bf16", 3, 0.3).to(DEV)
    attend_and_check(cache, small, q, [3], [147], True, "bf16")


@pytest.mark.parametrize("dtype,heads,group,dim,block", [("bf16", 2, 1, 64, 32), ("bf16", 1, 4, 128, 16), ("fp32", 1, 2, 32, 64)])
def test_more_rows_than_a_thread_block(dtype, heads, group, dim, block):
    """200 rows, most of them short or without queries, a few long ones whose keys are shared out over many CTAs."""
    g = np.random.default_rng(dim)
    new = [int(x) for x in g.integers(0, 4, 200)]
    lens = [int(x) for x in g.integers(0, 40, 200)]
    for b, n in ((0, 900), (57, 1500), (130, 2900), (199, 700)):
        lens[b], new[b] = n, 3
    cache, model = filled([p + n for p, n in zip(lens, new)], heads, dim, block, "int8", dtype, 8)
    q = numbers((sum(new), heads * group, dim), dtype, 6, 0.3).to(DEV)
    attend_and_check(cache, model, q, new, lens, True, dtype)
    attend_and_check(cache, model, q, new, lens, False, dtype)


def test_batches_without_any_query():
    cache, _ = filled([40, 70], 2, 64, 32, "e4m3", "bf16", 4)
    q = numbers((3, 2, 64), "bf16", 6, 0.3).to(DEV)
    out = torch.full((3, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for max_keys in (70, 4000):                              # (with and without a second kernel that joins parts)
        binding.cache_attention(cache, q, ints([1, 1, 1]), ints([40, 70]), 3, max_keys, causal=False, out=out, status_t=status)
        binding.cache_append(cache, q, q, ints([3, 3, 3]), ints([40, 70]), 3, status_t=status)
    assert bool((out == 9.0).all()) and int(status.item()) == 0


def test_calls_on_another_stream_and_in_a_graph():
    """The current stream is the one that counts; a captured step reads lengths that change between replays."""
    lens, heads, dim = [40, 70], 2, 64
    cache, model = filled(lens, heads, dim, 32, "e4m3", "bf16", 4, row_blocks=5)
    off, ln = ints([0, 2, 4]), ints(lens)
    x = numbers((4, 3, heads, dim), "bf16", 8, 0.3)
    d = x.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []

    def step():
        binding.cache_append(cache, d[:, 1], d[:, 2], off, ln, max_new=2)
        return binding.cache_attention(cache, d[:, 0], off, ln, max_new=2, max_keys=160)

    with torch.cuda.stream(side):
        outs.append(step().clone())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step()
    xs = x.double().numpy()
    for rep in range(3):
        if rep:
            ln += 2
            graph.replay()
            outs.append(res.clone())
        model.append(xs[:, 1], xs[:, 2], [0, 2, 4], [p + 2 * rep for p in lens])
        want, weight, size, floor = model.attend(xs[:, 0], [0, 2, 4], [p + 2 * rep for p in lens], True, dim ** -0.5)
        torch.cuda.synchronize()
        err = np.abs(outs[rep].double().cpu().numpy() - want)
        assert (err <= bound("bf16", want, weight, size, floor, 160, dim)).all()


def test_calls_that_are_refused():
    cache, _ = both(4, 2, 64, 32, "e4m3")
    x = numbers((4, 2, 64), "bf16", 1).to(DEV)
    off, ln = ints([0, 4]), ints([0])
    bad = [lambda: binding.cache_append(cache, x.half(), x.half(), off, ln, 4), lambda: binding.cache_append(cache, x, x.float(), off, ln, 4),
           lambda: binding.cache_append(cache, x[:, :1], x[:, :1], off, ln, 4), lambda: binding.cache_append(cache, x.cpu(), x.cpu(), off, ln, 4),
           lambda: binding.cache_append(cache, x, x, off.long(), ln, 4), lambda: binding.cache_append(cache, x, x, off[:1], ln, 4),
           lambda: binding.cache_append(cache, x, x, off, ln, 0), lambda: binding.cache_append(cache, x.transpose(1, 2), x.transpose(1, 2), off, ln, 4),
           lambda: binding.cache_append(cache, x, x, off.cpu(), ln, 4), lambda: binding.cache_append(cache, x, x, off, ln, 4, status_t=off),
           lambda: binding.cache_read(cache, off, ln, 4, 4, torch.float16), lambda: binding.cache_attention(cache, x[0], off, ln, 4, 4),
           lambda: binding.cache_attention(cache, x[:, :, :32], off, ln, 4, 4), lambda: binding.cache_attention(cache, x, off, ln, 4, -1),
           lambda: binding.cache_attention(cache, x, off, ln, 4, 4, scale=0.0), lambda: binding.cache_attention(cache, x, off, ln, 4, 4, out=x.float()),
           lambda: binding.cache_attention(cache, x[:, 0:1].expand(4, 4, 64), off, ln, 4, 4),
           lambda: binding.KvCache(4, 2, 64, 32, "e4m3", device=DEV, tensors=(cache.k_codes, cache.v_codes.view(torch.int8), cache.k_scale, cache.v_scale)),
           lambda: binding.KvCache(4, 2, 64, 32, "e4m3", device=DEV, table=torch.zeros((2, 2), device=DEV))]
    for call in bad:
        with pytest.raises(binding.AdError):
            call()
    # queries whose heads the cache's do not divide
    with pytest.raises(binding.AdError, match="multiple"):
        binding.cache_attention(cache, numbers((4, 3, 64), "bf16", 1).to(DEV), off, ln, 4, 4)


# ---------------------------------------------------------------------------------------------------------
# ends of the range
# ---------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("q_bits,k_bits,scale", [(0, 0, 1e30), (20, 0, 1e30), (60, -70, 1e30), (100, -100, 1e20), (120, 0, 0.125), (126, -120, 1e30), (-100, 80, 1e30), (-90, 110, 1.0)])
def test_scores_are_finite_wherever_their_factors_lie(fmt, dtype, dim, q_bits, k_bits, scale):
    """Scale, queries and keys at the ends of their ranges, scores inside of FP32's and far apart: each query gets its best key's value."""
    n = 40
    g = torch.Generator().manual_seed(dim)
    k, v = torch.randn((n, 1, dim), generator=g), torch.randn((n, 1, dim), generator=g)
    q = torch.randn((5, 1, dim), generator=g)
    q /= q.abs().amax(2, keepdim=True)
    k, q, v = ((x * 2.0 ** e).to(TORCH[dtype]) for x, e in ((k, k_bits), (q, q_bits), (v, 0)))
    cache, model = both(2, 1, dim, 32, fmt)
    binding.cache_append(cache, k.to(DEV), v.to(DEV), ints([0, n]), ints([0]), max_new=n)
    model.append(k.double().numpy(), v.double().numpy(), [0, n], [0])
    got = binding.cache_attention(cache, q.to(DEV), ints([0, 5]), ints([n]), 5, n, causal=False, scale=scale).double().cpu().numpy()[:, 0]
    kk, vv = model.values(0, 0, n)[:, 0], model.values(1, 0, n)[:, 0]
    scores = q.double().numpy()[:, 0] @ kk.T * float(np.float32(scale))
    assert np.abs(scores).max() < 2.0 ** 125
    rest = np.sort(scores, 1)
    assert (rest[:, -1] - rest[:, -2]).min() > 200            # (one key has all of it)
    assert (np.abs(got - vv[scores.argmax(1)]) <= 2.0 ** -8 * np.abs(vv[scores.argmax(1)])).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_live_codes_that_stand_for_more_than_fp32_holds(dtype, fmt):
    """The type's largest numbers round up to 2^128.  Tokens that come to them later leave them what they are."""
    block, heads, dim = 16, 2, 32
    cache, model = both(1, heads, dim, block, fmt)
    x = numbers((3, heads, dim), dtype, 5)
    x[0, 0, 3], x[0, 1, 4] = torch.finfo(TORCH[dtype]).max, torch.finfo(TORCH[dtype]).min
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for p in range(3):
        binding.cache_append(cache, x[p: p + 1].to(DEV), x[p: p + 1].to(DEV), ints([0, 1]), ints([p]), max_new=1, status_t=status)
        model.append(x[p: p + 1].double().numpy(), x[p: p + 1].double().numpy(), [0, 1], [p])
        same(cache, model)
    assert int(status.item()) == 0


def close_bound(dtype, want, weight, size, floor, keys, dim):
    """`bound` with the end to what small probabilities lose that the header gives: the product's steps are 2^-24, a largest operand is at least 2^12
    with BF16 queries, and 2^14 with FP32 ones, whose second number has steps of 2^-35: half of that over it, times the codes."""
    return bound(dtype, want, weight, size, 0.0 * floor, keys, dim) + (2.0 ** -37 if dtype == "bf16" else 2.0 ** -50) * floor


def leading_key(dtype, fmt, lead, n, heads, dim, block, value, seed):
    """A cache whose first key leads all others by about `lead` nats for every query, and whose value is `value` times the others'."""
    cache, model = both((n + block - 1) // block, heads, dim, block, fmt)
    k, v, q = numbers((n, heads, dim), dtype, seed, 0.0), numbers((n, heads, dim), dtype, seed + 1, 0.0), numbers((6, heads, dim), dtype, seed + 2, 0.0)
    k[:, :, 0], q[:, :, 0] = 0, 4.0
    k[0] = 0
    others = (torch.einsum("qhd,khd->qhk", q.double(), k.double()) * dim ** -0.5).amax((0, 1, 2)).item()
    k[0, :, 0] = (others + lead) * dim ** 0.5 / 4
    v[0] *= value
    binding.cache_append(cache, k.to(DEV), v.to(DEV), ints([0, n]), ints([0]), max_new=n)
    model.append(k.double().numpy(), v.double().numpy(), [0, n], [0])
    return cache, model, q


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("n,heads,dim,block", [(30, 1, 64, 32), (90, 2, 128, 16), (2000, 2, 64, 64), (2000, 1, 32, 16), (2000, 1, 128, 128)])
@pytest.mark.parametrize("lead", [10, 12, 14, 16, 18, 20])
def test_keys_that_another_one_outweighs(dtype, fmt, n, heads, dim, block, lead):
    """A first key that leads by many nats and has a value of zero or next to it, as a decoder's first token often does: what the others say is all there is to the result, and
    is as exact as it is for keys that lead."""
    for value in (0.0, 1e-3):
        cache, model, q = leading_key(dtype, fmt, lead, n, heads, dim, block, value, lead + dim)
        for causal in (False, True):
            off, lens = [0, 6], [n - 6 if causal else n]
            got = binding.cache_attention(cache, q.to(DEV), ints(off), ints(lens), 6, n, causal=causal)
            want, weight, size, floor = model.attend(q.double().numpy(), off, lens, causal, dim ** -0.5)
            tol = close_bound(dtype, want, weight, size, floor, n, dim)
            err = np.abs(got.double().cpu().numpy() - want)
            assert (err <= tol).all(), (value, causal, float((err / tol).max()))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 1, 32, 16), (2, 2, 64, 32), (1, 4, 128, 64), (2, 1, 128, 16)])
@pytest.mark.parametrize("spread", [0.3, 2.0])
def test_blocks_of_queries_within_the_close_bound(fmt, dtype, heads, group, dim, block, spread):
    """Ragged rows, scores close together and (where queries are large) tens of nats apart."""
    new, lens = [1, 7, 33, 20], [0, 3 * block + 5, 129, 700]
    cache, model = filled([p + n for p, n in zip(lens, new)], heads, dim, block, fmt, dtype, dim + block)
    q = numbers((sum(new), heads * group, dim), dtype, 5, spread).to(DEV)
    off = offsets(new)
    for causal in (True, False):
        got = binding.cache_attention(cache, q, ints(off), ints(lens), max(new), 720, causal=causal)
        want, weight, size, floor = model.attend(q.cpu().double().numpy(), off, lens, causal, dim ** -0.5)
        err = np.abs(got.double().cpu().numpy() - want)
        tol = close_bound(dtype, want, weight, size, floor, 720, dim)
        assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("gap", [60, 90, 99, 104, 112, 118])
def test_small_probabilities_of_large_values(dtype, block, gap):
    """Keys of probability 2^-gap whose values are 2^(gap + 7) times as large as those of the keys that lead: they are nearly all of the result."""
    dim, n = 64, 5 * block
    cache, model = both(5, 1, dim, block, "e4m3")
    k, v = torch.zeros((n, 1, dim)), numbers((n, 1, dim), "fp32", gap, 0.0)
    small = torch.arange(n) // block % 2 == 1                 # the second and the fourth block
    q = torch.zeros((2, 1, dim))
    q[:, :, 0], q[:, :, 1] = 1.0, 0.25
    k[:, 0, 1] = torch.linspace(0, 1, n)
    k[small, 0, 0] = -gap * float(np.log(2))
    v[small] *= 2.0 ** 10
    v[~small] *= 2.0 ** (3 - gap)
    k, v, q = (x.to(TORCH[dtype]) for x in (k, v, q))
    binding.cache_append(cache, k.to(DEV), v.to(DEV), ints([0, n]), ints([0]), max_new=n)
    model.append(k.double().numpy(), v.double().numpy(), [0, n], [0])
    attend_and_check(cache, model, q.to(DEV), [2], [n - 2], True, dtype, scale=1.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("block", [16, 64])
def test_scales_that_are_no_powers_of_two(dtype, fmt, block):
    """Memory that is adopted may come with any scales; blocks that grow by one part in fifty move the results' reference again and again."""
    heads, dim, n_blocks = 2, 64, 60
    g = torch.Generator().manual_seed(block)
    codes = [(torch.randn((n_blocks, heads, block, dim), generator=g) * (60 if fmt == "e4m3" else 30)).clamp(-127, 127) for _ in range(2)]
    codes = [x.to(torch.float8_e4m3fn) if fmt == "e4m3" else x.round().to(torch.int8) for x in codes]
    k_scale = 0.01 * (1 + torch.rand((n_blocks, heads), generator=g))
    v_scale = 0.3 * 1.02 ** torch.arange(n_blocks)[:, None] * (1 + 0.1 * torch.rand((n_blocks, heads), generator=g))
    v_scale[n_blocks // 2:] = v_scale[n_blocks // 2:].flip(0)
    held = [x.to(DEV) for x in (*codes, k_scale, v_scale)]
    cache = binding.KvCache(n_blocks, heads, dim, block, fmt, device=DEV, tensors=tuple(held))
    model = Model(n_blocks, heads, dim, block, fmt)
    model.codes = [x.double().numpy() for x in codes]
    model.scale = [k_scale.double().numpy(), v_scale.double().numpy()]
    n = n_blocks * block
    for new in (3, 20):
        q = numbers((new, 2 * heads, dim), dtype, new, 0.3).to(DEV)
        off = [0, new]
        got = binding.cache_attention(cache, q, ints(off), ints([n - new]), new, n)
        want, weight, size, floor = model.attend(q.cpu().double().numpy(), off, [n - new], True, dim ** -0.5)
        # (besides `close_bound`: the values' scale enters a probability through an exponent of 2^-22)
        err, tol = np.abs(got.double().cpu().numpy() - want), close_bound(dtype, want, weight, size, floor, n, dim) + 2.0 ** -22 * weight
        assert (err <= tol).all(), float((err / tol).max())
    # and tokens that come to such blocks
    x = numbers((5, heads, dim), dtype, 9)
    binding.cache_append(cache, x.to(DEV), x.to(DEV), ints([0, 5]), ints([n - 9]), max_new=5)
    model.append(x.double().numpy(), x.double().numpy(), [0, 5], [n - 9])
    assert np.array_equal(cache.v_scale.cpu().double().numpy()[-1], model.scale[1][-1])


# ---------------------------------------------------------------------------------------------------------
# larger calls
# ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("new,lens,heads,group,dim,block", [([300, 65, 129], [0, 700, 31], 2, 1, 64, 32), ([513], [1000], 1, 2, 128, 16), ([70, 1, 200], [5, 400, 0], 1, 4, 32, 128)])
def test_prompts_of_hundreds_of_queries(dtype, new, lens, heads, group, dim, block):
    """Tiles of queries far beyond a block's 64, within rows and across them."""
    cache, model = filled([p + n for p, n in zip(lens, new)], heads, dim, block, "e4m3", dtype, 31)
    q = numbers((sum(new), heads * group, dim), dtype, 6, 0.3).to(DEV)
    attend_and_check(cache, model, q, new, lens, True, dtype)
    attend_and_check(cache, model, q, new, lens, False, dtype, max_keys=10 ** 6)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 128, 64), (4, 1, 64, 16)])
def test_long_rows_under_fp32_queries(fmt, heads, group, dim, block):
    lens, new = [20011, 6000, 3001], [1, 5, 9]
    cache, model = filled([p + n for p, n in zip(lens, new)], heads, dim, block, fmt, "fp32", 13)
    q = numbers((sum(new), heads * group, dim), "fp32", 6, 0.3).to(DEV)
    attend_and_check(cache, model, q, new, lens, True, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("n,new,heads,group", [(400, 1, 1, 1), (3000, 2, 1, 4), (9000, 1, 1, 8), (9000, 30, 4, 1)])
def test_values_whose_sums_pass_fp32(dtype, fmt, n, new, heads, group):
    """Results are means of values: thousands of 2^120 and more have one, though no sum."""
    dim, block = 64, 64
    cache, model = both((n + block - 1) // block, heads, dim, block, fmt)
    k, v = numbers((n, heads, dim), dtype, 1, 0.0), numbers((n, heads, dim), dtype, 2, 0.0)
    v = (v.float().abs() * 2.0 ** 122).to(TORCH[dtype])
    binding.cache_append(cache, k.to(DEV), v.to(DEV), ints([0, n]), ints([0]), max_new=n)
    model.append(k.double().numpy(), v.double().numpy(), [0, n], [0])
    q = numbers((new, heads * group, dim), dtype, 3, 0.0).to(DEV)
    attend_and_check(cache, model, q, [new], [n - new], True, dtype)
