"""Attention over shared prefixes against the definition in 64 bits, and against the attention that reads them row by row."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding
from tests.test_gpu_kv_cache import DEV, Model, bound, ints, numbers, offsets

pytestmark = pytest.mark.gpu


def batch(groups, shared, tails, new, heads, dim, block, fmt, causal, seed=0, spread=1.0, gap=2, copies=False):
    """A cache and its model whose rows share their first positions: groups [G] rows each, shared [G], tails and new [B].  Shared blocks stand in all of
    a group's rows; one that is shared in part is copied for each (`copies`: all of them are)."""
    B = sum(groups)
    grp = [g for g, n in enumerate(groups) for _ in range(n)]
    lens = [shared[g] + t for g, t in zip(grp, tails)]
    ends = [n + m if causal else n for n, m in zip(lens, new)]
    row_blocks = max(1, max(-(-e // block) for e in ends)) + 60000      # (room for rows that make it worth reading shared positions once)
    r = np.random.default_rng(seed + block)
    most = sum(-(-e // block) for e in ends) + sum(-(-s // block) for s in shared) + gap
    ids = iter(r.permutation(most))
    table = np.full((B, row_blocks), -1, np.int32)
    k0, v0 = (numbers((max(1, max(shared)), heads, dim), "fp32", seed + i, spread) for i in range(2))
    first, b = [0], 0
    for g, n in enumerate(groups):
        whole = 0 if copies else shared[g] // block if any(tails[b + j] + (new[b + j] if causal else 0) for j in range(n)) else -(-shared[g] // block)
        common = [next(ids) for _ in range(whole)]
        for j in range(n):
            table[b, :whole] = common
            for i in range(whole, -(-ends[b] // block)):
                table[b, i] = next(ids)
            b += 1
        first.append(b)
    cache = binding.KvCache(most, heads, dim, block, fmt, table=ints(table), row_blocks=row_blocks, device=DEV)
    model = Model(most, heads, dim, block, fmt, table, row_blocks)
    # the shared positions into every row (the same numbers), then each row's own
    kt, vt = (torch.cat([x[: shared[g]] for g in grp]) if sum(shared[g] for g in grp) else x[:0] for x in (k0, v0))
    off = offsets([shared[g] for g in grp])
    if kt.shape[0]:
        binding.cache_append(cache, kt.to(DEV), vt.to(DEV), ints(off), ints([0] * B), max(shared))
    more = [e - shared[g] for e, g in zip(ends, grp)]
    if sum(more):
        kx, vx = (numbers((sum(more), heads, dim), "fp32", seed + 7 + i, spread) for i in range(2))
        binding.cache_append(cache, kx.to(DEV), vx.to(DEV), ints(offsets(more)), ints([shared[g] for g in grp]), max(more))
    for z, (codes, scale) in enumerate(((cache.k_codes, cache.k_scale), (cache.v_codes, cache.v_scale))):
        model.codes[z], model.scale[z] = codes.float().cpu().double().numpy(), scale.cpu().double().numpy()
    return cache, model, first, lens, ends


FAR = 1 << 21        # positions to plan for that make it worth reading shared ones once, whatever there are


def run(cache, q, new, lens, first, shared, ends, causal, plan=FAR, **kw):
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = binding.cache_attention_shared(cache, q, ints(offsets(new)), ints(lens), ints(first), ints(shared), max(1, max(new)), plan + max(1, max(ends)),
                                         max_shared=plan + max(shared), causal=causal, status_t=status, **kw)
    return out, int(status.item())


def check(groups, shared, tails, new, heads, per_kv, dim, block, fmt, dtype, causal, seed=0, spread=1.0, scale=None, copies=False):
    cache, model, first, lens, ends = batch(groups, shared, tails, new, heads, dim, block, fmt, causal, seed, spread, copies=copies)
    q = numbers((sum(new), heads * per_kv, dim), dtype, seed + 3, 0.3)
    out, status = run(cache, q.to(DEV), new, lens, first, shared, ends, causal, scale=scale)
    assert status == 0
    off = offsets(new)
    want, weight, size, floor = model.attend(q.double().numpy(), off, lens, causal, scale or dim ** -0.5)
    err = np.abs(out.double().cpu().numpy() - want)
    limit = bound(dtype, want, weight, size, floor, max(1, max(ends)), dim)
    assert (err <= limit).all(), (err / limit).max()
    return cache, q, out, (new, lens, first, shared, ends, causal)


SHAPES = [(1, 1, 32, 16), (2, 1, 64, 32), (1, 4, 128, 64), (2, 2, 128, 16), (1, 8, 64, 128), (3, 1, 32, 64), (1, 3, 128, 128)]


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("bf16", "int8"), ("fp32", "e4m3"), ("fp32", "int8")])
@pytest.mark.parametrize("heads,per_kv,dim,block", SHAPES)
def test_groups_of_all_kinds(dtype, fmt, heads, per_kv, dim, block):
    """Prefixes of none, one and many tiles of keys, that end inside blocks and tiles; tails of none and more; rows without queries; groups of one row."""
    check([3, 1, 4, 2], [300, 0, 17, 128], [0, 5, 140, 1, 16, 0, 33, 2, 0, 129], [1, 2, 1, 3, 0, 1, 4, 1, 2, 5], heads, per_kv, dim, block, fmt, dtype, True, seed=dim)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("bf16", "int8"), ("fp32", "e4m3"), ("fp32", "int8")])
@pytest.mark.parametrize("dim,block", [(32, 64), (64, 16), (128, 32)])
def test_more_rows_than_a_tile(dtype, fmt, dim, block):
    """Two tiles of rows at once (over 128), several items (over 256), prefixes over many CTAs."""
    check([9, 5], [1000, 257], [3 * b for b in range(14)], [8] * 9 + [7] * 5, 1, 4, dim, block, fmt, dtype, True, seed=5)
    check([20], [2500], [0] * 20, [9] * 20, 1, 4, dim, block, fmt, dtype, False, seed=6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [32, 64, 128])
def test_all_of_it_shared(dtype, dim):
    """An encoder's keys: no tails, all queries see the same positions, lengths around tiles and blocks; a source of no length."""
    for lens in ([127, 128, 129], [1, 0, 16], [255, 256, 400]):
        check([2, 3, 1], lens, [0] * 6, [5, 1, 0, 2, 3, 4], 2, 2, dim, 32, "int8", dtype, False, seed=lens[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_groups_and_heads(dtype):
    """More items than CTAs, most of them of a tile or two: every CTA goes through several, of all lengths."""
    groups = [1 + g % 4 for g in range(40)]
    rows = sum(groups)
    check(groups, [(37 * g) % 300 for g in range(40)], [b % 9 for b in range(rows)], [1 + b % 2 for b in range(rows)], 8, 2, 128, 16, "int8", dtype, True, seed=9)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_queries_behind_a_prefix(dtype):
    """Tails with more rows than a tile: every query sees a different number of keys."""
    check([2], [200], [10, 0], [150, 70], 1, 2, 64, 32, "e4m3", dtype, True)
    check([1, 1], [0, 40], [0, 0], [300, 1], 1, 1, 128, 16, "int8", dtype, True)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("fp32", "int8")])
def test_long_prefixes(dtype, fmt):
    check([16], [20001], [7 * b for b in range(16)], [1] * 16, 2, 4, 128, 64, fmt, dtype, True, seed=1)
    check([2, 1], [9000, 30], [0, 12000, 3], [1, 2, 1], 1, 2, 64, 16, fmt, dtype, True, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scales_and_scores_far_apart(dtype):
    """Blocks whose numbers differ by orders of magnitude, and scores that leave one key."""
    check([4], [700], [3, 60, 0, 200], [2] * 4, 1, 2, 64, 16, "e4m3", dtype, True, seed=1, spread=3.0)
    check([4], [700], [3, 60, 0, 200], [2] * 4, 1, 2, 128, 64, "int8", dtype, True, seed=2, scale=5.0)
    check([4], [700], [3, 60, 0, 200], [2] * 4, 1, 2, 32, 32, "int8", dtype, True, seed=3, scale=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_same_as_row_by_row_and_in_any_company(dtype):
    """Groups of one row each, one group, and the attention that reads every row's own blocks agree within two results' roundings."""
    groups, shared, tails, new = [4], [640], [0, 10, 100, 300], [3, 1, 2, 5]
    cache, q, out, (new, lens, first, shared, ends, causal) = check(groups, shared, tails, new, 2, 4, 64, 32, "int8", dtype, True)
    alone = binding.cache_attention(cache, q.to(DEV), ints(offsets(new)), ints(lens), max(new), max(ends))
    none, _ = run(cache, q.to(DEV), new, lens, [0, 1, 2, 3, 4], [0, 640, 7, 640], ends, True)
    tol = 2 ** -7 if dtype == "bf16" else 2 ** -17
    for x in (alone, none):
        assert float((x.float() - out.float()).abs().max()) <= tol * float(out.float().abs().max())


def test_what_lies_behind_is_not_looked_at():
    """Codes behind the rows' ends (NaN codes of E4M3), blocks that no row sees, and results behind the batch's."""
    cache, model, first, lens, ends = batch([3], [100], [5, 0, 40], [1, 2, 1], 1, 64, 32, "e4m3", True)
    q = numbers((4, 2, 64), "bf16", 1)
    want, _ = run(cache, q.to(DEV), [1, 2, 1], lens, first, [100], ends, True)
    used = {}
    for b, e in enumerate(ends):
        for i in range(-(-e // 32)):
            g = int(model.table[b, i])
            used[g] = max(used.get(g, 0), min(32, e - 32 * i))
    for codes in (cache.k_codes, cache.v_codes):
        raw = codes.view(torch.uint8)
        for g in range(raw.shape[0]):
            raw[g, :, used.get(g, 0):] = 0x7F
    for scale in (cache.k_scale, cache.v_scale):
        for g in range(scale.shape[0]):
            if g not in used:
                scale[g] = float("nan")
    out, status = run(cache, q.to(DEV), [1, 2, 1], lens, first, [100], ends, True)
    assert status == 0 and torch.equal(out, want)


def test_rows_and_groups_that_make_no_sense_are_left_out():
    groups, shared, tails, new = [2, 2], [64, 96], [3, 0, 5, 6], [1, 2, 1, 1]
    cache, model, first, lens, ends = batch(groups, shared, tails, new, 1, 64, 32, "int8", True)
    q = numbers((5, 1, 64), "bf16", 1).to(DEV)
    want, _ = run(cache, q, new, lens, first, shared, ends, True)
    off = offsets(new)
    capacity = cache.row_blocks * 32
    # (groups, shared, offsets, lengths, rows that stay right)
    for fi, sh, of, le, good in (([0, 2, 5], shared, off, lens, [0, 1]), ([0, 2, 4], [-1, 96], off, lens, [2, 3]), ([0, 2, 4], [64, capacity + 1], off, lens, [0, 1]),
                                 ([-1, 2, 4], shared, off, lens, [2, 3]), ([0, 2, 4], [64, 100], off, [*lens[:2], 98, *lens[3:]], [0, 1, 3]),
                                 ([1, 2, 4], shared, off, lens, [1, 2, 3]), ([0, 2, 4], shared, off, [-5, *lens[1:]], [1, 2, 3]),
                                 ([0, 2, 4], shared, [0, 1, 3, 4, 9], lens, [0, 1]), ([0, 4, 2], [64, 64], off, lens, None),
                                 ([2 ** 31 - 1, 2, 4], shared, off, lens, [2, 3]), ([0, 2, 4], [2 ** 31 - 1, 96], off, lens, [2, 3])):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.full_like(want, 7.0)
        binding.cache_attention_shared(cache, q, ints(of), ints(le), ints(fi), ints(sh), 2, FAR + max(ends), max_shared=FAR, causal=True, out=out, status_t=status)
        assert int(status.item()) == binding.AD_ERR_ARG
        for b in good or ():
            rows = slice(off[b], off[b + 1])
            assert torch.allclose(out[rows].float(), want[rows].float(), atol=0.02), (fi, sh, of, le, b)
    # a block that does not exist is left out like in the attention row by row
    cache.table[0, 1] = 10 ** 6
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = binding.cache_attention_shared(cache, q, ints(off), ints(lens), ints(first), ints(shared), 2, FAR + max(ends), max_shared=FAR, status_t=status)
    alone = binding.cache_attention(cache, q[:1], ints([0, 1]), ints(lens[:1]), 2, max(ends))
    assert int(status.item()) == binding.AD_ERR_ARG and torch.allclose(out[:1].float(), alone.float(), atol=0.02) and torch.allclose(out[3:].float(), want[3:].float(), atol=0.02)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strides_streams_and_graphs(dtype):
    """Queries inside a wider array, results given, two streams at once, and a captured call replayed with other lengths: every time the same bits."""
    groups, shared, tails, new = [5, 3], [1500, 64], [0, 3, 200, 1, 50, 0, 9, 300], [2] * 8
    cache, model, first, lens, ends = batch(groups, shared, tails, new, 2, 64, 32, "e4m3", True)
    wide = numbers((16, 12 + 8, 64), dtype, 4).to(DEV)
    q = wide[:, 4: 12]
    args = [ints(offsets(new)), ints(lens), ints(first), ints(shared)]
    call = lambda x, **kw: binding.cache_attention_shared(cache, x, *args, 2, FAR + max(ends), max_shared=FAR, causal=True, **kw)
    want = call(q.contiguous())
    out = torch.empty_like(want)
    assert call(q, out=out) is out and torch.equal(out, want)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(call(q))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = call(q)
        other = call(q * 0.5)
    args[1].copy_(ints([n - (n > 1500) for n in lens]))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(replayed, call(q)) and torch.equal(other, call(q * 0.5)) and not torch.equal(replayed, want)


def test_short_prefixes_are_left_to_the_attention_row_by_row():
    """Where reading them once would not pay, results are that one's, bit by bit; one call or the other by sizes that the host knows."""
    groups, shared, tails, new = [4], [640], [0, 10, 100, 300], [3, 1, 2, 5]
    cache, model, first, lens, ends = batch(groups, shared, tails, new, 2, 64, 32, "int8", True)
    q = numbers((11, 8, 64), "bf16", 3).to(DEV)
    out, status = run(cache, q, new, lens, first, shared, ends, True, plan=0)
    assert status == 0 and torch.equal(out, binding.cache_attention(cache, q, ints(offsets(new)), ints(lens), max(new), max(ends)))
    once, _ = run(cache, q, new, lens, first, shared, ends, True)
    assert not torch.equal(out, once) and float((out.float() - once.float()).abs().max()) <= 2 ** -7 * float(out.float().abs().max())


def test_nothing_to_do():
    cache, model, first, lens, ends = batch([2], [64], [0, 0], [1, 1], 1, 64, 32, "int8", True)
    empty = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    assert binding.cache_attention_shared(cache, empty, ints([0, 0, 0]), ints(lens), ints(first), ints([64]), 1, 65).shape == (0, 2, 64)
    out, status = run(cache, numbers((2, 1, 64), "bf16", 1).to(DEV), [2, 0], [0, 0], first, [0], [0], False)
    assert status == 0 and bool((out == 0).all())


@pytest.mark.parametrize("idle", [[0], [0, 1, 2], [0, 1, 2, 4], [1, 3], [0, 5, 6], [5, 6, 7, 8]])
def test_rows_that_were_given_up(idle):
    """Rows without tokens need no blocks, wherever they stand in their group, and none at all in a group: the others' results are what they were."""
    groups, shared = [5, 4], [300, 129]
    tails, new = [10, 0, 70, 5, 1, 33, 2, 0, 64], [0 if b in idle else 1 + b % 4 for b in range(9)]
    cache, model, first, lens, ends = batch(groups, shared, tails, new, 2, 64, 32, "e4m3", True)
    q = numbers((sum(new), 4, 64), "bf16", 3, 0.3).to(DEV)
    want, status = run(cache, q, new, lens, first, shared, ends, True)
    assert status == 0
    table = cache.table
    for b in idle:
        table[b] = -1
        lens[b] = -5 if b % 2 else 0
    got, status = run(cache, q, new, lens, first, shared, ends, True)
    assert status == 0 and torch.equal(got, want)
    exact = model.attend(q.double().cpu().numpy(), offsets(new), [max(n, 0) for n in lens], True, 64 ** -0.5)
    assert (np.abs(got.double().cpu().numpy() - exact[0]) <= bound("bf16", *exact, max(ends), 64)).all()


@pytest.mark.parametrize("dtype,dim,block", [("bf16", 64, 32), ("bf16", 128, 128), ("fp32", 32, 16)])
def test_many_prefixes_of_one_tile(dtype, dim, block):
    """One tile of keys after another, of as many groups: a half of a CTA that none of them gives any work keeps step with the other, call after call."""
    G, heads = 150, 8
    cache, q, out, (new, lens, first, shared, ends, causal) = check([2] * G, [128] * G, [b % 3 for b in range(2 * G)], [1] * (2 * G), heads, 1, dim, block, "int8", dtype, True, seed=11)
    for _ in range(20):
        again, status = run(cache, q.to(DEV), new, lens, first, shared, ends, causal)
        assert status == 0 and torch.equal(again, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,per_kv,dim,block", [(2, 4, 128, 64), (1, 1, 32, 16), (8, 2, 64, 32)])
def test_long_rows_beside_long_prefixes(dtype, heads, per_kv, dim, block):
    """A newcomer that shares nothing and is as long as a group's prefix, rows whose own positions are many behind a short prefix, and short ones among them: own positions in one
    part, in several, and in many."""
    check([4, 1, 2], [3000, 0, 100], [5, 0, 60, 511, 5000, 2000, 480], [1, 2, 1, 3, 2, 1, 4], heads, per_kv, dim, block, "int8", dtype, True, seed=21)
    check([3, 1], [1000, 0], [0, 700, 3, 9000], [2, 9, 1, 20], heads, per_kv, dim, block, "e4m3", dtype, False, seed=22)


def test_own_positions_around_where_they_are_split():
    """Longest own positions just below and from 512 on, where parts begin; calls in turn on the same scratch sizes."""
    for own in (495, 496, 511, 512, 513, 600):
        check([3, 2], [200, 64], [own, 3, 100, 0, 17], [1] * 5, 2, 2, 64, 32, "int8", "bf16", True, seed=own)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_planned_for_one_length_and_replayed_for_others(dtype):
    """A captured call whose rows grow from short own positions to long ones and back: what is split is decided anew by every replay."""
    shared, grow = [640, 0], ([3, 50, 1, 20], [3, 50, 1, 4000], [900, 50, 1, 4000], [3, 0, 400, 20])
    most = [max(t) for t in zip(*grow)]
    cache, model, first, lens, ends = batch([3, 1], shared, most, [2] * 4, 2, 64, 32, "int8", True)
    q = numbers((8, 4, 64), dtype, 5, 0.3)
    len_t, qd = ints(lens), q.to(DEV)
    call = lambda: binding.cache_attention_shared(cache, qd, ints_off, len_t, first_t, shared_t, 2, FAR + 5000, max_shared=FAR)
    ints_off, first_t, shared_t = ints(offsets([2] * 4)), ints(first), ints(shared)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for tails in grow:
        now = [s + t for s, t in zip([640] * 3 + [0], tails)]
        len_t.copy_(ints(now))
        graph.replay()
        torch.cuda.synchronize()
        want, weight, size, floor = model.attend(q.double().numpy(), offsets([2] * 4), now, True, 64 ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - want) <= bound(dtype, want, weight, size, floor, max(now) + 2, 64)).all()
        assert torch.equal(out, call())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_groups_that_overlap_are_left_out_as_a_whole(dtype):
    """Groups whose rows are others' as well: what there is no room for is left out, and does not come back as attention over its own positions alone."""
    groups, shared, tails, new = [8, 4], [96, 96], [3, 0, 5, 6, 1, 2, 3, 4, 9, 8, 7, 40], [1] * 12
    cache, model, first, lens, ends = batch(groups, shared, tails, new, 1, 64, 32, "int8", True)
    q = numbers((12, 1, 64), dtype, 1).to(DEV)
    want, status = run(cache, q, new, lens, first, shared, ends, True)
    assert status == 0
    for bounds, left in (([0, 8, 4, 12], range(8, 12)), ([0, 8, 0, 12], range(8, 12))):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.full_like(want, 7.0)
        binding.cache_attention_shared(cache, q, ints(range(13)), ints(lens), ints(bounds), ints([96, 96, 96]), 1, FAR + max(ends), max_shared=FAR, out=out, status_t=status)
        assert int(status.item()) == binding.AD_ERR_ARG and bool((out[list(left)] == 7).all())
        assert torch.allclose(out[:8].float(), want[:8].float(), atol=0.02)
