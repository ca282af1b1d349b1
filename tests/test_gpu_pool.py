"""Pools of cache blocks against a model on the host: forking, handing out blocks with copies of shared ones, giving back, moving to the front."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding
from tests.test_gpu_kv_cache import DEV, ints, offsets

pytestmark = pytest.mark.gpu


class Pool:
    """A pool in plain Python: rows are lists of block ids, contents are arrays that are copied."""

    def __init__(self, rows, row_blocks, n_blocks, block, layers=()):
        self.rows, self.row_blocks, self.n_blocks, self.block = [[] for _ in range(rows)], row_blocks, n_blocks, block
        self.layers = [[x.clone() for x in layer] for layer in layers]          # (k codes, v codes, k scale, v scale) as bytes and FP32

    def count(self, e):
        return sum(row.count(e) for row in self.rows)

    def refs(self):
        n = [0] * self.n_blocks
        for row in self.rows:
            for e in row:
                n[e] += 1
        return n

    def up(self, n):
        return -(-n // self.block)

    def fork(self, parent, lens):
        old = [list(r) for r in self.rows]
        for b, (p, n) in enumerate(zip(parent, lens)):
            self.rows[b] = old[p][: self.up(n)] if p >= 0 else []

    def spans(self, off, lens):
        return [range(n // self.block, (n + off[b + 1] - off[b] - 1) // self.block + 1) if off[b + 1] > off[b] else range(0) for b, n in enumerate(lens)]

    def reserve(self, off, lens):
        """False: not enough blocks, nothing has happened."""
        refs, spans = self.refs(), self.spans(off, lens)
        writers = {}
        for b, span in enumerate(spans):
            for i in span:
                if i < len(self.rows[b]):
                    writers.setdefault(self.rows[b][i], []).append((b, i))
        lacks = []
        for b, span in enumerate(spans):
            for i in span:
                e = self.rows[b][i] if i < len(self.rows[b]) else None
                keeps = e is not None and (refs[e] == 1 or (len(writers[e]) == refs[e] and writers[e][0] == (b, i)))
                if not keeps:
                    lacks.append((b, i, e))
        free = [e for e in range(self.n_blocks) if refs[e] == 0]
        if len(lacks) > len(free):
            return False
        for (b, i, e), to in zip(lacks, free):
            if e is None:
                assert i == len(self.rows[b]), "the model's rows have no gaps"
                self.rows[b].append(to)
                continue
            self.rows[b][i] = to
            live = lens[b] % self.block if i == lens[b] // self.block else 0
            if live:
                for layer in self.layers:
                    for x in layer[:2]:
                        x[to, :, :live] = x[e, :, :live]
                    for x in layer[2:]:
                        x[to] = x[e]
        return True

    def compact(self):
        refs = self.refs()
        used = sum(1 for r in refs if r)
        holes = [e for e in range(used) if not refs[e]]
        to = dict(zip([e for e in range(used, self.n_blocks) if refs[e]], holes))
        self.rows = [[to.get(e, e) for e in row] for row in self.rows]
        for layer in self.layers:
            for x in layer:
                for src, dst in to.items():
                    x[dst] = x[src]
        return used

    def same(self, pool):
        table = pool.table.cpu().tolist()
        assert [[e for e in row if e >= 0] for row in table] == self.rows
        assert all(row == r + [-1] * (self.row_blocks - len(r)) for row, r in zip(table, self.rows))
        assert pool.refs.cpu().tolist() == self.refs()
        for cache, layer in zip(pool.caches, self.layers):
            got = (cache.k_codes.view(torch.uint8), cache.v_codes.view(torch.uint8), cache.k_scale, cache.v_scale)
            assert all(torch.equal(a.cpu(), b) for a, b in zip(got, layer))


def both(rows, row_blocks, n_blocks, block, shapes=()):
    """A pool and its model; `shapes`: (heads, dim, format) of its caches, filled with any codes."""
    pool = binding.KvPool(rows, row_blocks, n_blocks, block, device=DEV)
    g = torch.Generator().manual_seed(n_blocks)
    layers = []
    for heads, dim, fmt in shapes:
        cache = pool.add_cache(heads, dim, fmt)
        for codes in (cache.k_codes, cache.v_codes):
            codes.view(torch.uint8).copy_(torch.randint(0, 256, codes.shape, generator=g, dtype=torch.uint8))
        for scale in (cache.k_scale, cache.v_scale):
            scale.copy_(torch.rand(scale.shape, generator=g) + 0.5)
        layers.append([cache.k_codes.view(torch.uint8).cpu(), cache.v_codes.view(torch.uint8).cpu(), cache.k_scale.cpu(), cache.v_scale.cpu()])
    return pool, Pool(rows, row_blocks, n_blocks, block, layers)


def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("rows,row_blocks,n_blocks,block,shapes", [
    (1, 1, 1, 16, [(1, 32, "int8")]), (4, 5, 30, 16, [(2, 32, "e4m3"), (3, 128, "int8")]), (7, 9, 90, 32, [(1, 64, "int8")]), (33, 6, 300, 64, [(2, 64, "e4m3")]),
    (40, 40, 2000, 16, []), (12, 4, 9000, 128, [(1, 128, "int8"), (1, 32, "int8"), (5, 64, "e4m3")])])
def test_any_sequence_of_calls(rows, row_blocks, n_blocks, block, shapes):
    """Rows grow, fork, are cut, dropped and moved, in any order and through shared blocks that are full, partly filled or behind a row's length."""
    pool, model = both(rows, row_blocks, n_blocks, block, shapes)
    r = np.random.default_rng(rows + block)
    lens, st = [0] * rows, status()
    refused = 0
    for step in range(14):
        new = [int(x) for x in r.integers(0, 2 * block + 2, rows) * (r.random(rows) < 0.7)]
        new = [min(n, row_blocks * block - lens[b]) for b, n in enumerate(new)]
        off = offsets(new)
        st.zero_()
        binding.cache_reserve(pool, ints(off), ints(lens), st)
        if model.reserve(off, lens):
            assert int(st.item()) == 0
            lens = [n + m for n, m in zip(lens, new)]
        else:
            assert int(st.item()) == binding.AD_ERR_CAPACITY
            refused += 1
        model.same(pool)
        parent = [int(x) for x in r.integers(-1, rows, rows)] if step % 3 == 0 else [b if r.random() < 0.7 else int(r.integers(0, rows)) for b in range(rows)]
        keep = [0 if p < 0 else int(r.integers(0, lens[p] + 1)) if r.random() < 0.5 else lens[p] for p in parent]
        st.zero_()
        binding.cache_fork(pool, ints(parent), ints(keep), st)
        model.fork(parent, keep)
        lens = keep
        assert int(st.item()) == 0
        model.same(pool)
        if step % 4 == 1:
            used = binding.cache_compact(pool)
            assert int(used.item()) == model.compact()
            model.same(pool)
    assert refused < 14


def test_batches_of_some_of_the_pools_rows():
    """Rows behind the batch are left as they were, and hold their blocks."""
    pool, model = both(9, 4, 40, 16, [(1, 32, "int8")])
    st = status()
    off, lens = offsets([20] * 9), [0] * 9
    binding.cache_reserve(pool, ints(off), ints(lens), st)
    assert model.reserve(off, lens)
    parent, keep = [2, 2, 2], [20, 17, 16]
    binding.cache_fork(pool, ints(parent), ints(keep), st)
    model.fork(parent, keep)
    model.same(pool)
    off = offsets([1, 1, 0])
    binding.cache_reserve(pool, ints(off), ints(keep), st)
    assert model.reserve(off, keep)
    model.same(pool)
    assert int(st.item()) == 0


def test_the_first_writer_keeps_a_block_that_nobody_else_holds():
    """Of four rows that share a partly filled block three get copies when all of them go on, and all four do while a fifth stays behind."""
    for behind in (False, True):
        pool, model = both(5, 3, 12, 16, [(2, 64, "e4m3")])
        st = status()
        binding.cache_reserve(pool, ints(offsets([21, 0, 0, 0, 0])), ints([0] * 5), st)
        assert model.reserve(offsets([21, 0, 0, 0, 0]), [0] * 5)
        parent = [0, 0, 0, 0, 0 if behind else -1]
        binding.cache_fork(pool, ints(parent), ints([21] * 5), st)
        model.fork(parent, [21] * 5)
        before = pool.table.cpu().clone()
        off = offsets([1, 1, 1, 1, 0])
        binding.cache_reserve(pool, ints(off), ints([21] * 4 + [21 if behind else 0]), st)
        assert model.reserve(off, [21] * 4 + [21 if behind else 0])
        model.same(pool)
        assert (pool.table.cpu()[:4, 1] == before[:4, 1]).tolist() == [not behind, False, False, False]
        assert int(st.item()) == 0


def test_a_pool_without_enough_blocks_stays_as_it_is():
    pool, model = both(3, 8, 5, 16, [(1, 32, "int8")])
    st = status()
    for new, good in (([16, 17, 16], True), ([1, 1, 0], False), ([1, 0, 0], True), ([0, 0, 1], False)):
        lens = [len(r) * 16 for r in model.rows]
        off = offsets(new)
        st.zero_()
        binding.cache_reserve(pool, ints(off), ints(lens), st)
        assert model.reserve(off, lens) == good and int(st.item()) == (0 if good else binding.AD_ERR_CAPACITY)
        model.same(pool)


def test_rows_that_make_no_sense_are_left_alone():
    pool, model = both(6, 4, 40, 16, [(1, 32, "int8")])
    st = status()
    off, lens = offsets([20, 30, 40, 10, 5, 1]), [0] * 6
    binding.cache_reserve(pool, ints(off), ints(lens), st)
    assert model.reserve(off, lens) and int(st.item()) == 0
    # parents that there are none of, lengths below zero or beyond a row: as they were
    for parent, keep, want in (([6, 0, 1, 2, 3, 4], [1, 20, 30, 40, 10, 5], binding.AD_ERR_ARG), ([0, 1, 2, 3, 4, 5], [20, -1, 40, 10, 5, 1], binding.AD_ERR_ARG),
                               ([0, 1, 2 ** 31 - 1, 3, 4, 5], [20, 30, 40, 10, 5, 1], binding.AD_ERR_ARG),
                               ([0, 1, 2, 3, 4, 5], [20, 30, 40, 65, 5, 1], binding.AD_ERR_CAPACITY), ([0, 1, 2, 3, 4, 5], [20, 30, 40, 2 ** 31 - 1, 5, 1], binding.AD_ERR_CAPACITY)):
        st.zero_()
        binding.cache_fork(pool, ints(parent), ints(keep), st)
        old = [list(r) for r in model.rows]
        for b, (p, n) in enumerate(zip(parent, keep)):
            if p < 6 and 0 <= n <= 64:
                model.rows[b] = old[p][: model.up(n)]
        model.same(pool)
        assert int(st.item()) == want
    # more than the parent holds: what there is
    st.zero_()
    binding.cache_fork(pool, ints([5] * 6), ints([1, 64, 16, 17, 0, 1]), st)
    model.fork([5] * 6, [1, 64, 16, 17, 0, 1])
    model.same(pool)
    assert int(st.item()) == binding.AD_ERR_ARG
    # offsets that descend or start below zero, lengths below zero, rows beyond their capacity
    lens = [len(r) * 16 for r in model.rows]
    for bad_off, bad_len, want in (([0, 5, 3, 4, 5, 6, 7], lens, binding.AD_ERR_ARG), ([-3, 1, 1, 1, 1, 1, 1], lens, binding.AD_ERR_ARG),
                                   ([0, 1, 1, 1, 1, 1, 1], [-1] + lens[1:], binding.AD_ERR_ARG), ([0, 1, 1, 1, 1, 1, 1], [64] + lens[1:], binding.AD_ERR_CAPACITY),
                                   ([0, 1, 1, 1, 1, 1, 1], [2 ** 31 - 1] + lens[1:], binding.AD_ERR_CAPACITY), ([0, 65, 65, 65, 65, 65, 65], [0] + lens[1:], binding.AD_ERR_CAPACITY)):
        st.zero_()
        binding.cache_reserve(pool, ints(bad_off), ints(bad_len), st)
        good = [max(0, bad_off[b + 1] - bad_off[b]) if bad_off[b] >= 0 and 0 <= bad_len[b] and bad_len[b] + bad_off[b + 1] - bad_off[b] <= 64 else 0 for b in range(6)]
        assert model.reserve(offsets(good), [max(0, min(n, 64)) for n in bad_len])
        lens = [len(r) * 16 for r in model.rows]
        model.same(pool)
        assert int(st.item()) == want


@pytest.mark.parametrize("rows,row_blocks", [(8192, 3), (2000, 40), (300, 700), (1, 5000)])
def test_large_batches_are_forked(rows, row_blocks):
    pool, model = both(rows, row_blocks, rows * row_blocks + 7, 16)
    r = np.random.default_rng(1)
    ids = r.permutation(pool.n_blocks)[: rows * row_blocks].reshape(rows, row_blocks)
    pool.table.copy_(torch.tensor(ids, dtype=torch.int32))
    pool.refs.copy_(torch.bincount(torch.tensor(ids).flatten(), minlength=pool.n_blocks).int())
    parent, keep = r.integers(-1, rows, rows), r.integers(0, row_blocks * 16 + 1, rows)
    st = status()
    binding.cache_fork(pool, ints(parent), ints(keep), st)
    held = np.where(parent < 0, 0, -(-keep // 16))
    want = np.where(np.arange(row_blocks)[None, :] < held[:, None], ids[np.maximum(parent, 0)], -1)
    assert np.array_equal(pool.table.cpu().numpy(), want) and int(st.item()) == 0
    assert np.array_equal(pool.refs.cpu().numpy(), np.bincount(want[want >= 0], minlength=pool.n_blocks))
    assert int(binding.cache_compact(pool).item()) == len(np.unique(want[want >= 0]))
    back = pool.table.cpu().numpy()
    assert (np.unique(back[back >= 0]) == np.arange(len(np.unique(want[want >= 0])))).all()
    # the same entries are equal as before, and blocks in front stay where they are
    used = len(np.unique(want[want >= 0]))
    assert ((back == want) | (want >= used)).all()
    order = np.unique(want[want >= used])
    holes = np.setdiff1d(np.arange(used), np.unique(want[want >= 0]))
    to = np.arange(pool.n_blocks)
    to[order] = holes
    assert np.array_equal(back, np.where(want >= 0, to[np.maximum(want, 0)], -1))


def test_replayed_from_a_graph_and_on_another_stream():
    """Fork, compaction and reservation captured once and replayed: a turnover of rows, step after step, as the model has it."""
    pool, model = both(6, 6, 60, 16, [(2, 32, "int8"), (1, 64, "e4m3")])
    st = status()
    off, lens = offsets([40, 50, 33, 40, 50, 33]), [0] * 6
    binding.cache_reserve(pool, ints(off), ints(lens), st)
    model.reserve(off, lens)
    parent, keep, new = [3, 4, 5, -1, -1, -1], [40, 50, 33, 0, 0, 0], [1, 15, 16, 40, 50, 33]
    args = (ints(parent), ints(keep), ints(offsets(new)))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.cache_fork(pool, args[0], args[1], st)
        used = binding.cache_compact(pool)
        binding.cache_reserve(pool, args[2], args[1], st)
    for _ in range(4):
        graph.replay()
        model.fork(parent, keep)
        want = model.compact()
        assert model.reserve(offsets(new), keep)
        torch.cuda.synchronize()
        assert int(used.item()) == want and int(st.item()) == 0
        model.same(pool)


def test_empty_and_adopted_pools():
    pool = binding.KvPool(3, 4, 10, 32, device=DEV)
    assert int(binding.cache_compact(pool).item()) == 0 and (pool.table == -1).all()
    table, refs = ints([[4, 2], [4, -1]]), ints([0, 0, 1, 0, 2])
    adopted = binding.KvPool(2, 2, 5, 16, device=DEV, tensors=(table, refs))
    assert int(binding.cache_compact(adopted).item()) == 2
    assert table.tolist() == [[0, 1], [0, -1]] or table.tolist() == [[1, 0], [1, -1]]
    assert refs.tolist()[:2] in ([2, 1], [1, 2]) and refs.tolist()[2:] == [0, 0, 0]


def contents(pool):
    return [x.clone() for c in pool.caches for x in (c.k_codes.view(torch.uint8), c.v_codes.view(torch.uint8), c.k_scale, c.v_scale)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("captured", [False, True])
def test_what_follows_a_refused_reservation_writes_nothing(captured, dtype):
    """Rows that share a partly filled block, and one that lacks its next, go on in a pool that is too small: reserve and append of all layers, one after the other as a program that
    does not look in between runs them, leave every row's tokens as they were.  Once there is room the same calls write what the plain append writes."""
    pool, model = both(5, 4, 4, 16, [(2, 64, "e4m3"), (1, 32, "int8"), (3, 128, "e4m3")])
    st, g = status(), torch.Generator().manual_seed(3)
    numbers = {c: [torch.randn((64, c.n_kv_heads, c.head_dim), generator=g).to(dtype).to(DEV) for _ in range(2)] for c in pool.caches}
    appended = lambda new, lens: [binding.cache_append(c, *(x[: sum(new)] * 50 for x in numbers[c]), ints(offsets(new)), ints(lens), max(new), st) for c in pool.caches]
    for new, lens in (([21, 0, 0, 0, 0], [0] * 5), ([0, 0, 0, 0, 16], [21, 0, 0, 0, 0])):
        binding.cache_reserve(pool, ints(offsets(new)), ints(lens), st)
        appended(new, lens)
    parent, lens = [0, 0, 0, 0, 4], [21] * 4 + [16]
    binding.cache_fork(pool, ints(parent), ints(lens), st)
    assert int(st.item()) == 0 and pool.refs.tolist() == [4, 4, 1, 0]
    before, off_t, len_t, new = contents(pool), ints(offsets([1] * 5)), ints(lens), [1] * 5

    def step():
        binding.cache_reserve(pool, off_t, len_t, st)
        for c in pool.caches:
            binding.cache_append(c, *(x[:5] for x in numbers[c]), off_t, len_t, 1, st)
    call = step
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        call = graph.replay
    for _ in range(2):
        call()
        assert int(st.item()) == binding.AD_ERR_CAPACITY
        assert all(torch.equal(a, b) for a, b in zip(contents(pool), before))
    # without a reservation at all, and a row that owns the first block it would write but lacks the next
    for new, at in (([1] * 5, lens), ([0, 0, 0, 0, 20], [21] * 4 + [10]), ([3, 1, 0, 0, 0], lens)):
        st.zero_()
        appended(new, at)
        assert int(st.item()) == binding.AD_ERR_ARG and all(torch.equal(a, b) for a, b in zip(contents(pool), before))
    # room for all that is left: what the plain append makes of the same blocks
    st.zero_()
    binding.cache_fork(pool, ints([0, -1, -1, -1, 4]), ints([21, 0, 0, 0, 16]), st)
    off_t.copy_(ints(offsets([1, 0, 0, 0, 1])))
    len_t.copy_(ints([21, 0, 0, 0, 16]))
    plain = [binding.KvCache(4, c.n_kv_heads, c.head_dim, 16, c.fmt, row_blocks=4, table=ints([[0, 1, -1, -1]] + [[-1] * 4] * 3 + [[2, 3, -1, -1]]), device=DEV,
                             tensors=[x.clone() for x in (c.k_codes, c.v_codes, c.k_scale, c.v_scale)]) for c in pool.caches]
    call()
    for c, p in zip(pool.caches, plain):
        binding.cache_append(p, *(x[:5] for x in numbers[c]), off_t, len_t, 1)
        assert torch.equal(pool.table, p.table)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((c.k_codes, c.v_codes, c.k_scale, c.v_scale), (p.k_codes, p.v_codes, p.k_scale, p.v_scale)))
    assert int(st.item()) == 0 and not all(torch.equal(a, b) for a, b in zip(contents(pool), before))


def test_a_pool_and_its_caches_go_when_nobody_has_them_any_more():
    """Neither holds the other back until the collector comes by: their memory is torch's again at once, and a cache whose pool went can still be written."""
    import gc
    import weakref
    torch.cuda.synchronize()
    gc.collect()
    gc.disable()
    try:
        before = torch.cuda.memory_allocated()
        pool = binding.KvPool(2, 8, 2048, 64, device=DEV)
        caches = [pool.add_cache(4, 128) for _ in range(2)]
        st, ref = status(), weakref.ref(pool)
        binding.cache_reserve(pool, ints([0, 3, 3]), ints([0, 0]), st)
        del pool
        assert ref() is None
        x = torch.ones((3, 4, 128), device=DEV)
        binding.cache_append(caches[0], x, x, ints([0, 3, 3]), ints([0, 0]), 3, st)
        assert int(st.item()) == 0 and bool((caches[0].k_codes[0, :, :3].float() != 0).all())
        assert torch.cuda.memory_allocated() - before > 2 * 2 * 2048 * 4 * 64 * 128
        del caches, x, st
        assert torch.cuda.memory_allocated() - before < 1 << 20
    finally:
        gc.enable()
