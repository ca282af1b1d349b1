"""Samples whose drafts are the ones that were fed and verified: rows go on by as many tokens as were accepted, across blocks, and branch from there; prefixes read once, in pools that run out
of blocks as well, and at addresses beyond 32 bits."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding
from tests.test_gpu_accept_sampled import accept
from tests.test_gpu_branching import contents
from tests.test_gpu_kv_cache import DEV, Model, bound, ints, numbers, offsets
from tests.test_gpu_pool import Pool

pytestmark = pytest.mark.gpu
FAR = 1 << 21        # positions to plan for that make it worth reading shared ones once, whatever there are


class Decoder:
    """Two layers of attention between an embedding and the projection to the vocabulary, on a pool, with a model of what the pool holds."""

    def __init__(self, B, V, n_blocks, dtype, fmt, heads, group, dim, block):
        self.B, self.V, self.dtype, self.fmt, self.heads, self.dim, self.block, self.H, self.d = B, V, dtype, fmt, heads, dim, block, heads * group, heads * group * dim
        self.dt, self.row_blocks = (torch.bfloat16 if dtype == "bf16" else torch.float32), 60000
        self.pool = binding.KvPool(B, self.row_blocks, n_blocks, block, device=DEV)
        self.layers = [self.pool.add_cache(heads, dim, fmt) for _ in range(2)]
        self.held = Pool(B, self.row_blocks, n_blocks, block, [contents(c) for c in self.layers])
        self.emb = numbers((V, self.d), dtype, 1).to(DEV)
        self.wqkv = (numbers((2 * (self.H + 2 * heads) * dim, self.d), dtype, 2) * self.d ** -0.5).to(self.dt).to(DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def same(self):
        """The pool as its model has it; its table."""
        for layer, cache in zip(self.held.layers, self.layers):
            assert all(torch.equal(a, b) for a, b in zip(layer, contents(cache)))
        table = self.pool.table[:, :16].cpu().numpy()
        assert [[int(e) for e in row if e >= 0] for row in table] == self.held.rows and self.pool.refs.cpu().tolist() == self.held.refs()
        return table

    def fork(self, parent, lens):
        binding.cache_fork(self.pool, ints(parent), ints(lens), self.status)
        self.held.fork(parent, lens)
        self.same()

    def forward(self, tokens, new, lens, shared, groups):
        """Scores behind every token that is fed; None: no room, and no row has changed that does not own what it would write."""
        B, block, dim, heads, H, st = self.B, self.block, self.dim, self.heads, self.H, self.status
        off, most, M = offsets(new), max(new), sum(new)
        o_t, l_t = ints(off), ints(lens)
        binding.cache_reserve(self.pool, o_t, l_t, st)
        room = self.held.reserve(off, lens)
        table = self.same()
        qkv = binding.linear(self.emb[torch.tensor(tokens, device=DEV)], self.wqkv, None, None).to(self.dt).view(M, 2, H + 2 * heads, dim)
        total = self.emb[torch.tensor(tokens, device=DEV)].float()
        for i, cache in enumerate(self.layers):
            q, k, v = (qkv[:, i, a:b] for a, b in ((0, H), (H, H + heads), (H + heads, H + 2 * heads)))
            binding.cache_append(cache, k, v, o_t, l_t, max_new=most, status_t=st)      # (whether there was room or not: a program does not look in between)
            if not room:
                continue
            read = lambda: ([c.float().cpu().double().numpy() for c in (cache.k_codes, cache.v_codes)], [s.cpu().double().numpy() for s in (cache.k_scale, cache.v_scale)])
            model = Model(self.pool.n_blocks, heads, dim, block, self.fmt, table, 16)
            model.codes, model.scale = read()
            self.held.layers[i] = contents(cache)
            args = (q, o_t, l_t, ints(groups), ints(shared), most, FAR)
            att = binding.cache_attention_shared(cache, *args, max_shared=FAR, status_t=st)
            want, weight, size, floor = model.attend(q.double().cpu().numpy(), off, lens, True, dim ** -0.5)
            assert (np.abs(att.double().cpu().numpy() - want) <= bound(self.dtype, want, weight, size, floor, 16 * block, dim)).all()
            total = total + att.reshape(M, self.d).float()
        if not room:
            assert int(st.item()) == binding.AD_ERR_CAPACITY
            # rows that own all they would write have been written, behind their ends; no other block has changed
            spans, refs = self.held.spans(off, lens), self.held.refs()
            owned = [[self.held.rows[b][i] if i < len(self.held.rows[b]) else -1 for i in span] for b, span in enumerate(spans)]
            written = {e for row in owned for e in row if all(x >= 0 and refs[x] == 1 for x in row)}
            still = torch.tensor([e for e in range(self.pool.n_blocks) if e not in written])
            for i, cache in enumerate(self.layers):
                now = contents(cache)
                assert all(torch.equal(a[still], b[still]) for a, b in zip(now, self.held.layers[i]))
                self.held.layers[i] = now
            self.same()
            st.zero_()
            return None
        assert int(st.item()) == 0
        return binding.linear(total.to(self.dt), self.emb, None, st) * (3.0 / self.dim ** 0.5)


@pytest.mark.parametrize("dtype,fmt,heads,group,dim,block", [("bf16", "e4m3", 2, 2, 64, 16), ("fp32", "int8", 1, 4, 32, 16), ("bf16", "int8", 1, 2, 128, 16)])
def test_accepted_drafts_are_kept_and_branched_from(dtype, fmt, heads, group, dim, block):
    """Two sources with three samples each.  Per step every sample drafts greedily, a token at a time; gives these positions up; feeds the same drafts as one block; keeps the ones that
    sampling accepts; and samples take each other's places.  Where the pool has no room, samples are given up, and the step is made again."""
    B, V, kmax, prompt, groups = 6, 300, 4, [70, 33], [0, 3, 6]
    dec = Decoder(B, V, 15, dtype, fmt, heads, group, dim, block)
    lib = binding.load()
    sizes = (1 if dtype == "bf16" else 0, dec.H, B, 8, kmax, FAR)
    assert lib.ad_cache_attention_shared_scratch_bytes(dec.layers[0]._ref, *sizes, 2, FAR) > lib.ad_cache_attention_scratch_bytes(dec.layers[0]._ref, *sizes[:3], *sizes[4:])   # (read once)
    r = np.random.default_rng(dim)
    dec.forward(r.integers(0, V, sum(prompt)), [prompt[0], 0, 0, prompt[1], 0, 0], [0] * B, [0, 0], groups)
    lens = [prompt[0]] * 3 + [prompt[1]] * 3
    dec.fork([0, 0, 0, 3, 3, 3], lens)
    last, alive = [int(x) for x in r.integers(0, V, B)], [True] * B
    kept = crossed = refused = 0
    for step in range(12):
        new = [int(x) * a for x, a in zip(r.integers(2, kmax + 1, B), alive)]
        # greedy drafts, one after the other behind the rows' ends; then these positions are given up
        drafts, fed, at = np.full((B, kmax), -1), list(last), list(lens)
        for i in range(kmax):
            one = [int(n > i) for n in new]
            scores = dec.forward([fed[b] for b in range(B) if one[b]], one, at, prompt, groups) if any(one) else None
            if scores is None:
                break
            best = scores.argmax(1).tolist()
            for b in range(B):
                if one[b]:
                    drafts[b, i] = fed[b] = best.pop(0)
                    at[b] += 1
        room = all((drafts[b, : new[b]] >= 0).all() for b in range(B))
        tokens = np.concatenate([[last[b]] + list(drafts[b, : new[b] - 1]) for b in range(B) if new[b]]) if room else None
        scores = dec.forward(tokens, new, lens, prompt, groups) if room else None
        if scores is None:                                    # the last of every source with more than one is given up
            refused += 1
            dec.fork([-1 if b % 3 and (b % 3 == 2 or not alive[b + 1]) and alive[b] else (b if alive[b] else -1) for b in range(B)], lens)
            alive = [bool(row) for row in dec.held.rows]
            lens = [n if a else 0 for n, a in zip(lens, alive)]
            continue
        off = offsets(new)
        left = torch.empty_like(scores)
        binding.sample(scores, torch.tensor(r.random(sum(new), dtype=np.float32), device=DEV), top_k=ints([20] * sum(new)), filtered=left, status_t=dec.status)
        u, rr = r.random((B, kmax), dtype=np.float32), r.random(B, dtype=np.float32)
        ids, n = (x.cpu().numpy() for x in binding.accept_sampled(left, None, ints(drafts), ints(off), torch.tensor(u, device=DEV), torch.tensor(rr, device=DEV), status_t=dec.status))
        t2, n2 = accept(left.double().cpu().numpy(), None, drafts, off, u, rr, 1.0)
        assert np.array_equal(ids, t2) and np.array_equal(n, n2)
        for b in range(B):
            if new[b]:
                # the last token and the accepted drafts in front of the newest one were fed: they stay
                kept += int(n[b]) - 1
                crossed += n[b] > 1 and lens[b] // block != (lens[b] + int(n[b]) - 1) // block
                lens[b], last[b] = lens[b] + int(n[b]), int(ids[b, n[b] - 1])
        parent = [-1 if not alive[b] else b if r.random() < 0.7 else int(r.choice([p for p in range(3 * (b // 3), 3 * (b // 3) + 3) if alive[p]])) for b in range(B)]
        lens, last = [lens[p] if p >= 0 else 0 for p in parent], [last[p] if p >= 0 else 0 for p in parent]
        dec.fork(parent, lens)
        if step % 3 == 2:
            assert int(binding.cache_compact(dec.pool).item()) == dec.held.compact()
            dec.same()
        if max(lens) + 2 * kmax > 15 * block:
            break
    assert int(dec.status.item()) == 0 and any(alive)
    assert kept > 0 and crossed > 0 and refused > 0, (kept, crossed, refused)


def test_shared_blocks_beyond_32_bits():
    """Prefixes read once from blocks that lie beyond 2^32 bytes of keys, before and after they are moved to the front."""
    heads, dim, block = 8, 128, 64
    n_blocks = (1 << 32) // (heads * dim * block) + 40
    pool = binding.KvPool(4, 60000, n_blocks, block, device=DEV)
    cache, st = pool.add_cache(heads, dim, "int8"), torch.zeros(1, dtype=torch.int32, device=DEV)
    pool.refs[: n_blocks - 9] = 1                               # (somebody else's)
    off, lens = ints([0, 150, 150, 150, 150]), ints([0] * 4)
    binding.cache_reserve(pool, off, lens, st)
    binding.cache_append(cache, numbers((150, heads, dim), "bf16", 1).to(DEV), numbers((150, heads, dim), "bf16", 2).to(DEV), off, lens, 150, status_t=st)
    binding.cache_fork(pool, ints([0, 0, 0, -1]), ints([150] * 3 + [0]), st)
    off, lens = ints([0, 3, 6, 9, 9]), ints([150] * 3 + [0])
    binding.cache_reserve(pool, off, lens, st)
    binding.cache_append(cache, numbers((9, heads, dim), "bf16", 3).to(DEV), numbers((9, heads, dim), "bf16", 4).to(DEV), off, lens, 3, status_t=st)
    assert int(pool.table[0, 0]) == n_blocks - 9
    q = numbers((9, 2 * heads, dim), "bf16", 5, 0.3).to(DEV)
    call = lambda plan: binding.cache_attention_shared(cache, q, off, lens, ints([0, 3, 4]), ints([150, 0]), 3, FAR, max_shared=plan, status_t=st)
    out, alone = call(FAR), call(0)
    assert not torch.equal(out, alone) and float((out.float() - alone.float()).abs().max()) <= 2 ** -7 * float(alone.float().abs().max())
    pool.refs[: n_blocks - 9] = 0
    assert int(binding.cache_compact(pool).item()) == 5 and torch.equal(call(FAR), out) and int(st.item()) == 0
