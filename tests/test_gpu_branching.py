"""The pool, the attention over shared prefixes and the sampling as a program uses them: samples of several sources that draft, are verified, branch and are given up;
and all of them at addresses beyond 32 bits."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding
from tests.test_gpu_accept_sampled import accept
from tests.test_gpu_kv_cache import DEV, Model, bound, ints, numbers, offsets
from tests.test_gpu_pool import Pool
from tests.test_gpu_sample import draw

pytestmark = pytest.mark.gpu


def contents(cache):
    return [cache.k_codes.view(torch.uint8).cpu(), cache.v_codes.view(torch.uint8).cpu(), cache.k_scale.cpu(), cache.v_scale.cpu()]


@pytest.mark.parametrize("dtype,fmt,heads,group,dim,block,wide", [("bf16", "e4m3", 2, 2, 64, 16, True), ("fp32", "int8", 1, 4, 32, 32, True), ("bf16", "int8", 1, 2, 128, 16, False)])
def test_samples_that_branch_are_verified_and_given_up(dtype, fmt, heads, group, dim, block, wide):
    """Two sources with three samples each, two layers.  Per step: blocks for the tokens, append, attention with the prompts read once (`wide`: rows planned long enough
    for that) or row by row, truncated scores, acceptance of drafts from them, then samples that take another one's place.  Everything against its model at every step."""
    B, V, kmax, row_blocks, n_blocks = 6, 300, 4, 60000 if wide else 12, 70
    prompt, groups = [70, 33], [0, 3, 6]
    H, d = heads * group, heads * group * dim
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    pool = binding.KvPool(B, row_blocks, n_blocks, block, device=DEV)
    layers = [pool.add_cache(heads, dim, fmt) for _ in range(2)]
    held = Pool(B, row_blocks, n_blocks, block, [contents(c) for c in layers])
    emb = numbers((V, d), dtype, 1).to(DEV)
    wqkv = (numbers((2 * (H + 2 * heads) * dim, d), dtype, 2) * d ** -0.5).to(dt).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = np.random.default_rng(dim)
    temperature = 0.7
    max_keys = (1 << 21) if wide else row_blocks * block

    def same():
        for layer, cache in zip(held.layers, layers):
            assert all(torch.equal(a, b) for a, b in zip(layer, contents(cache)))
        table = pool.table[:, :12].cpu().numpy()
        assert [[int(e) for e in row if e >= 0] for row in table] == held.rows and pool.refs.cpu().tolist() == held.refs()
        return table

    def forward(tokens, new, lens, shared, first):
        """Scores of the tokens that are fed, after both layers."""
        off, most = offsets(new), max(new)
        o_t, l_t = ints(off), ints(lens)
        binding.cache_reserve(pool, o_t, l_t, status)
        assert held.reserve(off, lens)
        table, M = same(), sum(new)
        x = emb[torch.tensor(tokens, device=DEV)]
        qkv = binding.linear(x, wqkv, None, status).to(dt).view(M, 2, (H + 2 * heads), dim)
        total = x.float()
        for i, cache in enumerate(layers):
            model = Model(n_blocks, heads, dim, block, fmt, table, 12)
            read = lambda: ([c.float().cpu().double().numpy() for c in (cache.k_codes, cache.v_codes)], [s.cpu().double().numpy() for s in (cache.k_scale, cache.v_scale)])
            model.codes, model.scale = read()
            q, k, v = (qkv[:, i, a:b] for a, b in ((0, H), (H, H + heads), (H + heads, H + 2 * heads)))
            binding.cache_append(cache, k, v, o_t, l_t, max_new=most, status_t=status)
            model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), off, lens)
            got = Model(n_blocks, heads, dim, block, fmt, table, 12)
            got.codes, got.scale = read()
            for b in range(B):
                assert all(np.array_equal(model.values(z, b, lens[b] + new[b]), got.values(z, b, lens[b] + new[b])) for z in range(2))
            held.layers[i] = contents(cache)
            att = binding.cache_attention_shared(cache, q, o_t, l_t, ints(first), ints(shared), most, max_keys, causal=True, status_t=status)
            want, weight, size, floor = model.attend(q.double().cpu().numpy(), off, lens, True, dim ** -0.5)
            err = np.abs(att.double().cpu().numpy() - want)
            assert (err <= bound(dtype, want, weight, size, floor, 12 * block, dim)).all()
            total = total + att.reshape(M, d).float()
        assert int(status.item()) == 0
        return binding.linear(total.to(dt), emb, None, status) * (2.0 / dim ** 0.5)

    # the prompts, in each source's first row, and samples of it in the others
    new = [prompt[0], 0, 0, prompt[1], 0, 0]
    forward(r.integers(0, V, sum(new)), new, [0] * B, [0, 0], groups)
    lens = [prompt[0]] * 3 + [prompt[1]] * 3
    parent = [0, 0, 0, 3, 3, 3]
    binding.cache_fork(pool, ints(parent), ints(lens), status)
    held.fork(parent, lens)
    same()
    last = [int(x) for x in r.integers(0, V, B)]
    accepted = 0
    for step in range(7):
        new = [int(x) for x in r.integers(1, kmax + 1, B)]
        if step == 3:
            new[int(r.integers(0, B))] = 0
        off, M = offsets(new), sum(new)
        drafts = np.full((B, kmax), -1)
        for b in range(B):
            drafts[b, : new[b]] = r.integers(0, V, new[b])
        tokens = np.concatenate([[last[b]] + list(drafts[b, : new[b] - 1]) for b in range(B) if new[b]])
        scores = forward(tokens, new, lens, prompt, groups)
        # truncated distributions, and what a draw from each would be
        left, rs = torch.empty_like(scores), r.random(M, dtype=np.float32)
        params = dict(temperature=[temperature] * M, top_k=[int(x) for x in r.integers(0, 50, M)], top_p=[float(x) for x in r.uniform(0.3, 1.1, M)], min_p=[0.001] * M)
        t = {n: torch.tensor(x, dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV) for n, x in params.items()}
        drawn, logp = binding.sample(scores, torch.tensor(rs, device=DEV), t["temperature"], t["top_k"], t["top_p"], t["min_p"], filtered=left, status_t=status)
        s64, l64 = scores.double().cpu().numpy(), left.double().cpu().numpy()
        for m in range(M):
            token, lp, ids = draw(s64[m], float(rs[m]), **{n: t[n][m].item() for n in t})
            kept = np.full(V, -np.inf)
            kept[ids] = s64[m, ids]
            assert int(drawn[m]) == token and np.array_equal(l64[m], kept) and abs(float(logp[m]) - lp) <= 2.0 ** -23 * max(1.0, abs(lp))
        u, rr = r.random((B, kmax), dtype=np.float32), r.random(B, dtype=np.float32)
        for b in range(B):                                    # (half of the drafts from what is left, so that some are accepted)
            for i in range(new[b]):
                if r.random() < 0.8:
                    drafts[b, i] = int(np.argmax(l64[off[b] + i]))
        ids, n = binding.accept_sampled(left, None, ints(drafts), ints(off), torch.tensor(u, device=DEV), torch.tensor(rr, device=DEV), temperature=temperature, status_t=status)
        ids, n = ids.cpu().numpy(), n.cpu().numpy()
        t2, n2 = accept(l64, None, drafts, off, u, rr, float(np.float32(temperature)))
        assert np.array_equal(ids, t2) and np.array_equal(n, n2)
        for b in range(B):
            if n[b]:
                # positions that were fed other tokens than were accepted are given up (the last accepted token is fed next)
                lens[b] += 1
                last[b] = int(ids[b, n[b] - 1])
        accepted += int(n.sum())
        # samples of a source take each other's places, at their lengths; what lies behind is given back
        parent = [b if r.random() < 0.6 else int(r.integers(0, 3)) + 3 * (b // 3) for b in range(B)]
        lens, last = [lens[p] for p in parent], [last[p] for p in parent]
        binding.cache_fork(pool, ints(parent), ints(lens), status)
        held.fork(parent, lens)
        same()
        if step % 3 == 2:
            assert int(binding.cache_compact(pool).item()) == held.compact()
            same()
    assert int(status.item()) == 0 and accepted >= B


def test_pools_beyond_32_bits():
    """A cache of more than 2^32 bytes of keys: copies and moves between its last blocks and its first, and attention over shared ones among the last."""
    heads, dim, block = 8, 128, 64
    n_blocks, row_blocks = (1 << 32) // (heads * dim * block) + 40, 60000
    pool = binding.KvPool(4, row_blocks, n_blocks, block, device=DEV)
    cache = pool.add_cache(heads, dim, "int8")
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    pool.refs[: n_blocks - 9] = 1                               # (somebody else's)
    off, lens = offsets([150, 0, 0, 0]), [0] * 4
    binding.cache_reserve(pool, ints(off), ints(lens), st)
    assert pool.table[0, :4].tolist() == [n_blocks - 9, n_blocks - 8, n_blocks - 7, -1]
    k, v = numbers((150, heads, dim), "bf16", 1).to(DEV), numbers((150, heads, dim), "bf16", 2).to(DEV)
    binding.cache_append(cache, k, v, ints(off), ints(lens), 150, status_t=st)
    binding.cache_fork(pool, ints([0, 0, 0, -1]), ints([150] * 3 + [0]), st)
    new = [3, 3, 3, 0]
    off, lens = offsets(new), [150] * 3 + [0]
    binding.cache_reserve(pool, ints(off), ints(lens), st)
    assert pool.table[:3, 2].tolist() == [n_blocks - 7, n_blocks - 6, n_blocks - 5]
    got = [binding.cache_read(cache, ints([0, 150, 300, 450, 450]), ints([0] * 4), 450, 150, torch.float32)[z].view(3, 150, heads, dim) for z in range(2)]
    assert all(torch.equal(x[0], x[1]) and torch.equal(x[0], x[2]) for x in got) and bool(got[1].any())
    kx, vx = numbers((9, heads, dim), "bf16", 3).to(DEV), numbers((9, heads, dim), "bf16", 4).to(DEV)
    binding.cache_append(cache, kx, vx, ints(off), ints(lens), 3, status_t=st)
    q = numbers((9, 2 * heads, dim), "bf16", 5, 0.3).to(DEV)

    def attend_and_check():
        table = pool.table[:, :3].cpu().numpy()
        ids = np.unique(table[table >= 0])
        small = Model(len(ids), heads, dim, block, "int8", np.searchsorted(ids, table), 3)
        at = torch.tensor(ids, device=DEV)
        small.codes = [x[at].float().cpu().double().numpy() for x in (cache.k_codes, cache.v_codes)]
        small.scale = [x[at].cpu().double().numpy() for x in (cache.k_scale, cache.v_scale)]
        out = binding.cache_attention_shared(cache, q, ints(off), ints(lens), ints([0, 3, 4]), ints([150, 0]), 3, 1 << 21, status_t=st)
        want, weight, size, floor = small.attend(q.double().cpu().numpy(), off, lens, True, dim ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - want) <= bound("bf16", want, weight, size, floor, 153, dim)).all() and int(st.item()) == 0
        return out

    out = attend_and_check()
    pool.refs[: n_blocks - 9] = 0
    assert int(binding.cache_compact(pool).item()) == 5
    assert sorted(set(pool.table[:, :3].flatten().tolist()) - {-1}) == [0, 1, 2, 3, 4]
    assert torch.equal(attend_and_check(), out)


def test_scores_beyond_32_bits():
    """Rows of scores that lie 2^31 numbers apart, filtered in place."""
    V, stride = 1000, 1 << 31
    buf = torch.empty(2 * stride + V, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((3, V), (stride, 1))
    g = torch.Generator().manual_seed(1)
    scores = (torch.randn((3, V), generator=g) * 3).bfloat16()
    x.copy_(scores)
    r = [0.1, 0.5, 0.9]
    k = ints([7, 0, 3])
    tokens, _ = binding.sample(x, torch.tensor(r, device=DEV), top_k=k, filtered=x)
    for m in range(3):
        token, _, ids = draw(scores[m].double().numpy(), float(np.float32(r[m])), top_k=int(k[m]))
        kept = np.full(V, -np.inf)
        kept[ids] = scores[m].double().numpy()[ids]
        assert int(tokens[m]) == token and np.array_equal(x[m].double().cpu().numpy(), kept)
