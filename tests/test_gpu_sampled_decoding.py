"""The cache and the sampled verification as a program uses them: a decoder layer built from operator-level calls that drafts, verifies and rolls back,
and the library's own models sampled from through a handle."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding, synth
from tests.test_gpu_accept_sampled import accept
from tests.test_gpu_kv_cache import DEV, Model, bound, ints, offsets, shuffled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,fmt,heads,group,dim,block", [("bf16", "e4m3", 4, 1, 64, 32), ("bf16", "int8", 1, 4, 128, 64), ("fp32", "int8", 2, 2, 32, 16)])
def test_a_decoder_that_drafts_verifies_and_rolls_back(dtype, fmt, heads, group, dim, block):
    """Per step: projections of the block's tokens, append, attention over prefix and block, scores, acceptance of random drafts; what is rejected is
    given up by a shorter length and overwritten.  Cache and attention against the definition in 64 bits at every step, decisions on the same scores."""
    B, V, kmax, row_blocks = 3, 500, 9, 8
    d, H = heads * group * dim, heads * group
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(dim)
    emb = (torch.randn((V, d), generator=g)).to(dt).to(DEV)
    wqkv = (torch.randn((H * dim + 2 * heads * dim, d), generator=g) * d ** -0.5).to(dt).to(DEV)
    table, n_blocks = shuffled(B, row_blocks, 1)
    cache = binding.KvCache(n_blocks, heads, dim, block, fmt, table=ints(table), row_blocks=row_blocks, device=DEV)
    model = Model(n_blocks, heads, dim, block, fmt, table, row_blocks)
    lens, last = [0, 0, 0], [3, 4, 5]
    r = np.random.default_rng(7)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    accepted = 0
    for step in range(8):
        new = [int(x) for x in r.integers(1, kmax + 1, B)]
        if step == 5:
            new[1] = 0
        off, M = offsets(new), sum(new)
        drafts = np.full((B, kmax), -1)
        for b in range(B):
            drafts[b, : new[b]] = r.integers(0, V, new[b])
        tokens = np.concatenate([[last[b]] + list(drafts[b, : new[b] - 1]) for b in range(B) if new[b]])
        x = emb[torch.tensor(tokens, device=DEV)]
        qkv = binding.linear(x, wqkv, None, status).to(dt)
        q = qkv[:, : H * dim].view(M, H, dim)
        k, v = qkv[:, H * dim: H * dim + heads * dim].view(M, heads, dim), qkv[:, H * dim + heads * dim:].view(M, heads, dim)
        o_t, l_t = ints(off), ints(lens)
        binding.cache_append(cache, k, v, o_t, l_t, max_new=kmax, status_t=status)
        att = binding.cache_attention(cache, q, o_t, l_t, max_new=kmax, max_keys=row_blocks * block, status_t=status)
        scores = binding.linear(att.reshape(M, d), emb, None, status) * 2.0
        u, rr = r.random((B, kmax), dtype=np.float32), r.random(B, dtype=np.float32)
        ids, n = binding.accept_sampled(scores, None, ints(drafts), o_t, torch.tensor(u, device=DEV), torch.tensor(rr, device=DEV), temperature=1.5,
                                        status_t=status)
        ids, n = ids.cpu().numpy(), n.cpu().numpy()
        # the definition, step by step
        model.append(k.double().cpu().numpy(), v.double().cpu().numpy(), off, lens)
        want, weight, size, floor = model.attend(q.double().cpu().numpy(), off, lens, True, dim ** -0.5)
        err = np.abs(att.double().cpu().numpy() - want)
        assert (err <= bound(dtype, want, weight, size, floor, row_blocks * block, dim)).all()
        t2, n2 = accept(scores.double().cpu().numpy(), None, drafts, off, u, rr, 1.5)
        assert np.array_equal(ids, t2) and np.array_equal(n, n2)
        for b in range(B):
            lens[b] += int(n[b])
            if n[b]:
                last[b] = int(ids[b, n[b] - 1])
        accepted += int(n.sum())
    assert int(status.item()) == 0 and accepted >= 8


def test_sampling_through_a_handle_follows_greedy_decoding_as_the_temperature_falls():
    """Draft, verify, accept from random numbers, commit: at a temperature that leaves one token its output is greedy decoding's, whatever the random
    numbers, and at an ordinary one the tokens are the decisions' on the handle's own scores."""
    w, wn = synth.make_weights(synth.TINY, 0), synth.make_weights(synth.TINY, 1)
    wl = synth.WORKLOADS[1]
    src, src_len = synth.make_sources(wl)
    dec = binding.AggressiveDecoder(synth.TINY, w, wn, max_batch=1, max_src=16, max_tgt=24, kmax=6)
    greedy, _ = dec.generate(src, src_len, mode="IAD", k=1, max_len=[24])
    V = synth.TINY.vocab
    r = np.random.default_rng(5)
    for temperature in (1e-5, 1.0):
        dec.encode(src, src_len)
        out = []
        for _ in range(24):
            ln, _, fin = dec.state()
            if fin[0] or ln[0] >= 24:
                break
            drafts, k = dec.draft_block(5)
            drafter = torch.tensor(dec.debug_logits(int(k[0]), which=1), device=DEV)
            dec.verify_block(drafts, k)
            scores = torch.tensor(dec.debug_logits(int(k[0])), device=DEV)
            u, rr = r.random((1, 6), dtype=np.float32), r.random(1, dtype=np.float32)
            # (the drafter's choice is its best token, not a sample: its own probability is one)
            ids, n = binding.accept_sampled(scores, None, ints(drafts), ints([0, int(k[0])]), torch.tensor(u, device=DEV), torch.tensor(rr, device=DEV),
                                            temperature=temperature, eos=synth.EOS)
            ids, n = ids.cpu().numpy(), n.cpu().numpy()
            want = accept(scores.double().cpu().numpy(), None, drafts, [0, int(k[0])], u, rr, float(np.float32(temperature)), synth.EOS)
            assert np.array_equal(ids, want[0]) and np.array_equal(n, want[1])
            assert drafter.shape == scores.shape == (int(k[0]), V)
            dec.force_commit(ids, n)
            out += [int(x) for x in ids[0, : n[0]]]
        if temperature < 1e-3:
            assert out[: len(greedy[0])] == [int(x) for x in greedy[0]]
        else:
            assert len(out) >= 1 and all(0 <= x < V for x in out)
    dec.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_calls_that_overlap_on_two_streams(dtype):
    """Attention over one cache and sampled verification, on two streams at once and again and again: what each gives alone."""
    heads, dim, block, n = 4, 64, 32, 3000
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(3)
    cache = binding.KvCache(2 * (n // block + 1), heads, dim, block, "int8", row_blocks=n // block + 1, device=DEV)
    k = torch.randn((2 * n, heads, dim), generator=g).to(dt).to(DEV)
    binding.cache_append(cache, k, k.flip(0), ints([0, n, 2 * n]), ints([0, 0]), n)
    work = []
    for new in (1, 9):
        q = torch.randn((2 * new, heads * 2, dim), generator=g).to(dt).to(DEV)
        scores = (torch.randn((2 * new, 9000), generator=g) * 3).to(dt).to(DEV)
        drafts = scores.argmax(1).view(2, new).int()
        u, r = torch.rand((2, new), generator=g).to(DEV), torch.rand(2, generator=g).to(DEV)
        off, lens = ints([0, new, 2 * new]), ints([n - new, n - 40 * new])
        work.append(lambda q=q, s=scores, d=drafts, u=u, r=r, o=off, l=lens, m=new: (binding.cache_attention(cache, q, o, l, m, n),
                                                                                     *binding.accept_sampled(s, s.flip(0).contiguous(), d, o, u, r)))
    alone = [f() for f in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[], []]
    for _ in range(20):
        for i, (f, s) in enumerate(zip(work, streams)):
            with torch.cuda.stream(s):
                got[i].append(f())
    torch.cuda.synchronize()
    for want, results in zip(alone, got):
        assert all(torch.equal(a, b) for res in results for a, b in zip(want, res))
