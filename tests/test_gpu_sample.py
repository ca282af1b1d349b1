"""Filtered sampling against its definition in 64 bits, row by row on the host."""
import math

import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}


def draw(x, r, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, its log-probability, kept ids) of scores x (64 bits)."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return 0, -np.inf, np.array([], dtype=int)
    order = np.argsort(-x, kind="stable")
    if temperature == 0:
        return int(order[0]), 0.0, order[:1]
    with np.errstate(invalid="ignore"):
        w = np.where(x == top, 1.0, 0.0) if np.isinf(top) else np.exp((x - top) / temperature)
    w = w[order]
    n = min(top_k, len(w)) if top_k > 0 else len(w)
    if top_p < 1:
        total = math.fsum(w[:n])
        front, kept = 0.0, 0
        c = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])
        kept = int((c < top_p * total).sum())
        n = min(n, max(kept, 1))
    n = int((w[:n] >= min(min_p, 1.0)).sum()) if min_p > 0 else n
    ids = np.sort(order[:n])
    rank = np.empty(len(w), dtype=int)
    rank[order] = np.arange(len(w))
    wi = w[rank[ids]]
    c = np.cumsum(wi)
    i = int(np.searchsorted(c, r * c[-1], side="right"))
    i = min(i, int(np.nonzero(wi)[0][-1]))
    return int(ids[i]), math.log(wi[i] / c[-1]), ids


def check(scores, r, filtered=True, **params):
    """scores [M, V] (torch, on the CPU); params: lists of M numbers.  Compares tokens, log-probabilities and what is left."""
    M, V = scores.shape
    dev = scores.to(DEV)
    t = {n: torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV) for n, v in params.items()}
    rt = torch.tensor(r, dtype=torch.float32)
    out = torch.full_like(dev, 7.0) if filtered else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tokens, logp = binding.sample(dev, rt.to(DEV), t.get("temperature"), t.get("top_k"), t.get("top_p"), t.get("min_p"), filtered=out, status_t=status)
    tokens, logp = tokens.cpu().numpy(), logp.cpu().numpy()
    assert int(status.item()) == 0
    x = scores.double().numpy()
    for m in range(M):
        p = {n: float(t[n][m]) if n != "top_k" else int(t[n][m]) for n in t}
        token, lp, ids = draw(x[m], float(rt[m]), **p)
        assert tokens[m] == token, (m, tokens[m], token, p)
        # one rounding of a number that is worked out in 64 bits, from a sum that is off by 2^-22 of itself at most
        assert logp[m] == lp or abs(logp[m] - lp) <= 2 ** -24 * abs(lp) + 2 ** -22
        if filtered:
            got = out[m].float().cpu().numpy()
            want = np.full(V, -np.inf)
            want[ids] = np.where(np.isnan(x[m][ids]), -np.inf, x[m][ids])
            assert np.array_equal(got, want), (m, np.nonzero(got != want)[0][:5], p)
    return tokens


def logits(M, V, dtype, seed, peaks=True, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, V), generator=g) * spread
    if peaks:
        x.scatter_add_(1, torch.randint(0, V, (M, 3), generator=g), torch.tensor([[9.0, 8.0, 7.0]]).expand(M, 3))
    return x.to(TORCH[dtype])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 1000, 2048, 2049, 4097, 32000, 50265])
def test_all_filters_at_all_sizes(dtype, V):
    M = 24
    r = np.random.default_rng(V).random(M).astype(np.float32)
    pick = lambda values, shift=0: [values[(m + shift) % len(values)] for m in range(M)]
    params = dict(temperature=pick([1.0, 0.7, 1.9, 0.3, 5.0]), top_k=pick([0, 50, 1, 7, V, V - 1, V + 5, -3, 1000]), top_p=pick([1.0, 0.9, 0.5, 0.99, 0.0, 0.2, 2.0]),
                  min_p=pick([0.0, 0.05, 0.0, 0.001, 1.0, -1.0, 0.3, 7.0], 2))
    check(logits(M, V, dtype, V), r, **params)
    check(logits(M, V, dtype, V + 1, peaks=False), r, filtered=False, **{n: params[n] for n in ("temperature", "top_p")})
    check(logits(M, V, dtype, V + 2), r, **{n: params[n] for n in ("top_k",)})
    check(logits(M, V, dtype, V + 3), r, **{n: params[n] for n in ("temperature", "min_p")})
    check(logits(M, V, dtype, V + 4), r)


@pytest.mark.parametrize("dtype,V", [("fp32", 131072), ("fp32", 400001), ("fp32", 1 << 20), ("bf16", 131073), ("bf16", 1 << 20)])
@pytest.mark.parametrize("M", [2, 40])
def test_vocabularies_beyond_shared_memory(dtype, V, M):
    if M == 40 and V == 1 << 20:
        M = 38
    r = np.random.default_rng(V).random(M).astype(np.float32)
    pick = lambda values: [values[m % len(values)] for m in range(M)]
    check(logits(M, V, dtype, 1), r, temperature=pick([0.8, 1.2]), top_k=pick([0, 0, 100, 200000]), top_p=pick([0.95, 0.9, 1.0]), min_p=pick([0.0, 0.0, 0.0, 0.0, 0.01]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_ties_go_to_the_lowest_ids(dtype):
    """Scores of few values, whole rows of one value, and the two zeros, which are the same score."""
    M, V = 30, 3000
    g = torch.Generator().manual_seed(3)
    x = torch.randint(-2, 3, (M, V), generator=g).float()
    x[3:6] = 1.5
    x[6:9] = torch.where(torch.rand((3, V), generator=g) < 0.5, 0.0, -0.0)
    x[9] = -0.0
    r = np.random.default_rng(1).random(M).astype(np.float32)
    pick = lambda values: [values[m % len(values)] for m in range(M)]
    for params in (dict(top_k=pick([1, 5, 700, 1234, 2999])), dict(top_p=pick([0.5, 0.25, 0.9, 0.03])), dict(top_k=pick([900, 1000, 100]), top_p=pick([0.5, 0.75])),
                   dict(top_k=pick([900, 1000, 100]), top_p=pick([0.5, 0.75]), min_p=pick([0.0, 0.2])), dict(min_p=pick([1.0, 0.5, 0.1]))):
        check(x.to(TORCH[dtype]), r, **params)


def test_borders_that_are_met_exactly():
    """Equal weights make all sums whole: a share that ends at an id does not take the next one, and r at a border goes on to it."""
    x = torch.zeros(6, 64)
    check(x, [0.5, 0.25, 0.0, 1 - 2 ** -24, 0.75, 0.5], top_p=[0.5, 0.25, 1 / 64, 1.0, 0.75, 0.515625])
    tokens = check(x, [0.0, 0.5, 0.25, 1 - 2 ** -24, 2 ** -6, 2 ** -6 - 2 ** -30])
    assert tokens.tolist() == [0, 32, 16, 63, 1, 0]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_infinities_and_nans(dtype):
    V = 700
    x = logits(12, V, dtype, 5)
    x[0, :] = -math.inf
    x[1, :] = math.nan
    x[2, ::2] = -math.inf
    x[3, ::3] = math.nan
    x[4, 17] = x[4, 300] = x[4, 301] = math.inf
    x[5, 17] = math.inf
    x[6, 1:] = -math.inf
    x[7, :-1] = math.nan
    x[8] = torch.finfo(x.dtype).max
    x[8, 5] = torch.finfo(x.dtype).min
    x[9] = x[9] * 1e30
    x[11] = torch.linspace(-1, 1, V) * 0.99 * torch.finfo(x.dtype).max
    x[10] = x[10] * 1e-38
    r = np.random.default_rng(1).random(12).astype(np.float32)
    for params in ({}, dict(top_k=[3] * 12), dict(top_k=[650] * 12, top_p=[0.8] * 12), dict(top_p=[0.5] * 12), dict(min_p=[0.5] * 12), dict(temperature=[0.0] * 12),
                   dict(temperature=[1e-30] * 12), dict(temperature=[1e30] * 12, top_p=[0.5] * 12), dict(temperature=[3e38] * 12, top_k=[5] * 12), dict(temperature=[3e38] * 12, top_p=[0.7] * 12),
                   dict(temperature=[3e38] * 12, min_p=[0.3] * 12), dict(temperature=[1e-42] * 12, top_p=[0.7] * 12)):
        check(x, r, **params)


def test_rows_whose_parameters_make_no_sense():
    """They latch an error and come back empty; the others are as ever."""
    x = logits(8, 900, "fp32", 2).to(DEV)
    ok = torch.full((8,), 0.5, device=DEV)
    for name, bad in (("temperature", -1.0), ("temperature", math.nan), ("temperature", math.inf), ("top_p", math.nan), ("min_p", math.nan), ("r_t", math.nan)):
        args = dict(r_t=ok.clone(), temperature=ok.clone(), top_p=ok.clone(), min_p=ok.clone() * 0.01)
        status, out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros_like(x)
        want, want_lp = binding.sample(x, filtered=out, **args)
        kept = out.clone()
        args[name][3] = bad
        tokens, lp = binding.sample(x, filtered=out, status_t=status, **args)
        assert int(status.item()) == binding.AD_ERR_ARG
        assert int(tokens[3]) == -1 and float(lp[3]) == -math.inf and bool((out[3] == -math.inf).all())
        rest = [m for m in range(8) if m != 3]
        assert torch.equal(tokens[rest], want[rest]) and torch.equal(lp[rest], want_lp[rest]) and torch.equal(out[rest], kept[rest])


@pytest.mark.parametrize("dtype,V", [("fp32", 1000), ("bf16", 50265), ("fp32", 500000)])
def test_in_place_and_strided(dtype, V):
    """What is left over the scores themselves; rows inside wider arrays, at any alignment."""
    M = 5
    wide = logits(M, V + 13, dtype, 9).to(DEV)
    r = torch.rand(M, generator=torch.Generator().manual_seed(1)).to(DEV)
    k, p = torch.tensor([0, 40, 3, 0, 77], dtype=torch.int32, device=DEV), torch.tensor([0.9, 1.0, 0.5, 0.3, 0.95], device=DEV)
    for shift in (0, 1, 13):
        x = wide[:, shift: shift + V].contiguous()
        out = torch.empty_like(x)
        tokens, lp = binding.sample(x, r, top_k=k, top_p=p, filtered=out)
        view = wide.clone()[:, shift: shift + V]
        t2, lp2 = binding.sample(view, r, top_k=k, top_p=p, filtered=view)
        assert torch.equal(tokens, t2) and torch.equal(lp, lp2) and torch.equal(out, view.contiguous())
        target = torch.zeros((M, V + 5), dtype=x.dtype, device=DEV)
        binding.sample(x, r, top_k=k, top_p=p, filtered=target[:, 3: 3 + V])
        assert torch.equal(target[:, 3: 3 + V], out) and bool((target[:, :3] == 0).all()) and bool((target[:, 3 + V:] == 0).all())
        assert torch.equal(tokens, binding.sample(x, r, top_k=k, top_p=p)[0])


def test_many_rows_and_none():
    x = logits(3000, 501, "bf16", 4)
    r = np.random.default_rng(2).random(3000).astype(np.float32)
    check(x, r, top_k=[(m * 7) % 90 for m in range(3000)], top_p=[0.1 + 0.3 * (m % 4) for m in range(3000)])
    tokens, lp = binding.sample(x.to(DEV)[:0], torch.empty(0, device=DEV))
    assert tokens.shape == (0,) and lp.shape == (0,)


def test_distribution_of_many_draws():
    """As many draws as numbers at even distances: each token as often as its share says, to one."""
    V, n = 40, 4096
    x = logits(1, V, "fp32", 8).expand(n, V).contiguous()
    r = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tokens = check(x, r, filtered=False, top_k=[12] * n, temperature=[0.9] * n)
    _, _, ids = draw(x[0].double().numpy(), 0.5, np.float32(0.9), 12)
    w = np.exp(x[0].double().numpy()[ids] / float(np.float32(0.9)))
    assert np.abs(np.bincount(tokens, minlength=V)[ids] - w / w.sum() * n).max() <= 1.0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_replayed_from_a_graph_and_on_two_streams(dtype):
    a, b = logits(6, 32000, dtype, 1).to(DEV), logits(40, 9000, dtype, 2).to(DEV)
    ra, rb = torch.rand(6, device=DEV), torch.rand(40, device=DEV)
    p = torch.full((40,), 0.9, device=DEV)
    want = [*binding.sample(a, ra, top_p=p[:6].contiguous()), *binding.sample(b, rb, top_p=p)]
    pa = p[:6].contiguous()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(s1):
            x = binding.sample(a, ra, top_p=pa)
        with torch.cuda.stream(s2):
            y = binding.sample(b, rb, top_p=p)
        torch.cuda.synchronize()
        assert all(torch.equal(i, j) for i, j in zip(want, [*x, *y]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x, y = binding.sample(a, ra, top_p=pa), binding.sample(b, rb, top_p=p)
    ra.fill_(0.25)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x[0], binding.sample(a, ra, top_p=pa)[0]) and torch.equal(y[0], want[2])


def test_truncated_distributions_are_verified_like_any_others():
    """Drafter and verifier truncated by their own filters: drafts drawn from the one, accepted against the other, come out with the verifier's kept ids only, as the
    decisions on the truncated scores in 64 bits have it."""
    from tests.test_gpu_accept_sampled import accept
    B, k, V = 6, 4, 1200
    g = torch.Generator().manual_seed(11)
    target = logits(B * k, V, "fp32", 21)
    drafter = target + torch.randn((B * k, V), generator=g) * 0.7
    temperature = torch.full((B * k,), 0.9, device=DEV)
    top_p, top_k = torch.full((B * k,), 0.8, device=DEV), torch.full((B * k,), 30, dtype=torch.int32, device=DEV)
    left = [torch.empty((B * k, V), device=DEV) for _ in range(2)]
    r = torch.rand(B * k, generator=g).to(DEV)
    drafts, _ = binding.sample(drafter.to(DEV), r, temperature, top_k, top_p, filtered=left[1])
    binding.sample(target.to(DEV), r, temperature, top_k, top_p, filtered=left[0])
    off = torch.arange(0, B * k + 1, k, dtype=torch.int32, device=DEV)
    u, rr = torch.rand((B, k), generator=g), torch.rand(B, generator=g)
    ids, n = binding.accept_sampled(left[0], left[1], drafts.view(B, k), off, u.to(DEV), rr.to(DEV), temperature=0.9)
    t2, n2 = accept(left[0].double().cpu().numpy(), left[1].double().cpu().numpy(), drafts.view(B, k).cpu().numpy(), off.tolist(), u.numpy(), rr.numpy(),
                    float(np.float32(0.9)))
    assert np.array_equal(ids.cpu().numpy(), t2) and np.array_equal(n.cpu().numpy(), n2)
    kept = torch.isfinite(left[0]).view(B, k, V).cpu().numpy()
    for b in range(B):
        for i in range(int(n[b])):
            assert kept[b, i, int(ids[b, i])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [40001, 131073])
def test_long_rows_of_all_kinds(dtype, V):
    """Rows whose weights are looked up by number: magnitudes far apart, borders among numbers too small for a bin, zeros of both signs, few numbers with thousands of ties each, scores
    below zero only, one infinity and many, masked ids, temperatures that make all of them alike or leave one."""
    g = torch.Generator().manual_seed(V)
    x = torch.randn((12, V), generator=g)
    x[1] *= 1e-4                                                # (all of it small, beside one larger number)
    x[1, 77] = 4.0
    x[2] = x[2].sign() * 0.0
    x[2, ::9] = -1.0
    x[3] = (x[3] * 2).round()                                  # (a dozen numbers)
    x[4] = -x[4].abs() * 3 - 100
    x[5, 1000] = float("inf")
    x[6, ::1000] = float("inf")
    x[7, torch.rand(V, generator=g) < 0.9] = float("-inf")
    x[8] *= torch.exp(torch.randn(V, generator=g) * 4)         # (many octaves)
    x[9] = torch.where(x[9] > 0, 1e-30, -1e-30) * x[9].abs()
    x[10, 5:] = float("-inf")
    x[11] = x[11].clamp(-0.01, 0.01)
    r = np.random.default_rng(V)
    for temperature in (0.7, 30.0, 1e5, 1e37, 1e-3):
        for k, p, least in ((0, 1.0, 0.0), (0, 0.83, 0.0), (V // 3, 1.0, 0.0), (V // 2, 0.71, 0.0), (40, 0.6, 0.0), (0, 0.9, 0.3), (0, 1.0, 0.2)):
            check(x.to(TORCH[dtype]), r.random(12), temperature=[temperature] * 12, top_k=[k] * 12, top_p=[p] * 12, min_p=[least] * 12)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,gap,swap", [(1000, 0, False), (1003, 5, False), (1003, 1, True), (40001, 3, True)])
def test_what_is_left_between_the_rows_of_scores(dtype, V, gap, swap):
    """Scores and what is left as two column ranges of one wide array, next to each other or apart, in either order: neither touches the other, nor what lies beside them."""
    M, g = 5, torch.Generator().manual_seed(V)
    wide = torch.full((M, 2 * V + gap + 7), 3.5, dtype=TORCH[dtype], device=DEV)
    first, second = wide[:, 2: 2 + V], wide[:, 2 + V + gap: 2 + 2 * V + gap]
    scores, out = (second, first) if swap else (first, second)
    x = logits(M, V, dtype, V)
    scores.copy_(x)
    r, k = torch.rand(M, generator=g).to(DEV), torch.tensor([0, 5, 1, 300, V], dtype=torch.int32, device=DEV)
    p = torch.tensor([0.9, 1.0, 0.5, 0.99, 0.2], device=DEV)
    tokens, logp = binding.sample(scores, r, top_k=k, top_p=p, filtered=out)
    want = torch.empty_like(x, device=DEV)
    alone = binding.sample(x.to(DEV), r, top_k=k, top_p=p, filtered=want)
    assert torch.equal(tokens, alone[0]) and torch.equal(logp, alone[1]) and torch.equal(out, want)
    assert torch.equal(scores.cpu(), x) and bool((wide[:, :2] == 3.5).all()) and bool((wide[:, 2 + V: 2 + V + gap] == 3.5).all()) and bool((wide[:, 2 + 2 * V + gap:] == 3.5).all())
    with pytest.raises(binding.AdError, match="overlap"):
        binding.sample(scores, r, top_k=k, filtered=wide[:, 3: 3 + V] if not swap else wide[:, 1 + V + gap: 1 + 2 * V + gap])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [700, 3000, 4096, 9001, 32000, 50265, 128000])
def test_a_row_is_drawn_alike_in_batches_of_any_size(dtype, V):
    """The same rows alone, among few and among many, which one, two, four or eight CTAs take together: the same tokens, log-probabilities and scores left, bit by bit."""
    rows, g = 6, torch.Generator().manual_seed(V)
    x = logits(rows, V, dtype, V)
    x[1] = (x[1].float() * 4).round().div(4).to(x.dtype)         # many ties
    x[2, ::3] = -math.inf
    r = torch.rand(rows, generator=g)
    t = dict(temperature=torch.tensor([1.0, 0.7, 1.3, 2.0, 0.5, 1.0]), top_k=torch.tensor([0, 40, 0, 300, V // 2, 0], dtype=torch.int32),
             top_p=torch.tensor([0.9, 0.95, 0.5, 0.99, 1.0, 1.0]), min_p=torch.tensor([0.0, 0.0, 0.01, 0.0, 0.001, 0.0]))
    want = None
    for M in (6, 30, 60, 150, 300, 600):
        if M * V > 40_000_000:
            continue
        many = lambda y: y.repeat((M // rows,) + (1,) * (y.dim() - 1)).to(DEV)
        scores = many(x)
        left = torch.empty_like(scores)
        tokens, logp = binding.sample(scores, many(r), **{n: many(y) for n, y in t.items()}, filtered=left)
        got = (tokens.view(-1, rows), logp.view(-1, rows), left.view(-1, rows, V))
        if want is None:
            want = [y[0].clone() for y in got]
            for m in range(rows):
                token, lp, ids = draw(x[m].double().numpy(), float(r[m]), **{n: y[m].item() for n, y in t.items()})
                kept = np.full(V, -np.inf)
                kept[ids] = x[m].double().numpy()[ids]
                assert int(want[0][m]) == token and np.array_equal(want[2][m].double().cpu().numpy(), kept)
        assert all(bool((y == w).all()) for y, w in zip(got, want)), M


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [5, 5000, 50000])
def test_min_p_of_one_leaves_what_ties_with_the_largest(dtype, V):
    """Scores a step or some below the largest, at temperatures that leave all of them a weight of one in 64 bits: none of them ties with it."""
    x = torch.full((6, V), 1.0).to(TORCH[dtype])
    step = torch.finfo(TORCH[dtype]).eps / 2                    # what numbers below one are apart: 24 and 8 bits
    for i, below in enumerate((1, 2, 3)):
        x[:, i] = 1.0 - below * step
    x[:, 4:] = 0.5
    x[3:, 0] = 1.0
    t = torch.tensor([1.0, 1e12, 1e30] * 2, device=DEV)
    for p in (1.0, 5.0):
        left, scores = torch.empty_like(x, device=DEV), x.to(DEV)
        tokens, logp = binding.sample(scores, torch.full((6,), 0.75, device=DEV), temperature=t, min_p=torch.full((6,), p, device=DEV), filtered=left)
        want = torch.where(x == 1, x, torch.full_like(x, -math.inf))
        assert torch.equal(left.cpu(), want) and tokens.tolist() == [3] * 6
        # (of one kept id, or of two that tie)
        assert torch.allclose(logp.cpu(), torch.tensor([0.0] * 3 + [-math.log(2.0)] * 3), atol=2 ** -22)
