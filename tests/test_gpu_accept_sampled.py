"""Sampled verification against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2205_10350_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}


def probabilities(scores, temperature):
    """softmax in 64 bits; a NaN counts as -inf, +inf share everything, nothing at all stays nothing."""
    x = np.where(np.isnan(scores), -np.inf, scores.astype(np.float64))
    top = x.max()
    if top == -np.inf:
        return np.zeros(x.shape)
    with np.errstate(invalid="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / temperature) if np.isfinite(top) else 0.0)
    return w / w.sum()


def accept(target, draft, drafts, off, u, r, temperature, eos=-1):
    B, kmax = drafts.shape
    tokens, counts = np.full((B, kmax), -1), []
    for b in range(B):
        n = 0
        for i in range(off[b + 1] - off[b]):
            d = drafts[b, i]
            d = d if 0 <= d < target.shape[1] else -1
            p = probabilities(target[off[b] + i], temperature)
            if draft is not None:
                q = probabilities(draft[off[b] + i], temperature)
            else:
                q = np.zeros(p.shape)
                q[d] = 1.0
            n += 1
            if d >= 0 and float(u[b, i]) * q[d] < p[d]:
                tokens[b, i] = d
                if d == eos:
                    break
                continue
            rest = np.maximum(p - q, 0) if d >= 0 else p
            if rest.sum() == 0:
                rest = p
            run = np.cumsum(rest)
            hit = np.nonzero(run > float(r[b]) * run[-1])[0]
            alive = np.nonzero(rest > 0)[0]
            tokens[b, i] = hit[0] if len(hit) else (alive[-1] if len(alive) else 0)
            break
        counts.append(n)
    return tokens, np.array(counts)


def problem(new, V, dtype, seed, drafter=True, temperature=1.0, agree=0.5):
    """Scores with a few likely tokens, a drafter that mostly agrees and drafts drawn from it (or the likeliest token of the verifier)."""
    g = np.random.default_rng(seed)
    M, kmax = sum(new), max(max(new), 1)
    target = g.standard_normal((M, V)) * 2
    for m in range(M):
        target[m, g.integers(0, V, 3)] += (9, 8, 7)
    target = torch.tensor(target, dtype=torch.float32).to(TORCH[dtype])
    draft, drafts, off, at = None, np.full((len(new), kmax), -1), [0], 0
    if drafter:
        draft = (target.float() + torch.tensor(g.standard_normal((M, V)) * agree, dtype=torch.float32)).to(TORCH[dtype])
    for b, n in enumerate(new):
        for i in range(n):
            if drafter:
                q = probabilities(draft[at + i].double().numpy(), temperature)
                drafts[b, i] = g.choice(V, p=q)
            else:
                drafts[b, i] = int(target[at + i].float().argmax()) if g.random() < 0.9 else -1
        at += n
        off.append(at)
    return target, draft, drafts, off, g.random((len(new), kmax), dtype=np.float32), g.random(len(new), dtype=np.float32)


def run(target, draft, drafts, off, u, r, status=None, **kw):
    t = lambda a, dt: torch.tensor(np.asarray(a), dtype=dt, device=DEV)
    tokens, n = binding.accept_sampled(target.to(DEV), None if draft is None else draft.to(DEV), t(drafts, torch.int32), t(off, torch.int32),
                                       t(u, torch.float32), t(r, torch.float32), status_t=status, **kw)
    return tokens.cpu().numpy(), n.cpu().numpy()


def check(target, draft, drafts, off, u, r, temperature=1.0, eos=-1, code=0):
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = run(target, draft, drafts, off, u, r, status, temperature=temperature, eos=eos)
    want = accept(target.double().numpy(), None if draft is None else draft.double().numpy(), drafts, off, u, r, float(np.float32(temperature)), eos)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[0], want[0])
    assert int(status.item()) == code
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("V", [1, 2, 7, 257, 1000, 4097, 32000, 50265])
def test_ragged_batches(dtype, drafter, V):
    new = [1, 5, 0, 25, 2, 64] if V < 10000 else [3, 0, 12, 1]
    temperature = {257: 0.7, 4097: 1.9}.get(V, 1.0)
    n = check(*problem(new, V, dtype, V, drafter, temperature), temperature=temperature)[1]
    assert n[new.index(0)] == 0


@pytest.mark.parametrize("dtype,drafter,V", [("bf16", True, 120001), ("fp32", False, 230000)])
def test_vocabularies_whose_weights_do_not_stay_in_shared_memory(dtype, drafter, V):
    check(*problem([3, 1, 2], V, dtype, 51, drafter))


def test_more_rows_than_clusters_of_eight():
    """Clusters of four CTAs, and of one where the vocabulary is small."""
    for V in (7000, 900):
        check(*problem([2, 1, 3, 0] * 12, V, "bf16", 53, True, 0.9), temperature=0.9)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [31, 5003])
def test_plain_sampling_follows_the_inverse_distribution(dtype, V):
    """A single negative slot a row: the token at which the running sum of probabilities passes r."""
    B = 40
    target, _, _, off, u, r = problem([1] * B, V, dtype, 3, False)
    r[:4] = 0.0, 1.0 - 2.0 ** -24, 0.5, 2.0 ** -24
    tokens, n = check(target, None, np.full((B, 1), -1), off, u, r)
    assert (n == 1).all() and (tokens >= 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_equal_distributions_keep_every_draft(dtype):
    """p = q: whatever u < 1 says, nothing is rejected, however the sums round."""
    new, V = [30, 17], 9001
    target, _, drafts, off, u, r = problem(new, V, dtype, 5, True, 1.3)
    u[:] = np.float32(1.0 - 2.0 ** -24)
    drafts = np.random.default_rng(1).integers(0, V, drafts.shape)
    tokens, n = check(target, target.clone(), drafts, off, u, r, temperature=1.3)
    assert list(n) == new


def test_random_numbers_at_the_border_of_a_decision():
    """u one step of its type to either side of p / q, position after position: 32-bit sums could not tell."""
    V, n = 3000, 24
    target, draft, drafts, off, u, r = problem([n] * 6, V, "fp32", 7, True, 1.0, 1.5)
    for b in range(6):
        for i in range(n):
            p, q = (probabilities(x[off[b] + i].double().numpy(), 1.0)[drafts[b, i]] for x in (target, draft))
            edge = np.float32(min(p / q, 1.0))
            for _ in range(3):                                # below the border, so that the row goes on; the last position beyond it
                if not float(edge) * q < p:
                    edge = np.nextafter(edge, np.float32(0))
            u[b, i] = edge if i < n - 1 or edge >= 1 - 2e-7 else np.nextafter(np.nextafter(edge, np.float32(2)), np.float32(2))
    check(target, draft, drafts, off, u, r)


def test_random_numbers_at_the_borders_of_the_draw():
    """r next to the running sum at some token, on either side."""
    V, B = 2000, 64
    target, _, _, off, u, r = problem([1] * B, V, "fp32", 11, False)
    g = np.random.default_rng(2)
    for b in range(B):
        run_sum = np.cumsum(probabilities(target[b].double().numpy(), 1.0))
        edge = np.float32(run_sum[g.integers(0, V - 1)] / run_sum[-1])
        r[b] = min(np.nextafter(edge, np.float32(b % 2 * 2)), np.float32(1 - 2.0 ** -24))
    check(target, None, np.full((B, 1), -1), off, u, r)


@pytest.mark.parametrize("drafter", [True, False])
def test_accepted_eos_ends_the_output(drafter):
    target, draft, drafts, off, u, r = problem([12, 12, 12], 500, "fp32", 13, drafter, 1.0, 0.05)
    for m in range(36):
        target[m, 2] += 9.0
        if drafter:
            draft[m, 2] += 9.0
    drafts[0, 5], drafts[1, 0], drafts[2, 11] = 2, 2, 2
    u[:] = 0.0
    for b in range(3):                                        # drafts that the verifier finds possible
        for i in range(12):
            if drafts[b, i] != 2:
                drafts[b, i] = int(target[off[b] + i].argmax())
    tokens, n = check(target, draft, drafts, off, u, r, eos=2)
    assert n[1] == 1 and n[0] <= 6


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("drafter", [True, False])
def test_scores_that_are_not_finite(dtype, drafter):
    """Masked tokens (-inf and the type's lowest value), whole rows of them, +inf, NaN: as in the definition."""
    V, B = 700, 12
    target, draft, drafts, off, u, r = problem([2] * B, V, dtype, 17, drafter)
    low = float(torch.finfo(TORCH[dtype]).min)
    target[0, 100:] = -np.inf
    target[2, 1:] = low
    target[4] = -np.inf                                       # nothing is possible: id 0
    target[6, 33] = np.inf
    target[8, 5], target[8, 600] = np.inf, np.inf
    target[10, ::2] = np.nan
    target[12] = np.nan
    target[14] = low
    if drafter:
        draft[1, 50:] = -np.inf
        draft[3] = -np.inf                                    # a drafter without a distribution
        draft[16, 9], draft[18, 3] = np.inf, np.nan
        draft[19] = np.nan
    drafts[3, 0], drafts[4, 0], drafts[8, 0] = 33, 600, 9
    tokens, n = check(target, draft, drafts, off, u, r)
    assert (n >= 1).all()
    drafts[:] = -1
    tokens, n = check(target, draft, drafts, off, u, r)
    assert tokens[2, 0] == 0 and tokens[6, 0] == 0


def test_drafts_and_rows_that_do_not_exist():
    target, draft, drafts, off, u, r = problem([3, 3, 3], 900, "bf16", 19)
    drafts[1, 0] = 900
    check(target, draft, drafts, off, u, r, code=binding.AD_ERR_ARG)
    drafts[1, 0], drafts[0, 0] = -7, -2147483648
    check(target, draft, drafts, off, u, r)
    for bad in ([0, 3, 7, 9], [0, 3, 2, 9], [0, 3, 6, 10], [0, -1, 6, 9]):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        tokens, n = run(target, draft, drafts, bad, u, r, status)
        assert int(status.item()) == binding.AD_ERR_ARG
        want = accept(target.double().numpy(), draft.double().numpy(), drafts, [0, 3, 3, 3], u, r, 1.0)
        if bad[:2] == [0, 3]:
            assert n[0] == want[1][0] and np.array_equal(tokens[0], want[0][0])
        for b in range(3):
            if bad[b] < 0 or not 0 <= bad[b + 1] - bad[b] <= 3 or bad[b + 1] > 9:
                assert n[b] == 0 and (tokens[b] == -1).all()


def test_random_numbers_outside_of_their_range():
    """r of one and more: the last token that has any weight; u of one and more rejects, below zero keeps what is possible."""
    target, draft, drafts, off, u, r = problem([2] * 6, 300, "fp32", 23)
    target[:, 250:] = -np.inf
    r[:] = 1.0, 5.0, 1.0, 0.5, 0.5, 0.5
    u[:] = 0.5
    u[:3], u[3:5, 0], u[5] = 2.0, 1.0, -1.0
    drafts[2] = -1
    check(target, draft, drafts, off, u, r)


@pytest.mark.parametrize("dtype,pad", [("fp32", 1), ("fp32", 3), ("bf16", 1), ("bf16", 5), ("bf16", 8)])
def test_rows_of_scores_at_any_alignment(dtype, pad):
    V = 6001
    target, draft, drafts, off, u, r = problem([4, 9], V, dtype, 29)
    wide = torch.full((13, V + pad + 7), float("nan"), dtype=TORCH[dtype])
    other = torch.full((13, V + pad), float("inf"), dtype=TORCH[dtype])
    wide[:, pad: pad + V], other[:, pad:] = target, draft
    want = run(target, draft, drafts, off, u, r)
    wide_d, other_d = wide.to(DEV), other.to(DEV)
    got = run(wide_d[:, pad: pad + V], other_d[:, pad:], drafts, off, u, r)
    assert all(np.array_equal(a, b) for a, b in zip(want, got))
    check(target, draft, drafts, off, u, r)


@pytest.mark.parametrize("drafter", [True, False])
def test_tokens_are_distributed_as_the_verifier_says(drafter):
    """20000 draws over a vocabulary of 6, first tokens counted: each share within six standard deviations of the verifier's probability, whatever
    the drafter thinks."""
    B, V = 20000, 6
    g = np.random.default_rng(31)
    p_scores, q_scores = np.array([1.0, 0.2, -0.5, 2.0, 0.0, -3.0], np.float32), np.array([2.0, 0.1, 1.0, -1.0, 0.5, -0.5], np.float32)
    q = probabilities(q_scores, 1.0)
    drafts = g.choice(V, size=(B, 1), p=q) if drafter else np.full((B, 1), 3)
    rows = lambda s: torch.tensor(s)[None].expand(B, V).contiguous()
    tokens, n = run(rows(p_scores), rows(q_scores) if drafter else None, drafts, np.arange(B + 1), g.random((B, 1), dtype=np.float32), g.random(B, dtype=np.float32))
    share = np.bincount(tokens[:, 0], minlength=V) / B
    p = probabilities(p_scores, 1.0)
    assert (n == 1).all() and (np.abs(share - p) <= 6 * np.sqrt(p * (1 - p) / B)).all()


def test_batches_without_any_draft():
    none = np.zeros((3, 4), np.int32)
    for M in (0, 5):
        tokens, n = run(torch.zeros((M, 100)), torch.zeros((M, 100)), none, [0, 0, 0, 0], np.zeros((3, 4)), np.zeros(3))
        assert (tokens == -1).all() and (n == 0).all()


def test_one_row_of_the_largest_vocabulary():
    target, _, drafts, off, u, r = problem([2], 1 << 20, "fp32", 61, False)
    check(target, None, drafts, off, u, r)


def test_captured_calls_and_other_streams():
    target, draft, drafts, off, u, r = problem([5, 9, 2], 7001, "bf16", 37)
    dev = [x.to(DEV) for x in (target, draft)] + [torch.tensor(np.asarray(x), dtype=dt, device=DEV) for x, dt in
                                                  ((drafts, torch.int32), (off, torch.int32), (u, torch.float32), (r, torch.float32))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = binding.accept_sampled(*dev)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens, n = binding.accept_sampled(*dev)
    g = np.random.default_rng(3)
    for rep in range(3):
        if rep:
            u, r = g.random(u.shape, dtype=np.float32), g.random(r.shape, dtype=np.float32)
            dev[4].copy_(torch.tensor(u)); dev[5].copy_(torch.tensor(r))
            graph.replay()
            first = (tokens, n)
        torch.cuda.synchronize()
        want = accept(target.double().numpy(), draft.double().numpy(), drafts, off, u, r, 1.0)
        assert np.array_equal(first[0].cpu().numpy(), want[0]) and np.array_equal(first[1].cpu().numpy(), want[1])


def test_calls_that_are_refused():
    target, draft, drafts, off, u, r = problem([2, 2], 50, "fp32", 41)
    a = dict(target_t=target.to(DEV), draft_t=draft.to(DEV), drafts_t=torch.tensor(drafts, dtype=torch.int32, device=DEV),
             off_t=torch.tensor(off, dtype=torch.int32, device=DEV), u_t=torch.tensor(u, device=DEV), r_t=torch.tensor(r, device=DEV))
    binding.accept_sampled(**a)
    for bad in (dict(target_t=target), dict(target_t=target.half().to(DEV)), dict(draft_t=draft.bfloat16().to(DEV)), dict(draft_t=draft[:, :40].to(DEV)),
                dict(drafts_t=a["drafts_t"].long()), dict(off_t=a["off_t"][:2]), dict(u_t=a["u_t"].double()), dict(u_t=a["u_t"][:, :1]), dict(r_t=a["r_t"][:1]),
                dict(temperature=0.0), dict(temperature=float("nan")), dict(target_t=a["target_t"].t()), dict(status_t=a["off_t"])):
        with pytest.raises(binding.AdError):
            binding.accept_sampled(**{**a, **bad})


# ---------------------------------------------------------------------------------------------------------
# ranges of scores and temperatures
# ---------------------------------------------------------------------------------------------------------
def sums_of_parts(target, draft, temperature):
    """(largest score, sum of exponentials) that a call leaves in its scratch for every part of every row of scores, [scores, M, parts, 2]."""
    lib = binding.load()
    M, V = target.shape
    z = 1 if draft is None else 2
    nbytes = lib.ad_accept_sampled_scratch_bytes(M, V, z - 1)
    dev = [None if x is None else x.to(DEV) for x in (target, draft)]
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=DEV)
    scratch = torch.full((nbytes // 4,), float("nan"), device=DEV)
    one, tokens, count = torch.zeros((1, M), device=DEV), i32(*[0] * M), i32(0)
    rc = lib.ad_accept_sampled(dev[0].data_ptr(), V, dev[1].data_ptr() if z == 2 else None, V, 1 if target.dtype is torch.bfloat16 else 0, temperature, V,
                               i32(0, M).data_ptr(), i32(*[0] * M).data_ptr(), M, 1, M, one.data_ptr(), one.data_ptr(), -1, tokens.data_ptr(),
                               count.data_ptr(), scratch.data_ptr(), nbytes, None, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    return scratch.view(z, M, -1, 2).cpu().double().numpy()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [3, 1000, 32000])
@pytest.mark.parametrize("shift,temperature", [(0.0, 1.0), (-100.0, 1.0), (-200.0, 0.7), (-3e4, 1.0), (-20.0, 0.01), (100.0, 0.05), (3e4, 1.0)])
def test_sums_are_finite_wherever_the_scores_lie(dtype, V, shift, temperature):
    """A row's maximum may lie anywhere: sums that are no numbers cost every position a sweep of its own."""
    g = torch.Generator().manual_seed(V)
    target, draft = ((torch.randn((3, V), generator=g) * 2 + shift).to(TORCH[dtype]) for _ in range(2))
    target[1, : V // 2] = -float("inf")
    stats = sums_of_parts(target, draft, temperature)
    assert np.isfinite(stats[..., 1]).all() and (stats[..., 1] >= 0).all()
    assert np.array_equal(stats[..., 0].max(2), torch.stack([target, draft]).double().amax(2).numpy())
    assert (stats[..., 1].max(2) > 0.1).all()
    check(*_drawn(target, draft, temperature, [3], V), temperature=temperature)


def _drawn(target, draft, temperature, new, seed):
    """The arguments of a call on these scores, with drafts drawn from the drafter (or the verifier)."""
    g = np.random.default_rng(seed)
    drafts, off = np.full((len(new), max(new)), -1), offsets_of(new)
    for b, n in enumerate(new):
        for i in range(n):
            drafts[b, i] = g.choice(target.shape[1], p=probabilities((target if draft is None else draft)[off[b] + i].double().numpy(), temperature))
    return target, draft, drafts, off, g.random(drafts.shape, dtype=np.float32), g.random(len(new), dtype=np.float32)


def offsets_of(new):
    return [0] + [int(x) for x in np.cumsum(new)]


def test_scores_far_below_zero_cost_no_more_than_others():
    """64 drafts that are all kept, where every one that 32 bits leave open would take a sweep over the vocabulary: scores around -200 within three
    times the time of scores around zero (sweeps one after the other would be twenty times it)."""
    V, n = 32000, 64
    target = problem([n], V, "fp32", 71, True)[0]
    args = [torch.tensor(np.asarray(a), dtype=dt, device=DEV) for a, dt in ((target.argmax(1)[None], torch.int32), ([0, n], torch.int32), (np.full((1, n), 0.1), torch.float32),
                                                                            ([0.5], torch.float32))]
    times = []
    for shift in (0.0, -200.0):
        t = (target + shift).to(DEV)
        best = 1e9
        for _ in range(8):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda._sleep(1000000)
            start.record()
            tokens, count = binding.accept_sampled(t, t, *args)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        assert int(count[0]) == n
        times.append(best)
    assert times[1] <= 3 * times[0], times


def test_scores_that_rise_over_a_large_vocabulary():
    """Every round and every part of a row moves the maximum, and random numbers lie next to the borders of decisions."""
    V, n = 1 << 20, 6
    g = np.random.default_rng(3)
    rise = torch.linspace(0, 9, V, dtype=torch.float64)
    target, draft = ((rise + 0.3 * torch.tensor(g.standard_normal((2 * n, V)))).float() for _ in range(2))
    drafts, u = g.integers(V - 2000, V, (2, n)), np.zeros((2, n), np.float32)
    for b in range(2):
        for i in range(n):
            p, q = (probabilities(x[b * n + i].double().numpy(), 1.0)[drafts[b, i]] for x in (target, draft))
            if p >= 0.999 * q:
                draft[b * n + i, drafts[b, i]] += float(np.log(p / q) + 0.5)
                q = probabilities(draft[b * n + i].double().numpy(), 1.0)[drafts[b, i]]
            edge = p / q * (1 + (-1e-5 if i < n - 1 else 1e-5))
            u[b, i] = edge
    tokens, count = check(target, draft, drafts, [0, n, 2 * n], u, g.random(2, dtype=np.float32))
    assert (count == n).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("temperature", [1e-6, 1e-8, 1e-9, 1e-10, 1e-20, 1e-30])
def test_temperatures_that_leave_next_to_one_token(dtype, drafter, temperature):
    """Scores over such a temperature lie beyond 2^24, 2^31 and FP32's range.  Tied best tokens, a step of the type between best and second, drafts on
    either, random numbers on both sides of the shares that ties leave."""
    V, n, B = 700, 3, 16
    g = np.random.default_rng(9)
    target = torch.tensor(g.standard_normal((B * n, V)), dtype=torch.float32).to(TORCH[dtype])
    drafts = np.zeros((B, n), np.int64)
    step = float(torch.finfo(TORCH[dtype]).eps)
    for b in range(B):
        for i in range(n):
            m, ids = b * n + i, g.permutation(V)[:3]
            top = float(torch.tensor(8 * (1 + g.random())).to(TORCH[dtype]))           # between 8 and 16: steps of 8 eps
            target[m, ids[0]] = top
            target[m, ids[1]] = top if b % 2 else top - 8 * step
            target[m, ids[2]] = top - 8 * step
            drafts[b, i] = ids[b // 2 % 3]
    draft = None
    if drafter:
        draft = target[:, torch.randperm(V, generator=torch.Generator().manual_seed(1))].clone()
        draft[::2] = target[::2]
    u = np.where(g.random((B, n)) < 0.5, 0.3, 0.7).astype(np.float32)
    check(target, draft, drafts, offsets_of([n] * B), u, g.random(B, dtype=np.float32), temperature=temperature)


@pytest.mark.parametrize("dtype,drafter,V", [("bf16", True, 60000), ("fp32", True, 60000), ("fp32", False, 110000)])
def test_many_rows_whose_weights_do_not_stay_in_shared_memory(dtype, drafter, V):
    """Clusters of four CTAs, which keep weights of half as many ids."""
    check(*problem([1] * 24, V, dtype, 57, drafter))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [5, 700, 60000])
def test_equal_distributions_leave_nothing_beyond_the_drafter(dtype, V):
    """A draft that a random number of one rejects all the same: the drafter has all of the verifier's probability, so that the draw is from the verifier's own."""
    B = 30
    target, _, drafts, off, u, r = problem([1] * B, V, dtype, 47, True, 1.7)
    u[:] = 1.0
    shifted = (target.float().round() - 64.0).to(TORCH[dtype])           # (the same distances from the top)
    check(target, target.clone(), drafts, off, u, r, temperature=1.7)
    check(target.float().round().to(TORCH[dtype]), shifted, drafts, off, u, r, temperature=1.7)
