"""Verification by sampling on the GPU (as2d_sampler_*), against the float64
oracle: accepted paths and tokens equal, log-probabilities to float32."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import trees                     # noqa: E402
from paper_2609_37617_amd import as2d        # noqa: E402
from tests.harness import ensure_built       # noqa: E402

pytestmark = pytest.mark.gpu

# logp is one rounding to float32 (2^-24 relative) of a value whose logits and
# 64-bit logarithm of a sum of float32 powers are good to 2^-22 absolute
LOGP_ABS, LOGP_REL = 2.0 ** -22, 2.0 ** -24


@pytest.fixture(scope="module")
def sampler():
    ensure_built()
    s = as2d.Sampler(64, 31, 160000)
    yield s
    s.close()


def heap(k, branch):
    return [i // branch - 1 for i in range(k)]


def inputs(n, k, vocab, branch, dtype=torch.float32, pad=0, seed=0, spread=2.0, temperature=1.0, noise=0.7):
    g = torch.Generator().manual_seed(seed)
    t = spread * torch.randn((n, k + 1, vocab), generator=g)
    d = t + noise * torch.randn((n, k + 1, vocab), generator=g)
    t, d = t.to(dtype), d.to(dtype)
    cands = torch.zeros((n, k), dtype=torch.int32)
    for i, p in enumerate(heap(k, branch)):
        cands[:, i] = torch.multinomial(torch.softmax(d[:, p + 1].double() / temperature, -1), 1, generator=g)[:, 0].int()
    u = torch.rand((n, k + 1), generator=g)

    def rows(x):
        out = torch.full((n, k + 1, vocab + pad), float("nan"), dtype=dtype, device="cuda")[:, :, :vocab]
        return out.copy_(x)
    return rows(t), rows(d), cands.cuda(), u.cuda()


def check(got, target, cands, u, parents, draft=None, temperature=1.0, draft_temperature=None, ks=None):
    got = {name: x.cpu() for name, x in got.items()}
    n, rows, vocab = target.shape
    k = rows - 1
    t = target.double().cpu().numpy()
    d = None if draft is None else draft.double().cpu().numpy()
    for r in range(n):
        kr = k if ks is None else ks[r]
        temp = float(temperature[r]) if hasattr(temperature, "__len__") else temperature
        uu = u[r].cpu().numpy()
        path, token, logp = trees.sample_walk(t[r, :kr + 1], cands[r, :kr].cpu().numpy(), np.append(uu[:kr], uu[k]), parents[:kr],
                                              temp, None if d is None else d[r], draft_temperature)
        assert got["path"][r].tolist() == path + [-1] * (k - len(path)), r
        assert (int(got["accepted"][r]), int(got["token"][r])) == (len(path), token), r
        mine = np.append(got["logp"][r, :kr].numpy(), got["logp"][r, k].numpy())
        # float32's range ends at 3.4e38: a finite -6e38 of 64 bits is its -inf
        with np.errstate(over="ignore"):
            fine = np.isfinite(np.asarray(logp).astype(np.float32))
        assert np.array_equal(np.isfinite(mine), fine)
        assert (np.abs(mine[fine] - np.array(logp)[fine]) <= LOGP_ABS + LOGP_REL * np.abs(np.array(logp)[fine])).all(), r
        assert torch.isnan(got["logp"][r, kr:k]).all()


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("n,k,vocab,branch", [(1, 0, 1, 1), (1, 0, 5, 1), (3, 1, 2, 1), (2, 4, 17, 1), (64, 3, 100, 2),
                                              (1, 31, 4096, 1), (2, 31, 4097, 31), (5, 8, 8191, 3), (1, 8, 152064, 1),
                                              (3, 15, 50257, 4)])
def test_against_the_oracle(sampler, n, k, vocab, branch, with_draft):
    t, d, cands, u = inputs(n, k, vocab, branch, seed=n + k + vocab)
    d = d if with_draft else None
    check(sampler.verify(t, cands, u, parents=heap(k, branch), draft_logits=d), t, cands, u, heap(k, branch), d)


@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_types_and_strides(sampler, dtype, pad):
    """Rows at any element's address; what lies between them (NaN here) is not read."""
    t, d, cands, u = inputs(3, 5, 5001, 2, dtype, pad, seed=pad, temperature=0.6)
    got = sampler.verify(t, cands, u, parents=heap(5, 2), draft_logits=d, temperature=0.6)
    check(got, t, cands, u, heap(5, 2), d, 0.6)


def test_temperatures(sampler):
    t, d, cands, u = inputs(4, 4, 3000, 1, seed=9)
    temps = torch.tensor([0.05, 0.5, 1.0, 4.0], device="cuda")
    check(sampler.verify(t, cands, u, draft_logits=d, temperature=temps, draft_temperature=1.3), t, cands, u, trees.chain(4), d,
          temps.cpu(), 1.3)
    check(sampler.verify(t, cands, u, draft_logits=d, temperature=temps), t, cands, u, trees.chain(4), d, temps.cpu())


def test_ragged_requests(sampler):
    """ks[r] candidates of k; logits, candidates and numbers past them are garbage."""
    t, d, cands, u = inputs(4, 6, 700, 2, seed=4)
    ks = [0, 1, 4, 6]
    for r, kr in enumerate(ks):
        t[r, kr + 1:] = float("nan")
        d[r, kr + 1:] = float("inf")
        cands[r, kr:] = -77
        u[r, kr:6] = float("nan")
    dev = torch.tensor(ks, dtype=torch.int32, device="cuda")
    for draft in (None, d):
        check(sampler.verify(t, cands, u, parents=heap(6, 2), ks=dev, draft_logits=draft), t, cands, u, heap(6, 2), draft, ks=ks)


def test_a_drafter_s_rows_without_children_are_not_read(sampler):
    t, d, cands, u = inputs(2, 4, 900, 2, seed=5)
    d[:, 2:] = float("nan")   # rows 0 and 1 have the four children
    got = sampler.verify(t, cands, u, parents=[-1, -1, 0, 0], draft_logits=d)
    check(got, t, cands, u, [-1, -1, 0, 0], d)


@pytest.mark.parametrize("with_draft", [False, True])
def test_masked_tokens(sampler, with_draft):
    """-inf logits are tokens of probability 0, whole chunks of them too; one allowed token is certain."""
    t, d, cands, u = inputs(3, 3, 9000, 1, seed=6)
    t[:, :, 100:8500] = -float("inf")
    t[1, 0] = -float("inf")
    t[1, 0, 4242] = -3.0
    t[2, 1, :] = -3.0e38
    t[2, 1, 17] = 3.0e38
    d = d if with_draft else None
    got = sampler.verify(t, cands, u, draft_logits=d)
    check(got, t, cands, u, trees.chain(3), d)


def test_the_same_candidate_twice(sampler):
    """A rejected token has no probability left when a sibling repeats it."""
    t, _, cands, u = inputs(1, 4, 50, 4, seed=7)
    cands[0] = torch.tensor([3, 3, 8, 3], dtype=torch.int32)
    u[0, :4] = 0.999999
    u[0, 4] = 0.0
    check(sampler.verify(t, cands, u, parents=[-1] * 4), t, cands, u, [-1] * 4)


def test_which_sibling_is_taken_from_call_to_call(sampler):
    """A child's mass is left out where an earlier sibling is accepted: in calls
    one after another on one workspace, what an earlier call left there has to
    be neither read nor missed.  The number 0 accepts a child with anything
    left; the last below 1 rejects most."""
    k, branch, n = 12, 3, 6
    parents = heap(k, branch)
    t, d, cands, u = inputs(n, k, 5003, branch, seed=31, noise=1.5)
    g = torch.Generator().manual_seed(5)
    lengths = []
    for first in (0, 3, 1, 3, 2, 0, None, None):   # the child that is given 0, 3: none, None: any
        pick = torch.randint(0, 4, (n, k), generator=g) if first is None else torch.full((n, k), first)
        turn = torch.arange(k) % branch   # which child of its node a candidate is
        u[:, :k] = torch.where(pick == turn, 0.0, 1.0 - 2.0 ** -24).cuda()
        got = sampler.verify(t, cands, u, parents=parents, draft_logits=d)
        check(got, t, cands, u, parents, d)
        lengths.append(got["accepted"].float().mean().item())
    assert lengths[0] > lengths[1]     # the two kinds of call differ


def test_candidates_outside_the_vocabulary_are_never_accepted(sampler):
    t, d, cands, u = inputs(1, 3, 60, 1, seed=8)
    cands[0] = torch.tensor([-1, 60, 2 ** 31 - 1], dtype=torch.int32)
    u[0, :3] = 0.0
    for draft in (None, d):
        got = sampler.verify(t, cands, u, parents=[-1, -1, -1], draft_logits=draft)
        assert int(got["accepted"][0]) == 0 and 0 <= int(got["token"][0]) < 60
        assert torch.isinf(got["logp"][0, :3]).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["target", "draft"])
def test_non_finite_logits_end_their_request_only(sampler, where, value):
    t, d, cands, u = inputs(3, 3, 5000, 1, seed=10)
    (t if where == "target" else d)[1, 2, 4999] = value
    got = sampler.verify(t, cands, u, draft_logits=d)
    assert got["accepted"].tolist()[1] == got["token"].tolist()[1] == -1
    assert got["path"][1].tolist() == [-1] * 3 and torch.isnan(got["logp"][1]).all()
    keep = [0, 2]
    check({name: x[keep] for name, x in got.items()}, t[keep], cands[keep], u[keep], trees.chain(3), d[keep])


def test_rows_of_minus_infinity_and_bad_parameters(sampler):
    t, d, cands, u = inputs(5, 2, 300, 1, seed=11)
    t[0, 1] = -float("inf")
    ks = torch.tensor([2, 3, -1, 2, 2], dtype=torch.int32, device="cuda")
    temps = torch.tensor([1.0, 1.0, 1.0, 0.0, float("nan")], device="cuda")
    got = sampler.verify(t, cands, u, ks=ks, temperature=temps)
    assert got["accepted"].tolist() == [-1] * 5 and got["token"].tolist() == [-1] * 5
    assert torch.isnan(got["logp"]).all()


@pytest.mark.parametrize("with_draft", [False, True])
def test_random_numbers_next_to_a_border(sampler, with_draft):
    """The float32 numbers on either side of the acceptance border p(x) / q(x), and the last and first of the range."""
    t, d, cands, _ = inputs(1, 1, 2000, 1, seed=12, noise=1.5)
    x = int(cands[0, 0])
    p = np.exp(trees.log_softmax(t[0, 0].double().cpu().numpy(), 1.0))[x]
    q = np.exp(trees.log_softmax(d[0, 0].double().cpu().numpy(), 1.0))[x] if with_draft else 1.0
    border = np.float32(min(p / q, 0.9))
    us = [0.0, 1 - 2.0 ** -24, border]
    for step in range(2, 5):   # float32 powers leave 2^-23 of the border open
        lo = hi = border
        for _ in range(4 * step):
            lo, hi = np.nextafter(lo, np.float32(0)), np.nextafter(hi, np.float32(1))
        us += [lo, hi]
    us = [w for w in us if w != border]
    n = len(us)
    u = torch.tensor([[w, 0.3] for w in us], dtype=torch.float32, device="cuda")
    tt, dd, cc = t.expand(n, -1, -1).contiguous(), d.expand(n, -1, -1).contiguous(), cands.expand(n, -1).contiguous()
    dd = dd if with_draft else None
    check(sampler.verify(tt, cc, u, draft_logits=dd), tt, cc, u, [-1], dd)


def test_the_extremes_of_the_last_number(sampler):
    t, d, cands, u = inputs(2, 2, 6000, 1, seed=13)
    u[0, 2], u[1, 2] = 0.0, 1 - 2.0 ** -24
    for draft in (None, d):
        check(sampler.verify(t, cands, u, draft_logits=draft), t, cands, u, trees.chain(2), draft)


def test_committed_tokens_follow_the_target(sampler):
    """64 x 400 calls: the first committed token's frequencies within five standard deviations of the target's."""
    V, k, branch = 7, 4, 2
    g = torch.Generator().manual_seed(14)
    t1, d1 = 1.5 * torch.randn((k + 1, V), generator=g), 1.5 * torch.randn((k + 1, V), generator=g)
    p = torch.softmax(t1[0].double(), -1).numpy()
    count, n = np.zeros(V), 64 * 400
    t, d = t1.expand(64, -1, -1).contiguous().cuda(), d1.expand(64, -1, -1).contiguous().cuda()
    for _ in range(400):
        cands = torch.stack([torch.multinomial(torch.softmax(d1[q + 1], -1), 64, replacement=True, generator=g)
                             for q in heap(k, branch)], 1).int().cuda()
        got = sampler.verify(t, cands, torch.rand((64, k + 1), generator=g).cuda(), parents=heap(k, branch), draft_logits=d)
        path, token, c = got["path"].cpu(), got["token"].cpu(), cands.cpu()
        first = torch.where(path[:, 0] >= 0, c.gather(1, path[:, :1].clamp(min=0).long())[:, 0], token)
        count += np.bincount(first.numpy(), minlength=V)
    assert (np.abs(count / n - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()


def test_a_replayed_graph_and_other_streams(sampler):
    """Captured once, replayed with new inputs and other calls of the sampler in between."""
    t, d, cands, u = inputs(2, 6, 20000, 2, seed=15)
    other = inputs(3, 3, 9000, 1, seed=16)
    sampler.verify(t, cands, u, parents=heap(6, 2), draft_logits=d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = sampler.verify(t, cands, u, parents=heap(6, 2), draft_logits=d)
    for seed in (17, 18, 19):
        nt, nd, nc, nu = inputs(2, 6, 20000, 2, seed=seed)
        for a, b in ((t, nt), (d, nd), (cands, nc), (u, nu)):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(got, t, cands, u, heap(6, 2), d)
        with torch.cuda.stream(side):
            check(sampler.verify(other[0], other[2], other[3]), other[0], other[2], other[3], trees.chain(3))
        check(sampler.verify(other[0], other[2], other[3], draft_logits=other[1]), other[0], other[2], other[3], trees.chain(3),
              other[1])
        torch.cuda.synchronize()


def test_two_streams_in_turn(sampler):
    """Calls on two streams with nothing waited for in between share the workspace in order."""
    a, b = inputs(4, 8, 60000, 1, seed=20), inputs(4, 8, 60000, 2, seed=21)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        with torch.cuda.stream(s1):
            got.append((sampler.verify(a[0], a[2], a[3], draft_logits=a[1]), a, 1))
        with torch.cuda.stream(s2):
            got.append((sampler.verify(b[0], b[2], b[3], parents=heap(8, 2), draft_logits=b[1]), b, 2))
    torch.cuda.synchronize()
    for out, x, branch in got:
        check(out, x[0], x[2], x[3], heap(8, branch), x[1])


def test_refusals(sampler):
    t, d, cands, u = inputs(2, 3, 100, 1, seed=22)

    def refused(**kw):
        args = dict(logits=t, cands=cands, uniforms=u)
        args.update(kw)
        with pytest.raises(as2d.As2dError) as e:
            sampler.verify(**args)
        assert e.value.code == as2d.EINVAL, e.value
    refused(parents=[-1, 1, 0])
    refused(parents=[-2, 0, 1])
    refused(parents=[-1, 0])
    refused(temperature=0.0)
    refused(temperature=float("nan"))
    refused(temperature=float("inf"))
    refused(draft_logits=d, draft_temperature=-1.0)
    refused(cands=cands.long())
    refused(cands=cands[:, :2])
    refused(cands=cands.cpu())
    refused(uniforms=u.double())
    refused(uniforms=u[:1])
    refused(logits=t.half())
    refused(logits=t[0])
    refused(logits=t.transpose(1, 2).contiguous().transpose(1, 2))
    refused(draft_logits=d.bfloat16())
    refused(draft_logits=d[:1])
    refused(ks=torch.tensor([3], dtype=torch.int32, device="cuda"))
    refused(temperature=torch.ones(3, device="cuda"))
    small = as2d.Sampler(1, 2, 50)
    for kw in (dict(), dict(logits=t[:1], cands=cands[:1], uniforms=u[:1])):
        with pytest.raises(as2d.As2dError):
            small.verify(**dict(dict(logits=t, cands=cands, uniforms=u), **kw))
    small.close()


def test_no_requests(sampler):
    got = sampler.verify(torch.empty((0, 4, 10), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"),
                         torch.empty((0, 4), device="cuda"))
    assert got["accepted"].shape == (0,) and got["path"].shape == (0, 3)


def test_a_call_captured_while_another_runs(sampler):
    """A long call runs on one stream while one is captured, and never
    replayed, on a second; calls on the second and a third, of other shapes and
    with nothing waited for, still come after the first."""
    long, captured, short = (inputs(8, 8, 152064, 2, seed=23), inputs(2, 3, 9000, 1, seed=24), inputs(3, 5, 30000, 1, seed=25))
    a, b, c = (torch.cuda.Stream() for _ in range(3))
    sampler.verify(captured[0], captured[2], captured[3], draft_logits=captured[1])
    for _ in range(3):
        torch.cuda.synchronize()
        graph, got = torch.cuda.CUDAGraph(), []
        with torch.cuda.stream(a):
            for _ in range(4):
                got.append((sampler.verify(long[0], long[2], long[3], parents=heap(8, 2), draft_logits=long[1]), long, 2))
        with torch.cuda.stream(b):
            graph.capture_begin()
            sampler.verify(captured[0], captured[2], captured[3], draft_logits=captured[1])
            graph.capture_end()
            got.append((sampler.verify(short[0], short[2], short[3], draft_logits=short[1]), short, 1))
        with torch.cuda.stream(c):
            got.append((sampler.verify(long[0], long[2], long[3], parents=heap(8, 2), draft_logits=long[1]), long, 2))
        torch.cuda.synchronize()
        for out, x, branch in got:
            check(out, x[0], x[2], x[3], heap(x[2].shape[1], branch), x[1])


def next_to_borders(p, n, near):
    """n float32 numbers in [0, 1) that lie `near` (a range of distances) a border of the running sums of p, either side."""
    run = np.cumsum(p)
    run /= run[-1]
    grid = np.round(run[:-1] * 2.0 ** 24)   # multiples of 2^-24 are float32 numbers
    away = grid * 2.0 ** -24 - run[:-1]
    pick = np.flatnonzero((np.abs(away) > near[0]) & (np.abs(away) < near[1]) & (grid < 2 ** 24))
    assert len(pick) >= n
    return (grid[pick[np.linspace(0, len(pick) - 1, n).astype(int)]] * 2.0 ** -24).astype(np.float32)


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("dtype,temperature", [(torch.float32, 1.0), (torch.bfloat16, 0.7)])
def test_tokens_next_to_the_borders_of_the_running_sum(sampler, dtype, temperature, with_draft):
    """Numbers close to a border between two tokens.  A term p or q is off by
    twice 2^-33.8 of itself (its power and its row's sum), so the running sum of
    what is left, and the whole one, by 2 (1 + 1) 2^-33.8 each, and their
    quotient by 8 2^-33.8 = 2^-30.8 over the mass S that is left.  With a drafter
    that is what one rejection leaves."""
    n, V = 64, 152064
    t, d, cands, _ = inputs(1, 1, V, 1, dtype, seed=26, noise=1.5)
    p = np.exp(trees.log_softmax(t[0, 0].double().cpu().numpy(), temperature))
    if with_draft:
        q = np.exp(trees.log_softmax(d[0, 0].double().cpu().numpy(), temperature))
        x = int(np.argmax(q / p))   # rejected by the largest number: q > p
        left = np.maximum(p - q, 0.0)
    else:
        x = int(np.argmin(p))
        left = p.copy()
        left[x] = 0.0
    assert left.sum() > 0.2
    us = next_to_borders(left, n, (2.0 ** -30.5 / left.sum(), 2.0 ** -26))
    u = torch.tensor([[1 - 2.0 ** -24, w] for w in us], dtype=torch.float32, device="cuda")
    tt = t.expand(n, -1, -1).contiguous()
    dd = d.expand(n, -1, -1).contiguous() if with_draft else None
    cc = torch.full((n, 1), x, dtype=torch.int32, device="cuda")
    got = sampler.verify(tt, cc, u, draft_logits=dd, temperature=temperature)
    assert not got["accepted"].any()
    check(got, tt, cc, u, [-1], dd, temperature)


@pytest.mark.parametrize("gap", [3.0, 8.0, 12.0])
def test_log_probabilities_of_a_token_that_carries_the_row(sampler, gap):
    """The sum of a row is as good as its terms: log p of a token near
    certainty is right to its own rounding (2^-24) and 2^-33.8 of the sum."""
    V = 50257
    g = torch.Generator().manual_seed(27)
    t = torch.randn((8, 1, V), generator=g)
    t[:, 0, 77] = gap + np.log(V) + torch.rand(8, generator=g)
    got = sampler.verify(t.cuda(), None, torch.full((8, 1), 0.5, device="cuda"))
    for r in range(8):
        lp = trees.log_softmax(t[r, 0].double().numpy(), 1.0)
        token = int(got["token"][r])
        assert abs(float(got["logp"][r, 0]) - lp[token]) <= 2.0 ** -24 * abs(lp[token]) + 2.0 ** -33


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("temperature", [1e-30, 1e-25, 1e-18, 1e-15, 1e-10, 1e-4, 1e4, 1e10, 1e30])
def test_the_whole_range_of_temperatures(sampler, temperature, with_draft):
    """From the largest logit alone to all tokens alike, over several chunks,
    with two tokens that share the largest logit."""
    n, k, V = 6, 3, 5000
    t, d, cands, u = inputs(n, k, V, 1, seed=28, spread=20.0)
    t[0, 0, [17, 4400]] = 200.0
    d[1, 0, [18, 19]] = 200.0
    cands[0, 0], cands[1, 0] = 4400, 19
    t[2, 0, :] = -1.0e30   # far logits: a difference of 1 is none in float32
    t[2, 0, 3000] = 2.0e37
    t[3, 1, 5:] = -float("inf")
    d = d if with_draft else None
    got = sampler.verify(t, cands, u, draft_logits=d, temperature=temperature)
    check(got, t, cands, u, trees.chain(k), d, temperature)


@pytest.mark.parametrize("top", [1e4, 1e20, 1e38])
def test_logits_of_any_size(sampler, top):
    """Equal large logits and ones a few float32 steps below them."""
    V, n = 3000, 5
    step = float(np.spacing(np.float32(top)))
    t = torch.full((n, 1, V), top)
    t[:, 0] -= step * torch.randint(0, 9, (n, V), generator=torch.Generator().manual_seed(29))
    u = torch.tensor([[0.0], [0.2], [0.5], [0.9], [1 - 2.0 ** -24]])
    for temperature in (step, 20 * step):
        if not 1e-30 <= temperature <= 1e30:
            continue
        check(sampler.verify(t.cuda(), None, u.cuda(), temperature=temperature), t, torch.zeros((n, 0), dtype=torch.int32), u, [],
              None, temperature)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(24, 3000), (24, 50257)])
@pytest.mark.parametrize("tokens", [[5, 6, 900, 901], [5, 2900, 1500, 10], [5, 5, 2900, 5], [2000, -1, 2047, 2048], [7, 2999, 2999, 8]])
def test_children_after_near_certain_ones(sampler, dtype, n, V, tokens):
    """Without a drafter's distribution the first two children have all but
    10^-7 each of what is left at their turn; the others share the rest, with
    numbers within 2^-20 of their borders.  In one workgroup's chunk of the
    vocabulary and in several, repeated and outside the vocabulary."""
    g = torch.Generator().manual_seed(30)
    t = torch.randn((1, 5, V), generator=g)
    large = [x for x in dict.fromkeys(tokens) if x >= 0]
    # about e^16 of the sum of what comes after, each time
    for i, x in enumerate(reversed(large[:2])):
        t[0, 0, x] = 16.6 * (i + 1) + np.log(V) + 0.5
    for x in large[2:]:
        t[0, 0, x] = np.log(V) - 1.0 if dtype == torch.float32 else 10.0
    t = t.to(dtype).expand(n, -1, -1).contiguous().cuda()
    cands = torch.tensor(tokens, dtype=torch.int32).expand(n, -1).contiguous().cuda()
    # the borders of the third and fourth child, in 64 bits
    left = np.exp(trees.log_softmax(t[0, 0].double().cpu().numpy(), 1.0))
    borders = []
    for x in tokens:
        borders.append(left[x] / left.sum() if x >= 0 else 0.0)
        if x >= 0:
            left[x] = 0.0
    rng = np.random.default_rng(1)
    u = np.full((n, 5), 1 - 2.0 ** -24, np.float32)
    for r in range(n):
        which = 2 + r % 2
        off = (1.0 + 2.0 ** -20 * rng.random()) ** (1 if r % 4 < 2 else -1)
        u[r, which] = np.float32(min(borders[which] * off, 1 - 2.0 ** -24))
        # a float32 step is 2^-23 at most: numbers that round onto the border itself are left out
        if abs(float(u[r, which]) - borders[which]) <= 2.0 ** -32 * borders[which]:
            u[r, which] = 0.5
        u[r, 4] = rng.random()
    u = torch.from_numpy(u).cuda()
    check(sampler.verify(t, cands, u, parents=[-1] * 4), t, cands, u, [-1] * 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,k,vocab,branch", [(16, 8, 152064, 1), (4, 15, 50257, 3), (1, 31, 152064, 1), (64, 31, 1025, 2),
                                              (1, 0, 152064, 1), (2, 4, 4097, 4)])
def test_without_a_drafter_on_both_sides_of_one_launch(sampler, n, k, vocab, branch, dtype):
    """One launch takes up to a workgroup per compute unit, as the last two do; the others take two."""
    t, _, cands, u = inputs(n, k, vocab, branch, dtype, seed=n + k, noise=0.1, temperature=0.4)
    ks = [k - (r % 3 if k > 3 else 0) for r in range(n)]
    dev = torch.tensor(ks, dtype=torch.int32, device="cuda")
    for temperature in (0.4, 1.0):
        check(sampler.verify(t, cands, u, parents=heap(k, branch), ks=dev, temperature=temperature), t, cands, u, heap(k, branch),
              None, temperature, ks=ks)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [262144, 262145, 300007, 1048576, 1048577, 1500001, 1 << 24])
def test_large_vocabularies(vocab, dtype):
    """Rows of more parts than a wave keeps (262,144 tokens) and more chunks
    than a workgroup has threads (1,048,576), up to the most; tokens far up the
    vocabulary, and rejected ones there."""
    n, k = (2, 3) if vocab < 1 << 24 else (1, 2)
    s = as2d.Sampler(n, k, vocab)
    t, d, cands, u = inputs(n, k, vocab, 1, dtype, seed=3) if vocab < 1 << 22 else (
        torch.randn((n, k + 1, vocab), generator=torch.Generator().manual_seed(1)).to(dtype).cuda(),) * 2 + (
        torch.tensor([[vocab - 1, 5]], dtype=torch.int32).cuda(), torch.tensor([[0.9, 0.9, 0.999]]).cuda())
    parents = [-1] * (k - 1) + [0]
    cands[0, 0] = vocab - 1
    t[0, 0, vocab - 1] = 10.0
    u[0, 0], u[0, k] = 1 - 2.0 ** -24, 1 - 2.0 ** -20
    for draft in (None, d):
        check(s.verify(t, cands, u, parents=parents, draft_logits=draft), t, cands, u, parents, draft)
    s.close()


@pytest.mark.parametrize("with_draft", [False, True])
def test_the_number_zero_takes_the_first_token_with_a_probability(sampler, with_draft):
    """In 64 bits: tokens below 2^-1074 of the whole have none, wherever in the
    vocabulary and in their chunk they stand; candidates of theirs are never
    accepted."""
    n, V = 4, 5000
    g = torch.Generator().manual_seed(33)
    t = -900.0 - 50.0 * torch.rand((n, 2, V), generator=g)      # e^-900: 0
    t[:, :, 3000:4000] = -600.0 - 50.0 * torch.rand((n, 2, 1000), generator=g)   # e^-650: a number
    t[1, :, 900] = -640.0
    t[2, :, 2047] = -500.0
    t[3, :, :10] = -float("inf")
    t[:, :, 4990] = 0.0
    d = t if with_draft else None
    cands = torch.full((n, 1), 17, dtype=torch.int32)
    u = torch.zeros((n, 2))
    got = sampler.verify(t.cuda(), cands.cuda(), u.cuda(), draft_logits=None if d is None else d.cuda())
    # (with the target's own logits as the drafter's nothing is left of a rejection, and the target's own are drawn from)
    assert got["accepted"].tolist() == [0] * n
    assert got["token"].tolist() == [3000, 900, 2047, 3000]
    for r in range(n):
        p = np.exp(trees.log_softmax(t[r, 0].double().numpy(), 1.0))
        assert int(np.argmax(np.cumsum(p) > 0)) == [3000, 900, 2047, 3000][r] and p[17] == 0
