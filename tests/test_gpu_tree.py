"""Trees of candidates on the GPU: attention over one layer of a cache against
float64, and whole passes (as2d_verify_tree, as2d_verify_sampled) against
chains, the oracle's walks on the pass's own logits, and fresh prefills."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import trees                                 # noqa: E402
from paper_2609_37617_amd import as2d                    # noqa: E402
from tests.harness import make_pair, prefix              # noqa: E402
from workload import QWEN05B, QWEN3B, QWEN7B, TINY, TINY_BF16   # noqa: E402

pytestmark = pytest.mark.gpu

LAYERS = dict(n_layers=2, hidden=128, ffn=64, vocab=128, qkv_bias=False)


def heap(k, branch):
    return [i // branch - 1 for i in range(k)]


def heads_model(shape, max_kv_len, max_requests=2):
    """Two narrow layers with the shape's heads: the operators see its caches."""
    from dataclasses import replace
    _, m = make_pair(replace(shape, name="heads", **LAYERS), max_requests=max_requests, max_kv_len=max_kv_len, max_k=31,
                     oracle=False)
    return m


def tensors(shape, rows, keys, seed, scale=1.5, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if shape.dtype == as2d.F32 else torch.bfloat16

    def normal(n, heads):
        return torch.randn((n, heads, shape.head_dim), generator=g)
    q, k, v = scale * normal(rows, shape.n_q_heads), normal(rows, shape.n_kv_heads), normal(rows, shape.n_kv_heads)
    K, V = normal(keys, shape.n_kv_heads), normal(keys, shape.n_kv_heads)
    return [x.to(t).to(device) for x in (q, k, v)] + [K.to(device), V.to(device)]


def bound(shape, q, K, k, V, v, keys):
    """Absolute error of an output, from the inputs' sizes.
    Scores: dim + 3 roundings of float32 over the sum of |q k|, and for bf16
    models two pairs of 2^-16 relative (the cache's, and the product of two
    low parts that is left out).  A weight is off by twice that (its own score
    and the sum's) and 2^-22 for the powers; sums over 32 keys of a chunk, 4
    chunks and the spans; for bf16 models three pairs of 2^-16 more (weights,
    values, low parts), and the output's own rounding of 2^-8."""
    d, bf = shape.head_dim, shape.dtype != as2d.F32
    size = max(float(torch.cat([K, k.float()]).abs().amax()) * float(q.float().abs().sum(-1).amax()), 1e-30) / np.sqrt(d)
    score = size * ((d + 3) * 2.0 ** -24 + (2 * 2.0 ** -16 if bf else 0))
    top = float(torch.cat([V, v.float()]).abs().amax())
    rel = 2 * np.expm1(score) + 2.0 ** -22 + (36 + keys / 128) * 2.0 ** -24 + (3 * 2.0 ** -16 if bf else 0)
    return rel * top * 2, 2.0 ** -8 if bf else 2.0 ** -24


def attend_and_check(m, shape, keys, rows, parents, seed, views=lambda x: x, stream=None):
    q, k, v, K, V = tensors(shape, rows, keys, seed)
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(keys, np.int32))
    m.write_kv(0, 1, K, V)
    got = m.tree_attention(0, 1, views(q), views(k), views(v), parents)
    full = parents if parents is not None else trees.chain(rows - 1)
    want = trees.attention(*(x.double().cpu().numpy() for x in (q, K, V, k, v)), full)
    err = np.abs(got.double().cpu().numpy() - want)
    a, r = bound(shape, q, K, k, V, v, keys)
    assert (err <= a + r * np.abs(want)).all(), (err.max(), a)
    assert m.state(0)[0] == keys   # the request is as it was
    return got


SHAPES = [TINY, TINY_BF16, QWEN05B, QWEN3B, QWEN7B]


@pytest.fixture(scope="module", params=SHAPES, ids=lambda s: s.name)
def served(request):
    m = heads_model(request.param, 4096)
    yield request.param, m
    m.close()


@pytest.mark.parametrize("keys,rows,branch", [(1, 1, 1), (1, 32, 2), (2, 5, 4), (31, 2, 1), (96, 32, 31), (97, 32, 1),
                                              (120, 32, 3), (127, 9, 2), (128, 17, 2), (300, 1, 1), (1024, 32, 4),
                                              (2047, 7, 2), (2100, 32, 2), (3999, 16, 3)])
def test_attention_against_64_bits(served, keys, rows, branch):
    """Cache lengths around the chunks of 32 keys, the spans of 128 and the
    16 spans that one launch merges; trees across those borders."""
    shape, m = served
    attend_and_check(m, shape, keys, rows, heap(rows - 1, branch), keys + rows)


def test_attention_over_two_trees_of_one_root(served):
    """Two chains below the root: a row's ancestors are not the rows before it."""
    shape, m = served
    parents = [-1, -1] + list(range(0, 22))   # even candidates follow even ones
    attend_and_check(m, shape, 125, 25, parents, 5)
    attend_and_check(m, shape, 500, 8, None, 6)   # parents None: a chain


def test_attention_with_large_scores_and_values(served):
    """One key has all the weight; values of stale cache rows never show."""
    shape, m = served
    m.prefill(1, np.zeros(0, np.uint16), np.zeros(900, np.int32))
    huge = torch.full((900, shape.n_kv_heads, shape.head_dim), 3.0e38, device="cuda")
    m.write_kv(1, 1, huge, huge)
    q, k, v, K, V = tensors(shape, 6, 40, 1)
    m.prefill(1, np.zeros(0, np.uint16), np.zeros(40, np.int32))   # the slot keeps what lies past the new length
    m.write_kv(1, 1, K, V)
    q[:] = 0
    q[:, :, 0] = 30.0
    k[:, :, 0] = 0
    K[:, :, 0] = 0
    K[7, :, 0] = 20.0
    m.write_kv(1, 1, K, V)
    got = m.tree_attention(1, 1, q, k, v, heap(5, 2))
    want = V[7].repeat_interleave(shape.n_q_heads // shape.n_kv_heads, 0)
    # the others' weight is 2^-50 and less: the value, in the cache's format
    assert (got.float() - want).abs().max() <= 4.0 * (2.0 ** -8 if shape.dtype != as2d.F32 else 2.0 ** -22)


@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_rows_reach_only_the_rows_that_see_them(served, what, value):
    shape, m = served
    parents = [-1, -1, 0, 1, 1, 3]
    for keys in (126, 2500):
        q, k, v, K, V = tensors(shape, 7, keys, 8)
        m.prefill(0, np.zeros(0, np.uint16), np.zeros(keys, np.int32))
        m.write_kv(0, 1, K, V)
        clean = m.tree_attention(0, 1, q, k, v, parents)
        (k if what == "k" else v)[2, :, 3] = value    # candidate 1, which candidates 3, 4 and 5 follow
        got = m.tree_attention(0, 1, q, k, v, parents)
        sees = trees.visible(parents)[:, 2]
        assert torch.equal(got[~sees], clean[~sees])
        if what == "v" or value != value:
            assert torch.isnan(got[sees]).any(-1).all()


@pytest.mark.parametrize("keys", [32, 64, 96, 97, 126, 127, 128, 160, 2144, 2528])
def test_a_key_of_nan_is_never_passed_over(served, keys):
    """Also where the NaN is all that a row sees of its chunk of 32 keys, the
    others being hidden: the maximum of their scores is then -inf."""
    shape, m = served
    # candidates 0 and 3 see little of the tree, 5 and 6 a long path
    parents = [-1, 0, 1, -1, 2, 4, 5]
    q, k, v, K, V = tensors(shape, 8, keys, 8)
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(keys, np.int32))
    m.write_kv(0, 1, K, V)
    clean = m.tree_attention(0, 1, q, k, v, parents)
    assert torch.isfinite(clean).all()
    for row in range(8):
        bad = k.clone()
        bad[row] = float("nan")
        got = m.tree_attention(0, 1, q, bad, v, parents)
        sees = trees.visible(parents)[:, row]
        assert torch.equal(got[~sees], clean[~sees]), row
        assert torch.isnan(got[sees]).all(), row


@pytest.mark.parametrize("keys", [2080, 2144, 2528, 4064])
def test_a_key_of_nan_in_runs_of_keys(served, keys):
    """The same with enough rows for runs of keys per workgroup (bf16 models), and values of NaN and infinity."""
    shape, m = served
    parents = heap(31, 3)
    q, k, v, K, V = tensors(shape, 32, keys, 9)
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(keys, np.int32))
    m.write_kv(0, 1, K, V)
    clean = m.tree_attention(0, 1, q, k, v, parents)
    for row in (0, 1, 9, 31):
        sees = trees.visible(parents)[:, row]
        for value, which in ((float("nan"), "k"), (float("nan"), "v"), (-float("inf"), "v")):
            kk, vv = k.clone(), v.clone()
            (kk if which == "k" else vv)[row, :, 5 if which == "v" else slice(None)] = value
            got = m.tree_attention(0, 1, q, kk, vv, parents)
            assert torch.equal(got[~sees], clean[~sees]), (row, which)
            assert torch.isnan(got[sees]).all(), (row, which)


LONG = [QWEN05B, QWEN7B]


@pytest.mark.parametrize("keys,rows,branch", [(8000, 32, 3), (7937, 31, 1), (8063, 9, 2), (5000, 32, 31), (8128, 18, 2)])
@pytest.mark.parametrize("shape", LONG, ids=lambda s: s.name)
def test_attention_over_long_caches(shape, keys, rows, branch):
    m = heads_model(shape, 8192, max_requests=1)
    attend_and_check(m, shape, keys, rows, heap(rows - 1, branch), keys + rows)
    m.set_cu_budget(64)   # longer runs, the last ones ragged
    attend_and_check(m, shape, keys, rows, heap(rows - 1, branch), keys + rows)
    m.set_cu_budget(1)    # one run holds every key
    attend_and_check(m, shape, 2100, rows, heap(rows - 1, branch), keys + rows)
    m.close()


@pytest.mark.parametrize("shape,keys,rows,branch", [(QWEN7B, 12345, 32, 2), (QWEN7B, 20001, 10, 3), (QWEN3B, 20000, 31, 2),
                                                    (QWEN05B, 20000, 32, 5)], ids=str)
def test_attention_of_two_row_tiles_a_wave(shape, keys, rows, branch):
    """Caches long enough for two tiles, the second partly or wholly past the rows."""
    m = heads_model(shape, keys + 64, max_requests=1)
    attend_and_check(m, shape, keys, rows, heap(rows - 1, branch), keys + rows)
    m.close()


@pytest.mark.parametrize("cus", [2, 16, 64])
def test_passes_of_two_row_tiles_a_wave(cus):
    """With few compute units passes over 3,000 keys take two tiles: logits are
    those of all units to rounding, for one request, three, and a graph of
    either used in turn."""
    from dataclasses import replace
    shape = replace(TINY_BF16, name="long", n_q_heads=28, n_kv_heads=4, head_dim=128, n_layers=1)
    _, m = make_pair(shape, max_requests=3, max_kv_len=4096, max_k=31, oracle=False)
    m.set_keep_logits(True)
    rng = np.random.default_rng(7)
    ks = [31, 9, 2]   # the last two fill one tile each
    parents = [[int(rng.integers(-1, i)) for i in range(k)] for k in ks]
    cands = [rng.integers(0, shape.vocab, k).tolist() for k in ks]

    def start():
        for r in range(3):
            m.prefill(r, np.zeros(0, np.uint16), np.arange(3000 + 300 * r, dtype=np.int32) % shape.vocab)

    def passes():
        out = []
        for reqs in ([0], [0, 1, 2], [1, 2], [1], [0]):
            start()
            m.verify_tree_batch(reqs, [cands[r] for r in reqs], [parents[r] for r in reqs])
            out += [m.logits(r) for r in reqs]
        return out
    want = passes()
    m.set_cu_budget(cus)
    for a, b in zip(want, passes()):
        assert close(a, b, shape)
    m.close()


def test_attention_of_other_strides(served):
    """Heads before rows, rows further apart, an output inside a larger tensor."""
    shape, m = served
    keys, rows, parents = 333, 11, heap(10, 2)
    plain = attend_and_check(m, shape, keys, rows, parents, 3)
    assert torch.equal(plain, attend_and_check(m, shape, keys, rows, np.array(parents), 3))
    heads_first = attend_and_check(m, shape, keys, rows, parents, 3,
                                   lambda x: x.transpose(0, 1).contiguous().transpose(0, 1))

    def spaced(x):   # odd element addresses
        big = torch.full((x.shape[0], x.shape[1] * x.shape[2] + 3), float("nan"), dtype=x.dtype, device="cuda")
        big[:, 1:-2] = x.reshape(x.shape[0], -1)
        return big[:, 1:-2].unflatten(1, x.shape[1:])
    odd = attend_and_check(m, shape, keys, rows, parents, 3, spaced)
    assert torch.equal(plain, heads_first) and torch.equal(plain, odd)
    q, k, v, _, _ = tensors(shape, rows, keys, 3)
    big = torch.zeros((rows, 2, shape.n_q_heads, shape.head_dim + 5), dtype=q.dtype, device="cuda")
    m.tree_attention(0, 1, q, k, v, parents, out=big[:, 1, :, 3:3 + shape.head_dim])
    assert torch.equal(big[:, 1, :, 3:3 + shape.head_dim], plain)
    assert not big[:, 0].any() and not big[:, 1, :, :3].any() and not big[:, 1, :, -2:].any()


def test_keys_and_values_shared_by_all_rows(served):
    """A broadcast input (stride 0) is read as it is."""
    shape, m = served
    q, k, v, K, V = tensors(shape, 6, 150, 4)
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(150, np.int32))
    m.write_kv(0, 1, K, V)
    one = m.tree_attention(0, 1, q, k[:1].expand(6, -1, -1), v[:1].expand(6, -1, -1), heap(5, 2))
    copies = m.tree_attention(0, 1, q, k[:1].repeat(6, 1, 1), v[:1].repeat(6, 1, 1), heap(5, 2))
    assert torch.equal(one, copies)


def test_an_output_of_equal_strides_is_refused(served):
    """Row 1 of head 0 would be row 0 of head 1; heads past the rows are an ordinary output."""
    shape, m = served
    q, k, v, K, V = tensors(shape, 5, 150, 4)
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(150, np.int32))
    m.write_kv(0, 1, K, V)
    d, nq = shape.head_dim, shape.n_q_heads
    room = torch.zeros((nq + 5) * d, dtype=q.dtype, device="cuda")
    with pytest.raises(as2d.As2dError) as e:
        m.tree_attention(0, 1, q, k, v, out=room.as_strided((5, nq, d), (d, d, 1)))
    assert e.value.code == as2d.EINVAL
    out = torch.empty((nq, 5, d), dtype=q.dtype, device="cuda").transpose(0, 1)
    assert torch.equal(m.tree_attention(0, 1, q, k, v, out=out), m.tree_attention(0, 1, q, k, v))


def test_write_kv_before_a_pass(served):
    """A pass on the context's stream waits for the rows another stream puts into the cache."""
    shape, m = served
    x = tensors(shape, 1, 3000, 9)[3:]
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(3000, np.int32))
    state = m.state(0)
    want = []
    for K, V in (x, [t.flip(0) for t in x]):
        for layer in range(2):
            m.write_kv(0, layer, K, V)
        torch.cuda.synchronize()
        want.append(m.decode_one(0))
        m.rollback(0, state[0], state[1])
    side = torch.cuda.Stream()
    for _ in range(4):
        for w, (K, V) in zip(want, (x, [t.flip(0) for t in x])):
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                for layer in range(2):
                    m.write_kv(0, layer, K, V)
            assert m.decode_one(0) == w
            m.rollback(0, state[0], state[1])


def test_attention_on_streams_in_turn(served):
    """Operators on two streams, a read of the cache and a pass of the context, nothing waited for in between."""
    shape, m = served
    x = [tensors(shape, rows, 1500, rows) for rows in (7, 20)]
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(1500, np.int32))
    m.write_kv(0, 1, x[0][3], x[0][4])
    alone = []
    for q, k, v, _, _ in x:
        alone.append(m.tree_attention(0, 1, q, k, v, heap(len(q) - 1, 2)))
        torch.cuda.synchronize()
    K0, _ = m.read_kv(0, 1, 1500)
    state = m.state(0)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for s, (q, k, v, _, _) in zip(streams, x):
            with torch.cuda.stream(s):
                got.append(m.tree_attention(0, 1, q, k, v, heap(len(q) - 1, 2)))
        K1, _ = m.read_kv(0, 1, 1500)
        m.decode_one(0)
        m.rollback(0, state[0], state[1])
        for a, b in zip(alone, got):
            torch.cuda.synchronize()
            assert torch.equal(a, b)
        assert np.array_equal(K0, K1)


def test_write_kv_is_read_back(served):
    shape, m = served
    m.prefill(1, np.zeros(0, np.uint16), np.zeros(200, np.int32))
    k0, v0 = m.read_kv(1, 0, 200)
    _, _, _, K, V = tensors(shape, 1, 61, 2)
    m.write_kv(1, 0, K, V, pos=70)
    k1, v1 = m.read_kv(1, 0, 200)
    tol = 0 if shape.dtype == as2d.F32 else 2.0 ** -16   # bf16 pairs
    for got, old, new in ((k1, k0, K), (v1, v0, V)):
        new = new.transpose(0, 1).cpu().numpy()
        assert (np.abs(got[:, 70:131] - new) <= tol * np.abs(new)).all()
        assert np.array_equal(got[:, :70], old[:, :70]) and np.array_equal(got[:, 131:], old[:, 131:])
    m.write_kv(1, 0, K.bfloat16(), V.bfloat16(), pos=139)
    k2, _ = m.read_kv(1, 0, 200)
    assert np.array_equal(k2[:, 139:], K.bfloat16().float().transpose(0, 1).cpu().numpy())
    m.write_kv(1, 0, K[:0], V[:0], pos=200)


def test_operator_refusals(served):
    shape, m = served
    m.prefill(1, np.zeros(0, np.uint16), np.zeros(4090, np.int32))
    q, k, v, K, V = tensors(shape, 5, 8, 0)

    def refused(code, f, *args, **kw):
        with pytest.raises(as2d.As2dError) as e:
            f(*args, **kw)
        assert e.value.code == code, e.value
    att = m.tree_attention
    refused(as2d.EINVAL, att, 9, 0, q, k, v)
    refused(as2d.EINVAL, att, 1, 2, q, k, v)
    refused(as2d.EINVAL, att, 1, -1, q, k, v)
    refused(as2d.EINVAL, att, 1, 0, q, k, v, [-1, 0, 3, 1])
    refused(as2d.EINVAL, att, 1, 0, q, k, v, [-1, 0, -2, 1])
    refused(as2d.EINVAL, att, 1, 0, q, k, v, [-1, 0])
    refused(as2d.EINVAL, att, 1, 0, q[:0], k[:0], v[:0])
    refused(as2d.EINVAL, att, 1, 0, q.cpu(), k, v)
    refused(as2d.EINVAL, att, 1, 0, q.half(), k, v)
    refused(as2d.EINVAL, att, 1, 0, q[:, :1], k, v)
    refused(as2d.EINVAL, att, 1, 0, q, k[:4], v)
    refused(as2d.EINVAL, att, 1, 0, q, k, v, out=torch.empty((5, 1, 1), device="cuda"))
    refused(as2d.EINVAL, att, 1, 0, q, k, v, out=torch.empty_like(q[:1]).expand(5, -1, -1))
    refused(as2d.EINVAL, att, 1, 0, q.transpose(1, 2).contiguous().transpose(1, 2), k, v)
    big = tensors(shape, 33, 1, 0)
    refused(as2d.EINVAL, att, 1, 0, *big[:3])
    refused(as2d.ECAPACITY, att, 1, 0, *tensors(shape, 7, 1, 0)[:3])   # 4,090 + 7 > 4,096
    m.release(0)
    refused(as2d.ESTATE, att, 0, 0, q, k, v)
    refused(as2d.ESTATE, m.write_kv, 0, 0, K, V)
    refused(as2d.EINVAL, m.write_kv, 1, 0, K, V, pos=4083)
    refused(as2d.EINVAL, m.write_kv, 1, 0, K, V, pos=-1)
    refused(as2d.EINVAL, m.write_kv, 1, 5, K, V)
    refused(as2d.EINVAL, m.write_kv, 1, 0, K.half(), V.half())
    refused(as2d.EINVAL, m.write_kv, 1, 0, K, V[:3])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = torch.empty_like(q)
        refused(as2d.ESTATE, att, 1, 0, q, k, v, out=out)
        out.zero_()
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(4, np.int32))


# ---------------------------------------------------------------------------
# Whole passes

PASS_SHAPES = [TINY, TINY_BF16]


@pytest.fixture(scope="module", params=PASS_SHAPES, ids=lambda s: s.name)
def model(request):
    _, m = make_pair(request.param, seed=0, max_requests=4, max_kv_len=512, max_k=31, oracle=False)
    m.set_keep_logits(True)
    yield request.param, m
    m.close()


def prefilled(m, shape, req=0, n_audio=70, n_instr=5, seed=3):
    _, a_dev, instr = prefix(shape, n_audio, n_instr, seed=seed, req=req)
    return m.prefill(req, a_dev, instr)


def cache(m, shape, req, n):
    return [np.stack(m.read_kv(req, l, n)) for l in range(shape.n_layers)]


def greedy_stream(m, req, n):
    """The next n greedy tokens after the pending root, and back."""
    kv, root, _ = m.state(req)
    out = [m.decode_one(req)["correction_token"] for _ in range(n)]
    m.rollback(req, kv, root)
    return out


def close(a, b, shape):
    """Two orders of the same float32 sums over a few layers: 2e-5 (float32) and 1e-3 (bf16 pairs) of values near 1."""
    return np.abs(np.asarray(a) - np.asarray(b)).max() <= (2e-5 if shape.dtype == as2d.F32 else 1e-3)


@pytest.mark.parametrize("mode", [as2d.EXEC_EAGER, as2d.EXEC_GRAPH, as2d.EXEC_PERSISTENT])
@pytest.mark.parametrize("n_audio", [70, 118, 123])
def test_a_chain_is_verify_bit_for_bit(model, mode, n_audio):
    shape, m = model
    m.set_exec_mode(mode)
    for k in (0, 1, 8, 31):
        _, L = prefilled(m, shape, 0, n_audio)
        y = greedy_stream(m, 0, 12)
        cands = (y + [7] * 31)[:k]
        if k > 3:
            cands[3] = (cands[3] + 1) % shape.vocab
        a = m.verify(0, cands)
        la, ka = m.logits(0), cache(m, shape, 0, a["kv_len"])
        prefilled(m, shape, 0, n_audio)
        b = m.verify_tree(0, cands)
        assert b.pop("path") == list(range(b["accepted_len"]))
        assert a == b and np.array_equal(la, m.logits(0))
        assert all(np.array_equal(x, y) for x, y in zip(ka, cache(m, shape, 0, a["kv_len"])))
        assert m.decode_one(0)["kv_len"] == a["kv_len"] + 1
    m.set_exec_mode(as2d.EXEC_GRAPH)


def planted(y, vocab, seed, k=20):
    """A tree that holds the greedy stream y along one path of siblings: every
    node of the path has a wrong child first, then the right one."""
    rng = np.random.default_rng(seed)
    cands, parents, node = [], [], -1
    for t in y[:k // 2]:
        cands += [int((t + 1 + rng.integers(vocab - 1)) % vocab), int(t)]
        parents += [node, node]
        node = len(cands) - 1
    return cands, parents


@pytest.mark.parametrize("n_audio", [20, 118, 123, 250])
def test_a_path_through_siblings(model, n_audio):
    """The planted path is accepted, its logits are a chain's, and the cache it
    leaves is a chain's: decoding goes on as after a chain."""
    shape, m = model
    _, L = prefilled(m, shape, 0, n_audio)
    y = greedy_stream(m, 0, 16)
    cands, parents = planted(y, shape.vocab, n_audio)
    out = m.verify_tree(0, cands, parents)
    assert out["path"] == list(range(1, 20, 2)) and out["accepted_len"] == 10 and out["correction_token"] == y[10]
    assert out["kv_len"] == L + 11 and out["committed"] == 11
    tree_logits, after = m.logits(0), cache(m, shape, 0, L + 11)
    assert trees.greedy_walk(m.row_tokens(0), cands, parents) == (out["path"], out["correction_token"])
    more = [m.decode_one(0)["correction_token"] for _ in range(4)]
    prefilled(m, shape, 0, n_audio)
    chain = m.verify(0, y[:10])
    assert chain["accepted_len"] == 10
    assert close(tree_logits[[0] + list(range(2, 21, 2))], m.logits(0), shape)
    for a, b in zip(after, cache(m, shape, 0, L + 11)):
        assert close(a, b, shape)
    assert more == y[11:15]


def test_every_branch_is_its_own_chain(model):
    """Each root-to-leaf path's logits are those of the path verified alone."""
    shape, m = model
    rng = np.random.default_rng(5)
    k = 31
    parents = [int(rng.integers(-1, i)) for i in range(k)]
    cands = rng.integers(0, shape.vocab, k).tolist()
    prefilled(m, shape, 0, 123)
    m.verify_tree(0, cands, parents)
    got = m.logits(0)
    sees = trees.visible(parents)
    for leaf in [i for i in range(k) if i not in parents]:
        rows = np.flatnonzero(sees[leaf + 1])
        prefilled(m, shape, 0, 123)
        m.verify(0, [cands[i - 1] for i in rows[1:]])
        assert close(got[rows], m.logits(0), shape), leaf


def test_passes_over_long_caches():
    """Trees at 7B heads over slots of more than 2,048 positions, one request and
    two: every branch is its own chain's to rounding; a call of chains alone
    has as2d_verify_batch's bits."""
    from dataclasses import replace
    shape = replace(TINY_BF16, name="long", n_q_heads=28, n_kv_heads=4, head_dim=128, n_layers=1)
    _, m = make_pair(shape, max_requests=2, max_kv_len=4096, max_k=31, oracle=False)
    m.set_keep_logits(True)
    rng = np.random.default_rng(6)
    k = 31
    parents = [[int(rng.integers(-1, i)) for i in range(k)] for _ in range(2)]
    cands = [rng.integers(0, shape.vocab, k).tolist() for _ in range(2)]

    def start():
        for r in range(2):
            m.prefill(r, np.zeros(0, np.uint16), np.arange(3000 + 700 * r, dtype=np.int32) % shape.vocab)
    start()
    m.verify_tree(0, cands[0], parents[0])
    alone = m.logits(0)
    start()
    m.verify_tree_batch([0, 1], cands, parents)
    both = [m.logits(0), m.logits(1)]
    assert close(alone, both[0], shape)
    for r in range(2):
        sees = trees.visible(parents[r])
        for leaf in [i for i in range(k) if i not in parents[r]][:8]:
            rows = np.flatnonzero(sees[leaf + 1])
            start()
            m.verify(r, [cands[r][i - 1] for i in rows[1:]])
            assert close(both[r][rows], m.logits(r), shape), (r, leaf)
    start()
    a = m.verify_batch([0, 1], cands)
    la = [m.logits(0), m.logits(1)]
    start()
    b = m.verify_tree_batch([0, 1], cands)
    assert [dict(x, path=list(range(x["accepted_len"]))) for x in a] == b
    assert all(np.array_equal(x, m.logits(r)) for r, x in enumerate(la))
    m.close()


@pytest.mark.parametrize("shape", [TINY, TINY_BF16], ids=lambda s: s.name)
@pytest.mark.parametrize("keys", [1, 40, 127, 300, 900])
def test_passes_over_short_caches_in_long_slots(shape, keys):
    """The usual serving layout: slots of more than 2,048 positions, whose span
    states a second launch joins, with little in them.  Every branch is its own
    chain's to rounding, alone and among other requests."""
    from dataclasses import replace
    shape = replace(shape, name="long", n_q_heads=14, n_kv_heads=2, n_layers=1)
    _, m = make_pair(shape, max_requests=3, max_kv_len=4096, max_k=31, oracle=False)
    m.set_keep_logits(True)
    rng = np.random.default_rng(keys)
    ks = [31, 6, 13]
    parents = [[int(rng.integers(-1, i)) for i in range(k)] for k in ks]
    cands = [rng.integers(0, shape.vocab, k).tolist() for k in ks]

    def start(r):
        m.prefill(r, np.zeros(0, np.uint16), np.arange(keys + 5 * r, dtype=np.int32) % shape.vocab)
    for r in range(3):
        start(r)
    m.verify_tree_batch([0, 1, 2], cands, parents)
    got = [m.logits(r) for r in range(3)]
    for r in range(3):
        start(r)
        m.verify_tree(r, cands[r], parents[r])
        assert close(got[r], m.logits(r), shape), r
        sees = trees.visible(parents[r])
        for leaf in [i for i in range(ks[r]) if i not in parents[r]][:6]:
            rows = np.flatnonzero(sees[leaf + 1])
            start(r)
            m.verify(r, [cands[r][i - 1] for i in rows[1:]])
            assert close(got[r][rows], m.logits(r), shape), (r, leaf)
    m.close()


def test_no_child_is_accepted(model):
    shape, m = model
    _, L = prefilled(m, shape)
    y = greedy_stream(m, 0, 2)
    wrong = [(y[0] + 1 + i) % shape.vocab for i in range(6)]
    out = m.verify_tree(0, wrong, [-1] * 6)
    assert (out["accepted_len"], out["path"], out["correction_token"], out["kv_len"]) == (0, [], y[0], L + 1)
    assert m.decode_one(0)["correction_token"] == y[1]


def test_equal_siblings_and_the_lowest_number(model):
    shape, m = model
    prefilled(m, shape)
    y = greedy_stream(m, 0, 3)
    out = m.verify_tree(0, [y[0], y[0], y[1], y[1]], [-1, -1, 1, 0])
    assert out["path"] == [0, 3] and out["correction_token"] == y[2]


def test_batches_of_trees(model):
    """Each request of a fused pass does what it does alone; more than 32 rows
    take the wide passes."""
    shape, m = model
    for sizes in ((4, 0, 9), (20, 20, 6, 20)):
        args, alone = [], []
        for r, k in enumerate(sizes):
            prefilled(m, shape, r, 60 + 20 * r)
            c, p = planted(greedy_stream(m, r, 12), shape.vocab, r, k // 2 * 2)
            args.append((c, p))
            out = m.verify_tree(r, c, p)
            alone.append((out, m.logits(r)))
        for r in range(len(sizes)):
            prefilled(m, shape, r, 60 + 20 * r)
        both = m.verify_tree_batch(list(range(len(sizes))), [a[0] for a in args], [a[1] for a in args])
        for r, (out, lg) in enumerate(alone):
            assert both[r] == out
            assert np.array_equal(m.logits(r), lg)


@pytest.mark.parametrize("with_draft", ["none", "host", "device"])
@pytest.mark.parametrize("branch", [1, 3])
def test_sampled_passes(model, branch, with_draft):
    """The walk of the oracle on the pass's own logits; the cache and the
    next step follow the accepted path."""
    shape, m = model
    k = 12
    parents = heap(k, branch)
    for seed in range(4):
        rng = np.random.default_rng(seed)
        _, L = prefilled(m, shape, 0, 100 + seed)
        base = m.verify_tree(0, rng.integers(0, shape.vocab, k).tolist(), parents)
        assert base["kv_len"] > L
        prefilled(m, shape, 0, 100 + seed)
        # logits over 4,096 tokens are nearly flat: a sharp temperature lets some candidates through
        temp = 0.01
        draft = np.tile(m.logits(0), (k + 1, 1)).astype(np.float32) + rng.normal(size=(k + 1, shape.vocab)).astype(np.float32) * 0.02
        y = greedy_stream(m, 0, 6)
        prefilled(m, shape, 0, 100 + seed)
        cands = [(y[d - 1] if rng.random() < 0.7 and d <= 6 else int(rng.integers(shape.vocab)))
                 for d in trees.depths(parents)[1:]]
        u = rng.random(k + 1).astype(np.float32)
        d = None if with_draft == "none" else draft if with_draft == "host" else torch.from_numpy(draft).cuda()
        out = m.verify_sampled(0, cands, u, parents, temperature=temp, draft_logits=d)
        lg = m.logits(0).astype(np.float64)
        path, token, _ = trees.sample_walk(lg, cands, u, parents, temp, None if d is None else draft.astype(np.float64))
        assert (out["path"], out["correction_token"], out["accepted_len"]) == (path, token, len(path))
        assert out["kv_len"] == L + len(path) + 1
        after = cache(m, shape, 0, out["kv_len"])
        step = m.decode_one(0)
        prefilled(m, shape, 0, 100 + seed)
        m.verify(0, [cands[i] for i in path])
        for a, b in zip(after, cache(m, shape, 0, out["kv_len"])):
            assert close(a, b, shape)
        m.rollback(0, out["kv_len"] if m.state(0)[0] >= out["kv_len"] else m.state(0)[0], token)
        assert step["kv_len"] == out["kv_len"] + 1


def test_sampled_batches_mix_temperatures_and_drafts(model):
    shape, m = model
    rng = np.random.default_rng(3)
    k = [5, 0, 9]
    for r in range(3):
        prefilled(m, shape, r, 60 + 20 * r)
    cands = [rng.integers(0, shape.vocab, n).tolist() for n in k]
    parents = [heap(5, 2), None, heap(9, 4)]
    draft = rng.normal(size=(10, shape.vocab)).astype(np.float32)
    s = [dict(uniforms=rng.random(n + 1).astype(np.float32), temperature=t) for n, t in zip(k, (0.02, 1.0, 0.5))]
    s[2].update(draft_logits=draft, draft_temperature=2.0)
    outs = m.verify_tree_batch([0, 1, 2], cands, parents, s)
    for r in range(3):
        want = trees.sample_walk(m.logits(r).astype(np.float64), cands[r], s[r]["uniforms"], parents[r] or [],
                                 s[r]["temperature"], draft.astype(np.float64) if r == 2 else None, 2.0)
        assert (outs[r]["path"], outs[r]["correction_token"]) == want[:2]


def test_sampling_leaves_keep_logits_as_it_was(model):
    shape, m = model
    m.set_keep_logits(False)
    prefilled(m, shape)
    m.verify_sampled(0, [1, 2], [0.5, 0.5, 0.5])
    with pytest.raises(as2d.As2dError):
        m.logits(0)
    m.set_keep_logits(True)


def test_rollback_and_the_other_calls_after_a_tree(model):
    """Rollback into a committed tree, another tree over it, the static call."""
    shape, m = model
    _, L = prefilled(m, shape, 0, 90)
    y = greedy_stream(m, 0, 14)
    c, p = planted(y, shape.vocab, 1, 12)
    assert m.verify_tree(0, c, p)["accepted_len"] == 6
    m.rollback(0, L + 3, y[2])
    assert m.verify_static(0, y[3:6])["accepted_len"] == 3
    m.rollback(0, L + 3, y[2])
    c, p = planted(y[3:], shape.vocab, 2, 8)
    out = m.verify_tree(0, c, p)
    assert out["accepted_len"] == 4 and out["correction_token"] == y[7]


def test_non_finite_logits_keep_the_request(model):
    """A non-finite audio row makes every later logit of its request NaN."""
    shape, m = model
    prefilled(m, shape, 1)
    y = greedy_stream(m, 1, 3)
    prefilled(m, shape, 0)
    bad = torch.full((3, shape.n_kv_heads, shape.head_dim), float("nan"), device="cuda")
    m.write_kv(0, 0, bad, bad)
    state = m.state(0)
    u = [0.5] * 4
    for sampling in (None, [dict(uniforms=u), dict(uniforms=u, temperature=1e-3)]):
        s1 = m.state(1)
        with pytest.raises(as2d.As2dError) as e:
            m.verify_tree_batch([0, 1], [[1, 2, 3], y], [[-1, -1, 0], None], sampling)
        assert e.value.code == as2d.ENUMERIC
        assert m.state(0) == state
        assert m.state(1)[0] > s1[0]
        m.rollback(1, s1[0], s1[1])


def test_pass_refusals(model):
    shape, m = model
    _, L = prefilled(m, shape)
    state = m.state(0)

    def refused(code, f, *args, **kw):
        with pytest.raises(as2d.As2dError) as e:
            f(*args, **kw)
        assert e.value.code == code, e.value
        assert m.state(0) == state
    refused(as2d.EINVAL, m.verify_tree, 0, [1, 2], [-1, 1])
    refused(as2d.EINVAL, m.verify_tree, 0, [1, 2], [-1, -3])
    refused(as2d.EINVAL, m.verify_tree, 0, [1, 2], [-1])
    refused(as2d.EINVAL, m.verify_tree, 0, [1, shape.vocab], [-1, 0])
    refused(as2d.EINVAL, m.verify_tree, 0, list(range(32)), heap(32, 2))
    refused(as2d.EINVAL, m.verify_tree, 9, [1], [-1])
    refused(as2d.EINVAL, m.verify_tree_batch, [0, 0], [[1], [2]])
    refused(as2d.EINVAL, m.verify_tree_batch, [], [])
    refused(as2d.EINVAL, m.verify_sampled, 0, [1], [0.5])
    refused(as2d.EINVAL, m.verify_sampled, 0, [1], [0.5, 1.0])
    refused(as2d.EINVAL, m.verify_sampled, 0, [1], [float("nan"), 0.5])
    refused(as2d.EINVAL, m.verify_sampled, 0, [1], [0.5, 0.5], temperature=0.0)
    refused(as2d.EINVAL, m.verify_sampled, 0, [1], [0.5, 0.5], draft_logits=np.zeros((1, 3), np.float32))
    refused(as2d.EINVAL, m.verify_sampled, 0, [1], [0.5, 0.5], draft_logits=np.zeros((1, shape.vocab), np.float32),
            draft_temperature=-1.0)
    m.release(3)
    refused(as2d.ESTATE, m.verify_tree, 3, [1], [-1])
    m.prefill(2, np.zeros(0, np.uint16), np.zeros(510, np.int32))
    refused(as2d.ECAPACITY, m.verify_tree, 2, [1, 2], [-1, -1])
