"""The operators on trees of drafted tokens, as cases that can be timed and checked.

attention   ``Model.tree_attention``: one layer's attention of the rows of a
            candidate tree (the pending root and its drafted descendants) over
            a request's cache.  A row sees every committed position and, of
            the tree, its ancestors and itself.
sampling    ``Sampler.verify``: the candidates of a tree tested against the
            target's probabilities with given random numbers, and the token
            that follows the accepted path.

Cases go over the head layouts of the model shapes this repository names,
cache lengths from a short window to a full slot, chains and trees of one to
32 rows, float32 and bfloat16, small to full vocabularies, candidates with and
without a drafter's distribution, and rows that are not a multiple of 16 bytes
apart.
"""
import collections
import math

import numpy as np
import torch

own = False   # True: the framework's calls; False: plain torch

Heads = collections.namedtuple("Heads", "n_q n_kv dim")
HEADS = {"tiny": Heads(4, 2, 64), "0.5b": Heads(14, 2, 64), "3b": Heads(16, 2, 128), "7b": Heads(28, 4, 128)}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCABS = [4096, 32001, 50257, 151936, 152064]
LONGEST = 32704   # positions a listed or drawn cache holds, at most


def _attention(name, heads, dtype, keys, rows, branch):
    return {"name": name, "op": "attention", "heads": heads, "dtype": dtype, "keys": keys, "rows": rows, "branch": branch}


def _sampling(name, requests, vocab, k, branch, draft, dtype, pad, temperature):
    return {"name": name, "op": "sampling", "requests": requests, "vocab": vocab, "k": k, "branch": branch,
            "draft": draft, "dtype": dtype, "pad": pad, "temperature": temperature}


def listed():
    return [
        # the smallest model in use, float32: launches and latency
        _attention("attn-tiny-f32", "tiny", "f32", 144, 5, 2),
        # one row: a draft head's single-token step over a drafter's cache
        _attention("attn-0.5b-one", "0.5b", "bf16", 290, 1, 1),
        # an ASR window (30 s of audio), eight candidates, two a node
        _attention("attn-7b-asr", "7b", "bf16", 782, 9, 2),
        # the middle of a conversation, a wider tree
        _attention("attn-3b-mid", "3b", "bf16", 2481, 17, 3),
        # five minutes of audio, the fullest tree
        _attention("attn-7b-long", "7b", "bf16", 7564, 32, 4),
        # the longest slot
        _attention("attn-7b-slot", "7b", "bf16", LONGEST, 32, 2),
        # the smallest vocabulary in use, a short chain without a drafter's distribution
        _sampling("sample-tiny", 1, 4096, 4, 1, False, "f32", 0, 1.0),
        # no candidate ready: one token drawn from the target
        _sampling("sample-one", 1, 152064, 0, 1, False, "f32", 0, 0.7),
        # the usual call: a chain of eight from published text
        _sampling("sample-chain", 1, 152064, 8, 1, False, "f32", 0, 1.0),
        # a chain of eight with the drafter's logits
        _sampling("sample-draft", 1, 151936, 8, 1, True, "f32", 0, 0.8),
        # trees with the drafter's logits, an odd vocabulary, rows at odd addresses
        _sampling("sample-tree-bf16", 4, 50257, 15, 3, True, "bf16", 3, 1.0),
        # a serving batch
        _sampling("sample-batch", 16, 152064, 8, 2, True, "f32", 0, 1.0),
    ]


def draw(rng):
    """One more case of the ranges above."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    branch = rng.choice([1, 1, 2, 2, 3, 4, 8])
    if rng.random() < 0.5:
        heads = rng.choice(list(HEADS))
        keys = log_int(1, 8192 if heads == "tiny" else LONGEST)
        return dict(op="attention", heads=heads, dtype="f32" if heads == "tiny" else "bf16", keys=keys,
                    rows=rng.randint(1, 32), branch=branch)
    requests, k = log_int(1, 16), rng.randint(0, 31)
    vocab = rng.choice(VOCABS + [log_int(16, 152064), log_int(16, 152064)])
    while requests * (k + 1) > 100:   # no more to read than the largest case above
        requests -= 1
    return dict(op="sampling", requests=requests, vocab=vocab, k=k, branch=branch, draft=rng.random() < 0.5,
                dtype=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 1, 3, 64]),
                temperature=round(rng.uniform(0.3, 1.5), 2))


def _parents(k, branch):
    """A tree of k candidates with `branch` children a node, level by level: the parent of each, -1 for the root."""
    return [i // branch - 1 for i in range(k)]


def _generator(*key):
    seed = 0x243F6A88
    for v in key:
        seed = (seed * 1000003 ^ int(v)) & 0x7FFFFFFFFFFF
    return torch.Generator(device="cuda").manual_seed(seed)


# ---------------------------------------------------------------------------
# Inputs

def _attention_inputs(case, seed):
    """Queries, keys and values of the rows [rows, heads, dim], those of the cache [keys, heads, dim] in float32.
    Scores reach a few units, so that some keys carry most of the weight."""
    h, t = HEADS[case["heads"]], TYPES[case["dtype"]]
    g = _generator(1, seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    return {"q": (1.5 * normal(case["rows"], h.n_q, h.dim)).to(t), "k": normal(case["rows"], h.n_kv, h.dim).to(t),
            "v": normal(case["rows"], h.n_kv, h.dim).to(t),
            "K": normal(case["keys"], h.n_kv, h.dim), "V": normal(case["keys"], h.n_kv, h.dim)}


def _gumbel(g, *shape):
    u = torch.rand(shape, generator=g, device="cuda").clamp_(1e-20, 1 - 1e-7)
    return -torch.log(-torch.log(u))


def _rows_of(values, pad):
    """`values` [n, rows, vocab] as a view of rows that are `pad` elements further apart."""
    n, rows, vocab = values.shape
    if not pad:
        return values
    return torch.empty((n, rows, vocab + pad), dtype=values.dtype, device="cuda")[:, :, :vocab].copy_(values)


def _sampling_inputs(case, seed):
    """Target logits [n, k + 1, vocab] with a few likely tokens a row, the drafter's (the target's and noise), candidates
    drawn from the drafter's distribution at their parent, and the random numbers [n, k + 1]."""
    n, k, vocab, t = case["requests"], case["k"], case["vocab"], TYPES[case["dtype"]]
    g = _generator(2, seed)
    target = 2.0 * torch.randn((n, k + 1, vocab), generator=g, device="cuda")
    likely = torch.randint(vocab, (n, k + 1, 6), generator=g, device="cuda")
    target.scatter_add_(2, likely, 8.0 + 4.0 * torch.rand((n, k + 1, 6), generator=g, device="cuda"))
    draft = target + 0.7 * torch.randn((n, k + 1, vocab), generator=g, device="cuda")
    cands = torch.zeros((n, k), dtype=torch.int32, device="cuda")
    for i, p in enumerate(_parents(k, case["branch"])):
        cands[:, i] = (draft[:, p + 1] / case["temperature"] + _gumbel(g, n, vocab)).argmax(-1).int()
    return {"target": _rows_of(target.to(t), case["pad"]),
            "draft": _rows_of(draft.to(t), case["pad"]) if case["draft"] else None,
            "cands": cands, "uniforms": torch.rand((n, k + 1), generator=g, device="cuda")}


# ---------------------------------------------------------------------------
# What a program holds between calls: a loaded model with its slots, a sampler

SLOTS = 4
_models, _samplers = collections.OrderedDict(), {}


class _Served:
    """A one-layer model of these heads: its requests' caches are what the operator reads."""

    def __init__(self, heads, dtype, capacity):
        from paper_2609_37617_amd import as2d
        Shape = collections.namedtuple("Shape", "n_layers hidden n_q_heads n_kv_heads head_dim ffn vocab rope_theta "
                                                "rms_eps dtype qkv_bias")
        hidden, ffn, vocab = 128, 64, 128
        shape = Shape(1, hidden, heads.n_q, heads.n_kv, heads.dim, ffn, vocab, 1e6, 1e-6,
                      as2d.F32 if dtype == "f32" else as2d.BF16, False)
        rng, es = np.random.default_rng(0), np.float32 if dtype == "f32" else np.uint16

        def matrix(rows, cols):
            w = (0.02 * rng.standard_normal((rows, cols))).astype(np.float32)
            return w if es is np.float32 else (w.view(np.uint32) >> 16).astype(np.uint16)
        one, qd, kvd = np.ones(hidden, np.float32), heads.n_q * heads.dim, heads.n_kv * heads.dim
        tensors = [matrix(vocab, hidden), one, matrix(qd, hidden), matrix(kvd, hidden), matrix(kvd, hidden),
                   matrix(hidden, qd), one, matrix(ffn, hidden), matrix(ffn, hidden), matrix(hidden, ffn), one,
                   matrix(vocab, hidden)]
        self.model = as2d.Model(shape, tensors, max_requests=SLOTS, max_kv_len=capacity, max_k=31)
        self.next = 0


def _served(case):
    """The loaded model of these heads with slots long enough, the latest few kept."""
    capacity = min(32768, (case["keys"] + 32 + 2047) // 2048 * 2048)
    key = (HEADS[case["heads"]], case["dtype"], capacity)
    if key not in _models:
        while len(_models) >= 2:
            _models.popitem(last=False)[1].model.close()
        _models[key] = _Served(*key)
    _models.move_to_end(key)
    return _models[key]


def _sampler(case):
    from paper_2609_37617_amd import as2d
    key = (16, 31, 152064)   # requests, candidates and vocabulary at most
    if key not in _samplers:
        _samplers[key] = as2d.Sampler(*key)
    return _samplers[key]


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    if case["op"] == "sampling":
        s.__dict__.update(_sampling_inputs(case, seed))
        s.parents = _parents(case["k"], case["branch"])
        s.parent_rows = torch.tensor([p + 1 for p in s.parents], dtype=torch.int64, device="cuda")
        if own:
            s.sampler = _sampler(case)
        return s
    x = _attention_inputs(case, seed)
    s.q, s.k, s.v, s.parents = x["q"], x["k"], x["v"], _parents(case["rows"] - 1, case["branch"])
    if own:
        served = _served(case)
        s.model, s.slot = served.model, served.next
        served.next = (served.next + 1) % SLOTS
        s.model.prefill(s.slot, np.zeros(0, np.uint16), np.zeros(case["keys"], np.int32))
        s.model.write_kv(s.slot, 0, x["K"], x["V"])
    else:
        h, n = HEADS[case["heads"]], case["keys"] + case["rows"]
        s.K, s.V = (torch.zeros((h.n_kv, n, h.dim), device="cuda") for _ in range(2))
        s.K[:, :case["keys"]], s.V[:, :case["keys"]] = x["K"].transpose(0, 1), x["V"].transpose(0, 1)
        s.visible = torch.ones((case["rows"], n), dtype=torch.bool, device="cuda")
        s.visible[:, case["keys"]:] = torch.from_numpy(_tree_mask(case)).cuda()
    return s


def _tree_mask(case):
    """[rows, rows]: row i sees tree row j."""
    m = np.eye(case["rows"], dtype=bool)
    for i, p in enumerate(_parents(case["rows"] - 1, case["branch"])):
        m[i + 1] |= m[p + 1]
    return m


def run(s):
    if s.case["op"] == "attention":
        return s.model.tree_attention(s.slot, 0, s.q, s.k, s.v, s.parents) if own else _plain_attention(s)
    if own:
        return s.sampler.verify(s.target, s.cands, s.uniforms, parents=s.parents, draft_logits=s.draft,
                                temperature=s.case["temperature"])
    return _plain_sampling(s)


# ---------------------------------------------------------------------------
# The plain forms

def _plain_attention(s):
    """Rows of the query heads that share a KV head as one product, float32."""
    (rows, n_q, dim), n_kv, keys = s.q.shape, s.k.shape[1], s.case["keys"]
    s.K[:, keys:], s.V[:, keys:] = s.k.float().transpose(0, 1), s.v.float().transpose(0, 1)
    q = s.q.float().view(rows, n_kv, n_q // n_kv, dim).permute(1, 2, 0, 3).reshape(n_kv, -1, dim)
    w = torch.bmm(q, s.K.transpose(1, 2)).div_(math.sqrt(dim)).view(n_kv, n_q // n_kv, rows, -1)
    w.masked_fill_(~s.visible, -math.inf)
    w = torch.exp(w - w.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    o = torch.bmm(w.view(n_kv, -1, w.shape[-1]), s.V)
    return o.view(n_kv, n_q // n_kv, rows, dim).permute(2, 0, 1, 3).reshape(rows, n_q, dim).to(s.q.dtype)


def _log_softmax(logits, temperature):
    x = logits.double() / temperature
    x = x - x.amax(-1, keepdim=True)
    return x - torch.log(torch.exp(x).sum(-1, keepdim=True))


def _plain_sampling(s):
    """All requests at once, the candidates in order (each may depend on the one before), in 64 bits: a random
    number may lie next to a border."""
    n, k = s.cands.shape
    dev, every = s.cands.device, torch.arange(n, device=s.cands.device)
    lp = _log_softmax(s.target, s.case["temperature"])
    p, u = torch.exp(lp), s.uniforms.double()
    q = torch.exp(_log_softmax(s.draft, s.case["temperature"])) if s.draft is not None else None
    cands = s.cands.long()
    at, left, mass = torch.zeros(n, dtype=torch.int64, device=dev), p[:, 0], torch.ones(n, dtype=torch.float64, device=dev)
    accepted, path = torch.zeros(n, dtype=torch.int64, device=dev), torch.full((n, k), -1, dtype=torch.int64, device=dev)
    for i in range(k):
        x = cands[:, i]
        qx = 1.0 if q is None else q[every, at, x]
        tested = at == s.parent_rows[i]
        yes = tested & (u[:, i] * mass * qx < left[every, x])
        less = left.scatter(1, x[:, None], 0.0) if q is None else (left - mass[:, None] * q[every, at]).clamp_(min=0.0)
        left = torch.where(yes[:, None], p[:, i + 1], torch.where(tested[:, None], less, left))
        mass = torch.where(yes, 1.0, torch.where(tested, less.sum(-1), mass))
        path = torch.where(yes[:, None] & (torch.arange(k, device=dev) == accepted[:, None]), i, path)
        accepted, at = accepted + yes, torch.where(yes, i + 1, at)
    left = torch.where((mass > 0)[:, None], left, p[every, at])
    run = left.cumsum(-1)
    token = (run <= (u[:, k] * run[:, -1])[:, None]).sum(-1).clamp_(max=p.shape[-1] - 1)
    logp = torch.cat([lp[every[:, None], s.parent_rows[None, :], cands], lp[every, at, token][:, None]], 1)
    return {"accepted": accepted.int(), "path": path.int(), "token": token.int(), "logp": logp.float()}


# ---------------------------------------------------------------------------

def work(case):
    """Cache read once at the 4 bytes an element takes in it, rows read and written once; logits read once (a
    drafter's only for rows with children), a few numbers written."""
    if case["op"] == "attention":
        h, n, keys = HEADS[case["heads"]], case["rows"], case["keys"]
        es = 4 if case["dtype"] == "f32" else 2
        pairs = n * keys + int(_tree_mask(case).sum())
        return {"bytes": 8 * h.n_kv * h.dim * (keys + n) + es * n * h.dim * (2 * h.n_q + 2 * h.n_kv),
                "flops": 4 * h.n_q * h.dim * pairs}
    es = 4 if case["dtype"] == "f32" else 2
    rows = case["k"] + 1 + (len(set(_parents(case["k"], case["branch"]))) if case["draft"] else 0)
    n = case["requests"]
    return {"bytes": n * (rows * case["vocab"] * es + 16 * (case["k"] + 1)), "flops": 4 * n * rows * case["vocab"]}


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits

def exact(case, seed):
    return _exact_attention(case, seed) if case["op"] == "attention" else _exact_sampling(case, seed)


def _exact_attention(case, seed):
    h = HEADS[case["heads"]]
    x = {name: t.double() for name, t in _attention_inputs(case, seed).items()}
    keys, values, mask = torch.cat([x["K"], x["k"]]), torch.cat([x["V"], x["v"]]), _tree_mask(case)
    out = torch.empty_like(x["q"])
    for i in range(case["rows"]):
        sees = list(range(case["keys"])) + [case["keys"] + int(j) for j in np.flatnonzero(mask[i])]
        sees = torch.tensor(sees, device="cuda")
        for g in range(h.n_kv):
            kk, vv = keys[sees, g], values[sees, g]
            heads = slice(g * (h.n_q // h.n_kv), (g + 1) * (h.n_q // h.n_kv))
            w = torch.softmax(x["q"][i, heads] @ kk.T / math.sqrt(h.dim), -1)
            out[i, heads] = w @ vv
    return out


def _exact_sampling(case, seed):
    """One request at a time, as the rule is told: walk down from the root, try the children in order."""
    x, k, parents = _sampling_inputs(case, seed), case["k"], _parents(case["k"], case["branch"])
    out = []
    for r in range(case["requests"]):
        def dist(logits, row):
            z = logits[r, row].double().cpu().numpy() / case["temperature"]
            z = z - z.max()
            return z - np.log(np.exp(z).sum())
        u, cands = x["uniforms"][r].double().cpu().numpy(), x["cands"][r].cpu().numpy()
        logs = {row: dist(x["target"], row) for row in range(k + 1)}
        node, path, i = -1, [], 0
        left, mass = np.exp(logs[0]), 1.0
        while i < k:
            if parents[i] != node:
                i += 1
                continue
            token = cands[i]
            q = np.exp(dist(x["draft"], node + 1)) if case["draft"] else np.eye(1, case["vocab"], token)[0]
            if u[i] * mass * q[token] < left[token]:
                path.append(i)
                node, left, mass = i, np.exp(logs[i + 1]), 1.0
            elif case["draft"]:
                left = np.maximum(left - mass * q, 0.0)
                mass = left.sum()
            else:
                left[token] = 0.0
                mass = left.sum()
            i += 1
        if not mass > 0:
            left = np.exp(logs[node + 1])
        run = np.cumsum(left)
        token = int(np.argmax(run > u[k] * run[-1]))
        logp = [logs[p + 1][t] for p, t in zip(parents, cands)] + [logs[node + 1][token]]
        out.append((len(path), path + [-1] * (k - len(path)), token, logp))
    return {"accepted": torch.tensor([o[0] for o in out], dtype=torch.int32),
            "path": torch.tensor([o[1] for o in out], dtype=torch.int32).view(len(out), k),
            "token": torch.tensor([o[2] for o in out], dtype=torch.int32),
            "logp": torch.tensor([o[3] for o in out], dtype=torch.float64)}
