"""Trees of candidates without a GPU: the oracle's rules pinned, and the
refusals that need no device."""
import ctypes

import numpy as np
import pytest

from oracle import trees


@pytest.fixture(scope="module")
def lib():
    from tests.harness import ensure_built
    ensure_built()
    from paper_2609_37617_amd import as2d
    return as2d.load_library()


def test_masks_and_depths():
    parents = [-1, -1, 0, 0, 2, 1]
    m = trees.visible(parents)
    assert [np.flatnonzero(r).tolist() for r in m] == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 4], [0, 1, 3, 5], [0, 2, 6]]
    assert trees.depths(parents) == [0, 1, 1, 2, 2, 3, 2]
    assert trees.depths(trees.chain(3)) == [0, 1, 2, 3]


def test_a_chain_is_causal_attention():
    from oracle import attention
    rng = np.random.default_rng(0)
    q, K, V = rng.normal(size=(3, 4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    k, v = rng.normal(size=(3, 2, 8)), rng.normal(size=(3, 2, 8))
    got = trees.attention(q, K, V, k, v, trees.chain(2))
    for i in range(3):
        kk, vv = np.concatenate([K, k[:i + 1]]), np.concatenate([V, v[:i + 1]])
        for h in range(4):
            s = kk[:, h // 2] @ q[i, h] / np.sqrt(8)
            p = np.exp(s) / np.exp(s).sum()
            assert np.allclose(got[i, h], p @ vv[:, h // 2], rtol=1e-12)
    assert callable(attention)


def test_greedy_walk():
    # the root says 5: candidates 0 and 2 have it, the first is taken; its child 3 has 7
    assert trees.greedy_walk([5, 7, 9, 1, 4], [5, 6, 5, 7], [-1, -1, -1, 0]) == ([0, 3], 4)
    assert trees.greedy_walk([8, 7, 9, 1, 4], [5, 6, 5, 7], [-1, -1, -1, 0]) == ([], 8)
    assert trees.greedy_walk([3], [], []) == ([], 3)


def test_masses_in_closed_form():
    """max(max(p - a q, 0) - b q, 0) = max(p - (a + b) q, 0), so a node's
    state after m rejections is one number: C_1 = 1, C_{m+1} = C_m + S_m."""
    rng = np.random.default_rng(1)
    for _ in range(50):
        p, q = rng.dirichlet(np.full(20, 0.3)), rng.dirichlet(np.full(20, 0.3))
        left, mass, cut = p, 1.0, 0.0
        for _ in range(4):
            left = np.maximum(left - mass * q, 0.0)
            cut += mass
            mass = left.sum()
            assert np.allclose(left, np.maximum(p - cut * q, 0.0), atol=1e-15)


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("branch", [1, 2])
def test_the_first_token_follows_the_target(with_draft, branch):
    """The first committed token's frequencies over 20,000 calls are the
    target's: each within five standard deviations."""
    rng = np.random.default_rng(2)
    V, k, n = 5, 3, 20000
    target, draft = rng.normal(size=(k + 1, V)) * 1.5, rng.normal(size=(k + 1, V)) * 1.5
    parents = [i // branch - 1 for i in range(k)]
    p, qs = np.exp(trees.log_softmax(target[0], 1.0)), [np.exp(trees.log_softmax(d, 1.0)) for d in draft]
    count = np.zeros(V)
    for _ in range(n):
        cands = [rng.choice(V, p=qs[parents[i] + 1]) for i in range(k)]
        path, token, _ = trees.sample_walk(target, cands, rng.random(k + 1), parents, draft=draft if with_draft else None)
        count[cands[path[0]] if path else token] += 1
    assert (np.abs(count / n - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()


def test_null_arguments(lib):
    from paper_2609_37617_amd import as2d
    out, h = as2d.VerifyOut(), ctypes.c_void_p()
    assert lib.as2d_verify_tree(None, 0, None, None, 0, ctypes.byref(out), None) == as2d.EINVAL
    assert lib.as2d_verify_sampled(None, 0, None, None, 0, None, ctypes.byref(out), None) == as2d.EINVAL
    assert lib.as2d_verify_tree_batch(None, 1, None, None, None, None, None, None, None) == as2d.EINVAL
    assert lib.as2d_tree_attention(None, 0, 0, 1, None, None, None, None, None, None) == as2d.EINVAL
    assert lib.as2d_write_kv(None, 0, 0, 0, 1, 0, None, None, None) == as2d.EINVAL
    assert lib.as2d_sampler_verify(None, None, None) == as2d.EINVAL
    assert lib.as2d_sampler_free(None) == as2d.EINVAL
    assert lib.as2d_sampler_last_error(None) == b"null sampler"
    assert lib.as2d_sampler_create(1, 1, 1, None) == as2d.EINVAL
    for bad in ((0, 4, 100), (5000, 4, 100), (1, -1, 100), (1, 32, 100), (1, 4, 0), (1, 4, (1 << 24) + 1)):
        assert lib.as2d_sampler_create(*bad, ctypes.byref(h)) == as2d.EINVAL and not h.value, bad
        assert b"max_requests" in lib.as2d_sampler_last_error(None)


def test_structs_have_the_abi_s_layout():
    """Sizes and offsets of the C structs under the System V rules (8-byte
    pointers and int64, natural alignment)."""
    from paper_2609_37617_amd import as2d
    assert ctypes.sizeof(as2d.Sampling) == 32 and as2d.Sampling.uniforms.offset == 16
    assert ctypes.sizeof(as2d.Rows) == 24
    s = as2d.SampleArgs
    assert (s.logits.offset, s.draft_logits.offset, s.cands.offset, s.temperature.offset, s.accepted.offset,
            ctypes.sizeof(s)) == (16, 32, 48, 88, 104, 136)


def test_the_binding_refuses_host_tensors(lib):
    import torch
    from paper_2609_37617_amd import as2d
    with pytest.raises(as2d.As2dError) as e:
        as2d._on_device(torch.zeros(2), "q", torch.float32, (2,))
    assert e.value.code == as2d.EINVAL
