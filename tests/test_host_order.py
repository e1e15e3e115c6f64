"""What the library's host code does, in which order, and after a call that
fails: against a HIP runtime that runs nothing (tests/host)."""
import ctypes
from dataclasses import replace

import numpy as np
import pytest

from paper_2609_37617_amd import as2d
from tests import host
from workload import TINY_BF16, gen

NARROW = replace(TINY_BF16, name="narrow", n_layers=2, hidden=128, ffn=64, vocab=128, qkv_bias=False)
OWN_STREAM = 1000   # the context's stream: the first one made


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = host.build(str(tmp_path_factory.mktemp("host")))
    saved, as2d._lib = as2d._lib, None
    try:
        yield as2d.load_library(path)
    finally:
        as2d._lib = saved


@pytest.fixture
def stub(lib, monkeypatch):
    monkeypatch.setattr(as2d, "_lib", lib)
    s = host.Stub(lib)
    s.reset()
    yield s
    s.reset()


@pytest.fixture
def model(stub):
    from workload.gen import _LIB_PATH
    import os
    if not os.path.exists(_LIB_PATH):
        gen.build()
    m = as2d.Model(NARROW, gen.make_weights(NARROW, 0, fmt="device"), max_requests=2, max_kv_len=256, max_k=31)
    m.lib.as2d_set_exec_mode(m.ctx, as2d.EXEC_EAGER)
    m.prefill(0, np.zeros(0, np.uint16), np.zeros(40, np.int32))
    stub.log()
    yield m
    m.close()


SAMPLED = dict(uniforms=np.full(5, 0.5, np.float32), parents=[-1, -1, 0, 0])
CANDS = [1, 2, 3, 4]


def launches(log):
    return [line.split()[1] for line in log if line.startswith("launch")]


def refused(code, f, *args, **kw):
    with pytest.raises(as2d.As2dError) as e:
        f(*args, **kw)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("with_draft", [False, True])
def test_a_sampled_pass_without_memory_launches_nothing(model, stub, with_draft):
    """The workspace is there before the pass starts, or the pass does not start."""
    s = dict(SAMPLED, draft_logits=np.zeros((4, NARROW.vocab), np.float32) if with_draft else None)
    state = model.state(0)
    stub.malloc_limit(64)
    refused(as2d.ENOMEM, model.verify_sampled, 0, CANDS, **s)
    assert launches(stub.log()) == [] and model.state(0) == state
    # the failed allocation is reported once, not by the next call's launches too
    assert stub.pending_error() == 0
    assert model.decode_one(0)["kv_len"] == state[0] + 1
    stub.malloc_limit(-1)
    stub.log()
    model.verify_sampled(0, CANDS, **s)
    log = stub.log()
    assert launches(log)[0] == "fill_zero" and launches(log)[-2:] == ["sample", "move_path"]
    assert log[-1] == f"sync {OWN_STREAM}"
    assert "malloc" not in log[log.index(f"launch embed {OWN_STREAM}"):]


@pytest.mark.parametrize("which", ["embed", "gemm", "attention", "finish", "tree_walk", "sample", "move_path"])
def test_a_pass_that_fails_is_waited_for(model, stub, which):
    """After an error nothing reads the descriptors or the caller's arrays any more, and the next call is as any other."""
    state = model.state(0)
    stub.fail_launch(which)
    refused(as2d.EHIP, model.verify_sampled, 0, CANDS, draft_logits=np.zeros((4, NARROW.vocab), np.float32), **SAMPLED)
    log = stub.log()
    failed = next(i for i, line in enumerate(log) if line.endswith("failed"))
    assert f"sync {OWN_STREAM}" in log[failed:] and model.state(0) == state and stub.pending_error() == 0
    stub.fail_launch("")
    assert model.verify_sampled(0, CANDS, **SAMPLED)["kv_len"] == state[0] + 1


@pytest.mark.parametrize("which", ["embed", "attention", "finish"])
def test_a_plain_pass_that_fails_is_waited_for(model, stub, which):
    state = model.state(0)
    stub.fail_launch(which)
    refused(as2d.EHIP, model.verify, 0, CANDS)
    assert stub.log()[-1] == f"sync {OWN_STREAM}" and model.state(0) == state
    stub.fail_launch("")
    assert model.verify(0, CANDS)["kv_len"] == state[0] + 1


# ---------------------------------------------------------------------------
# The sampler

class HostSampler:
    """Calls of a sampler on numbers as streams; the tensors are never read."""

    def __init__(self, lib):
        self.lib, self.h = lib, ctypes.c_void_p()
        assert lib.as2d_sampler_create(2, 3, 500, ctypes.byref(self.h)) == as2d.OK

    def verify(self, stream):
        some = 4096   # an address nothing reads
        a = as2d.SampleArgs(1, 2, 500, as2d.F32, some, 500, None, 0, some, None, None, some, None, 1.0, 0.0, some, some, some, None)
        return self.lib.as2d_sampler_verify(self.h, a, stream)


@pytest.fixture
def sampler(stub):
    s = HostSampler(stub.lib)
    stub.log()
    yield s
    stub.lib.as2d_sampler_free(s.h)


def order(log):
    """Records, waits and launches, without the event's number."""
    return [" ".join(w for i, w in enumerate(line.split()) if (line.split()[0], i) not in (("record", 1), ("wait", 2)))
            for line in log if line.split()[0] in ("record", "wait", "launch", "sync")]


def test_calls_on_several_streams_wait_for_the_last(sampler, stub):
    for s, want in ((0, []), (0, []), (12, ["record 0", "wait 12"]), (12, []), (0, ["record 12", "wait 0"])):
        assert sampler.verify(s) == as2d.OK
        assert order(stub.log()) == want + [f"launch sample {s}"]


def test_a_captured_call_does_not_hide_the_last_one_that_ran(sampler, stub):
    """A call on 11 still runs; one is captured on 12, which runs nothing: the
    next calls, on 12 and on 13, wait for 11's and for each other."""
    assert sampler.verify(11) == as2d.OK
    stub.log()
    stub.stream(12, capturing=True)
    assert sampler.verify(12) == as2d.OK
    assert order(stub.log()) == ["launch sample 12"]   # nothing recorded, nothing waited for
    stub.stream(12)
    assert sampler.verify(12) == as2d.OK
    assert order(stub.log()) == ["record 11", "wait 12", "launch sample 12"]
    assert sampler.verify(13) == as2d.OK
    assert order(stub.log()) == ["record 12", "wait 13", "launch sample 13"]


def test_the_first_call_captured(sampler, stub):
    stub.stream(12, capturing=True)
    assert sampler.verify(12) == as2d.OK
    assert sampler.verify(13) == as2d.OK
    assert order(stub.log()) == ["launch sample 12", "launch sample 13"]


def test_the_last_call_s_stream_is_captured_by_now(sampler, stub):
    """Its earlier work cannot be waited for (a record there would join the graph): refused, until the capture ends."""
    assert sampler.verify(11) == as2d.OK
    stub.log()
    stub.stream(11, capturing=True)
    assert sampler.verify(13) == as2d.ESTATE
    assert order(stub.log()) == []
    assert sampler.verify(11) == as2d.OK   # captured: behind its stream's earlier work wherever it is replayed there
    stub.stream(11)
    stub.log()
    assert sampler.verify(13) == as2d.OK
    assert order(stub.log()) == ["record 11", "wait 13", "launch sample 13"]


# ---------------------------------------------------------------------------
# Operators on one layer of a cache

SOME = 4096   # an address nothing reads


def rows(row=NARROW.n_q_heads * NARROW.head_dim, head=NARROW.head_dim):
    return as2d.Rows(SOME, row, head)


def attend(m, stream, n_rows=3, out=None):
    return m.call("as2d_tree_attention", 0, 0, n_rows, None, rows(), rows(), rows(), out or rows(), stream)


def put(m, stream):
    return m.call("as2d_write_kv", 0, 0, 0, 4, as2d.BF16, rows(), rows(), stream)


def test_operators_on_several_streams_wait_for_each_other(model, stub):
    assert put(model, 11) == as2d.OK
    assert attend(model, 11) == as2d.OK
    assert attend(model, 12) == as2d.OK
    assert put(model, 0) == as2d.OK
    assert order(stub.log()) == ["launch put_rows 11", "launch tree_attention 11", "record 11", "wait 12", "launch tree_attention 12",
                                 "record 12", "wait 0", "launch put_rows 0"]
    model.decode_one(0)
    assert order(stub.log())[:2] == ["sync 0", f"launch embed {OWN_STREAM}"]
    model.decode_one(0)
    assert order(stub.log())[0] == f"launch embed {OWN_STREAM}"   # waited for once


def test_an_operator_s_stream_that_is_captured_by_now(model, stub):
    """Neither an event of it nor a host wait may reach into the caller's
    capture: what would have to wait is refused, and the capture goes on."""
    assert put(model, 11) == as2d.OK
    stub.stream(11, capturing=True)
    stub.log()
    state = model.state(0)
    assert attend(model, 12) == as2d.ESTATE
    assert attend(model, 11) == as2d.ESTATE
    for f, args in ((model.decode_one, (0,)), (model.verify, (0, CANDS)), (model.verify_tree, (0, CANDS)),
                    (model.verify_static, (0, CANDS)), (model.read_kv, (0, 0, 8)), (model.set_stream, (13,)),
                    (lambda: model.verify_sampled(0, CANDS, **SAMPLED), ()),
                    (model.prefill, (0, np.zeros(0, np.uint16), np.zeros(5, np.int32)))):
        refused(as2d.ESTATE, f, *args)
    assert order(stub.log()) == [] and model.state(0) == state
    stub.stream(11)
    assert attend(model, 12) == as2d.OK
    assert order(stub.log()) == ["record 11", "wait 12", "launch tree_attention 12"]
    model.decode_one(0)
    assert order(stub.log())[0] == "sync 12"


def test_streams_restricted_by_a_mask_are_refused(model, sampler, stub):
    """As as2d_set_stream refuses them: the library never runs on one."""
    stub.stream(14, masked=True)
    stub.log()
    refused(as2d.EINVAL, model.set_stream, 14)
    assert attend(model, 14) == put(model, 14) == sampler.verify(14) == as2d.EINVAL
    assert stub.log() == []
    assert attend(model, 15) == put(model, 15) == sampler.verify(15) == as2d.OK
    assert order(stub.log()) == ["launch tree_attention 15", "launch put_rows 15", "launch sample 15"]


@pytest.mark.parametrize("row,head,n_rows,good", [
    ("nq d", "d", 3, True), ("nq d + 5", "d", 3, True), ("d", "3 d", 3, True), ("d + 1", "3 d + 3", 3, True),   # nested
    ("0", "d", 1, True), ("d", "d", 1, True),                                     # one row: its stride is not used
    ("0", "d", 3, False), ("nq d", "0", 3, False), ("nq d", "d - 1", 3, False),   # a dimension over itself
    ("d", "d", 3, False), ("d", "d + 1", 3, False), ("nq d - 1", "d", 3, False),   # one over the other
    ("d", "2 d", 3, False), ("d", "2 d", 2, True),                                # heads past two rows, not three
    ("2 d", "2 d", 3, False), ("9223372036854775807", "d", 3, True), ("d", "9223372036854775807", 3, True),
    ("9223372036854775807", "9223372036854775807", 3, False)])
def test_an_output_whose_rows_and_heads_overlap_is_refused(model, stub, row, head, n_rows, good):
    names = {"nq": NARROW.n_q_heads, "d": NARROW.head_dim}

    def value(text):
        return eval(text.replace("nq d", "nq * d").replace("2 d", "2 * d").replace("3 d", "3 * d"), names)
    rc = attend(model, 11, n_rows, rows(value(row), value(head)))
    assert rc == (as2d.OK if good else as2d.EINVAL)
    assert launches(stub.log()) == (["tree_attention"] if good else [])


# ---------------------------------------------------------------------------
# The binding

class Tensor:
    """What the binding asks of a device tensor."""
    is_cuda = True

    def __init__(self, shape, dtype, device=0):
        self.shape, self.dtype, self.device = tuple(shape), dtype, device

    def get_device(self):
        return self.device

    def data_ptr(self):
        return SOME

    def is_contiguous(self):
        return True

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def new_empty(self, shape, dtype=None):
        return Tensor(shape if isinstance(shape, tuple) else (shape,), dtype or self.dtype, self.device)


def test_tensors_of_another_device_are_refused(model, stub):
    """The default stream is the null handle on every device: on tensors of
    another one the library would run its kernels on its own."""
    torch = pytest.importorskip("torch")
    bf16, nq, nkv, d = torch.bfloat16, NARROW.n_q_heads, NARROW.n_kv_heads, NARROW.head_dim
    sampler = as2d.Sampler(2, 3, 500)

    def calls(other, which=None):
        def at(name):
            return other if which in (None, name) else 0
        q, out = Tensor((3, nq, d), bf16, at("q")), Tensor((3, nq, d), bf16, at("out"))
        k, v = Tensor((3, nkv, d), bf16, at("k")), Tensor((3, nkv, d), bf16, at("v"))
        yield "attention", lambda: model.tree_attention(0, 0, q, k, v, out=out, stream=0)
        yield "write", lambda: model.write_kv(0, 0, k, v, stream=0)
        t, dr = Tensor((2, 3, 500), torch.float32, at("logits")), Tensor((2, 3, 500), torch.float32, at("draft"))
        c, u = Tensor((2, 2), torch.int32, at("cands")), Tensor((2, 3), torch.float32, at("uniforms"))
        yield "sampler", lambda: sampler.verify(t, c, u, draft_logits=dr, stream=0)
    stub.log()
    for _, f in calls(1):
        refused(as2d.EINVAL, f)
    for which, ops in (("q", ["attention"]), ("out", ["attention"]), ("k", ["attention", "write"]), ("v", ["attention", "write"]),
                       ("logits", ["sampler"]), ("draft", ["sampler"]), ("cands", ["sampler"]), ("uniforms", ["sampler"])):
        for op, f in calls(1, which):
            if op in ops:
                refused(as2d.EINVAL, f)
    assert stub.log() == []
    for _, f in calls(0):
        f()
    assert launches(stub.log()) == ["tree_attention", "put_rows", "sample"]
    sampler.close()


def test_the_device_is_the_one_at_creation(model, stub):
    """Another current device later changes nothing; streams of another device are refused."""
    stub.lib.hipSetDevice(1)
    torch = pytest.importorskip("torch")
    sampler = as2d.Sampler(1, 0, 500)
    assert (model.device, sampler.device) == (0, 1)
    t, u = Tensor((1, 1, 500), torch.float32, 1), Tensor((1, 1), torch.float32, 1)
    refused(as2d.EINVAL, sampler.verify, t, None, u, stream=11)   # a stream of device 0
    stub.stream(16, device=1)
    sampler.verify(t, None, u, stream=16)
    k = Tensor((3, NARROW.n_kv_heads, NARROW.head_dim), torch.bfloat16)
    refused(as2d.EINVAL, model.write_kv, 0, 0, k, k, stream=16)
    model.write_kv(0, 0, k, k, stream=11)
    assert stub.lib.stub_device() == 1
    sampler.close()


def test_the_default_stream_during_a_capture_it_takes_part_in(model, sampler, stub):
    """The runtime gives an error, and no status, of the default stream while a stream that it synchronises with is captured."""
    assert put(model, 0) == as2d.OK and sampler.verify(0) == as2d.OK
    stub.stream(0, capturing=True)
    stub.log()
    state = model.state(0)
    assert attend(model, 12) == sampler.verify(12) == as2d.ESTATE
    refused(as2d.ESTATE, model.decode_one, 0)
    assert order(stub.log()) == [] and model.state(0) == state and stub.pending_error() == 0
    stub.stream(0)
    assert attend(model, 12) == sampler.verify(12) == as2d.OK
    assert order(stub.log()) == ["record 0", "wait 12", "launch tree_attention 12", "record 0", "wait 12", "launch sample 12"]
