"""ctypes binding of libas2d.so (include/as2d.h).

Argument marshalling only: every step of the verification path runs in the
library's HIP kernels.  Importing this module does not touch the GPU;
loading the library fails loudly if it has not been built.  Tensors on the
device are torch's; a program that uses torch imports it before the library
is loaded (before the first Model or Sampler), since both bring a HIP runtime
and the first one serves the process.
"""
import ctypes
import os
from typing import List, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libas2d.so")

OK, EINVAL, ECAPACITY, ESTATE, EHIP, ENUMERIC, ENOMEM = 0, -1, -2, -3, -4, -5, -6
EXEC_EAGER, EXEC_GRAPH, EXEC_PERSISTENT = 0, 1, 2
F32, BF16 = 0, 1

# Every symbol include/as2d.h declares.
EXPORTS = ["as2d_load_weights", "as2d_prefill_kv", "as2d_verify", "as2d_decode_one",
           "as2d_verify_batch", "as2d_set_keep_logits", "as2d_get_logits", "as2d_get_row_tokens",
           "as2d_get_row_margins",
           "as2d_rollback", "as2d_get_state", "as2d_read_kv", "as2d_release_request",
           "as2d_set_exec_mode", "as2d_get_exec_info", "as2d_set_step_trace", "as2d_step_trace_read",
           "as2d_set_timing", "as2d_timing_read", "as2d_timing_reset", "as2d_time_gemm",
           "as2d_stream_bandwidth", "as2d_step_bytes", "as2d_free", "as2d_last_error",
           "as2d_cbuf_create", "as2d_cbuf_free", "as2d_cbuf_publish", "as2d_cbuf_snapshot",
           "as2d_cbuf_read", "as2d_cbuf_n_records", "as2d_cbuf_get_record", "as2d_cursor_init",
           "as2d_cursor_propose", "as2d_cursor_update", "as2d_verify_from_buffer", "as2d_run_decoupled",
           "as2d_set_stream", "as2d_set_cu_budget", "as2d_verify_static",
           "as2d_verify_tree", "as2d_verify_sampled", "as2d_verify_tree_batch", "as2d_tree_attention",
           "as2d_write_kv", "as2d_sampler_create", "as2d_sampler_free", "as2d_sampler_verify",
           "as2d_sampler_last_error"]


class Config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("rope_theta", ctypes.c_float), ("rms_eps", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("qkv_bias", ctypes.c_int32),
                ("max_requests", ctypes.c_int32), ("max_kv_len", ctypes.c_int32),
                ("max_k", ctypes.c_int32)]


class VerifyOut(ctypes.Structure):
    _fields_ = [("accepted_len", ctypes.c_int32), ("correction_token", ctypes.c_int32),
                ("kv_len", ctypes.c_int32), ("committed", ctypes.c_int32)]

    def as_dict(self):
        return dict(accepted_len=self.accepted_len, correction_token=self.correction_token,
                    kv_len=self.kv_len, committed=self.committed)


class CbufRecord(ctypes.Structure):
    _fields_ = [("first", ctypes.c_int64), ("count", ctypes.c_int32), ("source_id", ctypes.c_int32),
                ("producer_id", ctypes.c_int32), ("pad", ctypes.c_int32), ("offset", ctypes.c_int64),
                ("publish_ns", ctypes.c_int64), ("confidence", ctypes.c_float), ("pad2", ctypes.c_int32)]


class ReadCursorC(ctypes.Structure):
    _fields_ = [("cursor", ctypes.c_int64), ("floor", ctypes.c_int64), ("radius", ctypes.c_int32),
                ("pad", ctypes.c_int32)]


class Interval(ctypes.Structure):
    _fields_ = [("start_ns", ctypes.c_int64), ("end_ns", ctypes.c_int64), ("kind", ctypes.c_int32),
                ("tokens", ctypes.c_int32)]


class Sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_double), ("draft_temperature", ctypes.c_double),
                ("uniforms", ctypes.c_void_p), ("draft_logits", ctypes.c_void_p)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class SampleArgs(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("k", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("draft_logits", ctypes.c_void_p),
                ("draft_row_stride", ctypes.c_int64), ("cands", ctypes.c_void_p), ("parents", ctypes.c_void_p),
                ("ks", ctypes.c_void_p), ("uniforms", ctypes.c_void_p), ("temperatures", ctypes.c_void_p),
                ("temperature", ctypes.c_double), ("draft_temperature", ctypes.c_double), ("accepted", ctypes.c_void_p),
                ("path", ctypes.c_void_p), ("token", ctypes.c_void_p), ("logp", ctypes.c_void_p)]


class As2dError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"as2d error {code}: {msg}")
        self.code = code


_lib = None
_P = ctypes.c_void_p
_I = ctypes.c_int32


def load_library(path: str = LIB_PATH):
    """Load libas2d.so; raises if it is missing (no fallback path exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is not built; run __graft_entry__.build() "
                                f"or python paper_2609_37617_amd/build.py")
    lib = ctypes.CDLL(path)
    lib.as2d_load_weights.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(_P), _I, _P,
                                      ctypes.POINTER(_P)]
    lib.as2d_prefill_kv.argtypes = [_P, _I, _P, _I, _P, _I, ctypes.POINTER(_I), ctypes.POINTER(_I)]
    lib.as2d_verify.argtypes = [_P, _I, _P, _I, ctypes.POINTER(VerifyOut)]
    lib.as2d_verify_static.argtypes = [_P, _I, _P, _I, ctypes.POINTER(VerifyOut)]
    lib.as2d_decode_one.argtypes = [_P, _I, ctypes.POINTER(VerifyOut)]
    lib.as2d_verify_batch.argtypes = [_P, _I, _P, _P, _P, _P]
    lib.as2d_set_keep_logits.argtypes = [_P, _I]
    lib.as2d_get_logits.argtypes = [_P, _I, _P, _I, ctypes.POINTER(_I)]
    lib.as2d_get_row_tokens.argtypes = [_P, _I, _P, _I, ctypes.POINTER(_I)]
    lib.as2d_get_row_margins.argtypes = [_P, _I, _P, _I, ctypes.POINTER(_I)]
    lib.as2d_rollback.argtypes = [_P, _I, _I, _I]
    lib.as2d_get_state.argtypes = [_P, _I, ctypes.POINTER(_I), ctypes.POINTER(_I), ctypes.POINTER(_I)]
    lib.as2d_read_kv.argtypes = [_P, _I, _I, _P, _P, _I]
    lib.as2d_release_request.argtypes = [_P, _I]
    lib.as2d_set_exec_mode.argtypes = [_P, _I]
    lib.as2d_set_step_trace.argtypes = [_P, _I]
    lib.as2d_step_trace_read.argtypes = [_P, _P, ctypes.c_int64, ctypes.POINTER(_I), ctypes.POINTER(_I)]
    lib.as2d_get_exec_info.argtypes = [_P, ctypes.POINTER(_I), ctypes.POINTER(_I)]
    lib.as2d_set_timing.argtypes = [_P, _I]
    lib.as2d_timing_read.argtypes = [_P, _P, _P, _P, _I]
    lib.as2d_timing_reset.argtypes = [_P]
    lib.as2d_time_gemm.argtypes = [_P, _I, _I, _I, ctypes.POINTER(ctypes.c_double)]
    lib.as2d_stream_bandwidth.argtypes = [_P, ctypes.c_int64, _I, ctypes.POINTER(ctypes.c_double)]
    lib.as2d_step_bytes.argtypes = [_P, _I, ctypes.c_int64]
    lib.as2d_step_bytes.restype = ctypes.c_int64
    _L = ctypes.c_int64
    lib.as2d_cbuf_create.argtypes = [_L, ctypes.POINTER(_P)]
    lib.as2d_cbuf_free.argtypes = [_P]
    lib.as2d_cbuf_publish.argtypes = [_P, _P, _I, _I, _I, _L, _L, ctypes.c_float, ctypes.POINTER(_L)]
    lib.as2d_cbuf_snapshot.argtypes = [_P, ctypes.POINTER(_L)]
    lib.as2d_cbuf_read.argtypes = [_P, _L, _I, _P]
    lib.as2d_cbuf_n_records.argtypes = [_P, ctypes.POINTER(_L)]
    lib.as2d_cbuf_get_record.argtypes = [_P, _L, ctypes.POINTER(CbufRecord)]
    lib.as2d_cursor_init.argtypes = [ctypes.POINTER(ReadCursorC), _I]
    lib.as2d_cursor_propose.argtypes = [_P, ctypes.POINTER(ReadCursorC), _L, _I, _P, ctypes.POINTER(_I)]
    lib.as2d_cursor_update.argtypes = [_P, ctypes.POINTER(ReadCursorC), _L, _I, _I, _I]
    lib.as2d_verify_from_buffer.argtypes = [_P, _I, _P, ctypes.POINTER(ReadCursorC), _I, _I,
                                            ctypes.POINTER(VerifyOut), ctypes.POINTER(_I)]
    lib.as2d_run_decoupled.argtypes = [_P, _I, _P, _I, _P, _I, _I, _I, _I, _P, ctypes.POINTER(ReadCursorC), _P,
                                       _P, _I, ctypes.POINTER(_I), ctypes.POINTER(_L), ctypes.POINTER(_I)]
    lib.as2d_verify_tree.argtypes = [_P, _I, _P, _P, _I, ctypes.POINTER(VerifyOut), _P]
    lib.as2d_verify_sampled.argtypes = [_P, _I, _P, _P, _I, ctypes.POINTER(Sampling), ctypes.POINTER(VerifyOut), _P]
    lib.as2d_verify_tree_batch.argtypes = [_P, _I, _P, _P, _P, _P, ctypes.POINTER(Sampling), _P, _P]
    _R = ctypes.POINTER(Rows)
    lib.as2d_tree_attention.argtypes = [_P, _I, _I, _I, _P, _R, _R, _R, _R, _P]
    lib.as2d_write_kv.argtypes = [_P, _I, _I, _I, _I, _I, _R, _R, _P]
    lib.as2d_sampler_create.argtypes = [_I, _I, _I, ctypes.POINTER(_P)]
    lib.as2d_sampler_free.argtypes = [_P]
    lib.as2d_sampler_verify.argtypes = [_P, ctypes.POINTER(SampleArgs), _P]
    lib.as2d_sampler_last_error.argtypes = [_P]
    lib.as2d_sampler_last_error.restype = ctypes.c_char_p
    lib.as2d_set_stream.argtypes = [_P, _P]
    lib.as2d_set_cu_budget.argtypes = [_P, _I]
    lib.as2d_free.argtypes = [_P]
    lib.as2d_free.restype = None
    lib.as2d_last_error.argtypes = [_P]
    lib.as2d_last_error.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("as2d_free", "as2d_last_error", "as2d_step_bytes", "as2d_sampler_last_error"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _ptr(a: np.ndarray) -> int:
    return a.ctypes.data


def _refuse(what: str):
    raise As2dError(EINVAL, what)


_dtypes = {}


def _types() -> dict:
    """The library's type of each torch type it takes."""
    if not _dtypes:
        import torch
        _dtypes.update({torch.float32: F32, torch.bfloat16: BF16})
    return _dtypes


def _on_device(t, name: str, dtype, shape) -> int:
    """Checks a device tensor (torch) and returns its address."""
    if not getattr(t, "is_cuda", False):
        _refuse(f"{name}: a device tensor is wanted")
    if t.dtype != dtype:
        _refuse(f"{name}: {dtype} is wanted, not {t.dtype}")
    if t.shape != shape:
        _refuse(f"{name}: shape {tuple(shape)} is wanted, not {tuple(t.shape)}")
    return t.data_ptr()


def _dense(t, name: str, dtype, shape) -> int:
    p = _on_device(t, name, dtype, shape)
    if not t.is_contiguous():
        _refuse(f"{name}: a contiguous tensor is wanted")
    return p


def _rows(t, name: str, dtype, shape) -> Rows:
    p, stride = _on_device(t, name, dtype, shape), t.stride()
    if stride[2] != 1 and shape[2] > 1:
        _refuse(f"{name}: adjacent dimensions are wanted")
    return Rows(p, stride[0], stride[1])


def _current_device(lib) -> int:
    """The calling thread's device, from the runtime the library is linked to."""
    dev = _I()
    if lib.hipGetDevice(ctypes.byref(dev)) != 0:
        raise As2dError(EHIP, "no device")
    return dev.value


def _device_of(tensors, owner: int) -> int:
    """The tensors' device, which has to be that of the model or sampler: its
    kernels run there, and torch's default stream is the same handle on every
    device, so that the library could not tell."""
    for t in tensors:
        if t.get_device() != owner:
            _refuse(f"a tensor on device {t.get_device()}, the model or sampler is on {owner}")
    return owner


def _stream_of(device: int, stream: Optional[int]) -> int:
    """The given stream's handle, or torch's current stream of the device."""
    if stream is not None:
        return stream
    import torch
    return torch._C._cuda_getCurrentRawStream(device)


def _int32(values) -> np.ndarray:
    return np.ascontiguousarray(values, dtype=np.int32)


def _parents(parents, k: int):
    """A host array of k parents, or None (null: a chain)."""
    if parents is None:
        return None
    if len(parents) != k:
        _refuse(f"parents: {k} entries are wanted, not {len(parents)}")
    return (ctypes.c_int32 * max(k, 1))(*parents)


def _opt(a: Optional[np.ndarray]):
    return _ptr(a) if a is not None and a.size else None


class Model:
    """One library context: a loaded target model with its KV slots."""

    def __init__(self, shape, tensors: Sequence[np.ndarray], max_requests: int = 1,
                 max_kv_len: int = 1024, max_k: int = 8, stream: Optional[int] = None):
        """shape: workload.configs.ModelShape; tensors: the canonical list
        in the 'device' format of workload.gen.make_weights."""
        self.lib = load_library()
        self.device = _current_device(self.lib)
        self.shape = shape
        cfg = Config(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                     shape.ffn, shape.vocab, shape.rope_theta, shape.rms_eps, shape.dtype,
                     int(shape.qkv_bias), max_requests, max_kv_len, max_k)
        self.cfg = cfg
        self._keep = [np.ascontiguousarray(t) for t in tensors]
        arr = (_P * len(self._keep))(*[_ptr(t) for t in self._keep])
        ctx = _P()
        rc = self.lib.as2d_load_weights(ctypes.byref(cfg), arr, len(self._keep), stream, ctypes.byref(ctx))
        self._keep = None
        if rc != OK:
            raise As2dError(rc, self.lib.as2d_last_error(None).decode())
        self.ctx = ctx

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.as2d_free(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc):
        if rc != OK:
            raise As2dError(rc, self.lib.as2d_last_error(self.ctx).decode())

    def call(self, name, *args):
        """Raw call returning the status code (for error-path tests)."""
        return getattr(self.lib, name)(self.ctx, *args)

    def prefill(self, req: int, audio: np.ndarray, instr: Sequence[int]):
        audio = np.ascontiguousarray(audio)
        instr = np.ascontiguousarray(instr, dtype=np.int32)
        first, kv = _I(), _I()
        n_audio = audio.shape[0] if audio.size else 0
        self._check(self.lib.as2d_prefill_kv(self.ctx, req, _ptr(audio) if n_audio else None, n_audio,
                                             _ptr(instr) if len(instr) else None, len(instr),
                                             ctypes.byref(first), ctypes.byref(kv)))
        return first.value, kv.value

    def verify(self, req: int, cands: Sequence[int], k: Optional[int] = None) -> dict:
        c = np.ascontiguousarray(cands, dtype=np.int32)
        k = len(c) if k is None else k
        out = VerifyOut()
        self._check(self.lib.as2d_verify(self.ctx, req, _ptr(c) if c.size else None, k, ctypes.byref(out)))
        return out.as_dict()

    def verify_static(self, req: int, cands: Sequence[int]) -> dict:
        """as2d_verify_static: the same call with the pass's buffers in the
        library's static scratch array (allocates nothing)."""
        c = np.ascontiguousarray(cands, dtype=np.int32)
        out = VerifyOut()
        self._check(self.lib.as2d_verify_static(self.ctx, req, _ptr(c) if c.size else None, len(c),
                                                ctypes.byref(out)))
        return out.as_dict()

    def decode_one(self, req: int) -> dict:
        out = VerifyOut()
        self._check(self.lib.as2d_decode_one(self.ctx, req, ctypes.byref(out)))
        return out.as_dict()

    def verify_batch(self, reqs: Sequence[int], cands: Sequence[Sequence[int]]) -> List[dict]:
        n = len(reqs)
        r = np.ascontiguousarray(reqs, dtype=np.int32)
        ks = np.array([len(c) for c in cands], dtype=np.int32)
        flat = np.ascontiguousarray(np.concatenate([np.asarray(c, dtype=np.int32) for c in cands])
                                    if ks.sum() else np.zeros(1, np.int32), dtype=np.int32)
        outs = (VerifyOut * n)()
        self._check(self.lib.as2d_verify_batch(self.ctx, n, _ptr(r), _ptr(flat), _ptr(ks), outs))
        return [o.as_dict() for o in outs]

    def verify_tree(self, req: int, cands: Sequence[int], parents: Optional[Sequence[int]] = None) -> dict:
        """One pass over a tree of candidates (parents[i]: the candidate that
        candidate i follows, -1 the root; None: a chain), greedily verified.
        The result has the accepted candidates' numbers under "path"."""
        return self._tree([req], [cands], None if parents is None else [parents], None)[0]

    def verify_sampled(self, req: int, cands: Sequence[int], uniforms, parents: Optional[Sequence[int]] = None,
                       temperature: float = 1.0, draft_logits=None, draft_temperature: float = 0.0) -> dict:
        """verify_tree with the candidates tested by sampling: `uniforms` has
        one number in [0, 1) per candidate and one for the token after the
        path; draft_logits (numpy or device float32, [rows, vocab]) the logits
        that the children of each row were drawn from (device logits of the
        current torch stream are waited for)."""
        return self._tree([req], [cands], None if parents is None else [parents],
                          [dict(uniforms=uniforms, temperature=temperature, draft_logits=draft_logits,
                                draft_temperature=draft_temperature)])[0]

    def verify_tree_batch(self, reqs: Sequence[int], cands: Sequence[Sequence[int]],
                          parents: Optional[Sequence[Optional[Sequence[int]]]] = None,
                          sampling: Optional[Sequence[dict]] = None) -> List[dict]:
        """Trees of several requests in one pass; `sampling`: None (greedy) or
        for each request the keyword arguments of verify_sampled."""
        return self._tree(reqs, cands, parents, sampling)

    def _tree(self, reqs, cands, parents, sampling):
        n = len(reqs)
        cands = [_int32(c) for c in cands]
        if len(cands) != n or (parents is not None and len(parents) != n) or (sampling is not None and len(sampling) != n):
            _refuse(f"{n} requests, but not as many candidates, parents or samplings")
        r, ks = _int32(reqs), _int32([len(c) for c in cands])
        flat = _int32(np.concatenate(cands)) if n else _int32([])
        up = None
        if parents is not None:
            for p, c in zip(parents, cands):
                if p is not None and len(p) != len(c):
                    _refuse(f"parents: {len(c)} entries are wanted, not {len(p)}")
            up = _int32(np.concatenate([_int32(range(-1, len(c) - 1) if p is None else p) for p, c in zip(parents, cands)])) \
                if n else None
        paths = np.full(max(flat.size, 1), -1, np.int32)
        outs, args, keep = (VerifyOut * max(n, 1))(), None, []
        if sampling is not None:
            args = (Sampling * max(n, 1))(*[self._sampling(s, c, p, keep) for s, c, p in
                                            zip(sampling, cands, parents if parents is not None else [None] * n)])
        self._check(self.lib.as2d_verify_tree_batch(self.ctx, n, _opt(r), _opt(flat), _opt(up), _opt(ks), args, outs,
                                                    _ptr(paths)))
        got, off = [], 0
        for o, c in zip(outs, cands):
            got.append(dict(o.as_dict(), path=[int(i) for i in paths[off:off + o.accepted_len]]))
            off += len(c)
        return got

    def _sampling(self, s: dict, cands, parents, keep: list) -> Sampling:
        u = np.ascontiguousarray(s["uniforms"], dtype=np.float32)
        if u.shape != (len(cands) + 1,):
            _refuse(f"uniforms: {len(cands) + 1} numbers are wanted, not {u.shape}")
        keep.append(u)
        d = s.get("draft_logits")
        p = None
        if d is not None and len(cands):
            rows = max((int(i) + 2 for i in parents), default=1) if parents is not None else len(cands)
            if len(d.shape) != 2 or d.shape[0] < rows or d.shape[1] != self.shape.vocab:
                _refuse(f"draft_logits: [{rows} or more, {self.shape.vocab}] is wanted, not {tuple(d.shape)}")
            if isinstance(d, np.ndarray):
                d = np.ascontiguousarray(d, dtype=np.float32)
                p = _ptr(d)
            else:
                import torch
                p = _dense(d, "draft_logits", torch.float32, tuple(d.shape))
                torch.cuda.current_stream(d.device).synchronize()   # the pass copies from it on its own stream
            keep.append(d)
        return Sampling(s.get("temperature", 1.0), s.get("draft_temperature", 0.0), _ptr(u), p)

    def tree_attention(self, req: int, layer: int, q, k, v, parents: Optional[Sequence[int]] = None, out=None,
                       stream: Optional[int] = None):
        """Attention of a tree's rows over one layer of the request's cache
        (as2d_tree_attention): q [rows, n_q_heads, head_dim], k and v
        [rows, n_kv_heads, head_dim], device tensors of the model's type, on
        the current torch stream or `stream` (a handle; the caller then sees to
        it that the tensors outlive the call's work).  Returns out (new if
        None)."""
        s, rows, t = self.shape, q.shape[0], q.dtype
        if _types().get(t) != s.dtype:
            _refuse(f"tree_attention: {t} tensors, the model's type is {s.dtype}")
        if rows < 1:
            _refuse("tree_attention: no rows")
        q_shape, kv_shape = (rows, s.n_q_heads, s.head_dim), (rows, s.n_kv_heads, s.head_dim)
        if out is None:
            out = q.new_empty(q_shape)
        self._check(self.lib.as2d_tree_attention(
            self.ctx, req, layer, rows, _parents(parents, rows - 1), _rows(q, "q", t, q_shape), _rows(k, "k", t, kv_shape),
            _rows(v, "v", t, kv_shape), _rows(out, "out", t, q_shape),
            _stream_of(_device_of((q, k, v, out), self.device), stream)))
        return out

    def write_kv(self, req: int, layer: int, k, v, pos: int = 0, stream: Optional[int] = None):
        """Keys and values [n, n_kv_heads, head_dim] (device, float32 or
        bfloat16) into positions pos .. of one layer of the request's cache."""
        s, t = self.shape, k.dtype
        if t not in _types():
            _refuse(f"k: float32 or bfloat16 is wanted, not {t}")
        a = [_rows(x, name, t, (k.shape[0], s.n_kv_heads, s.head_dim)) for x, name in ((k, "k"), (v, "v"))]
        dev = _device_of((k, v), self.device)
        if k.shape[0]:
            self._check(self.lib.as2d_write_kv(self.ctx, req, layer, pos, k.shape[0], _types()[t], *a, _stream_of(dev, stream)))

    def verify_batch_status(self, reqs: Sequence[int], cands: Sequence[Sequence[int]]):
        """as2d_verify_batch returning (status, per-request results) without
        raising: with AS2D_ENUMERIC the requests whose logits are finite are
        committed and the others report accepted_len -1."""
        n = len(reqs)
        r = np.ascontiguousarray(reqs, dtype=np.int32)
        ks = np.array([len(c) for c in cands], dtype=np.int32)
        flat = np.ascontiguousarray(np.concatenate([np.asarray(c, dtype=np.int32) for c in cands])
                                    if ks.sum() else np.zeros(1, np.int32), dtype=np.int32)
        outs = (VerifyOut * n)()
        rc = self.lib.as2d_verify_batch(self.ctx, n, _ptr(r), _ptr(flat), _ptr(ks), outs)
        return rc, [o.as_dict() for o in outs]

    def set_keep_logits(self, on: bool):
        self._check(self.lib.as2d_set_keep_logits(self.ctx, int(on)))

    def logits(self, req: int, max_rows: int = 32) -> np.ndarray:
        buf = np.empty((max_rows, self.shape.vocab), dtype=np.float32)
        n = _I()
        self._check(self.lib.as2d_get_logits(self.ctx, req, _ptr(buf), max_rows, ctypes.byref(n)))
        return buf[:n.value].copy()

    def row_tokens(self, req: int, max_rows: int = 32) -> List[int]:
        buf = np.empty(max_rows, dtype=np.int32)
        n = _I()
        self._check(self.lib.as2d_get_row_tokens(self.ctx, req, _ptr(buf), max_rows, ctypes.byref(n)))
        return [int(t) for t in buf[:n.value]]

    def row_margins(self, req: int, max_rows: int = 32) -> np.ndarray:
        """Top-2 logit margin of every row of the last call (device-side)."""
        buf = np.empty(max_rows, dtype=np.float32)
        n = _I()
        self._check(self.lib.as2d_get_row_margins(self.ctx, req, _ptr(buf), max_rows, ctypes.byref(n)))
        return buf[:n.value].copy()

    def rollback(self, req: int, kv_len: int, root: int):
        self._check(self.lib.as2d_rollback(self.ctx, req, kv_len, root))

    def state(self, req: int):
        kv, root, com = _I(), _I(), _I()
        self._check(self.lib.as2d_get_state(self.ctx, req, ctypes.byref(kv), ctypes.byref(root),
                                            ctypes.byref(com)))
        return kv.value, root.value, com.value

    def read_kv(self, req: int, layer: int, n_tok: int):
        s = self.shape
        k = np.empty((s.n_kv_heads, n_tok, s.head_dim), dtype=np.float32)
        v = np.empty_like(k)
        self._check(self.lib.as2d_read_kv(self.ctx, req, layer, _ptr(k), _ptr(v), n_tok))
        return k, v

    def release(self, req: int):
        self._check(self.lib.as2d_release_request(self.ctx, req))

    def set_exec_mode(self, mode: int):
        """EXEC_EAGER, EXEC_GRAPH or EXEC_PERSISTENT (include/as2d.h)."""
        self._check(self.lib.as2d_set_exec_mode(self.ctx, mode))

    def exec_info(self):
        mode, grid = _I(), _I()
        self._check(self.lib.as2d_get_exec_info(self.ctx, ctypes.byref(mode), ctypes.byref(grid)))
        return mode.value, grid.value

    def set_step_trace(self, on: bool):
        self._check(self.lib.as2d_set_step_trace(self.ctx, int(on)))

    def step_trace(self) -> np.ndarray:
        """[grid, n_phase, 3] wall-clock stamps of the last persistent pass."""
        n = 1 << 22
        buf = np.zeros(n, dtype=np.int64)
        g, ph = _I(), _I()
        self._check(self.lib.as2d_step_trace_read(self.ctx, _ptr(buf), n, ctypes.byref(g), ctypes.byref(ph)))
        return buf[:g.value * ph.value * 3].reshape(g.value, ph.value, 3)

    def set_timing(self, on: bool):
        self._check(self.lib.as2d_set_timing(self.ctx, int(on)))

    def timing_reset(self):
        self._check(self.lib.as2d_timing_reset(self.ctx))

    def timing(self) -> dict:
        names = ctypes.create_string_buffer(32 * 16)
        ms = (ctypes.c_double * 16)()
        cnt = (ctypes.c_int64 * 16)()
        n = self.lib.as2d_timing_read(self.ctx, names, ms, cnt, 16)
        out = {}
        for i in range(n):
            nm = names.raw[32 * i:32 * i + 32].split(b"\0")[0].decode()
            out[nm] = (ms[i], cnt[i])
        return out

    def time_gemm(self, which: int, rows: int, reps: int) -> float:
        """Average microseconds of one GEMM launch (0 QKV, 1 O, 2 gate/up,
        3 down, 4 LM head); measurement only, clobbers activations."""
        us = ctypes.c_double()
        self._check(self.lib.as2d_time_gemm(self.ctx, which, rows, reps, ctypes.byref(us)))
        return us.value

    def stream_bandwidth(self, nbytes: int = 1 << 30, reps: int = 10) -> float:
        """Achievable read bandwidth (GB/s) of a plain streaming kernel."""
        gbps = ctypes.c_double()
        self._check(self.lib.as2d_stream_bandwidth(self.ctx, nbytes, reps, ctypes.byref(gbps)))
        return gbps.value

    def set_stream(self, stream: Optional[int]):
        """Rebind to a HIP stream handle (None: a stream of its own)."""
        self._check(self.lib.as2d_set_stream(self.ctx, stream))

    def set_cu_budget(self, cus: int):
        """Size the balanced GEMM grids for `cus` compute units (0: all the
        stream's)."""
        self._check(self.lib.as2d_set_cu_budget(self.ctx, cus))

    def step_bytes(self, rows: int, kv_keys: int) -> int:
        return int(self.lib.as2d_step_bytes(self.ctx, rows, kv_keys))


def _rc(rc, what):
    if rc != OK:
        raise As2dError(rc, what)


class Sampler:
    """Verification of drafted tokens by sampling, on device tensors
    (as2d_sampler_verify has the rule and the conventions)."""

    def __init__(self, max_requests: int, max_k: int, max_vocab: int):
        self.lib = load_library()
        self.device = _current_device(self.lib)
        self.h = _P()
        rc = self.lib.as2d_sampler_create(max_requests, max_k, max_vocab, ctypes.byref(self.h))
        if rc != OK:
            raise As2dError(rc, self.lib.as2d_sampler_last_error(None).decode())

    def close(self):
        if getattr(self, "h", None):
            self.lib.as2d_sampler_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def verify(self, logits, cands, uniforms, parents: Optional[Sequence[int]] = None, ks=None, draft_logits=None,
               temperature=1.0, draft_temperature: float = 0.0, stream: Optional[int] = None) -> dict:
        """logits [n, k + 1, vocab] (float32 or bfloat16; rows may be further
        apart than vocab), draft_logits the same or None, cands [n, k] and ks
        [n] int32, uniforms [n, k + 1] float32, temperature a number or a
        float32 tensor [n]: device tensors.  parents: a host list of k entries
        or None (chains).  Returns device tensors accepted [n], path [n, k],
        token [n] and logp [n, k + 1], on the current torch stream or `stream`
        (a handle; the caller then sees to it that the tensors outlive the
        call's work)."""
        import torch
        shape, t = getattr(logits, "shape", ()), getattr(logits, "dtype", None)
        if len(shape) != 3 or shape[1] < 1 or t not in _types():
            _refuse("logits: [n, k + 1, vocab], float32 or bfloat16, is wanted")
        n, rows, vocab = shape
        k = rows - 1
        tensors = [logits, uniforms]
        p_logits, step = self._logits(logits, "logits", t, shape)
        p_draft, p_cands, p_ks, p_temps, draft_step = None, None, None, None, 0
        if k:
            p_cands = _dense(cands, "cands", torch.int32, (n, k))
            tensors.append(cands)
        if draft_logits is not None:
            p_draft, draft_step = self._logits(draft_logits, "draft_logits", t, shape)
            tensors.append(draft_logits)
        if ks is not None:
            p_ks = _dense(ks, "ks", torch.int32, (n,))
            tensors.append(ks)
        if hasattr(temperature, "data_ptr"):
            p_temps = _dense(temperature, "temperature", torch.float32, (n,))
            tensors.append(temperature)
            temperature = 0.0
        p_uniforms = _dense(uniforms, "uniforms", torch.float32, (n, rows))
        dev = _device_of(tensors, self.device)
        new = cands if k else uniforms.new_empty(0, dtype=torch.int32)
        out = dict(accepted=new.new_empty(n), path=new.new_empty((n, k)), token=new.new_empty(n),
                   logp=uniforms.new_empty((n, rows)))
        up = _parents(parents, k)
        a = SampleArgs(n, k, vocab, _types()[t], p_logits, step, p_draft, draft_step, p_cands,
                       ctypes.addressof(up) if up is not None and k else None, p_ks, p_uniforms, p_temps, temperature,
                       draft_temperature, *(x.data_ptr() for x in out.values()))
        rc = self.lib.as2d_sampler_verify(self.h, a, _stream_of(dev, stream))
        if rc != OK:
            raise As2dError(rc, self.lib.as2d_sampler_last_error(self.h).decode())
        return out

    @staticmethod
    def _logits(t, name, dtype, shape):
        """(address, elements between rows) of [n, rows, vocab] logits whose rows are evenly apart."""
        p, (n, rows, vocab), stride = _on_device(t, name, dtype, shape), shape, t.stride()
        step = stride[1] if rows > 1 else stride[0] if n > 1 else vocab
        if (vocab > 1 and stride[2] != 1) or (n > 1 and rows > 1 and stride[0] != rows * step):
            _refuse(f"{name}: rows of adjacent logits, evenly apart, are wanted")
        return p, step


class CandidateBuffer:
    """The library's candidate buffer (one producer, any readers)."""

    def __init__(self, capacity: int):
        self.lib = load_library()
        self.h = _P()
        _rc(self.lib.as2d_cbuf_create(capacity, ctypes.byref(self.h)), "as2d_cbuf_create")

    def close(self):
        if getattr(self, "h", None):
            self.lib.as2d_cbuf_free(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def publish(self, tokens, source_id=0, producer_id=0, offset=-1, publish_ns=0, confidence=float("nan")) -> int:
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        n = ctypes.c_int64()
        _rc(self.lib.as2d_cbuf_publish(self.h, _ptr(t) if t.size else None, len(t), source_id, producer_id, offset,
                                       publish_ns, confidence, ctypes.byref(n)), "as2d_cbuf_publish")
        return n.value

    def snapshot(self) -> int:
        n = ctypes.c_int64()
        _rc(self.lib.as2d_cbuf_snapshot(self.h, ctypes.byref(n)), "as2d_cbuf_snapshot")
        return n.value

    def read(self, start: int, n: int) -> List[int]:
        out = np.empty(max(n, 1), dtype=np.int32)
        _rc(self.lib.as2d_cbuf_read(self.h, start, n, _ptr(out)), "as2d_cbuf_read")
        return [int(v) for v in out[:n]]

    def records(self) -> List[dict]:
        n = ctypes.c_int64()
        _rc(self.lib.as2d_cbuf_n_records(self.h, ctypes.byref(n)), "as2d_cbuf_n_records")
        out = []
        for i in range(n.value):
            r = CbufRecord()
            _rc(self.lib.as2d_cbuf_get_record(self.h, i, ctypes.byref(r)), "as2d_cbuf_get_record")
            out.append(dict(first=r.first, count=r.count, source_id=r.source_id, producer_id=r.producer_id,
                            offset=r.offset, publish_ns=r.publish_ns, confidence=r.confidence))
        return out


class ReadCursor:
    """A read cursor over a CandidateBuffer (the library's alignment rule)."""

    def __init__(self, radius: int = 8):
        self.lib = load_library()
        self.c = ReadCursorC()
        _rc(self.lib.as2d_cursor_init(ctypes.byref(self.c), radius), "as2d_cursor_init")

    @property
    def cursor(self) -> int:
        return self.c.cursor

    @property
    def floor(self) -> int:
        return self.c.floor

    def propose(self, buf: CandidateBuffer, snapshot: int, k_max: int) -> List[int]:
        out = np.empty(max(k_max, 1), dtype=np.int32)
        k = _I()
        _rc(self.lib.as2d_cursor_propose(buf.h, ctypes.byref(self.c), snapshot, k_max, _ptr(out), ctypes.byref(k)),
            "as2d_cursor_propose")
        return [int(v) for v in out[:k.value]]

    def update(self, buf: CandidateBuffer, snapshot: int, k: int, accepted: int, token: int):
        _rc(self.lib.as2d_cursor_update(buf.h, ctypes.byref(self.c), snapshot, k, accepted, token),
            "as2d_cursor_update")

    def verify_from_buffer(self, model: "Model", req: int, buf: CandidateBuffer, budget: int, max_commit: int):
        """One decoding step of `model`'s request `req` from the buffer;
        returns (verify result dict, candidates verified)."""
        out = VerifyOut()
        k = _I()
        model._check(self.lib.as2d_verify_from_buffer(model.ctx, req, buf.h, ctypes.byref(self.c), budget,
                                                      max_commit, ctypes.byref(out), ctypes.byref(k)))
        return out.as_dict(), k.value


def run_decoupled(target: Model, treq: int, drafter: Model, dreq: int, draft: Sequence[int], budget: int,
                  n_commit: int, concurrent: bool, radius: int = 8, log_cap: int = 1 << 16) -> dict:
    """as2d_run_decoupled on a fresh buffer and cursor.  Returns the
    committed tokens, the stage intervals [(start_ns, end_ns, kind,
    tokens)] (kind 0 producer step, 1 verifier call), the run's total ns
    and the producer's status."""
    lib = load_library()
    d = np.ascontiguousarray(draft, dtype=np.int32)
    buf = CandidateBuffer(max(len(d), 1))
    cur = ReadCursor(radius)
    out = np.empty(n_commit, dtype=np.int32)
    log = (Interval * log_cap)()
    n_log, total, prc = _I(), ctypes.c_int64(), _I()
    rc = lib.as2d_run_decoupled(target.ctx, treq, drafter.ctx, dreq, _ptr(d) if d.size else None, len(d), budget,
                                n_commit, int(concurrent), buf.h, ctypes.byref(cur.c), _ptr(out), log, log_cap,
                                ctypes.byref(n_log), ctypes.byref(total), ctypes.byref(prc))
    target._check(rc)
    iv = [(log[i].start_ns, log[i].end_ns, log[i].kind, log[i].tokens) for i in range(n_log.value)]
    res = dict(committed=[int(t) for t in out], intervals=iv, total_ns=total.value, producer_rc=prc.value,
               published=buf.snapshot(), records=len(buf.records()))
    buf.close()
    return res

