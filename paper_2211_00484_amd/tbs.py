"""Python binding of libtbs.so (include/tbs.h): argument marshalling only.

Every step of the decode runs in the HIP library; torch supplies device memory
and the current HIP stream.  Importing this module does not load the library;
the first call does, and raises if ``libtbs.so`` has not been built.
"""
from __future__ import annotations

import atexit
import contextlib
import ctypes
import math
import os
import re
import weakref
from dataclasses import dataclass
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtbs.so")
HEADER_PATH = os.path.join(os.path.dirname(_HERE), "include", "tbs.h")

TBS_JOINER_FP32, TBS_JOINER_BF16 = 0, 1
STATUS_NAMES = {0: "TBS_OK", -1: "TBS_EINVAL", -2: "TBS_ENOMEM", -3: "TBS_EDEVICE",
                -4: "TBS_ECAPACITY", -5: "TBS_EUNSUPPORTED"}

_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_F32 = ctypes.c_float


class TbsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class KernelTime(ctypes.Structure):
    _fields_ = [("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


KERNEL_NAMES = ("joiner", "search", "final", "stream", "stream_group", "hyp_step")
SCHEDULES = {"auto": 0, "frame": 1, "stream": 2, "stream1": 3}


class BeamParams(ctypes.Structure):
    _fields_ = [("beam", ctypes.c_float), ("max_states", ctypes.c_int32),
                ("max_contexts", ctypes.c_int32)]


class Adjustments(ctypes.Structure):
    _fields_ = [("history", _P), ("ld_history", _I64), ("history_cols", _I32),
                ("history_lengths", _P), ("repetition", _F32), ("presence", _F32),
                ("frequency", _F32), ("row_penalties", _P), ("bias", _P), ("ld_bias", _I64),
                ("allowed", _P), ("ld_allowed", _I64), ("graph", _P), ("states", _P),
                ("normalize", _I32)]


_lib = None
# Set when the interpreter starts to exit: handles still open then are left to the
# process teardown instead of calling into the library (and HIP) from finalizers that
# may run after the runtime has begun shutting down.  Call close() to release earlier.
_exiting = False


def _at_exit():
    global _exiting
    _exiting = True


atexit.register(_at_exit)

_live = weakref.WeakSet()  # open handles (graphs, models, decode states, lattices)


def close_all():
    """Releases every handle still open: lattices and decode states first, then models
    and graphs (a lattice or state refers to its model).  For programs that want the
    device memory back before the interpreter exits."""
    order = {"Lattice": 0, "DecodeState": 1, "Model": 2, "Graph": 3}
    for obj in sorted(list(_live), key=lambda o: order.get(type(o).__name__, 4)):
        obj.close()


def declared_symbols() -> list:
    """Names of the functions declared in include/tbs.h."""
    with open(HEADER_PATH) as f:
        text = f.read()
    return sorted(set(re.findall(r"^\s*(?:const\s+)?[a-z_0-9]+\s*\*?\s*(tbs_[a-z_0-9]+)\s*\(",
                                 text, flags=re.M)))


def lib():
    """The loaded library; raises if it is missing (there is no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "(hipcc --offload-arch=gfx950); there is no CPU fallback")
    L = ctypes.CDLL(LIB_PATH)
    L.tbs_last_error.restype = ctypes.c_char_p
    L.tbs_last_error.argtypes = []
    L.tbs_graph_create.restype = _I32
    L.tbs_graph_create.argtypes = [_I32, _I32, _I32, _P, _P, _P, _P, _P, ctypes.POINTER(_P)]
    L.tbs_graph_create_trivial.restype = _I32
    L.tbs_graph_create_trivial.argtypes = [_I32, ctypes.POINTER(_P)]
    L.tbs_graph_destroy.restype = None
    L.tbs_graph_destroy.argtypes = [_P]
    L.tbs_model_create.restype = _I32
    L.tbs_model_create.argtypes = [_I32, _I32, _I32, _P, _P, _P, _P, _I32, _P, ctypes.POINTER(_P)]
    L.tbs_model_destroy.restype = None
    L.tbs_model_destroy.argtypes = [_P]
    L.tbs_decode.restype = _I32
    L.tbs_decode.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _P, _P, _I32, _I32,
                             _P, _P, _P, _P, _P, _P, _P]
    L.tbs_decode_noalloc.restype = _I32
    L.tbs_decode_noalloc.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _P, _P, _I32, _I32,
                                     _P, _P, _P, _P, _P, _P, _P]
    L.tbs_decode_graphs.restype = _I32
    L.tbs_decode_graphs.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _P, _P, _I32, _I32,
                                    _P, _P, _P, _P, _P, _P, _P]
    L.tbs_model_set_schedule.restype = _I32
    L.tbs_model_set_schedule.argtypes = [_P, _I32]
    L.tbs_model_set_graph_capture.restype = _I32
    L.tbs_model_set_graph_capture.argtypes = [_P, _I32]
    L.tbs_model_graph_stats.restype = _I32
    L.tbs_model_graph_stats.argtypes = [_P, ctypes.POINTER(_I32), ctypes.POINTER(_I32)]
    L.tbs_model_set_exchange_spin_limit.restype = _I32
    L.tbs_model_set_exchange_spin_limit.argtypes = [_P, _I32]
    L.tbs_model_set_profiling.restype = _I32
    L.tbs_model_set_profiling.argtypes = [_P, _I32]
    L.tbs_model_read_profile.restype = _I32
    L.tbs_model_read_profile.argtypes = [_P, ctypes.POINTER(KernelTime)]
    L.tbs_joiner_logp.restype = _I32
    L.tbs_joiner_logp.argtypes = [_P, _P, _P, _I32, _P, _P]
    L.tbs_state_create.restype = _I32
    L.tbs_state_create.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _I32, _I32, _P,
                                   ctypes.POINTER(_P)]
    L.tbs_state_create_graphs.restype = _I32
    L.tbs_state_create_graphs.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _I32, _I32, _P,
                                          ctypes.POINTER(_P)]
    L.tbs_transducer_forward.restype = _I32
    L.tbs_transducer_forward.argtypes = [_I32, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P]
    L.tbs_transducer_gradient_workspace.restype = _SZ
    L.tbs_transducer_gradient_workspace.argtypes = [_I32] * 3
    L.tbs_transducer_gradient.restype = _I32
    L.tbs_transducer_gradient.argtypes = [_I32, _P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P,
                                          _P, _SZ, _P]
    L.tbs_linear_workspace.restype = _SZ
    L.tbs_linear_workspace.argtypes = [_I32] * 4
    L.tbs_linear.restype = _I32
    L.tbs_linear.argtypes = [_I32, _P, _I64, _P, _I64, _P, _P, _I64, _I32, _I32, _I32, _I32, _I32,
                             _P, _I64, _P, _I64, _P, _SZ, _P]
    L.tbs_linear_backward_workspace.restype = _SZ
    L.tbs_linear_backward_workspace.argtypes = [_I32] * 9
    L.tbs_linear_backward.restype = _I32
    L.tbs_linear_backward.argtypes = [_I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _I32, _I32,
                                      _I32, _I32, _P, _I64, _P, _I64, _P, _P, _I64, _P, _SZ, _P]
    L.tbs_adjust_logits_workspace.restype = _SZ
    L.tbs_adjust_logits_workspace.argtypes = [_I32] * 4
    L.tbs_adjust_logits.restype = _I32
    L.tbs_adjust_logits.argtypes = [_I32, _P, _I64, _I32, _I32, ctypes.POINTER(Adjustments), _P,
                                    _I64, _P, _SZ, _P]
    L.tbs_hyp_search.restype = _I32
    L.tbs_hyp_search.argtypes = [_P, ctypes.POINTER(HypParams), _P, _P, _I32, _I32, _P, _P, _P,
                                 _P, _P]
    L.tbs_lattice_create.restype = _I32
    L.tbs_lattice_create.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _P, _P, _I32, _I32, _P,
                                     ctypes.POINTER(_P)]
    L.tbs_lattice_create_graphs.restype = _I32
    L.tbs_lattice_create_graphs.argtypes = [_P, _P, ctypes.POINTER(BeamParams), _P, _P, _I32,
                                            _I32, _P, ctypes.POINTER(_P)]
    L.tbs_lattice_num_arcs.restype = _I32
    L.tbs_lattice_num_arcs.argtypes = [_P, ctypes.POINTER(ctypes.c_int64)]
    L.tbs_lattice_export.restype = _I32
    L.tbs_lattice_export.argtypes = [_P] + [_P] * 8 + [_P]
    L.tbs_lattice_nbest.restype = _I32
    L.tbs_lattice_nbest.argtypes = [_P, _I32, _P] + [_P] * 7 + [_P]
    L.tbs_lattice_destroy.restype = None
    L.tbs_lattice_destroy.argtypes = [_P]
    L.tbs_decode_chunk.restype = _I32
    L.tbs_decode_chunk.argtypes = [_P, _P, _P, _I32, _P, _P]
    L.tbs_state_finish.restype = _I32
    L.tbs_state_finish.argtypes = [_P, _P, _P, _P, _P, _P, _P]
    L.tbs_state_destroy.restype = None
    L.tbs_state_destroy.argtypes = [_P]
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise TbsError(status, lib().tbs_last_error().decode())


def _host_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _dev_ptr(t):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return ctypes.c_void_p(t.data_ptr())


def _stream_ptr(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


class Graph:
    """Device copy of an epsilon-free decoding graph (tbs_graph_create)."""

    def __init__(self, handle, num_states: int, vocab_size: int, max_out_degree: int):
        self._h = handle
        _live.add(self)
        self.num_states, self.vocab_size, self.max_out_degree = num_states, vocab_size, max_out_degree

    @classmethod
    def from_csr(cls, num_states, start, vocab_size, row_ptr, dest, label, score, final=None):
        rp = np.ascontiguousarray(row_ptr, dtype=np.int32)
        de = np.ascontiguousarray(dest, dtype=np.int32)
        la = np.ascontiguousarray(label, dtype=np.int32)
        sc = np.ascontiguousarray(score, dtype=np.float32)
        fi = None if final is None else np.ascontiguousarray(final, dtype=np.float32)
        h = _P()
        _check(lib().tbs_graph_create(int(num_states), int(start), int(vocab_size), _host_ptr(rp),
                                      _host_ptr(de), _host_ptr(la), _host_ptr(sc), _host_ptr(fi),
                                      ctypes.byref(h)))
        deg = int(np.max(np.diff(rp))) if len(rp) > 1 else 0
        return cls(h, int(num_states), int(vocab_size), deg)

    @classmethod
    def trivial(cls, vocab_size: int):
        h = _P()
        _check(lib().tbs_graph_create_trivial(int(vocab_size), ctypes.byref(h)))
        return cls(h, 1, int(vocab_size), int(vocab_size) - 1)

    @classmethod
    def from_synth(cls, g):
        return cls.from_csr(g.num_states, g.start, g.vocab_size, g.row_ptr, g.dest, g.label,
                            g.score, g.final)

    def close(self):
        if self._h is not None and _lib is not None and not _exiting:
            _lib.tbs_graph_destroy(self._h)
        self._h = None

    def __del__(self):
        self.close()


class Model:
    """Stateless decoder + joiner weights on the device (tbs_model_create)."""

    def __init__(self, vocab_size: int, dim: int, embed, conv, w_out, b_out=None,
                 dtype: str = "fp32", stream=None):
        import torch
        self._h = None
        dev = torch.device("cuda", torch.cuda.current_device())

        def dt(x):
            if x is None:
                return None
            if isinstance(x, np.ndarray):
                x = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
            return x.to(device=dev, dtype=torch.float32).contiguous()

        E, cv, W, b = dt(embed), dt(conv), dt(w_out), dt(b_out)
        code = {"fp32": TBS_JOINER_FP32, "bf16": TBS_JOINER_BF16}[dtype]
        h = _P()
        _check(lib().tbs_model_create(int(vocab_size), int(dim), 2, _dev_ptr(E), _dev_ptr(cv),
                                      _dev_ptr(W), _dev_ptr(b), code, _stream_ptr(stream),
                                      ctypes.byref(h)))
        self._h = h
        _live.add(self)
        self.vocab_size, self.dim, self.dtype = int(vocab_size), int(dim), dtype

    def set_schedule(self, schedule: str):
        """Frame-loop schedule for later decodes: "auto", "frame", "stream" (several
        workgroups per stream where possible) or "stream1" (one per stream)."""
        _check(lib().tbs_model_set_schedule(self._h, SCHEDULES[schedule]))

    def set_graph_capture(self, enable: bool):
        """Capture the frame schedule's frame loop in a HIP graph when a decode repeats
        the previous one's launch arguments (default on)."""
        _check(lib().tbs_model_set_graph_capture(self._h, int(bool(enable))))

    def graph_stats(self) -> tuple:
        """(captures, replays) of the frame-loop graph so far."""
        c, r = _I32(), _I32()
        _check(lib().tbs_model_graph_stats(self._h, ctypes.byref(c), ctypes.byref(r)))
        return int(c.value), int(r.value)

    def set_exchange_spin_limit(self, polls: int):
        """Poll budget of the grouped kernel's exchange waits (0 = default); a
        diagnostic for the timeout path."""
        _check(lib().tbs_model_set_exchange_spin_limit(self._h, int(polls)))

    def set_profiling(self, enable: bool):
        _check(lib().tbs_model_set_profiling(self._h, int(bool(enable))))

    def read_profile(self) -> dict:
        """{kernel: (launches, total_ms)} accumulated since profiling was enabled."""
        arr = (KernelTime * len(KERNEL_NAMES))()
        _check(lib().tbs_model_read_profile(self._h, arr))
        return {n: (int(arr[i].launches), float(arr[i].total_ms)) for i, n in enumerate(KERNEL_NAMES)}

    @classmethod
    def from_synth(cls, m, dtype: str = "fp32"):
        return cls(m.vocab_size, m.dim, m.embed, m.conv, m.w_out, m.b_out, dtype=dtype)

    def close(self):
        if self._h is not None and _lib is not None and not _exiting:
            _lib.tbs_model_destroy(self._h)
        self._h = None

    def __del__(self):
        self.close()


@dataclass
class DecodeOutput:
    tokens: "object"      # int32 [B, T] device
    num_tokens: "object"  # int32 [B]
    scores: "object"      # float64 [B]
    status: "object"      # int32 [B] or None
    arcs: "object"        # int32 [B, T] or None
    trace: "object"       # int32 [T+1, B, Ns, 4] or None

    def token_lists(self):
        tok = self.tokens.cpu().numpy()
        n = self.num_tokens.cpu().numpy()
        return [list(tok[b, : n[b]]) for b in range(tok.shape[0])]


def allocate_outputs(B: int, T: int, max_states: int, status=True, arcs=False, trace=False,
                     device=None) -> DecodeOutput:
    import torch
    dev = device or torch.device("cuda", torch.cuda.current_device())
    i32 = dict(dtype=torch.int32, device=dev)
    return DecodeOutput(
        tokens=torch.empty((B, T), **i32), num_tokens=torch.empty(B, **i32),
        scores=torch.empty(B, dtype=torch.float64, device=dev),
        status=torch.empty(B, **i32) if status else None,
        arcs=torch.empty((B, T), **i32) if arcs else None,
        trace=torch.empty((T + 1, B, max_states, 4), **i32) if trace else None)


def _graph_table(graphs, B: int):
    """Host array of B graph handles (kept alive by the caller's list)."""
    graphs = list(graphs)
    if len(graphs) != B:
        raise ValueError(f"need one graph per stream: {len(graphs)} graphs for B = {B}")
    return (_P * max(B, 1))(*[g._h for g in graphs])


def decode_into(model: Model, graph, encoder_out, lengths, beam: float, max_states: int,
                max_contexts: int, out: DecodeOutput, stream=None) -> DecodeOutput:
    """tbs_decode into preallocated outputs (stream-ordered; no synchronisation).
    ``graph`` is one Graph shared by every stream, or a list of B graphs, one per
    stream (tbs_decode_graphs)."""
    lens = np.ascontiguousarray(np.asarray(lengths), dtype=np.int32)
    B, T = int(encoder_out.shape[0]), int(encoder_out.shape[1])
    if encoder_out.dim() != 3 or encoder_out.shape[2] != model.dim:
        raise ValueError("encoder_out must be [B, T, dim]")
    if lens.shape != (B,):
        raise ValueError("lengths must have shape [B]")
    params = BeamParams(float(math.inf if beam is None else beam), int(max_states),
                        int(max_contexts))
    if isinstance(graph, Graph):
        fn, gh = lib().tbs_decode, graph._h
    else:
        fn, gh = lib().tbs_decode_graphs, _graph_table(graph, B)
    _check(fn(model._h, gh, ctypes.byref(params), _dev_ptr(encoder_out),
              _host_ptr(lens), B, T, _dev_ptr(out.tokens), _dev_ptr(out.num_tokens),
              _dev_ptr(out.scores), _dev_ptr(out.status), _dev_ptr(out.arcs),
              _dev_ptr(out.trace), _stream_ptr(stream)))
    return out


def decode_noalloc_into(model: Model, graph: Graph, encoder_out, lengths_dev, beam: float,
                        max_states: int, max_contexts: int, out: DecodeOutput,
                        stream=None) -> DecodeOutput:
    """tbs_decode_noalloc: tbs_decode with its workspace in the library's fixed device
    array (no allocation); ``lengths_dev`` is a device int32 tensor [B]."""
    B, T = int(encoder_out.shape[0]), int(encoder_out.shape[1])
    if encoder_out.dim() != 3 or encoder_out.shape[2] != model.dim:
        raise ValueError("encoder_out must be [B, T, dim]")
    if tuple(lengths_dev.shape) != (B,) or str(lengths_dev.dtype) != "torch.int32":
        raise ValueError("lengths_dev must be a device int32 tensor of shape [B]")
    params = BeamParams(float(math.inf if beam is None else beam), int(max_states),
                        int(max_contexts))
    _check(lib().tbs_decode_noalloc(model._h, graph._h, ctypes.byref(params),
                                    _dev_ptr(encoder_out), _dev_ptr(lengths_dev), B, T,
                                    _dev_ptr(out.tokens), _dev_ptr(out.num_tokens),
                                    _dev_ptr(out.scores), _dev_ptr(out.status),
                                    _dev_ptr(out.arcs), _dev_ptr(out.trace), _stream_ptr(stream)))
    return out


def decode(model: Model, graph, encoder_out, lengths, beam: float = math.inf,
           max_states: int = 4, max_contexts: int = 4, want_arcs: bool = False,
           want_trace: bool = False, stream=None) -> DecodeOutput:
    """Batched FSA-constrained one-symbol-per-frame beam search; outputs on the device.
    ``graph``: one Graph for every stream, or a list of one Graph per stream."""
    B, T = int(encoder_out.shape[0]), int(encoder_out.shape[1])
    out = allocate_outputs(B, T, max_states, status=True, arcs=want_arcs, trace=want_trace,
                           device=encoder_out.device)
    return decode_into(model, graph, encoder_out, lengths, beam, max_states, max_contexts, out,
                       stream)


def joiner_logp(model: Model, enc_rows, ctx, stream=None):
    """log P(. | ctx, enc row) [R, V] from the HIP joiner (tbs_joiner_logp)."""
    import torch
    R = int(enc_rows.shape[0])
    out = torch.empty((R, model.vocab_size), dtype=torch.float32, device=enc_rows.device)
    ctx = ctx.to(device=enc_rows.device, dtype=torch.int32).contiguous()
    _check(lib().tbs_joiner_logp(model._h, _dev_ptr(enc_rows.contiguous()), _dev_ptr(ctx), R,
                                 _dev_ptr(out), _stream_ptr(stream)))
    return out


class DecodeState:
    """Streaming decode (tbs_state_create / tbs_decode_chunk / tbs_state_finish):
    each chunk continues every stream from where it stopped; finish traces the best
    paths back over all decoded frames."""

    def __init__(self, model: Model, graph, B: int, max_frames: int,
                 beam: float = math.inf, max_states: int = 4, max_contexts: int = 4,
                 stream=None):
        """``graph``: one Graph for every stream, or a list of one Graph per stream."""
        self._h = None
        params = BeamParams(float(math.inf if beam is None else beam), int(max_states),
                            int(max_contexts))
        h = _P()
        if isinstance(graph, Graph):
            fn, gh = lib().tbs_state_create, graph._h
        else:
            graph = list(graph)
            fn, gh = lib().tbs_state_create_graphs, _graph_table(graph, int(B))
        _check(fn(model._h, gh, ctypes.byref(params), int(B), int(max_frames),
                  _stream_ptr(stream), ctypes.byref(h)))
        self._h = h
        _live.add(self)
        self._refs = (model, graph)  # the state must not outlive them
        self.B, self.max_frames, self.max_states = int(B), int(max_frames), int(max_states)

    def chunk(self, encoder_chunk, lengths, trace=None, stream=None):
        """Decode the next frames: encoder_chunk [B, Tc, C] on the device, lengths [B]
        frames per stream (host); trace: optional [max_frames+1, B, Ns, 4] int32 buffer."""
        lens = np.ascontiguousarray(np.asarray(lengths), dtype=np.int32)
        B, Tc = int(encoder_chunk.shape[0]), int(encoder_chunk.shape[1])
        if B != self.B or lens.shape != (B,):
            raise ValueError("encoder_chunk / lengths do not match the state's batch")
        _check(lib().tbs_decode_chunk(self._h, _dev_ptr(encoder_chunk.contiguous()),
                                      _host_ptr(lens), Tc, _dev_ptr(trace), _stream_ptr(stream)))

    def finish(self, want_arcs: bool = False, stream=None) -> DecodeOutput:
        out = allocate_outputs(self.B, self.max_frames, self.max_states, status=True,
                               arcs=want_arcs)
        _check(lib().tbs_state_finish(self._h, _dev_ptr(out.tokens), _dev_ptr(out.num_tokens),
                                      _dev_ptr(out.scores), _dev_ptr(out.status),
                                      _dev_ptr(out.arcs), _stream_ptr(stream)))
        return out

    def close(self):
        if self._h is not None and _lib is not None and not _exiting:
            _lib.tbs_state_destroy(self._h)
        self._h = None

    def __del__(self):
        self.close()


@dataclass
class NBestOutput:
    tokens: "object"         # int32 [B, T] device: the best label sequence, -1 padded
    num_tokens: "object"     # int32 [B]
    scores: "object"         # float64 [B]: its total log probability in the lattice
    num_unique: "object"     # int32 [B]: distinct sequences among the sampled paths
    unique_scores: "object"  # float64 [B, n]
    unique_first: "object"   # int32 [B, n]: the path that first gave each sequence
    paths: "object"          # int32 [B, n, T+1] or None

    def token_lists(self):
        tok = self.tokens.cpu().numpy()
        n = self.num_tokens.cpu().numpy()
        return [list(tok[b, : n[b]]) for b in range(tok.shape[0])]


class Lattice:
    """The search's lattice (tbs_lattice_create) and the n-best label-sequence search on it
    (tbs_lattice_nbest).  ``graph``: one Graph, or a list of one Graph per stream."""

    def __init__(self, model: Model, graph, encoder_out, lengths, beam: float = math.inf,
                 max_states: int = 4, max_contexts: int = 4, stream=None):
        self._h = None
        lens = np.ascontiguousarray(np.asarray(lengths), dtype=np.int32)
        B, T = int(encoder_out.shape[0]), int(encoder_out.shape[1])
        if encoder_out.dim() != 3 or encoder_out.shape[2] != model.dim:
            raise ValueError("encoder_out must be [B, T, dim]")
        if lens.shape != (B,):
            raise ValueError("lengths must have shape [B]")
        params = BeamParams(float(math.inf if beam is None else beam), int(max_states),
                            int(max_contexts))
        h = _P()
        if isinstance(graph, Graph):
            fn, gh = lib().tbs_lattice_create, graph._h
        else:
            graph = list(graph)
            fn, gh = lib().tbs_lattice_create_graphs, _graph_table(graph, B)
        _check(fn(model._h, gh, ctypes.byref(params), _dev_ptr(encoder_out.contiguous()),
                  _host_ptr(lens), B, T, _stream_ptr(stream), ctypes.byref(h)))
        self._h = h
        _live.add(self)
        self._refs = (model, graph)
        self.device = encoder_out.device
        self.B, self.T, self.max_states = B, T, int(max_states)
        self.lengths = lens

    def num_arcs(self) -> int:
        n = ctypes.c_int64(0)
        _check(lib().tbs_lattice_num_arcs(self._h, ctypes.byref(n)))
        return int(n.value)

    def export(self, stream=None) -> dict:
        """Device tensors: frame_off [B*T+1], arcs [A, 4] (src, dst, label, graph arc),
        weights [A], nodes [T+1, B, Ns, 4], alpha [B, T+1, Ns], final_w [B, Ns], total [B],
        status [B]."""
        import torch
        A, B, T, Ns, dev = self.num_arcs(), self.B, self.T, self.max_states, self.device
        out = {"frame_off": torch.empty(B * T + 1, dtype=torch.int64, device=dev),
               "arcs": torch.empty((A, 4), dtype=torch.int32, device=dev),
               "weights": torch.empty(A, dtype=torch.float32, device=dev),
               "nodes": torch.empty((T + 1, B, Ns, 4), dtype=torch.int32, device=dev),
               "alpha": torch.empty((B, T + 1, Ns), dtype=torch.float64, device=dev),
               "final_w": torch.empty((B, Ns), dtype=torch.float64, device=dev),
               "total": torch.empty(B, dtype=torch.float64, device=dev),
               "status": torch.empty(B, dtype=torch.int32, device=dev)}
        _check(lib().tbs_lattice_export(self._h, *[_dev_ptr(out[k]) for k in (
            "frame_off", "arcs", "weights", "nodes", "alpha", "final_w", "total", "status")],
            _stream_ptr(stream)))
        return out

    def nbest(self, num_paths: int, uniforms, want_paths: bool = False,
              stream=None) -> NBestOutput:
        """n-best label-sequence search; uniforms: float64 [B, num_paths, T+1] on the
        device, each in [0, 1)."""
        import torch
        B, T, n, dev = self.B, self.T, int(num_paths), self.device
        if tuple(uniforms.shape) != (B, n, T + 1) or uniforms.dtype != torch.float64:
            raise ValueError(f"uniforms must be float64 [{B}, {n}, {T + 1}]")
        i32 = dict(dtype=torch.int32, device=dev)
        out = NBestOutput(tokens=torch.empty((B, T), **i32), num_tokens=torch.empty(B, **i32),
                          scores=torch.empty(B, dtype=torch.float64, device=dev),
                          num_unique=torch.empty(B, **i32),
                          unique_scores=torch.empty((B, n), dtype=torch.float64, device=dev),
                          unique_first=torch.empty((B, n), **i32),
                          paths=torch.empty((B, n, T + 1), **i32) if want_paths else None)
        _check(lib().tbs_lattice_nbest(self._h, n, _dev_ptr(uniforms.contiguous()),
                                       _dev_ptr(out.tokens), _dev_ptr(out.num_tokens),
                                       _dev_ptr(out.scores), _dev_ptr(out.num_unique),
                                       _dev_ptr(out.unique_scores), _dev_ptr(out.unique_first),
                                       _dev_ptr(out.paths), _stream_ptr(stream)))
        return out

    def close(self):
        if self._h is not None and _lib is not None and not _exiting:
            _lib.tbs_lattice_destroy(self._h)
        self._h = None

    def __del__(self):
        self.close()


class HypParams(ctypes.Structure):
    _fields_ = [("beam_size", _I32), ("merge", _I32)]


MERGES = {"max": 0, "logadd": 1}


def hyp_search(model: Model, encoder_out, lengths, beam_size: int = 4, merge: str = "logadd",
               want_trace: bool = False, stream=None) -> DecodeOutput:
    """Full-sequence beam search with max-symbols 1 (tbs_hyp_search, Table 5's comparison
    search); outputs on the device; trace [T+1, B, beam_size, 2] (parent rank, label)."""
    import torch
    lens = np.ascontiguousarray(np.asarray(lengths), dtype=np.int32)
    B, T = int(encoder_out.shape[0]), int(encoder_out.shape[1])
    if encoder_out.dim() != 3 or encoder_out.shape[2] != model.dim:
        raise ValueError("encoder_out must be [B, T, dim]")
    if lens.shape != (B,):
        raise ValueError("lengths must have shape [B]")
    dev = encoder_out.device
    i32 = dict(dtype=torch.int32, device=dev)
    out = DecodeOutput(tokens=torch.empty((B, T), **i32), num_tokens=torch.empty(B, **i32),
                       scores=torch.empty(B, dtype=torch.float64, device=dev), status=None,
                       arcs=None,
                       trace=torch.empty((T + 1, B, int(beam_size), 2), **i32) if want_trace
                       else None)
    params = HypParams(int(beam_size), MERGES[merge])
    _check(lib().tbs_hyp_search(model._h, ctypes.byref(params),
                                _dev_ptr(encoder_out.contiguous()), _host_ptr(lens), B, T,
                                _dev_ptr(out.tokens), _dev_ptr(out.num_tokens),
                                _dev_ptr(out.scores), _dev_ptr(out.trace), _stream_ptr(stream)))
    return out


TRANSDUCER_KINDS = {"standard": 0, "modified": 1, "constrained": 2}


def transducer_forward(kind: str, blank, label, lengths, want_alpha: bool = False,
                       stream=None):
    """Forward recursion of the standard (eq. 1), modified (eq. 2) or constrained (eq. 3)
    transducer (tbs_transducer_forward).  blank [B, T, U+1] and label [B, T, U] float32 on
    the device; lengths [B, 2] int32 (frames, labels).  Returns (total [B] float64,
    alpha [B, T+1, U+1] float32 or None, status [B] int32)."""
    import torch
    B, T, U1 = (int(x) for x in blank.shape)
    U = U1 - 1
    if tuple(label.shape) != (B, T, U):
        raise ValueError("label must be [B, T, U]")
    dev = blank.device
    lengths = torch.as_tensor(lengths, dtype=torch.int32).reshape(B, 2).to(dev).contiguous()
    total = torch.empty(B, dtype=torch.float64, device=dev)
    status = torch.empty(B, dtype=torch.int32, device=dev)
    alpha = torch.empty((B, T + 1, U1), dtype=torch.float32, device=dev) if want_alpha else None
    _check(lib().tbs_transducer_forward(TRANSDUCER_KINDS[kind], _dev_ptr(blank.contiguous()),
                                        _dev_ptr(label.contiguous()) if U > 0 else None,
                                        _dev_ptr(lengths), B, T, U, _dev_ptr(total),
                                        _dev_ptr(alpha), _dev_ptr(status), _stream_ptr(stream)))
    return total, alpha, status


_DTYPES = {}  # tbs_dtype of torch's dtypes (filled once torch is there)
ACTIVATIONS = {"none": 0, "relu": 1, "tanh": 2, "silu": 3, "gelu": 4}
_I32_MAX = 2 ** 31 - 1


_HERE_SCOPE = contextlib.nullcontext()


def _scope(t, stream):
    """Context in which the copies, outputs and workspace of a call on tensor ``t`` are
    allocated and its kernels launched: the given stream, or the current stream of the
    tensor's device."""
    import torch
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if stream is not None:
        if stream.device != t.device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {t.device}")
        return torch.cuda.stream(stream)
    if t.get_device() == torch.cuda.current_device():
        return _HERE_SCOPE
    return torch.cuda.device(t.device)


def _dtype_code(t) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"unsupported dtype {t.dtype}: float32, bfloat16 or float16")
    return code


def _matrix(t, like, cols: int, name: str, dtype=None, rows=None, one_row=False, lead=()):
    """(2-D tensor, row length) of ``t`` [..., cols]: a view where its rows are contiguous
    and no closer than their width, else a copy.  With one_row, a [cols] or [1, cols] tensor
    stands for all rows (row length 0).  lead: the leading dimensions that the rows stand for;
    those of ``t``, if both have several, must be the same."""
    dtype = dtype or like.dtype
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    shape = t.shape
    if len(shape) == 0 or shape[-1] != cols:
        raise ValueError(f"{name} must have {cols} columns, not shape {tuple(shape)}")
    if len(shape) == 2 and shape[0] == rows and t.is_contiguous():
        return t, cols
    m = t if len(shape) == 2 else t.reshape(-1, cols)
    n = m.shape[0]
    if rows is not None and n != rows and not (one_row and n == 1):
        raise ValueError(f"{name} must have {rows} rows, not {n}")
    if len(lead) > 1 and len(shape) > 2 and shape[:-1] != lead and not (one_row and n == 1):
        raise ValueError(f"{name} must have the leading dimensions {tuple(lead)}, not {tuple(shape[:-1])}")
    if cols > 1 and m.stride(1) != 1:
        m = m.contiguous()
    if one_row and (n == 1 or m.stride(0) == 0):
        return m, 0
    if n > 1 and m.stride(0) < cols:
        m = m.contiguous()
    return m, m.stride(0) if n > 1 else cols


def _vector(t, like, n: int, name: str, dtype=None):
    dtype = dtype or like.dtype
    if t.get_device() != like.get_device() or t.dtype is not dtype or tuple(t.shape) != (n,):
        raise ValueError(f"{name} must be {dtype} [{n}] on {like.device}, not {t.dtype} "
                         f"{list(t.shape)} on {t.device}")
    return t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream_of(t, stream):
    """The hipStream_t inside _scope(t, stream)."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _workspace(nbytes: int, like):
    import torch
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None


def _size(n: int, name: str) -> int:
    """n as an int32 argument (ctypes would drop its high bits)."""
    if n > _I32_MAX:
        raise ValueError(f"{name}: a dimension of {n}, at most {_I32_MAX}")
    return int(n)


def linear(x, weight, bias=None, residual=None, activation: str = "none",
           residual_after: bool = False, want_pre: bool = False, stream=None):
    """act(x weight^T + bias + residual), or act(x weight^T + bias) + residual with
    residual_after (tbs_linear): x [..., K], weight [N, K], bias [N], residual [..., N] or one
    row [N] for all, of one dtype (float32, bfloat16, float16); sums in fp32.  activation:
    "none", "relu", "tanh", "silu" or "gelu" (by erf).  Returns out [..., N], or (out, pre)
    with want_pre: the activation's argument, for linear_backward.  Tensors whose rows are
    not contiguous are copied; autograd does not see the call."""
    import torch
    with _scope(x, stream):
        code, act = _dtype_code(x), ACTIVATIONS[activation]
        if x.dim() == 0 or weight.dim() != 2:
            raise ValueError("x must be [..., K] and weight [N, K]")
        N, K = (_size(n, "weight") for n in weight.shape)
        x2, ldx = _matrix(x, x, K, "x")
        M = _size(x2.shape[0], "x")
        w2, ldw = _matrix(weight, x, K, "weight")
        b = None if bias is None else _vector(bias, x, N, "bias")
        r, ldr = (None, 0) if residual is None else _matrix(residual, x, N, "residual", rows=M,
                                                            one_row=True, lead=x.shape[:-1])
        out = torch.empty(x.shape[:-1] + (N,), dtype=x.dtype, device=x.device)
        pre = torch.empty_like(out) if want_pre else None
        L = lib()
        nbytes = L.tbs_linear_workspace(code, M, N, K)
        ws = _workspace(nbytes, x)
        _check(L.tbs_linear(code, _ptr(x2), ldx, _ptr(w2), ldw, _ptr(b), _ptr(r), ldr,
                            int(residual_after), act, M, N, K, _ptr(out), N, _ptr(pre), N,
                            _ptr(ws), nbytes, _stream_of(x, stream)))
    return (out, pre) if want_pre else out


@dataclass
class LinearGrads:
    x: "object"       # [..., K] or None
    weight: "object"  # [N, K] or None
    bias: "object"    # [N] or None
    pre: "object"     # [..., N] or None: of the activation's argument (and so of a residual
                      # added before it); a residual added after it has grad_out's


def linear_backward(grad_out, x, weight, pre=None, activation: str = "none",
                    want_x: bool = True, want_weight: bool = True, want_bias: bool = True,
                    want_pre: bool = False, stream=None) -> LinearGrads:
    """Gradients of ``linear`` (tbs_linear_backward) from grad_out [..., N], its x and weight,
    and, unless the activation is "none", the pre it returned.  Each is rounded once; autograd
    does not see the call."""
    import torch
    with _scope(grad_out, stream):
        code, act = _dtype_code(grad_out), ACTIVATIONS[activation]
        if x.dim() == 0 or weight.dim() != 2 or grad_out.dim() == 0:
            raise ValueError("grad_out must be [..., N], x [..., K] and weight [N, K]")
        N, K = (_size(n, "weight") for n in weight.shape)
        if grad_out.shape[:-1] != x.shape[:-1]:
            raise ValueError("grad_out and x differ in their leading dimensions")
        if (act != 0) != (pre is not None):
            raise ValueError("pre goes with an activation, and only with one")
        g, ldg = _matrix(grad_out, grad_out, N, "grad_out")
        M = _size(g.shape[0], "grad_out")
        x2, ldx = _matrix(x, grad_out, K, "x", rows=M)
        w2, ldw = _matrix(weight, grad_out, K, "weight")
        p, ldp = (None, 0) if pre is None else _matrix(pre, grad_out, N, "pre", rows=M,
                                                       lead=grad_out.shape[:-1])
        like = dict(dtype=grad_out.dtype, device=grad_out.device)
        dx = torch.empty(x.shape, **like) if want_x else None
        dw = torch.empty((N, K), **like) if want_weight else None
        db = torch.empty(N, **like) if want_bias else None
        dz = torch.empty(grad_out.shape, **like) if want_pre and act else None
        L = lib()
        nbytes = L.tbs_linear_backward_workspace(code, act, M, N, K, int(want_x),
                                                 int(want_weight), int(want_bias),
                                                 int(dz is not None))
        ws = _workspace(nbytes, grad_out)
        _check(L.tbs_linear_backward(code, _ptr(g), ldg, _ptr(x2), ldx, _ptr(w2), ldw, _ptr(p),
                                     ldp, act, M, N, K, _ptr(dx), K, _ptr(dw), K, _ptr(db),
                                     _ptr(dz), N, _ptr(ws), nbytes,
                                     _stream_of(grad_out, stream)))
    return LinearGrads(x=dx, weight=dw, bias=db,
                       pre=(dz if act else grad_out) if want_pre else None)


def adjust_logits(logits, history=None, history_lengths=None, repetition: float = 1.0,
                  presence: float = 0.0, frequency: float = 0.0, row_penalties=None, bias=None,
                  allowed=None, graph: Optional[Graph] = None, states=None,
                  normalize: bool = False, out=None, stream=None):
    """Logits [..., V] with penalties for the labels of each row's history, biases, masks
    and, with normalize, their log-softmax (tbs_adjust_logits); float32, bfloat16 or float16.
    history int32 [R, L] (entries outside [0, V), such as -1 padding, do not count),
    history_lengths int32 [R]; row_penalties float32 [R, 3] (repetition, presence, frequency)
    in place of the three numbers; bias float32 [V] or [R, V]; allowed int32 [W] or [R, W],
    W = (V + 31) // 32: bit v % 32 of word v // 32 allows label v; graph and states int32
    [R]: only blank and the labels on arcs out of each row's state (-1: no such mask).
    out: a tensor like logits, or logits itself.  A history of a transducer's labels holds no
    blank, so that penalties favour blank over every label that was given; a negative bias[0]
    counters that.  Autograd does not see the call."""
    import torch
    with _scope(logits, stream):
        code = _dtype_code(logits)
        if logits.dim() == 0 or logits.shape[-1] == 0:
            raise ValueError("logits must be [..., V]")
        V, i32 = _size(logits.shape[-1], "logits"), torch.int32
        z, ldz = _matrix(logits, logits, V, "logits")
        R, lead = _size(z.shape[0], "logits"), logits.shape[:-1]
        if (graph is None) != (states is None):
            raise ValueError("graph and states go together")
        a = Adjustments(repetition=float(repetition), presence=float(presence),
                        frequency=float(frequency), normalize=int(bool(normalize)))
        keep = []
        if history is not None:
            if history.dim() != 2:
                raise ValueError("history must be [R, L]")
            cols = _size(history.shape[1], "history")
            h, ldh = _matrix(history, logits, cols, "history", i32, rows=R)
            a.history, a.ld_history, a.history_cols = _ptr(h), ldh, cols
            keep.append(h)
        elif history_lengths is not None or row_penalties is not None:
            raise ValueError("history_lengths and row_penalties go with a history")
        if history_lengths is not None:
            keep.append(_vector(history_lengths, logits, R, "history_lengths", i32))
            a.history_lengths = _ptr(keep[-1])
        if row_penalties is not None:
            rp, _ = _matrix(row_penalties, logits, 3, "row_penalties", torch.float32, rows=R,
                            lead=lead)
            keep.append(rp.contiguous())
            a.row_penalties = _ptr(keep[-1])
        if bias is not None:
            m, a.ld_bias = _matrix(bias, logits, V, "bias", torch.float32, rows=R, one_row=True,
                                   lead=lead)
            a.bias = _ptr(m)
            keep.append(m)
        if allowed is not None:
            m, a.ld_allowed = _matrix(allowed, logits, (V + 31) // 32, "allowed", i32, rows=R,
                                      one_row=True, lead=lead)
            a.allowed = _ptr(m)
            keep.append(m)
        if graph is not None:
            keep.append(_vector(states, logits, R, "states", i32))
            a.graph, a.states = graph._h, _ptr(keep[-1])
        if out is None:
            out, o, ldo = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device), None, V
        else:
            if out.shape != logits.shape:
                raise ValueError("out must have the shape of logits")
            o, ldo = _matrix(out, logits, V, "out")
            if R > 0 and o.data_ptr() != out.data_ptr():
                raise ValueError("out must have contiguous rows at one distance")
        L = lib()
        nbytes = L.tbs_adjust_logits_workspace(code, R, V, 1) if normalize else 0
        ws = _workspace(nbytes, logits)
        _check(L.tbs_adjust_logits(code, _ptr(z), ldz, R, V, ctypes.byref(a),
                                   _ptr(out if o is None else o), ldo, _ptr(ws), nbytes,
                                   _stream_of(logits, stream)))
    return out


def transducer_gradient(kind: str, blank, label, lengths, weights=None, stream=None):
    """Log-likelihoods of ``transducer_forward`` and the gradient of
    sum(weights * total) with respect to blank and label (tbs_transducer_gradient); weights
    float64 [B] (None: 1 each).  Returns (total [B] float64, grad_blank [B, T, U+1],
    grad_label [B, T, U] float32, status [B] int32); gradients are 0 outside each utterance's
    lengths.  lengths as a device int32 tensor [B, 2] costs no host copy.  The gradients are
    results: autograd does not see the call."""
    import torch
    if blank.dim() != 3 or blank.shape[2] < 1:
        raise ValueError("blank must be [B, T, U + 1]")
    B, T, U1 = (_size(n, "blank") for n in blank.shape)
    U, f32 = U1 - 1, torch.float32
    if tuple(label.shape) != (B, T, U) or label.device != blank.device:
        raise ValueError("label must be [B, T, U] beside blank [B, T, U + 1]")
    if blank.dtype != f32 or label.dtype != f32:
        raise ValueError("blank and label must be float32")
    with _scope(blank, stream):
        dev = blank.device
        lengths = torch.as_tensor(lengths, dtype=torch.int32).reshape(B, 2).to(dev).contiguous()
        if weights is not None:
            weights = _vector(torch.as_tensor(weights, dtype=torch.float64, device=dev), blank, B,
                              "weights", torch.float64)
        blank, label = blank.contiguous(), label.contiguous()
        total = torch.empty(B, dtype=torch.float64, device=dev)
        status = torch.empty(B, dtype=torch.int32, device=dev)
        grad_blank, grad_label = torch.empty_like(blank), torch.empty_like(label)
        L = lib()
        nbytes = L.tbs_transducer_gradient_workspace(B, T, U)
        ws = _workspace(nbytes, blank)
        _check(L.tbs_transducer_gradient(
            TRANSDUCER_KINDS[kind], _ptr(blank), _ptr(label), _ptr(lengths), _ptr(weights), B, T,
            U, _ptr(total), _ptr(grad_blank), _ptr(grad_label), _ptr(status), _ptr(ws), nbytes,
            _stream_of(blank, stream)))
    return total, grad_blank, grad_label, status
