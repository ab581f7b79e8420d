"""MI355X-native sampler of multi-hop query training data (SMORE, arXiv 2110.14890).

Thin Python binding over the C ABI of ``libsmore.so`` (declared in
``include/smore.h``).  It only marshals arguments: graph building, reverse
directional sampling of positives and bidirectional rejection sampling of
negatives all run in the library's HIP kernels.  PyTorch provides device
memory and the current HIP stream.  There is no CPU fallback: if the library
is not built, every call raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
import weakref

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsmore.so")

TYPES = ("1p", "2p", "3p", "2i", "3i", "ip", "pi", "2u", "up", "2in", "3in", "inp", "pin", "pni")
ADD_INVERSE = 1
MAX_NEG_TRIES = 4096
OP_ANCHOR, OP_PROJ, OP_AND, OP_OR, OP_NOT = range(5)
ERRORS = {0: "OK", -1: "INVALID_ARG", -2: "RANGE", -3: "UNSUPPORTED", -4: "NOMEM", -5: "HIP",
          -6: "OVERFLOW"}

c_i32, c_i64, c_u32, c_u64, c_vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p


class DagNode(ctypes.Structure):
    _fields_ = [("op", c_i32), ("n_child", c_i32), ("child", c_i32 * 3), ("slot", c_i32)]


class QueryDag(ctypes.Structure):
    _fields_ = [("n_nodes", c_i32), ("root", c_i32), ("node", DagNode * 16)]


class SampleArgs(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("n_neg", c_i32), ("pos_tries", c_i32), ("neg_tries", c_i32),
                ("max_fanout", c_i32), ("seed", c_u64), ("query_offset", c_u64), ("flags", c_u32)]


class SampleOut(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in ("anchors", "relations", "positive", "negatives", "n_valid",
                                    "pos_attempts", "neg_draws")]


SHARED_FIELDS = ("anchors", "relations", "positive", "pos_attempts", "shared", "n_shared", "mask",
                 "n_valid")


class SharedOut(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in SHARED_FIELDS]


OUT_FIELDS = ("anchors", "relations", "positive", "negatives", "n_valid", "pos_attempts",
              "neg_draws")


F32, BF16, F16 = range(3)
PREFERENCE_KINDS = {"pairs": 0, "softmax": 1}
ADAMW_BLOCK = 128
ADAMW_STOCHASTIC = 1


class ScoreArgs(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("n", c_i32), ("dim", c_i32), ("n_rows", c_i32),
                ("table_stride", c_i64), ("query_stride", c_i64), ("candidate_stride", c_i64),
                ("score_stride", c_i64), ("table_type", c_i32), ("query_type", c_i32)]


class PreferenceArgs(ctypes.Structure):
    _fields_ = [("batch", c_i32), ("n", c_i32), ("kind", c_i32), ("score_type", c_i32),
                ("beta", ctypes.c_float), ("smoothing", ctypes.c_float), ("scale", ctypes.c_float),
                ("positive_stride", c_i64), ("negatives_stride", c_i64),
                ("ref_positive_stride", c_i64), ("ref_negatives_stride", c_i64),
                ("grad_positive_stride", c_i64), ("grad_negatives_stride", c_i64)]


class PreferenceIn(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in ("positive", "negatives", "ref_positive", "ref_negatives",
                                    "n_valid", "mask", "weight")]


class PreferenceOut(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in ("loss", "grad_positive", "grad_negatives")]


class AdamWTensor(ctypes.Structure):
    _fields_ = [(n, c_vp) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "rows",
                                    "order", "coef")] + \
               [(n, c_i64) for n in ("n_rows", "dim", "n_entries", "per")] + \
               [(n, c_i32) for n in ("param_type", "grad_type", "bits", "index")] + \
               [("weight_decay", ctypes.c_float)]


class AdamWArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps")] + \
               [("step", c_i64), ("step_device", c_vp), ("lr_device", c_vp), ("grad_scale", c_vp),
                ("seed", c_u64), ("flags", c_u32)]


class SmoreError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                               "(python paper_2110_14890_amd/build.py)")
        L = ctypes.CDLL(LIB_PATH)
        L.smore_last_error.restype = ctypes.c_char_p
        L.smore_build_graph.argtypes = [c_vp, c_i64, c_i32, c_i32, c_u32, ctypes.POINTER(c_vp)]
        L.smore_graph_info.argtypes = [c_vp] + [ctypes.POINTER(c_i64)] * 6
        L.smore_graph_copy.argtypes = [c_vp, c_i32, c_vp, c_i64]
        L.smore_query_preset.argtypes = [ctypes.c_char_p, ctypes.POINTER(QueryDag)]
        L.smore_plan.argtypes = [ctypes.POINTER(QueryDag), c_i32, ctypes.POINTER(c_i32),
                                 ctypes.POINTER(c_i32)]
        L.smore_sample_workspace_bytes.argtypes = [c_vp, ctypes.POINTER(QueryDag),
                                                   ctypes.POINTER(SampleArgs),
                                                   ctypes.POINTER(ctypes.c_size_t)]
        L.smore_sample.argtypes = [c_vp, ctypes.POINTER(QueryDag), ctypes.POINTER(SampleArgs),
                                   ctypes.POINTER(SampleOut), c_vp, ctypes.c_size_t, c_vp]
        L.smore_sample_noalloc.argtypes = [c_vp, ctypes.POINTER(QueryDag), ctypes.POINTER(SampleArgs),
                                           ctypes.POINTER(SampleOut), c_vp]
        L.smore_sample_shared.argtypes = [c_vp, ctypes.POINTER(QueryDag), ctypes.POINTER(SampleArgs),
                                          ctypes.POINTER(SharedOut), c_vp, ctypes.c_size_t, c_vp]
        L.smore_verify.argtypes = [c_vp, ctypes.POINTER(QueryDag), ctypes.POINTER(SampleArgs), c_vp,
                                   c_vp, c_vp, c_vp, c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.smore_sample_positives.argtypes = [c_vp, ctypes.POINTER(QueryDag),
                                             ctypes.POINTER(SampleArgs), ctypes.POINTER(SampleOut),
                                             c_vp]
        L.smore_sample_negatives.argtypes = [c_vp, ctypes.POINTER(QueryDag),
                                             ctypes.POINTER(SampleArgs), ctypes.POINTER(SampleOut),
                                             c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.smore_sample_negatives_part.argtypes = [c_vp, ctypes.POINTER(QueryDag),
                                                  ctypes.POINTER(SampleArgs),
                                                  ctypes.POINTER(SampleOut), c_vp, c_i32, c_vp,
                                                  ctypes.c_size_t, c_vp]
        L.smore_profile_kernel.argtypes = [c_vp, c_vp, c_i32]
        L.smore_wait_before_kernel.argtypes = [c_vp, c_i32]
        L.smore_gather_probe.argtypes = [c_vp, c_i64, c_i64, c_vp, c_i64, c_vp]
        sp = ctypes.POINTER(ctypes.c_size_t)
        L.smore_score.argtypes = [c_vp] * 6
        L.smore_score_grad_workspace_bytes.argtypes = [c_vp, sp]
        L.smore_score_grad.argtypes = [c_vp] * 6 + [ctypes.c_size_t, c_vp]
        L.smore_preference_loss.argtypes = [c_vp] * 4
        L.smore_sort_rows_workspace_bytes.argtypes = [c_i64, c_i32, sp]
        L.smore_sort_rows.argtypes = [c_vp, c_i64, c_i32, c_vp, c_vp, c_vp, ctypes.c_size_t, c_vp]
        L.smore_adamw_workspace_bytes.argtypes = [c_vp, c_i32, sp]
        L.smore_adamw.argtypes = [c_vp, c_i32, ctypes.POINTER(AdamWArgs), c_vp, ctypes.c_size_t,
                                  c_vp]
        L.smore_free_graph.argtypes = [c_vp]
        L.smore_free_graph.restype = None
        _lib = L
    return _lib


def last_error() -> str:
    return lib().smore_last_error().decode()


def _check(rc: int) -> None:
    if rc != 0:
        raise SmoreError(rc, last_error())


def query_preset(name: str) -> QueryDag:
    d = QueryDag()
    _check(lib().smore_query_preset(name.encode(), ctypes.byref(d)))
    return d


def plan(dag: "QueryDag | str", tie_break: int = 0) -> list:
    if isinstance(dag, str):
        dag = query_preset(dag)
    cut = (c_i32 * 16)()
    n = c_i32()
    _check(lib().smore_plan(ctypes.byref(dag), tie_break, cut, ctypes.byref(n)))
    return [cut[k] for k in range(n.value)]


class Graph:
    """Device adjacency owned by the library (smore_build_graph / smore_free_graph)."""

    def __init__(self, triples, n_entities: int, n_relations: int, add_inverse: bool = False):
        tr = np.ascontiguousarray(triples, dtype=np.int32).reshape(-1, 3)
        h = c_vp()
        _check(lib().smore_build_graph(tr.ctypes.data if len(tr) else None, len(tr), n_entities,
                                       n_relations, ADD_INVERSE if add_inverse else 0,
                                       ctypes.byref(h)))
        self._h = h
        vals = [c_i64() for _ in range(6)]
        _check(lib().smore_graph_info(h, *[ctypes.byref(v) for v in vals]))
        (self.V, self.R, self.E, self.S_fwd, self.S_rev, self.device_bytes) = [v.value for v in vals]

    @property
    def handle(self):
        return self._h

    _SIZES = {0: "V+1", 1: "2*(S_fwd+1)", 2: "E", 3: "V+1", 4: "2*(S_rev+1)", 5: "E", 6: "A"}

    def copy(self, which: int, count: int) -> np.ndarray:
        out = np.zeros(max(count, 1), np.int32)
        _check(lib().smore_graph_copy(self._h, which, out.ctypes.data, count))
        return out[:count]

    def close(self) -> None:
        if getattr(self, "_h", None):
            lib().smore_free_graph(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def build_graph(triples, n_entities: int, n_relations: int, add_inverse: bool = False) -> Graph:
    return Graph(triples, n_entities, n_relations, add_inverse)


def make_args(batch: int, n_neg: int, seed: int = 0, query_offset: int = 0, pos_tries: int = 64,
              neg_tries: int | None = None, max_fanout: int = 0, flags: int = 0) -> SampleArgs:
    if neg_tries is None:
        neg_tries = 4 * n_neg
    return SampleArgs(batch, n_neg, pos_tries, neg_tries, max_fanout, seed, query_offset, flags)


def alloc_outputs(batch: int, n_neg: int, device=None) -> dict:
    import torch
    dev = device if device is not None else torch.device("cuda", torch.cuda.current_device())
    z = lambda *s: torch.empty(s, dtype=torch.int32, device=dev)
    return {"anchors": z(batch, 3), "relations": z(batch, 3), "positive": z(batch),
            "negatives": z(batch, n_neg), "n_valid": z(batch), "pos_attempts": z(batch),
            "neg_draws": z(batch)}


def workspace_bytes(dag: QueryDag, args: SampleArgs) -> int:
    n = ctypes.c_size_t()
    _check(lib().smore_sample_workspace_bytes(None, ctypes.byref(dag), ctypes.byref(args),
                                              ctypes.byref(n)))
    return n.value


class Workspace:
    """Device scratch for the sampling calls, grown on demand (a uint8 torch
    tensor).  One per stream: calls that overlap must not share it."""

    def __init__(self, device=None):
        self.device = device
        self.buf = None

    def get(self, nbytes: int):
        import torch
        if self.buf is None or self.buf.numel() < nbytes:
            dev = self.device if self.device is not None else torch.device(
                "cuda", torch.cuda.current_device())
            self.buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
        return self.buf


_default_ws = {}


def _workspace(ws, dag, args, stream=None):
    """The caller's workspace, or a default one per (device, stream) the call
    runs on, so that calls on different streams never share scratch."""
    import torch
    if args.n_neg == 0:        # nothing is drawn: the library needs no workspace
        return None, 0
    if ws is None:
        st = stream if stream is not None else torch.cuda.current_stream()
        key = (st.device, st.cuda_stream)
        ws = _default_ws.setdefault(key, Workspace(st.device))
    buf = ws.get(workspace_bytes(dag, args))
    return c_vp(buf.data_ptr()), buf.numel()


def sample_into(graph: Graph, dag: QueryDag, args: SampleArgs, out: dict, stream=None,
                workspace: "Workspace | None" = None) -> dict:
    """smore_sample into caller-owned torch tensors on the current (or given) stream."""
    _require(out, _sample_shapes(args))
    wp, wn = _workspace(workspace, dag, args, stream)
    _check(lib().smore_sample(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                              ctypes.byref(_out_struct(out)), wp, wn, _stream_handle(stream)))
    return out


NOALLOC_SCRATCH_BYTES = 64 << 20


def sample_noalloc_into(graph: Graph, dag: QueryDag, args: SampleArgs, out: dict,
                        stream=None) -> dict:
    """smore_sample_noalloc: smore_sample without a workspace argument (the
    library's fixed per-device scratch; calls on one GPU must not overlap)."""
    _require(out, _sample_shapes(args))
    _check(lib().smore_sample_noalloc(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                                      ctypes.byref(_out_struct(out)), _stream_handle(stream)))
    return out


def alloc_shared_outputs(batch: int, n_shared: int, device=None) -> dict:
    """Device outputs of sample_shared_into (the mask is int32 storage of the
    uint32 words)."""
    import torch
    dev = device if device is not None else torch.device("cuda", torch.cuda.current_device())
    z = lambda *s: torch.empty(s, dtype=torch.int32, device=dev)
    return {"anchors": z(batch, 3), "relations": z(batch, 3), "positive": z(batch),
            "pos_attempts": z(batch), "shared": z(n_shared), "n_shared": z(1),
            "mask": z(batch, (n_shared + 31) // 32), "n_valid": z(batch)}


def sample_shared_into(graph: Graph, dag: QueryDag, args: SampleArgs, out: dict, stream=None,
                       workspace: "Workspace | None" = None) -> dict:
    """smore_sample_shared: args.n_neg is the size of the shared candidate set."""
    b, n = args.batch, args.n_neg
    _require(out, {"anchors": (b, 3), "relations": (b, 3), "positive": (b,), "pos_attempts": (b,),
                   "shared": (n,), "n_shared": (1,), "mask": (b, (n + 31) // 32), "n_valid": (b,)})
    wp, wn = _workspace(workspace, dag, args, stream)
    st = SharedOut(*[out[k].data_ptr() if out[k].numel() else None for k in SHARED_FIELDS])
    _check(lib().smore_sample_shared(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                                     ctypes.byref(st), wp, wn, _stream_handle(stream)))
    return out


def sample_shared(graph: Graph, qtype: "str | QueryDag", batch: int, n_shared: int, seed: int = 0,
                  query_offset: int = 0, pos_tries: int = 64, neg_tries: int | None = None,
                  max_fanout: int = 0, stream=None) -> dict:
    """A minibatch of `batch` queries sharing one set of `n_shared` candidate
    negatives, with the mask of verified negatives per query."""
    dag = query_preset(qtype) if isinstance(qtype, str) else qtype
    args = make_args(batch, n_shared, seed, query_offset, pos_tries, neg_tries, max_fanout)
    out = alloc_shared_outputs(batch, n_shared)
    return sample_shared_into(graph, dag, args, out, stream)


def verify(graph: Graph, qtype: "str | QueryDag", anchors, relations, candidates, stream=None,
           workspace: "Workspace | None" = None) -> dict:
    """smore_verify: which of the candidates (device int32 [batch, n]) are
    entities outside each query's answer set.  Returns {"mask" (int32
    storage of the uint32 words), "n_valid"}."""
    import torch
    dag = query_preset(qtype) if isinstance(qtype, str) else qtype
    batch, n = candidates.shape
    for name, t, shape in (("anchors", anchors, (batch, 3)), ("relations", relations, (batch, 3)),
                           ("candidates", candidates, (batch, n))):
        if tuple(t.shape) != shape or t.dtype != torch.int32 or not t.is_contiguous() \
                or t.device != candidates.device or not t.is_cuda:
            raise ValueError(f"{name} must be a contiguous int32 device tensor of shape {shape}")
    args = make_args(batch, n, neg_tries=n)
    dev = candidates.device
    out = {"mask": torch.empty((batch, (n + 31) // 32), dtype=torch.int32, device=dev),
           "n_valid": torch.empty(batch, dtype=torch.int32, device=dev)}
    wp, wn = _workspace(workspace, dag, args, stream)
    ptr = lambda t: t.data_ptr() if t.numel() else None
    _check(lib().smore_verify(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                              anchors.data_ptr(), relations.data_ptr(), ptr(candidates),
                              ptr(out["mask"]), out["n_valid"].data_ptr(), wp, wn,
                              _stream_handle(stream)))
    return out


def _require(tensors: dict, shapes: dict, dtype_name: str = "int32") -> None:
    """Caller-provided device buffers must have the sizes the kernels write:
    the C ABI cannot see a device buffer's length."""
    import torch
    dtype = getattr(torch, dtype_name)
    size = {}
    for k, shape in shapes.items():
        n = 1
        for d in shape:
            n *= d
        size[k] = n
        if tensors.get(k) is None and n:
            raise ValueError(f"{k}: missing (needs {n} {dtype_name})")
    dev = None
    for k, shape in shapes.items():
        t, n = tensors.get(k), size[k]
        if t is None:
            continue
        if t.dtype != dtype or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
            raise ValueError(f"{k} must be a contiguous {dtype_name} device tensor of shape "
                             f"{tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
        if dev is not None and t.device != dev:
            raise ValueError(f"{k} is on {t.device}, other buffers on {dev}")
        dev = t.device


def _sample_shapes(args: SampleArgs, negatives: bool = True) -> dict:
    b = args.batch
    shapes = {"anchors": (b, 3), "relations": (b, 3), "positive": (b,), "n_valid": (b,),
              "pos_attempts": (b,)}
    if negatives:
        shapes.update({"negatives": (b, args.n_neg), "neg_draws": (b,)})
    return shapes


def _out_struct(out: dict) -> SampleOut:
    return SampleOut(*[out[k].data_ptr() if k in out and out[k].numel() else None
                       for k in OUT_FIELDS])


def _stream_handle(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return c_vp(stream.cuda_stream)


def sample_positives(graph: Graph, dag: QueryDag, args: SampleArgs, out: dict, stream=None) -> dict:
    """First stage only (smore_sample_positives): anchors, relations, positive,
    pos_attempts, n_valid."""
    _require(out, _sample_shapes(args, negatives=False))
    _check(lib().smore_sample_positives(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                                        ctypes.byref(_out_struct(out)), _stream_handle(stream)))
    return out


NEG_PREPARE, NEG_CANDIDATES, NEG_REST = 0, 1, 2


def sample_negatives(graph: Graph, dag: QueryDag, args: SampleArgs, out: dict, stats=None,
                     stream=None, workspace: "Workspace | None" = None, part=None) -> dict:
    """Second stage only (smore_sample_negatives) on the queries in `out`;
    stats: optional int64 [batch, 4] device tensor: (bytes, 64-byte lines) of
    graph data read per query by the candidate kernel, then by the kernel
    that intersects long lists.  part: None for the whole stage, else one of
    NEG_PREPARE, NEG_CANDIDATES, NEG_REST (smore_sample_negatives_part: the
    caller orders the three parts and passes the same workspace to each)."""
    if part is not None and workspace is None:
        raise ValueError("the parts of one negatives call must share an explicit workspace")
    _require(out, _sample_shapes(args))
    if stats is not None:
        _require({"stats": stats}, {"stats": (args.batch, 4)}, "int64")
    sp = c_vp(stats.data_ptr()) if stats is not None else None
    wp, wn = _workspace(workspace, dag, args, stream)
    if part is None:
        _check(lib().smore_sample_negatives(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                                            ctypes.byref(_out_struct(out)), sp, wp, wn,
                                            _stream_handle(stream)))
    else:
        _check(lib().smore_sample_negatives_part(graph.handle, ctypes.byref(dag), ctypes.byref(args),
                                                 ctypes.byref(_out_struct(out)), sp, part, wp, wn,
                                                 _stream_handle(stream)))
    return out


KERNEL_CANDIDATES, KERNEL_HEAVY, KERNEL_SELECT = 0, 1, 2


def profile_kernel(start_event, stop_event, which: int = KERNEL_CANDIDATES) -> None:
    """Arm torch.cuda.Event objects (enable_timing=True) to be recorded around
    one kernel of the next negatives call on this thread (smore_profile_kernel)."""
    for ev in (start_event, stop_event):
        if not ev.cuda_event:          # torch creates the HIP event on first use
            ev.record()
    _check(lib().smore_profile_kernel(c_vp(start_event.cuda_event), c_vp(stop_event.cuda_event),
                                      which))


def wait_before_kernel(event, which: int = KERNEL_CANDIDATES) -> None:
    """The next negatives call on this thread waits on the torch.cuda.Event
    right before its first candidate kernel (smore_wait_before_kernel);
    None disarms."""
    if event is None:
        _check(lib().smore_wait_before_kernel(None, which))
        return
    if not event.cuda_event:           # torch creates the HIP event on first use
        event.record()
    _check(lib().smore_wait_before_kernel(c_vp(event.cuda_event), which))


def sample(graph: Graph, qtype: "str | QueryDag", batch: int, n_neg: int, seed: int = 0,
           query_offset: int = 0, pos_tries: int = 64, neg_tries: int | None = None,
           max_fanout: int = 0, stream=None) -> dict:
    """Sample `batch` queries: dict of int32 device tensors (see include/smore.h)."""
    dag = query_preset(qtype) if isinstance(qtype, str) else qtype
    args = make_args(batch, n_neg, seed, query_offset, pos_tries, neg_tries, max_fanout)
    out = alloc_outputs(batch, n_neg)
    return sample_into(graph, dag, args, out, stream)


def gather_probe(table, n_reads: int, stream=None):
    """Random-read ceiling probe (smore_gather_probe): n_reads random 4-byte
    reads from the device tensor `table`.  Returns the sink tensor; time it
    with events on `stream`."""
    import torch

    threads = (n_reads + 63) // 64
    sink = torch.empty(threads, dtype=torch.int32, device=table.device)
    st = stream if stream is not None else torch.cuda.current_stream(table.device)
    _check(lib().smore_gather_probe(c_vp(table.data_ptr()), table.numel() * table.element_size(),
                                    n_reads, c_vp(sink.data_ptr()), threads, c_vp(st.cuda_stream)))
    return sink


# ------------------------------------------------- training on sampled batches
# Gradients are outputs and inputs of these calls, as the C ABI has them:
# autograd does not see the calls (queries.backward(score_grad(...)) goes on
# into a model's own graph).
#
# A call's stream is the device's current one, or the one given as stream.  The
# caller makes a given stream wait for what made the inputs, and waits for it
# before using the outputs, which belong to that stream.  Inputs and outputs
# may be let go of as soon as the call returns: their memory is kept until the
# stream has got there.
#
# Small calls take as long as this binding does, so the checks of a call are
# plain comparisons; what is wrong is spelled out only where one fails.
_torch = None
_TYPES = {}          # element types of the C ABI


def _packer(structure):
    """struct.pack for a structure of the C ABI: the bytes of a call's
    arguments in one step (filling a ctypes structure takes microseconds)."""
    letters = {c_i32: "i", c_i64: "q", c_u32: "I", c_u64: "Q", c_vp: "P", ctypes.c_float: "f", ctypes.c_double: "d"}
    packed = struct.Struct("@" + "".join(letters[kind] for _, kind in structure._fields_) + "0q")
    assert packed.size == ctypes.sizeof(structure)
    return packed.pack


_pack_score, _pack_preference = _packer(ScoreArgs), _packer(PreferenceArgs)
_pack_in, _pack_out = _packer(PreferenceIn), _packer(PreferenceOut)


def _lazy_torch():
    global _torch
    if _torch is None:
        import torch
        _TYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
        _torch = torch
    return _torch


def _launch(device, stream, call, uses=()):
    """call(stream handle) with the device current and its stream: the given
    one, or the device's current stream.  Tensors that call makes belong to
    that stream; of a given one, the tensors of uses are not given back to the
    allocator before it has got there."""
    torch = _torch
    if device.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, not on {device}")
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
        with torch.cuda.stream(stream):
            result = call(stream.cuda_stream)
        for t in uses:
            if t is not None:
                t.record_stream(stream)
        return result
    if torch.cuda.current_device() == device.index:
        return call(torch._C._cuda_getCurrentRawStream(device.index))
    with torch.cuda.device(device):
        return call(torch._C._cuda_getCurrentRawStream(device.index))


def _fits(t, shape, dtype, index: int) -> bool:
    """A tensor of this shape and type on this GPU whose rows are contiguous
    (the distance of two rows is free)."""
    return t.shape == shape and t.dtype is dtype and t.get_device() == index and \
        (len(shape) < 2 or shape[1] < 2 or t.stride(1) == 1)


def _operand(name: str, t, shape, dtypes, device) -> None:
    """Says what of _fits() does not hold."""
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be one of {[str(d) for d in dtypes]}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on the device of the other tensors ({device}), it is on {t.device}")
    if len(shape) == 2 and shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"rows of {name} must be contiguous")


def _pitch(t, length: int) -> int:
    """Distance of two rows of a matrix (its length for a single row)."""
    return t.stride(0) if t.shape[0] > 1 else length


def _ptr(t):
    return t.data_ptr() if t is not None and t.numel() else None


def _score_args(table, candidates, other, other_name: str, grad_scores, grad_name: str) -> bytes:
    """Checks and sizes (ScoreArgs) of a score call: other [batch, dim], grad_scores [batch, n]."""
    torch = _torch
    if table.dim() != 2 or candidates.dim() != 2:
        raise ValueError("table and candidates must be matrices")
    v, dim = table.shape
    shape = candidates.shape
    batch, n = shape
    index, te, tq = table.get_device(), table.dtype, other.dtype
    wide = (torch.float32, torch.bfloat16)
    if not (te in wide and tq in wide and _fits(table, table.shape, te, index)
            and _fits(candidates, shape, torch.int32, index) and _fits(other, (batch, dim), tq, index)
            and _fits(grad_scores, shape, torch.float32, index)):
        device = table.device
        _operand("table", table, table.shape, wide, device)
        _operand("candidates", candidates, shape, (torch.int32,), device)
        _operand(other_name, other, (batch, dim), wide, device)
        _operand(grad_name, grad_scores, shape, (torch.float32,), device)
    if batch > 1:     # rows of the candidates may coincide: one set for all queries
        return _pack_score(batch, n, dim, v, _pitch(table, dim), other.stride(0), candidates.stride(0),
                           grad_scores.stride(0), _TYPES[te], _TYPES[tq])
    return _pack_score(batch, n, dim, v, _pitch(table, dim), dim, n, n, _TYPES[te], _TYPES[tq])


def score_into(table, queries, candidates, scores, stream=None):
    """smore_score into the caller's fp32 tensor [batch, n]."""
    _lazy_torch()
    args = _score_args(table, candidates, queries, "queries", scores, "scores")
    _check(_launch(table.device, stream, lambda st: lib().smore_score(
        args, _ptr(table), _ptr(queries), _ptr(candidates), _ptr(scores), st), (table, queries, candidates, scores)))
    return scores


def score(table, queries, candidates, stream=None):
    """Scores (fp32 [batch, n]) of each query's candidates (int32 [batch, n], as
    sampled): the product of queries [batch, dim] with the candidates' rows of
    table [V, dim], 0 for candidates outside [0, V) (smore_score).  For one
    candidate set shared by all queries, candidates.expand(batch, n) works,
    but a matrix product with the set's rows is the faster way.

    Autograd does not see the call, whether or not its inputs require
    gradients: the scores have no history.  Their gradients are score_grad()
    for the queries and row_grad() for the table.

    stream: a torch.cuda.Stream to run on instead of the current one.  The
    caller makes it wait for what made the inputs, and waits for it before
    using the scores; the inputs may be let go of at once.  The same holds for
    the other training calls."""
    torch = _lazy_torch()
    new = lambda _: torch.empty(candidates.shape, dtype=torch.float32, device=table.device)
    scores = new(None) if stream is None else _launch(table.device, stream, new)
    return score_into(table, queries, candidates, scores, stream)


def score_grad_into(table, candidates, grad_scores, grad_queries, stream=None):
    """smore_score_grad into the caller's tensor [batch, dim]."""
    torch = _lazy_torch()
    args = _score_args(table, candidates, grad_queries, "grad_queries", grad_scores, "grad_scores")
    L, need = lib(), ctypes.c_size_t()
    _check(L.smore_score_grad_workspace_bytes(args, ctypes.byref(need)))
    need = need.value

    def call(st):
        # a workspace of this call alone, from the stream's (or the capturing graph's) memory
        ws = torch.empty(need, dtype=torch.uint8, device=table.device) if need else None
        return L.smore_score_grad(args, _ptr(table), _ptr(candidates), _ptr(grad_scores),
                                  _ptr(grad_queries), _ptr(ws), need, st)

    _check(_launch(table.device, stream, call, (table, candidates, grad_scores, grad_queries)))
    return grad_queries


def score_grad(table, candidates, grad_scores, dtype=None, stream=None):
    """Gradient of score() for the queries, [batch, dim] in dtype (fp32): the
    sum of the candidates' rows, each times its entry of grad_scores (fp32
    [batch, n]).  The gradient for the table is AdamW's: row_grad().  Nothing is
    accumulated into .grad; queries.backward(score_grad(...)) goes on into the
    graph that the queries came from."""
    torch = _lazy_torch()
    new = lambda _: torch.empty((candidates.shape[0], table.shape[1]), dtype=dtype or torch.float32, device=table.device)
    out = new(None) if stream is None else _launch(table.device, stream, new)
    return score_grad_into(table, candidates, grad_scores, out, stream)


def _check_preference(batch, n, dtype, device, tensors: dict, vectors: dict) -> None:
    """Says what is wrong with the tensors of a preference_loss call."""
    torch = _torch
    if dtype not in _TYPES:
        raise ValueError(f"scores must be fp32, bf16 or fp16, got {dtype}")
    for name, t in tensors.items():
        if t is not None:
            _operand(name, t, (batch, n) if "negatives" in name else (batch,), (dtype,), device)
    for name, t in vectors.items():
        if t is not None:
            _operand(name, t, (batch, (n + 31) // 32) if name == "mask" else (batch,),
                     (torch.int32,) if name in ("n_valid", "mask") else (torch.float32,), device)
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")


def preference_loss_into(positive, negatives, out: dict, ref_positive=None, ref_negatives=None, n_valid=None,
                         mask=None, kind: str = "pairs", beta: float = 0.1, smoothing: float = 0.0, weight=None,
                         stream=None) -> dict:
    """smore_preference_loss into the caller's tensors: out has "loss" (fp32
    [batch]), or "grad_positive" [batch] and "grad_negatives" [batch, n] of
    the scores' type, or all three."""
    return _preference(positive, negatives, out, ref_positive, ref_negatives, n_valid, mask, kind, beta, smoothing,
                       weight, stream, False)


def _preference(positive, negatives, out, ref_positive, ref_negatives, n_valid, mask, kind, beta, smoothing, weight,
                stream, fits: bool) -> dict:
    """The call behind preference_loss; fits: out is known to."""
    torch = _lazy_torch()
    number = PREFERENCE_KINDS.get(kind)
    if number is None:
        raise ValueError(f"kind must be one of {sorted(PREFERENCE_KINDS)}, got {kind!r}")
    if negatives.dim() != 2:
        raise ValueError("negatives must be a matrix")
    shape = negatives.shape
    batch, n = shape
    device, dtype = negatives.device, negatives.dtype
    loss, grad_p, grad_n = out.get("loss"), out.get("grad_positive"), out.get("grad_negatives")
    if (ref_positive is None) != (ref_negatives is None):
        raise ValueError("reference scores are given for both, or for neither")
    if (grad_p is None) != (grad_n is None):
        raise ValueError("gradients are wanted for both, or for neither")
    scale = 1.0
    if weight is not None and not isinstance(weight, torch.Tensor):
        scale, weight = float(weight), None
    row, i32, f32, at = (batch,), torch.int32, torch.float32, negatives.get_device()
    good = dtype in _TYPES and _fits(positive, row, dtype, at) and (n < 2 or negatives.stride(1) == 1) \
        and (ref_positive is None or (_fits(ref_positive, row, dtype, at) and _fits(ref_negatives, shape, dtype, at))) \
        and (n_valid is None or (_fits(n_valid, row, i32, at) and n_valid.is_contiguous())) \
        and (mask is None or (_fits(mask, (batch, (n + 31) // 32), i32, at) and mask.is_contiguous())) \
        and (weight is None or (_fits(weight, row, f32, at) and weight.is_contiguous())) \
        and (fits or ((loss is None or (_fits(loss, row, f32, at) and loss.is_contiguous()))
                      and (grad_p is None or (_fits(grad_p, row, dtype, at) and _fits(grad_n, shape, dtype, at)))))
    if not good:
        _check_preference(batch, n, dtype, device,
                          {"positive": positive, "negatives": negatives, "ref_positive": ref_positive,
                           "ref_negatives": ref_negatives, "grad_positive": grad_p, "grad_negatives": grad_n},
                          {"n_valid": n_valid, "mask": mask, "weight": weight, "loss": loss})
    at = lambda t: 0 if t is None else t.data_ptr()
    step = lambda t: 0 if t is None else t.stride(0)
    uses = (positive, negatives, ref_positive, ref_negatives, n_valid, mask, weight, loss, grad_p, grad_n)
    if n == 0:
        negatives = ref_negatives = grad_n = mask = None
    args = _pack_preference(batch, n, number, _TYPES[dtype], beta, smoothing, scale, positive.stride(0), step(negatives),
                            step(ref_positive), step(ref_negatives), step(grad_p), step(grad_n))
    ins = _pack_in(positive.data_ptr(), at(negatives), at(ref_positive), at(ref_negatives), at(n_valid), at(mask), at(weight))
    outs = _pack_out(at(loss), at(grad_p), at(grad_n))
    _check(_launch(device, stream, lambda st: lib().smore_preference_loss(args, ins, outs, st), uses))
    return out


def preference_loss(positive, negatives, ref_positive=None, ref_negatives=None, n_valid=None, mask=None,
                    kind: str = "pairs", beta: float = 0.1, smoothing: float = 0.0, weight=None, grad: bool = True,
                    stream=None) -> dict:
    """Preference loss of each query's positive (scores [batch]) against its
    verified negatives (scores [batch, n]), optionally relative to a reference
    model's scores: {"loss" (fp32 [batch])}, with grad also {"grad_positive",
    "grad_negatives"}, the gradient of the sum of weight (a number or fp32
    [batch], default 1) times loss.  Which negatives count: n_valid as
    sample() gives it, or mask as sample_shared() and verify() give it.  kind
    "pairs" averages the paired losses, with label smoothing; "softmax"
    takes the positive against all negatives at once.  The formulas stand at
    smore_preference_loss.  Scores may be views of one matrix (a column, the
    columns behind it).  Autograd does not see the call: the loss has no
    history, and loss.backward() is not the way to the gradients, which are
    outputs."""
    torch = _lazy_torch()

    def new(_):
        if positive.is_contiguous() and negatives.is_contiguous():      # 9.0 us a call instead of 10.7
            like = torch.empty_like
            if grad:
                return {"loss": like(positive, dtype=torch.float32), "grad_positive": like(positive),
                        "grad_negatives": like(negatives)}
            return {"loss": like(positive, dtype=torch.float32)}
        shape = negatives.shape
        out = {"loss": negatives.new_empty(shape[:1], dtype=torch.float32)}
        if grad:
            out["grad_positive"] = negatives.new_empty(shape[:1])
            out["grad_negatives"] = negatives.new_empty(shape)
        return out

    out = new(None) if stream is None else _launch(negatives.device, stream, new)
    return _preference(positive, negatives, out, ref_positive, ref_negatives, n_valid, mask, kind, beta, smoothing,
                       weight, stream, True)


class RowGrad:
    """The gradient of a table in the rows that a batch touched: entry i of
    rows (int32, ascending, repeats allowed) adds coef[o] times
    grad[o // per], o = order[i], to its row (order int64 and coef fp32 by
    entry, both optional).  Entries outside the table are skipped.  With
    in_order False the rows may be in any order, and rows and coef of any shape
    and strides (order None): AdamW flattens and sorts them, on its stream."""

    def __init__(self, rows, grad, order=None, coef=None, per: int = 1, in_order: bool = True):
        self.rows, self.grad, self.order, self.coef, self.per, self.in_order = rows, grad, order, coef, per, in_order


def row_grad(ids, grad, coef=None, per: int = 1) -> RowGrad:
    """RowGrad of ids in any order and shape (int32): entry i, counted over
    the flattened ids, adds coef[i] times grad[i // per].  With score()'s
    candidates [batch, n] as ids, its queries as grad, the gradient of its
    scores as coef and per = n this is score()'s gradient for the table.
    Nothing is launched before the step."""
    return RowGrad(ids, grad, None, coef, per, in_order=False)


def sort_rows(ids, n_rows: int, stream=None):
    """smore_sort_rows: (rows, order) of ids (int32 [n], contiguous) for a table
    of n_rows rows: rows int32 ascending, ids outside the table last; order
    int64, equal ids in their first order."""
    torch = _lazy_torch()
    if ids.dim() != 1 or ids.dtype != torch.int32 or not ids.is_contiguous():
        raise ValueError(f"ids must be a contiguous int32 vector, got {ids.dtype} {tuple(ids.shape)}")
    L, n, size = lib(), ids.numel(), ctypes.c_size_t()
    _check(L.smore_sort_rows_workspace_bytes(n, n_rows, ctypes.byref(size)))

    def call(st):
        new = lambda count, dtype: torch.empty(count, dtype=dtype, device=ids.device)
        rows, order, ws = new(n, torch.int32), new(n, torch.int64), new(size.value, torch.uint8)
        _check(L.smore_sort_rows(_ptr(ids), n, n_rows, _ptr(rows), _ptr(order), _ptr(ws), size.value, st))
        return rows, order

    return _launch(ids.device, stream, call, (ids,))


def alloc_adamw_state(param, bits: int = 32, table: bool = False) -> dict:
    """Zero moments of a parameter: {"m", "v"}, fp32 of its shape, or in 8
    bits float8_e4m3fn codes of m and sqrt(v) with fp32 scales "m_scale",
    "v_scale" per block of ADAMW_BLOCK elements: of each row for a table
    [V, dim] whose rows are stepped, else of the parameter as one row."""
    torch = _lazy_torch()
    new = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=param.device)
    if bits == 32:
        return {k: new(tuple(param.shape), torch.float32) for k in ("m", "v")}
    if bits != 8:
        raise ValueError(f"moments have 8 or 32 bits, not {bits}")
    if table and param.dim() != 2:
        raise ValueError(f"a table has rows and columns, not shape {tuple(param.shape)}")
    blocks = lambda n: -(-n // ADAMW_BLOCK)
    shape = (param.shape[0], blocks(param.shape[1])) if table else (blocks(param.numel()),)
    state = {k: new(tuple(param.shape), torch.uint8).view(torch.float8_e4m3fn) for k in ("m", "v")}
    state.update({k: new(shape, torch.float32) for k in ("m_scale", "v_scale")})
    return state


class AdamW:
    """AdamW (smore_adamw) over a list of parameters (fp32 or bf16), with
    moments in 32 or 8 bits.

    tables: numbers of the parameters that are tables [V, dim] stepped by
    rows (RowGrad).  states: their moments as alloc_adamw_state makes them,
    e.g. of a checkpoint (they are used, not copied), steps the steps taken.
    seed: roundings to 8 bits and to bf16 are stochastic, keyed by it; None
    rounds to the nearest, with which moments in 8 bits hardly move once they
    have a code (a step changes v by 1 - beta2 of itself, a code is 1/16 to 1/8
    wide): for comparisons only.  "default" is 0 with moments in 8 bits, None
    with 32.  lr: a number, or an fp32 device tensor [1].  device_step:
    the step count is kept in an int64 device tensor, counted up by a kernel,
    so that a captured step counts when it is replayed.

    Moments are in .states, the count in .steps (.device_steps); .lr, .betas,
    .eps and .weight_decay may be changed between steps."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 bits: int = 32, seed: "int | str | None" = "default", tables=(), states=None, steps: int = 0,
                 device_step: bool = False):
        torch = _lazy_torch()
        self.params = list(params)
        if seed == "default":
            seed = 0 if bits == 8 else None
        self.lr, self.betas, self.eps, self.seed, self.steps = lr, betas, eps, seed, steps
        self.weight_decay, self._decays = self._decay_list(weight_decay), None
        if not self.params:
            raise ValueError("no parameters")
        self.device = self.params[0].device
        tables = set(tables)
        if states is None:
            states = [alloc_adamw_state(p, bits, k in tables) for k, p in enumerate(self.params)]
        self.states, self.bits = list(states), bits
        if len(self.states) != len(self.params):
            raise ValueError("one state per parameter is needed")
        self.device_steps = torch.full((1,), steps, dtype=torch.int64, device=self.device) if device_step else None
        # what the library gets for each parameter, the addresses it was made for,
        # whether scales allow steps by rows and of the whole, and its last gradient's type
        n = len(self.params)
        self._list = (AdamWTensor * n)()
        self._items = [self._list[k] for k in range(n)]
        self._seen, self._by_rows, self._whole, self._last, self._empty = ([None] * n for _ in range(5))
        self._take_decays()
        for k in range(n):
            self._describe(k)

    def _decay_list(self, decay) -> list:
        decays = list(decay) if isinstance(decay, (list, tuple)) else [decay] * len(self.params)
        if len(decays) != len(self.params):
            raise ValueError("weight_decay is a number or one per parameter")
        return decays

    def _take_decays(self) -> None:
        """Puts the parameters' decays into the list."""
        self.weight_decay = self._decay_list(self.weight_decay)
        self._decays = list(self.weight_decay)
        for x, decay in zip(self._items, self._decays):
            x.weight_decay = decay

    def _describe(self, k: int) -> None:
        """Checks parameter k and its moments and puts them into the list."""
        torch = _torch
        p, state = self.params[k], self.states[k]
        if p.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"parameter {k} must be fp32 or bf16, got {p.dtype}")
        shapes = {"m": p.shape, "v": p.shape}
        by_rows, whole = True, True
        if self.bits == 8:
            blocks = lambda n: -(-n // ADAMW_BLOCK)
            whole_shape = (blocks(p.numel()),)
            rows_shape = (p.shape[0], blocks(p.shape[1])) if p.dim() == 2 else None
            got = tuple(state["m_scale"].shape)
            by_rows, whole = got == rows_shape, got == whole_shape
            if not by_rows and not whole:
                raise ValueError(f"m_scale of parameter {k} must have shape {whole_shape}"
                                 + (f" or {rows_shape}" if rows_shape else "") + f", got {got}")
            shapes.update(m_scale=got, v_scale=got)
        elif self.bits != 32:
            raise ValueError(f"moments have 8 or 32 bits, not {self.bits}")
        code = torch.float32 if self.bits == 32 else torch.float8_e4m3fn
        for name, t, dtype in [("parameter", p, p.dtype)] + \
                [(n, state[n], code if n in ("m", "v") else torch.float32) for n in shapes]:
            numel = p.numel() if name in ("parameter", "m", "v") else None
            if t.device != self.device or not t.is_cuda or not t.is_contiguous() or t.dtype != dtype or \
                    (numel is not None and t.numel() != numel) or (numel is None and tuple(t.shape) != tuple(shapes[name])):
                raise ValueError(f"{name} of parameter {k} must be a contiguous {dtype} tensor on {self.device} that "
                                 f"fits {tuple(p.shape)}, got {t.dtype} {tuple(t.shape)} on {t.device}")
        x = self._items[k]
        x.param, x.m, x.v = p.data_ptr(), state["m"].data_ptr(), state["v"].data_ptr()
        x.m_scale, x.v_scale = (state["m_scale"].data_ptr(), state["v_scale"].data_ptr()) if self.bits == 8 else (None, None)
        x.n_rows, x.dim = (p.shape[0], p.shape[1]) if p.dim() == 2 else (1, p.numel())
        x.param_type, x.bits, x.index = _TYPES[p.dtype], self.bits, k
        moments = [state[n] for n in shapes]
        at = [t.data_ptr() for t in (p, *moments)]
        # a moment that goes away leaves its address to others: what was found out here ends with it
        ended = lambda _: at.__setitem__(0, None)
        self._seen[k] = (p.shape, p, p.dtype, at, [weakref.ref(t, ended) for t in moments])
        self._by_rows[k], self._whole[k], self._last[k], self._empty[k] = by_rows, whole, None, p.numel() == 0

    def step(self, grads, grad_scale=None, stream=None) -> None:
        """One step.  grads: for each parameter a contiguous tensor of its
        shape (fp32, bf16 or fp16), a RowGrad for a table, or None to leave
        it.  grad_scale: an fp32 device tensor [1] that multiplies every
        gradient (of a norm's clipping, of a scaled loss); nothing is written
        where it is not finite, though the step counts."""
        torch = _torch
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError(f"{len(grads)} gradients for {len(self.params)} parameters")
        used, device, scaled, tables, kept = [], self.device, self.bits == 8, False, []
        if self.weight_decay != self._decays:
            self._take_decays()
        for k, g in enumerate(grads):
            if g is None:
                continue
            p, state, seen = self.params[k], self.states[k], self._seen[k]
            shape = p.shape
            # a parameter or moments that were replaced are looked at again
            at = seen[3]
            if p is not seen[1] or shape != seen[0] or p.dtype is not seen[2] or not p.is_contiguous() \
                    or p.data_ptr() != at[0] or state["m"].data_ptr() != at[1] or state["v"].data_ptr() != at[2] or \
                    (scaled and (state["m_scale"].data_ptr() != at[3] or state["v_scale"].data_ptr() != at[4])):
                self._describe(k)
            if type(g) is RowGrad:
                if not self._rows(k, self._items[k], p, g, stream, kept):
                    continue
                tables = True
            else:
                if g.shape != shape or g.dtype not in _TYPES or g.device != device or not g.is_contiguous():
                    raise ValueError(f"gradient {k} must be a contiguous tensor of shape {tuple(shape)} on {device}, "
                                     f"got {g.dtype} {tuple(g.shape)} on {g.device}")
                x = self._items[k]
                x.grad = g.data_ptr()
                if self._last[k] is not g.dtype:
                    if not self._whole[k]:
                        raise ValueError(f"the moments of parameter {k} have scales per row: its gradient must be a RowGrad")
                    x.grad_type, x.rows, x.order, x.coef = _TYPES[g.dtype], None, None, None
                    self._last[k] = g.dtype
                if self._empty[k]:
                    continue
            used.append(k)
        for name, t, dtype in (("lr", self.lr if isinstance(self.lr, torch.Tensor) else None, torch.float32),
                               ("grad_scale", grad_scale, torch.float32)):
            if t is not None and (t.dtype != dtype or t.numel() != 1 or t.device != self.device):
                raise ValueError(f"{name} must be one {dtype} number on {self.device}")
        if len(used) == len(self.params):
            ts = self._list
        else:
            ts = (AdamWTensor * max(1, len(used)))(*[self._list[k] for k in used])
        device_lr = isinstance(self.lr, torch.Tensor)
        args = AdamWArgs(0.0 if device_lr else self.lr, self.betas[0], self.betas[1], self.eps, self.steps + 1,
                         _ptr(self.device_steps), self.lr.data_ptr() if device_lr else None, _ptr(grad_scale),
                         0 if self.seed is None else self.seed, 0 if self.seed is None else ADAMW_STOCHASTIC)
        L, n, need = lib(), len(used), 0
        if tables:
            size = ctypes.c_size_t()
            _check(L.smore_adamw_workspace_bytes(ts, n, ctypes.byref(size)))
            need = size.value

        def call(st):
            # a workspace of this call alone, from the stream's (or the capturing graph's) memory
            ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
            if self.device_steps is not None:
                self.device_steps.add_(1)
            rc = L.smore_adamw(ts, n, ctypes.byref(args), _ptr(ws), need, st)
            if rc and self.device_steps is not None:
                self.device_steps.sub_(1)
            return rc

        if stream is not None:
            kept += [grad_scale, self.lr if device_lr else None, self.device_steps]
            names = ("m", "v", "m_scale", "v_scale") if scaled else ("m", "v")
            for k in used:
                kept += [self.params[k], *(self.states[k][n] for n in names)]
                if type(grads[k]) is not RowGrad:
                    kept.append(grads[k])
        _check(_launch(device, stream, call, kept))
        self.steps += 1
        # autograd sees that they changed
        torch.autograd.graph.increment_version([p for p in (self.params[k] for k in used) if not p.is_inference()])

    def _rows(self, k: int, x, p, g: RowGrad, stream, kept: list) -> bool:
        """Puts a RowGrad into the list, and what the call has to keep into
        kept; False if it has no entries (whose address may be NULL, which
        would stand for a dense gradient)."""
        torch = _torch
        if p.dim() != 2 or not self._by_rows[k]:
            raise ValueError(f"parameter {k} is no table with moments per row: its gradient cannot be a RowGrad")
        n = g.rows.numel()
        rows, order, coef = g.rows, g.order, g.coef
        ok = lambda t, dtype, numel: t.dtype == dtype and t.device == self.device and t.numel() == numel and \
            (t.is_contiguous() or not g.in_order)
        of = "contiguous " if g.in_order else ""
        if not ok(rows, torch.int32, n):
            raise ValueError(f"rows of gradient {k} must be a {of}int32 tensor on {self.device}")
        if order is not None and not ok(order, torch.int64, n):
            raise ValueError(f"order of gradient {k} must be a contiguous int64 tensor of {n} entries on {self.device}")
        if coef is not None and not ok(coef, torch.float32, n):
            raise ValueError(f"coef of gradient {k} must be a {of}fp32 tensor of {n} entries on {self.device}")
        if g.per < 1 or g.grad.dim() != 2 or g.grad.shape[1] != p.shape[1] or g.grad.shape[0] * g.per < n or \
                g.grad.dtype not in _TYPES or g.grad.device != self.device or not g.grad.is_contiguous():
            raise ValueError(f"gradient {k} must hold contiguous rows of {p.shape[1]} on {self.device}, one for each "
                             f"{g.per} of {n} entries, got {g.grad.dtype} {tuple(g.grad.shape)} on {g.grad.device}")
        if not g.in_order and order is not None:
            raise ValueError(f"gradient {k} has an order, but its rows are not in order")
        if n == 0:
            return False
        if not g.in_order:
            # copies of what is not contiguous belong on the step's stream: a copy on the
            # current one would come behind what that stream was made to wait for
            flat = lambda: [t if t is None else t.reshape(-1) for t in (rows, coef)]
            if stream is None:
                rows, coef = flat()
            else:
                with torch.cuda.stream(stream):
                    rows, coef = flat()
            rows, order = sort_rows(rows, p.shape[0], stream)
        kept.extend((rows, order, coef, g.rows, g.grad, g.order, g.coef))
        x.grad, x.grad_type, x.rows, x.order, x.coef = g.grad.data_ptr(), _TYPES[g.grad.dtype], rows.data_ptr(), \
            None if order is None else order.data_ptr(), None if coef is None else coef.data_ptr()
        x.n_entries, x.per, self._last[k] = n, g.per, RowGrad
        return True
