"""ctypes binding of libmlip (argument marshalling only; every step runs in the HIP library).

PyTorch supplies device memory (tensors) and the stream; nothing is computed here.
The names mirror include/mlip.h.
"""
from __future__ import annotations

import array
import ctypes
import itertools
import operator
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# MLIP_LIBRARY selects another build of the same library (timing experiments); the default is the in-tree product build
_LIB_PATH = os.environ.get("MLIP_LIBRARY") or os.path.join(_HERE, "libmlip.so")

MODE_WHOLE, MODE_SLABS = 0, 1
PRECISION_FP32, PRECISION_BF16, PRECISION_FP32_SPLIT = 0, 1, 2
PROF_GROUPS = ("graph", "node", "edge_fwd", "edge_bwd", "ghost", "force", "bond", "triplet_fwd", "triplet_bwd",
               "edge_fwd_lower", "edge_bwd_lower")


class MlipError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libmlip error {code}: {msg}")
        self.code = code


class _Weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_species", "F", "L", "K", "p", "precision")] + \
               [(n, ctypes.c_void_p) for n in ("emb", "W1", "W2", "Wm", "Wo", "Wr1", "wr2")]


class _BondWeights(ctypes.Structure):
    _fields_ = [("r_bond", ctypes.c_float), ("A", ctypes.c_int32)] + \
               [(n, ctypes.c_void_p) for n in ("We0", "Wt1", "Wt2", "Wb")]


class _SlabInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("n_owned", "n_pure", "n_border", "n_ghost", "n_local",
                                              "n_edges_owned", "n_edges")] + \
               [(n, ctypes.c_void_p) for n in ("nodes", "markers", "row_ptr", "senders", "owned_sorted")]


_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
_FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class _Pairs(ctypes.Structure):
    _fields_ = [("n_upper", ctypes.c_int64), ("n_lower", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("u_row_ptr", "u_senders", "u_eid", "u_mirror", "u_d",
                                               "l_row_ptr", "l_senders", "l_slot")]


class _Tensor(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class _Alloc(ctypes.Structure):
    _fields_ = [("alloc", _ALLOC_FN), ("free", _FREE_FN), ("ctx", ctypes.c_void_p)]


class TorchAllocator:
    """mlip_alloc_t backed by torch tensors: every device block the library uses is a uint8 tensor from torch's
    caching allocator (so torch's memory accounting sees it).  Keeps the blocks alive until the library frees them."""

    def __init__(self):
        self.blocks = {}
        self.bytes_requested = 0
        self.n_alloc = self.n_free = 0
        self._a = _ALLOC_FN(self._alloc)
        self._f = _FREE_FN(self._free)
        self.c = _Alloc(self._a, self._f, None)

    def _alloc(self, nbytes, _ctx):
        try:
            t = torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device="cuda")
        except Exception:   # out of memory: the library reports MLIP_ENOMEM
            return None
        self.blocks[t.data_ptr()] = t
        self.bytes_requested += int(nbytes)
        self.n_alloc += 1
        return t.data_ptr()

    def _free(self, ptr, _ctx):
        self.n_free += 1
        self.blocks.pop(ptr, None)

    @property
    def bytes_held(self):
        return sum(t.numel() for t in self.blocks.values())


_lib = None


def lib():
    """Load libmlip.so; building it is `python -m paper_2506_02023_amd.build` (or __graft_entry__.build())."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: the HIP library has not been built "
                              "(run __graft_entry__.build()); there is no fallback path")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i64, i32, dbl = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double
        L.mlip_graph_create.argtypes = [ctypes.POINTER(_Alloc), ctypes.POINTER(vp)]
        L.mlip_graph_invalidate_weights.argtypes = [vp]
        L.mlip_graph_set_skin.argtypes = [vp, dbl]
        L.mlip_graph_skin_stats.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.mlip_forward_static.argtypes = [vp, ctypes.POINTER(_Weights), i32, vp, vp, vp]
        L.mlip_static_scratch_bytes.restype = ctypes.c_size_t
        L.mlip_build_graph.argtypes = [vp, ctypes.POINTER(dbl), vp, i64, dbl, i32, vp, ctypes.POINTER(vp)]
        L.mlip_forward.argtypes = [vp, ctypes.POINTER(_Weights), i32, vp, vp, vp]
        L.mlip_forward_bonds.argtypes = [vp, ctypes.POINTER(_Weights), ctypes.POINTER(_BondWeights), i32, vp, vp, vp]
        L.mlip_graph_bonds.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(i64)]
        L.mlip_graph_destroy.argtypes = [vp]
        L.mlip_graph_destroy.restype = None
        L.mlip_graph_sizes.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64), ctypes.POINTER(i32)]
        L.mlip_graph_csr.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp)]
        L.mlip_graph_shifts.argtypes = [vp, vp]
        L.mlip_graph_mirror.argtypes = [vp, ctypes.POINTER(vp)]
        L.mlip_graph_slab_of.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(i32)]
        L.mlip_graph_slab.argtypes = [vp, i32, ctypes.POINTER(_SlabInfo)]
        L.mlip_graph_pairs.argtypes = [vp, i32, ctypes.POINTER(_Pairs)]
        L.mlip_graph_from.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(i64)]
        L.mlip_graph_to.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(i64)]
        L.mlip_profile_enable.argtypes = [vp, i32]
        L.mlip_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i64), i32]
        L.mlip_copy_to_host.argtypes = [vp, vp, vp, ctypes.c_size_t]
        f32, size = ctypes.c_float, ctypes.c_size_t
        L.mlip_embed.argtypes = [vp, i32, i64, i64, i64, i64, vp, i32, i64, f32, vp, i32, i64, vp]
        L.mlip_embed_grad_workspace.argtypes = [i64, i64, i64]
        L.mlip_embed_grad_workspace.restype = size
        L.mlip_embed_grad.argtypes = [vp, i32, i64, i64, vp, i32, i64, i64, i64, f32, i32, vp, i32, i64, vp, size, vp]
        L.mlip_grad_workspace.argtypes = [i32]
        L.mlip_grad_workspace.restype = size
        L.mlip_grad_norm.argtypes = [vp, i32, vp, vp, size, vp]
        L.mlip_clip_grads.argtypes = [vp, i32, f32, vp, vp, size, vp]
        L.mlip_last_error.restype = ctypes.c_char_p
        L.mlip_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise MlipError(rc, lib().mlip_last_error().decode())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # the handle without a Stream object around it (0.1 us, not 3)


def _stream():
    if _raw_stream is not None:
        return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


class Graph:
    """Owner of a mlip_graph_t handle.  By default the handle takes its device memory from torch (TorchAllocator);
    allocator=False leaves allocation to the library (hipMalloc)."""

    def __init__(self, allocator=None):
        self._h = ctypes.c_void_p(None)
        self._weights = (None, None)   # serial numbers of the weights its packed operands belong to
        self.allocator = TorchAllocator() if allocator is None else (allocator or None)
        if self.allocator is not None:
            _check(lib().mlip_graph_create(ctypes.byref(self.allocator.c), ctypes.byref(self._h)))

    def set_skin(self, skin):
        """Verlet skin (same length unit as the positions) for repeated builds on this handle; 0 switches it off."""
        if not self._h.value:
            _check(lib().mlip_graph_create(None, ctypes.byref(self._h)))
        _check(lib().mlip_graph_set_skin(self._h, float(skin)))

    def skin_stats(self):
        """(candidate list rebuilds, reuses) since the handle was made."""
        a, b = ctypes.c_int64(), ctypes.c_int64()
        _check(lib().mlip_graph_skin_stats(self._h, ctypes.byref(a), ctypes.byref(b)))
        return a.value, b.value

    def invalidate_weights(self):
        _check(lib().mlip_graph_invalidate_weights(self._h))

    def __del__(self):
        self.destroy()

    def destroy(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            lib().mlip_graph_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    # -- sizes and host copies of the index structures (for parity checks and inspection)
    def sizes(self):
        n, e, p = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int32()
        _check(lib().mlip_graph_sizes(self._h, ctypes.byref(n), ctypes.byref(e), ctypes.byref(p)))
        return n.value, e.value, p.value

    def _host(self, ptr, count, dtype):
        out = np.empty(count, dtype)
        _check(lib().mlip_copy_to_host(self._h, out.ctypes.data_as(ctypes.c_void_p), ctypes.c_void_p(ptr),
                                       out.nbytes))
        return out

    def csr(self):
        """(row_ptr int64 [N+1], senders int32 [E], shifts int32 [E,3], d float32 [E]) as numpy arrays."""
        N, E, _ = self.sizes()
        rp, sd, dd = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        _check(lib().mlip_graph_csr(self._h, ctypes.byref(rp), ctypes.byref(sd), ctypes.byref(dd)))
        shifts = torch.empty((max(E, 1), 3), dtype=torch.int32, device="cuda")
        _check(lib().mlip_graph_shifts(self._h, ctypes.c_void_p(shifts.data_ptr())))
        torch.cuda.synchronize()
        return (self._host(rp.value, N + 1, np.int64), self._host(sd.value, E, np.int32),
                shifts[:E].cpu().numpy(), self._host(dd.value, E, np.float32))

    def mirror(self):
        """int32 [E]: position of every edge's reverse edge."""
        _, E, _ = self.sizes()
        ptr = ctypes.c_void_p()
        _check(lib().mlip_graph_mirror(self._h, ctypes.byref(ptr)))
        return self._host(ptr.value, E, np.int32)

    def bonds(self, p=-1):
        """(bond_edge int32 [n_bonds], bond_ptr int64 [rows+1]) of the last mlip_forward_bonds: whole graph (p = -1)
        or partition p."""
        rows = self.sizes()[0] if p < 0 else self.slab(p)["n_owned"]
        be, bp, n = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
        _check(lib().mlip_graph_bonds(self._h, p, ctypes.byref(be), ctypes.byref(bp), ctypes.byref(n)))
        return self._host(be.value, n.value, np.int32), self._host(bp.value, rows + 1, np.int64)

    def pairs(self, p=-1):
        """dict with the upper / lower split of the owned rows' edges of partition p (-1: the whole graph)."""
        rows = self.sizes()[0] if p < 0 else self.slab(p)["n_owned"]
        q = _Pairs()
        _check(lib().mlip_graph_pairs(self._h, p, ctypes.byref(q)))
        nu, nl = q.n_upper, q.n_lower
        d = {"n_upper": nu, "n_lower": nl}
        d["u_row_ptr"] = self._host(q.u_row_ptr, rows + 1, np.int64)
        d["l_row_ptr"] = self._host(q.l_row_ptr, rows + 1, np.int64)
        for k in ("u_senders", "u_eid", "u_mirror"):
            d[k] = self._host(getattr(q, k), nu, np.int32)
        d["u_d"] = self._host(q.u_d, nu, np.float32)
        for k in ("l_senders", "l_slot"):
            d[k] = self._host(getattr(q, k), nl, np.int32)
        return d

    def slab_of(self):
        N, _, _ = self.sizes()
        ptr, ax = ctypes.c_void_p(), ctypes.c_int32()
        _check(lib().mlip_graph_slab_of(self._h, ctypes.byref(ptr), ctypes.byref(ax)))
        return self._host(ptr.value, N, np.int32), ax.value

    def slab(self, p):
        """dict with the counts, nodes, markers, local row_ptr/senders and owned_sorted of partition p."""
        _, _, P = self.sizes()
        info = _SlabInfo()
        _check(lib().mlip_graph_slab(self._h, p, ctypes.byref(info)))
        d = {k: getattr(info, k) for k in ("n_owned", "n_pure", "n_border", "n_ghost", "n_local",
                                           "n_edges_owned", "n_edges")}
        d["nodes"] = self._host(info.nodes, d["n_local"], np.int32)
        d["markers"] = np.ctypeslib.as_array(ctypes.cast(info.markers, ctypes.POINTER(ctypes.c_int64)),
                                             shape=(P + 3,)).copy()
        d["row_ptr"] = self._host(info.row_ptr, d["n_local"] + 1, np.int64)
        d["senders"] = self._host(info.senders, d["n_edges"], np.int32)
        d["owned_sorted"] = self._host(info.owned_sorted, d["n_owned"], np.int32)
        return d

    def _bucket(self, fn, p, q):
        ptr, n = ctypes.c_void_p(), ctypes.c_int64()
        _check(fn(self._h, p, q, ctypes.byref(ptr), ctypes.byref(n)))
        return self._host(ptr.value, n.value, np.int32), ptr.value

    def frm(self, p, q):
        return self._bucket(lib().mlip_graph_from, p, q)[0]

    def to(self, p, q):
        return self._bucket(lib().mlip_graph_to, p, q)[0]

    def bucket_address(self, kind, p, q):
        return self._bucket(lib().mlip_graph_from if kind == "from" else lib().mlip_graph_to, p, q)[1]

    # -- profiling
    def profile_enable(self, on=True):
        _check(lib().mlip_profile_enable(self._h, 1 if on else 0))

    def profile_read(self, reset=True):
        ms = (ctypes.c_float * len(PROF_GROUPS))()
        n = (ctypes.c_int64 * len(PROF_GROUPS))()
        _check(lib().mlip_profile_read(self._h, ms, n, 1 if reset else 0))
        return {k: (ms[i], n[i]) for i, k in enumerate(PROF_GROUPS)}


def mlip_build_graph(positions, cell, species, r_cut, n_slabs=1, graph=None):
    """positions: cuda float64 [N,3]; cell: 3x3 host array (rows = lattice vectors); species: cuda int32 [N]."""
    assert positions.is_cuda and positions.dtype == torch.float64 and positions.is_contiguous()
    assert species.is_cuda and species.dtype == torch.int32 and species.is_contiguous()
    assert positions.dim() == 2 and positions.shape[1] == 3 and species.numel() == positions.shape[0]
    cell_h = np.ascontiguousarray(np.asarray(cell, dtype=np.float64).reshape(9))
    g = graph if graph is not None else Graph()
    _check(lib().mlip_build_graph(ctypes.c_void_p(positions.data_ptr()),
                                  cell_h.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                  ctypes.c_void_p(species.data_ptr()), positions.shape[0], float(r_cut),
                                  int(n_slabs), _stream(), ctypes.byref(g._h)))
    return g


_serial = itertools.count()   # one number per Weights / BondWeights object


def _note_weights(graph, weights, bond_weights=None):
    """The library keeps the packed operands of a weight struct and knows it by its addresses, at which the arrays of
    another object may lie once the first one's are freed: drop them when a call comes with another object."""
    last, bond_last = graph._weights
    now = (weights.serial, bond_last if bond_weights is None else bond_weights.serial)
    if (last is not None and last != now[0]) or (bond_last is not None and bond_last != now[1]):
        graph.invalidate_weights()
    graph._weights = now


class Weights:
    """Device copies of the model weights plus the POD struct the library takes."""

    def __init__(self, weights, p, K=8, device="cuda", precision=0):
        """precision: 0 = fp32, 1 = bf16 operands for the filter MLP's F x F products (fp32 accumulation),
        2 = those products as split-fp16 triples (fp32-grade results).  Filters looked up in tables: 1 rounds W2 to
        bf16, 2 is the same as 0."""
        self.t = {k: torch.as_tensor(np.ascontiguousarray(weights[k], np.float32)).to(device).contiguous()
                  for k in ("emb", "W1", "W2", "Wm", "Wo", "Wr1", "wr2")}
        self.serial = next(_serial)
        S, F = self.t["emb"].shape
        L = self.t["W1"].shape[0]
        self.F, self.L = F, L
        self.c = _Weights(S, F, L, K, p, int(precision), *[self.t[k].data_ptr() for k in
                                               ("emb", "W1", "W2", "Wm", "Wo", "Wr1", "wr2")])


class BondWeights:
    """Device copies of the three-body variant's extra weights plus the POD struct the library takes."""

    def __init__(self, weights, r_bond, A=8, device="cuda"):
        self.t = {k: torch.as_tensor(np.ascontiguousarray(weights[k], np.float32)).to(device).contiguous()
                  for k in ("We0", "Wt1", "Wt2", "Wb")}
        self.serial = next(_serial)
        self.c = _BondWeights(float(r_bond), int(A), *[self.t[k].data_ptr() for k in ("We0", "Wt1", "Wt2", "Wb")])


def mlip_forward_bonds(graph, weights, bond_weights, mode=MODE_WHOLE, out=None, want_atom_energy=True):
    """Three-body variant; returns as mlip_forward.  Builds the bond list on first use (one stream synchronisation)."""
    N, _, _ = graph.sizes()
    if out is None:
        energy = torch.empty(1, dtype=torch.float64, device="cuda")
        forces = torch.empty((N, 3), dtype=torch.float32, device="cuda")
        atom_e = torch.empty(N, dtype=torch.float32, device="cuda") if want_atom_energy else None
    else:
        energy, forces, atom_e = out
    _note_weights(graph, weights, bond_weights)
    _check(lib().mlip_forward_bonds(graph._h, ctypes.byref(weights.c), ctypes.byref(bond_weights.c), int(mode),
                                    ctypes.c_void_p(energy.data_ptr()), ctypes.c_void_p(forces.data_ptr()),
                                    ctypes.c_void_p(atom_e.data_ptr() if atom_e is not None else None)))
    return energy, forces, atom_e


def mlip_forward_static(graph, weights, mode=MODE_WHOLE, out=None, want_atom_energy=True):
    """mlip_forward with the library's fixed workspace (no device allocation inside the call); `out` as mlip_forward."""
    return mlip_forward(graph, weights, mode, out, want_atom_energy, _fn="mlip_forward_static")


def mlip_forward(graph, weights, mode=MODE_WHOLE, out=None, want_atom_energy=True, _fn="mlip_forward"):
    """Returns (energy cuda f64 [1], forces cuda f32 [N,3], atom_energy cuda f32 [N] or None); asynchronous."""
    N, _, _ = graph.sizes()
    if out is None:
        energy = torch.empty(1, dtype=torch.float64, device="cuda")
        forces = torch.empty((N, 3), dtype=torch.float32, device="cuda")
        atom_e = torch.empty(N, dtype=torch.float32, device="cuda") if want_atom_energy else None
    else:
        energy, forces, atom_e = out
    _note_weights(graph, weights)
    _check(getattr(lib(), _fn)(graph._h, ctypes.byref(weights.c), int(mode), ctypes.c_void_p(energy.data_ptr()),
                              ctypes.c_void_p(forces.data_ptr()),
                              ctypes.c_void_p(atom_e.data_ptr() if atom_e is not None else None)))
    return energy, forces, atom_e


# ---- per-species parameter tables and gradient clipping (no handle; results on the current stream)

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_ID_BITS = {torch.int32: 32, torch.int64: 64}


def _refuse(msg):
    raise MlipError(-1, msg)


# Tells torch that the library has written tensors, so that autograd notices a value of its own that has changed (increment_version without
# its look at the argument's type, in a third of its time)
_written = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version


def _stream_of(*tensors):
    """The current stream of the current GPU, on which all tensors must lie."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t.get_device() != here:
            _refuse("tensors must be on the current GPU")
    return _raw_stream(here) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _matrix(t, what):
    """(type code, rows, width, row stride, column stride) of a matrix, or of a vector as a matrix of one column."""
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        _refuse(f"{what} must be float32, bfloat16 or float16")
    if t.dim() == 2:
        return dtype, *t.shape, *t.stride()
    if t.dim() != 1:
        _refuse(f"{what} must be a matrix or a vector")
    return dtype, t.shape[0], 1, t.stride(0), 1


def _ids(species):
    """(address, bits, number) of a vector of species."""
    bits = _ID_BITS.get(species.dtype)
    if bits is None or species.dim() != 1 or not species.is_contiguous():
        _refuse("species must be a contiguous int32 or int64 vector")
    return species.data_ptr(), bits, species.shape[0]


def _output(out, rows, width, vector):
    """(type code, row stride) of an output of `rows` rows."""
    dtype, have_rows, have_width, rs, cs = _matrix(out, "out")
    if have_rows != rows or have_width != width or (out.dim() == 1) != vector:
        _refuse(f"out must have {rows} rows of {width} columns, and the dimensions of the input")
    if cs != 1 and width > 1:
        _refuse("the columns of out must lie one after another")
    return dtype, rs if rows > 1 else max(rs, width)


class _Embed(torch.autograd.Function):
    """mlip_embed in an autograd graph.  `out` comes first: where it is a view, torch takes the first input for what is written."""

    @staticmethod
    def forward(ctx, out, table, species, scale):
        ctx.save_for_backward(species)
        ctx.shape, ctx.dtype, ctx.scale = table.shape, table.dtype, scale
        if out is not None:
            ctx.mark_dirty(out)
        return mlip_embed(table, species, scale, out)

    @staticmethod
    def backward(ctx, bar):
        out_bar = torch.zeros_like(bar) if ctx.needs_input_grad[0] else None      # what out held is overwritten
        table_bar = None
        if ctx.needs_input_grad[1]:
            table_bar = mlip_embed_grad(bar, ctx.saved_tensors[0], ctx.shape[0], ctx.scale, bar.new_empty(ctx.shape, dtype=ctx.dtype))
        return out_bar, table_bar, None, None


class _EmbedGrad(torch.autograd.Function):
    """mlip_embed_grad in an autograd graph, `out` first as above"""

    @staticmethod
    def forward(ctx, out, grad, species, n_species, scale, accumulate):
        ctx.save_for_backward(species)
        ctx.shape, ctx.dtype, ctx.n_species, ctx.scale, ctx.accumulate = grad.shape, grad.dtype, n_species, scale, accumulate
        if out is not None:
            ctx.mark_dirty(out)
        return mlip_embed_grad(grad, species, n_species, scale, out, accumulate)

    @staticmethod
    def backward(ctx, bar):
        out_bar = grad_bar = None
        if ctx.needs_input_grad[0]:
            out_bar = bar if ctx.accumulate else torch.zeros_like(bar)
        if ctx.needs_input_grad[1]:
            species, = ctx.saved_tensors
            species = torch.where(species < ctx.n_species, species, -1)     # ids without a row brought nothing in: zeros, not NaN
            grad_bar = mlip_embed(bar, species, ctx.scale, bar.new_empty(ctx.shape, dtype=ctx.dtype))
        return out_bar, grad_bar, None, None, None, None


def mlip_embed(table, species, scale=1.0, out=None):
    """out[i] = scale * table[species[i]]: rows of a per-species table (zeros for a species < 0, NaN for one the table lacks).

    table: cuda [S, F] or [S], float32, bfloat16 or float16, any strides; species: cuda int32 or int64 [n]; out: [n, F] or [n] of any
    of the three types (default: the table's), its columns one after another.  Differentiable with respect to the table."""
    if (table.requires_grad or (out is not None and out.requires_grad)) and torch.is_grad_enabled():
        return _Embed.apply(out, table, species, scale)
    dtype, rows, width, rs, cs = _matrix(table, "table")
    ids, bits, n = _ids(species)
    given = out is not None
    if not given:
        out = table.new_empty((n,) if table.dim() == 1 else (n, width))
    out_dtype, out_rs = _output(out, n, width, table.dim() == 1)
    stream = _stream_of(table, species, out)
    _check(lib().mlip_embed(table.data_ptr(), dtype, rows, width, rs, cs, ids, bits, n, scale, out.data_ptr(), out_dtype, out_rs, stream))
    if given:
        _written((out,))
    return out


def mlip_embed_grad(grad, species, n_species, scale=1.0, out=None, accumulate=False):
    """out[s] = scale * sum of grad[i] over the atoms with species[i] == s: the gradient of mlip_embed for its table.

    grad: cuda [n, F] or [n], any strides (0 for a broadcast gradient); out: [n_species, F] or [n_species] (default: of grad's
    type); accumulate: add to what out holds.  Differentiable with respect to grad and to what is added to."""
    if (grad.requires_grad or (out is not None and out.requires_grad)) and torch.is_grad_enabled():
        return _EmbedGrad.apply(out, grad, species, n_species, scale, accumulate)
    dtype, rows, width, rs, cs = _matrix(grad, "grad")
    ids, bits, n = _ids(species)
    if rows != n:
        _refuse("grad must have a row for each atom")
    given = out is not None
    if not given:
        if accumulate:
            _refuse("accumulate needs out")
        out = grad.new_empty((n_species,) if grad.dim() == 1 else (n_species, width))
    out_dtype, out_rs = _output(out, n_species, width, grad.dim() == 1)
    stream = _stream_of(grad, species, out)
    L = lib()
    need = L.mlip_embed_grad_workspace(n, n_species, width)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    _check(L.mlip_embed_grad(grad.data_ptr(), dtype, rs, cs, ids, bits, n, n_species, width, scale, bool(accumulate), out.data_ptr(),
                             out_dtype, out_rs, ws.data_ptr() if need else None, need, stream))
    if given:
        _written((out,))
    return out


def _dense(t):
    """Whether a tensor's elements fill one piece of memory, in any order of its dimensions."""
    if t.is_contiguous():
        return True
    at = 1
    for stride, size in sorted((s, d) for s, d in zip(t.stride(), t.shape) if d != 1):
        if stride != at:
            return False
        at *= size
    return True


_Tensor_of, _dtype_of = torch.Tensor, operator.attrgetter("dtype")


def _listed(tensors):
    """The tensors of an iterable, which the first of several looks at them may use up, as a list; None as it is."""
    return tensors if tensors is None or type(tensors) is list else list(tensors)


def _tensor_list(grads, out):
    """The tensors as the library takes them (an array of _Tensor, as 64-bit words), checked.  Lists run to hundreds of tensors, so
    each property is taken of all of them in one map."""
    grads, out = _listed(grads), _listed(out)
    codes = list(map(_DTYPES.get, map(_dtype_of, grads)))
    if None in codes:
        _refuse("gradients must be float32, bfloat16 or float16")
    plain = all(map(_Tensor_of.is_contiguous, grads))
    if not plain and not all(map(_dense, grads)):
        _refuse("gradients must be dense")
    dst = src = list(map(_Tensor_of.data_ptr, grads))
    sizes = list(map(_Tensor_of.numel, grads))
    if out is not None:
        same = list(map(_DTYPES.get, map(_dtype_of, out))) == codes and list(map(_Tensor_of.numel, out)) == sizes and \
            (plain and all(map(_Tensor_of.is_contiguous, out)) or all(d.shape == t.shape and d.stride() == t.stride() for d, t in zip(out, grads)))
        if not same:
            _refuse("out must have a tensor for each gradient, of its type, size and layout")
        dst = list(map(_Tensor_of.data_ptr, out))
    if not {torch.cuda.current_device()}.issuperset(map(_Tensor_of.get_device, itertools.chain(grads, out or ()))):
        _refuse("tensors must be on the current GPU")
    words = [0] * (4 * len(src))
    words[::4], words[1::4], words[2::4], words[3::4] = src, dst, sizes, codes
    a = array.array("q", words)
    return a, a.buffer_info()[0], len(src)


def _norm_scratch(count):
    need = lib().mlip_grad_workspace(count)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    return torch.empty((), dtype=torch.float32, device="cuda"), ws, need


def mlip_grad_norm(grads):
    """Norm of all elements of the tensors together (cuda float32 scalar); asynchronous, not recorded by autograd.

    grads: an iterable of dense cuda tensors, float32, bfloat16 or float16, mixed as they come."""
    held, a, count = _tensor_list(grads, None)
    norm, ws, need = _norm_scratch(count)
    _check(lib().mlip_grad_norm(a, count, norm.data_ptr(), ws.data_ptr(), need, _stream()))
    return norm


def mlip_clip_grads(grads, max_norm, out=None):
    """Scales the tensors so that the norm of all of them together is at most max_norm; returns the norm before.

    grads, out: iterables of tensors.  In place, or into the tensors of `out` (of the same types, sizes and layouts).  Where the norm is infinite or NaN the values stay as
    they are: a caller that reads the norm skips the step."""
    grads, out = _listed(grads), _listed(out)
    held, a, count = _tensor_list(grads, out)
    norm, ws, need = _norm_scratch(count)
    _check(lib().mlip_clip_grads(a, count, max_norm, norm.data_ptr(), ws.data_ptr(), need, _stream()))
    _written(grads if out is None else out)
    return norm
