"""Mini-batch GNN hot path on MI355X: Python binding of libgmb.so.

Argument marshalling only: every step runs in the HIP kernels behind the C
ABI declared in include/gmb.h.  PyTorch provides device memory and the
current stream.  There is no CPU fallback: without the built library (or
without a GPU) every call raises.

    csr = CSRGraph(indptr, indices)                 # device tensors
    blocks = sample_blocks(csr, seeds, [15, 10, 5], seed=0)
    x = gather_features(blocks, feats)              # [cap_src0, D]
    logits = sage_forward(blocks, x, weights)       # [B, C] fp32

The three calls follow DistDGL (arXiv 2010.05337) Section II-B (sampling a
mini-batch), Section III-C (pulling its vertex features) and Section II-A
Eq. (1) with the GraphSAGE-mean model of Section IV.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libgmb.so")

GMB_MAX_LAYERS = 8
GMB_F32, GMB_BF16 = 0, 1
MXFP4, MXFP8 = 4, 8   # microscaled formats: the bits of an element
ENOSPC = -2
STATUS = {0: "OK", -1: "EINVAL", -2: "ENOSPC", -3: "EDEVICE", -4: "ERANGE", -5: "EDUP"}
EXPORTS = (
    "gmb_abi_version", "gmb_last_error", "gmb_sampler_state_bytes", "gmb_sampler_state_init",
    "gmb_state_status_word", "gmb_read_status", "gmb_sample_workspace_bytes", "gmb_sample_blocks",
    "gmb_read_sizes", "gmb_gather_features", "gmb_forward_workspace_bytes",
    "gmb_forward_hidden_offset", "gmb_sage_forward", "gmb_sage_forward_fused", "gmb_backward_workspace_bytes",
    "gmb_sage_backward", "gmb_sgd_update", "gmb_backward_embedding_workspace_bytes",
    "gmb_sage_backward_embedding", "gmb_sample_blocks_noalloc",
    "gmb_validate_blocks", "gmb_sgd_update_bf16",
    "gmb_mx_row_bytes", "gmb_mx_quantise", "gmb_mx_gather", "gmb_mx_mean", "gmb_mx_linear",
    "gmb_mx_forward_workspace_bytes", "gmb_mx_forward_offset", "gmb_sage_forward_mx",
    "gmb_distill_workspace_bytes", "gmb_distill_loss", "gmb_sage_backward_distill",
    "gmb_dropout_rows", "gmb_rms_norm", "gmb_rms_norm_workspace_bytes", "gmb_rms_norm_backward",
    "gmb_linear_loss_workspace_bytes", "gmb_linear_loss", "gmb_sage_forward_dropout", "gmb_sage_backward_from",
)


class GmbError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class CsrStruct(ctypes.Structure):
    _fields_ = [("num_nodes", ctypes.c_int64), ("num_edges", ctypes.c_int64),
                ("indptr", ctypes.c_void_p), ("indptr_bits", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("indices", ctypes.c_void_p)]


class BlockStruct(ctypes.Structure):
    _fields_ = [("indptr", ctypes.c_void_p), ("indices", ctypes.c_void_p), ("nbr", ctypes.c_void_p),
                ("src_ids", ctypes.c_void_p), ("sizes", ctypes.c_void_p),
                ("cap_dst", ctypes.c_int64), ("cap_src", ctypes.c_int64), ("cap_nnz", ctypes.c_int64),
                ("fanout", ctypes.c_int32), ("layer", ctypes.c_int32)]


class BlocksStruct(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_seeds", ctypes.c_int32),
                ("blk", BlockStruct * GMB_MAX_LAYERS)]


class WeightsStruct(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("dims", ctypes.c_int32 * (GMB_MAX_LAYERS + 1)),
                ("w_self", ctypes.c_void_p * GMB_MAX_LAYERS),
                ("w_neigh", ctypes.c_void_p * GMB_MAX_LAYERS),
                ("bias", ctypes.c_void_p * GMB_MAX_LAYERS)]


class GradsStruct(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("d_self", ctypes.c_void_p * GMB_MAX_LAYERS),
                ("d_neigh", ctypes.c_void_p * GMB_MAX_LAYERS),
                ("d_bias", ctypes.c_void_p * GMB_MAX_LAYERS)]


class MxOperandStruct(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_void_p), ("num_rows", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("ids", ctypes.c_void_p), ("weights", ctypes.c_void_p), ("weight_stride", ctypes.c_int64)]


class MxWeightsStruct(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32),
                ("dims", ctypes.c_int32 * (GMB_MAX_LAYERS + 1)),
                ("w_self", ctypes.c_void_p * GMB_MAX_LAYERS),
                ("w_neigh", ctypes.c_void_p * GMB_MAX_LAYERS),
                ("bias", ctypes.c_void_p * GMB_MAX_LAYERS)]


class TeacherStruct(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("classes", ctypes.c_void_p), ("top", ctypes.c_int32),
                ("alpha", ctypes.c_float), ("temperature", ctypes.c_float), ("reserved", ctypes.c_int32)]


class RowsStruct(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


class DropoutStruct(ctypes.Structure):
    _fields_ = [("seed", ctypes.c_uint64), ("p", ctypes.c_float), ("layer", ctypes.c_int32), ("step", ctypes.c_void_p)]


class LinearHeadStruct(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64), ("w", ctypes.c_void_p),
                ("w_row_stride", ctypes.c_int64), ("w_col_stride", ctypes.c_int64), ("bias", ctypes.c_void_p),
                ("labels", ctypes.c_void_p), ("rows", ctypes.c_int64), ("d", ctypes.c_int32),
                ("classes", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class LinearGradsStruct(ctypes.Structure):
    _fields_ = [("dx", ctypes.c_void_p), ("dw", ctypes.c_void_p), ("dbias", ctypes.c_void_p),
                ("turned", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded C ABI; raises if libgmb.so has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2010_05337_amd.build` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, u64, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                                 ctypes.c_size_t)
        L.gmb_abi_version.restype = i32
        L.gmb_last_error.restype = ctypes.c_char_p
        L.gmb_sampler_state_bytes.restype = sz
        L.gmb_sampler_state_bytes.argtypes = [i64]
        L.gmb_sampler_state_init.restype = ctypes.c_int
        L.gmb_sampler_state_init.argtypes = [vp, sz, i64, vp]
        L.gmb_state_status_word.restype = vp
        L.gmb_state_status_word.argtypes = [vp]
        L.gmb_read_status.restype = ctypes.c_int
        L.gmb_read_status.argtypes = [vp, vp]
        L.gmb_sample_workspace_bytes.restype = sz
        L.gmb_sample_workspace_bytes.argtypes = [i32, vp, i32, i64]
        L.gmb_sample_blocks.restype = ctypes.c_int
        L.gmb_sample_blocks.argtypes = [ctypes.POINTER(CsrStruct), vp, i32, vp, i32, u64, vp, sz, vp,
                                        sz, ctypes.POINTER(BlocksStruct), vp]
        L.gmb_sample_blocks_noalloc.restype = ctypes.c_int
        L.gmb_sample_blocks_noalloc.argtypes = [ctypes.POINTER(CsrStruct), vp, i32, vp, i32, u64, vp, sz, vp,
                                                sz, ctypes.POINTER(BlocksStruct), vp]
        L.gmb_validate_blocks.restype = ctypes.c_int
        L.gmb_validate_blocks.argtypes = [ctypes.POINTER(CsrStruct), ctypes.POINTER(BlocksStruct), vp, vp]
        L.gmb_read_sizes.restype = ctypes.c_int
        L.gmb_read_sizes.argtypes = [ctypes.POINTER(BlocksStruct), vp, vp]
        L.gmb_gather_features.restype = ctypes.c_int
        L.gmb_gather_features.argtypes = [vp, vp, i64, vp, i64, i32, i32, vp, vp, vp]
        L.gmb_forward_workspace_bytes.restype = sz
        L.gmb_forward_workspace_bytes.argtypes = [ctypes.POINTER(BlocksStruct),
                                                  ctypes.POINTER(WeightsStruct)]
        L.gmb_forward_hidden_offset.restype = i64
        L.gmb_forward_hidden_offset.argtypes = [ctypes.POINTER(BlocksStruct),
                                                ctypes.POINTER(WeightsStruct), i32]
        L.gmb_sage_forward.restype = ctypes.c_int
        L.gmb_sage_forward.argtypes = [ctypes.POINTER(BlocksStruct), vp, ctypes.POINTER(WeightsStruct),
                                       vp, vp, sz, vp]
        L.gmb_sage_forward_fused.restype = ctypes.c_int
        L.gmb_sage_forward_fused.argtypes = [ctypes.POINTER(BlocksStruct), vp, ctypes.c_int64, vp,
                                             ctypes.POINTER(WeightsStruct), vp, vp, sz, vp, vp]
        L.gmb_backward_workspace_bytes.restype = sz
        L.gmb_backward_workspace_bytes.argtypes = [ctypes.POINTER(BlocksStruct),
                                                   ctypes.POINTER(WeightsStruct)]
        L.gmb_sage_backward.restype = ctypes.c_int
        L.gmb_sage_backward.argtypes = [ctypes.POINTER(BlocksStruct), vp, ctypes.POINTER(WeightsStruct), vp, vp,
                                        vp, sz, ctypes.POINTER(GradsStruct), vp, vp, sz, vp]
        L.gmb_backward_embedding_workspace_bytes.restype = sz
        L.gmb_backward_embedding_workspace_bytes.argtypes = [ctypes.POINTER(BlocksStruct),
                                                             ctypes.POINTER(WeightsStruct)]
        L.gmb_sage_backward_embedding.restype = ctypes.c_int
        L.gmb_sage_backward_embedding.argtypes = [ctypes.POINTER(BlocksStruct), vp, ctypes.POINTER(WeightsStruct),
                                                  vp, vp, vp, sz, ctypes.POINTER(GradsStruct), vp, vp, sz, vp,
                                                  ctypes.c_int64, ctypes.c_float, vp]
        L.gmb_sgd_update_bf16.restype = ctypes.c_int
        L.gmb_sgd_update_bf16.argtypes = [ctypes.POINTER(WeightsStruct), ctypes.POINTER(WeightsStruct),
                                          ctypes.POINTER(GradsStruct), ctypes.c_float, vp]
        L.gmb_sgd_update.restype = ctypes.c_int
        L.gmb_sgd_update.argtypes = [ctypes.POINTER(WeightsStruct), ctypes.POINTER(GradsStruct),
                                     ctypes.c_float, vp]
        f32 = ctypes.c_float
        L.gmb_mx_row_bytes.restype = i64
        L.gmb_mx_row_bytes.argtypes = [i32, i32]
        L.gmb_mx_quantise.restype = ctypes.c_int
        L.gmb_mx_quantise.argtypes = [vp, i32, i64, i64, vp, vp, i64, i32, i32, vp, i64, i64, vp, sz, vp, vp]
        L.gmb_mx_gather.restype = ctypes.c_int
        L.gmb_mx_gather.argtypes = [vp, vp, i64, vp, i64, i64, i32, i32, vp, i32, vp, vp]
        L.gmb_mx_mean.restype = ctypes.c_int
        L.gmb_mx_mean.argtypes = [vp, vp, vp, i64, vp, i64, i64, i32, i32, vp, i32, vp]
        L.gmb_mx_linear.restype = ctypes.c_int
        L.gmb_mx_linear.argtypes = [ctypes.POINTER(MxOperandStruct), ctypes.POINTER(MxOperandStruct), vp, i64, i32,
                                    i32, vp, i32, vp, i32, vp, vp]
        L.gmb_mx_forward_workspace_bytes.restype = sz
        L.gmb_mx_forward_workspace_bytes.argtypes = [ctypes.POINTER(BlocksStruct), ctypes.POINTER(MxWeightsStruct)]
        L.gmb_mx_forward_offset.restype = i64
        L.gmb_mx_forward_offset.argtypes = [ctypes.POINTER(BlocksStruct), ctypes.POINTER(MxWeightsStruct), i32, i32]
        L.gmb_sage_forward_mx.restype = ctypes.c_int
        L.gmb_sage_forward_mx.argtypes = [ctypes.POINTER(BlocksStruct), vp, i64, i64, ctypes.POINTER(MxWeightsStruct),
                                          vp, vp, sz, vp, vp]
        L.gmb_distill_workspace_bytes.restype = sz
        L.gmb_distill_workspace_bytes.argtypes = [i64, i32]
        L.gmb_distill_loss.restype = ctypes.c_int
        L.gmb_distill_loss.argtypes = [vp, i32, i64, i32, ctypes.POINTER(TeacherStruct), vp, vp, vp, vp, sz, vp]
        L.gmb_sage_backward_distill.restype = ctypes.c_int
        L.gmb_sage_backward_distill.argtypes = [ctypes.POINTER(BlocksStruct), vp, ctypes.POINTER(WeightsStruct), vp,
                                                ctypes.POINTER(TeacherStruct), vp, vp, sz,
                                                ctypes.POINTER(GradsStruct), vp, vp, sz, vp, i64, f32, vp]
        rows, drop = ctypes.POINTER(RowsStruct), ctypes.POINTER(DropoutStruct)
        L.gmb_dropout_rows.restype = ctypes.c_int
        L.gmb_dropout_rows.argtypes = [rows, rows, drop, vp, vp, i64, i32, i32, rows, vp]
        L.gmb_rms_norm.restype = ctypes.c_int
        L.gmb_rms_norm.argtypes = [rows, rows, drop, vp, vp, i64, i32, i32, vp, f32, rows, i32, rows, vp]
        L.gmb_rms_norm_workspace_bytes.restype = sz
        L.gmb_rms_norm_workspace_bytes.argtypes = [i64, i32]
        L.gmb_rms_norm_backward.restype = ctypes.c_int
        L.gmb_rms_norm_backward.argtypes = [rows, rows, rows, drop, vp, vp, i64, i32, i32, vp, f32, rows, rows, vp, vp,
                                            sz, vp]
        head, grads = ctypes.POINTER(LinearHeadStruct), ctypes.POINTER(LinearGradsStruct)
        L.gmb_linear_loss_workspace_bytes.restype = sz
        L.gmb_linear_loss_workspace_bytes.argtypes = [head, grads]
        L.gmb_linear_loss.restype = ctypes.c_int
        L.gmb_linear_loss.argtypes = [head, grads, vp, vp, sz, vp]
        L.gmb_sage_forward_dropout.restype = ctypes.c_int
        L.gmb_sage_forward_dropout.argtypes = [ctypes.POINTER(BlocksStruct), vp, vp, i64,
                                               ctypes.POINTER(WeightsStruct), drop, vp, vp, sz, vp, vp]
        L.gmb_sage_backward_from.restype = ctypes.c_int
        L.gmb_sage_backward_from.argtypes = [ctypes.POINTER(BlocksStruct), vp, ctypes.POINTER(WeightsStruct), vp, drop,
                                             vp, sz, ctypes.POINTER(GradsStruct), vp, sz, vp, i64, f32, vp]
        _lib = L
    return _lib


def _check(code: int):
    if code != 0:
        raise GmbError(code, lib().gmb_last_error().decode(errors="replace"))


def _stream_handle() -> int:
    """The current stream's handle (0.3 us; through a torch.cuda.Stream object
    it is 2.9 us, three times per mini-batch)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _require_cuda(t: torch.Tensor, name: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _aligned_bytes(nbytes: int, device) -> tuple:
    """A uint8 device buffer with a 256-byte aligned view of nbytes."""
    buf = torch.empty(max(nbytes, 1) + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf, buf[off:off + max(nbytes, 1)]


class CSRGraph:
    """In-neighbour CSR on the device (row v lists the sources of the edges
    into v), plus the sampler state (a per-vertex dedup table) that
    sample_blocks needs."""

    def __init__(self, indptr: torch.Tensor, indices: torch.Tensor):
        _require_cuda(indptr, "indptr")
        _require_cuda(indices, "indices")
        if indptr.dtype not in (torch.int32, torch.int64):
            raise TypeError("indptr must be int32 or int64")
        if indices.dtype != torch.int32:
            raise TypeError("indices must be int32")
        self.indptr, self.indices = indptr, indices
        self.num_nodes = indptr.numel() - 1
        self.num_edges = indices.numel()
        self.struct = CsrStruct(self.num_nodes, self.num_edges, indptr.data_ptr(),
                                32 if indptr.dtype == torch.int32 else 64, 0,
                                indices.data_ptr() if self.num_edges else None)
        nbytes = lib().gmb_sampler_state_bytes(self.num_nodes)
        if nbytes == 0:
            raise GmbError(-1, f"num_nodes={self.num_nodes} unsupported")
        self._state_buf, self.state = _aligned_bytes(nbytes, indptr.device)
        self.state_bytes = nbytes
        _check(lib().gmb_sampler_state_init(ctypes.c_void_p(self.state.data_ptr()), nbytes,
                                            self.num_nodes, _stream_handle()))

    @property
    def status_word(self) -> int:
        return lib().gmb_state_status_word(ctypes.c_void_p(self.state.data_ptr()))

    def check_status(self):
        """Synchronises, then raises GmbError for a data error found on the device."""
        _check(lib().gmb_read_status(ctypes.c_void_p(self.state.data_ptr()), _stream_handle()))


class Block:
    """Host view of one block after the sizes were read (tensors are views
    into the workspace, cut to the device-side sizes)."""

    def __init__(self, n_dst, n_src, nnz, indptr, indices, nbr, src_ids, fanout, layer):
        self.n_dst, self.n_src, self.nnz = n_dst, n_src, nnz
        self.indptr, self.indices, self.nbr, self.src_ids = indptr, indices, nbr, src_ids
        self.fanout, self.layer = fanout, layer


class Blocks:
    """The L blocks of one mini-batch (index 0 = input layer).  Sizes stay on
    the device until sizes() is called."""

    def __init__(self, struct: BlocksStruct, workspace: torch.Tensor, csr: CSRGraph):
        self.struct = struct
        self.workspace = workspace
        self.csr = csr
        self.num_layers = struct.num_layers
        self.num_seeds = struct.num_seeds

    def _view(self, ptr: int, n: int) -> torch.Tensor:
        off = ptr - self.workspace.data_ptr()
        return self.workspace[off:off + 4 * n].view(torch.int32)

    @property
    def input_ids(self) -> torch.Tensor:
        """Block 0's source ids at full capacity (valid prefix: n_src of block 0)."""
        b = self.struct.blk[0]
        return self._view(b.src_ids, b.cap_src)

    @property
    def input_count_ptr(self) -> int:
        """Device address of block 0's n_src word."""
        return self.struct.blk[0].sizes + 4 * 1

    @property
    def input_capacity(self) -> int:
        return int(self.struct.blk[0].cap_src)

    def sizes(self):
        """[(n_dst, n_src, nnz)] per layer (synchronises the stream)."""
        out = (ctypes.c_int64 * (3 * self.num_layers))()
        _check(lib().gmb_read_sizes(ctypes.byref(self.struct), out, _stream_handle()))
        return [tuple(int(out[3 * l + i]) for i in range(3)) for l in range(self.num_layers)]

    def validate(self):
        """Enqueues the device consistency check of the blocks; a violation
        shows in the next csr.check_status() (GmbError EDEVICE)."""
        _check(lib().gmb_validate_blocks(ctypes.byref(self.csr.struct), ctypes.byref(self.struct),
                                         ctypes.c_void_p(self.csr.state.data_ptr()), _stream_handle()))

    def blocks(self):
        """Per-layer Block views cut to the device sizes (synchronises)."""
        res = []
        for l, (n_dst, n_src, nnz) in enumerate(self.sizes()):
            b = self.struct.blk[l]
            res.append(Block(n_dst, n_src, nnz, self._view(b.indptr, n_dst + 1),
                             self._view(b.indices, nnz), self._view(b.nbr, nnz),
                             self._view(b.src_ids, n_src), int(b.fanout), int(b.layer)))
        return res


def sample_workspace_bytes(num_seeds: int, fanouts, num_nodes: int) -> int:
    fo = (ctypes.c_int32 * len(fanouts))(*fanouts)
    return lib().gmb_sample_workspace_bytes(num_seeds, fo, len(fanouts), num_nodes)


def sample_blocks(csr: CSRGraph, seeds: torch.Tensor, fanouts, seed: int,
                  workspace: torch.Tensor | None = None) -> Blocks:
    """Samples an L-layer mini-batch from `seeds` (device int32, distinct);
    fanouts[l] belongs to model layer l (l = 0 is the input layer)."""
    _require_cuda(seeds, "seeds")
    if seeds.dtype != torch.int32:
        raise TypeError("seeds must be int32")
    fanouts = [int(f) for f in fanouts]
    layers, num_seeds = len(fanouts), seeds.numel()
    fo = (ctypes.c_int32 * layers)(*fanouts)
    L, out, stream = lib(), BlocksStruct(), _stream_handle()

    def call(ws):
        return L.gmb_sample_blocks(ctypes.byref(csr.struct), seeds.data_ptr() if num_seeds else None, num_seeds, fo,
                                   layers, seed & 0xFFFFFFFFFFFFFFFF, csr.state.data_ptr(), csr.state_bytes,
                                   ws.data_ptr(), ws.numel(), ctypes.byref(out), stream)

    # a workspace that is too small is refused before anything is enqueued
    code = ENOSPC if workspace is None or workspace.numel() == 0 or workspace.data_ptr() % 256 else call(workspace)
    if code == ENOSPC:
        need = L.gmb_sample_workspace_bytes(num_seeds, fo, layers, csr.num_nodes)
        if need == 0:
            _check(-1)
        if workspace is None or workspace.numel() < need or workspace.data_ptr() % 256:
            _, workspace = _aligned_bytes(need, seeds.device)
        code = call(workspace)
    _check(code)
    return Blocks(out, workspace, csr)


def gather_features(ids, feats: torch.Tensor, n: int | None = None,
                    out: torch.Tensor | None = None, status_word: int | None = None) -> torch.Tensor:
    """out[i] = feats[ids[i]] bit for bit.  `ids` is a Blocks (its input
    vertices; the count stays on the device and the result has the blocks'
    input capacity in rows) or a device int32 tensor (all of it, or the
    first n)."""
    _require_cuda(feats, "feats")
    if feats.dim() != 2:
        raise ValueError("feats must be [num_nodes, dim]")
    if feats.dtype == torch.float32:
        dtype = GMB_F32
    elif feats.dtype in (torch.bfloat16, torch.int16, torch.uint16):
        dtype = GMB_BF16
    else:
        raise TypeError("feats must be float32 or bfloat16")
    n_dev = None
    if isinstance(ids, Blocks):
        cap = ids.input_capacity
        n_dev = ids.input_count_ptr
        if status_word is None:
            status_word = ids.csr.status_word
        ids_ptr = ids.struct.blk[0].src_ids
    else:
        _require_cuda(ids, "ids")
        if ids.dtype != torch.int32:
            raise TypeError("ids must be int32")
        ids_ptr = ids.data_ptr()
        cap = ids.numel() if n is None else int(n)
        if cap > ids.numel():
            raise ValueError("n exceeds ids")
    if out is None:
        out = torch.empty((cap, feats.shape[1]), dtype=feats.dtype, device=feats.device)
    elif out.shape[0] < cap or out.shape[1] != feats.shape[1] or out.dtype != feats.dtype:
        raise ValueError("out has the wrong shape or dtype")
    _check(lib().gmb_gather_features(ids_ptr if cap else None, n_dev, cap, feats.data_ptr(), feats.shape[0],
                                     feats.shape[1], dtype, out.data_ptr() if cap else None, status_word or None,
                                     _stream_handle()))
    return out


class SageWeights:
    """GraphSAGE-mean weights on the device: W_self[l], W_neigh[l]
    [dims[l], dims[l+1]] (float32 or bfloat16) and bias[l] float32."""

    def __init__(self, w_self, w_neigh, bias):
        if not (len(w_self) == len(w_neigh) == len(bias)) or not w_self:
            raise ValueError("one W_self, W_neigh and bias per layer")
        if len(w_self) > GMB_MAX_LAYERS:
            raise ValueError("too many layers")
        self.w_self = [w.contiguous() for w in w_self]
        self.w_neigh = [w.contiguous() for w in w_neigh]
        self.bias = [b.contiguous().float() for b in bias]
        dt = self.w_self[0].dtype
        self.dtype = GMB_BF16 if dt == torch.bfloat16 else GMB_F32
        if dt not in (torch.float32, torch.bfloat16):
            raise TypeError("weights must be float32 or bfloat16")
        dims = [self.w_self[0].shape[0]] + [w.shape[1] for w in self.w_self]
        for l, (a, b) in enumerate(zip(self.w_self, self.w_neigh)):
            if a.shape != b.shape or a.shape != (dims[l], dims[l + 1]) or a.dtype != dt or b.dtype != dt:
                raise ValueError(f"layer {l}: W_self/W_neigh shapes or dtypes disagree")
            _require_cuda(a, "w_self")
            _require_cuda(b, "w_neigh")
            _require_cuda(self.bias[l], "bias")
        self.dims = dims
        s = WeightsStruct()
        s.num_layers = len(self.w_self)
        s.dtype = self.dtype
        for i, d in enumerate(dims):
            s.dims[i] = d
        for l in range(len(self.w_self)):
            s.w_self[l] = self.w_self[l].data_ptr()
            s.w_neigh[l] = self.w_neigh[l].data_ptr()
            s.bias[l] = self.bias[l].data_ptr()
        self.struct = s

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == GMB_BF16 else torch.float32

    def master(self) -> "SageWeights":
        """fp32 copies of the matrices (the biases are shared): the master
        weights that sgd_update_bf16 updates for a bf16 model."""
        return SageWeights([w.float() for w in self.w_self], [w.float() for w in self.w_neigh], self.bias)


def forward_workspace_bytes(blocks: Blocks, weights: SageWeights) -> int:
    return lib().gmb_forward_workspace_bytes(ctypes.byref(blocks.struct), ctypes.byref(weights.struct))


def _with_forward_workspace(call, blocks: Blocks, weights: SageWeights, workspace, device, drop):
    """call(workspace), or, where none is given or the call refuses it as too
    small (before anything is enqueued), call on one allocated here; returns
    (status, the workspace used).  The workspace keeps what the forward dropped
    out with, for _check_dropped."""
    code = ENOSPC
    if workspace is not None and workspace.numel() > 0 and workspace.data_ptr() % 256 == 0:
        code = call(workspace)
    if code == ENOSPC:
        need = forward_workspace_bytes(blocks, weights)
        if need == 0:
            _check(-1)
        _, workspace = _aligned_bytes(need, device)
        code = call(workspace)
    if code == 0:
        workspace.dropped = _dropped(drop)
    return code, workspace


def _dropped(drop) -> int:
    """What of 65536 elements a dropout (or None) drops, as the kernels round it."""
    return 0 if drop is None else int(65536.0 * drop.p + 0.5)


def _check_dropped(blocks: Blocks, fwd_workspace: torch.Tensor, drop):
    """A backward takes the probability that the forward dropped out with: without
    it the layers below a dropout would lack its factor.  (Known where the tensor
    is the one that the last forward was given; a copy or another view of its
    memory does not say.)"""
    want = _dropped(drop)
    had = getattr(fwd_workspace, "dropped", want)
    if had != want and blocks.num_layers > 1:
        raise ValueError(f"fwd_workspace is of a forward with dropout p={had / 65536:g}, the backward is asked for with"
                         f" p={want / 65536:g} (sage_backward_from takes the forward's dropout)")


def sage_forward(blocks: Blocks, feats: torch.Tensor, weights: SageWeights,
                 workspace: torch.Tensor | None = None, logits: torch.Tensor | None = None,
                 return_hidden: bool = False, dropout: "Dropout | None" = None):
    """GraphSAGE-mean forward over the blocks; feats holds the gathered input
    rows of block 0's sources.  Returns logits [num_seeds, C] float32 (and,
    with return_hidden, the hidden activations cut to their row counts).
    `dropout` drops out the hidden activations, layer l's with layer
    dropout.layer + l, keyed by vertex (train with sage_backward_from)."""
    _require_cuda(feats, "feats")
    if feats.dtype != weights.torch_dtype:
        raise TypeError("feats and weights must have the same dtype")
    if feats.dim() != 2 or feats.shape[1] != weights.dims[0] or feats.shape[0] < blocks.input_capacity:
        raise ValueError("feats must be [input capacity, dims[0]]")
    B, C = blocks.num_seeds, weights.dims[-1]
    if logits is None:
        logits = torch.empty((max(B, 0), C), dtype=torch.float32, device=feats.device)
    L, stream = lib(), _stream_handle()
    drop = None if dropout is None else _drop_struct(dropout, feats.get_device())

    def call(ws):
        if drop is not None:
            return L.gmb_sage_forward_dropout(ctypes.byref(blocks.struct), feats.data_ptr(), None, 0,
                                              ctypes.byref(weights.struct), drop, logits.data_ptr(),
                                              ws.data_ptr(), ws.numel(), None, stream)
        return L.gmb_sage_forward(ctypes.byref(blocks.struct), feats.data_ptr(), ctypes.byref(weights.struct),
                                  logits.data_ptr(), ws.data_ptr(), ws.numel(), stream)

    code, workspace = _with_forward_workspace(call, blocks, weights, workspace, feats.device, drop)
    _check(code)
    if not return_hidden:
        return logits
    return logits, _hidden_views(blocks, weights, workspace)


def _hidden_views(blocks: Blocks, weights: SageWeights, workspace: torch.Tensor):
    hidden = []
    sizes = blocks.sizes()
    es = 2 if weights.dtype == GMB_BF16 else 4
    for l in range(blocks.num_layers - 1):
        off = lib().gmb_forward_hidden_offset(ctypes.byref(blocks.struct), ctypes.byref(weights.struct), l)
        n = sizes[l][0]
        d = weights.dims[l + 1]
        h = workspace[off:off + n * d * es].view(weights.torch_dtype).view(n, d)
        hidden.append(h)
    return hidden


def dst_capacity(blocks: Blocks) -> int:
    """Rows of block 0's destinations (the x_dst buffer of the fused forward)."""
    return int(blocks.struct.blk[0].cap_dst)


def sage_forward_fused(blocks: Blocks, feats: torch.Tensor, weights: SageWeights,
                       x_dst: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                       logits: torch.Tensor | None = None, return_hidden: bool = False,
                       dropout: "Dropout | None" = None):
    """The forward with the feature pull folded into layer 0: `feats` is the
    whole feature table [num_nodes, dims[0]]; block 0's destination rows are
    gathered into x_dst ([dst capacity, dims[0]]), the layer-0 mean reads
    the table directly.  Returns (logits, x_dst) (and the hidden
    activations with return_hidden); x_dst serves as `x` of sage_backward.
    `dropout` as in sage_forward."""
    _require_cuda(feats, "feats")
    if feats.dtype != weights.torch_dtype:
        raise TypeError("feats and weights must have the same dtype")
    if feats.dim() != 2 or feats.shape[1] != weights.dims[0]:
        raise ValueError("feats must be [num_nodes, dims[0]]")
    if x_dst is None:
        x_dst = torch.empty((dst_capacity(blocks), weights.dims[0]), dtype=feats.dtype, device=feats.device)
    if x_dst.dtype != feats.dtype or x_dst.dim() != 2 or x_dst.shape[1] != weights.dims[0] or \
            x_dst.shape[0] < dst_capacity(blocks) or not x_dst.is_contiguous():
        raise ValueError("x_dst must be a contiguous [dst capacity, dims[0]] tensor of the features' dtype")
    B, C = blocks.num_seeds, weights.dims[-1]
    if logits is None:
        logits = torch.empty((max(B, 0), C), dtype=torch.float32, device=feats.device)
    L, stream, status = lib(), _stream_handle(), blocks.csr.status_word
    drop = None if dropout is None else _drop_struct(dropout, feats.get_device())

    def call(ws):
        if drop is not None:
            return L.gmb_sage_forward_dropout(ctypes.byref(blocks.struct), x_dst.data_ptr(), feats.data_ptr(),
                                              feats.shape[0], ctypes.byref(weights.struct), drop,
                                              logits.data_ptr(), ws.data_ptr(), ws.numel(), status, stream)
        return L.gmb_sage_forward_fused(ctypes.byref(blocks.struct), feats.data_ptr(), feats.shape[0],
                                        x_dst.data_ptr(), ctypes.byref(weights.struct), logits.data_ptr(),
                                        ws.data_ptr(), ws.numel(), status, stream)

    code, workspace = _with_forward_workspace(call, blocks, weights, workspace, feats.device, drop)
    _check(code)
    if not return_hidden:
        return logits, x_dst
    return logits, x_dst, _hidden_views(blocks, weights, workspace)


# ---------------------------------------------------------------- training

class SageGrads:
    """fp32 gradient arrays laid out like the weights (device tensors)."""

    def __init__(self, weights: SageWeights):
        dev = weights.w_self[0].device
        self.d_self = [torch.zeros(w.shape, dtype=torch.float32, device=dev) for w in weights.w_self]
        self.d_neigh = [torch.zeros(w.shape, dtype=torch.float32, device=dev) for w in weights.w_neigh]
        self.d_bias = [torch.zeros(b.shape, dtype=torch.float32, device=dev) for b in weights.bias]
        g = GradsStruct()
        g.num_layers = len(self.d_self)
        for l in range(g.num_layers):
            g.d_self[l] = self.d_self[l].data_ptr()
            g.d_neigh[l] = self.d_neigh[l].data_ptr()
            g.d_bias[l] = self.d_bias[l].data_ptr()
        self.struct = g


def backward_workspace_bytes(blocks: Blocks, weights: SageWeights) -> int:
    return lib().gmb_backward_workspace_bytes(ctypes.byref(blocks.struct), ctypes.byref(weights.struct))


def backward_embedding_workspace_bytes(blocks: Blocks, weights: SageWeights) -> int:
    return lib().gmb_backward_embedding_workspace_bytes(ctypes.byref(blocks.struct), ctypes.byref(weights.struct))


def sage_backward(blocks: Blocks, feats: torch.Tensor, weights: SageWeights, logits: torch.Tensor,
                  labels: torch.Tensor, fwd_workspace: torch.Tensor, grads: SageGrads | None = None,
                  loss: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                  embedding: torch.Tensor | None = None, emb_lr: float = 0.0, teacher: "Teacher | None" = None):
    """Gradients of the mean softmax cross-entropy of `logits` (from the
    sage_forward call that used `fwd_workspace`) against `labels` (device
    int32, one per seed), or, with `teacher`, of the loss of distill_loss
    (labels may be None then).  Returns (grads, loss) with loss a 1-element
    float32 device tensor.  With `embedding` (the fp32 [num_nodes, dims[0]]
    table the layer-0 inputs were taken from) the gradient in the input
    rows is applied to the table as an SGD step of size emb_lr.  A NaN loss
    may also mean that a bounded wait on the device ran out (gmb.h).  A forward
    with dropout is refused: its backward is sage_backward_from, which takes the
    dropout (distill_loss gives the gradient at the outputs)."""
    _check_dropped(blocks, fwd_workspace, None)
    if labels is not None or teacher is None:
        _require_cuda(labels, "labels")
        if labels.dtype != torch.int32 or labels.numel() < blocks.num_seeds:
            raise TypeError("labels must be int32 with one entry per seed")
    if teacher is not None:
        _current_device(teacher.logits, "teacher")
        if teacher.rows < blocks.num_seeds:
            raise ValueError("teacher must have one row per seed")
    if embedding is not None:
        _require_cuda(embedding, "embedding")
        if embedding.dtype != torch.float32 or embedding.dim() != 2 or embedding.shape[1] != weights.dims[0] \
                or not embedding.is_contiguous():
            raise ValueError("embedding must be a contiguous float32 [num_nodes, dims[0]] tensor")
        need = backward_embedding_workspace_bytes(blocks, weights)
    else:
        need = backward_workspace_bytes(blocks, weights)
    if need == 0:
        _check(-1)
    if workspace is None or workspace.numel() < need or workspace.data_ptr() % 256:
        _, workspace = _aligned_bytes(need, feats.device)
    if grads is None:
        grads = SageGrads(weights)
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=feats.device)
    common = (ctypes.byref(blocks.struct), ctypes.c_void_p(feats.data_ptr()), ctypes.byref(weights.struct),
              ctypes.c_void_p(logits.data_ptr()),
              None if labels is None else ctypes.c_void_p(labels.data_ptr()),
              ctypes.c_void_p(fwd_workspace.data_ptr()), fwd_workspace.numel(), ctypes.byref(grads.struct),
              ctypes.c_void_p(loss.data_ptr()), ctypes.c_void_p(workspace.data_ptr()), workspace.numel())
    if teacher is not None:
        table = (None, 0, 0.0) if embedding is None else (embedding.data_ptr(), embedding.shape[0], float(emb_lr))
        _check(lib().gmb_sage_backward_distill(*common[:4], ctypes.byref(teacher.struct), *common[4:], *table,
                                               _stream_handle()))
    elif embedding is None:
        _check(lib().gmb_sage_backward(*common, _stream_handle()))
    else:
        _check(lib().gmb_sage_backward_embedding(*common, ctypes.c_void_p(embedding.data_ptr()),
                                                 embedding.shape[0], float(emb_lr), _stream_handle()))
    return grads, loss


def sage_backward_from(blocks: Blocks, feats: torch.Tensor, weights: SageWeights, d_logits: torch.Tensor,
                       fwd_workspace: torch.Tensor, grads: SageGrads | None = None,
                       workspace: torch.Tensor | None = None, embedding: torch.Tensor | None = None,
                       emb_lr: float = 0.0, dropout: "Dropout | None" = None) -> SageGrads:
    """The backward of sage_forward (or its fused form) from the gradient at
    the model's outputs, float32 [num_seeds, C]: of a loss of your own or of
    layers behind the model.  `dropout` is the forward's (another probability
    than the forward's is refused); the others are sage_backward's."""
    dev = _current_device(d_logits, "d_logits")
    if d_logits.dtype is not torch.float32 or d_logits.dim() != 2 or not d_logits.is_contiguous() \
            or d_logits.shape[0] < blocks.num_seeds or d_logits.shape[1] != weights.dims[-1]:
        raise ValueError("d_logits must be a contiguous float32 [num_seeds, C] tensor")
    _same_device(feats, dev, "feats")
    table = (None, 0, 0.0)
    if embedding is not None:
        _same_device(embedding, dev, "embedding")
        if embedding.dtype != torch.float32 or embedding.dim() != 2 or embedding.shape[1] != weights.dims[0] \
                or not embedding.is_contiguous():
            raise ValueError("embedding must be a contiguous float32 [num_nodes, dims[0]] tensor")
        need = backward_embedding_workspace_bytes(blocks, weights)
        table = (embedding.data_ptr(), embedding.shape[0], float(emb_lr))
    else:
        need = backward_workspace_bytes(blocks, weights)
    if need == 0:
        _check(-1)
    drop = None if dropout is None else _drop_struct(dropout, dev)
    _check_dropped(blocks, fwd_workspace, drop)
    if workspace is None or workspace.numel() < need or workspace.data_ptr() % 256:
        _, workspace = _aligned_bytes(need, feats.device)
    if grads is None:
        grads = SageGrads(weights)
    _check(lib().gmb_sage_backward_from(ctypes.byref(blocks.struct), feats.data_ptr(), ctypes.byref(weights.struct),
                                        d_logits.data_ptr() or feats.data_ptr(), drop, fwd_workspace.data_ptr(),
                                        fwd_workspace.numel(), ctypes.byref(grads.struct), workspace.data_ptr(),
                                        workspace.numel(), *table, _stream_handle()))
    return grads


def sgd_update(weights: SageWeights, grads: SageGrads, lr: float):
    """W -= lr * dW and b -= lr * db in place (fp32 weights)."""
    _check(lib().gmb_sgd_update(ctypes.byref(weights.struct), ctypes.byref(grads.struct), float(lr),
                                _stream_handle()))


def sgd_update_bf16(weights: SageWeights, master: SageWeights, grads: SageGrads, lr: float):
    """One SGD step of a bf16 model: the fp32 master weights W -= lr * dW,
    then the bf16 matrices become the new masters rounded to nearest even
    (the biases, fp32 in both, are updated in the master and copied)."""
    _check(lib().gmb_sgd_update_bf16(ctypes.byref(weights.struct), ctypes.byref(master.struct),
                                     ctypes.byref(grads.struct), float(lr), _stream_handle()))


# ---------------------------------------------------------------- microscaled store and model

_DTYPES = {torch.float32: GMB_F32, torch.bfloat16: GMB_BF16}


def _current_device(t, name: str) -> int:
    """The device of the tensor `t`, which has to be the current one (the
    kernels run on its current stream)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    dev, now = t.get_device(), torch._C._cuda_getDevice()
    if dev != now:
        raise ValueError(f"{name} is on device {dev}, the current device is {now}")
    return dev


def _same_device(t, dev: int, name: str):
    if not isinstance(t, torch.Tensor) or t.get_device() != dev:
        _current_device(t, name)


def _dtype_code(dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError("dtype must be torch.float32 or torch.bfloat16")
    return code


def _int32(t, dev: int, name: str) -> int:
    """The length of a contiguous 1-d int32 tensor on `dev`."""
    _same_device(t, dev, name)
    if t.dtype is not torch.int32 or t.dim() != 1 or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous 1-d int32 tensor")
    return t.shape[0]


_row_bytes: dict = {}


def mx_row_bytes(dim: int, bits: int) -> int:
    """Bytes of the record of a row of `dim` elements in MXFP4 or MXFP8."""
    n = _row_bytes.get((dim, bits))
    if n is None:
        n = lib().gmb_mx_row_bytes(dim, bits)
        if n == 0:
            _check(-1)
        _row_bytes[dim, bits] = n
    return n


def _records(t, dim: int, bits: int, name: str):
    """(rows, row stride in bytes) of a table of records: uint8 [rows, >= row
    bytes], rows contiguous and at a stride.  (One row has any: its length,
    rounded down to 16.)"""
    if t.dtype is not torch.uint8 or t.dim() != 2:
        raise TypeError(f"{name} must be a uint8 [rows, row bytes] tensor")
    rows, width = t.shape
    stride, inner = t.stride()
    if inner != 1:
        raise TypeError(f"{name} must have contiguous rows")
    if width < mx_row_bytes(dim, bits):
        raise ValueError(f"{name} has {width} bytes a row, {mx_row_bytes(dim, bits)} needed")
    return rows, stride if rows > 1 else width // 16 * 16


def _output(out, rows: int, cols: int, dtype, like: torch.Tensor) -> torch.Tensor:
    """`out`, or a new [rows, cols] tensor beside `like`."""
    if out is None:
        return like.new_empty((rows, cols), dtype=dtype)
    _same_device(out, like.get_device(), "out")
    if out.dim() != 2 or out.shape[0] < rows or out.shape[1] != cols or out.dtype != dtype or not out.is_contiguous():
        raise ValueError(f"out must be a contiguous [{rows} or more, {cols}] {dtype} tensor")
    return out


def _rows_of(ids, n, table_rows: int, dev: int, status_word):
    """(ids pointer, device count pointer, rows, status word) of a Blocks (its
    input vertices), an int32 tensor, or None (every row of the table)."""
    if isinstance(ids, Blocks):
        if n is not None:
            raise ValueError("n goes with an id tensor")
        _same_device(ids.workspace, dev, "the blocks")
        return (ids.struct.blk[0].src_ids, ids.input_count_ptr, ids.input_capacity,
                ids.csr.status_word if status_word is None else status_word)
    have = table_rows if ids is None else _int32(ids, dev, "ids")
    cap = have if n is None else int(n)
    if not 0 <= cap <= have:
        raise ValueError("n exceeds the rows")
    return ids.data_ptr() if ids is not None and cap else None, None, cap, status_word


def mx_quantise(x: torch.Tensor, bits: int, ids=None, table: torch.Tensor | None = None, csr: CSRGraph | None = None,
                status_word: int | None = None) -> torch.Tensor:
    """Quantises the rows of x (float32 or bfloat16 [n, dim], any non-negative
    strides: w.t() for a weight matrix) into microscaled records and returns
    their table (uint8 [rows, row bytes]).  With `ids` (int32, one a row, or a
    Blocks: x holds its input rows) they replace those rows of `table`: ids
    are distinct, or, with `csr` (a graph of table's rows, whose sampler state
    is used), an id's last row counts.  Without ids, row i is record i of
    `table` or of a new one."""
    dev = _current_device(x, "x")
    if x.dim() != 2:
        raise ValueError("x must be [rows, dim]")
    code = _dtype_code(x.dtype)
    rows, dim = x.shape
    if table is None:
        if ids is not None:
            raise ValueError("ids need a table")
        table = x.new_empty((rows, mx_row_bytes(dim, bits)), dtype=torch.uint8)
    else:
        _same_device(table, dev, "table")
    table_rows, stride = _records(table, dim, bits, "table")
    if ids is None:
        if rows > table_rows:
            raise ValueError("x has more rows than the table")
        ids_ptr, n_dev, cap, status = None, None, rows, status_word
    else:
        ids_ptr, n_dev, cap, status = _rows_of(ids, None, table_rows, dev, status_word)
        if rows < cap or (rows > cap and n_dev is None):
            raise ValueError("x must have one row per id (or the blocks' input capacity in rows)")
    state, state_bytes = None, 0
    if csr is not None:
        if ids is None or csr.num_nodes != table_rows:
            raise ValueError("csr needs ids and a table of its graph's vertices")
        _same_device(csr.state, dev, "csr")
        state, state_bytes = csr.state.data_ptr(), csr.state_bytes
    if cap == 0:
        return table
    row_stride, col_stride = x.stride()
    code = lib().gmb_mx_quantise(x.data_ptr(), code, row_stride if rows > 1 else 0, col_stride, ids_ptr, n_dev, cap,
                                 dim, bits, table.data_ptr(), table_rows, stride, state, state_bytes, status or None,
                                 _stream_handle())
    if code:
        _check(code)
    return table


def mx_gather(ids, table: torch.Tensor, dim: int, bits: int, dtype: torch.dtype = torch.float32,
              n: int | None = None, out: torch.Tensor | None = None, status_word: int | None = None) -> torch.Tensor:
    """gather_features from a microscaled store: out[i] = the values of record
    ids[i] as float32 or bfloat16.  `ids` is a Blocks (its input vertices), an
    int32 tensor (all of it, or the first n), or None (the table's rows, or
    the first n)."""
    dev = _current_device(table, "table")
    rows, stride = _records(table, dim, bits, "table")
    code = _dtype_code(dtype)
    ids_ptr, n_dev, cap, status = _rows_of(ids, n, rows, dev, status_word)
    out = _output(out, cap, dim, dtype, table)
    if cap:
        code = lib().gmb_mx_gather(ids_ptr, n_dev, cap, table.data_ptr(), rows, stride, dim, bits, out.data_ptr(),
                                   code, status or None, _stream_handle())
        if code:
            _check(code)
    return out


def mx_mean(block, table: torch.Tensor, dim: int, bits: int, dtype: torch.dtype = torch.float32,
            out: torch.Tensor | None = None) -> torch.Tensor:
    """The mean of every destination's neighbours' rows, straight from a
    microscaled store (0 for a destination without any).  `block` is (indptr,
    ids): int32 row offsets and the neighbours' records, or a Blocks (block
    0's destinations, at their capacity, and sampled vertices).  A neighbour
    outside the table is read as record 0 and not reported."""
    dev = _current_device(table, "table")
    table_rows, stride = _records(table, dim, bits, "table")
    if isinstance(block, Blocks):
        _same_device(block.workspace, dev, "the blocks")
        b = block.struct.blk[0]
        indptr_ptr, ids_ptr, n_dev, rows = b.indptr, b.nbr, b.sizes, int(b.cap_dst)
    else:
        indptr, ids = block
        rows = _int32(indptr, dev, "indptr") - 1
        _int32(ids, dev, "ids")
        if rows < 0:
            raise ValueError("indptr needs one entry more than rows")
        # (without edges there are no ids to point at; none is read)
        indptr_ptr = indptr.data_ptr()
        ids_ptr, n_dev = ids.data_ptr() or indptr_ptr, None
    code = _dtype_code(dtype)
    out = _output(out, rows, dim, dtype, table)
    if rows:
        code = lib().gmb_mx_mean(indptr_ptr, ids_ptr, n_dev, rows, table.data_ptr(), table_rows, stride, dim, bits,
                                 out.data_ptr(), code, _stream_handle())
        if code:
            _check(code)
    return out


def mx_linear(a: torch.Tensor, w: torch.Tensor, d_in: int, bias: torch.Tensor | None = None,
              a2: torch.Tensor | None = None, w2: torch.Tensor | None = None, ids: torch.Tensor | None = None,
              relu: bool = False, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None,
              status_word: int | None = None) -> torch.Tensor:
    """act(A W^T [+ A2 W2^T] + bias) of MXFP4 records of d_in elements: a
    [rows, .], w [d_out, .] (mx_quantise(matrix.t(), MXFP4) of a [d_in, d_out]
    matrix), a2 and w2 a second pair.  With `ids` row i of A is record ids[i]
    of `a`."""
    dev = _current_device(a, "a")
    _same_device(w, dev, "w")
    a_rows, a_stride = _records(a, d_in, MXFP4, "a")
    d_out, w_stride = _records(w, d_in, MXFP4, "w")
    code, rows, ids_ptr = _dtype_code(dtype), a_rows, None
    if ids is not None:
        rows = _int32(ids, dev, "ids")
        ids_ptr = ids.data_ptr()
    first = MxOperandStruct(a.data_ptr(), a_rows, a_stride, ids_ptr, w.data_ptr(), w_stride)
    second = None
    if a2 is not None or w2 is not None:
        if a2 is None or w2 is None:
            raise ValueError("a2 and w2 go together")
        _same_device(a2, dev, "a2")
        _same_device(w2, dev, "w2")
        a2_rows, a2_stride = _records(a2, d_in, MXFP4, "a2")
        w2_rows, w2_stride = _records(w2, d_in, MXFP4, "w2")
        if a2_rows < rows or w2_rows != d_out:
            raise ValueError("a2 must have a row for each of the product's, w2 one for each column")
        second = MxOperandStruct(a2.data_ptr(), a2_rows, a2_stride, None, w2.data_ptr(), w2_stride)
    if bias is not None:
        _same_device(bias, dev, "bias")
        if bias.dtype is not torch.float32 or bias.dim() != 1 or bias.shape[0] != d_out or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous float32 [d_out] tensor")
    out = _output(out, rows, d_out, dtype, a)
    if rows and d_out:
        code = lib().gmb_mx_linear(first, second, None, rows, d_in, d_out, None if bias is None else bias.data_ptr(),
                                   1 if relu else 0, out.data_ptr(), code, status_word or None, _stream_handle())
        if code:
            _check(code)
    return out


class SageMxWeights:
    """A GraphSAGE-mean model's weights in MXFP4: the records of the
    transposed matrices of a SageWeights, and its biases (copies: matrices
    and biases are those of the last set that was quantised)."""

    def __init__(self, weights: SageWeights):
        self.dims = list(weights.dims)
        self.bias = [b.clone() for b in self._biases(weights)]
        self.w_self = [mx_quantise(w.t(), MXFP4) for w in weights.w_self]
        self.w_neigh = [mx_quantise(w.t(), MXFP4) for w in weights.w_neigh]
        s = MxWeightsStruct()
        s.num_layers = len(self.w_self)
        for i, d in enumerate(self.dims):
            s.dims[i] = d
        for l in range(s.num_layers):
            s.w_self[l] = self.w_self[l].data_ptr()
            s.w_neigh[l] = self.w_neigh[l].data_ptr()
            s.bias[l] = self.bias[l].data_ptr()
        self.struct = s

    def _biases(self, weights: SageWeights):
        if any(b.numel() < d for b, d in zip(weights.bias, self.dims[1:])):
            raise ValueError("a bias must have one entry per column of its layer")
        return [b.reshape(-1)[:d] for b, d in zip(weights.bias, self.dims[1:])]

    def requantise(self, weights: SageWeights):
        """The records and biases of `weights` (the same widths) in place of
        the old, at the same addresses (captured graphs serve the new ones)."""
        if list(weights.dims) != self.dims:
            raise ValueError("the widths differ")
        for l, bias in enumerate(self._biases(weights)):
            mx_quantise(weights.w_self[l].t(), MXFP4, table=self.w_self[l])
            mx_quantise(weights.w_neigh[l].t(), MXFP4, table=self.w_neigh[l])
            self.bias[l].copy_(bias)

    def values(self) -> SageWeights:
        """What the records stand for, as float32 weights (the model's own
        biases, not copies): what sage_forward and sage_backward take to train
        the model on float32 masters."""
        def mat(rec, d_in):
            return mx_gather(None, rec, d_in, MXFP4).t().contiguous()
        return SageWeights([mat(w, d) for w, d in zip(self.w_self, self.dims)],
                           [mat(w, d) for w, d in zip(self.w_neigh, self.dims)], self.bias)


def mx_forward_workspace_bytes(blocks: Blocks, weights: SageMxWeights) -> int:
    return lib().gmb_mx_forward_workspace_bytes(ctypes.byref(blocks.struct), ctypes.byref(weights.struct))


def sage_forward_mx(blocks: Blocks, table: torch.Tensor, weights: SageMxWeights,
                    workspace: torch.Tensor | None = None, logits: torch.Tensor | None = None) -> torch.Tensor:
    """The forward of an MXFP4 model over an MXFP4 store (table: one record of
    dims[0] elements a vertex); the layers' means and hidden outputs are
    quantised as they are written.  Returns logits [num_seeds, C] float32."""
    dev = _current_device(table, "table")
    _same_device(blocks.workspace, dev, "the blocks")
    _same_device(weights.w_self[0], dev, "weights")
    rows, stride = _records(table, weights.dims[0], MXFP4, "table")
    B, C = blocks.num_seeds, weights.dims[-1]
    logits = _output(logits, B, C, torch.float32, table)
    if workspace is not None:
        _same_device(workspace, dev, "workspace")
    L, stream, status = lib(), _stream_handle(), blocks.csr.status_word

    def call(ws):
        return L.gmb_sage_forward_mx(ctypes.byref(blocks.struct), table.data_ptr(), rows, stride,
                                     ctypes.byref(weights.struct), logits.data_ptr(), ws.data_ptr(), ws.numel(),
                                     status, stream)

    code = ENOSPC
    if workspace is not None and workspace.numel() > 0 and workspace.data_ptr() % 256 == 0:
        code = call(workspace)
    if code == ENOSPC:
        need = mx_forward_workspace_bytes(blocks, weights)
        if need == 0:
            _check(-1)
        _, workspace = _aligned_bytes(need, table.device)
        code = call(workspace)
    _check(code)
    return logits


# ---------------------------------------------------------------- distillation

def _teacher(logits, classes, alpha: float, temperature: float) -> TeacherStruct:
    dev = _current_device(logits, "the teacher's logits")
    _same_device(classes, dev, "the teacher's classes")
    if logits.dtype is not torch.float32 or logits.dim() != 2 or not logits.is_contiguous():
        raise TypeError("the teacher's logits must be a contiguous float32 [rows, k] tensor")
    if classes.dtype is not torch.int32 or classes.shape != logits.shape or not classes.is_contiguous():
        raise TypeError("the teacher's classes must be a contiguous int32 tensor of the logits' shape")
    return TeacherStruct(logits.data_ptr(), classes.data_ptr(), logits.shape[1], alpha, temperature, 0)


class Teacher:
    """A teacher's top logits for a student: `logits` float32 [rows, k] and
    their `classes` int32 [rows, k] (-1 pads a shorter list), the weight alpha
    of the teacher against the labels, and the temperature."""

    def __init__(self, logits: torch.Tensor, classes: torch.Tensor, alpha: float = 0.5, temperature: float = 1.0):
        self.struct = _teacher(logits, classes, alpha, temperature)
        self.logits, self.classes = logits, classes
        self.rows = logits.shape[0]


_distill_bytes: dict = {}


def distill_loss(logits: torch.Tensor, teacher_logits: torch.Tensor, teacher_classes: torch.Tensor,
                 labels: torch.Tensor | None = None, alpha: float = 0.5, temperature: float = 1.0,
                 grad: torch.Tensor | bool = True, loss: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None):
    """The mean over the rows of alpha T^2 KL(teacher || student) over the
    teacher's top entries plus (1 - alpha) times the cross-entropy against
    `labels` (int32, -1 for none), and its gradient in `logits` (float32 or
    bfloat16 [rows, C]).  Returns (loss, grad): a 1-element float32 tensor and
    a tensor like logits (None for grad=False)."""
    dev = _current_device(logits, "logits")
    if logits.dim() != 2 or not logits.is_contiguous():
        raise ValueError("logits must be a contiguous [rows, classes] tensor")
    code = _dtype_code(logits.dtype)
    rows, classes = logits.shape
    teacher = _teacher(teacher_logits, teacher_classes, alpha, temperature)
    if teacher_logits.shape[0] != rows:
        raise ValueError("the teacher must have one row per row of logits")
    if labels is not None and _int32(labels, dev, "labels") != rows:
        raise ValueError("labels must have one entry per row")
    if grad is True:
        grad = torch.empty_like(logits)
    elif grad is False:
        grad = None
    else:
        _same_device(grad, dev, "grad")
        if grad.shape != logits.shape or grad.dtype != logits.dtype or not grad.is_contiguous() \
                or (rows and grad.data_ptr() == logits.data_ptr()):
            raise ValueError("grad must be a contiguous tensor like logits, and another one")
    if loss is None:
        loss = logits.new_empty(1, dtype=torch.float32)
    else:
        _same_device(loss, dev, "loss")
        if loss.dtype != torch.float32 or loss.numel() != 1:
            raise ValueError("loss must be a 1-element float32 tensor")
    L = lib()
    need = _distill_bytes.get((rows, classes))
    if need is None:
        need = L.gmb_distill_workspace_bytes(rows, classes)
        if need == 0:
            _check(-1)
        if len(_distill_bytes) < 4096:
            _distill_bytes[rows, classes] = need
    if workspace is not None:
        _same_device(workspace, dev, "workspace")
    if workspace is None or workspace.numel() < need or workspace.data_ptr() % 256:
        workspace = logits.new_empty(need, dtype=torch.uint8)
        if workspace.data_ptr() % 256:   # (torch's own blocks are aligned)
            _, workspace = _aligned_bytes(need, logits.device)
    code = L.gmb_distill_loss(logits.data_ptr(), code, rows, classes, teacher,
                              None if labels is None else labels.data_ptr(),
                              None if grad is None else grad.data_ptr(), loss.data_ptr(), workspace.data_ptr(),
                              workspace.numel(), _stream_handle())
    if code:
        _check(code)
    return loss, grad


# ---------------------------------------------------------------- dropout, norm and loss of a residual model

class Dropout:
    """A dropout of probability p whose mask is never stored: which elements
    are dropped is a function of `seed`, the row's key, `layer`, the column and
    `step` (gmb.h), so that the backward draws it again.  `step` is a device
    int32 tensor of one element (or None: 0) that the kernels read: moved
    between replays, it gives a captured step other masks."""

    def __init__(self, p: float, seed: int, layer: int = 0, step: torch.Tensor | None = None):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must lie in 0 .. 1")
        if not 0 <= layer < 1 << 31:
            raise ValueError("layer must lie in 0 .. 2^31 - 1")
        if step is not None:
            _current_device(step, "step")
            if step.dtype is not torch.int32 or step.numel() != 1:
                raise TypeError("step must be an int32 tensor of one element")
        self.p, self.seed, self.layer, self.step = p, seed, layer, step
        self.struct = DropoutStruct(seed & 0xFFFFFFFFFFFFFFFF, p, layer, None if step is None else step.data_ptr())


def _row_struct(t, shape, dtype, dev: int, name: str) -> RowsStruct:
    """A tensor of that shape [rows, dim] and dtype with contiguous rows at any stride."""
    if not isinstance(t, torch.Tensor) or t.get_device() != dev:
        _current_device(t, name)
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name} must be a [{shape[0]}, {shape[1]}] {dtype} tensor")
    rows, dim = shape
    if t.is_contiguous():
        return RowsStruct(t.data_ptr(), dim)
    stride, inner = t.stride()
    if (inner != 1 and dim > 1) or (stride < dim and rows > 1):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return RowsStruct(t.data_ptr(), stride if rows > 1 else dim)


def _row_input(x, name: str):
    """(device, dtype code, shape, struct) of the tensor that the others of a call go by."""
    dev = _current_device(x, name)
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be [rows, dim]")
    return dev, _dtype_code(x.dtype), shape, _row_struct(x, shape, x.dtype, dev, name)


def _row_like(x: torch.Tensor) -> torch.Tensor:
    """A new contiguous tensor like x."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


def _drop_struct(drop, dev: int):
    if not isinstance(drop, Dropout):
        raise TypeError("dropout must be a Dropout")
    if drop.step is not None:
        _same_device(drop.step, dev, "the dropout's step")
    return drop.struct


def _row_keys(ids, count, rows: int, dev: int):
    """The pointers of the rows' keys and of their number on the device."""
    if ids is None and count is None:
        return None, None
    if ids is not None and _int32(ids, dev, "ids") != rows:
        raise ValueError("ids must have one entry per row")
    if count is not None and _int32(count, dev, "count") != 1:
        raise ValueError("count must have one element")
    return None if ids is None else ids.data_ptr(), None if count is None else count.data_ptr()


def dropout(x: torch.Tensor, drop: Dropout, ids: torch.Tensor | None = None, residual: torch.Tensor | None = None,
            out: torch.Tensor | None = None, count: torch.Tensor | None = None) -> torch.Tensor:
    """[residual +] x with elements dropped and the others scaled, float32 or
    bfloat16 [rows, dim] with contiguous rows at any stride.  Row i's key is
    ids[i] (int32: a vertex has the same mask wherever it stands), or i.  The
    backward is the same call on the gradient.  With `count` (device int32 of
    one element) only the first rows are read and written.  `out` may be x or
    residual."""
    dev, code, shape, a = _row_input(x, "x")
    rows, dim = shape
    d = _drop_struct(drop, dev)
    keys, n_dev = _row_keys(ids, count, rows, dev)
    b = None if residual is None else _row_struct(residual, shape, x.dtype, dev, "residual")
    if out is None:
        out = _row_like(x)
        o = RowsStruct(out.data_ptr(), dim)
    else:
        o = _row_struct(out, shape, x.dtype, dev, "out")
    if rows:
        code = lib().gmb_dropout_rows(a, b, d, keys, n_dev, rows, dim, code, o, _stream_handle())
        if code:
            _check(code)
    return out


def _norm_weight(weight, dim: int, dev: int):
    if weight is None:
        return None
    _same_device(weight, dev, "weight")
    if weight.dtype is not torch.float32 or weight.dim() != 1 or weight.shape[0] != dim or not weight.is_contiguous():
        raise ValueError("weight must be a contiguous float32 [dim] tensor")
    return weight.data_ptr()


def rms_norm(x: torch.Tensor, weight: torch.Tensor | None, eps: float = 1e-6, residual: torch.Tensor | None = None,
             dropout: Dropout | None = None, bits: int | None = None, ids: torch.Tensor | None = None,
             out: torch.Tensor | None = None, sum_out: torch.Tensor | None = None,
             count: torch.Tensor | None = None):
    """The root-mean-square norm of r = [residual +] x (x dropped out first with
    `dropout`, rows keyed as in gmb.dropout): returns (y, r), y = weight r /
    sqrt(mean(r^2) + eps).  y has x's dtype, or, with `bits` (MXFP4 or MXFP8),
    is a table of records like mx_quantise's.  r is rounded to x's dtype before
    it is normed; it is x itself if nothing is added or dropped (with out=x too:
    then it holds y).  `count` as in gmb.dropout; `sum_out` may be x or residual,
    so may `out` if `sum_out` is not."""
    dev, code, shape, a = _row_input(x, "x")
    rows, dim = shape
    keys, n_dev = _row_keys(ids, count, rows, dev)
    b = None if residual is None else _row_struct(residual, shape, x.dtype, dev, "residual")
    drop = None if dropout is None else _drop_struct(dropout, dev)
    g = _norm_weight(weight, dim, dev)
    r, total = x, None
    if sum_out is not None or residual is not None or dropout is not None:
        if sum_out is None:
            r = _row_like(x)
            total = RowsStruct(r.data_ptr(), dim)
        else:
            r = sum_out
            total = _row_struct(r, shape, x.dtype, dev, "sum_out")
    if bits is None:
        if out is None:
            out = _row_like(x)
            o = RowsStruct(out.data_ptr(), dim)
        else:
            o = _row_struct(out, shape, x.dtype, dev, "out")
    elif out is None:
        stride = mx_row_bytes(dim, bits)
        out = x.new_empty((rows, stride), dtype=torch.uint8)
        o = RowsStruct(out.data_ptr(), stride)
    else:
        _same_device(out, dev, "out")
        have, stride = _records(out, dim, bits, "out")
        if have < rows:
            raise ValueError("out has fewer rows than x")
        o = RowsStruct(out.data_ptr(), stride)
    if rows:
        code = lib().gmb_rms_norm(a, b, drop, keys, n_dev, rows, dim, code, g, eps, total, bits or 0, o,
                                  _stream_handle())
        if code:
            _check(code)
    return out, r


class NormGrads(NamedTuple):
    """Gradients of rms_norm's x, residual and weight (without dropout x's and
    the residual's are one tensor)."""
    x: torch.Tensor
    residual: torch.Tensor
    weight: torch.Tensor | None


def _workspace(workspace, need: int, like: torch.Tensor, dev: int) -> torch.Tensor:
    """`workspace` if it holds `need` bytes at an aligned address, or a new one."""
    if workspace is not None:
        _same_device(workspace, dev, "workspace")
        if workspace.dtype is torch.uint8 and workspace.numel() >= need and workspace.data_ptr() % 256 == 0:
            return workspace
    workspace = like.new_empty(need, dtype=torch.uint8)
    if workspace.data_ptr() % 256:   # (torch's own blocks are aligned)
        _, workspace = _aligned_bytes(need, like.device)
    return workspace


def rms_norm_backward(dy: torch.Tensor, r: torch.Tensor, weight: torch.Tensor | None, eps: float = 1e-6,
                      carry: torch.Tensor | None = None, dropout: Dropout | None = None,
                      ids: torch.Tensor | None = None, count: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None) -> NormGrads:
    """The gradients of rms_norm from dy, that of y, and r, the sum that it
    returned (both of x's dtype).  `carry` is the gradient that reaches r from
    elsewhere (the residual stream); `dropout`, `ids` and `count` are the
    forward's.  The weight's gradient is float32 (None without a weight), summed
    in a fixed order."""
    dev, code, shape, a = _row_input(r, "r")
    rows, dim = shape
    b = _row_struct(dy, shape, r.dtype, dev, "dy")
    keys, n_dev = _row_keys(ids, count, rows, dev)
    c = None if carry is None else _row_struct(carry, shape, r.dtype, dev, "carry")
    drop = None if dropout is None else _drop_struct(dropout, dev)
    g = _norm_weight(weight, dim, dev)
    d_residual = _row_like(r)
    to = RowsStruct(d_residual.data_ptr(), dim)
    dx, to_x = d_residual, None
    if drop is not None:
        dx = _row_like(r)
        to_x = RowsStruct(dx.data_ptr(), dim)
    dw = dw_ptr = ws = None
    need = 0
    if weight is not None:
        dw = torch.empty_like(weight)
        dw_ptr = dw.data_ptr()
        need = lib().gmb_rms_norm_workspace_bytes(rows, dim)
        if need == 0:
            _check(-1)
        workspace = _workspace(workspace, need, r, dev)
        ws, need = workspace.data_ptr(), workspace.numel()
    code = lib().gmb_rms_norm_backward(b, a, c, drop, keys, n_dev, rows, dim, code, g, eps, to, to_x, dw_ptr, ws, need,
                                       _stream_handle())
    if code:
        _check(code)
    return NormGrads(dx, d_residual, dw)


class LinearGrads(NamedTuple):
    """Gradients of linear_loss (None where they were not asked for)."""
    x: torch.Tensor | None
    w: torch.Tensor | None
    bias: torch.Tensor | None


def linear_loss(x: torch.Tensor, w: torch.Tensor, labels: torch.Tensor, bias: torch.Tensor | None = None,
                grad=True, loss: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """The mean over the rows of the softmax cross-entropy of x W^T + bias
    against `labels` (int32; a row whose label is no class, -1 for instance,
    counts as 0), and its gradients, without the logits ever being stored.  x
    is float32 or bfloat16 [rows, d] with contiguous rows, w [classes, d] of the
    same dtype with any non-negative strides: an embedding table, or matrix.t()
    of a [d, classes] matrix; bias float32 [classes] (-inf or the type's lowest
    value: a class that cannot be).  Returns (loss,
    LinearGrads): the loss float32 of one element, the gradients of x and w of
    their dtype (w's laid out like w), the bias's float32.  `grad` is True,
    False, or the names of the gradients wanted ("x", "w", "bias")."""
    dev, code, shape, a = _row_input(x, "x")
    rows, d = shape
    _same_device(w, dev, "w")
    if w.dim() != 2 or w.shape[1] != d or w.dtype is not x.dtype:
        raise ValueError(f"w must be a [classes, {d}] {x.dtype} tensor")
    classes = w.shape[0]
    if _int32(labels, dev, "labels") != rows:
        raise ValueError("labels must have one entry per row")
    if bias is not None:
        _same_device(bias, dev, "bias")
        if bias.dtype is not torch.float32 or bias.dim() != 1 or bias.shape[0] != classes or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous float32 [classes] tensor")
    if grad is True or grad is False:
        want_x = want_w = want_bias = grad
    else:
        grad = set(grad)
        if grad - {"x", "w", "bias"}:
            raise ValueError("grad names x, w and bias")
        want_x, want_w, want_bias = "x" in grad, "w" in grad, "bias" in grad
    row_stride, col_stride = w.stride()
    turned = row_stride == 1 and col_stride >= classes and d > 1 and classes > 1
    dx = _row_like(x) if want_x else None
    dw = None
    if want_w:
        dw = w.new_empty((d, classes)).t() if turned else _row_like(w)
    db = torch.empty_like(bias) if want_bias and bias is not None else None
    if loss is None:
        loss = x.new_empty(1, dtype=torch.float32)
    else:
        _same_device(loss, dev, "loss")
        if loss.dtype != torch.float32 or loss.numel() != 1:
            raise ValueError("loss must be a 1-element float32 tensor")
    head = LinearHeadStruct(a.data, a.stride, w.data_ptr(), row_stride, col_stride,
                            None if bias is None else bias.data_ptr(), labels.data_ptr(), rows, d, classes, code, 0)
    grads = None
    if dx is not None or dw is not None or db is not None:
        grads = LinearGradsStruct(None if dx is None else dx.data_ptr(), None if dw is None else dw.data_ptr(),
                                  None if db is None else db.data_ptr(), 1 if turned else 0, 0)
    L = lib()
    need = L.gmb_linear_loss_workspace_bytes(head, grads)
    if need == 0:
        _check(-1)
    workspace = _workspace(workspace, need, x, dev)
    code = L.gmb_linear_loss(head, grads, loss.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream_handle())
    if code:
        _check(code)
    return loss, LinearGrads(dx, dw, db)
