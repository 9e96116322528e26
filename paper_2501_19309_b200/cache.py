"""What runs around a verification call, as tensors: rotary positions, the paged key / value cache and the attention of
a drafted block over it (the second half of ``include/jd.h``).

One decoding step of a stack of target layers::

    cache.reserve(T)                                             # pages for the block
    for layer in ...:
        q = cache.append(layer, k, v, tree, rotary=rotary, q=q)  # turn q and k, write k and v
        o = cache.attend(layer, q, tree)["out"]                  # context + the nodes each node may see
    out = verifier.verify(H, draft_tokens, draft_logits, ...)    # accept_len stays on the device
    cache.commit(out["accept_len"])                              # keep the accepted nodes, drop the rest (of a tree: with paths)

Argument marshalling only; every step runs inside the library's kernels.  All calls are enqueued on ``stream`` (default:
torch's current stream of the cache's device) and none waits for the device, except :meth:`PagedCache.status`.  Outputs that a
call makes itself are allocated on the current stream: with another ``stream``, pass them in.  Nothing here records a graph for
autograd: inputs that require gradients are refused while gradients are enabled, and so are inputs with a forward-mode tangent.
"""
from __future__ import annotations

import ctypes as C
import math
import struct
from typing import Optional

import torch
import torch.autograd.forward_ad as _fw

from . import jd

LAYOUTS = {"half": jd.JD_ROPE_HALF, "interleaved": jd.JD_ROPE_INTERLEAVED}
SCALINGS = {None: jd.JD_ROPE_SCALE_NONE, "none": jd.JD_ROPE_SCALE_NONE, "linear": jd.JD_ROPE_SCALE_LINEAR,
            "bands": jd.JD_ROPE_SCALE_BANDS, "yarn": jd.JD_ROPE_SCALE_YARN}
ATTEND_VARIANTS = {"auto": jd.JD_ATTEND_AUTO, "simt": jd.JD_ATTEND_SIMT, "tensor": jd.JD_ATTEND_TENSOR}
_DTYPES = {torch.float32: jd.JD_DTYPE_F32, torch.bfloat16: jd.JD_DTYPE_BF16}


def _check(status: int, where: str) -> None:
    if status != jd.JD_OK:
        raise jd.JdError(status, where)


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


# These calls are made for every layer of every token: what follows avoids what costs microseconds in Python (stream objects,
# device comparisons, messages that are formatted before they are needed; new_empty with a plain tuple takes 1.8 us where torch.empty with
# another tensor's shape and device takes 5.5).
# Argument structs are packed in one go, in the C compiler's layout, instead of field by field.
_raw_stream = torch._C._cuda_getCurrentRawStream
_TREE = "iiPPP"
_ROPE_ARGS = struct.Struct("@qiiiiPPqqPPiif")
_APPEND_ARGS = struct.Struct("@iiP" + _TREE + "PPPPqqqqP")
_ATTEND_ARGS = struct.Struct("@iiP" + _TREE + "PPqqPfi")
_COMMIT_ARGS = struct.Struct("@iPPiiPP")


def _has_tangent(x: torch.Tensor) -> bool:
    return _fw.unpack_dual(x).tangent is not None


def _stream(stream, index: int) -> int:
    return stream.cuda_stream if stream is not None else _raw_stream(index)


def _ints(x, name: str, index: int, shape=None) -> int:
    """Pointer of an int32 device tensor, 0 for None."""
    if x is None:
        return 0
    if x.dtype is not torch.int32 or x.get_device() != index or not x.is_contiguous() or (shape is not None and x.shape != shape):
        raise ValueError("%s: a contiguous int32 tensor%s on the cache's device" % (name, "" if shape is None else " of shape %s" % (shape,)))
    return x.data_ptr()


def rope_frequencies(rot_dim: int, base: float = 500000.0, scaling: Optional[str] = None, factor: float = 1.0,
                     original_len: float = 8192.0, low: float = 1.0, high: float = 4.0):
    """(frequencies [rot_dim / 2] as a float32 CPU tensor, amplitude); see ``jd_rope_frequencies``."""
    out = torch.empty(max(0, rot_dim // 2), dtype=torch.float32)
    amplitude = C.c_float(0.0)
    st = jd.load().jd_rope_frequencies(rot_dim, base, SCALINGS[scaling], factor, original_len, low, high,
                                       out.data_ptr(), C.addressof(amplitude))
    _check(st, "jd_rope_frequencies")
    return out, amplitude.value


class Rotary:
    """Rotary positions: frequencies [rot_dim / 2] (float32, on the device), layout and amplitude."""

    def __init__(self, inv_freq: torch.Tensor, layout: str = "half", amplitude: float = 1.0):
        _require(inv_freq.dtype == torch.float32 and inv_freq.is_contiguous() and inv_freq.dim() == 1,
                 "inv_freq: a contiguous float32 vector")
        _require(not inv_freq.requires_grad, "inv_freq: no autograd here; detach it")
        self.inv_freq, self.layout, self.amplitude = inv_freq, layout, float(amplitude)
        self.rot_dim = 2 * inv_freq.numel()
        self._layout = LAYOUTS[layout]
        self.c = jd.jd_rope_t(inv_freq.data_ptr(), self.rot_dim, self._layout, self.amplitude)
        self.ref = C.addressof(self.c)
        self.index = inv_freq.get_device()
        self._lib = jd.load()

    def rotate(self, x: torch.Tensor, positions: torch.Tensor, out: Optional[torch.Tensor] = None, inverse: bool = False,
               stream=None) -> torch.Tensor:
        """Turns x [tokens, heads, head_dim] (tokens may be strided) to its positions [tokens] (int32). ``inverse`` turns back: with
        the gradient of the output as x, the result is the gradient of the input. ``out`` may be x."""
        if x.dim() != 3 or x.dtype not in _DTYPES or not x.is_cuda:
            raise ValueError("x: [tokens, heads, head_dim], float32 or bfloat16, on the device")
        n, heads, dim = x.shape
        index = x.get_device()
        if out is None:
            out = x.new_empty((n, heads, dim))
        elif out.shape != x.shape or out.dtype is not x.dtype or out.get_device() != index:
            raise ValueError("out: like x")
        x_step, out_step = self._step(x, "x", n, heads, dim), self._step(out, "out", n, heads, dim)
        at = _ints(positions, "positions", index, (n,))
        if self.index != index:
            raise ValueError("inv_freq and x on one device")
        if n == 0:
            return out
        a = jd.jd_rope_args_t()
        _ROPE_ARGS.pack_into(a, 0, n, heads, dim, _DTYPES[x.dtype], 1 if inverse else 0, x.data_ptr(), out.data_ptr(), x_step, out_step, at,
                             self.inv_freq.data_ptr(), self.rot_dim, self._layout, self.amplitude)
        if torch._C._cuda_getDevice() == index:
            st = self._lib.jd_rope(a, _stream(stream, index))
        else:
            with torch.cuda.device(index):
                st = self._lib.jd_rope(a, _stream(stream, index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_rope")
        return out

    @staticmethod
    def _step(t: torch.Tensor, name: str, n: int, heads: int, dim: int) -> int:
        """Elements between tokens, 0: dense."""
        if t.requires_grad and torch.is_grad_enabled() or _fw._current_level >= 0 and _has_tangent(t):
            raise ValueError("%s: no autograd here; detach it, the gradient is rotate(grad, positions, inverse=True)" % name)
        if t.is_contiguous():
            return 0
        step, by_head, by_element = t.stride()
        if (dim > 1 and by_element != 1) or (heads > 1 and by_head != dim):
            raise ValueError("%s: heads of a token contiguous" % name)
        if n > 1 and step < heads * dim:      # a broadcast among them: its step of 0 would stand for dense
            raise ValueError("%s: tokens must not overlap" % name)
        return step if n > 1 else 0


class Tree:
    """A block of ``nodes`` drafted tokens (node 0: the last context token). mask [T, W] or [B, T, W] and depth [T] or [B, T]
    as in ``jd_tree_t`` (int32 words, W = ceil(T / 32)); both per sequence or neither; None: a chain. num_nodes [B]: nodes of each
    sequence of a padded batch."""

    def __init__(self, nodes: int, mask: Optional[torch.Tensor] = None, depth: Optional[torch.Tensor] = None,
                 num_nodes: Optional[torch.Tensor] = None):
        self.nodes, self.mask, self.depth, self.num_nodes = int(nodes), mask, depth, num_nodes
        words = (self.nodes + 31) // 32
        batched = set()
        for x, tail, name in ((mask, (self.nodes, words), "mask"), (depth, (self.nodes,), "depth")):
            if x is None:
                continue
            _require(x.dtype == torch.int32 and x.is_contiguous(), "%s: a contiguous int32 tensor" % name)
            _require(tuple(x.shape[-len(tail):]) == tail and x.dim() <= len(tail) + 1, "%s: shape %s, or with B in front" % (name, tail))
            _require(x.numel() > 0, "%s: at least one sequence" % name)
            batched.add(int(x.shape[0]) if x.dim() > len(tail) else 0)
        if num_nodes is not None:
            _require(num_nodes.dtype == torch.int32 and num_nodes.is_contiguous() and num_nodes.dim() == 1, "num_nodes: a contiguous int32 vector")
        _require(len(batched) <= 1, "mask and depth: both per sequence, of one batch size, or neither")
        self.batch = batched.pop() if batched else 0            # 0: shared
        self.index = next((x.get_device() for x in (mask, depth, num_nodes) if x is not None), None)
        for x in (mask, depth, num_nodes):
            _require(x is None or x.get_device() == self.index, "mask, depth and num_nodes on one device")
        self.sequences = None if num_nodes is None else num_nodes.shape[0]
        self.c = (self.nodes, 1 if self.batch else 0, *(0 if x is None else x.data_ptr() for x in (mask, depth, num_nodes)))

    @classmethod
    def from_parents(cls, parents, device, num_nodes: Optional[torch.Tensor] = None) -> "Tree":
        """parents: for every node the number of its parent, -1 for node 0, [T] or [B, T] (host lists or a CPU tensor); a
        parent comes before its children."""
        p = torch.as_tensor(parents, dtype=torch.int64, device="cpu")
        _require(p.dim() in (1, 2) and p.shape[-1] >= 1, "parents: [T] or [B, T]")
        rows = p.reshape(-1, p.shape[-1])
        T = rows.shape[1]
        ids = torch.arange(T)
        _require(bool((rows[:, 0] == -1).all()) and bool(((rows[:, 1:] >= 0) & (rows[:, 1:] < ids[1:])).all()),
                 "parents: -1 for node 0, an earlier node for every other")
        see = torch.zeros(rows.shape[0], T, T, dtype=torch.bool)
        for i in range(T):
            if i:
                see[:, i] = see[torch.arange(rows.shape[0]), rows[:, i]]
            see[:, i, i] = True
        depth = (see.sum(2) - 1).to(torch.int32)
        mask = mask_words(see)
        if p.dim() == 1:
            mask, depth = mask[0], depth[0]
        return cls(T, mask.to(device), depth.to(device), num_nodes)


def mask_words(see: torch.Tensor) -> torch.Tensor:
    """Truth values [..., T, T] (node i sees node j) as the int32 words [..., T, ceil(T / 32)] of :class:`Tree`."""
    T = see.shape[-1]
    words = (T + 31) // 32
    bits = torch.zeros(*see.shape[:-1], words * 32, dtype=torch.int64, device=see.device)
    bits[..., :T] = see
    w = (bits.view(*see.shape[:-1], words, 32) << torch.arange(32, device=see.device)).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


class PagedCache:
    """Keys and values of many sequences in pages, and the tables that say whose they are (``jd_cache_buffers_t``). Adopts the
    tensors it is given, which the caller may read between calls; :meth:`allocate` makes an empty cache."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, seq_len: torch.Tensor, held: torch.Tensor,
                 refs: torch.Tensor, free_bits: torch.Tensor, q_heads: int, max_nodes: int = 64):
        self.h = None
        _require(not (k.requires_grad or v.requires_grad), "k, v: no autograd here; detach them")
        _require(k.dim() == 5 and k.is_cuda and k.is_contiguous() and k.dtype in _DTYPES, "k: contiguous [layers, pages, kv_heads, page_size, head_dim]")
        _require(v.shape == k.shape and v.dtype == k.dtype and v.device == k.device and v.is_contiguous(), "v: like k")
        self.device, self.index, self.dtype = k.device, k.get_device(), k.dtype
        dev = self.index
        layers, pages, kv_heads, page_size, dim = k.shape
        _require(page_table.dim() == 2, "page_table: [seqs, pages of a sequence]")
        seqs, per_seq = page_table.shape
        ptrs = [_ints(x, n, dev, s) for x, n, s in (
            (page_table, "page_table", (seqs, per_seq)), (seq_len, "seq_len", (seqs,)), (held, "held", (seqs,)),
            (refs, "refs", (pages,)), (free_bits, "free_bits", ((pages + 31) // 32,)))]
        self.k, self.v, self.page_table, self.seq_len, self.held, self.refs, self.free_bits = k, v, page_table, seq_len, held, refs, free_bits
        self.q_heads, self.kv_heads, self.head_dim, self.max_nodes, self.max_seqs = int(q_heads), kv_heads, dim, int(max_nodes), seqs
        self.cfg = jd.jd_cache_config_t(layers, pages, page_size, self.q_heads, kv_heads, dim, seqs, per_seq, self.max_nodes,
                                        _DTYPES[k.dtype], dev)
        self._lib = lib = jd.load()
        need = lib.jd_cache_workspace_bytes(C.byref(self.cfg))
        if need == 0:
            raise jd.JdError(jd.JD_ERR_INVALID_ARG, "jd_cache_workspace_bytes")
        self.workspace = torch.zeros(need, dtype=torch.uint8, device=self.device)
        buf = jd.jd_cache_buffers_t(k.data_ptr(), v.data_ptr(), *ptrs, self.workspace.data_ptr(), need)
        h = C.c_void_p()
        _check(lib.jd_cache_create(C.byref(h), C.byref(self.cfg), C.byref(buf)), "jd_cache_create")
        self.h = h
        self._scale = 1.0 / math.sqrt(dim)
        torch.cuda.current_stream(dev).synchronize()     # the zeroes are there, whatever stream the first call is on

    @classmethod
    def allocate(cls, num_layers: int, num_pages: int, page_size: int, q_heads: int, kv_heads: int, head_dim: int, max_seqs: int,
                 max_pages: int, max_nodes: int = 64, dtype: str = "bf16", device: int = 0) -> "PagedCache":
        t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        dev = torch.device("cuda", device)
        shape = (num_layers, num_pages, kv_heads, page_size, head_dim)
        ints = dict(dtype=torch.int32, device=dev)
        see = torch.zeros((num_pages + 31) // 32 * 32, dtype=torch.bool)
        see[:num_pages] = True
        w = (see.view(-1, 32).to(torch.int64) << torch.arange(32)).sum(1)
        free = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32).to(dev)
        return cls(torch.zeros(shape, dtype=t, device=dev), torch.zeros(shape, dtype=t, device=dev),
                   torch.full((max_seqs, max_pages), -1, **ints), torch.zeros(max_seqs, **ints), torch.zeros(max_seqs, **ints),
                   torch.zeros(num_pages, **ints), free, q_heads, max_nodes)

    def close(self) -> None:
        if getattr(self, "h", None) is not None:
            self._lib.jd_cache_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _batch(self, slots, B: Optional[int] = None) -> int:
        if slots is None:
            return self.max_seqs if B is None else B
        if slots.dim() != 1 or (B is not None and slots.shape[0] != B):
            raise ValueError("slots: one for each sequence")
        return slots.shape[0]

    def _tokens(self, x: torch.Tensor, name: str, shape) -> int:
        """Elements between tokens (0: dense) of [B, T, heads, head_dim] whose tokens lie evenly, heads contiguous."""
        if x.shape != shape or x.dtype is not self.dtype or x.get_device() != self.index:
            raise ValueError("%s: %s of the cache's type, on its device" % (name, list(shape)))
        if x.requires_grad and torch.is_grad_enabled() or _fw._current_level >= 0 and _has_tangent(x):
            raise ValueError("%s: no autograd here; detach it" % name)
        if x.is_contiguous():
            return 0
        B, T, H, D = shape
        sb, st, sh, sd = x.stride()
        step = st if T > 1 else sb
        if (D > 1 and sd != 1) or (H > 1 and sh != D) or (B > 1 and T > 1 and sb != T * st):
            raise ValueError("%s: heads of a token contiguous, tokens evenly spaced" % name)
        if B * T > 1 and step < H * D:        # a broadcast among them: its step of 0 would stand for dense
            raise ValueError("%s: tokens must not overlap" % name)
        return step if B * T > 1 else 0

    def _tree(self, tree: Optional[Tree], B: int, T: int):
        if tree is None:
            return (T, 0, 0, 0, 0)
        if tree.nodes != T or (tree.batch != 0 and tree.batch != B) or (tree.sequences is not None and tree.sequences != B):
            raise ValueError("tree: of %d nodes, shared or for %d sequences" % (T, B))
        if tree.index is not None and tree.index != self.index:
            raise ValueError("tree: on the cache's device")
        return tree.c

    def reserve(self, n: int, slots: Optional[torch.Tensor] = None, stream=None) -> None:
        """Pages for n more tokens of every sequence (``jd_cache_reserve``)."""
        if not -1 << 31 <= n < 1 << 31:           # ctypes would drop the upper bits
            raise ValueError("n: a number of tokens")
        B = self._batch(slots)
        st = self._lib.jd_cache_reserve(self.h, B, _ints(slots, "slots", self.index), n, _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_reserve")

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, tree: Optional[Tree] = None, rotary: Optional[Rotary] = None,
               q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None, stream=None):
        """Writes a block's keys and values [B, T, kv_heads, head_dim] behind the sequences' tokens, turned to their positions,
        and returns the turned queries (q_out; a new tensor if None), or None without q."""
        if k.dim() != 4:
            raise ValueError("k, v: [B, T, kv_heads, head_dim]")
        B, T, _, D = k.shape
        if slots is not None:
            self._batch(slots, B)
        at = _ints(slots, "slots", self.index)
        t0, t1, t2, t3, t4 = self._tree(tree, B, T)
        kv = (B, T, self.kv_heads, self.head_dim)
        k_step, v_step = self._tokens(k, "k", kv), self._tokens(v, "v", kv)
        q_ptr = o_ptr = q_step = o_step = rope = 0
        if q is not None:
            if q_out is None:
                q_out = q.new_empty((B, T, self.q_heads, self.head_dim))
            qs = (B, T, self.q_heads, self.head_dim)
            q_ptr, q_step = q.data_ptr(), self._tokens(q, "q", qs)
            o_ptr, o_step = q_out.data_ptr(), self._tokens(q_out, "q_out", qs)
        else:
            q_out = None
        if rotary is not None:
            if rotary.index != self.index:
                raise ValueError("rotary: on the cache's device")
            rope = rotary.ref
        a = jd.jd_append_args_t()
        _APPEND_ARGS.pack_into(a, 0, B, layer, at, t0, t1, t2, t3, t4, k.data_ptr(), v.data_ptr(), q_ptr, o_ptr, k_step, v_step, q_step, o_step, rope)
        st = self._lib.jd_cache_append(self.h, a, _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_append")
        return q_out

    def attend(self, layer: int, q: torch.Tensor, tree: Optional[Tree] = None, scale: Optional[float] = None, out: Optional[dict] = None,
               slots: Optional[torch.Tensor] = None, variant="auto", stream=None) -> dict:
        """Attention of q [B, T, q_heads, head_dim] over the sequences' tokens and the block's visible nodes; scale: on q . k,
        default head_dim ** -0.5. Returns (and takes) a dict with "out" like q and "lse" [B, T, q_heads] (may be absent in a
        dict that is given)."""
        if q.dim() != 4:
            raise ValueError("q: [B, T, q_heads, head_dim]")
        B, T, H, D = q.shape
        if slots is not None:
            self._batch(slots, B)
        if out is None:
            out = dict(out=q.new_empty((B, T, H, D)), lse=q.new_empty((B, T, H), dtype=torch.float32))
        o, lse = out["out"], out.get("lse")
        at = _ints(slots, "slots", self.index)
        t0, t1, t2, t3, t4 = self._tree(tree, B, T)
        shape = (B, T, self.q_heads, self.head_dim)
        q_step, o_step, l_ptr = self._tokens(q, "q", shape), self._tokens(o, "out", shape), 0
        if lse is not None:
            if lse.dtype is not torch.float32 or lse.get_device() != self.index or not lse.is_contiguous() or lse.shape != shape[:3]:
                raise ValueError("lse: contiguous float32 [B, T, q_heads]")
            l_ptr = lse.data_ptr()
        a = jd.jd_attend_args_t()
        _ATTEND_ARGS.pack_into(a, 0, B, layer, at, t0, t1, t2, t3, t4, q.data_ptr(), o.data_ptr(), q_step, o_step, l_ptr,
                               self._scale if scale is None else scale, ATTEND_VARIANTS[variant] if isinstance(variant, str) else int(variant))
        st = self._lib.jd_cache_attend(self.h, a, _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_attend")
        return out

    def commit(self, accept_len: torch.Tensor, paths: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
               chosen: Optional[torch.Tensor] = None, path_len: Optional[int] = None, stream=None) -> torch.Tensor:
        """Keeps node 0 and the accepted nodes. accept_len [B] or [B, num_paths] (int32, as ``Verifier.verify`` returns it); paths
        [B, num_paths, path_len] nodes of the draft tokens along every path, None: a chain (path_len then bounds
        accept_len, default max_nodes - 1). Returns the number of the kept path of every sequence, [B]
        (entries of padding sequences stay as they were)."""
        if accept_len.dim() not in (1, 2):
            raise ValueError("accept_len: [B] or [B, num_paths]")
        B = accept_len.shape[0]
        n = accept_len.shape[1] if accept_len.dim() == 2 else 1
        if slots is not None:
            self._batch(slots, B)
        if paths is not None:
            if paths.dim() != 3 or paths.shape[0] != B or paths.shape[1] != n:
                raise ValueError("paths: [B, num_paths, path_len]")
            path_len = paths.shape[2]
        elif path_len is None:
            path_len = self.max_nodes - 1
        if chosen is None:
            chosen = self.seq_len.new_empty((B,))
        a = jd.jd_commit_args_t()
        _COMMIT_ARGS.pack_into(a, 0, B, _ints(slots, "slots", self.index), _ints(accept_len, "accept_len", self.index), n, path_len,
                               _ints(paths, "paths", self.index), _ints(chosen, "chosen", self.index, (B,)))
        st = self._lib.jd_cache_commit(self.h, a, _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_commit")
        return chosen

    def fork(self, src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
        """The empty slots dst[i] become copies of src[i] that share its pages until they part (``jd_cache_fork``)."""
        if src.dim() != 1 or src.shape != dst.shape:
            raise ValueError("src, dst: [n]")
        st = self._lib.jd_cache_fork(self.h, src.shape[0], _ints(src, "src", self.index), _ints(dst, "dst", self.index), _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_fork")

    def truncate(self, length: Optional[torch.Tensor], slots: Optional[torch.Tensor] = None, stream=None) -> None:
        """Cuts the sequences to length [B] tokens (None: 0); pages behind are released."""
        B = self._batch(slots, None if length is None else length.shape[0])
        st = self._lib.jd_cache_truncate(self.h, B, _ints(slots, "slots", self.index), _ints(length, "length", self.index, (B,)),
                                         _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_truncate")

    def free(self, slots: torch.Tensor, stream=None) -> None:
        """Empties slots."""
        if slots is None:
            raise ValueError("slots: which to empty")
        self.truncate(None, slots, stream)

    def compact(self, used: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Moves the pages in use to the front of the pool; returns their number, [1] (``jd_cache_compact``)."""
        if used is None:
            used = self.seq_len.new_empty((1,))
        st = self._lib.jd_cache_compact(self.h, _ints(used, "used", self.index, (1,)), _stream(stream, self.index))
        if st != jd.JD_OK:
            raise jd.JdError(st, "jd_cache_compact")
        return used

    def status(self) -> int:
        """Waits for the stream of the cache's last call (a replayed graph's stream is the caller's to wait for); the first device-side problem since the last query, or JD_OK."""
        out = C.c_int(0)
        _check(self._lib.jd_cache_last_status(self.h, C.byref(out)), "jd_cache_last_status")
        return out.value
