"""Verification of drafted tokens against probabilities that are there already, from given random numbers (``jd_verify_probs``): chains
and, by sampling, trees.  Where the target's hidden states are at hand instead, ``Verifier.verify`` forms the probabilities itself."""
from __future__ import annotations

import struct
from typing import Optional

import torch

from . import jd
from .cache import _DTYPES, _has_tangent, _fw, _raw_stream

SIBLINGS = {"independent": jd.JD_SIBLINGS_INDEPENDENT, "distinct": jd.JD_SIBLINGS_DISTINCT}
_ARGS = struct.Struct("@iiiiPPqqPPiPPPPfiiiPPPP")


def _rows(x: torch.Tensor, name: str, shape, dtype, index: int) -> int:
    """Elements between rows (0: dense) of [B, n, V] whose rows lie evenly."""
    if x.shape != shape or x.dtype is not dtype or x.get_device() != index:
        raise ValueError("%s: %s of one type with target, on its device" % (name, list(shape)))
    if x.requires_grad and torch.is_grad_enabled() or _fw._current_level >= 0 and _has_tangent(x):
        raise ValueError("%s: no autograd here; detach it" % name)
    if x.is_contiguous():
        return 0
    B, n, V = shape
    sb, sn, sv = x.stride()
    step = sn if n > 1 else sb
    if (V > 1 and sv != 1) or (B > 1 and n > 1 and sb != n * sn):
        raise ValueError("%s: rows of neighbouring entries, evenly spaced" % name)
    if B * n > 1 and step < V:                # a broadcast among them: its step of 0 would stand for dense
        raise ValueError("%s: rows must not overlap" % name)
    return step if B * n > 1 else 0


def _plain(x: torch.Tensor, name: str, shape, dtype, index: int) -> int:
    if x.shape != shape or x.dtype is not dtype or x.get_device() != index or not x.is_contiguous():
        raise ValueError("%s: a contiguous %s tensor of shape %s on the target's device" % (name, dtype, list(shape)))
    return x.data_ptr()


def verify_probs(target: torch.Tensor, draft: Optional[torch.Tensor], tokens: torch.Tensor, accept_u: torch.Tensor, sample_u: torch.Tensor,
                 parents: Optional[torch.Tensor] = None, num_nodes: Optional[torch.Tensor] = None, judge_scores: Optional[torch.Tensor] = None,
                 tau: float = 0.5, mode="standard", resample="residual", siblings="independent", out: Optional[dict] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> dict:
    """Accepts drafted tokens and draws the next one. target [B, T, V] (float32 or bfloat16): probabilities behind node 0, the last context
    token, and behind each of the T - 1 drafted tokens; draft [B, T - 1, V]: the distributions that the children of each node were drawn from
    (row i: of node i); tokens [B, T - 1] (int32); accept_u [B, T - 1] and sample_u [B]: uniform float32 numbers of [0, 1). parents [T] or [B, T]
    (int32, a parent before its children): trees, None: chains; ``siblings``: whether children of a node were drawn "independent" of one another or
    "distinct" (without replacement). judge_scores [B, T - 1] and tau as in ``Verifier.verify``, read by the modes that judge. num_nodes [B]: nodes of
    each sequence of a padded batch (0: its outputs stay as they were, -1 in those that the call makes; ``commit`` leaves the sequence out by slot -1). Returns (and takes as ``out``) a dict with "accept_len" [B],
    "next_token" [B] and "path" [B, T - 1], the nodes of the accepted tokens, -1 behind them: ``cache.commit(out["accept_len"][:, None],
    out["path"][:, None])``. status: int32 [1] that becomes the first problem (a token or parent out of range) if it holds 0.
    All tensors on one device; enqueued on ``stream`` (default: the current one), where tensors that the call makes are allocated."""
    if target.dim() != 3 or target.dtype not in _DTYPES or not target.is_cuda:
        raise ValueError("target: [B, T, V], float32 or bfloat16, on the device")
    B, T, V = target.shape
    index, i32, f32, dt = target.get_device(), torch.int32, torch.float32, target.dtype
    M = T - 1
    t_step = _rows(target, "target", (B, T, V), dt, index)
    if draft is None and M > 0:
        raise ValueError("draft: [B, T - 1, V]")
    d_step = 0 if M <= 0 else _rows(draft, "draft", (B, M, V), dt, index)
    if parents is not None and (parents.dtype is not i32 or parents.get_device() != index or not parents.is_contiguous() or
                                parents.shape not in ((T,), (B, T))):
        raise ValueError("parents: contiguous int32 [T] or [B, T] on the target's device")
    if out is None:
        # parts of one allocation, cut in one call: 2 us where slices take 1.4 each
        flat = tokens.new_empty((B * (M + 2),))
        if num_nodes is not None:      # where there are no nodes nothing is written: -1, on the call's stream
            if stream is None:
                flat.fill_(-1)
            else:
                with torch.cuda.stream(stream):
                    flat.fill_(-1)
        length, token, path = flat.unsafe_split_with_sizes((B, B, B * M))
        out = dict(accept_len=length, next_token=token, path=path.view(B, M))
        len_ptr = flat.data_ptr()
        next_ptr, path_ptr = len_ptr + 4 * B, len_ptr + 8 * B
    else:
        path = out.get("path")
        len_ptr, next_ptr = _plain(out["accept_len"], "accept_len", (B,), i32, index), _plain(out["next_token"], "next_token", (B,), i32, index)
        path_ptr = 0 if path is None else _plain(path, "path", (B, M), i32, index)
    mode = jd.MODES[mode] if isinstance(mode, str) else int(mode)
    if mode != jd.JD_MODE_STANDARD and judge_scores is None:
        raise ValueError("judge_scores: [B, T - 1] for a mode that judges")
    a = jd.jd_verify_probs_args_t()
    bm = (B, M)
    _ARGS.pack_into(a, 0, B, T, V, _DTYPES[dt], target.data_ptr(), 0 if M <= 0 else draft.data_ptr(), t_step, d_step,
                    _plain(tokens, "tokens", bm, i32, index), 0 if parents is None else parents.data_ptr(),
                    1 if parents is not None and parents.dim() == 2 else 0,
                    0 if num_nodes is None else _plain(num_nodes, "num_nodes", (B,), i32, index),
                    _plain(accept_u, "accept_u", bm, f32, index), _plain(sample_u, "sample_u", (B,), f32, index),
                    0 if judge_scores is None else _plain(judge_scores, "judge_scores", bm, f32, index), tau, mode,
                    jd.RESAMPLE[resample] if isinstance(resample, str) else int(resample),
                    SIBLINGS[siblings] if isinstance(siblings, str) else int(siblings), len_ptr, next_ptr, path_ptr,
                    0 if status is None else _plain(status, "status", (1,), i32, index))
    lib = jd.load()
    if torch._C._cuda_getDevice() == index:
        st = lib.jd_verify_probs(a, stream.cuda_stream if stream is not None else _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = lib.jd_verify_probs(a, stream.cuda_stream if stream is not None else _raw_stream(index))
    if st != jd.JD_OK:
        raise jd.JdError(st, "jd_verify_probs")
    return out
