"""verify_drafts: which drafted tokens stay, and the token behind them.  Computed in the library's kernels; PyTorch is used for device
memory and streams only."""
from __future__ import annotations

import struct

import torch

from . import binding as B

# rr_verify_args as bytes
_VERIFY = struct.Struct("@11P2q4i")

_DTYPES = {torch.bfloat16: B.RR_BF16, torch.float32: B.RR_F32}


def _tensor(t, name, dtype, shape, index):
    """t is a contiguous tensor of this type, shape and device; its address."""
    if t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be contiguous {dtype} {tuple(shape)} on cuda:{index}, not {t.dtype} {tuple(t.shape)} on {t.device}"
                     + ("" if t.is_contiguous() else " (not contiguous)"))


def _rows(t, name, dtype, shape, index):
    """t has this type, shape and device and contiguous rows; its row stride."""
    apart, side = t.stride()
    if t.dtype is dtype and t.get_device() == index and side == 1 and not t.requires_grad and t.shape == shape:
        return apart
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which the verification does not have: call it under torch.no_grad()")
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on cuda:{index}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    if shape[1] > 1 and shape[0] > 0 and side != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    return apart


def verify_drafts(target: torch.Tensor, tokens: torch.Tensor, cu: torch.Tensor | None = None, *, draft: torch.Tensor | None = None,
                  uniform: torch.Tensor | None = None, lens: torch.Tensor | None = None, new_lens: torch.Tensor | None = None,
                  status: torch.Tensor | None = None, room: torch.Tensor | None = None) -> "tuple[torch.Tensor, torch.Tensor]":
    """Verifies the drafted tokens of a step.  Sequence b owns the rows cu[b] .. cu[b + 1] - 1: its last known token and the drafts behind it;
    rows behind cu[batch] are padding.  Returns (next, accepted):
        next      [rows] int32: the token that follows each row: the accepted drafts, one token more, then -1 (padding: not written)
        accepted  [batch] int32: how many drafts were accepted
    target    [rows, vocab] bf16 or fp32 (rows contiguous, any row stride): what the target predicts behind each row's token
    tokens    [rows] int32
    cu        [batch + 1] int32; None: one row per sequence, no drafts
    uniform   [rows] float32 in [0, 1): target and draft hold probabilities.  Draft x behind row t is accepted if
              target[t, x] > uniform[t] * draft[t, x]; the token more is drawn by the sequence's last random number, from max(target - draft, 0) of
              the row that was rejected or from the last row of the target.  The tokens are then distributed as the target's.
              None: greedy; target holds scores, a draft is accepted if it is its row's best (the lowest of several), the token more is the next row's best
    draft     [rows, vocab] as target: row t is what tokens[t + 1] was drawn from (a sequence's last row is not read); None: the draft's
              probability was 1
    new_lens  [batch] int32: gets lens + accepted + 1, the tokens that stay of sequences that had lens tokens before the step's rows were
              appended (may be lens itself, else memory of its own): what PagePool.reserve takes next
    status    [1] int32: RR_STATUS_BAD_INDEX is OR-ed into it if a drafted token is outside the vocabulary (it is rejected)
    room      [batch] int32, PagePool.room, with lens: a sequence whose rows had no room, so that they were not appended, has accepted = -1 and keeps its lens; its
              next tokens are not to be used
    Work goes to the current stream of target's device.  No gradient."""
    if target.dim() != 2 or tokens.dim() != 1:
        raise ValueError("target must be [rows, vocab] and tokens [rows]")
    code, index = _DTYPES.get(target.dtype), target.get_device()
    if code is None:
        raise TypeError(f"target must be bfloat16 or float32, not {target.dtype}")
    if index < 0:
        raise ValueError("target must be on a CUDA device (there is no CPU path)")
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return verify_drafts(target, tokens, cu, draft=draft, uniform=uniform, lens=lens, new_lens=new_lens, status=status, room=room)
    rows, vocab = shape = tuple(target.shape)
    stride = _rows(target, "target", target.dtype, shape, index)
    i32, one = torch.int32, (rows,)
    p_tokens = _tensor(tokens, "tokens", i32, one, index)
    p_cu = p_draft = p_uniform = p_lens = p_new = p_status = p_room = draft_stride = 0
    batch = rows
    if cu is not None:
        batch = cu.shape[0] - 1 if cu.dim() == 1 else 0
        if batch < 1:
            raise ValueError("cu must be [batch + 1]")
        p_cu = _tensor(cu, "cu", i32, (batch + 1,), index)
    elif rows == 0:
        raise ValueError("no rows")
    if uniform is not None:
        p_uniform = _tensor(uniform, "uniform", torch.float32, one, index)
        if draft is not None:
            if draft.dim() != 2:
                raise ValueError("draft must be [rows, vocab]")
            draft_stride = _rows(draft, "draft", target.dtype, shape, index)
            p_draft = draft.data_ptr()
    elif draft is not None:
        raise ValueError("draft without uniform: greedy verification has no probabilities")
    if lens is not None:
        p_lens = _tensor(lens, "lens", i32, (batch,), index)
    if new_lens is not None:
        if lens is None:
            raise ValueError("new_lens without lens")
        p_new = _tensor(new_lens, "new_lens", i32, (batch,), index)
    if status is not None:
        p_status = _tensor(status, "status", i32, (1,), index)
    if room is not None:
        if lens is None:
            raise ValueError("room without lens")
        p_room = _tensor(room, "room", i32, (batch,), index)
    after = torch.empty_like(tokens)
    accepted = tokens.new_empty((batch,)) if lens is None else torch.empty_like(lens)
    if rows == 0:                                      # (an empty tensor has no address, and nothing is read)
        p_tokens = p_out = p_cu
        p_uniform = p_draft = 0
    else:
        p_out = after.data_ptr()
    rc = B.lib().rr_verify_drafts(_VERIFY.pack(target.data_ptr(), p_draft, p_tokens, p_cu, p_uniform, p_lens, p_out, accepted.data_ptr(), p_new, p_status, p_room,
                                               stride, draft_stride, code, rows, batch, vocab),
                                  torch._C._cuda_getCurrentRawStream(index))
    if rc != B.RR_OK:
        raise B.RouteRelayError(rc, "rr_verify_drafts")
    return after, accepted
