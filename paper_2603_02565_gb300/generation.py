"""The candidate generator's operators: a paged cache of keys and values that the
candidates of a request share a prefix of, and the policy loss that learns from
the evaluator's scores.

A request's context is a prefix, its K candidate sequences a group that shares
it.  A step of the generator appends the new rows (`PagedKV.append`, which
rotates keys and queries by their position) and attends to prefix and own rows
(`PagedKV.attend`).  `policy_loss` turns logits, chosen tokens and advantages into
a loss and its gradient to the logits.

As in `binding`, arguments are checked and passed on: every computation runs in
the library's kernels, on the tensors' device, whichever is current, and its
current stream unless `stream` (a torch.cuda.Stream of that device or its handle)
says otherwise.  Nothing waits.  Outputs and
workspaces that are not passed in are allocated by torch for that stream; only
attend's workspace is kept.  Indices
in device memory are checked by the kernels, which report through `status`, a
CUDA int32 tensor of one element that the caller zeroes and `check_status` reads.
"""
from __future__ import annotations

import math
import struct
import threading
import warnings
import weakref

import torch

from . import binding as _b
from .binding import FeError, _check, load_library

_TYPES = {torch.bfloat16: _b.FE_IO_BF16, torch.float16: _b.FE_IO_F16, torch.float32: _b.FE_IO_F32}
_PAIRS = {"half": 0, "interleaved": 1}
# The argument structures of fe.h, fields in their order.  (A call of a few microseconds on the GPU is worth a lean
# one here: packing all fields at once takes a tenth of the time that setting them one by one does.)
_APPEND = struct.Struct("@5i2P8i7P6q3P")
_PREFIX = struct.Struct("@5i2P6ifi7P2q3PQP")
_POLICY = struct.Struct("@3i5fP2q12P")
_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        _LIB = load_library()
    return _LIB


def check_status(status) -> None:
    """Wait for `status` and raise FeError if a kernel reported anything."""
    st = int(status.item())
    if st & _b.FE_ST_TIMEOUT:
        raise FeError(_b.FE_ERR_TIMEOUT, "device-side wait timed out")
    if st & _b.FE_ST_INDEX:
        raise FeError(_b.FE_ERR_INDEX, "an index or length in device memory is out of range")


def rotary_table(n_positions: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """[n_positions, rot_dim / 2, 2] fp32: cosine and sine of p base^(-2 i / rot_dim), computed in 64 bits."""
    inv = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    a = torch.arange(n_positions, dtype=torch.float64)[:, None] * inv
    return torch.stack([a.cos(), a.sin()], -1).to(torch.float32).to(device)


# the current stream's handle by device index, without a stream object where torch offers that
_current = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_capturing = torch.cuda.is_current_stream_capturing


def _on_device(index, entry):
    """`entry`, called with CUDA device `index` current: the library's calls, and what torch says of the current stream,
    are that device's."""
    if index == _current_device():
        return entry

    def call(*args):
        with torch.cuda.device(index):
            return entry(*args)
    return call


def _cut_off(name):
    """Called where tensors of a call require a gradient."""
    if torch.is_grad_enabled():
        warnings.warn(f"{name} has no backward: its results are cut off from tensors that require a gradient (call it "
                      "under torch.no_grad(), or with detached tensors)", stacklevel=3)


def _stream_of(stream, index):
    """(handle, torch stream to allocate for; None: the current one) of a `stream` argument."""
    if stream is None:
        return _current(index), None
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=index)
    elif stream.device_index != index:
        raise ValueError(f"stream is one of cuda:{stream.device_index}, the tensors are on cuda:{index}")
    return stream.cuda_stream, stream


def _captured(on, index):
    """Whether calls on stream `on` (None: the current one of device `index`) are being captured."""
    if on is None:
        return _on_device(index, _capturing)()
    with torch.cuda.stream(on):
        return _capturing()


class _Kept(threading.local):
    """A PagedKV's workspaces by stream, each thread's its own: they go with the thread."""

    def __init__(self):
        self.spaces = {}


class _Shared(threading.local):
    """The same by device and stream over all PagedKV, as long as one of them keeps them: a model's layers share one."""

    def __init__(self):
        self.spaces = weakref.WeakValueDictionary()


_shared = _Shared()


def _like(t, on):
    """A contiguous tensor of t's shape and type, allocated for stream `on`."""
    if on is None:
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    with torch.cuda.stream(on):
        return torch.empty_like(t, memory_format=torch.contiguous_format)


def _new(t, shape, on, dtype=None):
    if on is None:
        return torch.empty(shape, dtype=dtype or t.dtype, device=t.device)
    with torch.cuda.stream(on):
        return torch.empty(shape, dtype=dtype or t.dtype, device=t.device)


def _i32(name, t, n, index):
    """The pointer of a contiguous int32 tensor [n] on CUDA device `index`."""
    if t.dtype is not torch.int32 or t.shape != (n,) or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor [{n}] on cuda:{index}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _table(name, t, n, index):
    """(pointer, columns) of a contiguous int32 table [n, columns]."""
    if t.dtype is not torch.int32 or t.dim() != 2 or t.get_device() != index or not t.is_contiguous() or t.shape[0] != n:
        raise ValueError(f"{name} must be a contiguous int32 tensor [{n}, columns] on cuda:{index}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr(), t.shape[1]


def _f32(name, t, n, index):
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.get_device() != index or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{name} must be a contiguous float32 tensor of {n} elements on cuda:{index}")
    return t.data_ptr()


def _status(status, index):
    return 0 if status is None else _i32("status", status, 1, index)


class PagedKV:
    """Keys and values in pages: two tensors [n_pages, kv_heads, page_rows, head_dim] of the caller's,
    bf16 or f16, page_rows 16, 32, 64 or 128, head_dim 32, 64 or 128.  Row c of a sequence is place
    c % page_rows of the page that entry c // page_rows of its page-table row names."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("k and v must be [n_pages, kv_heads, page_rows, head_dim], both bf16 or both f16")
        if not (k.is_cuda and k.device == v.device and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("k and v must be contiguous CUDA tensors on one device")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self.n_pages, self.kv_heads, self.page_rows, self.head_dim = k.shape
        self._index = k.get_device()
        self._fields = (_TYPES[k.dtype], self.n_pages, self.page_rows, self.kv_heads, self.head_dim, k.data_ptr(),
                        v.data_ptr())
        self._scale = 1.0 / math.sqrt(self.head_dim)
        self._kept = _Kept()

    @classmethod
    def empty(cls, n_pages, page_rows, kv_heads, head_dim, dtype=torch.bfloat16, device="cuda"):
        shape = (n_pages, kv_heads, page_rows, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))

    def _rows(self, name, x, n, heads=None):
        """(pointer, heads, row stride, head stride) of rows [n, heads, head_dim]."""
        if x.dim() == 3 and x.dtype is self.dtype and x.get_device() == self._index:
            rows, h, d = x.shape
            row, head, one = x.stride()
            if rows == n and d == self.head_dim and (one == 1 or rows == 0) and (heads is None or h == heads):
                return x.data_ptr(), h, row, head
        raise ValueError(f"{name} must be [{n}, {heads or 'heads'}, {self.head_dim}] of {self.dtype} on {self.device}, "
                         f"its last dimension contiguous; got {x.dtype} {tuple(x.shape)} on {x.device}")

    def _out(self, name, x, like):
        if x.shape != like.shape or x.dtype is not like.dtype or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous, with q's shape, type and device")
        return x

    def append(self, k, v, row_start, first, pages, *, q=None, rope=None, pairs="half", shift=None, q_out=None,
               status=None, stream=None):
        """Append rows to paged sequences (fe_kv_append).

        k, v [rows, kv_heads, head_dim] (any row and head strides that keep 16-byte alignment): the rows
        row_start[s] .. row_start[s + 1] - 1 go to rows first[s], first[s] + 1, ... of sequence s, whose pages are
        pages[s].  With rope ([positions, rot_dim / 2, 2] fp32, see rotary_table) keys, and the queries
        q [rows, q_heads, head_dim] when given, are rotated at position shift[s] + first[s] + j; pairs: "half"
        or "interleaved".  Returns the rotated queries (q_out, contiguous), or None without q.  There is no backward."""
        dev = self._index
        S, T = first.shape[0], k.shape[0]
        kp, _, k_row, k_head = self._rows("k", k, T, self.kv_heads)
        vp, _, v_row, v_head = self._rows("v", v, T, self.kv_heads)
        if k.requires_grad or v.requires_grad or (q is not None and q.requires_grad):
            _cut_off("append")
        if pairs not in _PAIRS:
            raise ValueError("pairs must be 'half' or 'interleaved'")
        rope_p = rope_rows = rot = 0
        if rope is not None:
            if rope.dim() != 3 or rope.shape[2] != 2:
                raise ValueError("rope must be [positions, rot_dim / 2, 2]")
            rope_rows, half, _ = rope.shape
            rot = 2 * half
            rope_p = _f32("rope", rope, rope_rows * rot, dev)
        table, cols = _table("pages", pages, S, dev)
        handle, on = _stream_of(stream, dev)
        qp = hq = q_row = q_head = out_p = 0
        if q is not None:
            qp, hq, q_row, q_head = self._rows("q", q, T)
            q_out = _like(q, on) if q_out is None else self._out("q_out", q_out, q)
            out_p = q_out.data_ptr()
        rc = _on_device(dev, _lib().fe_kv_append)(_APPEND.pack(
            *self._fields, S, T, cols, hq, rope_rows, rot, _PAIRS[pairs], 0, _i32("row_start", row_start, S + 1, dev),
            _i32("first", first, S, dev), 0 if shift is None else _i32("shift", shift, S, dev), table, kp, vp, qp, k_row,
            k_head, v_row, v_head, q_row, q_head, out_p, rope_p, _status(status, dev)), handle)
        if rc:
            _check(rc)
        return q_out if q is not None else None

    def attend(self, q, row_start, lengths, pages, group_start, prefix_lengths, prefix_pages, *, scale=None, out=None,
               with_lse=False, workspace=None, status=None, stream=None):
        """Attention of sequences that share a prefix (fe_prefix_attention).

        q [rows, q_heads, head_dim]: rows row_start[s] .. row_start[s + 1] - 1 are the last ones of the lengths[s] rows
        that sequence s holds in pages[s]; each sees the rows up to itself, and the prefix_lengths[g] rows in
        prefix_pages[g] of the group g with group_start[g] <= s < group_start[g + 1].  scale: 1 / sqrt(head_dim)
        unless given.  Returns out [rows, q_heads, head_dim], with with_lse (out, lse [rows, q_heads] fp32); a
        row that sees nothing gets 0 and -inf.  workspace: a uint8 tensor to use instead of the one that is kept for
        each thread and stream, for all PagedKV of a device (workspace_bytes says how much); not to be shared by calls
        that may overlap.  There is no backward."""
        dev = self._index
        G, S, T = prefix_lengths.shape[0], lengths.shape[0], q.shape[0]
        qp, hq, q_row, q_head = self._rows("q", q, T)
        if q.requires_grad or self.k.requires_grad or self.v.requires_grad:
            _cut_off("attend")
        table, cols = _table("pages", pages, S, dev)
        pre_table, pre_cols = _table("prefix_pages", prefix_pages, G, dev)
        handle, on = _stream_of(stream, dev)
        out = _like(q, on) if out is None else self._out("out", out, q)
        lse = _new(q, (T, hq), on, torch.float32) if with_lse else None
        if workspace is None:
            # A thread's calls on a stream run one after another and share a workspace (another thread's kernels could
            # come between the three of a call); a call that is being captured has one of its own, in the graph's memory.
            keep = None if _captured(on, dev) else handle
            workspace = self._kept.spaces.get(keep)
            if workspace is None:
                workspace = self._workspace(keep, G, S, T, hq, q, on)
        elif workspace.dtype is not torch.uint8 or workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {self.device}")
        else:
            keep = None
        entry = _on_device(dev, _lib().fe_prefix_attention)
        while True:
            rc = entry(_PREFIX.pack(
                *self._fields, G, S, T, hq, pre_cols, cols, self._scale if scale is None else scale, 0,
                _i32("group_start", group_start, G + 1, dev), _i32("prefix_lengths", prefix_lengths, G, dev), pre_table,
                _i32("row_start", row_start, S + 1, dev), _i32("lengths", lengths, S, dev), table, qp, q_row, q_head,
                out.data_ptr(), 0 if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.numel(),
                _status(status, dev)), handle)
            if rc == 0:
                break
            if rc != _b.FE_ERR_WORKSPACE or keep is None:
                _check(rc)
            # the kept workspace is one of smaller calls (nothing has been enqueued)
            workspace, keep = self._workspace(keep, G, S, T, hq, q, on), None
        return (out, lse) if with_lse else out

    _spaces = property(lambda self: self._kept.spaces)  # this thread's workspaces by stream handle

    def _workspace(self, keep, G, S, T, hq, q, on):
        """A workspace for a call of these sizes, to be kept for the stream with handle `keep` unless that is None."""
        need = self.workspace_bytes(G, S, T, hq)
        if keep is None:
            return _new(q, need, on, torch.uint8)
        workspace = _shared.spaces.get((self._index, keep))
        if workspace is None or workspace.numel() < need:
            workspace = _shared.spaces[self._index, keep] = _new(q, need, on, torch.uint8)
        self._spaces[keep] = workspace
        return workspace

    def workspace_bytes(self, n_groups: int, n_seqs: int, n_rows: int, q_heads: int) -> int:
        """Workspace of attend for these sizes."""
        at = self._fields[5]  # (any pointer: only sizes count)
        n = _on_device(self._index, _lib().fe_prefix_attention_workspace)(_PREFIX.pack(
            *self._fields, n_groups, n_seqs, n_rows, q_heads, 1, 1, 1.0, 0, at, at, at, at, at, at, at, 8, 8, at + 32, 0, 0, 0,
            0))
        if n == 0:
            raise FeError(_b.FE_ERR_INVALID_ARG, _lib().fe_last_error_message().decode())
        return int(n)


class PolicyLoss:
    """Outputs of policy_loss: loss (a 0-d tensor), and per token terms (the weighted summands), logp (log
    probability), lse (logsumexp) and coef (the slope of the loss to logp), all fp32; grad [tokens, vocab] or None."""

    __slots__ = ("_stats", "_tokens", "grad")

    def __init__(self, stats, tokens, grad):
        self._stats, self._tokens, self.grad = stats, tokens, grad  # [1 + 4 tokens]: the loss, then the four rows

    def _row(self, i):
        return self._stats.narrow(0, 1 + i * self._tokens, self._tokens)

    loss = property(lambda self: self._stats.select(0, 0))
    terms = property(lambda self: self._row(0))
    logp = property(lambda self: self._row(1))
    lse = property(lambda self: self._row(2))
    coef = property(lambda self: self._row(3))


def _logits(logits):
    """(tokens, vocab, type, device index, row stride) of logits."""
    if logits.dim() == 2 and logits.is_cuda and logits.dtype in _TYPES:
        T, V = logits.shape
        row, one = logits.stride()
        if one == 1 or V <= 1:
            return T, V, _TYPES[logits.dtype], logits.get_device(), row if T > 1 else max(V, row)
    raise ValueError("logits must be a CUDA tensor [tokens, vocab] of bf16, f16 or fp32 with contiguous rows")


def _grad(logits, row, grad, on):
    """(tensor, row stride) of the gradient: a new one has its rows as far apart as the logits', and as far off a
    16-byte boundary (so they leave the kernels in whole pieces)."""
    T, V = logits.shape
    if grad is None:
        off = logits.data_ptr() % 16 // logits.element_size()
        if off == 0 and logits.is_contiguous():
            return _like(logits, on), row
        return _new(logits, off + max(0, (T - 1) * row + V), on).as_strided((T, V), (row, 1), off), row
    if grad.shape != logits.shape or grad.dtype is not logits.dtype or grad.get_device() != logits.get_device() or (
            grad.stride(1) != 1 and V > 1):
        raise ValueError("grad must have the logits' shape, type and device, and contiguous rows")
    return grad, grad.stride(0) if T > 1 else max(V, grad.stride(0))


def policy_loss(logits, tokens, advantages, weights=None, *, old_logp=None, ref_logp=None, clip=(0.2, 0.2), beta=0.0,
                temperature=1.0, with_grad=True, grad_scale=1.0, grad=None, status=None, stream=None) -> PolicyLoss:
    """Clipped policy loss with a KL term (fe_policy_loss), and its gradient to the logits.

    logits [tokens, vocab] bf16, f16 or fp32; tokens int32, the chosen ones; advantages, weights (1 / tokens each
    unless given; 0: the token takes no part), old_logp (None: the present policy's), ref_logp (None: no KL term)
    fp32.  clip: how far the ratio may go below and above 1; beta: the KL term's weight.  grad: where to
    write the gradient times grad_scale (may be logits itself)."""
    T, V, dtype, dev, row = _logits(logits)
    handle, on = _stream_of(stream, dev)
    grad_p = grad_row = 0
    if with_grad:
        grad, grad_row = _grad(logits, row, grad, on)
        grad_p = grad.data_ptr()
    else:
        grad = None
    stats = _new(logits, 4 * T + 1, on, torch.float32)
    at, n = stats.data_ptr(), 4 * T
    rc = _on_device(dev, _lib().fe_policy_loss)(_POLICY.pack(
        dtype, T, V, clip[0], clip[1], beta, temperature, grad_scale, logits.data_ptr(), row, grad_row,
        _i32("tokens", tokens, T, dev), _f32("advantages", advantages, T, dev), _f32("weights", weights, T, dev),
        _f32("old_logp", old_logp, T, dev), _f32("ref_logp", ref_logp, T, dev), at, at + 4, at + 4 + n, at + 4 + 2 * n,
        at + 4 + 3 * n, grad_p, _status(status, dev)), handle)
    if rc:
        _check(rc)
    return PolicyLoss(stats, T, grad)


def policy_loss_backward(logits, tokens, result: PolicyLoss, weights=None, *, upstream=None, temperature=1.0,
                         grad_scale=1.0, grad=None, status=None, stream=None):
    """The gradient to the logits from an earlier policy_loss (with_grad=False) on the same tokens, weights and
    temperature, times upstream (a CUDA fp32 tensor of one element; None: 1) and grad_scale."""
    T, V, dtype, dev, row = _logits(logits)
    handle, on = _stream_of(stream, dev)
    grad, grad_row = _grad(logits, row, grad, on)
    rc = _on_device(dev, _lib().fe_policy_loss_backward)(_POLICY.pack(
        dtype, T, V, 0.0, 0.0, 0.0, temperature, grad_scale, logits.data_ptr(), row, grad_row,
        _i32("tokens", tokens, T, dev), 0, _f32("weights", weights, T, dev), 0, 0, 0, 0, 0,
        _f32("lse", result.lse, T, dev), _f32("coef", result.coef, T, dev), grad.data_ptr(), _status(status, dev)),
        _f32("upstream", upstream, 1, dev), handle)
    if rc:
        _check(rc)
    return grad
