"""The candidate generator's operators: a paged cache of keys and values that the
candidates of a request share a prefix of, and the policy loss that learns from
the evaluator's scores.

A request's context is a prefix, its K candidate sequences a group that shares
it.  A step of the generator appends the new rows (`PagedKV.append`, which
rotates keys and queries by their position) and attends to prefix and own rows
(`PagedKV.attend`).  `policy_loss` turns logits, chosen tokens and advantages into
a loss and its gradient to the logits.

As in `binding`, arguments are checked and passed on: every computation runs in
the library's kernels, on the current stream unless `stream` (a
torch.cuda.Stream or its handle) says otherwise.  Nothing waits.  Outputs and
workspaces that are not passed in are allocated by torch for that stream.  Indices
in device memory are checked by the kernels, which report through `status`, a
CUDA int32 tensor of one element that the caller zeroes and `check_status` reads.
"""
from __future__ import annotations

import collections
import ctypes
import math

import torch

from . import binding as _b
from .binding import FeError, _check, load_library

_TYPES = {torch.bfloat16: _b.FE_IO_BF16, torch.float16: _b.FE_IO_F16, torch.float32: _b.FE_IO_F32}
_PAIRS = {"half": 0, "interleaved": 1}


def check_status(status) -> None:
    """Wait for `status` and raise FeError if a kernel reported anything."""
    st = int(status.item())
    if st & _b.FE_ST_TIMEOUT:
        raise FeError(_b.FE_ERR_TIMEOUT, "device-side wait timed out")
    if st & _b.FE_ST_INDEX:
        raise FeError(_b.FE_ERR_INDEX, "an index or length in device memory is out of range")
    if st & _b.FE_ST_NUMERIC:
        raise FeError(_b.FE_ERR_NUMERIC, "NaN")


def rotary_table(n_positions: int, rot_dim: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """[n_positions, rot_dim / 2, 2] fp32: cosine and sine of p base^(-2 i / rot_dim), computed in 64 bits."""
    inv = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    a = torch.arange(n_positions, dtype=torch.float64)[:, None] * inv
    return torch.stack([a.cos(), a.sin()], -1).to(torch.float32).to(device)


def _on(stream, device):
    """(handle, torch stream to allocate for or None) of a `stream` argument."""
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream, None
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    return stream.cuda_stream, stream


def _empty(on, make):
    if on is None:
        return make()
    with torch.cuda.stream(on):
        return make()


def _i32(name, t, shape, device):
    """The pointer of a contiguous int32 CUDA tensor; None in `shape` stands for any size."""
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor on {device}")
    if t.dim() != len(shape) or any(w is not None and n != w for n, w in zip(t.shape, shape)):
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    return t.data_ptr()


def _f32(name, t, n, device):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.device != device or not t.is_contiguous() or t.numel() != n:
        raise ValueError(f"{name} must be a contiguous float32 tensor of {n} elements on {device}")
    return t.data_ptr()


class PagedKV:
    """Keys and values in pages: two tensors [n_pages, kv_heads, page_rows, head_dim] of the caller's,
    bf16 or f16, page_rows 16, 32, 64 or 128, head_dim 32, 64 or 128.  Row c of a sequence is place
    c % page_rows of the page that entry c // page_rows of its page-table row names."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in _TYPES or k.device != v.device:
            raise ValueError("k and v must be [n_pages, kv_heads, page_rows, head_dim] of one type on one device")
        if not (k.is_cuda and k.is_contiguous() and v.is_contiguous()):
            raise ValueError("k and v must be contiguous CUDA tensors")
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        self.n_pages, self.kv_heads, self.page_rows, self.head_dim = k.shape
        self._kv = _b.FePagedKv(_TYPES[k.dtype], *k.shape[:1], k.shape[2], k.shape[1], k.shape[3], k.data_ptr(),
                                v.data_ptr())

    @classmethod
    def empty(cls, n_pages, page_rows, kv_heads, head_dim, dtype=torch.bfloat16, device="cuda"):
        shape = (n_pages, kv_heads, page_rows, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))

    def _rows(self, name, x, heads=None):
        if x.dim() != 3 or x.dtype != self.dtype or x.device != self.device or x.shape[2] != self.head_dim or (
                heads is not None and x.shape[1] != heads) or (x.stride(2) != 1 and x.numel() > 0):
            raise ValueError(f"{name} must be [rows, {heads or 'heads'}, {self.head_dim}] of {self.dtype} on "
                             f"{self.device}, its last dimension contiguous")
        return x.data_ptr()

    def append(self, k, v, row_start, first, pages, *, q=None, rope=None, pairs="half", shift=None, q_out=None,
               status=None, stream=None):
        """Append rows to paged sequences (fe_kv_append).

        k, v [rows, kv_heads, head_dim] (any row and head strides that keep 16-byte alignment): the rows
        row_start[s] .. row_start[s + 1] - 1 go to rows first[s], first[s] + 1, ... of sequence s, whose pages are
        pages[s].  With rope ([positions, rot_dim / 2, 2] fp32, see rotary_table) keys, and the queries
        q [rows, q_heads, head_dim] when given, are rotated at position shift[s] + first[s] + j; pairs: "half"
        or "interleaved".  Returns the rotated queries (q_out, contiguous), or None without q."""
        dev = self.device
        a = _b.FeAppendArgs(kv=self._kv)
        a.n_seqs, a.n_rows = first.shape[0], k.shape[0]
        a.k, a.v = self._rows("k", k, self.kv_heads), self._rows("v", v, self.kv_heads)
        if v.shape[0] != a.n_rows:
            raise ValueError("k and v must have as many rows")
        a.k_row, a.k_head, _ = k.stride()
        a.v_row, a.v_head, _ = v.stride()
        a.row_start = _i32("row_start", row_start, (a.n_seqs + 1,), dev)
        a.first = _i32("first", first, (a.n_seqs,), dev)
        a.pages = _i32("pages", pages, (a.n_seqs, None), dev)
        a.page_cols = pages.shape[1]
        if shift is not None:
            a.shift = _i32("shift", shift, (a.n_seqs,), dev)
        if pairs not in _PAIRS:
            raise ValueError("pairs must be 'half' or 'interleaved'")
        a.pairs = _PAIRS[pairs]
        if rope is not None:
            if rope.dim() != 3 or rope.shape[2] != 2:
                raise ValueError("rope must be [positions, rot_dim / 2, 2]")
            a.rope = _f32("rope", rope, rope.numel(), dev)
            a.rope_rows, a.rot_dim = rope.shape[0], 2 * rope.shape[1]
        if status is not None:
            a.status = _i32("status", status, (1,), dev)
        handle, on = _on(stream, dev)
        if q is not None:
            a.q, a.q_heads = self._rows("q", q), q.shape[1]
            if q.shape[0] != a.n_rows:
                raise ValueError("q and k must have as many rows")
            a.q_row, a.q_head, _ = q.stride()
            if q_out is None:
                q_out = _empty(on, lambda: torch.empty(q.shape, dtype=q.dtype, device=dev))
            elif q_out.shape != q.shape or not q_out.is_contiguous():
                raise ValueError("q_out must be contiguous and have q's shape")
            a.q_out = self._rows("q_out", q_out)
        _check(load_library().fe_kv_append(ctypes.byref(a), handle))
        return q_out if q is not None else None

    def attend(self, q, row_start, lengths, pages, group_start, prefix_lengths, prefix_pages, *, scale=None, out=None,
               with_lse=False, workspace=None, status=None, stream=None):
        """Attention of sequences that share a prefix (fe_prefix_attention).

        q [rows, q_heads, head_dim]: rows row_start[s] .. row_start[s + 1] - 1 are the last ones of the lengths[s] rows
        that sequence s holds in pages[s]; each sees the rows up to itself, and the prefix_lengths[g] rows in
        prefix_pages[g] of the group g with group_start[g] <= s < group_start[g + 1].  scale: 1 / sqrt(head_dim)
        unless given.  Returns out [rows, q_heads, head_dim], with with_lse (out, lse [rows, q_heads] fp32); a
        row that sees nothing gets 0 and -inf.  workspace: a uint8 tensor to use instead of a fresh one
        (workspace_bytes says how much); not to be shared by calls that may overlap."""
        dev = self.device
        a = _b.FePrefixArgs(kv=self._kv)
        a.n_groups, a.n_seqs, a.n_rows = prefix_lengths.shape[0], lengths.shape[0], q.shape[0]
        a.q, a.q_heads = self._rows("q", q), q.shape[1]
        a.q_row, a.q_head, _ = q.stride()
        a.row_start = _i32("row_start", row_start, (a.n_seqs + 1,), dev)
        a.seq_len = _i32("lengths", lengths, (a.n_seqs,), dev)
        a.pages = _i32("pages", pages, (a.n_seqs, None), dev)
        a.page_cols = pages.shape[1]
        a.group_start = _i32("group_start", group_start, (a.n_groups + 1,), dev)
        a.prefix_len = _i32("prefix_lengths", prefix_lengths, (a.n_groups,), dev)
        a.prefix_pages = _i32("prefix_pages", prefix_pages, (a.n_groups, None), dev)
        a.prefix_cols = prefix_pages.shape[1]
        a.scale = 1.0 / math.sqrt(self.head_dim) if scale is None else scale
        if status is not None:
            a.status = _i32("status", status, (1,), dev)
        handle, on = _on(stream, dev)
        if out is None:
            out = _empty(on, lambda: torch.empty(q.shape, dtype=q.dtype, device=dev))
        elif out.shape != q.shape or not out.is_contiguous():
            raise ValueError("out must be contiguous and have q's shape")
        a.out = self._rows("out", out)
        lse = None
        if with_lse:
            lse = _empty(on, lambda: torch.empty(q.shape[:2], dtype=torch.float32, device=dev))
            a.lse = lse.data_ptr()
        lib = load_library()
        if workspace is None:
            n = lib.fe_prefix_attention_workspace(ctypes.byref(a))
            workspace = _empty(on, lambda: torch.empty(n, dtype=torch.uint8, device=dev))
        elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}")
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
        _check(lib.fe_prefix_attention(ctypes.byref(a), handle))
        return (out, lse) if with_lse else out

    def workspace_bytes(self, n_groups: int, n_seqs: int, n_rows: int, q_heads: int) -> int:
        """Workspace of attend for these sizes."""
        one = self.k.data_ptr()  # (any pointer: only sizes count)
        a = _b.FePrefixArgs(kv=self._kv, n_groups=n_groups, n_seqs=n_seqs, n_rows=n_rows, q_heads=q_heads, prefix_cols=1,
                            page_cols=1, scale=1.0, group_start=one, prefix_len=one, prefix_pages=one, row_start=one,
                            seq_len=one, pages=one, q=one, out=one, q_row=8, q_head=8)
        n = load_library().fe_prefix_attention_workspace(ctypes.byref(a))
        if n == 0:
            raise FeError(_b.FE_ERR_INVALID_ARG, load_library().fe_last_error_message().decode())
        return int(n)


PolicyLoss = collections.namedtuple("PolicyLoss", "loss terms logp lse coef grad")
PolicyLoss.__doc__ = """Outputs of policy_loss: loss (a 0-d tensor), and per token the weighted term, log probability,
logsumexp and the slope of the loss to the log probability; grad [tokens, vocab] or None."""


def _policy_args(logits, tokens, weights, temperature, grad_scale, status):
    if logits.dim() != 2 or logits.dtype not in _TYPES or not logits.is_cuda or (logits.stride(1) != 1 and logits.shape[1] > 1):
        raise ValueError("logits must be a CUDA tensor [tokens, vocab] of bf16, f16 or fp32 with contiguous rows")
    T, V = logits.shape
    dev = logits.device
    a = _b.FePolicyArgs(dtype=_TYPES[logits.dtype], rows=T, vocab=V, temperature=temperature, grad_scale=grad_scale)
    a.logits, a.logits_row = logits.data_ptr(), logits.stride(0) if T > 1 else max(V, logits.stride(0))
    a.tokens = _i32("tokens", tokens, (T,), dev)
    a.weights = _f32("weights", weights, T, dev)
    if status is not None:
        a.status = _i32("status", status, (1,), dev)
    return a


def _policy_grad(a, logits, grad, on):
    if grad is None:  # rows as far apart as the logits': the same alignment
        grad = _empty(on, lambda: torch.empty_strided(logits.shape, (a.logits_row, 1), dtype=logits.dtype,
                                                      device=logits.device))
    elif grad.shape != logits.shape or grad.dtype != logits.dtype or grad.device != logits.device or (
            grad.stride(1) != 1 and grad.shape[1] > 1):
        raise ValueError("grad must have the logits' shape, type and device, and contiguous rows")
    a.grad, a.grad_row = grad.data_ptr(), grad.stride(0) if a.rows > 1 else max(a.vocab, grad.stride(0))
    return grad


def policy_loss(logits, tokens, advantages, weights=None, *, old_logp=None, ref_logp=None, clip=(0.2, 0.2), beta=0.0,
                temperature=1.0, with_grad=True, grad_scale=1.0, grad=None, status=None, stream=None) -> PolicyLoss:
    """Clipped policy loss with a KL term (fe_policy_loss), and its gradient to the logits.

    logits [tokens, vocab] bf16, f16 or fp32; tokens int32, -- the chosen ones; advantages, weights (1 / tokens each
    unless given; 0: the token takes no part), old_logp (None: the present policy's), ref_logp (None: no KL term)
    fp32.  clip: how far the ratio may go below and above 1; beta: the KL term's weight.  grad: where to
    write the gradient times grad_scale (may be logits itself)."""
    a = _policy_args(logits, tokens, weights, temperature, grad_scale, status)
    T, dev = a.rows, logits.device
    a.advantages = _f32("advantages", advantages, T, dev)
    a.old_logp = _f32("old_logp", old_logp, T, dev)
    a.ref_logp = _f32("ref_logp", ref_logp, T, dev)
    a.clip_low, a.clip_high = clip
    a.beta = beta
    handle, on = _on(stream, dev)
    grad = _policy_grad(a, logits, grad, on) if with_grad else None
    buf = _empty(on, lambda: torch.empty(4 * T + 1, dtype=torch.float32, device=dev))
    at = buf.data_ptr()
    a.loss, a.terms, a.logp, a.lse, a.coef = at, at + 4, at + 4 + 4 * T, at + 4 + 8 * T, at + 4 + 12 * T
    _check(load_library().fe_policy_loss(ctypes.byref(a), handle))
    return PolicyLoss(buf[0], *buf[1:].view(4, T).unbind(0), grad)


def policy_loss_backward(logits, tokens, result: PolicyLoss, weights=None, *, upstream=None, temperature=1.0,
                         grad_scale=1.0, grad=None, status=None, stream=None):
    """The gradient to the logits from an earlier policy_loss (with_grad=False) on the same tokens, weights and
    temperature, times upstream (a CUDA fp32 tensor of one element; None: 1) and grad_scale."""
    a = _policy_args(logits, tokens, weights, temperature, grad_scale, status)
    dev = logits.device
    a.lse, a.coef = _f32("lse", result.lse, a.rows, dev), _f32("coef", result.coef, a.rows, dev)
    up = _f32("upstream", upstream, 1, dev)
    handle, on = _on(stream, dev)
    grad = _policy_grad(a, logits, grad, on)
    _check(load_library().fe_policy_loss_backward(ctypes.byref(a), up, handle))
    return grad
