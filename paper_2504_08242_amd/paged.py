"""ctypes front end of the paged-cache operators (see include/jupiter_paged.h): keys and values in pages of one pool.

A pool is two tensors ``k_pool`` and ``v_pool`` [n_blocks, n_kv_heads, page_size, head_dim] (one layer each; any strides
whose last is 1, the same for both), a block table an int32 tensor [n_requests, width], a ragged batch a tensor of rows with
``row_start`` [n_requests + 1].  One step::

    step = extend(lengths, n_new, owned, table, free_blocks, free_count, page_size, max_rows)
    for layer in ...:
        q = append(k, v, step.slots, k_pool, v_pool, positions=step.positions, rope_theta=1e4, q=q)
        out = attention(q, k_pool, v_pool, table, step.row_start, step.lengths, max_new, workspace)
    verdict = verify(tokens, target_probs, step.row_start, u_accept, u_sample, workspace, lengths=lengths)

Argument marshalling only: every operator is a HIP kernel of the library.  The calls are asynchronous on ``stream`` (default: the
current one of the tensors' device) and read nothing back.  ``ValueError`` for tensors that do not fit together,
``binding.JupiterError`` for what the library refuses.
"""
import collections
import ctypes
import math

import torch

from . import binding as jb

_i32, _i64, _f32, _vp, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t


class _Pool(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("block_stride", _i64), ("head_stride", _i64), ("slot_stride", _i64), ("n_blocks", _i32),
                ("page_size", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32)]


class _Extend(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_seqs", "page_size", "table_width", "n_free", "max_rows")] + [("table_stride", _i64)] + [
        (n, _vp) for n in ("lengths", "n_new", "owned", "table", "free_blocks", "free_count", "row_start", "positions", "slots",
                           "new_lengths", "new_owned", "new_free_count", "status")]


class _Append(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("n_heads", _i32), ("q", _vp), ("k", _vp), ("v", _vp), ("q_out", _vp)] + [
        (n, _i64) for n in ("q_row_stride", "q_head_stride", "k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride",
                            "q_out_row_stride", "q_out_head_stride")] + [("positions", _vp), ("slots", _vp), ("rope_theta", _f32)]


class _Attention(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_seqs", "n_rows", "n_heads", "max_new", "table_width")] + [
        ("table_stride", _i64), ("q", _vp), ("out", _vp), ("q_row_stride", _i64), ("q_head_stride", _i64), ("out_row_stride", _i64),
        ("out_head_stride", _i64), ("row_start", _vp), ("lengths", _vp), ("table", _vp), ("scale", _f32), ("workspace", _vp),
        ("workspace_bytes", _sz)]


class _Verify(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_seqs", "n_rows", "vocab", "probs_dtype")] + [
        (n, _vp) for n in ("tokens", "row_start", "target_probs", "draft_probs")] + [
        ("target_row_stride", _i64), ("draft_row_stride", _i64)] + [
        (n, _vp) for n in ("u_accept", "u_sample", "n_accepted", "next_token", "emitted", "lengths", "new_lengths", "workspace")] + [
        ("workspace_bytes", _sz)]


_bound = None


def _lib():
    global _bound
    if _bound is None:
        L = jb.lib()
        for name, (res, args) in {
            "jup_paged_extend": (_i32, [_vp, _vp]),
            "jup_paged_append": (_i32, [_vp, _vp, _vp]),
            "jup_paged_attention": (_i32, [_vp, _vp, _vp]),
            "jup_paged_workspace_bytes": (_sz, []),
            "jup_verify_drafts": (_i32, [_vp, _vp]),
        }.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _bound = L
    return _bound


Step = collections.namedtuple("Step", "row_start positions slots lengths owned free_count status")
Verdict = collections.namedtuple("Verdict", "n_accepted next_token emitted lengths")

_DTYPES = {torch.float32: jb.JUP_F32, torch.bfloat16: jb.JUP_BF16}


def _need(ok, message):
    if not ok:
        raise ValueError(message)


def _ints(name, t, device, *shape):
    """An int32 tensor on the call's device; shape None: any length."""
    _need(t.dtype == torch.int32 and t.device == device, f"{name} must be an int32 tensor on {device}")
    _need(t.dim() == len(shape) and all(want is None or n == want for n, want in zip(t.shape, shape)),
          f"{name} has shape {tuple(t.shape)}, {shape} wanted (None: any)")
    _need(t.is_contiguous(), f"{name} must be contiguous")


def _table(t, device, n):
    _need(t.dtype == torch.int32 and t.device == device and t.dim() == 2 and t.shape[0] == n,
          f"table must be an int32 tensor [{n}, width] on {device}")
    _need(t.shape[1] < 2 or n == 0 or t.stride(1) == 1, "entries of a row of the table must be neighbours")
    return max(t.stride(0), t.shape[1]) if n > 1 else t.shape[1]


def _heads(name, t, dtype, device, n_heads, head_dim, rows=None):
    """[rows, heads, head_dim], elements of a head neighbours; (row stride, head stride)."""
    _need(t.dtype == dtype and t.device == device, f"{name} must be a {dtype} tensor on {device}")
    _need(t.dim() == 3 and (n_heads is None or t.shape[1] == n_heads) and t.shape[2] == head_dim and (rows is None or t.shape[0] == rows),
          f"{name} has shape {tuple(t.shape)}, [{rows}, {n_heads}, {head_dim}] wanted (None: any)")
    _need(t.stride(2) == 1 or t.numel() == 0, f"elements of a head of {name} must be neighbours")
    # (the stride of an axis of one entry is not used, and says nothing)
    return t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0


def _pool(k_pool, v_pool):
    _need(k_pool.dtype in _DTYPES and k_pool.dim() == 4 and k_pool.device.type == "cuda",
          "k_pool must be a float32 or bfloat16 tensor [n_blocks, n_kv_heads, page_size, head_dim] on the GPU")
    _need(v_pool.dtype == k_pool.dtype and v_pool.shape == k_pool.shape and v_pool.device == k_pool.device,
          "v_pool must have the type, shape and device of k_pool")
    strides = [n if size > 1 else 0 for n, size in zip(k_pool.stride(), k_pool.shape)]
    _need(strides == [n if size > 1 else 0 for n, size in zip(v_pool.stride(), v_pool.shape)] and strides[3] == 1,
          "k_pool and v_pool must have the same strides, the last one 1")
    n_blocks, heads, page, dim = k_pool.shape
    return _Pool(k_pool.data_ptr(), v_pool.data_ptr(), strides[0], strides[1], strides[2], n_blocks, page, heads, dim, _DTYPES[k_pool.dtype])


def _call(fn, device, stream, made, *structs):
    """The call on `stream`, with the tensors' device current; made: tensors that were allocated for it."""
    if stream is None:
        handle = torch.cuda.current_stream(device).cuda_stream
    else:
        _need(stream.device == device, f"the stream is on {stream.device}, the tensors on {device}")
        handle = stream.cuda_stream
        for t in made:
            if t is not None:
                t.record_stream(stream)
    structs = [ctypes.byref(s) for s in structs]
    if device.index == torch.cuda.current_device():
        jb._check(fn(*structs, handle))
    else:
        with torch.cuda.device(device):
            jb._check(fn(*structs, handle))


class Workspace:
    """Scratch of ``attention`` and ``verify`` calls that follow one another (calls that overlap need one each)."""

    def __init__(self, device="cuda:0"):
        self.buf = torch.zeros(_lib().jup_paged_workspace_bytes(), dtype=torch.uint8, device=device)


def _scratch(workspace, device):
    _need(isinstance(workspace, Workspace) and workspace.buf.device == device, f"workspace must be a Workspace on {device}")
    return workspace.buf.data_ptr(), workspace.buf.numel()


def extend(lengths, n_new, owned, table, free_blocks, free_count, page_size, max_rows, in_place=False, stream=None):
    """Pages, positions and slots of a step (jup_paged_extend): ``Step(row_start, positions, slots, lengths, owned, free_count,
    status)``, int32 tensors; ``table`` gets the new pages.  in_place: lengths, owned and free_count are updated themselves."""
    device, n = lengths.device, lengths.numel()
    _need(device.type == "cuda", "lengths must be on the GPU")
    for name, t in (("lengths", lengths), ("n_new", n_new), ("owned", owned)):
        _ints(name, t, device, n)
    _ints("free_blocks", free_blocks, device, None)
    _ints("free_count", free_count, device, 1)
    stride = _table(table, device, n)
    max_rows = int(max_rows)
    _need(max_rows >= 0, "max_rows must not be negative")
    made = torch.empty(n + 1 + 2 * max_rows + 1 + (0 if in_place else 2 * n + 1), dtype=torch.int32, device=device)
    sizes = [n + 1, max_rows, max_rows, 1] + ([] if in_place else [n, n, 1])
    row_start, positions, slots, status, *new = made.split(sizes)
    new_lengths, new_owned, new_count = (lengths, owned, free_count) if in_place else new
    args = _Extend(n, int(page_size), table.shape[1], free_blocks.numel(), max_rows, stride, lengths.data_ptr(), n_new.data_ptr(),
                   owned.data_ptr(), table.data_ptr(), free_blocks.data_ptr(), free_count.data_ptr(), row_start.data_ptr(),
                   positions.data_ptr(), slots.data_ptr(), new_lengths.data_ptr(), new_owned.data_ptr(), new_count.data_ptr(),
                   status.data_ptr())
    _call(_lib().jup_paged_extend, device, stream, (made,), args)
    return Step(row_start, positions, slots, new_lengths, new_owned, new_count, status)


def append(k, v, slots, k_pool, v_pool, positions=None, rope_theta=None, q=None, q_out=None, stream=None):
    """Rows k, v [rows, n_kv_heads, head_dim] into their slots (jup_paged_append), k rotated at ``positions`` if rope_theta is
    given; q [rows, n_heads, head_dim] is rotated into q_out (may be q; default: a new tensor), which is returned."""
    pool = _pool(k_pool, v_pool)
    dtype, device, rows = k_pool.dtype, k_pool.device, k.shape[0]
    a = _Append(n_rows=rows, k=k.data_ptr(), v=v.data_ptr(), slots=slots.data_ptr())
    a.k_row_stride, a.k_head_stride = _heads("k", k, dtype, device, pool.n_kv_heads, pool.head_dim)
    a.v_row_stride, a.v_head_stride = _heads("v", v, dtype, device, pool.n_kv_heads, pool.head_dim, rows)
    _ints("slots", slots, device, rows)
    made = None
    if rope_theta is None:
        _need(q is None and q_out is None and positions is None, "q and positions go with rope_theta")
    else:
        _need(positions is not None, "rope_theta goes with positions")
        _need(rope_theta > 0, "rope_theta must be positive")
        _ints("positions", positions, device, rows)
        a.rope_theta, a.positions = rope_theta, positions.data_ptr()
    if q is not None:
        a.q_row_stride, a.q_head_stride = _heads("q", q, dtype, device, None, pool.head_dim, rows)
        if q_out is None:
            q_out = made = torch.empty(q.shape, dtype=dtype, device=device)
        a.q_out_row_stride, a.q_out_head_stride = _heads("q_out", q_out, dtype, device, q.shape[1], pool.head_dim, rows)
        a.n_heads, a.q, a.q_out = q.shape[1], q.data_ptr(), q_out.data_ptr()
    else:
        _need(q_out is None, "q_out goes with q")
    _call(_lib().jup_paged_append, device, stream, (made,), pool, a)
    return q_out


def attention(q, k_pool, v_pool, table, row_start, lengths, max_new, workspace=None, scale=None, out=None, stream=None):
    """Attention of the rows q [rows, n_heads, head_dim] of a ragged batch over the pages (jup_paged_attention): out, of q's
    shape (default: a new tensor, whose rows outside the batch are not set).  lengths count the new tokens.  max_new: the most new tokens
    a request is expected to have.  workspace: a ``Workspace`` (not needed by float32 pools); scale: 1 / sqrt(head_dim) if None."""
    pool = _pool(k_pool, v_pool)
    dtype, device, n = k_pool.dtype, k_pool.device, lengths.numel()
    a = _Attention(n_seqs=n, n_rows=q.shape[0], max_new=int(max_new), table_width=table.shape[-1])
    a.q_row_stride, a.q_head_stride = _heads("q", q, dtype, device, None, pool.head_dim)
    a.n_heads = q.shape[1]
    made = None
    if out is None:
        out = made = torch.empty(q.shape, dtype=dtype, device=device)
    a.out_row_stride, a.out_head_stride = _heads("out", out, dtype, device, q.shape[1], pool.head_dim, q.shape[0])
    _ints("lengths", lengths, device, None)
    _ints("row_start", row_start, device, n + 1)
    a.table_stride = _table(table, device, n)
    a.q, a.out, a.row_start, a.lengths, a.table = q.data_ptr(), out.data_ptr(), row_start.data_ptr(), lengths.data_ptr(), table.data_ptr()
    a.scale = 1.0 / math.sqrt(pool.head_dim) if scale is None else scale
    if workspace is not None or dtype != torch.float32:
        a.workspace, a.workspace_bytes = _scratch(workspace, device)
    _call(_lib().jup_paged_attention, device, stream, (made,), pool, a)
    return out


def verify(tokens, target_probs, row_start, u_accept, u_sample, workspace, draft_probs=None, lengths=None, in_place=False, stream=None):
    """Verification of drafted tokens (jup_verify_drafts): ``Verdict(n_accepted, next_token, emitted, lengths)``, int32 tensors.
    tokens, u_accept [rows], probabilities [rows, vocab] (float32 or bfloat16), u_sample [n]; lengths: cached positions before the
    step (Verdict.lengths: those behind it, None without; in_place: in the same tensor)."""
    device, n, rows = row_start.device, row_start.numel() - 1, tokens.numel()
    _need(device.type == "cuda" and n >= 0, "row_start must be on the GPU and have an entry more than there are requests")
    _ints("row_start", row_start, device, n + 1)
    _ints("tokens", tokens, device, rows)
    dtype = target_probs.dtype
    _need(dtype in _DTYPES, "target_probs must be float32 or bfloat16")
    a = _Verify(n_seqs=n, n_rows=rows, vocab=target_probs.shape[-1], probs_dtype=_DTYPES[dtype])
    for name, t in (("target", target_probs), ("draft", draft_probs)):
        if t is None:
            continue
        _need(t.dtype == dtype and t.device == device and t.dim() == 2 and tuple(t.shape) == (rows, a.vocab),
              f"{name}_probs must be a {dtype} tensor [{rows}, {a.vocab}] on {device}")
        _need(t.shape[1] < 2 or rows == 0 or t.stride(1) == 1, f"probabilities of a row of {name}_probs must be neighbours")
        setattr(a, name + "_probs", t.data_ptr())
        setattr(a, name + "_row_stride", t.stride(0) if rows > 1 else 0)
    for name, t, size in (("u_accept", u_accept, rows), ("u_sample", u_sample, n)):
        _need(t.dtype == torch.float32 and t.device == device and t.is_contiguous() and tuple(t.shape) == (size,),
              f"{name} must be a contiguous float32 tensor [{size}] on {device}")
        setattr(a, name, t.data_ptr())
    new_lengths = None
    made = torch.empty(2 * n + rows + (n if lengths is not None and not in_place else 0), dtype=torch.int32, device=device)
    n_accepted, next_token, emitted, rest = made.split([n, n, rows, made.numel() - 2 * n - rows])
    if lengths is not None:
        _ints("lengths", lengths, device, n)
        new_lengths = lengths if in_place else rest
        a.lengths, a.new_lengths = lengths.data_ptr(), new_lengths.data_ptr()
    a.tokens, a.row_start = tokens.data_ptr(), row_start.data_ptr()
    a.n_accepted, a.next_token, a.emitted = n_accepted.data_ptr(), next_token.data_ptr(), emitted.data_ptr()
    a.workspace, a.workspace_bytes = _scratch(workspace, device)
    _call(_lib().jup_verify_drafts, device, stream, (made,), a)
    return Verdict(n_accepted, next_token, emitted, new_lengths)
