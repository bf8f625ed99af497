"""ctypes front end of the paged-cache operators (see include/jupiter_paged.h): keys and values in pages of one pool.

A pool is two tensors ``k_pool`` and ``v_pool`` [n_blocks, n_kv_heads, page_size, head_dim] (one layer each; any strides
whose last is 1, the same for both), a block table an int32 tensor [n_requests, width], a ragged batch a tensor of rows with
``row_start`` [n_requests + 1].  Requests may name the same pages for a prefix that they share, as far as it fills them: a page that is
partly filled is written by the next step.  One step::

    step = extend(lengths, n_new, owned, table, free_blocks, free_count, page_size, max_rows)
    for layer in ...:
        q = append(k, v, step.slots, k_pool, v_pool, positions=step.positions, rope_theta=1e4, q=q)
        out = attention(q, k_pool, v_pool, table, step.row_start, step.lengths, max_new, workspace)
    # ... or, for a stage of this package: hidden = prefill(stage, hidden, step, k_pools, v_pools, table, max_new, workspace)
    verdict = verify(tokens, target_probs, step.row_start, u_accept, u_sample, workspace, lengths=lengths)

A pool in 8 bits is two tensors of codes, int8 or float8_e4m3fn, and two of their scales, float32 [n_blocks, n_kv_heads, page_size], which
``append``, ``attention``, ``prefill``, ``read`` and ``copy_pages`` take as ``scales=(k_scale, v_scale)``; the rows that go with it are bfloat16.  ``read``
gets rows back out of their slots.  Where requests are the beams of a search a step ends, and the next one begins, with::

    beams = beam_select(logits, scores, n_keep, workspace)
    after = reorder(beams.parents.view(-1), table, step.lengths, step.owned, free_blocks, step.free_count, page_size, workspace)
    copy_pages(after.copy_from, after.copy_to, k_pools, v_pools, lengths=after.lengths)

Argument marshalling only: every operator is a HIP kernel of the library.  The calls are asynchronous on ``stream`` (default: the
current one of the tensors' device) and read nothing back.  On another stream than the current one, that stream waits for what made
the tensors that are handed in, and the caller keeps them until the call is done; results that the call makes itself are that stream's.
``ValueError`` for tensors that do not fit together, ``binding.JupiterError`` for what the library refuses.
"""
import collections
import ctypes
import math
import struct

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


class _Batch(ctypes.Structure):
    _fields_ = [("pool", _Pool), ("layer_stride", _i64)] + [(n, _i32) for n in ("n_seqs", "max_new", "table_width")] + [
        ("table_stride", _i64)] + [(n, _vp) for n in ("row_start", "lengths", "table", "positions", "slots", "workspace")] + [
        ("workspace_bytes", _sz)]


class _Scales(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("block_stride", _i64), ("head_stride", _i64), ("layer_stride", _i64)]


class _Read(ctypes.Structure):
    _fields_ = [("n_rows", _i32), ("k", _vp), ("v", _vp)] + [
        (n, _i64) for n in ("k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride")] + [("slots", _vp)]


class _Beam(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_seqs", "n_beams", "n_keep", "vocab", "logits_dtype", "end_token")] + [("logits", _vp), ("row_stride", _i64)] + [
        (n, _vp) for n in ("scores", "ended", "parents", "tokens", "new_scores", "new_ended", "workspace")] + [("workspace_bytes", _sz)]


class _Reorder(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("n_in", "n_out", "page_size", "table_width", "new_table_width", "n_free")] + [
        ("table_stride", _i64), ("new_table_stride", _i64)] + [
        (n, _vp) for n in ("parents", "table", "lengths", "owned", "free_blocks", "free_count", "held", "new_table", "new_lengths", "new_owned",
                           "new_free_blocks", "new_free_count", "copy_from", "copy_to", "status", "workspace")] + [("workspace_bytes", _sz)]


class _Copy(ctypes.Structure):
    _fields_ = [("n_copies", _i32), ("n_layers", _i32), ("layer_stride", _i64), ("copy_from", _vp), ("copy_to", _vp), ("lengths", _vp)]


# The structs as one pack() each: a ctypes object of 25 fields takes longer to fill than the GPU to answer a small call.
_FORMATS = {_i32: "i", _i64: "q", _vp: "P", _f32: "f", _sz: "N"}


def _packer(struct_type):
    packer = struct.Struct("@" + "".join(_FORMATS[t] for _, t in struct_type._fields_) + "0q")
    assert packer.size == ctypes.sizeof(struct_type), struct_type

    def pack(*values):
        try:
            return packer.pack(*values)
        except (struct.error, OverflowError) as e:
            raise ValueError(f"a number is too large for the field it goes into: {e}") from None
    return pack


_pack_pool, _pack_extend, _pack_append, _pack_attention, _pack_verify = map(_packer, (_Pool, _Extend, _Append, _Attention, _Verify))
_pack_scales, _pack_read, _pack_beam, _pack_reorder, _pack_copy = map(_packer, (_Scales, _Read, _Beam, _Reorder, _Copy))

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
            "jup_stage_prefill_paged": (_i32, [_vp, _vp, _i32, _vp, _vp, _vp]),
            "jup_verify_drafts": (_i32, [_vp, _vp]),
            "jup_paged_append8": (_i32, [_vp] * 4),
            "jup_paged_attention8": (_i32, [_vp] * 4),
            "jup_paged_read": (_i32, [_vp] * 3),
            "jup_paged_read8": (_i32, [_vp] * 4),
            "jup_stage_prefill_paged8": (_i32, [_vp, _vp, _i32, _vp, _vp, _vp, _vp]),
            "jup_beam_select": (_i32, [_vp, _vp]),
            "jup_paged_reorder": (_i32, [_vp, _vp]),
            "jup_paged_copy": (_i32, [_vp] * 4),
        }.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _bound = L
    return _bound


Step = collections.namedtuple("Step", "row_start positions slots lengths owned free_count status")
Verdict = collections.namedtuple("Verdict", "n_accepted next_token emitted lengths")
Beams = collections.namedtuple("Beams", "parents tokens scores ended")
Reordered = collections.namedtuple("Reordered", "table lengths owned free_blocks free_count copy_from copy_to status")

JUP_I8, JUP_E4M3 = 3, 4

_F32, _BF16, _I32, _CONTIGUOUS = torch.float32, torch.bfloat16, torch.int32, torch.contiguous_format
_DTYPES = {_F32: jb.JUP_F32, _BF16: jb.JUP_BF16}
_CODES = {torch.int8: JUP_I8, torch.float8_e4m3fn: JUP_E4M3}


# (messages are made where they are needed: in a call of a few microseconds they would be half of it)


def _ints(name, t, at, *shape):
    """Address of a contiguous int32 tensor on GPU number `at`, of that shape."""
    if t.dtype is not _I32 or t.get_device() != at or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def _table(t, at, n):
    """(address, width, stride) of block tables."""
    if t.dtype is not _I32 or t.get_device() != at or t.dim() != 2 or t.shape[0] != n:
        raise ValueError(f"table must be an int32 tensor [{n}, width] on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    width, (stride, step) = t.shape[1], t.stride()
    if n < 2:
        stride = width
    if (step != 1 and width > 1 and n > 0) or stride < width:
        raise ValueError("entries of a row of the table must be neighbours, and rows must not overlap")
    return t.data_ptr(), width, stride


def _overlap(rows, heads, dim, row, head):
    """Whether two heads of a tensor with these strides (0 where there is one entry) share an element."""
    if (row < dim and rows > 1) or (head < dim and heads > 1):
        return True
    if rows == 1 or heads == 1 or row >= (heads - 1) * head + dim or head >= (rows - 1) * row + dim:
        return False
    # neither lies whole between two of the other: the rows next to h heads further on
    return any(abs(h * head - r * row) < dim for h in range(1, heads) for r in (h * head // row, h * head // row + 1) if r < rows)


def _heads(name, t, dtype, at, rows, heads, dim, written=False):
    """(address, row stride, head stride) of a tensor [rows, heads, dim] whose heads are contiguous."""
    if t.dtype is not dtype or t.get_device() != at or t.shape != (rows, heads, dim):
        raise ValueError(f"{name} must be a {dtype} tensor [{rows}, {heads}, {dim}] on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    row, head, step = t.stride()
    if step != 1 and dim > 1 and t.numel():
        raise ValueError(f"elements of a head of {name} must be neighbours")
    # (the stride of an axis of one entry is not used, and says nothing)
    row, head = row if rows > 1 else 0, head if heads > 1 else 0
    if written and t.numel() and _overlap(rows, heads, dim, row, head):
        raise ValueError(f"heads of {name} overlap")
    return t.data_ptr(), row, head


def _used(strides, shape):
    """Strides, 0 for an axis of one entry: its own says nothing."""
    return tuple(step if size > 1 else 0 for step, size in zip(strides, shape))


def _pool(k_pool, v_pool, scales=None, layered=False):
    """(struct, struct of the scales or None, dtype of rows, GPU number, heads, head size) of a pool; layered: of the first layer of tensors that
    _layers() has looked at."""
    dtype, at, shape, strides, v_strides = k_pool.dtype, k_pool.get_device(), k_pool.shape, k_pool.stride(), v_pool.stride()
    if layered:
        shape, strides, v_strides = shape[1:], strides[1:], v_strides[1:]
    if scales is None:
        if dtype not in _DTYPES or len(shape) != 4 or at < 0:
            raise ValueError("k_pool must be a float32 or bfloat16 tensor [n_blocks, n_kv_heads, page_size, head_dim] on the GPU (with scales an int8 "
                             "or float8_e4m3fn one)")
    elif dtype not in _CODES or len(shape) != 4 or at < 0:
        raise ValueError("k_pool must be an int8 or float8_e4m3fn tensor [n_blocks, n_kv_heads, page_size, head_dim] on the GPU, as there are scales")
    if v_pool.dtype is not dtype or v_pool.shape != k_pool.shape or v_pool.get_device() != at:
        raise ValueError("v_pool must have the type, shape and device of k_pool")
    blocks, heads, page, dim = shape
    if scales is None:
        if v_strides != strides or strides[3] != 1:
            raise ValueError("k_pool and v_pool must have the same strides, the last one 1")
        return (_pack_pool(k_pool.data_ptr(), v_pool.data_ptr(), strides[0], strides[1], strides[2], blocks, page, heads, dim, _DTYPES[dtype]),
                None, dtype, at, heads, dim)
    k_scale, v_scale = scales
    places = k_pool.shape[:-1]
    for x in scales:
        if x.dtype is not _F32 or x.get_device() != at or x.shape != places:
            raise ValueError(f"scales must be two float32 tensors {list(places)} on cuda:{at}, not {x.dtype} {list(x.shape)} on {x.device}")
    k_steps, v_steps, layer = k_scale.stride(), v_scale.stride(), 0
    if layered:
        layer, k_steps, v_steps = k_steps[0], k_steps[1:], v_steps[1:]
    if v_strides != strides or v_steps != k_steps or strides[3] != 1 or k_steps[2] != 1 or blocks == 1 or heads == 1 or page == 1:
        # (the stride of an axis of one entry is not used, and says nothing)
        strides, k_steps = _used(strides, shape), _used(k_steps, shape)
        if _used(v_strides, shape) != strides or (strides[3] != 1 and dim > 1):
            raise ValueError("k_pool and v_pool must have the same strides, the last one 1")
        if _used(v_steps, shape) != k_steps or (k_steps[2] != 1 and page > 1):
            raise ValueError("the scales must have the same strides, the last one 1")
    return (_pack_pool(k_pool.data_ptr(), v_pool.data_ptr(), strides[0], strides[1], strides[2], blocks, page, heads, dim, _CODES[dtype]),
            _pack_scales(k_scale.data_ptr(), v_scale.data_ptr(), k_steps[0], k_steps[1], layer), _BF16, at, heads, dim)


def _layers(k_pools, v_pools, scales):
    """Stride between the layers of tensors with an axis of layers in front."""
    if k_pools.dim() != 5 or v_pools.shape != k_pools.shape or (k_pools.shape[0] > 1 and v_pools.stride(0) != k_pools.stride(0)):
        raise ValueError("k_pools and v_pools must be tensors [n_layers, n_blocks, n_heads, page_size, head_dim] of the same strides")
    if k_pools.shape[0] == 0:
        raise ValueError("there are no layers")
    if scales is not None:
        k_scale, v_scale = scales
        if k_scale.dim() != 4 or k_scale.shape != k_pools.shape[:4] or v_scale.shape != k_scale.shape or (
                k_scale.shape[0] > 1 and v_scale.stride(0) != k_scale.stride(0)):
            raise ValueError(f"scales must be two float32 tensors {list(k_pools.shape[:4])} of the same strides")
    return k_pools.stride(0)


_current_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice  # (the tensors are on the GPU: it is initialised)


def _new(stream, at, allocate):
    """A result that the call makes itself.  It is written on `stream`, so its memory is that stream's: what another stream has freed may
    still be written there by work that `stream` does not wait for.  The current stream, whose caller reads it, holds it too."""
    if stream is None:
        return allocate()
    with torch.cuda.stream(stream):
        t = allocate()
    t.record_stream(torch.cuda.current_stream(at))
    return t


def _call(fn, at, stream, *structs):
    """The call on `stream`, with the tensors' device current."""
    if stream is None:
        handle = _current_stream(at)
    else:
        if stream.device.index != at:
            raise ValueError(f"the stream is on {stream.device}, the tensors on cuda:{at}")
        handle = stream.cuda_stream
    if at == _current_device():
        status = fn(*structs, handle)
    else:
        with torch.cuda.device(at):
            status = fn(*structs, handle)
    if status:
        jb._check(status)


class Workspace:
    """Scratch of ``attention``, ``verify``, ``beam_select`` and ``reorder`` calls that follow one another (calls that overlap need one each)."""

    def __init__(self, device="cuda:0"):
        self.buf = torch.zeros(_lib().jup_paged_workspace_bytes(), dtype=torch.uint8, device=device)
        if not torch.cuda.is_current_stream_capturing():   # (the first call may be on another stream)
            torch.cuda.current_stream(self.buf.device).synchronize()
        self.args = self.buf.data_ptr(), self.buf.numel()
        self.at = self.buf.get_device()


def _scratch(workspace, at, stream):
    if not isinstance(workspace, Workspace) or workspace.at != at:
        raise ValueError(f"workspace must be a Workspace on cuda:{at}")
    if stream is not None:
        workspace.buf.record_stream(stream)
    return workspace.args


def extend(lengths, n_new, owned, table, free_blocks, free_count, page_size, max_rows, in_place=False, stream=None):
    """Pages, positions and slots of a step (jup_paged_extend): ``Step(row_start, positions, slots, lengths, owned, free_count,
    status)``, int32 tensors; ``table`` gets the new pages.  in_place: lengths, owned and free_count are updated themselves."""
    at, n = lengths.get_device(), lengths.numel()
    if at < 0:
        raise ValueError("lengths must be on the GPU")
    max_rows = int(max_rows)
    if max_rows < 0:
        raise ValueError("max_rows must not be negative")
    n_free = free_blocks.numel()
    inputs = (_ints("lengths", lengths, at, n), _ints("n_new", n_new, at, n), _ints("owned", owned, at, n))
    tables, width, stride = _table(table, at, n)
    free = (_ints("free_blocks", free_blocks, at, n_free), _ints("free_count", free_count, at, 1))
    sizes = [n + 1, max_rows, max_rows, 1] if in_place else [n + 1, max_rows, max_rows, 1, n, n, 1]
    made = _new(stream, at, lambda: lengths.new_empty(sum(sizes)))
    row_start, positions, slots, status, *new = made.split_with_sizes(sizes)
    new_lengths, new_owned, new_count = (lengths, owned, free_count) if in_place else new
    base = made.data_ptr()
    ends = base + 4 * (n + 1), base + 4 * (n + 1 + max_rows), base + 4 * (n + 1 + 2 * max_rows)
    after = (inputs[0], inputs[2], free[1]) if in_place else (ends[2] + 4, ends[2] + 4 * (n + 1), ends[2] + 4 * (2 * n + 1))
    _call(_lib().jup_paged_extend, at, stream,
          _pack_extend(n, int(page_size), width, n_free, max_rows, stride, *inputs, tables, *free, base, ends[0], ends[1], *after, ends[2]))
    return Step(row_start, positions, slots, new_lengths, new_owned, new_count, status)


def append(k, v, slots, k_pool, v_pool, positions=None, rope_theta=None, q=None, q_out=None, stream=None, scales=None):
    """Rows k, v [rows, n_kv_heads, head_dim] into their slots (jup_paged_append), k rotated at ``positions`` if rope_theta is
    given; q [rows, n_heads, head_dim] is rotated into q_out (may be q; default: a new tensor), which is returned.  scales: of a pool in 8
    bits (jup_paged_append8): the rows are quantised as they are written."""
    pool, scale, dtype, at, kv_heads, dim = _pool(k_pool, v_pool, scales)
    rows = k.shape[0]
    k_at, *k_strides = _heads("k", k, dtype, at, rows, kv_heads, dim)
    v_at, *v_strides = _heads("v", v, dtype, at, rows, kv_heads, dim)
    slots_at = _ints("slots", slots, at, rows)
    if rope_theta is None:
        if q is not None or q_out is not None or positions is not None:
            raise ValueError("q and positions go with rope_theta")
        theta, positions_at = 0.0, 0
    else:
        if positions is None or not rope_theta > 0:
            raise ValueError("rope_theta must be positive, and goes with positions")
        theta, positions_at = rope_theta, _ints("positions", positions, at, rows)
    heads, q_at, q_strides, out_at, out_strides = 0, 0, (0, 0), 0, (0, 0)
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else -1
        q_at, *q_strides = _heads("q", q, dtype, at, rows, heads, dim)
        if q_out is None:
            q_out = _new(stream, at, lambda: torch.empty_like(q, memory_format=_CONTIGUOUS))
            out_at, out_strides = q_out.data_ptr(), (heads * dim, dim)
        else:
            out_at, *out_strides = _heads("q_out", q_out, dtype, at, rows, heads, dim, written=True)
    elif q_out is not None:
        raise ValueError("q_out goes with q")
    args = _pack_append(rows, heads, q_at, k_at, v_at, out_at, *q_strides, *k_strides, *v_strides, *out_strides, positions_at, slots_at, theta)
    if scale is None:
        _call(_lib().jup_paged_append, at, stream, pool, args)
    else:
        _call(_lib().jup_paged_append8, at, stream, pool, scale, args)
    return q_out


def read(slots, k_pool, v_pool, scales=None, k_out=None, v_out=None, stream=None):
    """Rows out of their slots (jup_paged_read): k_out, v_out [rows, n_kv_heads, head_dim] (default: new tensors), zeros for slots outside the
    pool.  scales: of a pool in 8 bits, whose rows come back as bfloat16."""
    pool, scale, dtype, at, heads, dim = _pool(k_pool, v_pool, scales)
    rows = slots.numel()
    row = heads * dim
    if k_out is None and v_out is None:
        k_out, v_out = _new(stream, at, lambda: k_pool.new_empty((2, rows, heads, dim), dtype=dtype)).unbind()
        args = (k_out.data_ptr(), v_out.data_ptr(), row, dim, row, dim)
    else:
        if k_out is None:
            k_out = _new(stream, at, lambda: torch.empty((rows, heads, dim), dtype=dtype, device=k_pool.device))
        if v_out is None:
            v_out = _new(stream, at, lambda: torch.empty((rows, heads, dim), dtype=dtype, device=k_pool.device))
        k_at, *k_strides = _heads("k_out", k_out, dtype, at, rows, heads, dim, written=True)
        v_at, *v_strides = _heads("v_out", v_out, dtype, at, rows, heads, dim, written=True)
        args = (k_at, v_at, *k_strides, *v_strides)
    args = _pack_read(rows, *args, _ints("slots", slots, at, rows))
    if scale is None:
        _call(_lib().jup_paged_read, at, stream, pool, args)
    else:
        _call(_lib().jup_paged_read8, at, stream, pool, scale, args)
    return k_out, v_out


def attention(q, k_pool, v_pool, table, row_start, lengths, max_new, workspace=None, scale=None, out=None, stream=None, scales=None):
    """Attention of the rows q [rows, n_heads, head_dim] of a ragged batch over the pages (jup_paged_attention): out, of q's
    shape (default: a new tensor, whose rows outside the batch are not set).  lengths count the new tokens.  max_new: the most new tokens
    a request is expected to have.  workspace: a ``Workspace`` (not needed by float32 pools); scale: 1 / sqrt(head_dim) if None; scales: of a
    pool in 8 bits (jup_paged_attention8)."""
    pool, code_scales, dtype, at, kv_heads, dim = _pool(k_pool, v_pool, scales)
    n = lengths.numel()
    if q.dim() != 3:
        raise ValueError("q must be a tensor [rows, n_heads, head_dim]")
    rows, heads = q.shape[0], q.shape[1]
    q_at, *q_strides = _heads("q", q, dtype, at, rows, heads, dim)
    if out is None:
        out = _new(stream, at, lambda: torch.empty_like(q, memory_format=_CONTIGUOUS))
        out_at, out_strides = out.data_ptr(), (heads * dim, dim)
    else:
        out_at, *out_strides = _heads("out", out, dtype, at, rows, heads, dim, written=True)
    tables, width, stride = _table(table, at, n)
    args = _pack_attention(n, rows, heads, int(max_new), width, stride, q_at, out_at, *q_strides, *out_strides,
                           _ints("row_start", row_start, at, n + 1), _ints("lengths", lengths, at, n), tables,
                           1.0 / math.sqrt(dim) if scale is None else scale,
                           *(_scratch(workspace, at, stream) if workspace is not None or dtype is not _F32 else (0, 0)))
    if code_scales is None:
        _call(_lib().jup_paged_attention, at, stream, pool, args)
    else:
        _call(_lib().jup_paged_attention8, at, stream, pool, code_scales, args)
    return out


def prefill(stage, hidden_in, step, k_pools, v_pools, table, max_new, workspace=None, hidden_out=None, stream=None, scales=None):
    """A ``binding.Stage`` over the rows hidden_in [rows, d_model] of a ragged batch (jup_stage_prefill_paged): hidden_out (default: a new
    tensor).  step: what ``extend`` returned; k_pools, v_pools [n_layers, n_blocks, n_heads, page_size, head_dim]; scales: of pools in 8
    bits, [n_layers, n_blocks, n_heads, page_size] each (jup_stage_prefill_paged8)."""
    layer_stride = _layers(k_pools, v_pools, scales)
    if k_pools.shape[0] != stage.cfg["n_layers"]:
        raise ValueError(f"k_pools and v_pools have {k_pools.shape[0]} layers, the stage {stage.cfg['n_layers']}")
    packed, code_scales, dtype, at, _, _ = _pool(k_pools, v_pools, scales, True)
    n, rows, width = step.lengths.numel(), hidden_in.shape[0], stage.cfg["d_model"]
    for name, t in (("hidden_in", hidden_in), ("hidden_out", hidden_in if hidden_out is None else hidden_out)):
        if t.dtype is not dtype or t.get_device() != at or t.shape != (rows, width) or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor [{rows}, {width}] on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    if stage.workspace.get_device() != at:
        raise ValueError(f"the stage is on {stage.workspace.device}, the tensors on cuda:{at}")
    if step.positions.numel() < rows or step.slots.numel() < rows:
        raise ValueError(f"the step has positions of {step.positions.numel()} rows, hidden_in {rows}")
    tables, table_width, stride = _table(table, at, n)
    scratch = _scratch(workspace, at, stream) if workspace is not None or dtype is not _F32 else (0, 0)
    batch = _Batch(_Pool.from_buffer_copy(packed), layer_stride, n, int(max_new), table_width, stride, _ints("row_start", step.row_start, at, n + 1),
                   _ints("lengths", step.lengths, at, n), tables, _ints("positions", step.positions, at, step.positions.numel()),
                   _ints("slots", step.slots, at, step.slots.numel()), *scratch)
    if hidden_out is None:
        hidden_out = _new(stream, at, lambda: torch.empty_like(hidden_in))
    fn, given = (_lib().jup_stage_prefill_paged, ()) if code_scales is None else (_lib().jup_stage_prefill_paged8, (code_scales,))
    _call(lambda handle: fn(stage.handle, hidden_in.data_ptr(), rows, ctypes.byref(batch), *given, hidden_out.data_ptr(), handle), at, stream)
    return hidden_out


def _probs(name, t, dtype, at, rows, vocab):
    if t.dtype is not dtype or t.get_device() != at or t.shape != (rows, vocab):
        raise ValueError(f"{name} must be a {dtype} tensor [{rows}, {vocab}] on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    row, step = t.stride()
    if step != 1 and vocab > 1 and rows > 0:
        raise ValueError(f"probabilities of a row of {name} must be neighbours")
    return t.data_ptr(), row if rows > 1 else 0


def _uniforms(name, t, at, n):
    if t.dtype is not _F32 or t.get_device() != at or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor [{n}] on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def verify(tokens, target_probs, row_start, u_accept, u_sample, workspace, draft_probs=None, lengths=None, in_place=False, stream=None):
    """Verification of drafted tokens (jup_verify_drafts): ``Verdict(n_accepted, next_token, emitted, lengths)``, int32 tensors.
    tokens, u_accept [rows], probabilities [rows, vocab] (float32 or bfloat16), u_sample [n]; lengths: cached positions before the
    step (Verdict.lengths: those behind it, None without; in_place: in the same tensor)."""
    at, n, rows, dtype = row_start.get_device(), row_start.numel() - 1, tokens.numel(), target_probs.dtype
    if at < 0 or n < 0:
        raise ValueError("row_start must be on the GPU and have an entry more than there are requests")
    if dtype not in _DTYPES or target_probs.dim() != 2:
        raise ValueError("target_probs must be a float32 or bfloat16 tensor [rows, vocab]")
    vocab = target_probs.shape[1]
    target, target_stride = _probs("target_probs", target_probs, dtype, at, rows, vocab)
    draft, draft_stride = (0, 0) if draft_probs is None else _probs("draft_probs", draft_probs, dtype, at, rows, vocab)
    tokens_at = _ints("tokens", tokens, at, rows)
    sizes = [n, n, rows] if lengths is None or in_place else [n, n, rows, n]
    made = _new(stream, at, lambda: tokens.new_empty(sum(sizes)))
    n_accepted, next_token, emitted, *new = made.split_with_sizes(sizes)
    base = made.data_ptr()
    lengths_at = after_at = 0
    new_lengths = None
    if lengths is not None:
        lengths_at = after_at = _ints("lengths", lengths, at, n)
        new_lengths = lengths
        if not in_place:
            new_lengths, after_at = new[0], base + 4 * (2 * n + rows)
    _call(_lib().jup_verify_drafts, at, stream,
          _pack_verify(n, rows, vocab, _DTYPES[dtype], tokens_at, _ints("row_start", row_start, at, n + 1), target,
                       draft, target_stride, draft_stride, _uniforms("u_accept", u_accept, at, rows), _uniforms("u_sample", u_sample, at, n),
                       base, base + 4 * n, base + 8 * n, lengths_at, after_at, *_scratch(workspace, at, stream)))
    return Verdict(n_accepted, next_token, emitted, new_lengths)


def _floats(name, t, at, n):
    if t.dtype is not _F32 or t.get_device() != at or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor of {n} on cuda:{at}, not {t.dtype} {list(t.shape)} on {t.device}")
    return t.data_ptr()


def beam_select(logits, scores, n_keep, workspace, end_token=-1, ended=None, stream=None):
    """The best continuations over the beams and the vocabulary (jup_beam_select): ``Beams(parents, tokens, scores, ended)``, [n_requests,
    n_keep] each, best first.  scores [n_requests, n_beams] float32, sums of log probabilities; logits [n_requests * n_beams, vocab] float32 or
    bfloat16; ended [n_requests, n_beams] int32: not 0 where a beam has come to end_token."""
    dtype, at = logits.dtype, logits.get_device()
    if dtype not in _DTYPES or logits.dim() != 2 or at < 0:
        raise ValueError("logits must be a float32 or bfloat16 tensor [rows, vocab] on the GPU")
    if scores.dim() != 2 or scores.numel() != logits.shape[0]:
        raise ValueError(f"scores must be a tensor [n_requests, n_beams] of as many as there are rows of logits ({logits.shape[0]}), not {list(scores.shape)}")
    (n, beams), (rows, vocab), keep = scores.shape, logits.shape, int(n_keep)
    logits_at, stride = _probs("logits", logits, dtype, at, rows, vocab)
    scores_at = _floats("scores", scores, at, rows)
    if ended is not None and ended.shape != scores.shape:
        raise ValueError(f"ended must have the shape of scores, not {list(ended.shape)}")
    ended_at = 0 if ended is None else _ints("ended", ended, at, n, beams)
    if not 0 < keep <= 64:
        raise ValueError(f"n_keep={keep} is outside 1..64")
    made = _new(stream, at, lambda: torch.empty((4, n, keep), dtype=_I32, device=logits.device))
    parents, tokens, new_scores, new_ended = made.unbind()
    base, size = made.data_ptr(), 4 * n * keep
    _call(_lib().jup_beam_select, at, stream,
          _pack_beam(n, beams, keep, vocab, _DTYPES[dtype], int(end_token), logits_at, stride, scores_at, ended_at, base, base + size, base + 2 * size,
                     base + 3 * size, *_scratch(workspace, at, stream)))
    return Beams(parents, tokens, new_scores.view(_F32), new_ended)


def reorder(parents, table, lengths, owned, free_blocks, free_count, page_size, workspace, held=None, width=None, in_place=False, stream=None):
    """Block tables of requests that go on from others (jup_paged_reorder): ``Reordered(table, lengths, owned, free_blocks, free_count, copy_from,
    copy_to, status)``, int32 tensors of parents.numel() requests.  parents: rows of ``table``, or -1; free_blocks has room for every block of the
    pool; held: uint8, one per entry of free_blocks, not 0 for blocks that others hold; width: of the new table (default: table's).
    in_place: free_blocks and free_count are updated themselves.  The copies that are due: ``copy_pages``."""
    at, n, n_in, n_free = parents.get_device(), parents.numel(), lengths.numel(), free_blocks.numel()
    if at < 0:
        raise ValueError("parents must be on the GPU")
    parents_at = _ints("parents", parents, at, n)
    tables, old_width, stride = _table(table, at, n_in)
    inputs = (_ints("lengths", lengths, at, n_in), _ints("owned", owned, at, n_in), _ints("free_blocks", free_blocks, at, n_free),
              _ints("free_count", free_count, at, 1))
    if held is not None and (held.dtype is not torch.uint8 or held.get_device() != at or held.shape != (n_free,) or not held.is_contiguous()):
        raise ValueError(f"held must be a contiguous uint8 tensor [{n_free}] on cuda:{at}, not {held.dtype} {list(held.shape)} on {held.device}")
    width = old_width if width is None else int(width)
    if width < 0:
        raise ValueError("width must not be negative")
    sizes = [n, n, n, n, 1, n * width] + ([] if in_place else [1, n_free])
    made = _new(stream, at, lambda: parents.new_empty(sum(sizes)))
    new_lengths, new_owned, copy_from, copy_to, status, new_table, *new = made.split_with_sizes(sizes)
    new_table = new_table.view(n, width)
    new_count, new_free = (free_count, free_blocks) if in_place else new
    base = made.data_ptr()
    status_at = base + 16 * n
    table_at = status_at + 4
    after = (inputs[2], inputs[3]) if in_place else (table_at + 4 * n * width + 4, table_at + 4 * n * width)
    _call(_lib().jup_paged_reorder, at, stream,
          _pack_reorder(n_in, n, int(page_size), old_width, width, n_free, stride, width, parents_at, tables, *inputs,
                        0 if held is None else held.data_ptr(), table_at, base, base + 4 * n, *after, base + 8 * n, base + 12 * n, status_at,
                        *_scratch(workspace, at, stream)))
    return Reordered(new_table, new_lengths, new_owned, new_free, new_count, copy_from, copy_to, status)


def copy_pages(copy_from, copy_to, k_pools, v_pools, lengths=None, scales=None, stream=None):
    """Pages copy_from[i] to copy_to[i] of every layer (jup_paged_copy), whole ones, or with lengths the first lengths[i] mod page_size slots.
    k_pools, v_pools, scales: of one layer, or with an axis of layers in front."""
    layered = k_pools.dim() == 5
    layers, layer_stride = (k_pools.shape[0], _layers(k_pools, v_pools, scales)) if layered else (1, 0)
    pool, code_scales, _, at, _, _ = _pool(k_pools, v_pools, scales, layered)
    n = copy_from.numel()
    _call(_lib().jup_paged_copy, at, stream, pool, code_scales,
          _pack_copy(n, layers, layer_stride, _ints("copy_from", copy_from, at, n), _ints("copy_to", copy_to, at, n),
                     0 if lengths is None else _ints("lengths", lengths, at, n)))
