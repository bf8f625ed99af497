"""Keys and values in pages: every operator of include/jupiter_paged.h against its definition in 64 bits (paged_reference.py).

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value.  Attention rounds the probabilities (2^-8 of sum p|v|) and the
result (2^-8 of it); fp32 sums over n keys and 128 products add at most (n 2^-24 + 2 x 128 x 2^-24 x sum|q k| scale) sum p|v|, and
the exponentials a few 2^-23.  Rotated rows: one rounding, of a result whose fp32 products and cosines are 2^-22 of the pair off.
"""
import ctypes
import random
import types

import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2504_08242_amd import binding as jb
from paper_2504_08242_amd import paged as jp

gpu = pytest.mark.gpu
DEV = "cuda:0"
BF16 = 2.0 ** -8


def f64(t):
    return t.detach().double().cpu().numpy()


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device=DEV)


def starts(new):
    return [sum(new[:i]) for i in range(len(new) + 1)]


@pytest.fixture(scope="module")
def workspace():
    return jp.Workspace(DEV)


# ---- refusals: no GPU -------------------------------------------------------------------------------------------------------

FAKE = 0x7000_0000_0000


def pool_args(**change):
    a = dict(k=FAKE, v=FAKE, block_stride=4 * 16 * 128, head_stride=16 * 128, slot_stride=128, n_blocks=10, page_size=16, n_kv_heads=4,
             head_dim=128, dtype=jb.JUP_BF16)
    return jp._Pool(**dict(a, **change))


def extend_args(**change):
    a = dict(n_seqs=2, page_size=16, table_width=4, n_free=3, max_rows=8, table_stride=4)
    a.update({n: FAKE for n in ("lengths", "n_new", "owned", "table", "free_blocks", "free_count", "row_start", "positions", "slots",
                                "new_lengths", "new_owned", "new_free_count", "status")})
    return jp._Extend(**dict(a, **change))


def append_args(**change):
    a = dict(n_rows=3, n_heads=8, q=FAKE, k=FAKE, v=FAKE, q_out=FAKE, positions=FAKE, slots=FAKE, rope_theta=1e4)
    for x in ("q", "k", "v", "q_out"):
        a[x + "_row_stride"], a[x + "_head_stride"] = 1024, 128
    return jp._Append(**dict(a, **change))


def attention_args(**change):
    a = dict(n_seqs=2, n_rows=3, n_heads=8, max_new=2, table_width=4, table_stride=4, q=FAKE, out=FAKE, q_row_stride=1024, q_head_stride=128,
             out_row_stride=1024, out_head_stride=128, row_start=FAKE, lengths=FAKE, table=FAKE, scale=0.1, workspace=FAKE,
             workspace_bytes=jp._lib().jup_paged_workspace_bytes())
    return jp._Attention(**dict(a, **change))


def verify_args(**change):
    a = dict(n_seqs=2, n_rows=6, vocab=100, probs_dtype=jb.JUP_F32, target_row_stride=100, draft_row_stride=100, workspace=FAKE,
             workspace_bytes=jp._lib().jup_paged_workspace_bytes())
    a.update({n: FAKE for n in ("tokens", "row_start", "target_probs", "draft_probs", "u_accept", "u_sample", "n_accepted", "next_token",
                                "emitted", "lengths", "new_lengths")})
    return jp._Verify(**dict(a, **change))


def refused(rc, word):
    assert rc == jb.JUP_EINVAL, (rc, word)
    assert word in jb.last_error(), (word, jb.last_error())


@pytest.mark.parametrize("change,word", [
    (dict(n_seqs=-1), "n_seqs"), (dict(n_seqs=16385), "n_seqs"), (dict(page_size=12), "page_size"), (dict(page_size=4), "page_size"),
    (dict(page_size=131072), "page_size"), (dict(table_width=-1), "table_width"), (dict(table_width=1 << 27, table_stride=1 << 27), "2^31"),
    (dict(table_stride=3), "table_stride"), (dict(n_free=-1), "n_free"), (dict(max_rows=-1), "max_rows"), (dict(free_count=None), "free_count"),
    (dict(status=None), "status"), (dict(free_blocks=None), "free_blocks"), (dict(slots=None), "slots"), (dict(lengths=None), "lengths"),
    (dict(new_owned=None), "new_owned"), (dict(table=None), "table"), (dict(row_start=None), "row_start")])
def test_extend_refuses(change, word):
    refused(jp._lib().jup_paged_extend(ctypes.byref(extend_args(**change)), None), word)


POOL_FAULTS = [(dict(dtype=2), "dtype"), (dict(n_blocks=0), "positive"), (dict(n_kv_heads=0), "positive"), (dict(page_size=24), "page_size"),
               (dict(n_blocks=1 << 28), "2^31"), (dict(k=None), "k and v"), (dict(v=FAKE + 8), "aligned"), (dict(head_dim=64), "128"),
               (dict(slot_stride=132), "multiples of 8"), (dict(block_stride=-8), "negative"), (dict(slot_stride=(1 << 25) + 8), "slot_stride"),
               (dict(dtype=0, head_dim=258), "256"), (dict(dtype=0, head_dim=63), "even")]


@pytest.mark.parametrize("change,word", POOL_FAULTS)
def test_pools_are_refused_by_append_and_attention(change, word):
    p = ctypes.byref(pool_args(**change))
    refused(jp._lib().jup_paged_append(p, ctypes.byref(append_args()), None), word)
    refused(jp._lib().jup_paged_attention(p, ctypes.byref(attention_args()), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(n_rows=-1), "n_rows"), (dict(rope_theta=-1.0), "rope_theta"), (dict(rope_theta=float("nan")), "rope_theta"),
    (dict(rope_theta=float("inf")), "rope_theta"), (dict(rope_theta=0.0), "rotation"), (dict(q_out=None), "together"), (dict(n_heads=0), "n_heads"),
    (dict(k=None), "NULL"), (dict(slots=None), "NULL"), (dict(positions=None), "positions"), (dict(k=FAKE + 2), "aligned"),
    (dict(v_row_stride=1020), "multiples of 8"), (dict(q_head_stride=-128), "negative"), (dict(q_out=FAKE + 4), "aligned")])
def test_append_refuses(change, word):
    refused(jp._lib().jup_paged_append(ctypes.byref(pool_args()), ctypes.byref(append_args(**change)), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(n_seqs=-1), "n_seqs"), (dict(n_rows=-1), "n_rows"), (dict(max_new=-1), "max_new"), (dict(n_heads=6), "multiple"), (dict(n_heads=0), "multiple"),
    (dict(n_rows=1 << 30), "2^31"), (dict(table_width=-1), "table_width"), (dict(table_stride=3), "table_stride"), (dict(scale=0.0), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(q=None), "NULL"), (dict(lengths=None), "NULL"),
    (dict(table=None), "NULL"), (dict(q=FAKE + 8), "aligned"), (dict(out_row_stride=1028), "multiples of 8"), (dict(workspace=None), "workspace"),
    (dict(workspace=FAKE + 16), "workspace"), (dict(workspace_bytes=0), "workspace")])
def test_attention_refuses(change, word):
    refused(jp._lib().jup_paged_attention(ctypes.byref(pool_args()), ctypes.byref(attention_args(**change)), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(n_seqs=-1), "n_seqs"), (dict(n_rows=-1), "n_rows"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 30) + 1), "vocab"),
    (dict(probs_dtype=2), "probs_dtype"), (dict(target_row_stride=-1), "negative"), (dict(lengths=None), "together"),
    (dict(new_lengths=None), "together"), (dict(workspace=None), "workspace"), (dict(workspace_bytes=1), "workspace"), (dict(row_start=None), "NULL"),
    (dict(next_token=None), "NULL"), (dict(tokens=None), "NULL"), (dict(u_accept=None), "NULL")])
def test_verify_refuses(change, word):
    refused(jp._lib().jup_verify_drafts(ctypes.byref(verify_args(**change)), None), word)


@pytest.mark.parametrize("change,word", [(dict(scale=1.1e38), "scale"), (dict(table_width=(1 << 27) - 1, table_stride=1 << 27), "2^31 - 256")])
def test_attention_refuses_what_would_overflow(change, word):
    a = attention_args(**change)
    refused(jp._lib().jup_paged_attention(ctypes.byref(pool_args()), ctypes.byref(a), None), word)


def test_sizes_that_indices_would_wrap_at_are_refused():
    L = jp._lib()
    refused(L.jup_paged_extend(ctypes.byref(extend_args(n_free=(1 << 30) + 1)), None), "n_free")
    refused(L.jup_verify_drafts(ctypes.byref(verify_args(n_rows=(1 << 30) + 1)), None), "n_rows")


def test_null_arguments_and_empty_calls():
    L = jp._lib()
    refused(L.jup_paged_extend(None, None), "NULL")
    refused(L.jup_paged_append(None, ctypes.byref(append_args()), None), "pool")
    refused(L.jup_paged_append(ctypes.byref(pool_args()), None, None), "args")
    refused(L.jup_paged_attention(ctypes.byref(pool_args()), None, None), "args")
    refused(L.jup_verify_drafts(None, None), "NULL")
    # nothing to do: nothing is launched, pointers may be missing
    assert L.jup_paged_append(ctypes.byref(pool_args()), ctypes.byref(append_args(n_rows=0, k=None, v=None, slots=None)), None) == 0
    assert L.jup_paged_attention(ctypes.byref(pool_args()), ctypes.byref(attention_args(n_rows=0, q=None)), None) == 0
    assert L.jup_paged_attention(ctypes.byref(pool_args()), ctypes.byref(attention_args(n_seqs=0, lengths=None)), None) == 0
    assert L.jup_verify_drafts(ctypes.byref(verify_args(n_seqs=0, tokens=None)), None) == 0


def test_the_front_end_refuses_tensors_that_do_not_fit():
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        jp.extend(i, i, i, torch.zeros((3, 2), dtype=torch.int32), i, i[:1], 16, 4)
    p = torch.zeros((2, 1, 16, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        jp.append(p[:, :, 0], p[:, :, 0], i, p, p)
    with pytest.raises(ValueError, match="GPU"):
        jp.verify(i, p[0, 0], i, i, i, None)


@pytest.mark.parametrize("shape,strides,fits", [
    ((5, 3, 8), (24, 8, 1), True), ((5, 3, 8), (8, 40, 1), True), ((5, 3, 8), (100, 9, 1), True), ((5, 1, 8), (8, 0, 1), True), ((1, 3, 8), (0, 8, 1), True),
    ((2, 3, 8), (8, 16, 1), True),                                                # heads between the rows of another
    ((5, 3, 8), (8, 8, 1), False), ((5, 3, 8), (23, 8, 1), False), ((5, 3, 8), (8, 39, 1), False), ((5, 3, 8), (0, 8, 1), False), ((5, 3, 8), (24, 7, 1), False),
    ((3, 3, 8), (8, 16, 1), False), ((4, 40, 8), (50, 10, 1), False), ((2, 7, 8), (60, 10, 1), False), ((2, 6, 8), (58, 10, 1), True)])
def test_results_whose_heads_overlap_are_refused(shape, strides, fits):
    t = torch.empty(10000).as_strided(shape, strides)
    offsets = [r * strides[0] + h * strides[1] + i for r in range(shape[0]) for h in range(shape[1]) for i in range(shape[2])]
    assert fits == (len(set(offsets)) == len(offsets))
    if fits:
        jp._heads("out", t, torch.float32, -1, *shape, written=True)
    else:
        with pytest.raises(ValueError, match="overlap"):
            jp._heads("out", t, torch.float32, -1, *shape, written=True)


@gpu
def test_the_front_end_refuses_tensors_that_do_not_fit_on_the_gpu(workspace):
    k = torch.zeros((5, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    row, i = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=DEV), ints([0, 1, 2])
    q, table = torch.zeros((3, 4, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    at, n = ints([0, 1, 2, 3]), ints([1, 1, 1])
    for bad in (lambda: jp.append(row.float(), row, i, k, k), lambda: jp.append(row, row[:2], i, k, k), lambda: jp.append(row, row, i.long(), k, k),
                lambda: jp.append(row, row, i, k, k[:4]), lambda: jp.append(row, row, i, k, k, positions=i), lambda: jp.append(row, row, i, k, k, rope_theta=1e4),
                lambda: jp.append(row, row, i, k, k, positions=i[:2], rope_theta=1e4), lambda: jp.append(row, row, i, k, k, q=q),
                lambda: jp.append(row.transpose(1, 2), row, i, k, k), lambda: jp.append(row, row, i, k, torch.zeros((5, 16, 2, 128), dtype=torch.bfloat16, device=DEV).transpose(1, 2)),
                lambda: jp.attention(q, k, k, table, at[:3], n, 1, workspace), lambda: jp.attention(q, k, k, table[:2], at, n, 1, workspace),
                lambda: jp.attention(q, k, k, table, at, n, 1), lambda: jp.attention(q.float(), k, k, table, at, n, 1, workspace),
                lambda: jp.attention(q, k, k, table, at, n.cpu(), 1, workspace), lambda: jp.attention(q, k, k, table.t(), at, n, 1, workspace),
                lambda: jp.attention(q, k, k, table, at, n, 1, workspace, out=q[:, :2]),
                lambda: jp.verify(i, q[:, 0], at, i.float(), n.float(), workspace, draft_probs=q[:, 0].float()),
                lambda: jp.verify(i, q[:, 0].half(), at, i.float(), n.float(), workspace), lambda: jp.verify(i, q[:, 0], at, i, n.float(), workspace)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: jp.attention(q[:, :3], k, k, table, at, n, 1, workspace), lambda: jp.attention(q, k, k, table, at, n, 1, workspace, scale=-1.0),
                lambda: jp.attention(q, k, k, table, at, n, -1, workspace), lambda: jp.extend(n, n, n, table, i, n[:1], 10, 4)):
        with pytest.raises(jb.JupiterError) as e:
            bad()
        assert e.value.status == jb.JUP_EINVAL


@gpu
def test_numbers_too_large_for_their_fields_are_refused(workspace):
    k = torch.zeros((5, 2, 16, 128), dtype=torch.bfloat16, device=DEV)
    q, i = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=DEV), ints([0, 1, 2])
    table, at = torch.zeros((3, 2), dtype=torch.int32, device=DEV), ints([0, 1, 2, 3])
    for bad in (lambda: jp.attention(q, k, k, table, at, i, 2 ** 31, workspace), lambda: jp.attention(q, k, k, table, at, i, 1, workspace, scale=1e300),
                lambda: jp.attention(q, k, k, table, at, i, 1, workspace, scale=3e38), lambda: jp.append(q, q, i, k, k, positions=i, rope_theta=1e300),
                lambda: jp.extend(i, i, i, table, i, i[:1], 2 ** 40, 4)):
        with pytest.raises((ValueError, jb.JupiterError)):
            bad()


# ---- tables -----------------------------------------------------------------------------------------------------------------


def check_extend(lengths, new, owned, table, free, count, page, max_rows, in_place=False):
    table = np.array(table, dtype=np.int64)
    want = ref.extend(lengths, new, owned, table, free, count, page, max_rows)
    t = torch.from_numpy(table).to(DEV, torch.int32)
    dev = [ints(x) for x in (lengths, new, owned)]
    cnt = ints([count])
    step = jp.extend(*dev, t, ints(free), cnt, page, max_rows, in_place=in_place)
    got = [step.status, step.row_start, step.positions, step.slots, step.lengths, step.owned, step.free_count]
    for name, g, w in zip(("status", *jp.Step._fields), got, [[want[0]], *want[1:6], [want[6]]]):
        assert g.cpu().tolist() == list(w), (name, want[0])
    assert np.array_equal(t.cpu().numpy(), want[7])
    if in_place:
        assert step.lengths.data_ptr() == dev[0].data_ptr() and step.free_count.data_ptr() == cnt.data_ptr()
    else:  # what went in is as it was
        assert dev[0].cpu().tolist() == list(lengths) and dev[2].cpu().tolist() == list(owned) and cnt.cpu().tolist() == [count]
    return want[0]


def random_step(rng, n, page, width, most_new):
    lengths = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, page * width // 2)]) for _ in range(n)]
    lengths = [min(a, page * width) for a in lengths]
    new = [rng.choice([0, 1, 1, 5, rng.randint(0, most_new)]) for _ in range(n)]
    new = [min(b, page * width - a) for a, b in zip(lengths, new)]
    owned = [min(width, -(-a // page) + rng.choice([0, 0, 0, 1, 2])) for a in lengths]   # pages left over from rejected drafts
    fresh = sum(max(0, -(-(a + b) // page) - c) for a, b, c in zip(lengths, new, owned))
    blocks = rng.sample(range(10 * n * width + 10), n * width + fresh + 5)
    table = [blocks[i * width:(i + 1) * width] for i in range(n)]
    table = [[b if j < c else -1 for j, b in enumerate(row)] for row, c in zip(table, owned)]
    return lengths, new, owned, table, blocks[n * width:], fresh


@gpu
@pytest.mark.parametrize("n,page,width,most_new", [(1, 8, 1, 8), (1, 16, 40, 600), (7, 16, 9, 40), (64, 32, 5, 10), (300, 8, 30, 100),
                                                   (1024, 16, 12, 3), (1025, 16, 6, 9), (2500, 64, 3, 6), (16, 65536, 2, 300)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_of_a_step(n, page, width, most_new, in_place):
    rng = random.Random(n * page + width)
    lengths, new, owned, table, free, fresh = random_step(rng, n, page, width, most_new)
    rows = sum(new)
    for max_rows in (rows, rows + 3, rows + 5000):  # the last: positions and slots in a launch of their own
        assert check_extend(lengths, new, owned, table, free, fresh + (len(free) - fresh) // 2, page, max_rows, in_place) == 0


@gpu
def test_tables_of_no_requests_and_of_idle_ones():
    assert check_extend([], [], [], np.zeros((0, 3)), [4, 5], 2, 16, 0) == 0
    assert check_extend([], [], [], np.zeros((0, 3)), [4, 5], 2, 16, 5) == 0
    assert check_extend([], [], [], np.zeros((0, 3)), [4, 5], 2, 16, 5000) == 0
    assert check_extend([17, 0, 3], [0, 0, 0], [2, 0, 1], [[3, 4], [-1, -1], [7, -1]], [], 0, 16, 4) == 0


@gpu
@pytest.mark.parametrize("max_rows", [40, 5000])
@pytest.mark.parametrize("status,change", [
    (1, dict(lengths=[16, -1, 3])), (1, dict(new=[3, 2, -2])), (1, dict(owned=[1, -1, 1])), (1, dict(owned=[1, 5, 1])), (1, dict(count=-1)),
    (1, dict(count=7)), (2, dict(lengths=[16, 60, 3])), (2, dict(lengths=[16, 2147483647, 3], new=[3, 2147483647, 2])), (3, dict(new=[3, 6000, 2], width=1000)),
    (4, dict(count=2)), (4, dict(count=0)), (1, dict(count=0, lengths=[-16, 4, 3])), (2, dict(count=0, lengths=[100, 4, 3]))])
def test_a_step_that_does_not_fit_changes_nothing(status, change, max_rows):
    a = dict(dict(lengths=[16, 4, 3], new=[3, 30, 2], owned=[1, 1, 1], count=6, width=4), **change)
    table = np.full((3, a["width"]), -1)
    table[:, 0] = [8, 9, 10]
    assert check_extend(a["lengths"], a["new"], a["owned"], table, [20, 21, 22, 23, 24, 25], a["count"], 16, max_rows) == status


@gpu
def test_blocks_that_no_pool_has_get_no_slots():
    # page numbers a caller got wrong: negative ones, and one whose slots would pass 2^31
    step = jp.extend(ints([0, 0]), ints([3, 2]), ints([0, 0]), torch.full((2, 1), -1, dtype=torch.int32, device=DEV), ints([-7, 2 ** 31 - 1]), ints([2]), 16, 6)
    assert step.status.tolist() == [0] and step.slots.tolist() == [-1] * 6 and step.positions.tolist() == [0, 1, 2, 0, 1, 0]


# ---- rows into their slots ---------------------------------------------------------------------------------------------------


def make_pool(dtype, n_blocks, heads, page, dim, order, gen, fill=None):
    """k and v [block, head, slot, i] in one of the orders a pool may have in memory."""
    def one():
        shape = (n_blocks, heads, page, dim)
        if order == "block-head-slot":
            t = torch.empty(shape, dtype=dtype, device=DEV)
        elif order == "block-slot-head":
            t = torch.empty((n_blocks, page, heads, dim), dtype=dtype, device=DEV).transpose(1, 2)
        elif order == "head-block-slot":
            t = torch.empty((heads, n_blocks, page, dim), dtype=dtype, device=DEV).transpose(0, 1)
        else:  # wide rows: something else lies between the heads
            t = torch.empty((n_blocks, heads, page, dim + 24), dtype=dtype, device=DEV)[..., :dim]
        t.copy_(torch.randn(shape, generator=gen) if fill is None else torch.full(shape, fill))
        return t
    if order == "k-v-together":
        both = torch.empty((n_blocks, 2, heads, page, dim), dtype=dtype, device=DEV)
        both.copy_(torch.randn(both.shape, generator=gen) if fill is None else torch.full(both.shape, fill))
        return both[:, 0], both[:, 1]
    return one(), one()


ORDERS = ["block-head-slot", "block-slot-head", "head-block-slot", "wide", "k-v-together"]


@gpu
@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float32, 128), (torch.float32, 6), (torch.float32, 256)])
@pytest.mark.parametrize("rows,heads,kv_heads,page,order", [(1, 4, 4, 16, "block-head-slot"), (5, 8, 2, 8, "block-slot-head"), (33, 5, 1, 32, "head-block-slot"),
                                                            (70, 12, 12, 64, "wide"), (9, 40, 8, 16, "k-v-together")])
def test_rows_go_into_their_slots(dtype, dim, rows, heads, kv_heads, page, order):
    gen = torch.Generator().manual_seed(rows * heads + dim)
    n_blocks = -(-rows // page) + 3
    k_pool, v_pool = make_pool(dtype, n_blocks, kv_heads, page, dim, order, gen)
    before = f64(k_pool), f64(v_pool)
    # one projection's output holds q, k and v of a row side by side
    fused = torch.randn((rows, heads + 2 * kv_heads, dim), generator=gen).to(DEV, dtype)
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
    slots = torch.randperm(n_blocks * page, generator=gen)[:rows]
    if rows > 4:
        slots[1], slots[3], slots[4] = -1, n_blocks * page, 2 ** 31 - 1   # a row behind the last one, and slots no pool has
    positions = torch.randint(0, 100000, (rows,), generator=gen)
    positions[0] = 0
    if rows > 2:
        positions[2] = -3
    got = jp.append(k, v, slots.to(DEV, torch.int32), k_pool, v_pool, positions=positions.to(DEV, torch.int32), rope_theta=1e4, q=q)
    want_q, want_k = ref.rotate(f64(q), positions.numpy(), 1e4), ref.rotate(f64(k), positions.numpy(), 1e4)
    rounding = BF16 if dtype == torch.bfloat16 else 0.0
    half = dim // 2

    def bound(x, w):  # x: what was rotated
        size = np.hypot(x[..., :half], x[..., half:])
        return rounding * np.abs(w) + 2.0 ** -21 * np.concatenate([size, size], -1)

    assert (np.abs(f64(got) - want_q) <= bound(f64(q), want_q)).all()
    pools, wants, sources = (f64(k_pool), f64(v_pool)), before, (want_k, f64(v))
    for name, have, want, src in zip("kv", pools, wants, sources):
        limit = np.zeros_like(want)
        for r, s in enumerate(slots.tolist()):
            if 0 <= s < n_blocks * page:
                want[s // page, :, s % page] = src[r]
                if name == "k":
                    limit[s // page, :, s % page] = bound(f64(k)[r], src[r])
        assert (np.abs(have - want) <= limit).all(), name   # values as they were given, all else as it was
    # without a rotation, and the queries in place
    again_k, again_v = k_pool.clone(), v_pool.clone()
    assert jp.append(k, v, slots.to(DEV, torch.int32), k_pool, v_pool) is None
    assert torch.equal(again_v, v_pool)
    s = next(s for s in slots.tolist() if 0 <= s < n_blocks * page)
    assert torch.equal(k_pool[s // page, :, s % page], k[slots.tolist().index(s)])
    mine = q.clone()
    assert jp.append(k, v, slots.to(DEV, torch.int32), k_pool, v_pool, positions=positions.to(DEV, torch.int32), rope_theta=1e4, q=mine, q_out=mine) is mine
    assert torch.equal(mine, got) and torch.equal(k_pool, again_k)


@gpu
def test_no_rows_go_nowhere():
    k_pool = torch.randn((3, 2, 16, 128), device=DEV).bfloat16()
    keep = k_pool.clone()
    none = torch.empty((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    q = jp.append(none, none, ints([]), k_pool, k_pool, positions=ints([]), rope_theta=1e4, q=none)
    assert q.shape == (0, 2, 128) and torch.equal(k_pool, keep)


# ---- attention ------------------------------------------------------------------------------------------------------------------


class Batch:
    """A ragged batch over pages that lie anywhere; places nobody wrote hold NaN."""

    def __init__(self, dtype, heads, kv_heads, page, requests, dim=128, order="block-head-slot", seed=0, spare=3, pad_rows=0, spread=1.0):
        gen = torch.Generator().manual_seed(seed + 17 * len(requests) + page)
        self.page, self.scale = page, dim ** -0.5
        self.new = [b for _, b in requests]
        self.lengths = [a + b for a, b in requests]
        need = [-(-x // page) for x in self.lengths]
        width, n_blocks = max([1, *need]) + 2, sum(need) + spare
        at = torch.randperm(n_blocks, generator=gen).tolist()
        self.table = np.full((len(requests), width), -1)
        for i, x in enumerate(need):
            self.table[i, :x] = [at.pop() for _ in range(x)]
        self.k, self.v = make_pool(dtype, n_blocks, kv_heads, page, dim, order, gen, fill=float("nan"))
        for i, x in enumerate(self.lengths):
            for j in range(need[i]):
                m = min(page, x - j * page)
                for pool, scale in ((self.k, spread), (self.v, 1.0)):
                    pool[int(self.table[i, j]), :, :m] = (torch.randn((kv_heads, m, dim), generator=gen) * scale).to(DEV, dtype)
        self.rows = sum(self.new)
        self.q = torch.randn((self.rows + pad_rows, heads, dim), generator=gen).to(DEV, dtype)
        self.row_start = starts(self.new)

    def run(self, workspace, max_new=None, table=None, **kw):
        t = torch.from_numpy(self.table if table is None else table).to(DEV, torch.int32)
        return jp.attention(self.q, self.k, self.v, t, ints(self.row_start), ints(self.lengths), max(self.new) if max_new is None else max_new,
                            workspace, **kw)

    def check(self, got, table=None, scale=None):
        scale = self.scale if scale is None else scale
        want, size, most = ref.attention(f64(self.q)[:self.rows], f64(self.k), f64(self.v), self.table if table is None else table,
                                         self.row_start, self.lengths, scale, self.page)
        keys = max(self.lengths)
        dim = self.q.shape[-1]
        small = (keys + 2 * dim * most + 32) * 2.0 ** -24
        rounding = BF16 if got.dtype == torch.bfloat16 else 0.0
        off = np.abs(f64(got)[:self.rows] - want)
        limit = (rounding + small) * size + rounding * np.abs(want) + 1e-38
        assert (off <= limit).all(), (float((off - limit).max()), [int(x) for x in np.unravel_index(np.argmax(off - limit), off.shape)])


SHAPES = [
    # heads, kv heads, page, (cached, new) of every request
    (1, 1, 16, [(0, 1)]),
    (4, 4, 16, [(576, 1)]),
    (4, 2, 8, [(0, 5), (31, 1), (32, 1), (33, 2), (100, 5), (7, 0), (63, 1), (64, 3)]),
    (8, 1, 32, [(300, 4), (0, 33), (95, 17)]),
    (6, 2, 64, [(1000, 1), (10, 70), (500, 5), (0, 1)]),
    (2, 2, 128, [(0, 130), (200, 64), (1, 257)]),
    (3, 3, 16, [(777, 100), (0, 300)]),
    (4, 4, 1024, [(1500, 3), (900, 40)]),
    (16, 2, 16, [(40, 16), (3000, 1), (5, 2)]),
    (5, 1, 16, [(129, 13), (64, 51), (0, 77)]),
    (2, 1, 16, [(0, 600)]),
]


@gpu
@pytest.mark.parametrize("heads,kv_heads,page,requests", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_over_pages(workspace, dtype, heads, kv_heads, page, requests):
    b = Batch(dtype, heads, kv_heads, page, requests)
    got = b.run(workspace)
    b.check(got)
    # whatever was expected of the lengths, and once more on the same workspace
    for expected in (0, 1, 40, 5000):
        b.check(b.run(workspace, max_new=expected))
    assert torch.equal(got, b.run(workspace))


MANY_HEADS = [
    # enough key/value heads that tiles of 128 (60 heads) or 256 rows (150) fill the GPU; more than 128: keys are not divided
    (60, 60, 16, [(100, 70), (0, 150), (33, 40), (700, 1)]),
    (120, 60, 32, [(10, 129), (333, 17), (64, 0)]),
    (150, 150, 16, [(30, 70), (0, 41), (257, 2)]),
    (300, 150, 64, [(5, 140), (0, 33), (63, 1)]),
    (200, 200, 16, [(900, 1), (31, 4)]),
    (160, 160, 8, [(70, 30)]),
]


@gpu
@pytest.mark.parametrize("heads,kv_heads,page,requests", MANY_HEADS)
def test_attention_of_many_heads(workspace, heads, kv_heads, page, requests):
    b = Batch(torch.bfloat16, heads, kv_heads, page, requests)
    b.check(b.run(workspace))
    b.check(b.run(workspace, max_new=1))


@gpu
@pytest.mark.parametrize("heads", [60, 150])
def test_holes_and_unseen_values_with_many_heads(workspace, heads):
    requests = [(100, 90), (0, 50)]
    b = Batch(torch.bfloat16, heads, heads, 16, requests)
    t = b.table.copy()
    t[0, [0, 5, 6]] = [-1, b.k.shape[0], 2 ** 31 - 1]
    t[1, 0] = -5
    got = b.run(workspace, table=t)
    b.check(got, table=t)
    assert (got[90:106] == 0).all()
    want = b.run(workspace)
    for bad in (float("nan"), float("inf")):
        c = Batch(torch.bfloat16, heads, heads, 16, requests)
        pos = 100 + 60
        c.k[int(c.table[0, pos // 16]), :, pos % 16, 5] = bad
        c.v[int(c.table[0, pos // 16]), :, pos % 16, 7] = bad
        got = c.run(workspace)
        assert torch.equal(got[:60], want[:60]) and torch.equal(got[90:], want[90:])
        assert not torch.isfinite(got[60:90, :, 7]).any()


@gpu
@pytest.mark.parametrize("requests", [[(3000, 40), (0, 33)], [(0, 33)] * 6 + [(3000, 40)]])
def test_a_long_cache_among_many_heads(workspace, requests):
    """Tiles of 128 and of 256 rows whose keys are divided; with pages that are not there, values that are no numbers, and in place."""
    b = Batch(torch.bfloat16, 60, 60, 16, requests)
    want = b.run(workspace)
    b.check(want)
    long = int(np.argmax(b.lengths))
    t = b.table.copy()
    t[long, [0, 7, 100, 150, 151]] = [-1, b.k.shape[0], 2 ** 31 - 1, -2, -3]
    b.check(b.run(workspace, table=t), table=t)
    c = Batch(torch.bfloat16, 60, 60, 16, requests)
    new = requests[long][1]
    pos, at = 3000 + new // 2, c.row_start[long] + new // 2
    c.v[int(c.table[long, pos // 16]), :, pos % 16, 7] = float("inf")
    got = c.run(workspace)
    assert torch.equal(got[:at], want[:at]) and torch.equal(got[c.row_start[long + 1]:], want[c.row_start[long + 1]:])
    assert (got[at:c.row_start[long + 1], :, 7] == float("inf")).all()
    got[at:c.row_start[long + 1], :, 7] = want[at:c.row_start[long + 1], :, 7]
    assert torch.equal(got, want)
    assert b.run(workspace, out=b.q) is b.q and torch.equal(b.q, want)


@gpu
@pytest.mark.parametrize("heads,requests", [(20, [(0, 1)] * 5 + [(2000, 200)]), (20, [(0, 1)] * 19 + [(2000, 200)]), (4, [(3000, 200), (10, 3)]),
                                            (64, [(0, 2)] * 6 + [(1500, 36)]), (65, [(0, 2)] * 6 + [(1500, 36)])])
def test_tall_tiles_put_together(workspace, heads, requests):
    """All rows of tiles of 128, 256 and 64 whose keys are divided; and as many heads as keys are divided for, and one more."""
    b = Batch(torch.bfloat16, heads, heads, 32, requests)
    got = b.run(workspace)
    b.check(got)
    assert torch.equal(got, b.run(workspace))


@gpu
@pytest.mark.parametrize("heads,kv_heads,requests", [(80, 80, [(100, 120), (0, 50)]), (200, 200, [(100, 120), (0, 50)]), (32, 4, [(100, 400), (0, 150)]),
                                                     (60, 60, [(1000, 120)] + [(0, 1)] * 5), (60, 60, [(1000, 120)] + [(0, 1)] * 7), (32, 4, [(2500, 33), (0, 500)])])
def test_tall_tiles(workspace, heads, kv_heads, requests):
    """Tiles of 128, 256 and 64 rows, the keys of one request divided in the last three: pages that are not there, infinities that some rows see, in
    place of the queries."""
    b = Batch(torch.bfloat16, heads, kv_heads, 16, requests)
    want = b.run(workspace)
    b.check(want)
    t = b.table.copy()
    t[0, [0, 5, 6]] = [-1, b.k.shape[0], 2 ** 31 - 1]
    t[1, 0] = -5
    b.check(b.run(workspace, table=t), table=t)
    c = Batch(torch.bfloat16, heads, kv_heads, 16, requests)
    cached, new = requests[0]
    pos = cached + new // 2
    c.v[int(c.table[0, pos // 16]), :, pos % 16, 7] = float("inf")
    got = c.run(workspace)
    sees = slice(new // 2, new)
    assert (got[sees, :, 7] == float("inf")).all()
    got[sees, :, 7] = want[sees, :, 7]
    assert torch.equal(got, want)
    assert b.run(workspace, out=b.q) is b.q and torch.equal(b.q, want)


@gpu
@pytest.mark.parametrize("heads,kv_heads,requests,gone", [(1, 1, [(13000, 1)], 11500), (1, 1, [(9000, 30)], 6400), (32, 4, [(6400, 33), (0, 500)], 6000)])
def test_old_pages_that_were_dropped(workspace, heads, kv_heads, requests, gone):
    """Divided keys whose first pieces hold nothing (more of them than are put together at a time), and scores far below 0 behind them."""
    b = Batch(torch.bfloat16, heads, kv_heads, 16, requests)
    b.q += 4.0
    b.k -= 4.0
    b.table[0, :gone // 16] = -1
    got = b.run(workspace)
    b.check(got)
    assert got[:requests[0][1]].any()


@gpu
@pytest.mark.parametrize("heads,kv_heads,requests", [(30, 30, [(0, 1)] * 10 + [(2000, 300)]), (20, 20, [(0, 1)] * 20 + [(2000, 200)]), (32, 4, [(3000, 200), (10, 300)]),
                                                     (64, 64, [(0, 2)] * 7 + [(1500, 100)]), (65, 65, [(0, 2)] * 7 + [(1500, 100)])])
def test_divided_keys_of_tall_tiles(workspace, heads, kv_heads, requests):
    """Tiles of 128, 256 and 64 rows: requests of more than 96 rows, more than 512 tiles of 32.  Keys are divided for up to 64 heads."""
    b = Batch(torch.bfloat16, heads, kv_heads, 32, requests)
    got = b.run(workspace)
    b.check(got)
    assert torch.equal(got, b.run(workspace))


def many_requests(n, most_cached, most_new, seed):
    rng = np.random.default_rng(seed)
    requests = [(int(rng.integers(0, most_cached + 1)), int(rng.integers(0, most_new + 1))) for _ in range(n)]
    requests[n // 3] = (3000, 2)       # one long cache among them
    requests[-1] = (5, 1)
    return requests


@gpu
@pytest.mark.parametrize("n,most_cached,most_new,heads,kv_heads", [
    (64, 100, 3, 4, 2), (65, 100, 3, 4, 2), (200, 300, 1, 2, 2), (1000, 40, 2, 2, 1), (1025, 20, 1, 16, 1), (4097, 12, 1, 1, 1), (16384, 3, 1, 1, 1),
    (70, 60, 40, 4, 1), (130, 200, 17, 8, 2),
])
def test_attention_of_many_requests(workspace, n, most_cached, most_new, heads, kv_heads):
    b = Batch(torch.bfloat16, heads, kv_heads, 16, many_requests(n, most_cached, most_new, n))
    got = b.run(workspace)
    b.check(got)
    b.check(b.run(workspace, max_new=100))
    assert torch.equal(got, b.run(workspace))


@gpu
@pytest.mark.parametrize("n", [70, 3000])
def test_many_requests_without_tokens(workspace, n):
    b = Batch(torch.bfloat16, 2, 2, 16, [(20, 0)] * (n - 1) + [(30, 2)])
    b.check(b.run(workspace))
    b = Batch(torch.bfloat16, 2, 2, 16, [(20, 0)] * n, pad_rows=1)
    out = torch.full_like(b.q, 3.0)
    b.run(workspace, out=out)
    assert (out == 3.0).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv_heads,requests", [(4, 2, [(500, 3), (2000, 1)]), (4, 4, [(0, 300), (1700, 70)]), (60, 60, [(0, 150)]), (150, 150, [(9, 70)])])
def test_results_in_place_of_the_queries(workspace, dtype, heads, kv_heads, requests):
    b = Batch(dtype, heads, kv_heads, 16, requests)
    want, q = b.run(workspace), b.q.clone()
    assert b.run(workspace, out=b.q) is b.q
    assert torch.equal(b.q, want) and not torch.equal(b.q, q)


@gpu
@pytest.mark.parametrize("new", [2, 60])
def test_pages_of_several_requests(workspace, new):
    """Branches that share a prefix name the same pages; a page may even be named twice in a row."""
    b = Batch(torch.bfloat16, 4, 2, 16, [(160 + 5, new), (160 + 9, new), (160, new)])
    b.table[1:, :10] = b.table[0, :10]
    b.table[2, 3] = b.table[2, 4]
    b.check(b.run(workspace))


@gpu
def test_rows_of_requests_that_overlap_spoil_no_later_call():
    """A row_start that makes no sense: more pieces of work than a launch has room for.  Later calls on the workspace are right."""
    workspace = jp.Workspace(DEV)
    b = Batch(torch.bfloat16, 4, 2, 16, [(4000, 1), (50, 2), (3000, 1)])
    want = b.run(workspace)
    n = 60
    table = torch.from_numpy(np.repeat(b.table[:1], n, 0)).to(DEV, torch.int32)
    for ends in ([0, 4], [4, 0], [0, 1]):
        row_start = ints((ends * n)[:n + 1])
        for expected in (1, 100):
            jp.attention(b.q, b.k, b.v, table, row_start, ints([4001] * n), expected, workspace)
    assert torch.equal(b.run(workspace), want)


@gpu
def test_a_workspace_made_behind_work_and_used_on_another_stream():
    b = Batch(torch.bfloat16, 4, 2, 16, [(4000, 1), (300, 3)])
    want = b.run(jp.Workspace(DEV))
    dirt = torch.full_like(jp.Workspace(DEV).buf, 1)
    torch.cuda.synchronize()
    del dirt                                 # (the next workspace may get this memory)
    x = torch.randn((4096, 4096), device=DEV)
    for _ in range(20):
        x = x @ x * 1e-2
    side = torch.cuda.Stream()
    got = b.run(jp.Workspace(DEV), stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@gpu
def test_two_graphs_share_a_workspace(workspace):
    """Replayed one after the other, with eager calls on the same workspace between them."""
    batches = [Batch(torch.bfloat16, 4, 2, 16, r) for r in ([(3000, 1), (700, 4)], [(2500, 40), (100, 90)], many_requests(100, 60, 2, 1))]
    want = [b.run(workspace) for b in batches]
    graphs, outs = [], []
    for b in batches:
        args = b.q, b.k, b.v, torch.from_numpy(b.table).to(DEV, torch.int32), ints(b.row_start), ints(b.lengths), max(b.new), workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = jp.attention(*args)
        graphs.append((graph, args))
        outs.append(out)
    for _ in range(4):
        for (graph, _), out, w, b in zip(graphs, outs, want, batches):
            out.zero_()
            graph.replay()
            assert torch.equal(out, w)
            assert torch.equal(b.run(workspace), w)


@gpu
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_over_pools_in_any_order(workspace, dtype, order):
    for requests in ([(70, 3), (200, 1)], [(40, 150), (0, 300)]):
        b = Batch(dtype, 4, 2, 16, requests, order=order)
        b.check(b.run(workspace))


@gpu
@pytest.mark.parametrize("dim", [2, 6, 64, 130, 256])
def test_check_mode_takes_any_even_head_size(dim):
    b = Batch(torch.float32, 4, 2, 16, [(70, 3), (0, 40)], dim=dim)
    b.check(b.run(None))


@gpu
@pytest.mark.parametrize("new", [1, 5, 40, 260])
def test_rows_and_columns_of_other_tensors(workspace, new):
    """Queries out of a fused projection, results into a wider tensor: what lies around them stays as it is."""
    b = Batch(torch.bfloat16, 4, 4, 16, [(100, new), (33, new)], pad_rows=5)
    fused = torch.full((b.q.shape[0], 12, 128), float("nan"), device=DEV).bfloat16()
    fused[:, 4:8] = b.q
    want, b.q = b.run(workspace)[:b.rows], fused[:, 4:8]
    wide = torch.full((b.q.shape[0] + 2, 9, 136), 7.0, device=DEV).bfloat16()
    keep = wide.clone()
    out = wide[1:-1, 2:6, :128]
    assert b.run(workspace, out=out) is out
    assert torch.equal(out[:b.rows], want)
    out[:b.rows] = keep[1:1 + b.rows, 2:6, :128]
    assert torch.equal(wide, keep)   # rows behind the last one among it


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pages_that_are_not_there(workspace, dtype):
    """Table entries outside the pool: their positions are not seen; rows that see nothing get zeros."""
    for requests in ([(90, 4), (40, 2), (0, 3)], [(200, 160), (0, 140), (64, 33)]):
        b = Batch(dtype, 4, 2, 16, requests)
        n_blocks = b.k.shape[0]
        t = b.table.copy()
        t[0, [0, 2, 3]] = [-1, n_blocks, 2 ** 31 - 1]
        t[1, :] = -(2 ** 31)                 # nothing left of this one
        t[2, 0] = -5                         # its first rows see nothing
        got = b.run(workspace, table=t)
        b.check(got, table=t)
        assert (got[b.row_start[1]:b.row_start[2]] == 0).all()
        if requests[2][0] == 0:
            assert (got[b.row_start[2]] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("requests", [[(50, 6)], [(20, 40), (70, 3)], [(100, 200)]])
def test_values_a_row_does_not_see_do_not_reach_it(workspace, dtype, requests):
    """NaN and infinities in the keys and values of later tokens of the same step."""
    b = Batch(dtype, 2, 2, 16, requests)
    want = b.run(workspace)
    for bad in (float("nan"), float("inf"), -float("inf")):
        c = Batch(dtype, 2, 2, 16, requests)
        cached, new = requests[0]
        for t in (new - 1, new // 2):        # the last token's keys and values, and one in the middle
            pos = cached + t
            c.k[int(c.table[0, pos // 16]), :, pos % 16, 5] = bad
            c.v[int(c.table[0, pos // 16]), :, pos % 16] = bad
        got = c.run(workspace)
        clean = [r for r in range(b.rows) if not (new // 2 <= r < new)]
        assert torch.equal(got[clean], want[clean]), bad
        assert not torch.isfinite(got[new // 2]).all()


@gpu
def test_infinite_values_that_are_seen_come_out(workspace):
    for requests in ([(50, 6)], [(100, 200)]):
        b = Batch(torch.bfloat16, 2, 2, 16, requests)
        cached, new = requests[0]
        pos = cached + new // 2
        page = int(b.table[0, pos // 16])
        b.v[page, 0, pos % 16, 3], b.v[page, 0, pos % 16, 4], b.v[page, 0, pos % 16, 5] = float("inf"), -float("inf"), float("nan")
        got = b.run(workspace).float().cpu()
        after, before = got[new // 2:, 0], got[:new // 2, 0]
        assert torch.isfinite(before).all()
        assert (after[:, 3] == float("inf")).all() and (after[:, 4] == -float("inf")).all() and torch.isnan(after[:, 5]).all()
        rest = after.clone()
        rest[:, 3:6] = 0
        assert torch.isfinite(rest).all() and torch.isfinite(got[:, 1]).all()


@gpu
@pytest.mark.parametrize("requests", [[(600, 3)], [(100, 200)]])
def test_scores_far_apart(workspace, requests):
    """Scores of spread 40: a few keys carry a row, and the running maximum moves by more than 2^8 at a time."""
    b = Batch(torch.bfloat16, 4, 2, 16, requests, spread=40.0)
    b.check(b.run(workspace))
    b = Batch(torch.bfloat16, 4, 2, 16, requests)
    b.check(b.run(workspace, scale=3.0), scale=3.0)


@gpu
@pytest.mark.parametrize("requests", [[(3000, 2)], [(2500, 40), (0, 600)]])
def test_values_near_the_largest(workspace, requests):
    """2^104 times normal ones: sums of 3000 weights of up to 2^8 stay below 2^128."""
    b = Batch(torch.bfloat16, 32, 4, 16, requests)
    b.v *= 2.0 ** 104
    b.check(b.run(workspace))


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lengths_that_make_no_sense_stay_inside_the_buffers(workspace, dtype):
    """Lengths shorter than the new tokens, negative, or beyond the table; rows beyond n_rows."""
    b = Batch(dtype, 4, 2, 16, [(90, 4), (40, 60), (0, 3)])
    b.lengths = [2, 40, 2 ** 31 - 1]
    t = b.table.copy()
    t[2, :] = t[0, 0]
    b.k[torch.isnan(b.k)], b.v[torch.isnan(b.v)] = 0.5, 0.25
    got = b.run(workspace, table=t)
    b.check(got, table=t)
    assert (got[:2] == 0).all() and (got[4:24] == 0).all()
    b.lengths = [-5, -(2 ** 31), 0]
    assert (b.run(workspace)[:b.rows] == 0).all()
    full = torch.zeros((b.rows + 50, 4, 128), dtype=dtype, device=DEV)
    out = full[:b.rows]
    jp.attention(b.q, b.k, b.v, torch.from_numpy(b.table).to(DEV, torch.int32), ints([0, 4, 64, 100]), ints([94, 100, 3]), 60, workspace, out=out)
    assert (full[b.rows:] == 0).all()
    jp.attention(b.q, b.k, b.v, torch.from_numpy(b.table).to(DEV, torch.int32), ints([5, 2, -7, 3]), ints([94, 100, 3]), 60, workspace, out=out)
    torch.cuda.synchronize()


@gpu
def test_no_requests_and_no_rows(workspace):
    k = torch.zeros((2, 1, 16, 128), dtype=torch.bfloat16, device=DEV)
    q = torch.zeros((3, 1, 128), dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 4.0)
    t = torch.zeros((0, 1), dtype=torch.int32, device=DEV)
    jp.attention(q, k, k, t, ints([0]), ints([]), 1, workspace, out=out)
    jp.attention(q, k, k, torch.zeros((2, 1), dtype=torch.int32, device=DEV), ints([0, 0, 0]), ints([5, 0]), 1, workspace, out=out)
    assert (out == 4.0).all()
    assert jp.attention(q[:0], k, k, t, ints([0]), ints([]), 1, workspace).shape == (0, 1, 128)
    # a table without columns: nothing is there
    assert (jp.attention(q, k, k, torch.zeros((1, 0), dtype=torch.int32, device=DEV), ints([0, 3]), ints([9]), 1, workspace) == 0).all()


@gpu
@pytest.mark.parametrize("new", [1, 200])
def test_pools_beyond_32_bit_offsets(workspace, new):
    """Pools of 4.3 GB each: 2^31 elements lie between the pages of one request."""
    n_blocks, heads, page = 66000, 8, 32
    k = torch.empty((n_blocks, heads, page, 128), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    blocks = [n_blocks - 1, 3, n_blocks - 2, 0, 65999 // 2, 7, n_blocks - 3, 9]
    gen = torch.Generator().manual_seed(5)
    small_k, small_v = (torch.randn((len(blocks), heads, page, 128), generator=gen).to(DEV, torch.bfloat16) for _ in range(2))
    k[blocks], v[blocks] = small_k, small_v
    q = torch.randn((new, heads, 128), generator=gen).to(DEV, torch.bfloat16)
    args = ints([0, new]), ints([250]), new, workspace
    far = jp.attention(q, k, v, ints(blocks)[None], *args)
    near = jp.attention(q, small_k, small_v, ints(range(len(blocks)))[None], *args)
    assert torch.equal(far, near) and torch.isfinite(far).all()
    slot = ints([(n_blocks - 1) * page + 5])
    jp.append(small_k[:1, :, 0], small_v[:1, :, 0], slot, k, v)
    assert torch.equal(k[n_blocks - 1, :, 5], small_k[0, :, 0]) and torch.equal(v[n_blocks - 1, :, 5], small_v[0, :, 0])


@gpu
def test_another_stream(workspace):
    b = Batch(torch.bfloat16, 4, 2, 16, [(300, 3), (50, 1)])
    want = b.run(workspace)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = b.run(jp.Workspace(DEV), stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@gpu
def test_results_made_for_another_stream_are_not_written_by_this_one(workspace):
    """Memory that the current stream has freed, with its work on it still ahead, is not what a call on another stream gets."""
    b = Batch(torch.bfloat16, 4, 2, 16, [(300, 3), (50, 1)])
    lengths, table, at = ints(b.lengths), torch.from_numpy(b.table).to(DEV, torch.int32), ints(b.row_start)
    n_new, owned, free, count = ints(b.new), ints([b.table.shape[1]] * 2), ints([]), ints([0])
    slots, positions = torch.full((4,), -1, dtype=torch.int32, device=DEV), ints([5, 6, 7, 8])
    probs, u = torch.softmax(torch.randn((4, 100), device=DEV), -1), torch.rand(4, device=DEV)
    tokens, new_k = ints([3, 1, 4, 1]), b.q[:, :2].contiguous()
    cfg, stage, _ = small_stage("bf16", 8)
    pools = [torch.zeros((2, 4, 8, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    hidden, step = torch.randn((4, 1024), device=DEV).bfloat16(), jp.Step(ints([0, 4]), ints([0, 1, 2, 3]), ints([0, 1, 2, 3]), ints([4]), None, None, None)
    stage_table, space = ints([1])[None], jp.Workspace(DEV)
    calls = [lambda s: [jp.attention(b.q, b.k, b.v, table, at, lengths, 3, space, stream=s)],
             lambda s: [jp.append(new_k, new_k, slots, b.k, b.v, positions=positions, rope_theta=1e4, q=b.q, stream=s)],
             lambda s: list(jp.extend(lengths, n_new, owned, table, free, count, 16, 4, stream=s)),
             lambda s: list(jp.verify(tokens, probs, at, u, u[:2].clone(), space, lengths=lengths, stream=s)),
             lambda s: [jp.prefill(stage, hidden, step, *pools, stage_table, 4, space, stream=s)]]
    side, x = torch.cuda.Stream(), torch.randn((4096, 4096), device=DEV)
    for call in calls:
        want = [t.clone() for t in call(None)]
        freed = [torch.empty(t.untyped_storage().nbytes(), dtype=torch.uint8, device=DEV) for t in call(None)[:1] for _ in range(20)]
        torch.cuda.synchronize()
        for _ in range(30):
            x = x @ x * 1e-2
        for f in freed:
            f.fill_(77)
        del f, freed
        got = call(side)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))


@gpu
def test_two_streams_at_once():
    """Calls that overlap, each stream with a workspace of its own."""
    batches = [Batch(torch.bfloat16, 4, 2, 16, r, seed=s) for s, r in enumerate(([(3000, 2), (900, 1)], [(2500, 70), (40, 3)]))]
    spaces, streams = [jp.Workspace(DEV) for _ in batches], [torch.cuda.Stream() for _ in batches]
    want = [b.run(w) for b, w in zip(batches, spaces)]
    args = [(b.q, b.k, b.v, torch.from_numpy(b.table).to(DEV, torch.int32), ints(b.row_start), ints(b.lengths), max(b.new), w)
            for b, w in zip(batches, spaces)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        got.append([jp.attention(*a, stream=s) for a, s in zip(args, streams)])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for run in got for x, y in zip(run, want))


@gpu
def test_more_rows_than_a_launch_has_workgroups_in_a_line():
    """2^24 rows of two features and more: 2^32 threads if a row had a workgroup of its own in one line of them."""
    rows = (1 << 24) + 3
    pools = [torch.zeros((rows // 65536 + 1, 1, 65536, 2), device=DEV) for _ in "kv"]
    k, v = torch.rand((rows, 1, 2), device=DEV), torch.rand((rows, 1, 2), device=DEV)
    slots = torch.arange(rows, device=DEV, dtype=torch.int32).flip(0)
    jp.append(k, v, slots, *pools)
    for x, pool in zip((k, v), pools):
        assert torch.equal(pool.view(-1, 2)[:rows], x[:, 0].flip(0)) and not pool.view(-1, 2)[rows:].any()


@gpu
def test_more_rows_and_heads_than_a_launch_has_workgroups_in_a_line():
    """Check mode has a wave per row and head: 2^26 and more of them."""
    rows, heads = (1 << 20) + 5, 64
    q = torch.rand((rows, heads, 2), device=DEV)
    k, v = torch.zeros((1, 1, 8, 2), device=DEV), torch.rand((1, 1, 8, 2), device=DEV)
    out = torch.full_like(q, 9.0)
    jp.attention(q, k, v, ints([0])[None], ints([0, rows]), ints([rows]), rows, scale=1.0, out=out)
    # (a table of one page of eight: row r sees the first r + 1 positions, the last rows all eight; keys of 0 weigh the same, and sums of
    # eight numbers below 1 are off by at most 8 x 2^-24)
    for r in (0, 1, 5, 7, 100, rows // 2, rows - 1):
        want = v[0, 0, :min(r + 1, 8)].double().mean(0)
        assert (out[r].double() - want).abs().max() <= 1e-6, r
    assert ((out[7:] - out[7]).abs() <= 1e-6).all()


@gpu
@pytest.mark.parametrize("max_new", [1, 100])
def test_more_pieces_of_work_than_a_launch_has_workgroups_in_a_line(workspace, max_new):
    """2^24 requests times key/value heads, of 256 threads and more each."""
    n, heads = 16384, 1024
    gen = torch.Generator().manual_seed(4)
    q1, k, v = ((torch.randn(shape, generator=gen)).to(DEV, torch.bfloat16) for shape in ((1, heads, 128), (1, heads, 8, 128), (1, heads, 8, 128)))
    lengths = [1 + i % 8 for i in range(n)]
    out = torch.full((n, heads, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    jp.attention(q1.expand(n, heads, 128), k, v, torch.zeros((n, 1), dtype=torch.int32, device=DEV), ints(range(n + 1)), ints(lengths), max_new, workspace, out=out)
    want, size, most = ref.attention(f64(q1.expand(8, heads, 128)), f64(k), f64(v), np.zeros((8, 1), dtype=np.int64), list(range(9)), lengths[:8], 128 ** -0.5, 8)
    off = np.abs(f64(out[:8]) - want)
    assert (off <= (BF16 + (8 + 256 * most + 32) * 2.0 ** -24) * size + BF16 * np.abs(want)).all()
    assert (out.view(n // 8, 8, heads, 128) == out[:8]).all()


@gpu
def test_a_call_on_another_stream_is_captured():
    """A graph whose call is on a stream of its own, replayed with eager calls in between."""
    batches = [Batch(torch.bfloat16, 4, 2, 16, r) for r in ([(3000, 1), (700, 4)], [(500, 40), (100, 90)])]
    space, eager = jp.Workspace(DEV), jp.Workspace(DEV)
    want = [b.run(eager) for b in batches]
    args = [(b.q, b.k, b.v, torch.from_numpy(b.table).to(DEV, torch.int32), ints(b.row_start), ints(b.lengths), max(b.new), space) for b in batches]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        outs = [jp.attention(*a, stream=side) for a in args]
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for out in outs:
            out.zero_()
        graph.replay()
        assert all(torch.equal(b.run(eager), w) for b, w in zip(batches, want))
        assert all(torch.equal(out, w) for out, w in zip(outs, want))


# ---- verification ----------------------------------------------------------------------------------------------------------------


def make_verify(n, most, vocab, dtype, from_draft, seed):
    gen = torch.Generator().manual_seed(seed)
    new = torch.randint(0, most + 2, (n,), generator=gen).tolist()
    new[0] = most + 1
    rows = sum(new)
    g = 2.0 * torch.randn((rows, vocab), generator=gen)
    target = torch.softmax(g, -1).to(dtype)
    draft = torch.softmax(g + 0.5 * torch.randn((rows, vocab), generator=gen), -1).to(dtype)
    tokens = torch.randint(vocab, (rows,), generator=gen, dtype=torch.int32)
    tokens[1:] = torch.multinomial(draft.float(), 1, generator=gen)[:-1, 0].int()
    if not from_draft:
        sure = 0.8 * torch.rand(rows - 1, generator=gen)
        target = target.float() * 0.5
        target[torch.arange(rows - 1), tokens[1:].long()] += sure
        target = target.to(dtype)
        draft = None
    return new, target, draft, tokens, torch.rand(rows, generator=gen), torch.rand(n, generator=gen)


def check_verify(workspace, new, target, draft, tokens, u_accept, u_sample):
    lengths = [10 + 3 * i for i in range(len(new))]
    got = jp.verify(tokens.to(DEV), target.to(DEV), ints(starts(new)), u_accept.to(DEV), u_sample.to(DEV), workspace,
                    draft_probs=None if draft is None else draft.to(DEV), lengths=ints(lengths))
    want = ref.verify(tokens.tolist(), target.double().numpy(), None if draft is None else draft.double().numpy(), starts(new),
                      u_accept.tolist(), u_sample.tolist(), lengths)
    for name, g, w in zip(jp.Verdict._fields, got, want):
        assert g.tolist() == w, (name, g.tolist()[:20], w[:20])
    return want


@gpu
@pytest.mark.parametrize("n,most,vocab", [(1, 4, 32000), (3, 0, 1), (5, 3, 7), (4, 2, 64), (6, 5, 1000), (17, 8, 4097), (2, 3, 131072), (3, 1500, 50), (40, 2, 65537)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("from_draft", [True, False])
def test_verification(workspace, n, most, vocab, dtype, from_draft):
    if n * most * vocab > 3e6:
        most = 2
    want = check_verify(workspace, *make_verify(n, most, vocab, dtype, from_draft, n * vocab + most))
    assert len(want[0]) == n


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [524288, 700001])
def test_verification_of_a_very_large_vocabulary(workspace, dtype, vocab):
    """Slices of more than one round each."""
    check_verify(workspace, *make_verify(2, 1, vocab, dtype, True, vocab))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,most,vocab", [(64, 1, 65536), (61, 1, 65537), (66, 2, 65537), (260, 0, 16385), (1100, 1, 60)])
def test_verification_of_many_requests(workspace, dtype, n, most, vocab):
    """So many that slices are longer (more than 1024 short ones), and just not so many."""
    check_verify(workspace, *make_verify(n, most, vocab, dtype, most != 2, vocab))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verification_of_unusual_numbers(workspace, dtype):
    nan, inf = float("nan"), float("inf")
    V = 300
    flat = torch.full((V,), 1.0 / 256)
    one = torch.zeros(V)
    one[123] = 1.0
    odd = flat.clone()
    odd[[0, 5, 70, 299]] = torch.tensor([nan, inf, -0.25, nan])
    zero = torch.zeros(V)
    cases = [  # target, draft, token, u_accept, u_sample; two rows per request, the second row's target is flat
        (flat, flat, 4, 0.5, 0.5), (flat, flat, 4, 1.0, 0.25), (one, flat, 123, 0.9, 0.1), (one, flat, 7, 0.0, 0.7), (one, one, 7, 0.3, 0.7),
        (zero, flat, 4, 0.0, 0.5), (zero, zero, 4, 0.0, 0.5), (odd, flat, 9, 1.0, 0.999), (flat, odd, 5, 0.5, 0.3), (odd, zero, 0, 0.5, 0.0),
        (flat, flat, -1, 0.0, 0.4), (flat, one, V, 0.0, 0.4), (flat, one, 2 ** 31 - 1, 0.0, 0.4), (one, flat, 4, nan, nan), (flat, one, 4, nan, 1.0),
        (flat, one, 123, 1.0, -0.5), (flat, one, 123, 1.0, 7.0), (flat, one, 123, 1.0, nan), (zero, one, 123, 0.5, 0.5)]
    for with_draft in (True, False):
        target = torch.stack([x for t, d, *_ in cases for x in (t, flat)]).to(dtype)
        draft = torch.stack([x for t, d, *_ in cases for x in (d, flat)]).to(dtype) if with_draft else None
        tokens = torch.tensor([x for c in cases for x in (3, c[2])], dtype=torch.int32)
        u_accept = torch.tensor([x for c in cases for x in (c[3], 0.5)])
        check_verify(workspace, [2] * len(cases), target, draft, tokens, u_accept, torch.tensor([c[4] for c in cases]))


@gpu
def test_verification_leaves_other_rows_alone_and_works_in_place(workspace):
    new, target, draft, tokens, ua, us = make_verify(4, 3, 500, torch.float32, True, 3)
    want = check_verify(workspace, new, target, draft, tokens, ua, us)
    # a batch of wider rows, read every second one, with rows behind the last
    rows = sum(new)
    wide = torch.full((2 * rows + 8, 512), float("nan"), device=DEV)
    wide[0:2 * rows:2, :500] = target.to(DEV)
    wide_q = torch.full((rows + 4, 501), float("nan"), device=DEV)
    wide_q[:rows, :500] = draft.to(DEV)
    pad = lambda t: torch.cat([t, t[:4]]).to(DEV)  # noqa: E731
    lengths = ints([10 + 3 * i for i in range(4)])
    got = jp.verify(pad(tokens), wide[::2, :500], ints(starts(new)), pad(ua), us.to(DEV), workspace, draft_probs=wide_q[:, :500], lengths=lengths, in_place=True)
    assert got.lengths is lengths and lengths.tolist() == want[3]
    assert got.emitted[:rows].tolist() == want[2] and got.next_token.tolist() == want[1]
    got = jp.verify(pad(tokens), wide[::2, :500], ints(starts(new)), pad(ua), us.to(DEV), workspace)
    assert got.lengths is None
    # row starts that make no sense stay inside the buffers
    jp.verify(pad(tokens), wide[::2, :500], ints([-4, 2, 1, 10 ** 6, 2 * 10 ** 6]), pad(ua), us.to(DEV), workspace)
    torch.cuda.synchronize()


@gpu
def test_tokens_come_out_as_often_as_the_target_says(workspace):
    """20000 requests of one drafted token, in two calls: the first emitted token has the target's distribution (five tokens; a share of
    p is off by at most 5 sqrt(p (1 - p) / 20000) but for one draw in a million)."""
    n, V = 10000, 5
    target = torch.tensor([0.1, 0.4, 0.05, 0.25, 0.2], device=DEV)
    draft = torch.tensor([0.3, 0.1, 0.3, 0.2, 0.1], device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(8)
    count = torch.zeros(V, device=DEV)
    for _ in range(2):
        tokens = torch.zeros(2 * n, dtype=torch.int32, device=DEV)
        tokens[1::2] = torch.multinomial(draft.expand(n, V), 1, generator=gen)[:, 0].int()
        u = torch.rand(3 * n, generator=gen, device=DEV)
        got = jp.verify(tokens, target.expand(2 * n, V), ints(range(0, 2 * n + 1, 2)), u[:2 * n].clone(), u[2 * n:].clone(), workspace,
                        draft_probs=draft.expand(2 * n, V))
        count += torch.bincount(got.emitted[::2].long(), minlength=V)
    p = target.cpu().numpy()
    assert (np.abs(count.cpu().numpy() / (2 * n) - p) <= 5 * np.sqrt(p * (1 - p) / (2 * n))).all(), count


# ---- a step, as a server runs it ---------------------------------------------------------------------------------------------------


class Server:
    """Requests that draft and verify over one pool: two layers of attention, random rows in place of a model.  Everything stays on
    the GPU, in the same buffers from step to step."""

    def __init__(self, page, cached, drafts, vocab, seed):
        gen = torch.Generator().manual_seed(seed)
        self.page, self.n, self.vocab = page, len(cached), vocab
        self.heads, self.kv_heads, self.layers = 4, 2, 2
        width, n_blocks = 24, 24 * len(cached)
        order = torch.randperm(n_blocks, generator=gen)
        self.table = torch.full((self.n, width), -1, dtype=torch.int32)
        shared = [int(order[0]), int(order[1])]            # every request begins with the same two pages
        at = 2
        for i, c in enumerate(cached):
            for j in range(-(-c // page)):
                self.table[i, j] = shared[j] if j < 2 else int(order[at])
                at += j >= 2
        self.table = self.table.to(DEV)
        self.owned, self.lengths = ints([-(-c // page) for c in cached]), ints(cached)
        self.free, self.free_count = ints(order[at:].tolist()), ints([n_blocks - at])
        self.pools = [[torch.randn((n_blocks, self.kv_heads, page, 128), generator=gen).to(DEV, torch.bfloat16) for _ in "kv"] for _ in range(self.layers)]
        self.n_new = ints([d + 1 for d in drafts])
        self.rows = sum(drafts) + self.n
        self.max_rows, self.most = self.rows + 3, max(drafts) + 1
        self.workspace = jp.Workspace(DEV)
        self.inputs = {}
        self.draw(gen)

    def draw(self, gen):
        """The step's random inputs, into the buffers that hold them."""
        H, V, R = self.heads + 2 * self.kv_heads, self.vocab, self.max_rows
        new = dict(qkv=torch.randn((self.layers, R, H, 128), generator=gen).bfloat16(), target=torch.softmax(2 * torch.randn((R, V), generator=gen), -1),
                   u_accept=0.2 * torch.rand(R, generator=gen), u_sample=torch.rand(self.n, generator=gen), tokens=torch.randint(V, (R,), generator=gen).int())
        new["draft"] = torch.softmax(new["target"].log() + 0.3 * torch.randn((R, V), generator=gen), -1)
        for name, x in new.items():
            if name in self.inputs:
                self.inputs[name].copy_(x)
            else:
                self.inputs[name] = x.to(DEV)

    def step(self):
        x = self.inputs
        before = self.lengths.clone()
        s = jp.extend(self.lengths, self.n_new, self.owned, self.table, self.free, self.free_count, self.page, self.max_rows, in_place=True)
        outs = []
        for layer, (k_pool, v_pool) in enumerate(self.pools):
            q, k, v = x["qkv"][layer].split([self.heads, self.kv_heads, self.kv_heads], 1)
            q = jp.append(k, v, s.slots, k_pool, v_pool, positions=s.positions, rope_theta=1e4, q=q)
            outs.append(jp.attention(q, k_pool, v_pool, self.table, s.row_start, s.lengths, self.most, self.workspace)[:self.rows])
        verdict = jp.verify(x["tokens"], x["target"], s.row_start, x["u_accept"], x["u_sample"], self.workspace, draft_probs=x["draft"], lengths=before)
        self.lengths.copy_(verdict.lengths)
        return dict(status=s.status, slots=s.slots, emitted=verdict.emitted[:self.rows], n_accepted=verdict.n_accepted, lengths=verdict.lengths, outs=outs)


def as_lists(result):
    return {k: v.tolist() for k, v in result.items() if k != "outs"}


@gpu
@pytest.mark.parametrize("page,cached,drafts", [(16, [40, 33, 64, 200, 35], [4, 0, 2, 4, 1]), (8, [16, 17], [9, 3]), (32, [70] * 9, [3] * 9)])
def test_steps_of_a_server(page, cached, drafts):
    """Six steps: tables, appends, attention and verification together, against a cache kept in order on the CPU."""
    srv = Server(page, cached, drafts, 600, seed=page)
    gen = torch.Generator().manual_seed(100)
    # what every request has cached, in order: [layer][k|v][request] -> [kv heads, positions, 128]
    table = srv.table.cpu().numpy()
    kept = [[[f64(pool)[table[i, :-(-c // page)]].transpose(1, 0, 2, 3).reshape(srv.kv_heads, -1, 128)[:, :c] for i, c in enumerate(cached)]
             for pool in pools] for pools in srv.pools]
    lengths = list(cached)
    start = starts([d + 1 for d in drafts])
    accepted = 0
    for step in range(6):
        srv.draw(gen)
        got = srv.step()
        assert got["status"].tolist() == [0]
        x = {k: f64(v) for k, v in srv.inputs.items()}
        want = ref.verify(srv.inputs["tokens"].tolist(), x["target"], x["draft"], start, x["u_accept"], x["u_sample"], lengths)
        assert got["n_accepted"].tolist() == want[0] and got["lengths"].tolist() == want[3]
        assert got["emitted"].tolist() == want[2][:srv.rows]
        accepted += sum(want[0])
        for layer in range(srv.layers):
            for i, c in enumerate(lengths):
                rows = slice(start[i], start[i + 1])
                m = start[i + 1] - start[i]
                q, k, v = (x["qkv"][layer][rows, a:b] for a, b in ((0, 4), (4, 6), (6, 8)))
                pos = np.arange(c, c + m)
                bf = lambda a: torch.from_numpy(a).bfloat16().double().numpy()  # noqa: E731
                for what, new in ((0, bf(ref.rotate(k, pos, 1e4))), (1, v)):
                    kept[layer][what][i] = np.concatenate([kept[layer][what][i][:, :c], new.transpose(1, 0, 2)], 1)
                keys, values = kept[layer][0][i], kept[layer][1][i]
                blocks = -(-(c + m) // page)
                pad = np.zeros((srv.kv_heads, blocks * page - c - m, 128))
                pages = [np.concatenate([a, pad], 1).reshape(srv.kv_heads, blocks, page, 128).transpose(1, 0, 2, 3) for a in (keys, values)]
                out, size, most = ref.attention(bf(ref.rotate(q, pos, 1e4)), *pages, np.arange(blocks)[None], [0, m], [c + m], 128 ** -0.5, page)
                # rotated queries and keys may round the other way (a step of 2^-7 of one element in a thousand or so): scores are off by at
                # most 2 x 2^-7 x the largest product, and by the root of 128 less as the products add up
                loose = 2.0 ** -6 * most / np.sqrt(128)
                off = np.abs(f64(got["outs"][layer][rows]) - out)
                assert (off <= (BF16 + loose) * size + BF16 * np.abs(out)).all(), (step, layer, i)
        lengths = want[3]
    assert accepted > 0
    # pages are distinct but for the shared ones
    t = srv.table.cpu().numpy()
    own = [int(b) for i, o in enumerate(srv.owned.tolist()) for b in t[i, 2:o]]
    assert len(set(own)) == len(own) and srv.free_count.item() == 24 * len(cached) - 2 - len(own)


@gpu
def test_a_captured_step_is_replayed():
    """The whole step in a graph, replayed with other inputs and eager work in between: every replay gives what an eager server gives."""
    args = 16, [40, 33, 64, 200, 35], [4, 0, 2, 4, 1], 600
    one, other = Server(*args, seed=3), Server(*args, seed=3)
    gens = [torch.Generator().manual_seed(9) for _ in range(2)]
    for srv, gen in zip((one, other), gens):   # a step outside the graph
        srv.draw(gen)
        srv.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        recorded = one.step()
    for _ in range(5):
        for srv, gen in zip((one, other), gens):
            srv.draw(gen)
        graph.replay()
        want = other.step()
        torch.cuda.synchronize()
        assert as_lists(recorded) == as_lists(want)
        assert all(torch.equal(a, b) for a, b in zip(recorded["outs"], want["outs"]))
        for a, b in zip(one.pools, other.pools):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert torch.equal(one.table, other.table) and one.free_count.tolist() == other.free_count.tolist()


# ---- a stage over pages -------------------------------------------------------------------------------------------------------------


def small_stage(dtype, max_rows, w4_expanded=False):
    """A stage, one oracle per request on demand, and the config; bars are those of the parity tests."""
    import oracle
    from oracle import w4
    from paper_2504_08242_amd import synth_inputs as si
    cfg = dict(si.TINY) if dtype == "f32" else dict(si.LLAMA7B_STAGE, n_layers=2, d_model=1024, n_heads=8, d_ffn=2816)
    if dtype == "w4":
        layers = si.make_w4_layers(cfg, seed=5)
        dev, full = jb.upload_w4_layers(layers), w4.dequantize_layers(layers)
    else:
        layers = full = si.make_layers(cfg, seed=5, bf16=dtype == "bf16")
        dev = jb.upload_layers(layers, dtype)
    stage = jb.Stage(cfg, dtype, dev, max_rows, w4_expanded=w4_expanded)
    torch.cuda.synchronize()
    return cfg, stage, lambda n: oracle.OracleStage(cfg, full, n)


@gpu
@pytest.mark.parametrize("dtype,steps", [
    ("f32", [[37, 5, 0, 16], [1, 3, 20, 1], [1, 1, 1, 1]]),
    ("bf16", [[37, 5, 0, 16], [1, 3, 20, 1], [1, 1, 1, 1], [5, 5, 1, 5]]),     # 58, 25, 4 and 16 rows
    ("bf16", [[300, 0, 140, 64], [1, 200, 1, 1]]),
    ("bf16", [[900, 20, 0, 40], [1, 130, 700, 1], [1, 1, 1, 5]]),             # keys divided among workgroups
    ("bf16", [[2000, 20, 0, 40], [1, 5, 1, 1]]),                              # tiles of 64 rows
    ("bf16", [[2700, 20, 0, 40], [1, 5, 1, 1]]),                              # and of 128
    ("w4", [[37, 5, 0, 16], [1, 3, 7, 1], [1, 1, 1, 1]]),
    ("w4+bf16", [[90, 5, 0, 16], [1, 1, 1, 1]])])
def test_a_stage_over_pages(dtype, steps, workspace):
    """Ragged steps of four requests through a stage, rows of every request and what it caches against the oracle."""
    import helpers
    from paper_2504_08242_amd import synth_inputs as si
    expanded, dtype = dtype == "w4+bf16", dtype.split("+")[0]
    page, spare, n = 16, 3, 4
    most = max(sum(s) for s in steps) + spare
    cfg, stage, new_oracle = small_stage(dtype, most, expanded)
    total = [sum(s[i] for s in steps) for i in range(n)]
    oracles = [new_oracle(max(1, t)) for t in total]
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    hidden = [si.make_hidden(cfg, 5, max(1, t), tag=i, bf16=dtype != "f32") for i, t in enumerate(total)]
    heads, D = cfg["n_heads"], cfg["head_dim"]
    n_blocks = sum(-(-t // page) for t in total) + 2
    gen = torch.Generator().manual_seed(1)
    k_pools, v_pools = (torch.full((cfg["n_layers"], n_blocks, heads, page, D), float("nan"), dtype=td, device=DEV) for _ in "kv")
    table = torch.full((n, max(-(-t // page) for t in total)), -1, dtype=torch.int32, device=DEV)
    free, count = ints(torch.randperm(n_blocks, generator=gen).tolist()), ints([n_blocks])
    lengths, owned = ints([0] * n), ints([0] * n)
    at = [0] * n
    for new in steps:
        rows = sum(new)
        step = jp.extend(lengths, ints(new), owned, table, free, count, page, rows + spare, in_place=True)
        x = torch.full((rows + spare, cfg["d_model"]), 0.5, dtype=td, device=DEV)
        x[:rows] = torch.from_numpy(np.concatenate([h[a:a + m] for h, a, m in zip(hidden, at, new)])).to(DEV, td)
        y = jp.prefill(stage, x, step, k_pools, v_pools, table, max(new), workspace)
        assert step.status.item() == 0
        got, row = y[:rows].float().cpu().numpy(), 0
        for i, m in enumerate(new):
            if m:
                want = oracles[i].prefill_chunk(hidden[i][at[i]:at[i] + m], at[i])
                if dtype == "f32":
                    assert helpers.rel_l2(got[row:row + m], want) <= helpers.F32_REL_L2
                else:
                    helpers.assert_rows_close(got[row:row + m], want, what=f"request {i}, {m} rows at {at[i]}")
            row += m
            at[i] += m
        again = x.clone()
        assert jp.prefill(stage, again, step, k_pools, v_pools, table, 1, workspace, hidden_out=again) is again   # in place, wrong hint
        helpers.assert_rows_close(again[:rows].float().cpu().numpy(), got, bound=1e-6 if dtype == "f32" else helpers.BF16_ROW_REL_L2)
    assert lengths.tolist() == total
    t = table.cpu().numpy()
    for i, m in enumerate(total):
        for which, pools in enumerate((k_pools, v_pools)):
            kept = f64(pools[:, t[i, :-(-m // page)]].transpose(1, 2).reshape(cfg["n_layers"], heads, -1, D)[:, :, :m])
            want = oracles[i].kv[:, which, :, :m]
            if dtype == "f32":
                assert helpers.rel_l2(kept, want) <= helpers.F32_REL_L2
            else:
                helpers.assert_rows_close(kept, want, what=f"cache of request {i}")


@gpu
def test_a_stage_over_pages_in_a_graph(workspace):
    """Decoding steps of a stage, captured: tables, all layers; every replay gives what the same calls give outside."""
    cfg, stage, _ = small_stage("bf16", 16)
    states = []
    for _ in range(2):
        gen = torch.Generator().manual_seed(2)
        s = dict(lengths=ints([40, 7, 100]), owned=ints([3, 1, 7]), table=torch.full((3, 12), -1, dtype=torch.int32, device=DEV), free=ints(range(11, 40)),
                 count=ints([29]), pools=[torch.randn((2, 40, 8, 16, 128), generator=gen).to(DEV, torch.bfloat16) for _ in "kv"],
                 x=torch.randn((16, 1024), generator=gen).to(DEV, torch.bfloat16), n_new=ints([5, 1, 3]))
        for i, row in enumerate(([0, 1, 2], [3], [4, 5, 6, 7, 8, 9, 10])):
            s["table"][i, :len(row)] = ints(row)
        states.append(s)

    def run(s, space):
        step = jp.extend(s["lengths"], s["n_new"], s["owned"], s["table"], s["free"], s["count"], 16, 16, in_place=True)
        return step, jp.prefill(stage, s["x"], step, *s["pools"], s["table"], 5, space)

    one, other = states
    run(one, workspace), run(other, workspace)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph, space = torch.cuda.CUDAGraph(), jp.Workspace(DEV)
    with torch.cuda.graph(graph, stream=side):
        step, y = run(one, space)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want_step, want = run(other, workspace)
        torch.cuda.synchronize()
        assert step.slots.tolist() == want_step.slots.tolist() and one["lengths"].tolist() == other["lengths"].tolist()
        assert torch.equal(y[:9], want[:9]) and torch.equal(one["pools"][0], other["pools"][0])
        one["x"].copy_(y), other["x"].copy_(want)
        one["x"][9:] = other["x"][9:] = 0.25


@gpu
def test_a_stage_over_pages_refuses(workspace):
    cfg, stage, _ = small_stage("bf16", 8)
    k = torch.zeros((2, 4, 8, 16, 128), dtype=torch.bfloat16, device=DEV)
    table = torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    x = torch.zeros((4, 1024), dtype=torch.bfloat16, device=DEV)
    step = jp.Step(ints([0, 4]), ints([0, 1, 2, 3]), ints([0, 1, 2, 3]), ints([4]), None, None, None)
    run = lambda **c: jp.prefill(**dict(dict(stage=stage, hidden_in=x, step=step, k_pools=k, v_pools=k, table=table, max_new=4, workspace=workspace), **c))  # noqa: E731
    run()
    torch.cuda.synchronize()
    for change in (dict(hidden_in=x[:, :512]), dict(hidden_in=x.float()), dict(k_pools=k[:1]), dict(v_pools=k[:, :2]), dict(hidden_out=x[:3]), dict(workspace=None),
                   dict(step=step._replace(slots=ints([0]))), dict(step=step._replace(row_start=ints([0]))), dict(table=table[:0]),
                   dict(hidden_in=torch.zeros((5, 1024), dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(ValueError):
            run(**change)
    many = jp.Step(ints([0, 4]), ints(range(9)), ints(range(9)), ints([9]), None, None, None)
    with pytest.raises(jb.JupiterError) as e:
        run(hidden_in=torch.zeros((9, 1024), dtype=torch.bfloat16, device=DEV), step=many)
    assert e.value.status == jb.JUP_ECAP
    few = torch.zeros((2, 4, 4, 16, 128), dtype=torch.bfloat16, device=DEV)   # pools of four heads
    with pytest.raises(jb.JupiterError) as e:
        run(k_pools=few, v_pools=few)
    assert e.value.status == jb.JUP_EINVAL and "configuration" in str(e.value)
    none = x[:0]
    assert run(hidden_in=none).shape == (0, 1024)
    L, batch = jp._lib(), jp._Batch(pool=pool_args(n_kv_heads=8), n_seqs=1, max_new=1, table_width=2, table_stride=2, row_start=FAKE, lengths=FAKE,
                                    table=FAKE, positions=FAKE, slots=FAKE, workspace=FAKE, workspace_bytes=workspace.args[1])
    for change, word in ((dict(layer_stride=-8), "layer_stride"), (dict(layer_stride=4), "layer_stride"), (dict(positions=None), "positions"),
                         (dict(slots=None), "slots"), (dict(n_seqs=0), "requests"), (dict(max_new=-1), "max_new"), (dict(workspace=None), "workspace"),
                         (dict(table_stride=1), "table_stride"), (dict(lengths=None), "NULL")):
        b = jp._Batch.from_buffer_copy(batch)
        for name, value in change.items():
            setattr(b, name, value)
        refused(L.jup_stage_prefill_paged(stage.handle, FAKE, 2, ctypes.byref(b), FAKE, None), word)
    refused(L.jup_stage_prefill_paged(stage.handle, FAKE, -1, ctypes.byref(batch), FAKE, None), "n_rows")
    refused(L.jup_stage_prefill_paged(stage.handle, FAKE + 2, 2, ctypes.byref(batch), FAKE, None), "aligned")
    refused(L.jup_stage_prefill_paged(stage.handle, None, 2, ctypes.byref(batch), FAKE, None), "NULL")
    refused(L.jup_stage_prefill_paged(stage.handle, FAKE, 2, None, FAKE, None), "batch")


@gpu
def test_a_stage_on_another_device_is_refused(workspace):
    k = torch.zeros((2, 4, 8, 16, 128), dtype=torch.bfloat16, device=DEV)
    x, table = torch.zeros((4, 1024), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    step = jp.Step(ints([0, 4]), ints([0, 1, 2, 3]), ints([0, 1, 2, 3]), ints([4]), None, None, None)
    elsewhere = types.SimpleNamespace(cfg=dict(n_layers=2, d_model=1024), handle=None, workspace=torch.empty(1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="stage"):
        jp.prefill(elsewhere, x, step, k, k, table, 4, workspace)


@gpu
def test_a_stage_over_more_activations_than_a_launch_has_threads_in_a_line(workspace):
    """Check mode has a thread per row and feature of the MLP: 2^32 and more of them.  The second half of the requests alone gives the same bits."""
    from paper_2504_08242_amd import synth_inputs as si
    cfg = dict(si.TINY, n_layers=1, d_model=64, n_heads=1, d_ffn=4096)
    n, rows = 16384, 64 * 16384 + 64
    stage = jb.Stage(cfg, "f32", jb.upload_layers(si.make_layers(cfg, seed=3), "f32"), rows)
    x = torch.randn((rows, 64), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)

    def run(x, new):
        k, v = (torch.zeros((1, len(new) + 1, 1, 64, 64), device=DEV) for _ in "kv")
        table, none = torch.full((len(new), 2), -1, dtype=torch.int32, device=DEV), [0] * len(new)
        step = jp.extend(ints(none), ints(new), ints(none), table, ints(range(len(new) + 1)), ints([len(new) + 1]), 64, x.shape[0])
        assert step.status.item() == 0
        return jp.prefill(stage, x, step, k, v, table, max(new))

    whole = run(x, [128] + [64] * (n - 1))
    assert torch.equal(run(x[-64 * 8192:].contiguous(), [64] * 8192), whole[-64 * 8192:])
    assert torch.equal(run(x[:64 * 8193], [128] + [64] * 8191), whole[:64 * 8193])


@gpu
def test_a_stage_over_more_rows_than_a_launch_has_workgroups_in_a_line():
    """2^24 rows and more, in check mode.  No row has a slot and the pool is zero: what is left is x + down(silu(gate n) up n), n = x / rms."""
    cfg = dict(n_layers=1, d_model=2, n_heads=1, head_dim=2, d_ffn=1, rms_eps=1e-5, rope_theta=1e4)
    weight = {n: torch.ones((2,) if n.startswith("g_") else (1, 2) if n in ("w_gate", "w_up") else (2, 1) if n == "w_down" else (2, 2), device=DEV) for n in jb.WEIGHT_NAMES}
    rows = (1 << 24) + 70
    stage = jb.Stage(cfg, "f32", [weight], rows)
    zero, pool = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros((1, 1, 1, 8, 2), device=DEV)
    x = torch.randn((rows, 2), generator=torch.Generator(device=DEV).manual_seed(7), device=DEV)
    got = jp.prefill(stage, x, jp.Step(ints([0, rows]), zero, zero - 1, ints([rows]), None, None, None), pool, pool, ints([0])[None], rows)
    v = x.double()
    v = (v / (v.square().mean(-1, keepdim=True) + 1e-5).sqrt()).sum(-1, keepdim=True)   # at most 2.83 in size
    # roundings: five in each of the two that make v, 14 x 2^-24 with their sum, times the slope of silu(v) v, 5.8; six in that product of up to
    # 7.6; one of the result
    assert ((got - (x.double() + torch.nn.functional.silu(v) * v)).abs() <= (81 + 46 + 8) * 2.0 ** -24 + 2.0 ** -24 * x.abs()).all()


def test_a_missing_stage_is_refused():
    refused(jp._lib().jup_stage_prefill_paged(None, FAKE, 2, ctypes.byref(jp._Batch()), FAKE, None), "stage")
