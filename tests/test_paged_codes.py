"""Pools in 8 bits: rows stored, read back and attended over, against the definitions in 64 bits (codes_reference.py, paged_reference.py).

Tolerances.  A value quantised is off by half a step: scale / 2 (int8), or the larger of 2^-4 of it and 2^-10 scale (e4m3); x * (T / m) has three
fp32 roundings on the way, 2^-22 of 448 steps of e4m3's least size, or of 127.  Attention: as over bf16 pools (a probability times a scale is
rounded once, 2^-8 of it, the result once more; fp32 sums).
"""
import ctypes
import inspect

import numpy as np
import pytest
import torch

import codes_reference as cref
import paged_reference as ref
from paper_2504_08242_amd import binding as jb
from paper_2504_08242_amd import paged as jp
from test_paged import (BF16, DEV, FAKE, MANY_HEADS, ORDERS, SHAPES, Batch, append_args, attention_args, f64, ints, many_requests, pool_args, refused)

gpu = pytest.mark.gpu
KINDS = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
kinds = pytest.mark.parametrize("kind", list(KINDS))


@pytest.fixture(scope="module")
def workspace():
    return jp.Workspace(DEV)


def raw(t):
    """The bytes of a tensor of codes."""
    return t.view(torch.uint8).cpu().numpy()


# ---- refusals: no GPU -------------------------------------------------------------------------------------------------------


def pool8_args(**change):
    return pool_args(**dict(dict(dtype=jp.JUP_I8), **change))


def scales_args(**change):
    return jp._Scales(**dict(dict(k=FAKE, v=FAKE, block_stride=64, head_stride=16, layer_stride=640), **change))


def read_args(**change):
    a = dict(n_rows=3, k=FAKE, v=FAKE, k_row_stride=512, k_head_stride=128, v_row_stride=512, v_head_stride=128, slots=FAKE)
    return jp._Read(**dict(a, **change))


def copy_args(**change):
    return jp._Copy(**dict(dict(n_copies=2, n_layers=1, layer_stride=0, copy_from=FAKE, copy_to=FAKE, lengths=None), **change))


def batch_args(pool, **change):
    a = dict(pool=pool, layer_stride=1 << 20, n_seqs=1, max_new=1, table_width=4, table_stride=4, workspace=FAKE,
             workspace_bytes=jp._lib().jup_paged_workspace_bytes())
    a.update({n: FAKE for n in ("row_start", "lengths", "table", "positions", "slots")})
    return jp._Batch(**dict(a, **change))


POOL8 = [(dict(dtype=jb.JUP_BF16), {}, "dtype"), (dict(dtype=0), {}, "dtype"), (dict(dtype=5), {}, "dtype"), (dict(n_blocks=0), {}, "positive"),
         (dict(page_size=24), {}, "page_size"), (dict(n_blocks=1 << 28), {}, "2^31"), (dict(k=None), {}, "k and v"), (dict(v=FAKE + 8), {}, "aligned"),
         (dict(head_dim=64), {}, "128"), (dict(slot_stride=136), {}, "multiples of 16"), (dict(head_stride=-16), {}, "negative"),
         (dict(slot_stride=(1 << 26) + 16), {}, "slot_stride"), ({}, dict(k=None), "scales"), ({}, dict(v=FAKE + 4), "aligned"),
         ({}, dict(block_stride=-4), "negative"), ({}, dict(layer_stride=-4), "negative"), ({}, dict(head_stride=18), "multiples of 4")]


@pytest.mark.parametrize("pool,scales,word", POOL8)
def test_pools_are_refused_by_every_call(pool, scales, word):
    L, p, x = jp._lib(), ctypes.byref(pool8_args(**pool)), ctypes.byref(scales_args(**scales))
    refused(L.jup_paged_append8(p, x, ctypes.byref(append_args()), None), word)
    refused(L.jup_paged_attention8(p, x, ctypes.byref(attention_args()), None), word)
    refused(L.jup_paged_read8(p, x, ctypes.byref(read_args()), None), word)
    refused(L.jup_paged_copy(p, x, ctypes.byref(copy_args()), None), word)


def test_pools_and_calls_of_the_other_kind_do_not_go_together():
    L = jp._lib()
    for dtype in (jp.JUP_I8, jp.JUP_E4M3):
        p = ctypes.byref(pool_args(dtype=dtype))
        refused(L.jup_paged_append(p, ctypes.byref(append_args()), None), "dtype")
        refused(L.jup_paged_attention(p, ctypes.byref(attention_args()), None), "dtype")
        refused(L.jup_paged_read(p, ctypes.byref(read_args()), None), "dtype")
        refused(L.jup_paged_copy(p, None, ctypes.byref(copy_args()), None), "dtype")
    p = ctypes.byref(pool8_args())
    for call, args in ((L.jup_paged_append8, append_args()), (L.jup_paged_attention8, attention_args()), (L.jup_paged_read8, read_args())):
        refused(call(p, None, ctypes.byref(args), None), "scales")
        refused(call(None, ctypes.byref(scales_args()), ctypes.byref(args), None), "pool")
        refused(call(p, ctypes.byref(scales_args()), None, None), "args")
    refused(L.jup_paged_copy(p, ctypes.byref(scales_args()), None, None), "args")
    refused(L.jup_paged_read(ctypes.byref(pool_args()), None, None), "args")
    refused(L.jup_stage_prefill_paged8(None, None, 1, ctypes.byref(batch_args(pool8_args())), ctypes.byref(scales_args()), None, None), "stage")


@pytest.mark.parametrize("change,word", [(dict(n_rows=-1), "n_rows"), (dict(slots=None), "slots"), (dict(k=FAKE + 2), "aligned"),
                                         (dict(v_row_stride=-128), "negative"), (dict(k_head_stride=129), "multiples of 8")])
def test_read_refuses(change, word):
    refused(jp._lib().jup_paged_read8(ctypes.byref(pool8_args()), ctypes.byref(scales_args()), ctypes.byref(read_args(**change)), None), word)
    refused(jp._lib().jup_paged_read(ctypes.byref(pool_args()), ctypes.byref(read_args(**change)), None), word)


@pytest.mark.parametrize("change,word", [(dict(n_copies=-1), "n_copies"), (dict(n_copies=16385), "n_copies"), (dict(n_layers=-1), "n_layers"),
                                         (dict(layer_stride=-16), "layer_stride"), (dict(layer_stride=24), "layer_stride"), (dict(copy_to=None), "NULL"),
                                         (dict(n_copies=16384, n_layers=1 << 20), "2^31")])
def test_copy_refuses(change, word):
    refused(jp._lib().jup_paged_copy(ctypes.byref(pool8_args()), ctypes.byref(scales_args()), ctypes.byref(copy_args(**change)), None), word)


def test_calls_of_nothing_launch_nothing():
    L, p, x = jp._lib(), ctypes.byref(pool8_args()), ctypes.byref(scales_args())
    assert L.jup_paged_append8(p, x, ctypes.byref(append_args(n_rows=0, k=None, v=None, slots=None)), None) == 0
    assert L.jup_paged_attention8(p, x, ctypes.byref(attention_args(n_rows=0, q=None)), None) == 0
    assert L.jup_paged_read8(p, x, ctypes.byref(read_args(n_rows=0, slots=None)), None) == 0
    assert L.jup_paged_read8(p, x, ctypes.byref(read_args(k=None, v=None, slots=None)), None) == 0
    assert L.jup_paged_copy(p, x, ctypes.byref(copy_args(n_copies=0, copy_from=None, copy_to=None)), None) == 0
    assert L.jup_paged_copy(p, x, ctypes.byref(copy_args(n_layers=0)), None) == 0


@pytest.mark.parametrize("call,names", [
    (jp.append, "k v slots k_pool v_pool positions rope_theta q q_out stream"), (jp.attention, "q k_pool v_pool table row_start lengths max_new workspace scale out stream"),
    (jp.prefill, "stage hidden_in step k_pools v_pools table max_new workspace hidden_out stream")])
def test_arguments_of_calls_over_other_pools_keep_their_places(call, names):
    """What a call over values takes by its place is where it was before there were scales."""
    assert list(inspect.signature(call).parameters) == names.split() + ["scales"]


@gpu
def test_the_front_end_refuses_tensors_that_do_not_fit(workspace):
    k, s = torch.zeros((5, 2, 16, 128), dtype=torch.int8, device=DEV), torch.zeros((5, 2, 16), device=DEV)
    row, i = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=DEV), ints([0, 1, 2])
    q, table = torch.zeros((3, 4, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    at, n = ints([0, 1, 2, 3]), ints([1, 1, 1])
    wide = torch.zeros((5, 2, 16, 136), dtype=torch.int8, device=DEV)
    for bad in (lambda: jp.append(row, row, i, k, k), lambda: jp.append(row, row, i, row, row, scales=(s, s)), lambda: jp.append(row, row, i, k, k, scales=(s, s[:4])),
                lambda: jp.append(row, row, i, k, k, scales=(s.double(), s)), lambda: jp.append(row.float(), row, i, k, k, scales=(s, s)),
                lambda: jp.append(row, row, i, k, k.view(torch.float8_e4m3fn), scales=(s, s)), lambda: jp.append(row, row, i, k, wide[..., :128], scales=(s, s)),
                lambda: jp.append(row, row, i, k, k, scales=(s, torch.zeros((2, 5, 16), device=DEV).transpose(0, 1))),
                lambda: jp.append(row, row, i, k, k, scales=(s.cpu(), s)), lambda: jp.attention(q, k, k, table, at, n, 1, workspace, scales=(s, s[..., :8])),
                lambda: jp.attention(q, k, k, table, at, n, 1, scales=(s, s)), lambda: jp.attention(q.float(), k, k, table, at, n, 1, workspace, scales=(s, s)),
                lambda: jp.read(i, k, k), lambda: jp.read(i.long(), k, k, scales=(s, s)), lambda: jp.read(i, k, k, scales=(s, s), k_out=row.float()),
                lambda: jp.read(i, k, k, scales=(s, s), v_out=row[:2]), lambda: jp.read(i, k, k, scales=(s, s), k_out=row[:, :1].expand(3, 2, 128)),
                lambda: jp.copy_pages(i, i[:2], k, k, scales=(s, s)), lambda: jp.copy_pages(i, i, k[None], k[None], scales=(s, s)),
                lambda: jp.copy_pages(i, i, k, k, lengths=i[:2], scales=(s, s))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: jp.append(row, row, i, wide[..., :128], wide[..., :128], scales=(s, s)),
                lambda: jp.attention(q[:, :3], k, k, table, at, n, 1, workspace, scales=(s, s))):
        with pytest.raises(jb.JupiterError) as e:
            bad()
        assert e.value.status == jb.JUP_EINVAL


# ---- rows stored and read back --------------------------------------------------------------------------------------------------


def make_codes(kind, n_blocks, heads, page, order, gen):
    """Codes of any kind [block, head, slot, i] in one of the orders a pool may have in memory, and scales [block, head, slot]."""
    def one():
        if order == "block-head-slot":
            t, s = torch.empty((n_blocks, heads, page, 128), dtype=torch.uint8, device=DEV), torch.empty((n_blocks, heads, page), device=DEV)
        elif order == "block-slot-head":  # (scales always have their slots side by side)
            t, s = torch.empty((n_blocks, page, heads, 128), dtype=torch.uint8, device=DEV).transpose(1, 2), torch.empty((n_blocks, heads, page + 4), device=DEV)[..., :page]
        elif order == "head-block-slot":
            t, s = torch.empty((heads, n_blocks, page, 128), dtype=torch.uint8, device=DEV).transpose(0, 1), torch.empty((heads, n_blocks, page), device=DEV).transpose(0, 1)
        else:
            t, s = torch.empty((n_blocks, heads, page, 160), dtype=torch.uint8, device=DEV)[..., :128], torch.empty((n_blocks, heads, page + 8), device=DEV)[..., :page]
        t.copy_(torch.randint(256, t.shape, generator=gen, dtype=torch.uint8))
        s.copy_(torch.rand(s.shape, generator=gen))
        return t.view(KINDS[kind]), s
    if order == "k-v-together":
        t = torch.randint(256, (n_blocks, 2, heads, page, 128), generator=gen, dtype=torch.uint8).to(DEV).view(KINDS[kind])
        s = torch.rand((n_blocks, 2, heads, page), generator=gen).to(DEV)
        return t[:, 0], t[:, 1], (s[:, 0], s[:, 1])
    (k, ks), (v, vs) = one(), one()
    return k, v, (ks, vs)


def whole(codes, scale, kind):
    """What a pool holds, in float64."""
    return cref.numbers(raw(codes), kind) * f64(scale)[..., None]


def rows_at(pool, slots, page):
    return pool[slots // page, :, slots % page]


@gpu
@kinds
@pytest.mark.parametrize("rows,heads,kv_heads,page,order", [(1, 4, 4, 16, "block-head-slot"), (5, 8, 2, 8, "block-slot-head"), (33, 5, 1, 32, "head-block-slot"),
                                                            (70, 12, 12, 64, "wide"), (9, 40, 8, 16, "k-v-together"), (600, 2, 1, 16, "block-head-slot")])
def test_rows_are_quantised_into_their_slots(kind, rows, heads, kv_heads, page, order):
    gen = torch.Generator().manual_seed(rows * heads)
    n_blocks = -(-rows // page) + 3
    k_pool, v_pool, scales = make_codes(kind, n_blocks, kv_heads, page, order, gen)
    before = [raw(x).copy() for x in (k_pool, v_pool)] + [x.cpu().numpy().copy() for x in scales]
    fused = (torch.randn((rows, heads + 2 * kv_heads, 128), generator=gen) * torch.randn((rows, heads + 2 * kv_heads, 1), generator=gen).mul(3).exp()).to(DEV, torch.bfloat16)
    q, k, v = fused[:, :heads], fused[:, heads:heads + kv_heads], fused[:, heads + kv_heads:]
    slots = torch.randperm(n_blocks * page, generator=gen)[:rows]
    if rows > 4:
        slots[1], slots[3], slots[4] = -1, n_blocks * page, 2 ** 31 - 1   # a row behind the last one, and slots no pool has
    positions = torch.randint(0, 100000, (rows,), generator=gen)
    positions[0] = 0
    if rows > 2:
        positions[2] = -3
    got = jp.append(k, v, slots.to(DEV, torch.int32), k_pool, v_pool, positions=positions.to(DEV, torch.int32), rope_theta=1e4, q=q, scales=scales)
    plain = torch.zeros((n_blocks, kv_heads, page, 128), dtype=torch.bfloat16, device=DEV)
    assert torch.equal(got, jp.append(k, v, slots.to(DEV, torch.int32), plain, plain.clone(), positions=positions.to(DEV, torch.int32), rope_theta=1e4, q=q))
    stored = np.array([s for s in slots.tolist() if 0 <= s < n_blocks * page])
    of = np.array([r for r, s in enumerate(slots.tolist()) if 0 <= s < n_blocks * page])
    # values: the definition to the bit
    codes, scale = cref.quantise(v.float().cpu().numpy()[of], kind)
    assert np.array_equal(rows_at(raw(v_pool), stored, page), codes)
    assert np.array_equal(rows_at(scales[1].cpu().numpy(), stored, page), scale)
    # keys: rotated in fp32 first, each 2^-21 of its pair off
    want = ref.rotate(f64(k)[of], positions.numpy()[of], 1e4)
    off = 2.0 ** -21 * np.tile(np.hypot(f64(k)[of][..., :64], f64(k)[of][..., 64:]), 2)
    m = np.abs(want).max(-1)
    have = rows_at(scales[0].cpu().numpy(), stored, page).astype(np.float64)
    assert (np.abs(have * cref.TOP[kind] - m) <= off.max(-1) + 2.0 ** -23 * m).all()
    value = cref.numbers(rows_at(raw(k_pool), stored, page), kind) * have[..., None]
    half = have[..., None] / 2 if kind == "int8" else np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * have[..., None])
    assert (np.abs(value - want) <= half * (1 + 2.0 ** -20) + 2 * off + 2.0 ** -22 * m[..., None]).all()
    # all else as it was
    for x, b in zip([raw(k_pool), raw(v_pool)] + [x.cpu().numpy() for x in scales], before):
        x, b = x.copy(), b.copy()
        x[stored // page, :, stored % page] = b[stored // page, :, stored % page] = 0
        assert np.array_equal(x, b)
    # without a rotation keys are the definition to the bit too
    assert jp.append(k, v, slots.to(DEV, torch.int32), k_pool, v_pool, scales=scales) is None
    codes, scale = cref.quantise(k.float().cpu().numpy()[of], kind)
    assert np.array_equal(rows_at(raw(k_pool), stored, page), codes) and np.array_equal(rows_at(scales[0].cpu().numpy(), stored, page), scale)


@gpu
@kinds
def test_heads_of_every_size(kind):
    """Zeros, the least and the largest numbers, infinities and NaN, one large value among small ones."""
    x = torch.randn((9, 2, 128), generator=torch.Generator().manual_seed(3)).to(DEV, torch.bfloat16)
    x[0] = 0
    x[1] *= 1e-39                     # subnormal ones
    x[2] *= 2.0 ** -101
    x[3] *= 1e37
    x[4, 0, 7] = float("inf")
    x[4, 1, 9] = -float("inf")
    x[5, 0, 0] = float("nan")
    x[6, 0, 127] = 1000.0
    x[7] = 3.3e38
    x[8] = -0.0
    pool, scales = torch.full((2, 2, 16, 128), 99, dtype=torch.uint8, device=DEV).view(KINDS[kind]), torch.full((2, 2, 2, 16), 7.0, device=DEV)
    v_pool = pool.clone()
    slots = ints(range(3, 12))
    jp.append(x, x, slots, pool, v_pool, scales=(scales[0], scales[1]))
    codes, scale = cref.quantise(x.float().cpu().numpy(), kind)
    at = np.arange(3, 12)
    for p, s in ((pool, scales[0]), (v_pool, scales[1])):
        assert np.array_equal(rows_at(raw(p), at, 16), codes)
        assert np.array_equal(rows_at(s.cpu().numpy(), at, 16), scale, equal_nan=True)
    assert np.isnan(scale[4]).all() and np.isnan(scale[5]).tolist() == [True, False] and np.isfinite(scale[[0, 1, 2, 3, 6, 7, 8]]).all()
    k, v = jp.read(slots, pool, v_pool, scales=(scales[0], scales[1]))
    assert torch.equal(k.isnan(), v.isnan()) and k.isnan().flatten(2).all(-1).nonzero().tolist() == [[4, 0], [4, 1], [5, 0]]
    assert (k[0] == 0).all() and torch.isfinite(k[7]).all()
    assert (k[7] == x[7]).all()       # the largest code stands for the largest value


def bf16_of(x):
    """float64 products of a code and an fp32 scale, rounded as fp32 products are and then to bf16."""
    return torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)


@gpu
@kinds
@pytest.mark.parametrize("order", ORDERS)
def test_rows_are_read_out_of_their_slots(kind, order):
    gen = torch.Generator().manual_seed(5)
    for rows, heads, page in ((1, 1, 16), (77, 3, 8), (40, 40, 32)):
        n_blocks = 6
        k_pool, v_pool, scales = make_codes(kind, n_blocks, heads, page, order, gen)
        slots = torch.randint(0, n_blocks * page, (rows,), generator=gen)
        if rows > 4:
            slots[1], slots[3], slots[4], slots[5] = -1, n_blocks * page, 2 ** 31 - 1, int(slots[0])
        wide = torch.full((rows, heads + 2, 136), 5.0, device=DEV).bfloat16()
        keep = wide.clone()
        k, v = jp.read(slots.to(DEV, torch.int32), k_pool, v_pool, scales=scales, v_out=wide[:, 1:-1, :128])
        for got, pool, scale in ((k, k_pool, scales[0]), (v, v_pool, scales[1])):
            want = bf16_of(rows_at(whole(pool, scale, kind), slots.numpy() % (n_blocks * page), page))
            want[(slots < 0) | (slots >= n_blocks * page)] = 0
            assert torch.equal(got.cpu().isnan(), want.isnan())
            assert torch.equal(got.cpu().nan_to_num(), want.nan_to_num())
        wide[:, 1:-1, :128] = keep[:, 1:-1, :128]
        assert torch.equal(wide, keep)


@gpu
@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float32, 128), (torch.float32, 6), (torch.float32, 256)])
def test_rows_of_other_pools_are_read_as_they_are(dtype, dim):
    from test_paged import make_pool
    gen = torch.Generator().manual_seed(dim)
    for order in ORDERS:
        k_pool, v_pool = make_pool(dtype, 5, 3, 16, dim, order, gen)
        slots = torch.tensor([0, 79, 33, -1, 80, 33])
        k, v = jp.read(slots.to(DEV, torch.int32), k_pool, v_pool)
        for got, pool in ((k, k_pool), (v, v_pool)):
            want = pool[(slots.clamp(0, 79) // 16).to(DEV), :, (slots.clamp(0, 79) % 16).to(DEV)]
            want[3:5] = 0
            assert got.dtype == dtype and torch.equal(got, want)


@gpu
@kinds
def test_no_rows(kind):
    k_pool, v_pool, scales = make_codes(kind, 3, 2, 16, "block-head-slot", torch.Generator().manual_seed(1))
    keep = raw(k_pool).copy()
    none = torch.empty((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    assert jp.append(none, none, ints([]), k_pool, v_pool, positions=ints([]), rope_theta=1e4, q=none, scales=scales).shape == (0, 2, 128)
    assert jp.read(ints([]), k_pool, v_pool, scales=scales)[0].shape == (0, 2, 128)
    assert np.array_equal(raw(k_pool), keep)


# ---- attention ----------------------------------------------------------------------------------------------------------------------


class Batch8(Batch):
    """A ragged batch over pages in 8 bits; places nobody wrote hold any code, and NaN as their scale."""

    def __init__(self, kind, heads, kv_heads, page, requests, order="block-head-slot", **kw):
        super().__init__(torch.bfloat16, heads, kv_heads, page, requests, **kw)
        self.kind = kind
        gen = torch.Generator().manual_seed(len(requests))
        n_blocks = self.k.shape[0]
        *pools, self.scales = make_codes(kind, n_blocks, kv_heads, page, order, gen)
        for x, codes, scale in zip((self.k, self.v), pools, self.scales):
            c, s = cref.quantise(x.float().cpu().numpy(), kind)
            there = torch.from_numpy(~np.isnan(s)).to(DEV)
            bytes_of(codes)[there] = torch.from_numpy(c).to(DEV)[there]
            scale.copy_(torch.from_numpy(s))
        self.k, self.v = pools

    def run(self, workspace, **kw):
        return super().run(workspace, scales=self.scales, **kw)

    def check(self, got, table=None):
        k, v = (whole(x, s, self.kind) for x, s in zip((self.k, self.v), self.scales))
        want, size, most = ref.attention(f64(self.q)[:self.rows], k, v, self.table if table is None else table, self.row_start, self.lengths, self.scale, self.page)
        keys = max(self.lengths)
        small = (keys + 2 * 128 * most + 32) * 2.0 ** -24
        # fp32 exponentials below 2^-126 are 0, and a value may be that much larger than what a row comes to: each key's |v| 2^-126 (of sums that are
        # divided by 1 at least, as the largest exponential is)
        least = keys * 2.0 ** -126 * np.abs(v[np.isfinite(v)]).max(initial=1.0)
        off = np.abs(f64(got)[:self.rows] - want)
        limit = (BF16 + small) * size + BF16 * np.abs(want) + least
        assert (off <= limit).all(), (float((off - limit).max()), [int(x) for x in np.unravel_index(np.argmax(off - limit), off.shape)])


def bytes_of(codes):
    """A view of codes as bytes that shares their memory, whatever their order."""
    return codes.view(torch.uint8)


@gpu
@kinds
@pytest.mark.parametrize("heads,kv_heads,page,requests", SHAPES)
def test_attention_over_codes(workspace, kind, heads, kv_heads, page, requests):
    b = Batch8(kind, heads, kv_heads, page, requests)
    got = b.run(workspace)
    b.check(got)
    for expected in (0, 1, 40, 5000):
        b.check(b.run(workspace, max_new=expected))
    assert torch.equal(got, b.run(workspace))


@gpu
@kinds
@pytest.mark.parametrize("heads,kv_heads,requests", [(4, 4, [(200, 1), (37, 3)]), (8, 1, [(0, 13), (0, 18)]), (32, 32, [(0, 23), (0, 73)]), (4, 2, [(100, 40), (0, 30)]),
                                                     (40, 8, [(0, 16), (0, 19)]), (64, 64, [(30, 70), (0, 90), (0, 60)]), (2, 2, [(3000, 60)]), (16, 1, [(1500, 2)])])
def test_tiles_of_few_rows_lose_nothing_to_probabilities_of_fewer_bits(workspace, kind, heads, kv_heads, requests):
    """In tiles of up to 32 rows a probability times its value's scale goes into the product as two numbers: its first 8 bits, cut off, which leaves less than
    2^-7 of it, and the rest, rounded, 2^-8 of that.  What is left is 2^-15, fp32 sums and the rounding of the result."""
    b = Batch8(kind, heads, kv_heads, 16, requests)
    got = b.run(workspace)
    k, v = (whole(x, s, kind) for x, s in zip((b.k, b.v), b.scales))
    want, size, most = ref.attention(f64(b.q)[:b.rows], k, v, b.table, b.row_start, b.lengths, b.scale, b.page)
    keys = max(b.lengths)
    small = (keys + 2 * 128 * most + 32) * 2.0 ** -24
    least = keys * 2.0 ** -126 * np.abs(v[np.isfinite(v)]).max(initial=1.0)
    off = np.abs(f64(got)[:b.rows] - want) - ((2.0 ** -15 + small) * size + BF16 * np.abs(want) + least)
    assert (off <= 0).all(), float(off.max())


@gpu
@kinds
@pytest.mark.parametrize("heads,kv_heads,page,requests", MANY_HEADS)
def test_attention_of_many_heads(workspace, kind, heads, kv_heads, page, requests):
    b = Batch8(kind, heads, kv_heads, page, requests)
    b.check(b.run(workspace))
    b.check(b.run(workspace, max_new=1))


@gpu
@kinds
@pytest.mark.parametrize("order", ORDERS)
def test_attention_over_pools_in_any_order(workspace, kind, order):
    for requests in ([(70, 3), (200, 1)], [(40, 150), (0, 300)]):
        b = Batch8(kind, 4, 2, 16, requests, order=order)
        b.check(b.run(workspace))


@gpu
@kinds
@pytest.mark.parametrize("n,most_cached,most_new,heads,kv_heads", [(64, 100, 3, 4, 2), (65, 100, 3, 4, 2), (1000, 40, 2, 2, 1), (70, 60, 40, 4, 1), (130, 200, 17, 8, 2),
                                                                   (4097, 12, 1, 1, 1)])
def test_attention_of_many_requests(workspace, kind, n, most_cached, most_new, heads, kv_heads):
    b = Batch8(kind, heads, kv_heads, 16, many_requests(n, most_cached, most_new, n))
    got = b.run(workspace)
    b.check(got)
    b.check(b.run(workspace, max_new=100))
    assert torch.equal(got, b.run(workspace))


@gpu
@kinds
@pytest.mark.parametrize("heads,kv_heads,requests", [(30, 30, [(0, 1)] * 10 + [(2000, 300)]), (20, 20, [(0, 1)] * 20 + [(2000, 200)]), (32, 4, [(3000, 200), (10, 300)]),
                                                     (64, 64, [(0, 2)] * 7 + [(1500, 100)]), (65, 65, [(0, 2)] * 7 + [(1500, 100)]), (1, 1, [(13000, 1)]),
                                                     (8, 1, [(9000, 5)])])
def test_divided_keys(workspace, kind, heads, kv_heads, requests):
    b = Batch8(kind, heads, kv_heads, 32, requests)
    got = b.run(workspace)
    b.check(got)
    assert torch.equal(got, b.run(workspace))


@gpu
@kinds
def test_pages_that_are_not_there(workspace, kind):
    for heads, requests in ((4, [(90, 4), (40, 2), (0, 3)]), (4, [(200, 160), (0, 140), (64, 33)]), (60, [(100, 90), (0, 50), (0, 3)]), (150, [(100, 90), (0, 50), (0, 3)])):
        b = Batch8(kind, heads, heads, 16, requests)
        t = b.table.copy()
        t[0, [0, 2, 3]] = [-1, b.k.shape[0], 2 ** 31 - 1]
        t[1, :] = -(2 ** 31)                 # nothing left of this one
        t[2, 0] = -5                         # its first rows see nothing
        got = b.run(workspace, table=t)
        b.check(got, table=t)
        assert (got[b.row_start[1]:b.row_start[2]] == 0).all()
        if requests[2][0] == 0:
            assert (got[b.row_start[2]] == 0).all()


@gpu
@kinds
@pytest.mark.parametrize("heads,requests", [(2, [(50, 6)]), (2, [(20, 40), (70, 3)]), (2, [(100, 200)]), (60, [(100, 90), (0, 50)]), (150, [(100, 90), (0, 50)]),
                                            (4, [(3000, 200), (10, 3)])])
def test_codes_and_scales_that_a_row_does_not_see_do_not_reach_it(workspace, kind, heads, requests):
    """Scales that are no numbers, and codes that are none, of later tokens of the same step; those that see them get NaN."""
    b = Batch8(kind, heads, heads, 16, requests)
    want = b.run(workspace)
    cached, new = requests[0]
    for what in ("k_scale", "v_scale", "v_inf", "inf", "codes"):
        c = Batch8(kind, heads, heads, 16, requests)
        for t in (new - 1, new // 2):        # the last token's keys and values, and one in the middle
            pos = cached + t
            block, slot = int(c.table[0, pos // 16]), pos % 16
            if what == "k_scale":
                c.scales[0][block, :, slot] = float("nan")
            elif what == "v_scale":
                c.scales[1][block, :, slot] = float("nan")
            elif what == "v_inf":
                c.scales[1][block, :, slot] = -float("inf")
            elif what == "inf":              # a probability of 0, or none that is a number
                c.scales[0][block, :, slot] = float("inf")
            else:
                for x in (c.k, c.v):
                    bytes_of(x)[block, :, slot, 5] = 0x7F if kind == "e4m3" else 0x80
        got = c.run(workspace)
        clean = [r for r in range(b.rows) if not (new // 2 <= r < new)]
        assert torch.equal(got[clean], want[clean]), what
        if what == "codes" and kind == "int8":
            c.check(got)
        elif what != "inf":
            assert not torch.isfinite(got[new // 2:new]).flatten(1).all(1).any()


@gpu
@pytest.mark.parametrize("heads,requests", [(2, [(50, 6)]), (2, [(100, 200)]), (60, [(100, 90), (0, 50)]), (150, [(100, 90), (0, 50)])])
def test_values_that_are_no_numbers_reach_one_feature(workspace, heads, requests):
    b = Batch8("e4m3", heads, heads, 16, requests)
    want = b.run(workspace)
    cached, new = requests[0]
    pos = cached + new // 2
    bytes_of(b.v)[int(b.table[0, pos // 16]), :, pos % 16, 7] = 0xFF
    got = b.run(workspace)
    sees = slice(new // 2, new)
    assert got[sees, :, 7].isnan().all()
    got[sees, :, 7] = want[sees, :, 7]
    assert torch.equal(got, want)


@gpu
@kinds
def test_scales_of_every_size(workspace, kind):
    """Scores and values far apart in size: what counts is the products."""
    for requests in ([(400, 3)], [(100, 200)]):
        b = Batch8(kind, 4, 2, 16, requests)
        g = torch.Generator().manual_seed(9)
        b.scales[1].mul_((torch.randn(b.scales[1].shape, generator=g) * 6).exp().to(DEV))
        b.scales[0].mul_((torch.randn(b.scales[0].shape, generator=g)).exp().to(DEV))
        b.check(b.run(workspace))
        b.scales[1].fill_(2.0 ** 100)
        b.check(b.run(workspace))
        b.scales[0].zero_()
        b.check(b.run(workspace))


@gpu
@kinds
def test_results_in_place_and_in_wider_tensors(workspace, kind):
    for new in (1, 5, 40, 260):
        b = Batch8(kind, 4, 4, 16, [(100, new), (33, new)], pad_rows=5)
        fused = torch.full((b.q.shape[0], 12, 128), float("nan"), device=DEV).bfloat16()
        fused[:, 4:8] = b.q
        want, b.q = b.run(workspace)[:b.rows], fused[:, 4:8]
        wide = torch.full((b.q.shape[0] + 2, 9, 136), 7.0, device=DEV).bfloat16()
        keep = wide.clone()
        out = wide[1:-1, 2:6, :128]
        assert b.run(workspace, out=out) is out and torch.equal(out[:b.rows], want)
        out[:b.rows] = keep[1:1 + b.rows, 2:6, :128]
        assert torch.equal(wide, keep)   # rows behind the last one among it
        assert b.run(workspace, out=b.q) is b.q and torch.equal(b.q[:b.rows], want)


@gpu
@kinds
def test_two_graphs_and_other_streams(workspace, kind):
    """Graphs that share a workspace, replayed with eager calls between them; a call on another stream."""
    batches = [Batch8(kind, 4, 2, 16, r) for r in ([(3000, 1), (700, 4)], [(2500, 40), (100, 90)], many_requests(100, 60, 2, 1))]
    want = [b.run(workspace) for b in batches]
    graphs = []
    for b in batches:
        args = b.q, b.k, b.v, torch.from_numpy(b.table).to(DEV, torch.int32), ints(b.row_start), ints(b.lengths), max(b.new), workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = jp.attention(*args, scales=b.scales)
        graphs.append((graph, args, out))
    for _ in range(4):
        for (graph, _, out), w, b in zip(graphs, want, batches):
            out.zero_()
            graph.replay()
            assert torch.equal(out, w)
            assert torch.equal(b.run(workspace), w)
    side = torch.cuda.Stream()
    other = jp.Workspace(DEV)
    got = batches[0].run(other, stream=side)
    side.synchronize()
    assert torch.equal(got, want[0])


@gpu
@kinds
def test_blocks_beyond_32_bits(workspace, kind):
    """Codes 2^31 bytes apart and scales 2^32: rows stored, read, attended over (few and many of them) and copied."""
    far, heads, page, n_blocks = (1 << 31) + 4096, 2, 16, 4
    memory = torch.empty(4 * far + (1 << 20), dtype=torch.uint8, device=DEV)
    shape, strides = (n_blocks, heads, page, 128), (far, page * 128, 128, 1)
    k_pool, v_pool = (memory.as_strided(shape, strides, at).view(KINDS[kind]) for at in (0, 1 << 16))
    apart = tuple(memory.view(torch.float32).as_strided((2, heads, page), (far // 2, page, 1), at // 4) for at in (1 << 17, (1 << 17) + 4096))
    scales = tuple(torch.zeros(shape[:3], device=DEV) for _ in range(2))
    gen = torch.Generator().manual_seed(2)
    rows = torch.randn((n_blocks * page, heads, 128), generator=gen).to(DEV, torch.bfloat16)
    small = [torch.zeros(shape, dtype=torch.uint8, device=DEV).view(KINDS[kind]) for _ in range(2)]
    near = [torch.zeros(shape[:3], device=DEV) for _ in range(2)]
    slots = ints(range(n_blocks * page))
    for pool, x in (((k_pool, v_pool), scales), (small, near)):
        jp.append(rows, rows.flip(0), slots, *pool, scales=x)
    assert torch.equal(k_pool.view(torch.uint8), small[0].view(torch.uint8)) and torch.equal(v_pool.view(torch.uint8), small[1].view(torch.uint8))
    for a, b in zip(jp.read(slots, k_pool, v_pool, scales=scales), jp.read(slots, *small, scales=near)):
        assert torch.equal(a, b)
    table = ints([2, 0, 3, 1]).view(1, 4)
    for new in (1, 33, 60):
        q = torch.randn((new, 4, 128), generator=gen).to(DEV, torch.bfloat16)
        call = lambda *pool, scales: jp.attention(q, *pool, table, ints([0, new]), ints([61]), new, workspace, scales=scales)  # noqa: E731
        assert torch.equal(call(k_pool, v_pool, scales=scales), call(*small, scales=near))
    # two blocks whose scales are as far apart
    codes = [x[:2].contiguous() for x in (small[0].view(torch.uint8), small[1].view(torch.uint8))]
    codes = [x.view(KINDS[kind]) for x in codes]
    for mine, x in zip(apart, near):
        mine.copy_(x[:2])
    for a, b in zip(jp.read(slots[:32], *codes, scales=apart), jp.read(slots[:32], *small, scales=near)):
        assert torch.equal(a, b)
    for new in (1, 30):
        q = torch.randn((new, 4, 128), generator=gen).to(DEV, torch.bfloat16)
        call = lambda *pool, scales: jp.attention(q, *pool, ints([1, 0]).view(1, 2), ints([0, new]), ints([31]), new, workspace, scales=scales)  # noqa: E731
        assert torch.equal(call(*codes, scales=apart), call(*small, scales=near))
    jp.copy_pages(ints([0]), ints([3]), k_pool, v_pool, scales=scales)
    assert torch.equal(k_pool.view(torch.uint8)[3], small[0].view(torch.uint8)[0]) and torch.equal(scales[1][3], near[1][0])


@gpu
@kinds
def test_stores_on_another_stream(kind):
    """Rows stored and read on a stream that is not the current one, twice at once."""
    gen = torch.Generator().manual_seed(4)
    k_pool, v_pool, scales = make_codes(kind, 40, 4, 16, "block-head-slot", gen)
    rows = torch.randn((600, 4, 128), generator=gen).to(DEV, torch.bfloat16)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    halves = ints(range(300)), ints(range(300, 600))
    for s, x, stream in zip(halves, (rows[:300], rows[300:]), (None, side)):
        jp.append(x, x, s, k_pool, v_pool, scales=scales, stream=stream)
    got = jp.read(halves[1], k_pool, v_pool, scales=scales, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    codes, scale = cref.quantise(rows.float().cpu().numpy(), kind)
    want = bf16_of(cref.numbers(codes, kind) * scale[..., None].astype(np.float64))
    assert all(torch.equal(x.cpu(), want[300:]) for x in got)
    assert all(torch.equal(x.cpu(), want) for x in jp.read(ints(range(600)), k_pool, v_pool, scales=scales))


# ---- a stage over pages in 8 bits ------------------------------------------------------------------------------------------------------


def stage_in_64_bits(layer, cfg, hidden, cached_k, cached_v, position, kind):
    """One layer over new rows of one request behind cached keys and values [H, n, 128] that are as they are; those of the new rows are
    quantised.  float64; weights [out, in]."""
    H, D, d = cfg["n_heads"], 128, cfg["d_model"]

    def norm(x, g):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + cfg["rms_eps"]) * g

    w = {name: np.asarray(x, np.float64) for name, x in layer.items()}
    n = len(hidden)
    x = norm(hidden, w["g_attn"])
    q, k, v = ((x @ w[name].T).reshape(n, H, D) for name in ("wq", "wk", "wv"))
    at = position + np.arange(n)
    q, k = ref.rotate(q, at, cfg["rope_theta"]), ref.rotate(k, at, cfg["rope_theta"])
    held = []
    for new, old in ((k, cached_k), (v, cached_v)):
        codes, scale = cref.quantise(new, kind)
        held.append(np.concatenate([old, (cref.numbers(codes, kind) * scale[..., None].astype(np.float64)).transpose(1, 0, 2)], 1))
    out = np.empty((n, H, D))
    for t in range(n):
        s = np.einsum("hd,hjd->hj", q[t], held[0][:, :position + t + 1]) / np.sqrt(D)
        p = np.exp(s - s.max(-1, keepdims=True))
        out[t] = np.einsum("hj,hjd->hd", p / p.sum(-1, keepdims=True), held[1][:, :position + t + 1])
    x = hidden + out.reshape(n, d) @ w["wo"].T
    y = norm(x, w["g_mlp"])
    gate = y @ w["w_gate"].T
    return x + (gate / (1 + np.exp(-gate)) * (y @ w["w_up"].T)) @ w["w_down"].T, held


@gpu
@kinds
@pytest.mark.parametrize("dtype", ["bf16", "w4"])
def test_a_stage_over_pages_in_8_bits(workspace, kind, dtype):
    """Two layers, checked one by one: a prompt, then a step of a few tokens; uneven requests; rel-L2 2e-2 of all rows, 4e-2 of each, as for other
    stages (a code that falls on the other side of a border is one step off, half a step more than the definition allows anyway)."""
    from oracle import w4
    from paper_2504_08242_amd import synth_inputs as si
    page, D = 16, 128
    for n_layers in (1, 2):
        cfg = dict(si.LLAMA7B_STAGE, n_layers=n_layers, d_model=512, n_heads=4, d_ffn=768)
        if dtype == "w4":
            given = si.make_w4_layers(cfg, seed=3)
            layers, up = w4.dequantize_layers(given), jb.upload_w4_layers(given)
        else:
            layers = given = si.make_layers(cfg, seed=3, bf16=True)
            up = jb.upload_layers(given, dtype)
        stage = jb.Stage(cfg, dtype, up, 96)
        n_blocks, width = 24, 8
        codes = [torch.randint(256, (n_layers, n_blocks, 4, page, D), dtype=torch.uint8, device=DEV).view(KINDS[kind]) for _ in range(2)]
        scales = [torch.full((n_layers, n_blocks, 4, page), float("nan"), device=DEV) for _ in range(2)]
        table, free, count = torch.full((2, width), -1, dtype=torch.int32, device=DEV), ints(torch.randperm(n_blocks).tolist()), ints([n_blocks])
        lengths, owned = ints([0, 0]), ints([0, 0])
        hidden = si.make_hidden(cfg, seed=3, n_tokens=100, bf16=True)
        at = [0, 50]       # rows of the two requests in hidden
        kept = [[(np.zeros((4, 0, D)), np.zeros((4, 0, D))) for _ in range(n_layers)] for _ in range(2)]
        done = [0, 0]
        for new in ([40, 21], [1, 5], [3, 1]):
            step = jp.extend(lengths, ints(new), owned, table, free, count, page, sum(new), in_place=True)
            x = np.concatenate([hidden[a:a + m] for a, m in zip(at, new)])
            y = jp.prefill(stage, torch.from_numpy(x).to(DEV, torch.bfloat16), step, *codes, table, max(new), workspace, scales=scales)
            row = 0
            for i, m in enumerate(new):
                want = hidden[at[i]:at[i] + m].astype(np.float64)
                blocks = table[i, :-(-(done[i] + m) // page)].long()
                for l in range(n_layers):
                    want, held = stage_in_64_bits(layers[l], cfg, want, *kept[i][l], done[i], kind)
                    mine = []
                    for c, s, h in zip(codes, scales, held):
                        have = whole(c[l][blocks], s[l][blocks], kind).transpose(1, 0, 2, 3).reshape(4, -1, D)[:, :done[i] + m]
                        # what is stored is the definition's up to the rounding of what came in
                        off = np.linalg.norm(have - h) / np.linalg.norm(h)
                        assert off <= 2e-2 + (0.0 if kind == "int8" else 2e-2), (l, i, off)
                        mine.append(have)
                    kept[i][l] = mine
                got = f64(y)[row:row + m]
                assert np.linalg.norm(got - want) <= 2e-2 * np.linalg.norm(want)
                assert (np.linalg.norm(got - want, axis=1) <= 4e-2 * np.linalg.norm(want, axis=1)).all()
                row += m
                at[i] += m
                done[i] += m
        # the same captured and replayed: a step of one token each whose lengths move on
        x = torch.from_numpy(hidden[90:92]).to(DEV, torch.bfloat16)
        one = ints([1, 1])
        state = [t.clone() for t in (lengths, owned, count, table, *codes, *scales)]

        def again():
            s = jp.extend(lengths, one, owned, table, free, count, page, 2, in_place=True)
            return jp.prefill(stage, x, s, *codes, table, 1, workspace, scales=scales)

        want = [again().clone() for _ in range(3)]
        for t, s in zip((lengths, owned, count, table, *codes, *scales), state):
            t.copy_(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = again()
        for w in want:
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)


@gpu
def test_a_stage_refuses_pools_that_do_not_fit(workspace):
    from paper_2504_08242_amd import synth_inputs as si
    cfg = dict(si.LLAMA7B_STAGE, n_layers=1, d_model=512, n_heads=4, d_ffn=768)
    stage = jb.Stage(cfg, "bf16", jb.upload_layers(si.make_layers(cfg, seed=3, bf16=True), "bf16"), 16)
    k, s = torch.zeros((1, 4, 4, 16, 128), dtype=torch.int8, device=DEV), torch.zeros((1, 4, 4, 16), device=DEV)
    table, x = torch.zeros((1, 2), dtype=torch.int32, device=DEV), torch.zeros((1, 512), dtype=torch.bfloat16, device=DEV)
    step = jp.Step(ints([0, 1]), ints([0]), ints([0]), ints([1]), ints([1]), ints([0]), ints([0]))
    for bad in (lambda: jp.prefill(stage, x, step, k, k, table, 1, workspace), lambda: jp.prefill(stage, x, step, k, k, table, 1, workspace, scales=(s[0], s[0])),
                lambda: jp.prefill(stage, x, step, k, k, table, 1, workspace, scales=(s, s[..., :8])), lambda: jp.prefill(stage, x, step, k, k, table, 1, scales=(s, s))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(jb.JupiterError):   # fewer heads than the stage has
        jp.prefill(stage, x, step, k[:, :, :2], k[:, :, :2], table, 1, workspace, scales=(s[:, :, :2], s[:, :, :2]))
    tiny = jb.Stage(si.TINY, "f32", jb.upload_layers(si.make_layers(si.TINY, seed=3), "f32"), 16)
    with pytest.raises((ValueError, jb.JupiterError)):
        jp.prefill(tiny, x, step, k.expand(2, -1, -1, -1, -1), k.expand(2, -1, -1, -1, -1), table, 1, workspace, scales=(s.expand(2, -1, -1, -1),) * 2)
