"""The end of a step of a beam search, tables of requests that go on from others, copies of pages: against codes_reference.py.

Tolerances.  Scores: exponentials are fp32 (2^-23 each, and 2^-22 for the sums of eight), so a score is off by 2^-21 and by its own rounding, 2^-24 of
it.  Where two scores are nearer than that their order is open; the inputs here have ties that are exact (they go by the order of beams and tokens) or
differ by more, which the tests assert.  Tables and copies: exact.
"""
import ctypes
import random

import numpy as np
import pytest
import torch

import codes_reference as cref
from paper_2504_08242_amd import binding as jb
from paper_2504_08242_amd import paged as jp
from test_paged import DEV, FAKE, f64, ints, make_pool, refused

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def workspace():
    return jp.Workspace(DEV)


# ---- refusals: no GPU -------------------------------------------------------------------------------------------------------


def beam_args(**change):
    a = dict(n_seqs=2, n_beams=3, n_keep=3, vocab=100, logits_dtype=jb.JUP_F32, end_token=-1, row_stride=100, ended=None, workspace=FAKE,
             workspace_bytes=jp._lib().jup_paged_workspace_bytes())
    a.update({n: FAKE for n in ("logits", "scores", "parents", "tokens", "new_scores", "new_ended")})
    return jp._Beam(**dict(a, **change))


def reorder_args(**change):
    a = dict(n_in=2, n_out=3, page_size=16, table_width=4, new_table_width=4, n_free=9, table_stride=4, new_table_stride=4, held=None, workspace=FAKE,
             workspace_bytes=jp._lib().jup_paged_workspace_bytes())
    a.update({n: FAKE for n in ("parents", "table", "lengths", "owned", "free_blocks", "free_count", "new_lengths", "new_owned", "new_free_blocks",
                                "new_free_count", "copy_from", "copy_to", "status")})
    a["new_table"] = FAKE + 4096
    return jp._Reorder(**dict(a, **change))


@pytest.mark.parametrize("change,word", [
    (dict(n_seqs=-1), "n_seqs"), (dict(n_seqs=6000), "n_seqs"), (dict(n_beams=0), "n_beams"), (dict(n_beams=65), "n_beams"), (dict(n_keep=0), "n_keep"),
    (dict(n_keep=65), "n_keep"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 30) + 1), "vocab"), (dict(logits_dtype=2), "logits_dtype"),
    (dict(end_token=-2), "end_token"), (dict(end_token=100), "end_token"), (dict(ended=FAKE), "ended"), (dict(row_stride=-1), "row_stride"),
    (dict(workspace=None), "workspace"), (dict(workspace=FAKE + 8), "workspace"), (dict(workspace_bytes=9), "workspace"), (dict(logits=None), "NULL"),
    (dict(scores=None), "NULL"), (dict(parents=None), "NULL"), (dict(tokens=None), "NULL"), (dict(new_scores=None), "NULL")])
def test_selection_refuses(change, word):
    refused(jp._lib().jup_beam_select(ctypes.byref(beam_args(**change)), None), word)


@pytest.mark.parametrize("change,word", [
    (dict(n_in=-1), "n_in"), (dict(n_out=16385), "n_out"), (dict(page_size=20), "page_size"), (dict(page_size=4), "page_size"), (dict(table_width=-1), "table_width"),
    (dict(new_table_width=1 << 28, new_table_stride=1 << 28), "2^31"), (dict(table_stride=3), "table_stride"), (dict(new_table_stride=3), "table_stride"),
    (dict(n_free=-1), "n_free"), (dict(n_free=(1 << 26) + 1), "n_free"), (dict(workspace=None), "workspace"), (dict(free_count=None), "free_count"),
    (dict(status=None), "status"), (dict(new_free_blocks=None), "free_blocks"), (dict(owned=None), "owned"), (dict(table=None), "table"),
    (dict(parents=None), "parents"), (dict(new_table=None), "new_table"), (dict(copy_to=None), "copy_to"), (dict(new_table=FAKE), "must not be table")])
def test_reordering_refuses(change, word):
    refused(jp._lib().jup_paged_reorder(ctypes.byref(reorder_args(**change)), None), word)


def test_null_arguments_and_nothing_to_select():
    L = jp._lib()
    refused(L.jup_beam_select(None, None), "NULL")
    refused(L.jup_paged_reorder(None, None), "NULL")
    assert L.jup_beam_select(ctypes.byref(beam_args(n_seqs=0, logits=None, scores=None)), None) == 0


def test_the_front_end_refuses_tensors_on_the_cpu():
    i, x = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 5))
    with pytest.raises(ValueError, match="GPU"):
        jp.beam_select(x, x[:, :1], 1, None)
    with pytest.raises(ValueError, match="GPU"):
        jp.reorder(i, i.view(3, 1), i, i, i, i[:1], 16, None)


@gpu
def test_the_front_end_refuses_tensors_that_do_not_fit(workspace):
    x, s, i = torch.zeros((6, 50), device=DEV), torch.zeros((2, 3), device=DEV), ints([0, 1, 2])
    e = torch.zeros((2, 3), dtype=torch.int32, device=DEV)
    t, one = torch.zeros((3, 2), dtype=torch.int32, device=DEV), ints([0])
    free = ints([0] * 8)
    for bad in (lambda: jp.beam_select(x.half(), s, 2, workspace), lambda: jp.beam_select(x, s[:, :2], 2, workspace), lambda: jp.beam_select(x, s.view(-1), 2, workspace),
                lambda: jp.beam_select(x, s.double(), 2, workspace), lambda: jp.beam_select(x, s, 0, workspace), lambda: jp.beam_select(x, s, 65, workspace),
                lambda: jp.beam_select(x, s, 2, None), lambda: jp.beam_select(x, s, 2, workspace, end_token=1, ended=e.bool()),
                lambda: jp.beam_select(x, s, 2, workspace, end_token=1, ended=e[:1]), lambda: jp.beam_select(x.t().contiguous().t(), s, 2, workspace),
                lambda: jp.beam_select(x, s.t().contiguous().t(), 2, workspace),
                lambda: jp.reorder(i.long(), t, i, i, free, one, 16, workspace), lambda: jp.reorder(i, t[:2], i, i, free, one, 16, workspace),
                lambda: jp.reorder(i, t, i, i[:2], free, one, 16, workspace), lambda: jp.reorder(i, t, i, i, free, i, 16, workspace),
                lambda: jp.reorder(i, t, i, i, free, one, 16, workspace, held=free), lambda: jp.reorder(i, t, i, i, free, one, 16, workspace, width=-1),
                lambda: jp.reorder(i, t, i, i, free, one, 16, None), lambda: jp.reorder(i, t, i, i, free, one, 16, workspace, held=torch.zeros(7, dtype=torch.uint8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: jp.beam_select(x, s, 2, workspace, ended=e), lambda: jp.beam_select(x, s, 2, workspace, end_token=50), lambda: jp.reorder(i, t, i, i, free, one, 10, workspace)):
        with pytest.raises(jb.JupiterError) as err:
            bad()
        assert err.value.status == jb.JUP_EINVAL


# ---- selection ------------------------------------------------------------------------------------------------------------------


def check_select(workspace, logits, scores, keep, end_token=-1, ended=None):
    n, B = scores.shape
    got = jp.beam_select(logits, scores, keep, workspace, end_token=end_token, ended=ended)
    over = None if ended is None else ended.cpu().numpy()
    parents, tokens, best, after = cref.beam_select(f64(logits).reshape(n, B, -1), f64(scores), keep + 1, end_token, over)
    with np.errstate(invalid="ignore"):
        gap = best[:, :-1] - best[:, 1:]
    assert not ((gap > 0) & (gap < 2.0 ** -19)).any(), "the inputs leave an order open"
    assert got.parents.cpu().tolist() == parents[:, :keep].tolist()
    assert got.tokens.cpu().tolist() == tokens[:, :keep].tolist()
    assert got.ended.cpu().tolist() == after[:, :keep].tolist()
    have, want = f64(got.scores), best[:, :keep]
    assert np.array_equal(np.isfinite(have), np.isfinite(want)) and (have[~np.isfinite(want)] == -np.inf).all()
    there = np.isfinite(want)
    assert (np.abs(have - want)[there] <= 2.0 ** -21 + 2.0 ** -24 * np.abs(want[there])).all(), np.abs(have - want)[there].max()
    return got


def make_logits(n, B, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    logits = (spread * torch.randn((n * B, V), generator=g, dtype=torch.float64)).to(dtype)
    scores = -torch.rand((n, B), generator=g, dtype=torch.float64).cumsum(1).float() * 3
    return logits.to(DEV), scores.to(DEV)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,B,keep,V", [(1, 1, 1, 1), (1, 1, 4, 3), (2, 3, 3, 5), (3, 4, 4, 63), (1, 2, 5, 64), (5, 8, 8, 1000), (1, 4, 4, 32000), (2, 16, 16, 4097), (3, 1, 16, 8191),
                                        (1, 64, 64, 300), (1, 5, 64, 20011), (700, 2, 3, 130), (2, 7, 2, 50257), (1, 3, 3, 131073)])
def test_selection(workspace, dtype, n, B, keep, V):
    logits, scores = make_logits(n, B, V, dtype, n * V + keep)
    got = check_select(workspace, logits, scores, keep)
    again = jp.beam_select(logits, scores, keep, workspace)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_a_wider_tensor_that_begin_anywhere(workspace, dtype):
    logits, scores = make_logits(3, 4, 1003, dtype, 7)
    wide = torch.full((12, 1017), float("nan"), device=DEV).to(dtype)
    for at in (0, 1, 3, 8):
        wide[:, at:at + 1003] = logits
        check_select(workspace, wide[:, at:at + 1003], scores, 4)
        wide.fill_(float("nan"))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,keep", [(40, 7), (9000, 8), (33000, 64)])
def test_equal_scores_go_to_the_lower_beam_and_token(workspace, dtype, V, keep):
    n, B = 2, 4
    g = torch.Generator().manual_seed(V)
    for values in (1, 2, 5):   # so many different logits in a row; every beam's row is the same, and some beams' scores are
        row = torch.randint(values, (n, 1, V), generator=g).float() * 0.5
        logits = row.expand(n, B, V).reshape(n * B, V).contiguous().to(DEV, dtype)
        scores = torch.tensor([[-1.0, -1.0, -1.0, -3.2], [-2.0, -1.7, -2.0, -1.7]], device=DEV)
        check_select(workspace, logits, scores, keep)
    signed = torch.zeros((n * B, V), device=DEV).to(dtype)
    signed[:, ::2] = -0.0      # the same number
    check_select(workspace, signed, scores, keep)


@gpu
@pytest.mark.parametrize("order", ["up", "down", "steps", "far", "late"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_in_order(workspace, dtype, order):
    """Ascending rows (every logit is better than those before it), descending ones, large and far-apart numbers, the best at the very end."""
    V = 20000
    j = torch.arange(V, dtype=torch.float64)
    x = {"up": j / 64, "down": -j / 64, "steps": (j // 1000) * 70.0, "far": (j - V / 2) * 1e34, "late": torch.where(j > V - 5, j - V + 40, j * 0)}[order]
    logits = torch.stack([x, x.flip(0) if order == "late" else x * 0.75, x * 0.5]).to(DEV, dtype)
    check_select(workspace, logits, torch.tensor([[-1.0, -2.03, -0.57]], device=DEV), 5)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_numbers_that_are_none_and_beams_that_are_gone(workspace, dtype):
    n, B, V = 4, 5, 5000
    logits, scores = make_logits(n, B, V, dtype, 11)
    logits[::3, ::2] = -float("inf")
    logits[1, 100:200] = float("nan")
    logits[2, 7], logits[2, 4999] = float("inf"), -float("nan")
    logits[5:7] = -float("inf")              # nothing left of two beams
    logits[8, :] = float("nan")
    logits[10:15] = -float("inf")            # of a whole request
    logits[15:20, 3:] = -float("inf")        # at most three candidates of a beam
    scores[0, 1], scores[1, 4], scores[3, 0], scores[3, 2] = -float("inf"), float("nan"), float("inf"), -float("inf")
    for keep in (1, 5, 9, 20):
        got = check_select(workspace, logits, scores, keep)
        assert (got.parents[2] == -1).all() and (got.tokens[2] == -1).all()
    assert (got.parents[3] == -1).sum() == 20 - 7   # three of two beams, one of a third


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_beams_that_have_ended(workspace, dtype):
    n, B, V = 6, 8, 3001
    logits, scores = make_logits(n, B, V, dtype, 12)
    logits[:, 2] += 6.0                      # the end is likely
    ended = (torch.rand((n, B), generator=torch.Generator().manual_seed(1)) < 0.4).int().to(DEV)
    ended[1], ended[2] = 0, 1
    logits[8 * 2:8 * 3] = float("nan")       # rows that are not read
    scores[3, 0] = -float("inf")             # ended or not, it is gone
    ended[3, 0] = 1
    for keep in (1, 8, 12):
        got = check_select(workspace, logits, scores, keep, end_token=2, ended=ended)
        assert (got.tokens[2, :min(keep, 8)] == 2).all() and got.ended[2, :min(keep, 8)].all()
    check_select(workspace, logits[:16], scores[:2], 8, end_token=2)   # none has, some do now
    # a result goes into the next call as it is
    first = jp.beam_select(logits[:8], scores[:1], 8, workspace, end_token=2)
    check_select(workspace, logits[8:16], first.scores, 8, end_token=2, ended=first.ended)


def beams_apart(x, scores, keep):
    """(parents, tokens) of one request whose beams' scores are equal or so far apart that no logit brings one past another: beam after beam, by
    score and number, each in the order of its logits, then of its tokens.  x [B, V], scores [B] on the CPU; NaN and infinities are no candidates."""
    out = []
    for b in sorted(range(len(scores)), key=lambda b: (-scores[b], b)):
        best = np.argsort(-x[b], kind="stable")[:keep]
        out += [(b, int(j)) for j in best if np.isfinite(x[b, j])]
    out = (out + [(-1, -1)] * keep)[:keep]
    return [b for b, _ in out], [j for _, j in out]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V,keep", [(1, 131072, 4), (2, 40000, 4), (1, 131072, 16), (3, 100000, 12), (8, 131072, 64), (5, 30011, 33)])
@pytest.mark.parametrize("scores", [[-1e12 - 1e9 * b for b in range(8)], [-1e30] * 8, [-1e30, -3e12, -1e30, -2e20, -1e12, -3e38, -5e25, 7e14]], ids=["far", "off", "mixed"])
def test_logits_of_a_beam_are_compared_whatever_its_score(workspace, dtype, B, V, keep, scores):
    """Scores in which logits vanish: within a beam the best logits come first, wherever in the row they lie (the rows are slices of several
    workgroups), and equal ones by token.  Few candidates, some hundreds and thousands are put together in ways of their own."""
    g = torch.Generator().manual_seed(B * V + keep)
    x = torch.randn((2 * B, V), generator=g, dtype=torch.float64).to(dtype)
    x[:, V - 5 * keep:] += 3.0                        # the best are late
    x[0, :V // 2 * 2:2] = x[0, 1::2]                  # and, in one row, all are there twice
    for b in range(1, 2 * B, 2):
        x[b, torch.randperm(V, generator=g)[keep // 2:]] = -float("inf")   # fewer of this beam than are kept
    s = torch.tensor([scores[:B]] * 2, dtype=torch.float32)
    # ended beams, and none of them
    for ended in (None, (torch.arange(2 * B).view(2, B) % 4 == 1).int()):
        got = jp.beam_select(x.to(DEV), s.to(DEV), keep, workspace, **({} if ended is None else dict(end_token=7, ended=ended.to(DEV))))
        for i in range(2):
            rows = f64(x)[i * B:i * B + B].copy()
            for b in range(B):
                if ended is not None and ended[i, b]:
                    rows[b] = -np.inf
                    rows[b, 7] = 0.0
            parents, tokens = beams_apart(rows, s[i].tolist(), keep)
            assert got.parents[i].tolist() == [p if p < 0 else p + i * B for p in parents]
            assert got.tokens[i].tolist() == tokens
            there = [p >= 0 for p in parents]
            want = np.array([s[i, p].item() for p in parents], np.float64)[there]
            assert (np.abs(f64(got.scores)[i][there] - want) <= 2.0 ** -24 * np.abs(want) + 400).all()   # (no logit is that far from the sum)


@gpu
@pytest.mark.parametrize("B,V,keep", [(1, 131072, 4), (1, 131072, 16), (3, 100000, 12), (8, 131072, 64)])
def test_logits_that_vanish_in_a_sum_are_compared(workspace, B, V, keep):
    """Logits that differ by less than 64 bits of a score hold, all over a row, among others far below them."""
    g = torch.Generator().manual_seed(V + keep)
    x = torch.randn((B, V), generator=g) - 30.0
    for b in range(B):
        x[b, torch.randperm(V, generator=g)[:100]] = torch.arange(100, dtype=torch.float32).add(1)[torch.randperm(100, generator=g)] * 1e-18
    s = torch.tensor([[-3.0 - 2.0 * b for b in range(B)]])   # (a beam's logits among the best lie within 1 of each other)
    got = jp.beam_select(x.to(DEV), s.to(DEV), keep, workspace)
    parents, tokens = beams_apart(f64(x), s[0].tolist(), keep)
    assert got.parents[0].tolist() == parents and got.tokens[0].tolist() == tokens


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [32000, 131072, 1 << 20])
@pytest.mark.parametrize("first", [True, False])
def test_scores_of_rows_whose_sum_lies_far_below_the_largest_logit(workspace, dtype, V, first):
    """One logit, and all others the same distance d below it, so that what the rounding of d and of d log2(e) loses does not average out: d 2^-24 each,
    and d 2^-26 of log2(e) itself.  The mean of d over the probabilities is ln V at most; an exponential is 2^-23 off and sums of eight 2^-22."""
    for d in (3.3, 6.7, 9.1, 10.1, 11.3, 12.7):
        x = torch.full((2, V), -d).to(dtype)
        x[:, 5 if first else V - 3] = 0.0
        got = jp.beam_select(x.to(DEV), torch.tensor([[-1.0, -40.0]], device=DEV), 1, workspace)
        d = -float(x[0, 0])
        want = -1.0 - np.log1p((V - 1) * np.exp(-d))
        assert got.tokens.tolist() == [[5 if first else V - 3]]
        assert abs(float(got.scores) - want) <= 2.0 ** -21 + 2.0 ** -22 * np.log(V) + 2.0 ** -24 * abs(want)


@gpu
def test_selection_in_graphs_and_on_other_streams(workspace):
    cases = [make_logits(2, 4, 32000, torch.float32, 1), make_logits(9, 3, 5000, torch.bfloat16, 2)]
    want = [jp.beam_select(x, s, 4, workspace) for x, s in cases]
    graphs = []
    for x, s in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = jp.beam_select(x, s, 4, workspace)
        graphs.append((graph, got))
    for _ in range(4):
        for (graph, got), w, (x, s) in zip(graphs, want, cases):
            for t in got:
                t.zero_()
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(got, w))
            check_select(workspace, x, s, 4)
    side, other = torch.cuda.Stream(), jp.Workspace(DEV)
    got = jp.beam_select(*cases[0], 4, other, stream=side)
    here = jp.beam_select(*cases[0], 4, workspace)          # two at once
    side.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(got, want[0], here))


@gpu
def test_no_requests(workspace):
    got = jp.beam_select(torch.zeros((0, 10), device=DEV), torch.zeros((0, 3), device=DEV), 2, workspace)
    assert got.parents.shape == (0, 2) and got.scores.dtype == torch.float32


# ---- tables ---------------------------------------------------------------------------------------------------------------------


def check_reorder(workspace, parents, table, lengths, owned, free, count, page, width=None, held=None, in_place=False):
    t = torch.tensor(table, dtype=torch.int32, device=DEV).view(len(lengths), -1 if len(lengths) else 3)
    width = t.shape[1] if width is None else width
    want = cref.reorder(parents, t.tolist(), lengths, owned, free, count, page, width, held)
    dev = dict(parents=ints(parents), lengths=ints(lengths), owned=ints(owned), free=ints(free), count=ints([count]))
    h = None if held is None else torch.tensor(held, dtype=torch.uint8, device=DEV)
    got = jp.reorder(dev["parents"], t, dev["lengths"], dev["owned"], dev["free"], dev["count"], page, workspace, held=h, width=width, in_place=in_place)
    assert got.status.tolist() == [want["status"]]
    assert got.free_count.tolist() == [want["free_count"]]
    for name in ("lengths", "owned", "copy_from", "copy_to", "free_blocks"):
        assert getattr(got, name).tolist() == want[name], name
    assert got.table.shape == (len(parents), width) and got.table.tolist() == want["table"]
    assert t.flatten().tolist() == [x for row in (table if len(table) else []) for x in row] and dev["lengths"].tolist() == list(lengths)
    if in_place:
        assert got.free_blocks is dev["free"] and got.free_count is dev["count"]
    else:
        assert dev["free"].tolist() == list(free) and dev["count"].tolist() == [count]
    return want


def random_beams(rng, n, page, width, shared=True):
    """Requests that share the pages of a prefix now and then, and some that have pages left over."""
    blocks = rng.sample(range(3 * n * width + 20), 3 * n * width + 20)
    table, lengths, owned, last = [], [], [], None
    for _ in range(n):
        length = rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, page * width)])
        length = min(length, page * width)
        need = -(-length // page)
        row = [blocks.pop() for _ in range(need)]
        if shared and last is not None and rng.random() < 0.6:
            full = rng.randint(0, min(last[1] // page, length // page))
            for j in range(full):
                blocks.append(row[j])
                row[j] = last[0][j]
        more = rng.choice([0, 0, 1, 2])
        row += [blocks.pop() for _ in range(min(more, width - need))]
        table.append(row + [-1] * (width - len(row)))
        lengths.append(length), owned.append(len(row))
        last = table[-1], length
    return table, lengths, owned, blocks


@gpu
@pytest.mark.parametrize("n,page,width,n_out", [(1, 8, 3, 1), (4, 16, 5, 4), (4, 16, 5, 9), (9, 8, 12, 4), (64, 32, 7, 64), (300, 8, 20, 300), (1500, 16, 4, 1100), (2, 65536, 2, 5), (3, 16, 700, 8)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_of_requests_that_go_on(workspace, n, page, width, n_out, in_place):
    rng = random.Random(n * page + width + n_out)
    for _ in range(3):
        table, lengths, owned, free = random_beams(rng, n, page, width)
        n_blocks = 3 * n * width + 20
        parents = [rng.randrange(n) if rng.random() < 0.9 else -1 for _ in range(n_out)]
        count = len(free)
        stack = free + [-7] * (n_blocks - count)
        assert check_reorder(workspace, parents, table, lengths, owned, stack, count, page, in_place=in_place)["status"] == 0
        held = [int(rng.random() < 0.3) for _ in range(n_blocks)]
        check_reorder(workspace, parents, table, lengths, owned, stack, count, page, width=width + 3, held=held, in_place=in_place)


@gpu
def test_tables_of_nothing(workspace):
    table, lengths, owned = [[0, 1, 2], [3, 4, -1]], [40, 17], [3, 2]
    check_reorder(workspace, [], table, lengths, owned, [9] * 8, 1, 16)                  # all go
    check_reorder(workspace, [-1, -1], table, lengths, owned, [9] * 8, 1, 16)
    check_reorder(workspace, [], [], [], [], [5, 6, 0, 0], 2, 16, width=3)
    check_reorder(workspace, [-1], [], [], [], [5, 6, 0, 0], 2, 16, width=3)
    check_reorder(workspace, [], [], [], [], [], 0, 16, width=3)
    check_reorder(workspace, [1, 0, 1], table, [0, 0], [0, 0], [9] * 8, 1, 16, width=0)  # no pages at all
    check_reorder(workspace, [0, 1], table, lengths, owned, [9] * 8, 0, 16)              # as it was; nothing is free, nothing is needed
    check_reorder(workspace, [0, 0], table, [32, 17], owned, [9] * 8, 0, 16)             # a page that is full is shared


@gpu
@pytest.mark.parametrize("status,change", [
    (1, dict(parents=[0, 2])), (1, dict(parents=[0, -2])), (1, dict(lengths=[-1, 17])), (1, dict(owned=[2, 2])), (1, dict(owned=[4, 2])), (1, dict(owned=[-1, 2])),
    (1, dict(count=-1)), (1, dict(count=9)), (2, dict(width=2)), (4, dict(parents=[0, 0, 1, 1], count=1)), (4, dict(parents=[0, 0], count=0)),
    (1, dict(parents=[0, 5], width=2)), (1, dict(width=2, owned=[3, 1]))])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_reordering_that_does_not_fit_changes_nothing(workspace, status, change, in_place):
    a = dict(dict(parents=[0, 1], table=[[0, 1, 2], [3, 4, -1]], lengths=[40, 17], owned=[3, 2], free=[7, 6, 5, 0, 0, 0, 0, 0], count=3, page=16, width=3), **change)
    assert check_reorder(workspace, in_place=in_place, **a)["status"] == status


@gpu
def test_requests_that_nobody_goes_on_from_may_hold_anything(workspace):
    """Owned numbers out of range of a request that is no parent, entries that are no blocks: nothing outside the tables is touched."""
    table = [[0, 1, 2], [3, 900, -4], [2 ** 31 - 1, -(2 ** 31), 8]]
    check_reorder(workspace, [0, 0], table, [40, 5, 7], [3, 99, -3], [5, 6, 7, 0, 0, 0, 0, 0, 0], 3, 16)
    check_reorder(workspace, [1, 1, 2], table, [40, 40, 33], [3, 3, 3], [5, 6, 7, 0, 0, 0, 0, 0, 0], 3, 16)


@gpu
def test_many_requests_and_blocks(workspace):
    n, page, width = 16384, 8, 3
    rng = np.random.default_rng(4)
    n_blocks = 200000
    order = rng.permutation(n_blocks)
    table = order[:n * width].reshape(n, width).tolist()
    lengths = rng.integers(0, 25, n).tolist()
    owned = [-(-x // page) for x in lengths]
    free = order[n * width:].tolist() + [0] * (n * width)
    check_reorder(workspace, rng.integers(0, n, n).tolist(), table, lengths, owned, free, n_blocks - n * width, page)


@gpu
@pytest.mark.parametrize("n", [2047, 2048, 2049])
def test_where_the_plan_leaves_the_workgroups_memory(workspace, n):
    rng = random.Random(n)
    table, lengths, owned, free = random_beams(rng, n, 8, 2)
    parents = [rng.choice([-1, n - 1, 0, rng.randrange(n), rng.randrange(n)]) for _ in range(1500)]
    check_reorder(workspace, parents, table, lengths, owned, free + [0] * (6 * n + 20 - len(free)), len(free), 8)


@gpu
@pytest.mark.parametrize("rows,n_free", [(32, 32768), (33, 32768), (32, 32769)])
def test_where_one_launch_ends_and_three_begin(workspace, rows, n_free):
    rng = np.random.default_rng(rows)
    lengths = rng.integers(0, 25, 32).tolist()
    owned = [-(-x // 8) for x in lengths]
    table = [[i * 3 + j if j < n else -1 for j in range(3)] for i, n in enumerate(owned)]
    free = rng.permutation(np.arange(96, 32700))[:100].tolist() + [0] * (n_free - 100)
    for in_place in (False, True):
        check_reorder(workspace, rng.integers(0, 32, rows).tolist(), table, lengths, owned, free, 100, 8, in_place=in_place)


@gpu
def test_other_rows_of_a_wider_table(workspace):
    wide = torch.arange(60, dtype=torch.int32, device=DEV).view(4, 15)
    got = jp.reorder(ints([1, 1]), wide[:, 3:6], ints([33, 40, 1, 0]), ints([3, 3, 1, 0]), ints([50] * 70), ints([5]), 16, workspace)
    assert got.table.tolist() == [[18, 19, 20], [18, 19, 50]] and got.copy_from.tolist() == [-1, 20] and got.status.tolist() == [0]


# ---- copies ---------------------------------------------------------------------------------------------------------------------


def codes_pool(kind, n_layers, n_blocks, heads, page, order, gen):
    shape = (n_layers, n_blocks, heads, page, 128)
    c = torch.randint(256, shape, generator=gen, dtype=torch.uint8).to(DEV)
    if order != "plain":
        c = c.permute(1, 0, 3, 2, 4).contiguous().permute(1, 0, 3, 2, 4)   # layers inside blocks, heads inside slots
    s = torch.rand(shape[:4], generator=gen).to(DEV)
    return c.view(kind), s


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("n_layers,heads,page", [(1, 1, 8), (3, 5, 16), (2, 40, 64), (1, 2, 4096)])
def test_pages_are_copied(dtype, n_layers, heads, page):
    gen = torch.Generator().manual_seed(page)
    n_blocks, scales = 9, None
    for order in ("plain", "inside"):
        if dtype in (torch.int8, torch.float8_e4m3fn):
            (k, ks), (v, vs) = (codes_pool(dtype, n_layers, n_blocks, heads, page, order, gen) for _ in range(2))
            scales = ks, vs
        else:
            dim = 128 if dtype == torch.bfloat16 else 6
            k, v = (torch.randn((n_layers, n_blocks, heads, page, dim), generator=gen).to(DEV, dtype) for _ in range(2))
            if order == "inside":
                k, v = (x.permute(1, 0, 3, 2, 4).contiguous().permute(1, 0, 3, 2, 4) for x in (k, v))
        source, target = [0, 3, -1, 8, 2, n_blocks, 1], [4, 5, 6, -1, 7, 1, 2 ** 31 - 1]
        lengths = [page + 3, 2 * page, 5, 5, 3 * page - 1, 5, 5]
        for given in (None, lengths):
            before = [(x.view(torch.uint8) if x.element_size() == 1 else x).clone() for x in (k, v, *(scales or ()))]
            jp.copy_pages(ints(source), ints(target), k, v, lengths=None if given is None else ints(given), scales=scales)
            for x, want in zip((k, v, *(scales or ())), before):
                for i, (a, b) in enumerate(zip(source, target)):
                    if 0 <= a < n_blocks and 0 <= b < n_blocks:
                        slots = page if given is None else lengths[i] % page
                        want[:, b, :, :slots] = want[:, a, :, :slots]
                assert torch.equal(x.view(torch.uint8) if x.element_size() == 1 else x, want)
        # one layer
        one = k[0].clone(), v[0].clone()
        jp.copy_pages(ints([0]), ints([6]), *one, scales=None if scales is None else (ks[0].clone(), vs[0].clone()))
        assert torch.equal(one[0].view(torch.uint8)[6], one[0].view(torch.uint8)[0])


# ---- together -------------------------------------------------------------------------------------------------------------------


@gpu
@pytest.mark.parametrize("kind", [None, torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("captured", [False, True])
def test_a_beam_search_over_pages(workspace, kind, captured):
    """Steps of a search, from prompts to beams: tables, rows, attention, selection, reordering, copies.  What a beam holds in its pages is, to the bit, what
    it would hold if every beam had a cache of its own that is copied whole."""
    n, B, heads, page, width, V = 3, 4, 2, 8, 9, 200
    gen = torch.Generator().manual_seed(17)
    n_blocks, rows = 150, n * B
    pool_type = kind or torch.bfloat16
    k_pool, v_pool = (torch.zeros((n_blocks, heads, page, 128), dtype=pool_type, device=DEV) for _ in range(2))
    scales = None if kind is None else tuple(torch.zeros((n_blocks, heads, page), device=DEV) for _ in range(2))
    free, count = ints(torch.randperm(n_blocks, generator=gen).tolist()), ints([n_blocks])
    # prompts of different lengths: one row each, which then become B beams
    prompt = [5, 16, 11]
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    step = jp.extend(ints([0] * n), ints(prompt), ints([0] * n), table, free, count, page, sum(prompt))
    k, v = (torch.randn((sum(prompt), heads, 128), generator=gen).to(DEV, torch.bfloat16) for _ in range(2))
    jp.append(k, v, step.slots, k_pool, v_pool, scales=scales)
    logits = torch.randn((n, V), generator=gen).to(DEV)
    beams = jp.beam_select(logits, torch.zeros((n, 1), device=DEV), B, workspace)
    after = jp.reorder(beams.parents.view(-1), table, step.lengths, step.owned, free, step.free_count, page, workspace)
    jp.copy_pages(after.copy_from, after.copy_to, k_pool, v_pool, lengths=after.lengths, scales=scales)
    at = np.cumsum([0] + prompt)
    plain = [[list(range(at[i], at[i + 1]))] * B for i in range(n)]        # the rows (numbers into `every`) of each beam
    plain = [p for group in plain for p in group]
    every = [(k, v)]
    total = sum(prompt)
    table, lengths, owned = after.table.clone(), after.lengths.clone(), after.owned.clone()
    free, count, scores = after.free_blocks.clone(), after.free_count.clone(), beams.scores.clone()
    k_in, v_in, q_in = (torch.empty((rows, heads, 128), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    mix = torch.randn((heads * 128, V), generator=gen).to(DEV)

    def one():
        s = jp.extend(lengths, torch.ones_like(lengths), owned, table, free, count, page, rows)
        jp.append(k_in, v_in, s.slots, k_pool, v_pool, scales=scales)
        out = jp.attention(q_in, k_pool, v_pool, table, s.row_start, s.lengths, 1, workspace, scales=scales)
        b = jp.beam_select(torch.mm(out.view(rows, -1).float(), mix), scores, B, workspace)
        r = jp.reorder(b.parents.view(-1), table, s.lengths, s.owned, free, s.free_count, page, workspace)
        jp.copy_pages(r.copy_from, r.copy_to, k_pool, v_pool, lengths=r.lengths, scales=scales)
        for mine, new in zip((table, lengths, owned, free, count, scores), (r.table, r.lengths, r.owned, r.free_blocks, r.free_count, b.scores)):
            mine.copy_(new)
        return out, b, r, s

    graph = None
    if captured:
        state = [x.clone() for x in (table, lengths, owned, free, count, scores)] + [x.view(torch.uint8).clone() for x in (k_pool, v_pool)] + [x.clone() for x in scales or ()]
        for x in (k_in, v_in, q_in):
            x.normal_()
        one()                                   # (libraries are loaded outside of the capture)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, b, r, s = one()
        torch.cuda.synchronize()
        for x, was in zip((table, lengths, owned, free, count, scores, k_pool.view(torch.uint8), v_pool.view(torch.uint8), *(scales or ())), state):
            x.copy_(was)
    for t in range(25):
        k, v, q = (torch.randn((rows, heads, 128), generator=gen).to(DEV, torch.bfloat16) for _ in range(3))
        for x, y in zip((k_in, v_in, q_in), (k, v, q)):
            x.copy_(y)
        before = [p + [total + i] for i, p in enumerate(plain)]
        every.append((k, v))
        total += rows
        if graph is None:
            out, b, r, s = one()
        else:
            graph.replay()
        assert s.status.tolist() == [0] and r.status.tolist() == [0], t
        parents = b.parents.flatten().tolist()
        assert all(p // B == i // B for i, p in enumerate(parents))
        plain = [list(before[p]) for p in parents]
        # pages in use are the tables', each once on the stack or in a table
        used = {x for row, m in zip(table.tolist(), owned.tolist()) for x in row[:m]}
        stack = free.tolist()[:count.item()]
        assert len(set(stack)) == len(stack) and not used & set(stack) and len(used) + len(stack) == n_blocks
        # what the beams hold
        ks, vs = torch.cat([x for x, _ in every]), torch.cat([x for _, x in every])
        slots = [int(table[i, p // page]) * page + p % page for i in range(rows) for p in range(len(plain[i]))]
        have = jp.read(ints(slots), k_pool, v_pool, scales=scales)
        for got, x in zip(have, (ks, vs)):
            want = x[torch.tensor([j for p in plain for j in p], device=DEV)]
            if kind is not None:
                name = "int8" if kind == torch.int8 else "e4m3"
                codes, scale = cref.quantise(want.float().cpu().numpy(), name)
                want = torch.from_numpy((cref.numbers(codes, name) * scale[..., None].astype(np.float64)).astype(np.float32)).to(DEV, torch.bfloat16)
            assert torch.equal(got, want), t
