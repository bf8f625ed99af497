"""Operators of a step over pages held in 8 bits, and of a step of a beam search, as measurable cases.

A server that keeps its requests' keys and values in 8 bits writes them with ``append`` (quantised as they are written), reads
them back with ``read`` and attends over them with ``attention``, all of ``paper_2504_08242_amd.paged`` and given the pool's
``scales``.  A step of a beam search ends with ``beam_select`` (the best continuations over all beams and the vocabulary) and
``reorder`` with ``copy_pages`` (block tables of the beams that go on, and copies of the pages that two of them would write to).
A case is one call of one of them, or of the two that go together.

An 8-bit pool holds codes, int8 or e4m3, and a scale for each head of each position: with m the largest magnitude among the
head's values (2^-100 at least), scale = m / T and code = x * (T / m) rounded to the nearest code, T = 127 or 448.

Where ``own`` is false ``run`` computes the same in plain torch operations.  ``exact`` is the definition in 64 bits.  The
lengths of a case's requests follow from the case, everything else from the seed.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
THETA = 1e4  # rotary base of the repository's configurations
D = 128      # head size of them
LEAST = 2.0 ** -100
CODES = {"int8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}

if torch.cuda.is_available():
    torch.backends.cuda.matmul.allow_tf32 = False


# ---- the cases ----------------------------------------------------------------------------------------------------------


def _rows(op, codes, n, heads, kv_heads, page, length, new, name=None):
    """n requests with cached lengths and new tokens spread over the given (least, most)."""
    return _named(dict(op=op, codes=codes, n=n, heads=heads, kv_heads=kv_heads, page=page, length_lo=length[0], length_hi=length[1],
                       new_lo=new[0], new_hi=new[1]), name)


def _beam(n, beams, keep, vocab, dtype, ended, name=None):
    return _named(dict(op="beam", n=n, beams=beams, keep=keep, vocab=vocab, dtype=dtype, ended=ended), name)


def _reorder(n, beams, layers, kv_heads, page, prompt, since, name=None):
    """n requests whose prompts are (least, most) tokens long, `beams` beams each that went apart `since` tokens ago."""
    return _named(dict(op="reorder", n=n, beams=beams, layers=layers, kv_heads=kv_heads, page=page, length_lo=prompt[0], length_hi=prompt[1],
                       since=since), name)


def _named(case, name):
    return dict(case, name=name) if name else case


def listed():
    return [
        # the rows of a decoding step: 16 branches of five candidates, 7B heads
        _rows("store", "e4m3", 16, 32, 32, 16, (300, 900), (5, 5), "store_branches_16x5"),
        # the rows of several prompts at once, 13B heads
        _rows("store", "int8", 6, 40, 40, 64, (0, 700), (300, 2600), "store_prompts"),
        # one request leaves the pool, grouped heads
        _rows("read", "int8", 1, 32, 8, 16, (577, 577), (0, 0), "read_request"),
        # many requests of uneven lengths leave it (they move to another device, or into a contiguous cache), 7B heads
        _rows("read", "e4m3", 12, 32, 32, 32, (40, 4100), (0, 0), "read_many"),
        # plain decoding of one request, 7B heads: the smallest attention there is
        _rows("attention", "int8", 1, 32, 32, 16, (576, 576), (1, 1), "attend_token"),
        # a decoding step of 64 requests of very different lengths, grouped heads
        _rows("attention", "e4m3", 64, 32, 8, 16, (16, 8192), (1, 1), "attend_decode_64"),
        # a chunk of a long prompt behind what earlier chunks left, 7B heads
        _rows("attention", "int8", 1, 32, 32, 64, (1536, 1536), (512, 512), "attend_chunk_512"),
        # whole prompts of uneven lengths in one call, 13B heads
        _rows("attention", "e4m3", 4, 40, 40, 128, (0, 0), (700, 4100), "attend_prompts"),
        # one request with four beams, none of which has ended
        _beam(1, 4, 4, 32000, "f32", False, "beams_1x4"),
        # a large batch and a large vocabulary, some beams ended
        _beam(64, 8, 8, 131072, "bf16", True, "beams_64x8_wide"),
        # one request with four beams goes on, eight layers of 7B heads
        _reorder(1, 4, 8, 32, 16, (300, 300), 20, "reorder_1x4"),
        # a batch of beams, grouped heads
        _reorder(64, 8, 4, 8, 16, (30, 1000), 40, "reorder_64x8"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["store", "read", "attention", "attention", "attention", "beam", "reorder"])
    page, codes = rng.choice([8, 16, 16, 32, 64, 128, 256]), rng.choice(["int8", "e4m3"])
    if op == "beam":
        vocab = rng.choice([32000, 32000, 50257, 65537, 131072, 20000 + rng.randrange(40000)])
        beams = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
        n = _log_int(rng, 1, min(64, 64 * 8 * 131072 // (beams * vocab)))
        keep = rng.randint(2, 16) if beams == 1 else beams
        return _beam(n, beams, keep, vocab, rng.choice(["f32", "bf16"]), beams > 1 and rng.random() < 0.5)
    if op == "reorder":
        beams, layers, kv_heads = rng.choice([2, 3, 4, 5, 8, 12]), rng.choice([1, 2, 4]), rng.choice([4, 8, 32])
        n = _log_int(rng, 1, min(64, 512 // beams))
        most = _log_int(rng, 16, max(16, min(1000, 500000 // (n * layers * kv_heads))))
        return _reorder(n, beams, layers, kv_heads, min(page, 64), (rng.randint(1, most), most), rng.randint(1, 60))
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (40, 40), (40, 8), (16, 2), (12, 12), (8, 1)])
    if op == "store":
        n = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, max(1, 6000 // n))
        most = _log_int(rng, 1, 2048)
        return _rows("store", codes, n, heads, kv_heads, page, (rng.randint(0, most), most), (rng.randint(1, new), new))
    if op == "read":
        n = _log_int(rng, 1, 64)
        most = _log_int(rng, 1, max(1, min(8192, 15000 // n)))
        return _rows("read", codes, n, heads, kv_heads, page, (rng.randint(0, most - 1), most), (0, 0))
    kind = rng.choice(["decode", "verify", "chunk", "prompts"])
    if kind in ("decode", "verify"):
        n = _log_int(rng, 1, 64)
        most = _log_int(rng, 64, min(16384, 1000000 // (kv_heads * n)))
        new = 1 if kind == "decode" else rng.randint(2, 16)
        return _rows("attention", codes, n, heads, kv_heads, page, (rng.randint(1, most), most), (1 if rng.random() < 0.5 else new, new))
    n = rng.randint(1, 4)
    new = _log_int(rng, 17, 2048 // n)
    most = _log_int(rng, 1, 4096) - 1 if kind == "chunk" else 0
    return _rows("attention", codes, n, heads, kv_heads, page, (rng.randint(0, most), most), (rng.randint(max(1, new // 4), new), new))


# ---- lengths: from the case alone -----------------------------------------------------------------------------------------


def _spread(n, lo, hi, salt):
    """n whole numbers between lo and hi, both among them where n allows, dense at the short end (cubes), in a mixed order."""
    if lo == hi:
        return [lo] * n
    at = [hi if n == 1 else lo + round((hi - lo) * (k / (n - 1)) ** 3) for k in range(n)]
    g = torch.Generator().manual_seed(salt)
    return [at[k] for k in torch.randperm(n, generator=g).tolist()]


def _lengths(case):
    """(cached, new) tokens of every request."""
    n = case["n"]
    return _spread(n, case["length_lo"], case["length_hi"], 2), _spread(n, case["new_lo"], case["new_hi"], 3)


def _blocks(tokens, page):
    return -(-tokens // page)


def _row_start(new):
    at = [0]
    for x in new:
        at.append(at[-1] + x)
    return at


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _generator(seed, stream):
    return torch.Generator(device=DEVICE).manual_seed((int(seed) * 1_000_003 + stream) % (1 << 62))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)


def _keys(gen, rows, heads):
    """Keys: a few features of a head are much larger than the others."""
    wide = (0.6 * torch.randn((1, heads, D), generator=gen, device=DEVICE)).exp().to(torch.bfloat16)
    return _normal(gen, rows, heads, D) * wide


def _tables(case, gen, tokens):
    """A pool in use for a while: every request's pages lie anywhere.  Block tables that hold `tokens` of each request, width
    rounded up to 8 entries with one to spare, unused entries -1; (table, blocks of the pool)."""
    page = case["page"]
    need = [_blocks(x, page) for x in tokens]
    n_blocks = sum(need) + 3
    order = torch.randperm(n_blocks, generator=gen, device=DEVICE).to(torch.int32)
    width = (max(need) // 8 + 1) * 8
    start = _ints(_row_start(need))
    column = torch.arange(width, device=DEVICE)
    at = start[:-1, None] + column[None]
    used = column[None] < _ints(need)[:, None]
    return torch.where(used, order[at.clamp(max=n_blocks - 1)], -1).contiguous(), n_blocks


def _quantised(x, codes):
    """(codes, scales) of x [..., D] in 32 bits.  (Divisions of two tensors: by a number they would be products.)"""
    dtype, top = CODES[codes]
    m = x.abs().amax(-1, keepdim=True).clamp(min=LEAST)
    t = torch.full_like(m, top)
    y = x * (t / m)
    return (y.round() if codes == "int8" else y).to(dtype), (m / t)[..., 0]


def _slots(table, page, start, first):
    """Slots of the rows that begin at `start` (rows of a ragged batch), at positions first[i], first[i] + 1, .. of request i."""
    at = torch.arange(start[-1], device=DEVICE)
    request = torch.searchsorted(_ints(start)[1:].contiguous(), at.int(), right=True)
    position = (at + _ints([a - b for a, b in zip(first, start)])[request]).to(torch.int32)
    slot = table[request, (position // page).long()] * page + position % page
    return position, slot.to(torch.int32)


def prepare(case, seed):
    gen = _generator(seed, 1)
    if case["op"] == "beam":
        return _prepare_beam(case, gen)
    if case["op"] == "reorder":
        return _prepare_reorder(case, gen)
    cached, new = _lengths(case)
    start = _row_start(new)
    rows = start[-1]
    H, Hkv, page = case["heads"], case["kv_heads"], case["page"]
    total = [a + b for a, b in zip(cached, new)]
    table, n_blocks = _tables(case, gen, total)
    s = dict(case=case, rows=rows, most_new=max(new), most_keys=max(total), table=table)
    if case["op"] == "store":  # what earlier requests left, codes of any kind
        for name in ("k", "v"):
            s[name + "_pool"], s[name + "_scale"] = _quantised(torch.zeros((n_blocks, Hkv, page, D), device=DEVICE), case["codes"])
        position, slot = _slots(table, page, start, cached)
        return s | dict(q=_normal(gen, rows, H, D), k=_keys(gen, rows, Hkv), v=_normal(gen, rows, Hkv, D), positions=position, slots=slot)
    for name in ("k", "v"):
        x = _keys(gen, n_blocks * page, Hkv) if name == "k" else _normal(gen, n_blocks * page, Hkv, D)
        codes, scale = _quantised(x.float(), case["codes"])
        s[name + "_pool"] = codes.view(torch.uint8).view(n_blocks, page, Hkv, D).transpose(1, 2).contiguous().view(codes.dtype)
        s[name + "_scale"] = scale.view(n_blocks, page, Hkv).transpose(1, 2).contiguous()
    if case["op"] == "read":
        return s | dict(slots=_slots(table, page, _row_start(total), [0] * case["n"])[1])
    return s | dict(q=_normal(gen, rows, H, D), row_start=_ints(start), lengths=_ints(total))


def _prepare_beam(case, gen):
    n, B, V = case["n"], case["beams"], case["vocab"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    # (beams of one request have read nearly the same tokens: their logits are alike)
    logits = (2.0 * torch.randn((n, 1, V), generator=gen, device=DEVICE) + 0.7 * torch.randn((n, B, V), generator=gen, device=DEVICE)).to(dtype)
    scores = -(10.0 + torch.rand((n, B), generator=gen, device=DEVICE).cumsum(1))
    ended = (torch.rand((n, B), generator=gen, device=DEVICE) < 0.2).int() if case["ended"] else None
    return dict(case=case, logits=logits.view(n * B, V), scores=scores, ended=ended, end=2 if case["ended"] else -1)


def _prepare_reorder(case, gen):
    """Beams that share their prompt's full pages and have pages of their own behind it; half of the beams have children."""
    n, B, page = case["n"], case["beams"], case["page"]
    prompt = _spread(n, case["length_lo"], case["length_hi"], 4)
    total = [p + case["since"] for p in prompt]
    shared, need = [p // page for p in prompt], [_blocks(t, page) for t in total]
    width = (max(need) // 8 + 2) * 8
    held = [a + B * (b - a) for a, b in zip(shared, need)]
    used, spare = sum(held), n * B + 40
    order = torch.randperm(used + spare, generator=gen, device=DEVICE).to(torch.int32)
    first = _ints(_row_start(held))[:-1, None, None]
    a, b = _ints(shared)[:, None, None], _ints(need)[:, None, None]
    beam, column = torch.arange(B, device=DEVICE)[:, None], torch.arange(width, device=DEVICE)
    at = torch.where(column < a, first + column, first + a + beam * (b - a) + column - a)
    table = torch.where(column < b, order[at.clamp(0, used + spare - 1).long()], -1).view(n * B, width).contiguous()
    alive = -(-B // 2)
    order_of = torch.rand((n, B), generator=gen, device=DEVICE).argsort(1)[:, :alive]
    pick = torch.cat([torch.arange(alive, device=DEVICE).expand(n, alive), torch.randint(alive, (n, B - alive), generator=gen, device=DEVICE)], 1)
    parents = (order_of.gather(1, pick) + B * torch.arange(n, device=DEVICE)[:, None]).view(-1).int()
    free = torch.full((used + spare,), -1, dtype=torch.int32, device=DEVICE)
    free[:spare] = order[used:]
    shape = (case["layers"], used + spare, case["kv_heads"], page, D)
    lengths = _ints([t for t in total for _ in range(B)])
    return dict(case=case, table=table, parents=parents, lengths=lengths, owned=_ints([x for x in need for _ in range(B)]), free=free,
                free_count=_ints([spare]), k_pools=_normal(gen, *shape), v_pools=_normal(gen, *shape))


# ---- one pass ---------------------------------------------------------------------------------------------------------------


_workspaces = []  # a program's one workspace, on the stream that all its calls are on


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"store": _plain_store, "read": _plain_read, "attention": _plain_attention, "beam": _plain_beam, "reorder": _plain_reorder}[op](s)
    from paper_2504_08242_amd import paged
    if not _workspaces:
        _workspaces.append(paged.Workspace(DEVICE))
    if op == "beam":
        return paged.beam_select(s["logits"], s["scores"], s["case"]["keep"], _workspaces[0], end_token=s["end"], ended=s["ended"])._asdict()
    if op == "reorder":
        after = paged.reorder(s["parents"], s["table"], s["lengths"], s["owned"], s["free"], s["free_count"], s["case"]["page"], _workspaces[0])
        paged.copy_pages(after.copy_from, after.copy_to, s["k_pools"], s["v_pools"], lengths=after.lengths)
        return dict(after._asdict(), k_pools=s["k_pools"], v_pools=s["v_pools"])
    scales = (s["k_scale"], s["v_scale"])
    if op == "store":
        q = paged.append(s["k"], s["v"], s["slots"], s["k_pool"], s["v_pool"], positions=s["positions"], rope_theta=THETA, q=s["q"], scales=scales)
        k, v = paged.read(s["slots"], s["k_pool"], s["v_pool"], scales=scales)
        return dict(q=q, k=k, v=v, k_scale=s["k_scale"], v_scale=s["v_scale"])
    if op == "read":
        return paged.read(s["slots"], s["k_pool"], s["v_pool"], scales=scales)
    return paged.attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["row_start"], s["lengths"], s["most_new"], _workspaces[0], scales=scales)


def _rotate(x, position):
    """x [rows, heads, D] in 32 bits, halves rotated against each other; angles in 64 bits."""
    half = D // 2
    angle = position.double()[:, None] * THETA ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * n, b * c + a * n], -1)


def _plain_read_rows(s, name):
    page, slot = s["case"]["page"], s["slots"].long()
    block, at = slot // page, slot % page
    pool = s[name + "_pool"]  # (indexing knows no 8-bit floats)
    rows = pool.view(torch.uint8)[block, :, at].view(pool.dtype)
    return (rows.float() * s[name + "_scale"][block, :, at][..., None]).to(torch.bfloat16)


def _plain_read(s):
    return _plain_read_rows(s, "k"), _plain_read_rows(s, "v")


def _plain_store(s):
    page, slot = s["case"]["page"], s["slots"].long()
    block, at = slot // page, slot % page
    for name, x in (("k", _rotate(s["k"].float(), s["positions"])), ("v", s["v"].float())):
        codes, scale = _quantised(x, s["case"]["codes"])
        s[name + "_pool"].view(torch.uint8)[block, :, at] = codes.view(torch.uint8)
        s[name + "_scale"][block, :, at] = scale
    k, v = _plain_read(s)
    return dict(q=_rotate(s["q"].float(), s["positions"]).to(torch.bfloat16), k=k, v=v, k_scale=s["k_scale"], v_scale=s["v_scale"])


def _padded_rows(s):
    """(request, place in it) of every row: where a [requests, most new tokens] layout has it."""
    at = torch.arange(s["rows"], device=DEVICE, dtype=torch.int32)
    request = torch.searchsorted(s["row_start"][1:].contiguous(), at, right=True)
    return request, at - s["row_start"][request]


def _plain_attention(s):
    H, Hkv, page, n = s["case"]["heads"], s["case"]["kv_heads"], s["case"]["page"], s["case"]["n"]
    most, keys = s["most_new"], s["most_keys"]
    request, place = _padded_rows(s)
    pages = s["table"][:, :_blocks(keys, page)].clamp(min=0).long()

    def whole(name):
        codes, scale = s[name + "_pool"], s[name + "_scale"]
        x = codes.view(torch.uint8)[pages].view(codes.dtype).float() * scale[pages][..., None]
        return x.transpose(1, 2).reshape(n, Hkv, -1, D)

    k, v = whole("k"), whole("v")
    q = torch.zeros((n, most, H, D), device=DEVICE)
    q[request, place] = s["q"].float() / math.sqrt(D)
    q = q.view(n, most, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, H // Hkv * most, D)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).view(n, Hkv, H // Hkv, most, -1)
    new = s["row_start"][1:] - s["row_start"][:-1]
    last = (s["lengths"] - new)[:, None] + torch.arange(most, device=DEVICE)  # the last key that each row sees
    hidden = torch.arange(score.shape[-1], device=DEVICE) > last[:, :, None]
    p = torch.where(hidden[:, None, None], -math.inf, score)
    p = (p - p.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(n, Hkv, -1, p.shape[-1]), v).view(n, Hkv, H // Hkv, most, D)
    return out.permute(0, 3, 1, 2, 4).reshape(n, most, H, D)[request, place].to(s["q"].dtype)


def _plain_beam(s):
    n, B, K, V, end = s["case"]["n"], s["case"]["beams"], s["case"]["keep"], s["case"]["vocab"], s["end"]
    # (64 bits: what is chosen goes by comparisons of neighbouring values)
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    score = s["scores"].double().view(-1, 1) + (x - (top + (x - top).exp().sum(-1, keepdim=True).log()))
    if s["ended"] is not None:
        ended = s["ended"].view(-1, 1) != 0
        at_end = torch.arange(V, device=DEVICE) == end
        score = torch.where(ended, torch.where(at_end, s["scores"].double().view(-1, 1), -math.inf), score)
    best, at = score.view(n, B * V).sort(dim=1, descending=True, stable=True)
    best, at = best[:, :K], at[:, :K]
    beam, token = at // V, (at % V).int()
    parents = (beam + B * torch.arange(n, device=DEVICE)[:, None]).int()
    before = s["ended"].gather(1, beam) if s["ended"] is not None else torch.zeros_like(token)
    return dict(parents=parents, tokens=token, scores=best.float(), ended=((before != 0) | (token == end)).int())


def _plain_reorder(s):
    page, parents, table = s["case"]["page"], s["parents"].long(), s["table"]
    n, n_free = parents.numel(), s["free"].numel()
    length = s["lengths"][parents]
    full, rest = length // page, length % page
    need = full + (rest > 0).int()
    first = ~(parents[:, None] == parents[None]).tril(-1).any(1)
    copied = ~first & (rest > 0)
    rank = copied.cumsum(0) - copied.long()
    taken = s["free"][(s["free_count"] - 1 - rank).clamp(0, n_free - 1).long()]
    column = torch.arange(table.shape[1], device=DEVICE, dtype=torch.int32)
    old = table[parents]
    new = torch.where(column < need[:, None], old, -1)
    new = torch.where(copied[:, None] & (column == full[:, None]), taken[:, None], new)
    # pages that were in use and are not any more, in the order of their numbers
    before, after = torch.zeros(n_free + 1, dtype=torch.bool, device=DEVICE), torch.zeros(n_free + 1, dtype=torch.bool, device=DEVICE)
    before[torch.where(column < s["owned"][:, None], table, n_free).long().view(-1)] = True
    after[torch.where(column < need[:, None], new, n_free).long().view(-1)] = True
    gone = (before & ~after)[:n_free]
    left = s["free_count"] - copied.sum()
    free = torch.cat([s["free"], s["free"][:1]])
    free[torch.where(gone, left + gone.cumsum(0) - 1, n_free).long()] = torch.arange(n_free, device=DEVICE, dtype=torch.int32)
    from_block = old.gather(1, full.clamp(max=table.shape[1] - 1)[:, None].long())[:, 0]
    # (a row without a copy copies its page onto itself)
    source = torch.where(rest > 0, from_block, new[:, 0]).long()
    target = torch.where(copied, taken, source.int()).long()
    inside = torch.arange(page, device=DEVICE)[None] < rest[:, None]
    for pools in (s["k_pools"], s["v_pools"]):
        pools[:, target] = torch.where(inside[None, :, None, :, None], pools[:, source], pools[:, target])
    return dict(table=new, lengths=length, owned=need.int(), free_blocks=free[:n_free], free_count=(left + gone.sum()).int(),
                copy_from=torch.where(copied, from_block, -1), copy_to=torch.where(copied, taken, -1), status=torch.zeros_like(s["free_count"]),
                k_pools=s["k_pools"], v_pools=s["v_pools"])


# ---- what a pass cannot do without --------------------------------------------------------------------------------------


def work(case):
    op, n = case["op"], case["n"]
    if op == "beam":
        size, rows = 4 if case["dtype"] == "f32" else 2, n * case["beams"]
        read = rows * (0.8 if case["ended"] else 1.0)  # (rows of beams that have ended are not read)
        return {"bytes": float(read * case["vocab"] * size + 4 * rows + 16 * n * case["keep"]), "flops": 4.0 * read * case["vocab"]}
    if op == "reorder":
        prompt = _spread(n, case["length_lo"], case["length_hi"], 4)
        page, B = case["page"], case["beams"]
        need = [_blocks(p + case["since"], page) for p in prompt]
        copied = sum((p + case["since"]) % page for p in prompt) * (B - -(-B // 2))
        # tables in and out, lengths, and pages of which two beams would write to the rest: in and out, keys and values
        return {"bytes": float(8 * B * sum(need) + 32 * n * B + copied * 2 * 2 * 2 * D * case["kv_heads"] * case["layers"]), "flops": 0.0}
    cached, new = _lengths(case)
    rows, H, Hkv = sum(new), case["heads"], case["kv_heads"]
    if op == "store":  # rows in, codes and scales out; and the same rows from codes and scales back
        return {"bytes": float(rows * (4 * H * D + 2 * Hkv * (2 * D + D + 4) + 2 * Hkv * (D + 4 + 2 * D)) + 12 * rows), "flops": 8.0 * rows * (H + Hkv) * D}
    if op == "read":
        rows = sum(cached)
        return {"bytes": float(rows * (2 * Hkv * (D + 4 + 2 * D) + 4)), "flops": 2.0 * rows * Hkv * D}
    keys = sum(a + b for a, b in zip(cached, new))
    pairs = sum(b * a + b * (b + 1) / 2 for a, b in zip(cached, new))
    return {"bytes": 4.0 * rows * H * D + 2.0 * keys * Hkv * (D + 4) + 4.0 * keys / case["page"] + 8.0 * n, "flops": 4.0 * D * H * pairs}


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------------


def _nearest(y, codes):
    """The code nearest to y, in 64 bits; ties to even."""
    if codes == "int8":
        return torch.round(y).clamp(-127, 127)
    _, exponent = torch.frexp(y)  # |y| in [2^(e-1), 2^e): three bits behind the first, down to steps of 2^-9
    step = torch.ldexp(torch.ones_like(y), (exponent - 4).clamp(min=-9))
    return (torch.round(y / step) * step).clamp(-448, 448)


def _turned(x, position):
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       position.double()[:, None, None] / THETA ** (torch.arange(0, D, 2, device=DEVICE, dtype=torch.float64) / D))
    z = torch.complex(x[..., :D // 2].double(), x[..., D // 2:].double()) * turn
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    """The definitions, request by request (no plain form, no kernel).  Whole numbers are the same whatever the bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "reorder":
        return None
    if op == "beam":
        n, B, K, V = case["n"], case["beams"], case["keep"], case["vocab"]
        scores = torch.empty((n, K), dtype=torch.float64, device=DEVICE)
        for i in range(n):
            candidates = []
            for b in range(B):
                so_far = s["scores"][i, b].double()
                if s["ended"] is not None and int(s["ended"][i, b]):
                    candidates.append(so_far.view(1))
                else:
                    candidates.append(so_far + torch.log_softmax(s["logits"][i * B + b].double(), 0).topk(K).values)
            scores[i] = torch.cat(candidates).topk(K).values
        return dict(parents=None, tokens=None, scores=scores, ended=None)
    H, Hkv, page = case["heads"], case["kv_heads"], case["page"]
    if op == "store":
        out = dict(q=_turned(s["q"], s["positions"]))
        block, at = s["slots"].long().div(page, rounding_mode="floor"), s["slots"].long() % page
        top = CODES[case["codes"]][1]
        for name, x in (("k", _turned(s["k"], s["positions"])), ("v", s["v"].double())):
            scale = x.abs().max(-1).values / top
            out[name] = _nearest(x / scale[..., None], case["codes"]) * scale[..., None]
            pool = s[name + "_scale"].double()
            pool[block, :, at] = scale
            out[name + "_scale"] = pool
        return out
    whole = {name: s[name + "_pool"].double() * s[name + "_scale"].double()[..., None] for name in ("k", "v")}
    if op == "read":
        block, at = s["slots"].long().div(page, rounding_mode="floor"), s["slots"].long() % page
        return whole["k"][block, :, at], whole["v"][block, :, at]
    cached, new = _lengths(case)
    start = _row_start(new)
    out = torch.empty((s["rows"], H, D), dtype=torch.float64, device=DEVICE)
    for i in range(case["n"]):
        keys = cached[i] + new[i]
        blocks = s["table"][i, :_blocks(keys, page)].long()
        k = whole["k"][blocks].transpose(1, 2).flatten(0, 1)[:keys]  # [keys, Hkv, D]
        v = whole["v"][blocks].transpose(1, 2).flatten(0, 1)[:keys]
        q = s["q"][start[i]:start[i + 1]].double()
        seen = torch.ones((new[i], keys), dtype=torch.bool, device=DEVICE).tril(cached[i])
        for h in range(H):
            g = h // (H // Hkv)
            score = (q[:, h] @ k[:, g].T.contiguous() / D ** 0.5).masked_fill(~seen, -math.inf)
            out[start[i]:start[i + 1], h] = torch.softmax(score, -1) @ v[:, g].contiguous()
    return out
