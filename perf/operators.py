"""The operators of a step over a paged cache, as measurable cases.

A step of a server that keeps its requests' keys and values in pages of one pool goes through four operators of
``paper_2504_08242_amd.paged``: ``extend`` (block tables, positions and slots of the step from the requests' lengths),
``append`` (rotary embedding, keys and values into their slots), ``attention`` (the new tokens over the pages) and ``verify``
(drafted tokens against the target's probabilities, from given random numbers).  A case is one call of one of them.

Where ``own`` is false ``run`` computes the same in plain torch operations.  ``exact`` is the definition in 64 bits.  The
lengths of a case's requests follow from the case, everything else from the seed.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
THETA = 1e4  # rotary base of the repository's configurations

if torch.cuda.is_available():
    torch.backends.cuda.matmul.allow_tf32 = False


# ---- the cases ----------------------------------------------------------------------------------------------------------


def _extend(n, page, length, new, name=None):
    """n requests with cached lengths and new tokens spread over the given (least, most)."""
    return _named(dict(op="extend", n=n, page=page, length_lo=length[0], length_hi=length[1], new_lo=new[0], new_hi=new[1]), name)


def _rows(op, n, heads, kv_heads, page, length, new, name=None):
    return _named(dict(op=op, n=n, heads=heads, kv_heads=kv_heads, page=page, length_lo=length[0], length_hi=length[1],
                       new_lo=new[0], new_hi=new[1]), name)


def _verify(n, drafts, vocab, dtype, from_draft, name=None):
    return _named(dict(op="verify", n=n, drafts_lo=drafts[0], drafts_hi=drafts[1], vocab=vocab, dtype=dtype, from_draft=from_draft), name)


def _named(case, name):
    return dict(case, name=name) if name else case


def listed():
    return [
        # the tables of a decoding step: eight outline branches of one token and four candidates each
        _extend(8, 16, (200, 900), (5, 5), "tables_branches_8x5"),
        # a large server's step in which most requests decode and some bring prompts: 60 000 rows
        _extend(1024, 16, (0, 8192), (1, 230), "tables_mixed_1024"),
        # keys, values and queries of 16 branches of five candidates, 7B heads
        _rows("append", 16, 32, 32, 16, (300, 900), (5, 5), "append_branches_16x5"),
        # the rows of several prompts at once, 13B heads
        _rows("append", 6, 40, 40, 64, (0, 700), (300, 2600), "append_prompts"),
        # plain decoding of one request, 7B heads: the smallest call there is
        _rows("attention", 1, 32, 32, 16, (576, 576), (1, 1), "attend_token"),
        # a decoding step of 64 requests of very different lengths, grouped heads
        _rows("attention", 64, 32, 8, 16, (16, 8192), (1, 1), "attend_decode_64"),
        # speculative verification: 16 requests, one token and four candidates each, 7B heads
        _rows("attention", 16, 32, 32, 32, (500, 2100), (5, 5), "attend_verify_16x5"),
        # a chunk of a long prompt behind what earlier chunks left, 7B heads
        _rows("attention", 1, 32, 32, 64, (1536, 1536), (512, 512), "attend_chunk_512"),
        # whole prompts of uneven lengths in one call, 13B heads
        _rows("attention", 4, 40, 40, 128, (0, 0), (700, 4100), "attend_prompts"),
        # one request's four candidates, taken for certain by the drafting heads
        _verify(1, (4, 4), 32000, "bf16", False, "verify_1x4"),
        # a step of 16 requests whose drafts come from a small model's distribution
        _verify(16, (4, 4), 32000, "f32", True, "verify_16x4"),
        # a large batch and a large vocabulary, uneven numbers of drafts
        _verify(64, (0, 8), 131072, "f32", True, "verify_64_wide"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["extend", "append", "attention", "attention", "attention", "verify"])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    if op == "extend":
        n, most = _log_int(rng, 1, 1024), _log_int(rng, 1, 8192)
        new = _log_int(rng, 1, max(1, min(2000, 60000 // n)))
        return _extend(n, page, (rng.randint(0, most), most), (rng.randint(0, new), new))
    if op == "verify":
        n, vocab = _log_int(rng, 1, 64), rng.choice([32000, 32000, 50257, 65537, 131072, 20000 + rng.randrange(40000)])
        drafts = rng.randint(0, 8)
        return _verify(n, (rng.randint(0, drafts), drafts), vocab, rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.6)
    heads, kv_heads = rng.choice([(32, 32), (32, 8), (40, 40), (40, 8), (16, 2), (12, 12), (8, 1)])
    if op == "append":
        n = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, max(1, 6000 // n))
        most = _log_int(rng, 1, 2048)
        return _rows("append", n, heads, kv_heads, page, (rng.randint(0, most), most), (rng.randint(1, new), new))
    kind = rng.choice(["decode", "verify", "chunk", "prompts"])
    if kind in ("decode", "verify"):
        n = _log_int(rng, 1, 64)
        most = _log_int(rng, 64, min(16384, 1000000 // (kv_heads * n)))
        new = 1 if kind == "decode" else rng.randint(2, 16)
        return _rows("attention", n, heads, kv_heads, page, (rng.randint(1, most), most), (1 if rng.random() < 0.5 else new, new))
    n = rng.randint(1, 4)
    new = _log_int(rng, 17, 2048 // n)
    most = _log_int(rng, 1, 4096) - 1 if kind == "chunk" else 0
    return _rows("attention", n, heads, kv_heads, page, (rng.randint(0, most), most), (rng.randint(max(1, new // 4), new), new))


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
    if case["op"] == "verify":
        return [500] * n, [1 + d for d in _spread(n, case["drafts_lo"], case["drafts_hi"], 1)]
    return _spread(n, case["length_lo"], case["length_hi"], 2), _spread(n, case["new_lo"], case["new_hi"], 3)


def _blocks(tokens, page):
    return -(-tokens // page)


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _generator(seed, stream):
    return torch.Generator(device=DEVICE).manual_seed((int(seed) * 1_000_003 + stream) % (1 << 62))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)


def _row_start(new):
    at = [0]
    for x in new:
        at.append(at[-1] + x)
    return at


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


def prepare(case, seed):
    cached, new = _lengths(case)
    start = _row_start(new)
    rows = start[-1]
    gen = _generator(seed, 1)
    s = dict(case=case, rows=rows, most_new=max(new), most_keys=max(a + b for a, b in zip(cached, new)))
    if case["op"] == "extend":
        page = case["page"]
        held, n_blocks = _tables(case, gen, cached)
        width = (max(_blocks(a + b, page) for a, b in zip(cached, new)) // 8 + 1) * 8
        fresh = sum(_blocks(a + b, page) - _blocks(a, page) for a, b in zip(cached, new))
        table = torch.full((case["n"], width), -1, dtype=torch.int32, device=DEVICE)
        table[:, :min(width, held.shape[1])] = held[:, :width]
        # the blocks nobody holds, in the order in which they were given back
        free = n_blocks + torch.randperm(fresh + 64, generator=gen, device=DEVICE).to(torch.int32)
        s |= dict(table=table, lengths=_ints(cached), new=_ints(new), owned=_ints([_blocks(a, page) for a in cached]),
                  free=free, free_count=_ints([free.numel()]), max_rows=rows + 7)
        return s
    if case["op"] == "verify":
        V, dtype = case["vocab"], torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        g = torch.randn((rows, V), generator=gen, device=DEVICE)
        target = torch.softmax(2.0 * g, -1)
        if case["from_draft"]:
            near = torch.softmax(2.0 * g + 0.7 * torch.randn((rows, V), generator=gen, device=DEVICE), -1).to(dtype)
            s["draft"] = near
            drawn = torch.multinomial(near.float(), 1, generator=gen)[:, 0]
        else:
            s["draft"] = None
            drawn = torch.multinomial(target, 1, generator=gen)[:, 0]
            if rows > 1:  # two drafts of three are what the target would say, the others the target's most likely
                drawn = torch.where(torch.rand(rows, generator=gen, device=DEVICE) < 0.67, target.argmax(-1), drawn)
        tokens = torch.randint(V, (rows,), generator=gen, device=DEVICE, dtype=torch.int32)
        tokens[1:] = drawn[:-1].to(torch.int32)  # row r's distribution is that of the token in row r + 1
        s |= dict(target=target.to(dtype), tokens=tokens, row_start=_ints(start), lengths=_ints(cached),
                  u_accept=torch.rand(rows, generator=gen, device=DEVICE), u_sample=torch.rand(case["n"], generator=gen, device=DEVICE))
        if not case["from_draft"]:
            # drafts taken for certain are accepted with the target's own probability of them: a real target is that sure
            likely = torch.zeros(rows, device=DEVICE)
            likely[:-1] = 0.8 * torch.rand(rows - 1, generator=gen, device=DEVICE)
            mixed = target * (1.0 - likely[:, None])
            mixed[torch.arange(rows - 1, device=DEVICE), tokens[1:].long()] += likely[:-1]
            s["target"] = mixed.to(dtype)
        return s
    H, Hkv, page, D = case["heads"], case["kv_heads"], case["page"], 128
    total = [a + b for a, b in zip(cached, new)]
    table, n_blocks = _tables(case, gen, total)
    s |= dict(q=_normal(gen, rows, H, D), k_pool=_normal(gen, n_blocks, Hkv, page, D), v_pool=_normal(gen, n_blocks, Hkv, page, D),
              table=table, row_start=_ints(start), lengths=_ints(total))
    if case["op"] == "append":
        at = torch.arange(rows, device=DEVICE)
        request = torch.searchsorted(s["row_start"][1:].contiguous(), at.int(), right=True)
        position = (at + _ints([a - b for a, b in zip(cached, start)])[request]).to(torch.int32)
        slot = table[request, (position // page).long()] * page + position % page
        s |= dict(k=_normal(gen, rows, Hkv, D), v=_normal(gen, rows, Hkv, D), positions=position, slots=slot.to(torch.int32))
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------


_workspaces = []  # a program's one workspace, on the stream that all its calls are on


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"extend": _plain_extend, "append": _plain_append, "attention": _plain_attention, "verify": _plain_verify}[op](s)
    from paper_2504_08242_amd import paged
    if op == "extend":
        step = paged.extend(s["lengths"], s["new"], s["owned"], s["table"], s["free"], s["free_count"], s["case"]["page"], s["max_rows"])
        return dict(step._asdict(), table=s["table"])
    if op == "append":
        q = paged.append(s["k"], s["v"], s["slots"], s["k_pool"], s["v_pool"], positions=s["positions"], rope_theta=THETA, q=s["q"])
        return dict(q=q, k_pool=s["k_pool"], v_pool=s["v_pool"])
    if not _workspaces:
        _workspaces.append(paged.Workspace(DEVICE))
    if op == "attention":
        return paged.attention(s["q"], s["k_pool"], s["v_pool"], s["table"], s["row_start"], s["lengths"], s["most_new"], _workspaces[0])
    return paged.verify(s["tokens"], s["target"], s["row_start"], s["u_accept"], s["u_sample"], _workspaces[0], draft_probs=s["draft"],
                        lengths=s["lengths"])._asdict()


def _plain_extend(s):
    page, table, owned, free, most = s["case"]["page"], s["table"], s["owned"], s["free"], s["max_rows"]
    total = s["lengths"] + s["new"]
    fresh = ((total + page - 1) // page - owned).clamp(min=0)
    before = fresh.cumsum(0) - fresh
    left = s["free_count"] - fresh.sum()
    row_start = torch.cat([torch.zeros_like(total[:1]), s["new"].cumsum(0)])
    rows = torch.arange(most, device=DEVICE, dtype=torch.int32)
    column = torch.arange(table.shape[1], device=DEVICE, dtype=torch.int32)
    j = column[None] - owned[:, None]
    taken = (s["free_count"] - 1 - before[:, None] - j).clamp(0, free.numel() - 1)
    table.copy_(torch.where((j >= 0) & (j < fresh[:, None]), free[taken], table))
    request = torch.searchsorted(row_start[1:].contiguous(), rows.long(), right=True).clamp(max=total.numel() - 1)
    position = s["lengths"][request] + rows - row_start[request]
    there = rows < row_start[-1]
    block = table[request, (position // page).clamp(0, table.shape[1] - 1).long()]
    return dict(row_start=row_start.int(), positions=torch.where(there, position, 0).int(),
                slots=torch.where(there, block * page + position % page, -1).int(), lengths=total, owned=owned + fresh.int(),
                free_count=left.int(), status=torch.zeros_like(s["free_count"]), table=table)


def _rotate(x, position, dtype):
    """x [rows, heads, D] in `dtype`, halves rotated against each other; angles in 64 bits."""
    half = x.shape[-1] // 2
    angle = position.double()[:, None] * THETA ** (-torch.arange(half, device=x.device, dtype=torch.float64) / half)
    c, n = angle.cos().to(dtype)[:, None], angle.sin().to(dtype)[:, None]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * c - b * n, b * c + a * n], -1)


def _plain_append(s):
    page, slot = s["case"]["page"], s["slots"].long()
    block, at = slot // page, slot % page
    s["k_pool"][block, :, at] = _rotate(s["k"].float(), s["positions"], torch.float32).to(torch.bfloat16)
    s["v_pool"][block, :, at] = s["v"]
    return dict(q=_rotate(s["q"].float(), s["positions"], torch.float32).to(torch.bfloat16), k_pool=s["k_pool"], v_pool=s["v_pool"])


def _padded_rows(s):
    """(request, place in it) of every row: where a [requests, most new tokens] layout has it."""
    at = torch.arange(s["rows"], device=DEVICE, dtype=torch.int32)
    request = torch.searchsorted(s["row_start"][1:].contiguous(), at, right=True)
    return request, at - s["row_start"][request]


def _plain_attention(s):
    H, Hkv, page, n = s["case"]["heads"], s["case"]["kv_heads"], s["case"]["page"], s["case"]["n"]
    D, most, keys = s["q"].shape[-1], s["most_new"], s["most_keys"]
    request, place = _padded_rows(s)
    pages = s["table"][:, :_blocks(keys, page)].clamp(min=0).long()
    k = s["k_pool"][pages].transpose(1, 2).reshape(n, Hkv, -1, D).float()
    v = s["v_pool"][pages].transpose(1, 2).reshape(n, Hkv, -1, D).float()
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
    # (slots behind a request's last token hold what earlier requests left: finite here, and weighted by 0)
    out = torch.matmul(p.view(n, Hkv, -1, p.shape[-1]), v).view(n, Hkv, H // Hkv, most, D)
    return out.permute(0, 3, 1, 2, 4).reshape(n, most, H, D)[request, place].to(s["q"].dtype)


def _plain_verify(s):
    start, tokens, V, n = s["row_start"], s["tokens"], s["case"]["vocab"], s["case"]["n"]
    rows, most = s["rows"], s["most_new"]
    new = start[1:] - start[:-1]
    # every row's draft (the token of the next row), its probabilities and whether it would be accepted; 64 bits, as these
    # are comparisons of neighbouring values
    drafted = torch.cat([tokens[1:], tokens[:1]]).long()
    at = torch.arange(rows, device=DEVICE)
    p = s["target"][at, drafted].double()
    q = s["draft"][at, drafted].double() if s["draft"] is not None else torch.ones_like(p)
    accepted = s["u_accept"].double() * q < p
    column = torch.arange(most, device=DEVICE)
    padded = (start[:-1, None] + column).clamp(max=rows - 1).long()
    run_of = (accepted[padded] & (column < new[:, None] - 1)).int().cumprod(1)
    n_accepted = run_of.sum(1).int()
    row = (start[:-1] + n_accepted).long()
    rejected = n_accepted < new - 1
    w = s["target"][row].double()
    if s["draft"] is not None:
        w = torch.where(rejected[:, None], (w - s["draft"][row].double()).clamp(min=0), w)
    else:
        w = torch.where(rejected[:, None] & (torch.arange(V, device=DEVICE) == drafted[row][:, None]), 0.0, w)
    total = w.cumsum(1)
    following = (total <= s["u_sample"].double()[:, None] * total[:, -1:]).sum(1).clamp(max=V - 1).int()
    request, place = _padded_rows(s)
    emitted = torch.where(place < n_accepted[request], drafted.int(), torch.where(place == n_accepted[request], following[request], -1))
    return dict(n_accepted=n_accepted, next_token=following, emitted=emitted, lengths=s["lengths"] + 1 + n_accepted)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------


def work(case):
    cached, new = _lengths(case)
    n, rows = case["n"], sum(new)
    if case["op"] == "extend":
        page = case["page"]
        fresh = sum(_blocks(a + b, page) - _blocks(a, page) for a, b in zip(cached, new))
        touched = sum(_blocks(a + b, page) - a // page for a, b in zip(cached, new))  # table entries that rows go through
        return {"bytes": 4.0 * (6 * n + 4 + 2 * fresh + touched + 2 * (rows + 7)), "flops": 0.0}
    if case["op"] == "verify":  # a few single values per request, and one row of the vocabulary of it (of the draft's too)
        size = 4 if case["dtype"] == "f32" else 2
        both = 2 if case["from_draft"] else 1
        return {"bytes": float(n * case["vocab"] * size * both + rows * (8 + 2 * 32 + 4) + 24 * n), "flops": 3.0 * n * case["vocab"]}
    H, Hkv, D = case["heads"], case["kv_heads"], 128
    if case["op"] == "append":
        return {"bytes": 2.0 * 2 * rows * (H + 2 * Hkv) * D + 8.0 * rows, "flops": 3.0 * rows * (H + Hkv) * D}
    keys = sum(a + b for a, b in zip(cached, new))
    pairs = sum(b * a + b * (b + 1) / 2 for a, b in zip(cached, new))
    return {"bytes": 2.0 * 2 * (rows * H + keys * Hkv) * D + 4.0 * keys / case["page"] + 8.0 * n, "flops": 4.0 * D * H * pairs}


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions, request by request (no plain form, no kernel).  Whole numbers are the same whatever the bits."""
    s = prepare(case, seed)
    cached, new = _lengths(case)
    start = _row_start(new)
    if case["op"] == "extend":
        return None
    if case["op"] == "append":
        D = 128
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                           s["positions"].double()[:, None, None] / THETA ** (torch.arange(0, D, 2, device=DEVICE, dtype=torch.float64) / D))

        def turned(x):
            z = torch.complex(x[..., :D // 2].double(), x[..., D // 2:].double()) * turn
            return torch.cat([z.real, z.imag], -1)

        k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
        block, at = s["slots"].long().div(case["page"], rounding_mode="floor"), s["slots"].long() % case["page"]
        k_pool[block, :, at] = turned(s["k"])
        v_pool[block, :, at] = s["v"].double()
        return dict(q=turned(s["q"]), k_pool=k_pool, v_pool=v_pool)
    if case["op"] == "attention":
        H, Hkv, page, D = case["heads"], case["kv_heads"], case["page"], 128
        out = torch.empty((s["rows"], H, D), dtype=torch.float64, device=DEVICE)
        for i in range(case["n"]):
            keys = cached[i] + new[i]
            blocks = s["table"][i, :_blocks(keys, page)].long()
            k = s["k_pool"][blocks].transpose(1, 2).flatten(0, 1)[:keys].double()  # [keys, Hkv, D]
            v = s["v_pool"][blocks].transpose(1, 2).flatten(0, 1)[:keys].double()
            q = s["q"][start[i]:start[i + 1]].double()
            seen = torch.ones((new[i], keys), dtype=torch.bool, device=DEVICE).tril(cached[i])
            for h in range(H):
                g = h // (H // Hkv)
                score = (q[:, h] @ k[:, g].T.contiguous() / D ** 0.5).masked_fill(~seen, -math.inf)
                out[start[i]:start[i + 1], h] = torch.softmax(score, -1) @ v[:, g].contiguous()
        return out
    tokens, u, us = s["tokens"].tolist(), s["u_accept"].double().tolist(), s["u_sample"].double().tolist()
    n_accepted, following, emitted, lengths = [], [], [], []
    for i in range(case["n"]):
        row, said = start[i], []
        while row + 1 < start[i + 1]:
            x = tokens[row + 1]
            q = float(s["draft"][row, x].double()) if s["draft"] is not None else 1.0
            if not u[row] * q < float(s["target"][row, x].double()):
                break
            said.append(x)
            row += 1
        w = s["target"][row].double().cpu()
        if row + 1 < start[i + 1]:  # rejected there
            if s["draft"] is not None:
                w = torch.relu(w - s["draft"][row].double().cpu())
            else:
                w[tokens[row + 1]] = 0.0
        total = torch.cumsum(w, 0)
        x = int(torch.searchsorted(total, us[i] * total[-1:], right=True))
        n_accepted.append(len(said))
        following.append(x)
        lengths.append(cached[i] + 1 + len(said))
        emitted += said + [x] + [-1] * (new[i] - len(said) - 1)
    return dict(n_accepted=_ints(n_accepted), next_token=_ints(following), emitted=_ints(emitted), lengths=_ints(lengths))
