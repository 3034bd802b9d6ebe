"""More of the library's calls for serving outside a fixed generation, with their inputs, their work and their plain forms.

Four kinds of pass:
  attend   attention over a paged cache whose scores are capped by a tanh or fall with the distance, or whose tokens see a window, a
           document or a prefix; and any attention over pages of 4 bits
  cache    keys and values of new tokens filed into pages of 4 bits, then read back
  assign   the next block table of a batch (rows forked, reordered and grown, written pages no longer shared) and the copies of pages it asks for
  compact  the pages in use moved to the lowest places, with the copies of pages

Pages are what include/skd.h documents (skd_kv).  4-bit pages hold e2m1 codes, and a power of two for every 32 neighbouring elements.
"""
import math

import torch

own = False

BF16, FP8, FP4 = "bf16", "fp8", "fp4"
CAUSAL, WINDOW, DOCUMENTS, PREFIX = "causal", "window", "documents", "prefix"


# ---------------------------------------------------------------------------------------------- cases
def _attend(elem, rows, heads, kv_heads, dh, page, new, past, files=False, cap=0.0, slopes=False, mask=CAUSAL, size=0, **name):
    """new, past: tokens of the longest row; the others have between half and all of it.  files: the call files the new tokens too;
    else the cache holds them already.  cap: of the scores (0: none).  slopes: they fall with the distance.  size: of the window, of a
    document on average, or of the prefix."""
    return dict(name, kind="attend", elem=elem, rows=rows, heads=heads, kv_heads=kv_heads, dh=dh, page=page, new=new, past=past, files=files,
                cap=cap, slopes=slopes, mask=mask, size=size)


def _cache(rows, heads, dh, page, new, past, whole=False, **name):
    """whole: the rows are read back from position 0 on, not only what was filed."""
    return dict(name, kind="cache", elem=FP4, rows=rows, kv_heads=heads, dh=dh, page=page, new=new, past=past, whole=whole)


def _assign(groups, beams, kv_heads, dh, page, past, more, **name):
    """groups of `beams` rows that share the whole pages of a prompt and have `past` positions at most; each goes on from some row of its
    group with up to `more` tokens."""
    return dict(name, kind="assign", elem=BF16, groups=groups, beams=beams, kv_heads=kv_heads, dh=dh, page=page, past=past, more=more)


def _compact(rows, kv_heads, dh, page, past, pages, **name):
    """rows of up to `past` positions, scattered over a pool of `pages` pages."""
    return dict(name, kind="compact", elem=BF16, rows=rows, kv_heads=kv_heads, dh=dh, page=page, past=past, pages=pages)


def listed():
    return [
        # the smallest step with a distance bias: two short rows of a narrow model, latency alone
        _attend(BF16, 2, 4, 4, 64, 64, 1, 31, True, slopes=True, name="slopes_bf16_b2_ctx31"),
        # a decode step of a model with capped scores and a sliding window, tokens filed by the same call
        _attend(BF16, 32, 32, 32, 128, 64, 1, 1535, True, cap=50.0, mask=WINDOW, size=512, name="cap_window_bf16_b32_ctx1536"),
        # one user at a long context with a distance bias, over 8-bit pages
        _attend(FP8, 1, 32, 8, 128, 64, 1, 32766, slopes=True, name="slopes_fp8_b1_ctx32k_group4"),
        # documents packed into prompts of an odd length
        _attend(BF16, 2, 32, 8, 128, 64, 2047, 0, mask=DOCUMENTS, size=500, name="documents_bf16_b2_prompt2047_group4"),
        # the second piece of prompts whose beginning sees itself in both directions, capped scores, 64-wide heads
        _attend(FP8, 8, 32, 32, 64, 64, 511, 1024, cap=30.0, mask=PREFIX, size=1300, name="cap_prefix_fp8_b8_chunk511"),
        # five drafted tokens a row to be verified at once, capped scores over 4 bits
        _attend(FP4, 16, 32, 8, 128, 64, 5, 1994, cap=50.0, name="cap_fp4_b16_draft5_group4"),
        # a decode step of a large ragged batch over 4 bits
        _attend(FP4, 128, 32, 32, 128, 64, 1, 1023, name="fp4_b128_ctx1024"),
        # the next turn of eight conversations over 4 bits
        _attend(FP4, 8, 32, 32, 128, 64, 512, 2048, name="fp4_b8_chunk512"),
        # one decode step's tokens of a large batch into 4-bit pages: hardly any bytes
        _cache(128, 32, 128, 64, 1, 640, name="cache_fp4_b128_step"),
        # chunks of an odd length behind earlier turns, rows handed on whole
        _cache(8, 32, 128, 64, 509, 1539, True, name="cache_fp4_b8_chunk509"),
        # a step of beam search: 32 prompts, four beams each
        _assign(32, 4, 32, 128, 64, 640, 1, name="assign_32x4_beams"),
        # a pool that is to shrink after many of its rows have ended
        _compact(64, 8, 128, 64, 1500, 2048, name="compact_2048_pages"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend", "cache", "assign", "compact"])
    dh = rng.choice([64, 128, 128])
    kv_heads, page = rng.choice([1, 2, 4, 8, 12, 32]), rng.choice([32, 64, 64, 96, 128, 256])
    page_bytes = kv_heads * page * 4 * dh
    if kind == "assign":
        beams, past = rng.choice([1, 2, 3, 4, 8]), _log(rng, 1, 4096)
        more = rng.choice([1, 1, _log(rng, 2, 64)])
        groups = _log(rng, 1, max(1, min(128 // beams, (544 << 20) // (page_bytes * (2 * beams + (past + more) // page + 1)))))
        return _assign(groups, beams, kv_heads, dh, page, past, more)
    if kind == "compact":
        pages = _log(rng, 2, max(2, min(8192, (512 << 20) // page_bytes)))
        rows = _log(rng, 1, min(128, pages))
        return _compact(rows, kv_heads, dh, page, _log(rng, 1, max(1, pages // rows * page)), pages)
    rows = _log(rng, 1, 128)
    room = 4 * 131072 // (rows * kv_heads)  # positions of a row: no cache is larger than the largest listed one
    if kind == "cache":
        new = min(rng.choice([1, _log(rng, 2, 64), _log(rng, 64, 2048)]), max(1, room // 4))
        return _cache(rows, kv_heads, dh, page, new, _log(rng, 1, max(1, min(4096, room // 2 - new))) - 1, rng.choice([False, True]))
    elem, group = rng.choice([BF16, FP8, FP4, FP4]), rng.choice([1, 1, 2, 3, 4, 8]) if kv_heads <= 8 else 1
    new = min(rng.choice([1, 1, _log(rng, 2, 32), _log(rng, 32, 2048)]), room // 2)
    past = _log(rng, 1, min(32768, room - new)) - 1
    heads = kv_heads * group
    while rows * heads * new * (new + past) > 32 * 8 * 512 * 2560:  # scores: no more than those of the largest listed case
        if new > 1 and new * 8 > past:
            new = (new + 1) // 2
        elif past > 1:
            past //= 2
        else:
            rows = max(1, rows // 2)
    cap, slopes, mask = rng.choice([0.0, 0.0, 20.0, 30.0, 50.0]), rng.choice([False, False, True]), rng.choice([CAUSAL, WINDOW, DOCUMENTS, PREFIX])
    if elem != FP4 and not cap and not slopes and mask == CAUSAL:
        cap = 50.0
    size = 0 if mask == CAUSAL else _log(rng, 1, new + past) if new + past > 1 else 1
    return _attend(elem, rows, heads, kv_heads, dh, page, new, past, new == 1 and elem == BF16 and rng.choice([False, True]), cap, slopes, mask, size)


# ---------------------------------------------------------------------------------------------- inputs
def _generator(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + part)
    return g


def _lengths(case):
    """(new, past) of each row, on the host; the first row has the longest of both."""
    g = torch.Generator().manual_seed(11)
    new = case["new"] - (torch.rand(case["rows"], generator=g) * (case["new"] // 2 + 1)).long().clamp_(max=case["new"] // 2)
    past = case["past"] - (torch.rand(case["rows"], generator=g) * (case["past"] // 2 + 1)).long().clamp_(max=case["past"] // 2)
    new[0], past[0] = case["new"], case["past"]
    return new, past


def _seen(case):
    """[tokens] each on the host: position of each new token, the first that it sees and the one behind the last."""
    new, past = _lengths(case)
    at = torch.cat([p + torch.arange(n) for n, p in zip(new.tolist(), past.tolist())])
    begin, end, size = torch.zeros_like(at), at + 1, case["size"]
    if case["mask"] == WINDOW:
        begin = (at - size + 1).clamp(min=0)
    if case["mask"] == PREFIX:
        longest = torch.repeat_interleave(torch.minimum(torch.tensor(size), new + past), new)
        end = torch.maximum(end, torch.where(at < longest, longest, 0))
    if case["mask"] == DOCUMENTS:
        g, parts = torch.Generator().manual_seed(13), []
        for n, p in zip(new.tolist(), past.tolist()):
            starts = torch.rand(n + p, generator=g) < 1.0 / size
            first = torch.where(starts, torch.arange(n + p), 0).cummax(0).values
            parts.append(first[p:])
        begin = torch.cat(parts)
    return at, begin, end


def _normal(g, *size):
    return torch.empty(*size, dtype=torch.float32, device="cuda").normal_(generator=g)


def _tokens(case, seed):
    """Keys and values [tokens][kv head][dh] of all rows, what is cached and what is new, one row behind the other, and whether
    each is new; a few channels of the keys are large, as in trained models."""
    new, past = _lengths(case)
    n = int((new + past).sum())
    g = _generator(seed, 1)
    gain = torch.where(_normal(g, case["kv_heads"], case["dh"]).abs() > 2.2, 4.0, 0.7)
    k = (_normal(g, n, case["kv_heads"], case["dh"]) * gain).bfloat16()
    v = _normal(g, n, case["kv_heads"], case["dh"]).bfloat16()
    row = torch.repeat_interleave(torch.arange(case["rows"]), new + past)
    pos = torch.arange(n) - (torch.cumsum(new + past, 0) - new - past)[row]
    return k, v, row.cuda(), pos.cuda(), (pos >= past[row]).cuda()


def _queries(case, seed, tokens):
    """Scores of capped models are large: some of them are where the tanh bends."""
    return (_normal(_generator(seed, 2), tokens, case["heads"], case["dh"]) * (4.0 if case["cap"] else 1.0)).bfloat16()


def _slopes(case):
    return torch.exp2(-8.0 * torch.arange(1, case["heads"] + 1, dtype=torch.float32) / case["heads"])


def _rows_of_table(case):
    """Host lists of an assign or compact case: positions of each row; for assign also the tokens to come, the row that each goes on
    from, and how many of its first pages a row shares with its group."""
    g = torch.Generator().manual_seed(17)
    if case["kind"] == "compact":
        n = case["rows"]
        length = (torch.rand(n, generator=g) * case["past"]).long() + 1
        return length.tolist(), None, None, None
    G, B = case["groups"], case["beams"]
    length = case["past"] - (torch.rand(G, generator=g) * (case["past"] // 2 + 1)).long().clamp_(max=case["past"] // 2)
    more = (torch.rand(G, generator=g) * case["more"]).long() + 1
    more[0] = case["more"]
    source = torch.arange(G)[:, None] * B + torch.randint(B, (G, B), generator=g)
    share = (length * 3 // 4) // case["page"]
    return [x.repeat_interleave(B).tolist() for x in (length, more)] + [source.flatten().tolist(), share.repeat_interleave(B).tolist()]


def _table(case, seed):
    """The block table of such a case and the number of pages of its pool; pages are dealt out in the order of the seed."""
    length, _, _, share = _rows_of_table(case)
    page, rows = case["page"], len(length)
    need = [-(-n // page) for n in length]
    if case["kind"] == "compact":
        pages = max(case["pages"], sum(need))
        width = max(need)
    else:
        width = -(-(case["past"] + case["more"]) // page)
        pages = sum(need) + rows * (-(-case["more"] // page) + 1)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed * 1009 + 5)).tolist()
    table = torch.full((rows, width), -1, dtype=torch.int32)
    for r in range(rows):
        first = r - r % case["beams"] if share else r
        for i in range(need[r]):
            table[r, i] = table[first, i] if share and r != first and i < share[r] else order.pop()
    return table, pages


# ---------------------------------------------------------------------------------------------- pages
def _parts(case, pool):
    """Views of the pool in which a token's place is an index: keys [page][block][half][key][head][..codes..], values
    [page][block][half][quarter][key][head][..codes..] and their exponents, indexed alike (8 bits: [page][block][k | v][position][head])."""
    H, dh, nb = case["kv_heads"], case["dh"], case["page"] // 32
    if case["elem"] == FP4:
        G = dh // 32
        b = pool.unflatten(1, (H, nb, 34 * dh))
        k = b[..., :16 * dh].unflatten(-1, (G // 2, 4, 16, 4 // G, G, 4)).permute(0, 2, 3, 6, 5, 1, 7, 4, 8)
        k = k.flatten(2, 3)  # one of the two is 1: [page][block][half][key][head][32 elements][8 of them][2 of these]
        v = b[..., 16 * dh:32 * dh].unflatten(-1, (G // 2, 4, 16, 2, 2, 4)).permute(0, 2, 7, 4, 8, 1, 3, 6, 5)
        ke = b[..., 32 * dh:33 * dh].unflatten(-1, (16, 2, G)).permute(0, 2, 4, 3, 1, 5)
        ve = b[..., 33 * dh:].unflatten(-1, (4, G, 2, 4)).permute(0, 2, 5, 3, 6, 1, 4)
        return k, v, (ke, ve)
    at = H * nb * 64 * dh
    k, v = pool[:, :at].unflatten(1, (H, nb, 2, 32 * dh)).unbind(3)
    if case["elem"] == BF16:
        k = k.unflatten(-1, (2, dh // 32, 4, 16, 8)).permute(0, 2, 3, 6, 1, 4, 5, 7)
        v = v.unflatten(-1, (dh // 16, 4, 16, 2, 4)).permute(0, 2, 6, 4, 7, 1, 3, 5)
        return k, v, None
    k = k.unflatten(-1, (2, dh // 64, 4, 16, 2, 8)).permute(0, 2, 3, 6, 1, 4, 7, 5, 8)
    v = v.unflatten(-1, (dh // 32, 4, 16, 2, 2, 4)).permute(0, 2, 7, 4, 8, 1, 3, 6, 5)
    return k, v, pool[:, at:].unflatten(1, (H, nb, 2, 32)).permute(0, 2, 3, 4, 1)


def _codes8(x):
    """e4m3 codes and exponent bytes of [..., dh]: the smallest power of two that leaves no value above 448."""
    m, e = torch.frexp(x.float().abs().amax(-1))
    e = torch.where(m == 0, -127, e - torch.where(m <= 0.875, 9, 8)).clamp_(min=-127)
    return torch.ldexp(x.float(), -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values8(codes, exponents):
    return torch.ldexp(codes.contiguous().view(torch.float8_e4m3fn).float(), exponents[..., None].int() - 127)


def _codes4(x):
    """e2m1 codes [..., dh / 32, 32] and exponent bytes [..., dh / 32]: the smallest power of two that leaves none of 32 values above 6."""
    x = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m == 0, -124, e - torch.where(m <= 0.75, 3, 2)).clamp_(min=-124)
    y = torch.ldexp(x, -e[..., None])
    a = y.abs()
    a = torch.where(a < 2, (2 * a).round(), torch.where(a < 4, a.round() + 2, (0.5 * a).round() + 4))  # (halves to even; 1.75 .. 2: code 4)
    a = torch.where(e[..., None] == 126, a.clamp(max=5), a)
    return a.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3), (e + 127).to(torch.uint8)


def _values4(codes, exponents):
    """Values [..., dh] of codes [..., dh / 32, 32]."""
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    value = torch.cat([value, -value])[codes.int()]
    return torch.ldexp(value, exponents[..., None].int() - 127).flatten(-2)


def _keys4(b):  # [..., dh / 32, 4, 4] bytes of neighbouring elements -> codes [..., dh / 32, 32]
    return torch.stack([b & 15, b >> 4], -1).flatten(-3)


def _vals4(b):  # [..., dh / 64, 2, 16] bytes of elements 16 apart
    return torch.cat([b & 15, b >> 4], -1).flatten(-3, -2)


def _file(case, pool, table, row, pos, k, v):
    """k, v [tokens][kv head][dh] into the pages, at position `pos` of row `row`."""
    K, V, E = _parts(case, pool)
    page, slot = table[row, pos // case["page"]].long(), pos % case["page"]
    block, half, key = slot // 32, slot // 16 % 2, slot % 16
    if case["elem"] == FP4:
        (k, ke), (v, ve) = _codes4(k), _codes4(v)
        E[0][page, block, half, key] = ke
        E[1][page, block, half, key // 4, key % 4] = ve
        k = k.unflatten(-1, (4, 4, 2))
        k = k[..., 0] | k[..., 1] << 4
        v = (v[..., :16] | v[..., 16:] << 4).unflatten(-2, (-1, 2))
    elif E is not None:
        (k, ke), (v, ve) = _codes8(k), _codes8(v)
        E[page, block, 0, slot % 32] = ke
        E[page, block, 1, slot % 32] = ve
    K[page, block, half, key] = k.reshape(k.shape[:2] + K.shape[5:])
    V[page, block, half, key // 4, key % 4] = v.reshape(v.shape[:2] + V.shape[6:])


def _read(case, pool, table, row, pos):
    """fp32 keys and values [tokens][kv head][dh] of 4-bit pages at position `pos` of row `row`."""
    K, V, E = _parts(case, pool)
    page, slot = table[row, pos // case["page"]].long(), pos % case["page"]
    block, half, key = slot // 32, slot // 16 % 2, slot % 16
    k = _values4(_keys4(K[page, block, half, key]), E[0][page, block, half, key])
    return k, _values4(_vals4(V[page, block, half, key // 4, key % 4]), E[1][page, block, half, key // 4, key % 4])


def _read_pages(case, pool, table):
    """fp32 keys and values [row][kv head][position][dh] of whole rows."""
    K, V, E = _parts(case, pool)
    pages = table.clamp(min=0).long()
    if case["elem"] == FP4:
        k = _values4(_keys4(K[pages]), E[0][pages]).flatten(1, 4)
        v = _values4(_vals4(V[pages]), E[1][pages]).flatten(1, 5)
        return k.transpose(1, 2), v.transpose(1, 2)
    k, v = K[pages].flatten(6).flatten(1, 4), V[pages].flatten(7).flatten(1, 5)
    if E is None:
        k, v = k.float(), v.float()
    else:
        e = E[pages]
        k, v = _values8(k, e[:, :, :, 0].flatten(1, 3)), _values8(v, e[:, :, :, 1].flatten(1, 3))
    return k.transpose(1, 2), v.transpose(1, 2)


# ---------------------------------------------------------------------------------------------- the passes
def prepare(case, seed):
    """The cache as earlier calls left it (pool, block table, lengths), what the pass is given, and the buffers for its results."""
    page, H, dh = case["page"], case["kv_heads"], case["dh"]
    if case["kind"] in ("assign", "compact"):
        length, more, source, _ = _rows_of_table(case)
        table, pages = _table(case, seed)
        ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        st = {"case": case, "table": table.cuda(), "len": ints(length), "more": ints(more), "source": ints(source),
              "pool": torch.empty(pages, H * page * 2 * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=_generator(seed, 4)),
              "table_out": torch.zeros_like(table, device="cuda"), "counts": torch.zeros(3, dtype=torch.int32, device="cuda"),
              "copies": torch.zeros(len(length) if more else pages // 2, 2, dtype=torch.int32, device="cuda")}
        torch.cuda.synchronize()
        return st
    new, past = _lengths(case)
    k, v, row, pos, fresh = _tokens(case, seed)
    need = (new + past + page - 1) // page
    order = torch.randperm(int(need.sum()), generator=torch.Generator().manual_seed(seed * 1009 + 5))
    table = torch.full((case["rows"], int(need.max())), -1, dtype=torch.int32)
    table[torch.arange(table.shape[1])[None] < need[:, None]] = order.int()
    size = H * page * 2 * dh if case["elem"] == BF16 else H * page * (2 * dh + 2) if case["elem"] == FP8 else H * page // 32 * 34 * dh
    pool = torch.zeros(len(order), size, dtype=torch.bfloat16 if case["elem"] == BF16 else torch.uint8, device="cuda")
    table = table.cuda()
    files = case["kind"] == "cache" or case["files"]
    held = ~fresh if files else torch.ones_like(fresh)
    _file(case, pool, table, row[held], pos[held], k[held], v[held])
    zero = torch.zeros(1, dtype=torch.int64)
    st = {"case": case, "pool": pool, "table": table, "tokens": int(new.sum()), "new": int(new.max()), "longest": int(past.max()),
          "first": torch.cat([zero, torch.cumsum(new, 0)]).int().cuda(), "past": past.int().cuda()}
    if files:
        st["k"], st["v"] = k[fresh].contiguous(), v[fresh].contiguous()
    if case["kind"] == "cache":
        whole = case["whole"]
        st["read_first"] = torch.cat([zero, torch.cumsum(new + past, 0)]).int().cuda() if whole else st["first"]
        st["read_past"] = torch.zeros_like(st["past"]) if whole else st["past"]
        st["read"], st["read_new"] = (int((new + past).sum()), int((new + past).max())) if whole else (st["tokens"], st["new"])
        st["k_out"], st["v_out"] = (torch.zeros(st["read"], H, dh, device="cuda") for _ in range(2))
    else:
        _, begin, end = _seen(case)
        st["begin"], st["end"], st["slopes"] = begin.int().cuda(), end.int().cuda(), _slopes(case).cuda()
        st["q"] = _queries(case, seed, st["tokens"])
        st["out"] = torch.zeros_like(st["q"])
    torch.cuda.synchronize()
    return st


def _places(first, past, tokens):
    """Row and position of each token of a call."""
    n = torch.arange(tokens, device="cuda")
    row = torch.searchsorted(first, n, right=True) - 1
    return row, n - first[row] + past[row]


def run(st):
    case = st["case"]
    if own:
        return _own(st)
    if case["kind"] in ("assign", "compact"):
        table, copies, counts = (_plain_assign if case["kind"] == "assign" else _plain_compact)(st)
        named = copies[copies[:, 0] >= 0].long()
        st["pool"][named[:, 1]] = st["pool"][named[:, 0]]
        return {"table": table, "copies": copies, "counts": counts, "pool": st["pool"]}
    if case["kind"] == "cache":
        _file(case, st["pool"], st["table"], *_places(st["first"], st["past"], st["tokens"]), st["k"], st["v"])
        k, v = _read(case, st["pool"], st["table"], *_places(st["read_first"], st["read_past"], st["read"]))
        return {"k": k, "v": v}
    if case["files"]:
        _file(case, st["pool"], st["table"], *_places(st["first"], st["past"], st["tokens"]), st["k"], st["v"])
        return {"out": _plain_attend(st), "pool": st["pool"]}
    return {"out": _plain_attend(st)}


def _plain_attend(st):
    case, H, dh = st["case"], st["case"]["kv_heads"], st["case"]["dh"]
    k, v = _read_pages(case, st["pool"], st["table"])
    row, pos = _places(st["first"], st["past"], st["tokens"])
    place = torch.arange(st["tokens"], device="cuda") - st["first"][row]
    q = torch.zeros(case["rows"], st["new"], case["heads"], dh, device="cuda")
    q[row, place] = st["q"].float()
    q = q.unflatten(2, (H, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [row][kv head][query head of the group, token][dh]
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(dh)).unflatten(2, (-1, st["new"]))
    if case["cap"]:
        s.div_(case["cap"]).tanh_().mul_(case["cap"])
    j = torch.arange(k.shape[2], device="cuda")
    if case["slopes"]:
        away = (st["past"][:, None, None] + torch.arange(st["new"], device="cuda")[:, None] - j).abs().float()
        s.sub_(st["slopes"].view(1, H, -1, 1, 1) * away[:, None, None])
    seen = torch.zeros(case["rows"], st["new"], k.shape[2], dtype=torch.bool, device="cuda")
    seen[row, place] = (j >= st["begin"][:, None]) & (j < st["end"][:, None])
    s.masked_fill_(~seen[:, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    s = s.div_(s.sum(-1, keepdim=True).clamp(min=1e-38)).flatten(2, 3)
    o = torch.matmul(s, v).unflatten(2, (-1, st["new"])).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return o[row, place].bfloat16()


def _plain_assign(st):
    table, pages, page = st["table"], st["pool"].shape[0], st["case"]["page"]
    rows, width = table.shape
    i, length, upto = torch.arange(width, device="cuda"), st["len"][:, None], (st["len"] + st["more"])[:, None]
    keep = torch.where(i * page < upto, table[st["source"].long()], -1)
    named = keep >= 0
    write = (i * page < upto) & (i * page + page > length) & (upto > length)
    bucket = torch.where(named, keep, pages).long().flatten()
    uses = torch.zeros(pages + 1, dtype=torch.int64, device="cuda").index_add_(0, bucket, torch.ones_like(bucket))
    written = torch.zeros_like(uses).index_add_(0, bucket, write.flatten().long())
    entry = torch.arange(rows * width, device="cuda")
    lowest = torch.full_like(uses, rows * width).scatter_reduce_(0, bucket, torch.where(write.flatten(), entry, rows * width), "amin")
    alone = (uses[bucket] == 1) | ((uses == written)[bucket] & (lowest[bucket] == entry))
    fresh = write & ~(named & alone.view(rows, width))
    free = torch.nonzero(uses[:pages] == 0).flatten()
    enough = fresh.sum() <= len(free)
    fresh &= enough
    out, at = keep.clone(), torch.cumsum(fresh.flatten(), 0).view(rows, width)
    got = free[(at - 1).clamp(0, max(len(free) - 1, 0))].int() if len(free) else torch.zeros_like(out)
    out = torch.where(fresh, got, torch.where(enough | (i * page < length), keep, -1))
    moved = fresh & named & (i * page < length)
    copies = torch.full_like(st["copies"], -1)
    pairs = torch.stack([keep[moved], out[moved]], -1)
    copies[:len(pairs)] = pairs
    distinct = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
    distinct[torch.where(out >= 0, out, pages).long().flatten()] = 1
    counts = torch.stack([distinct[:pages].sum(), (write & ~(named & alone.view(rows, width))).sum().sub(len(free)).clamp(min=0), moved.sum()]).int()
    return out, copies, counts


def _plain_compact(st):
    table, pages = st["table"], st["pool"].shape[0]
    used = torch.zeros(pages + 1, dtype=torch.bool, device="cuda")
    used[torch.where(table >= 0, table, pages).long().flatten()] = True
    used = used[:pages]
    number, n = torch.arange(pages, device="cuda"), used.sum()
    source, target = torch.nonzero(used & (number >= n)).flatten(), torch.nonzero(~used & (number < n)).flatten()
    place = torch.cat([number, number.new_full((1,), -1)])
    place[source] = target
    copies = torch.full_like(st["copies"], -1)
    copies[:len(source)] = torch.stack([source, target], -1).int()
    counts = torch.stack([n, torch.zeros_like(n), n.new_tensor(len(source))]).int()
    return place[torch.where(table >= 0, table, pages).long()].int(), copies, counts


def _own(st):
    from paper_2307_02628_amd import skd

    case = st["case"]
    if "cache" not in st:  # the handles that such a program keeps
        elem = {BF16: skd.KV_BF16, FP8: skd.KV_FP8, FP4: skd.KV_FP4}[case["elem"]]
        st["cache"] = cache = skd.KvCache(st["pool"], st["table"], case["kv_heads"], case["dh"], case["page"], elem)
        scores = None
        if case["kind"] == "assign":
            need = cache.assign_workspace()
        elif case["kind"] == "compact":
            need = cache.compact_workspace()
        else:
            st["chunk"] = skd.KvChunk(st["first"], st["past"], st["tokens"], st["new"], st["longest"])
            if case["kind"] == "cache":
                st["read_chunk"] = skd.KvChunk(st["read_first"], st["read_past"], st["read"], st["read_new"], st["longest"])
                need = 0
            elif case["cap"] or case["slopes"] or case["mask"] != CAUSAL:
                scores = skd.KvScores(case["cap"], st["slopes"] if case["slopes"] else None, case["size"] if case["mask"] == WINDOW else 0,
                                      st["begin"] if case["mask"] == DOCUMENTS else None, st["end"] if case["mask"] == PREFIX else None)
                need = cache.attend_scores_workspace(st["chunk"], case["heads"], scores)
            else:
                need = cache.attend_workspace(st["chunk"], case["heads"])
        st["scores"], st["workspace"] = scores, torch.empty(need, dtype=torch.uint8, device="cuda")
    cache = st["cache"]
    if case["kind"] in ("assign", "compact"):
        if case["kind"] == "assign":
            cache.assign(st["table_out"], st["copies"], st["counts"], st["len"], st["more"], st["source"], workspace=st["workspace"])
        else:
            cache.compact(st["table_out"], st["copies"], st["counts"], workspace=st["workspace"])
        cache.copy_pages(st["copies"], st["counts"][2:])
        return {"table": st["table_out"], "copies": st["copies"], "counts": st["counts"], "pool": st["pool"]}
    if case["kind"] == "cache":
        cache.append(st["chunk"], st["k"], st["v"])
        cache.read(st["read_chunk"], st["k_out"], st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    args = (st["chunk"], st["q"], st["out"], 1.0 / math.sqrt(case["dh"]))
    if st["scores"] is None:
        cache.attend(*args, st.get("k"), st.get("v"), workspace=st["workspace"])
    else:
        cache.attend_scores(*args, st["scores"], st.get("k"), st.get("v"), workspace=st["workspace"])
    return {"out": st["out"], "pool": st["pool"]} if case["files"] else {"out": st["out"]}


# ---------------------------------------------------------------------------------------------- work, reference
def work(case):
    H, dh = case["kv_heads"], case["dh"]
    if case["kind"] in ("assign", "compact"):
        table, pages = _table(case, 0)
        moved = len(_expected(case, table.tolist(), pages)[1])
        return {"bytes": 2 * moved * H * case["page"] * 4 * dh + 8 * table.numel() + 8 * moved, "flops": 0}
    new, past = (x.double() for x in _lengths(case))
    held = 4 * dh if case["elem"] == BF16 else 2 * dh + 2 if case["elem"] == FP8 else 17 * dh / 16  # bytes of one position and head, keys and values
    n, every = float(new.sum()), float((new + past).sum())
    if case["kind"] == "cache":
        read = every if case["whole"] else n
        return {"bytes": H * (n * (4 * dh + held) + read * (held + 8 * dh)), "flops": H * (n + read) * 4 * dh}
    _, begin, end = _seen(case)
    at, wanted = 0, 0  # positions that some token of a row sees
    for m in new.long().tolist():
        marks = torch.zeros(int(end[at:at + m].max()) + 1, dtype=torch.long)
        marks.index_add_(0, begin[at:at + m], torch.ones(m, dtype=torch.long)).index_add_(0, end[at:at + m], -torch.ones(m, dtype=torch.long))
        wanted += int((marks.cumsum(0) > 0).sum())
        at += m
    size = H * (wanted * held + (n * held if case["files"] else 0)) + 4 * dh * n * (case["heads"] + (H if case["files"] else 0))
    each = 4 * dh + (2 if case["slopes"] else 0) + (3 if case["cap"] else 0)
    return {"bytes": size, "flops": each * case["heads"] * float((end - begin).sum())}


def _rounded(x, bits):
    """What pages of 8 or 4 bits hold of [..., dh], in 64 bits: multiples of a power of two for the vector or for 32 of it."""
    x = x.double()
    top, digits, low, shape = (448.0, 3, -6, x.shape) if bits == 8 else (6.0, 1, 0, x.shape[:-1] + (-1, 32))
    x, whole = x.reshape(shape), x.shape
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a / top))
    e = torch.where(a > top * torch.exp2(e), e + 1, torch.where(a <= top / 2 * torch.exp2(e), e - 1, e))
    y = torch.where(a > 0, x / torch.exp2(e), 0.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** low))) - digits)
    return torch.where(a > 0, torch.round(y / step) * step * torch.exp2(e), 0.0).reshape(whole)


def _expected(case, table, pages):
    """The next table and the copies, entry by entry on the host."""
    length, more, source, _ = _rows_of_table(case)
    page = case["page"]
    if case["kind"] == "compact":
        used = sorted({p for row in table for p in row if p >= 0})
        free = sorted(set(range(len(used))) - set(used))
        copies = list(zip([p for p in used if p >= len(used)], free))
        place = dict(copies)
        return [[place.get(p, p) for p in row] for row in table], copies, [len(used), 0, len(copies)]
    rows = [[p if i * page < length[r] + more[r] else -1 for i, p in enumerate(table[source[r]])] for r in range(len(table))]
    holders, writers = {}, {}
    for r, row in enumerate(rows):
        for i, p in enumerate(row):
            if p >= 0:
                holders.setdefault(p, []).append((r, i))
                if (i + 1) * page > length[r] and i * page < length[r] + more[r]:
                    writers.setdefault(p, []).append((r, i))
    free = iter(p for p in range(pages) if p not in holders)
    copies = []
    for r, row in enumerate(rows):
        for i in range(length[r] // page, -(-(length[r] + more[r]) // page)):
            p = row[i]
            if p >= 0 and (len(holders[p]) == 1 or (holders[p] == writers[p] and writers[p][0] == (r, i))):
                continue
            row[i] = next(free)
            if p >= 0 and i * page < length[r]:
                copies.append((p, row[i]))
    return rows, copies, [len({p for row in rows for p in row if p >= 0}), 0, len(copies)]


def exact(case, seed):
    if case["kind"] in ("assign", "compact"):
        before = prepare(case, seed)
        rows, copies, counts = _expected(case, before["table"].tolist(), before["pool"].shape[0])
        pool, listed_copies = before["pool"].double(), torch.full_like(before["copies"], -1)
        for n, (a, b) in enumerate(copies):
            pool[b], listed_copies[n] = before["pool"][a].double(), torch.tensor([a, b])
        return {"table": torch.tensor(rows, dtype=torch.int32), "copies": listed_copies, "counts": torch.tensor(counts, dtype=torch.int32), "pool": pool}
    new, past = _lengths(case)
    k, v, row, pos, fresh = _tokens(case, seed)
    if case["elem"] == BF16:
        k, v = k.double(), v.double()
    else:
        k, v = (_rounded(x, 8 if case["elem"] == FP8 else 4) for x in (k, v))
    if case["kind"] == "cache":
        return {"k": k, "v": v} if case["whole"] else {"k": k[fresh], "v": v[fresh]}
    tokens, group = int(new.sum()), case["heads"] // case["kv_heads"]
    where, begin, end = (x.cuda() for x in _seen(case))
    slopes = _slopes(case).double().tolist()
    q, out = _queries(case, seed, tokens).double(), torch.zeros(tokens, case["heads"], case["dh"], dtype=torch.float64, device="cuda")
    at = first = 0
    for n, p in zip(new.tolist(), past.tolist()):
        j, me = torch.arange(n + p, device="cuda")[None], slice(at, at + n)
        hidden = (j < begin[me, None]) | (j >= end[me, None])
        for h in range(case["heads"]):
            kh, vh = k[first:first + n + p, h // group], v[first:first + n + p, h // group]
            s = q[me, h] @ kh.t() / math.sqrt(case["dh"])
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            if case["slopes"]:
                s = s - slopes[h] * (where[me, None] - j).abs()
            out[me, h] = s.masked_fill(hidden, -math.inf).softmax(-1) @ vh
        at, first = at + n, first + n + p
    if not case["files"]:
        return {"out": out}
    return {"out": out, "pool": prepare(dict(case, files=False), seed)["pool"].double()}
