"""The library's calls for serving outside a fixed generation, with their inputs, their work and their plain forms.

Three kinds of pass:
  cache   keys and values of new tokens filed into the pages of a cache (bf16 or 8 bits), then read back
  attend  attention of new tokens over a paged cache: one token a row, a few, or a chunk of a prompt
  sample  one token a row drawn from logits with the row's own temperature, top-k, top-p and min-p

Pages are what include/skd.h documents (skd_kv): per kv head and block of 32 positions, keys and values in the order in which the
matrix instructions take them; 8-bit pages hold e4m3 codes and, behind them, one power of two for each token and head.
"""
import math

import torch

own = False

BF16, FP8 = "bf16", "fp8"
TEMPERATURE, TOP_P = 0.3, 0.7  # the sampling setting that the repository's benchmark uses


# ---------------------------------------------------------------------------------------------- cases
def _cache(elem, rows, heads, dh, page, new, past, whole=False, **name):
    """new, past: tokens of the longest row; the others have between half and all of it.  whole: the rows are read back from
    position 0 on, not only what was filed."""
    return dict(name, kind="cache", elem=elem, rows=rows, kv_heads=heads, dh=dh, page=page, new=new, past=past, whole=whole)


def _attend(elem, rows, heads, kv_heads, dh, page, new, past, files=False, **name):
    """files: the call files the new tokens too, as a decode step does; else the cache holds them already."""
    return dict(name, kind="attend", elem=elem, rows=rows, heads=heads, kv_heads=kv_heads, dh=dh, page=page, new=new, past=past, files=files)


def _sample(rows, vocab, spread, top_k, top_p, min_p, **name):
    """spread: standard deviation of the logits; top_k, top_p, min_p: the loosest of the rows (0, 1, 0: off)."""
    return dict(name, kind="sample", rows=rows, vocab=vocab, spread=spread, top_k=top_k, top_p=top_p, min_p=min_p)


def listed():
    return [
        # one decode step's tokens of a large batch into 8-bit pages: a launch or two, hardly any bytes
        _cache(FP8, 128, 32, 128, 64, 1, 640, name="cache_fp8_b128_step"),
        # chunks of an odd length behind earlier turns, rows handed on whole
        _cache(FP8, 8, 32, 128, 64, 509, 1539, True, name="cache_fp8_b8_chunk509"),
        # prompts of 64-wide heads in bf16 pages
        _cache(BF16, 3, 32, 64, 64, 301, 0, name="cache_bf16_b3_prompt301"),
        # the smallest step: two short rows of a narrow model, latency alone
        _attend(BF16, 2, 4, 4, 64, 64, 1, 31, True, name="attend_bf16_b2_ctx31"),
        # a decode step of the benchmark's batch, tokens filed by the same call
        _attend(BF16, 32, 32, 32, 128, 64, 1, 639, True, name="attend_bf16_b32_ctx640"),
        # the large ragged batch over 8-bit pages
        _attend(FP8, 128, 32, 32, 128, 64, 1, 1023, name="attend_fp8_b128_ctx1024"),
        # one user at a long context, four query heads to a kv head
        _attend(FP8, 1, 32, 8, 128, 64, 1, 32766, name="attend_fp8_b1_ctx32k_group4"),
        # five drafted tokens a row to be verified at once
        _attend(BF16, 16, 32, 8, 128, 64, 5, 1994, name="attend_bf16_b16_draft5"),
        # the next turn of eight conversations
        _attend(BF16, 8, 32, 32, 128, 64, 512, 2048, name="attend_bf16_b8_chunk512"),
        # a piece of a long prompt over 8-bit pages, odd lengths, grouped heads
        _attend(FP8, 2, 32, 8, 128, 128, 1023, 8193, name="attend_fp8_b2_chunk1023_group4"),
        # one request with the repository's own sampling setting
        _sample(1, 50272, 1.5, 0, TOP_P, 0.0, name="sample_b1_50272"),
        # a large batch of requests that all ask for something else, over a large vocabulary
        _sample(128, 131072, 2.5, 1000, 0.95, 0.05, name="sample_b128_131072"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["cache", "attend", "attend", "attend", "sample"])
    if kind == "sample":
        return _sample(_log(rng, 1, 128), _log(rng, 1000, 131072), rng.choice([0.5, 1.5, 2.5, 4.0]), rng.choice([0, 1, _log(rng, 2, 2000)]),
                       rng.choice([1.0, 0.7, 0.9, 0.95, 0.99]), rng.choice([0.0, 0.01, 0.05, 0.1]))
    elem, dh = rng.choice([BF16, FP8]), rng.choice([64, 128, 128])
    kv_heads, page = rng.choice([1, 2, 4, 8, 12, 32]), rng.choice([32, 64, 64, 96, 128, 256])
    rows = _log(rng, 1, 128)
    room = 4 * 131072 // (rows * kv_heads)  # positions of a row: no cache is larger than the largest listed one
    if kind == "cache":
        new = min(rng.choice([1, _log(rng, 2, 64), _log(rng, 64, 2048)]), max(1, room // 4))
        return _cache(elem, rows, kv_heads, dh, page, new, _log(rng, 1, max(1, min(4096, room // 2 - new))) - 1, rng.choice([False, True]))
    group = rng.choice([1, 1, 2, 3, 4, 8]) if kv_heads <= 8 else 1
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
    return _attend(elem, rows, heads, kv_heads, dh, page, new, past, new == 1 and elem == BF16 and rng.choice([False, True]))


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
    return _normal(_generator(seed, 2), tokens, case["heads"], case["dh"]).bfloat16()


def _logits(case, seed):
    """Logits, and the parameters of each row: temperature 0.3 to 1.2, top-k, top-p and min-p between off and the case's."""
    g, B = _generator(seed, 3), case["rows"]
    z = _normal(g, B, case["vocab"]) * case["spread"]
    z[::3] = z[::3].bfloat16().float()  # logits that were rounded: many of them are equal
    r = torch.rand(4, B, generator=g, device="cuda")
    on = torch.rand(3, B, generator=g, device="cuda") < 0.75
    on[:, 0] = True
    t = TEMPERATURE + 0.9 * r[0]
    t[0] = TEMPERATURE
    k = torch.where(on[0], (case["top_k"] * (0.25 + 0.75 * r[1])).round().int(), 0).int()
    p = torch.where(on[1], 1 - (1 - case["top_p"]) * (0.25 + 0.75 * r[2]), 1.0)
    p[0] = case["top_p"]
    m = torch.where(on[2], case["min_p"] * r[3], 0.0)
    u = torch.rand(B, generator=g, device="cuda").clamp_(max=0.999999)
    return z, t, k, p.float(), m.float(), u


# ---------------------------------------------------------------------------------------------- pages
def _parts(case, pool):
    """Views of the pool in which a token's place is an index: keys [page][block][half][key][head][..dh..], values
    [page][block][half][quarter][key][head][..dh..] and, for 8 bits, exponents [page][block][k | v][position][head]."""
    H, dh, nb = case["kv_heads"], case["dh"], case["page"] // 32
    at = H * nb * 64 * dh
    k, v = pool[:, :at].unflatten(1, (H, nb, 2, 32 * dh)).unbind(3)
    if case["elem"] == BF16:
        k = k.unflatten(-1, (2, dh // 32, 4, 16, 8)).permute(0, 2, 3, 6, 1, 4, 5, 7)
        v = v.unflatten(-1, (dh // 16, 4, 16, 2, 4)).permute(0, 2, 6, 4, 7, 1, 3, 5)
        return k, v, None
    k = k.unflatten(-1, (2, dh // 64, 4, 16, 2, 8)).permute(0, 2, 3, 6, 1, 4, 7, 5, 8)
    v = v.unflatten(-1, (dh // 32, 4, 16, 2, 2, 4)).permute(0, 2, 7, 4, 8, 1, 3, 6, 5)
    return k, v, pool[:, at:].unflatten(1, (H, nb, 2, 32)).permute(0, 2, 3, 4, 1)


def _codes(x):
    """e4m3 codes and exponent bytes of [..., dh]: the smallest power of two that leaves no value above 448."""
    m, e = torch.frexp(x.float().abs().amax(-1))
    e = torch.where(m == 0, -127, e - torch.where(m <= 0.875, 9, 8)).clamp_(min=-127)
    return torch.ldexp(x.float(), -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, exponents):
    return torch.ldexp(codes.contiguous().view(torch.float8_e4m3fn).float(), exponents[..., None].int() - 127)


def _file(case, pool, table, row, pos, k, v):
    """k, v [tokens][kv head][dh] into the pages, at position `pos` of row `row`."""
    K, V, E = _parts(case, pool)
    page, slot = table[row, pos // case["page"]].long(), pos % case["page"]
    block, half, key = slot // 32, slot // 16 % 2, slot % 16
    if E is not None:
        (k, ke), (v, ve) = _codes(k), _codes(v)
        E[page, block, 0, slot % 32] = ke
        E[page, block, 1, slot % 32] = ve
    K[page, block, half, key] = k.unflatten(-1, K.shape[5:])
    V[page, block, half, key // 4, key % 4] = v.unflatten(-1, V.shape[6:])


def _read(case, pool, table, row, pos):
    """fp32 keys and values [tokens][kv head][dh] at position `pos` of row `row`."""
    K, V, E = _parts(case, pool)
    page, slot = table[row, pos // case["page"]].long(), pos % case["page"]
    block, half, key = slot // 32, slot // 16 % 2, slot % 16
    k, v = K[page, block, half, key].flatten(2), V[page, block, half, key // 4, key % 4].flatten(2)
    if E is None:
        return k.float(), v.float()
    return _values(k, E[page, block, 0, slot % 32]), _values(v, E[page, block, 1, slot % 32])


def _read_pages(case, pool, table):
    """fp32 keys and values [row][kv head][position][dh] of whole rows."""
    K, V, E = _parts(case, pool)
    pages = table.clamp(min=0).long()
    k, v = K[pages].flatten(6).flatten(1, 4), V[pages].flatten(7).flatten(1, 5)
    if E is None:
        k, v = k.float(), v.float()
    else:
        e = E[pages]
        k, v = _values(k, e[:, :, :, 0].flatten(1, 3)), _values(v, e[:, :, :, 1].flatten(1, 3))
    return k.transpose(1, 2), v.transpose(1, 2)


# ---------------------------------------------------------------------------------------------- the passes
def prepare(case, seed):
    """The cache as earlier calls left it (pool, block table, lengths), what the pass is given, and the buffers for its results."""
    if case["kind"] == "sample":
        z, t, k, p, m, u = _logits(case, seed)
        return {"case": case, "logits": z, "temperature": t, "top_k": k, "top_p": p, "min_p": m, "u": u,
                "out": torch.zeros(case["rows"], dtype=torch.int32, device="cuda")}
    new, past = _lengths(case)
    k, v, row, pos, fresh = _tokens(case, seed)
    page, H, dh = case["page"], case["kv_heads"], case["dh"]
    need = (new + past + page - 1) // page
    order = torch.randperm(int(need.sum()), generator=torch.Generator().manual_seed(seed * 1009 + 5))
    table = torch.full((case["rows"], int(need.max())), -1, dtype=torch.int32)
    table[torch.arange(table.shape[1])[None] < need[:, None]] = order.int()
    size = H * page * 2 * dh if case["elem"] == BF16 else H * page * (2 * dh + 2)
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
    if case["kind"] == "sample":
        return {"tokens": _plain_sample(st)}
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
    last = st["past"][:, None] + torch.arange(st["new"], device="cuda")
    s.masked_fill_((torch.arange(k.shape[2], device="cuda") > last[..., None])[:, None, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    s = s.div_(s.sum(-1, keepdim=True)).flatten(2, 3)
    o = torch.matmul(s, v).unflatten(2, (-1, st["new"])).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return o[row, place].bfloat16()


def _plain_sample(st):
    z, top_k, top_p, V = st["logits"], st["top_k"][:, None].long(), st["top_p"][:, None].double(), st["case"]["vocab"]
    by_size = torch.sort(z, dim=-1, descending=True).values
    highest, t = by_size[:, :1].double(), st["temperature"][:, None].double()
    kth = torch.where(top_k > 0, by_size.gather(1, top_k.clamp(1, V) - 1), -math.inf)
    mass = torch.exp((z.double() - highest) / t)
    keep = (z >= kth) & (mass >= st["min_p"][:, None].double())
    ordered = torch.exp((by_size.double() - highest) / t)
    ordered = torch.where((by_size >= kth) & (ordered >= st["min_p"][:, None].double()), ordered, 0.0).cumsum(-1)
    enough = (ordered < top_p * ordered[:, -1:]).sum(-1, keepdim=True).clamp(max=V - 1)
    keep &= (z >= by_size.gather(1, enough)) | (top_p >= 1)
    mass = torch.where(keep, mass, 0.0).cumsum(-1)
    return (mass <= st["u"][:, None].double() * mass[:, -1:]).sum(-1).int()


def _own(st):
    from paper_2307_02628_amd import skd

    case = st["case"]
    if case["kind"] == "sample":
        if "workspace" not in st:
            st["workspace"] = torch.empty(skd.sample_workspace(case["rows"], case["vocab"]), dtype=torch.uint8, device="cuda")
        skd.sample(st["logits"], st["u"], st["out"], st["temperature"], st["top_k"], st["top_p"], st["min_p"], st["workspace"])
        return {"tokens": st["out"]}
    if "cache" not in st:  # the handles that such a program keeps
        st["cache"] = skd.KvCache(st["pool"], st["table"], case["kv_heads"], case["dh"], case["page"],
                                  skd.KV_BF16 if case["elem"] == BF16 else skd.KV_FP8)
        st["chunk"] = skd.KvChunk(st["first"], st["past"], st["tokens"], st["new"], st["longest"])
        if case["kind"] == "cache":
            st["read_chunk"] = skd.KvChunk(st["read_first"], st["read_past"], st["read"], st["read_new"], st["longest"])
        else:
            st["workspace"] = torch.empty(st["cache"].attend_workspace(st["chunk"], case["heads"]), dtype=torch.uint8, device="cuda")
    if case["kind"] == "cache":
        st["cache"].append(st["chunk"], st["k"], st["v"])
        st["cache"].read(st["read_chunk"], st["k_out"], st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    st["cache"].attend(st["chunk"], st["q"], st["out"], 1.0 / math.sqrt(case["dh"]), st.get("k"), st.get("v"), workspace=st["workspace"])
    return {"out": st["out"], "pool": st["pool"]} if case["files"] else {"out": st["out"]}


# ---------------------------------------------------------------------------------------------- work, reference
def work(case):
    B = case["rows"]
    if case["kind"] == "sample":  # a subtraction, a product, an exponential, two comparisons and two sums a value
        return {"bytes": 4 * B * case["vocab"] + 24 * B, "flops": 7 * B * case["vocab"]}
    new, past = (x.double() for x in _lengths(case))
    H, dh = case["kv_heads"], case["dh"]
    held = 4 * dh if case["elem"] == BF16 else 2 * dh + 2  # bytes of one position and head, keys and values
    n, every = float(new.sum()), float((new + past).sum())
    if case["kind"] == "cache":
        read = every if case["whole"] else n
        return {"bytes": H * (n * (4 * dh + held) + read * (held + 8 * dh)), "flops": H * (n + read) * 4 * dh}
    size = H * every * held + 4 * dh * n * (case["heads"] + (H if case["files"] else 0))
    return {"bytes": size, "flops": 4 * dh * case["heads"] * float((new * (past + (new + 1) / 2)).sum())}


def _rounded(x):
    """The e4m3 values times their power of two that stand for [..., dh], in 64 bits."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a / 448.0))
    e = torch.where(a > 448.0 * torch.exp2(e), e + 1, torch.where(a <= 224.0 * torch.exp2(e), e - 1, e))
    y = torch.where(a > 0, x / torch.exp2(e), 0.0)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(a > 0, torch.round(y / step) * step * torch.exp2(e), 0.0)


def exact(case, seed):
    if case["kind"] == "sample":
        return _exact_sample(case, seed)
    new, past = _lengths(case)
    k, v, row, pos, fresh = _tokens(case, seed)
    if case["elem"] == FP8:
        k, v = _rounded(k), _rounded(v)
    else:
        k, v = k.double(), v.double()
    if case["kind"] == "cache":
        return {"k": k, "v": v} if case["whole"] else {"k": k[fresh], "v": v[fresh]}
    tokens, group = int(new.sum()), case["heads"] // case["kv_heads"]
    q, out = _queries(case, seed, tokens).double(), torch.zeros(tokens, case["heads"], case["dh"], dtype=torch.float64, device="cuda")
    at = seen = 0
    for n, p in zip(new.tolist(), past.tolist()):
        ahead = torch.arange(n + p, device="cuda")[None] > p + torch.arange(n, device="cuda")[:, None]
        for h in range(case["heads"]):
            kh, vh = k[seen:seen + n + p, h // group], v[seen:seen + n + p, h // group]
            w = (q[at:at + n, h] @ kh.t() / math.sqrt(case["dh"])).masked_fill(ahead, -math.inf).softmax(-1)
            out[at:at + n, h] = w @ vh
        at, seen = at + n, seen + n + p
    if not case["files"]:
        return {"out": out}
    return {"out": out, "pool": prepare(dict(case, files=False), seed)["pool"].double()}


def _exact_sample(case, seed):
    import numpy as np

    z, t, k, p, m, u = (x.cpu().double().numpy() for x in _logits(case, seed))
    got = []
    for b in range(case["rows"]):
        w = np.exp((z[b] - z[b].max()) / t[b])
        kept = w >= m[b]
        if k[b] > 0:
            kept &= z[b] >= np.partition(z[b], -min(int(k[b]), len(w)))[-min(int(k[b]), len(w))]
        if p[b] < 1:
            size = np.sort(z[b][kept])[::-1]
            mass = np.cumsum(np.exp((size - z[b].max()) / t[b]))
            kept &= z[b] >= size[min(int(np.searchsorted(mass, p[b] * mass[-1])), len(size) - 1)]
        mass = np.cumsum(np.where(kept, w, 0.0))
        got.append(int(np.searchsorted(mass, u[b] * mass[-1], side="right")))
    return {"tokens": torch.tensor(got, dtype=torch.int32)}
