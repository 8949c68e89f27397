"""What a program that decodes from the library's 8-bit paged cache asks of it, as cases that can be timed and compared.

`op` says which operator a case is about:

  rope     rotary embedding of query and key rows whose positions have several axes (time, height, width), in place
           in the rows that a fused projection of queries, keys and values leaves
  store    key and value rows into pages of 64 tokens, 8 bits an element (e4m3), one power-of-two scale for each page and kv head
  attend   causal attention of a few rows of each sequence (one when decoding, some when several tokens are checked at once,
           hundreds when a prompt arrives in pieces) over the sequence's pages
  copy     pages copied to other pages: sequences forked for several answers, a pool made compact

With `own` false the operators are computed in their plain form, from elementary tensor operations in 32 bits (angles in
64); with `own` true by the calls of `paper_2603_05353_amd.Layer`.  Head shapes are the repository's own (32/8 heads of
128, 28/4 for vision-language layers, an fp32 layer with 8 heads of 64) and, in `draw`, others of the same kinds.

A page's keys lie as [kv head, token, d], its values as [kv head, d, byte], where the 64 tokens of a page take the byte
order of ORDER: what one lane of a matrix instruction needs lies in 16 consecutive bytes.
"""
import math

import torch

own = False

DEV = "cuda:0"
THETA = 1e6
PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn

# byte of token t in a value row of a page: bits 3:2 of t go to the top, then bit 5, bit 4 and bits 1:0
ORDER = [((t >> 2) & 3) << 4 | (t >> 5) << 3 | ((t >> 4) & 1) << 2 | (t & 3) for t in range(PAGE)]


def listed():
    wide = dict(dtype="bf16", hq=32, hkv=8, d=128)
    vlm = dict(dtype="bf16", hq=28, hkv=4, d=128)
    return [
        # the smallest call: the next token of one short conversation
        dict(name="attend-1x300", op="attend", seqs=1, longest=300, least=1.0, rows=1, lse=False, **wide),
        # a decoding batch of uneven conversations
        dict(name="attend-64x8k", op="attend", seqs=64, longest=8191, least=0.1, rows=1, lse=False, **wide),
        # one request over a very long context: few rows, the work has to be cut along the cache
        dict(name="attend-1x130k", op="attend", seqs=1, longest=130078, least=1.0, rows=1, lse=True, **wide),
        # five proposed tokens of each sequence checked at once, grouped heads of a vision-language layer
        dict(name="attend-12x20k-5", op="attend", seqs=12, longest=20480, least=0.5, rows=5, lse=False, **vlm),
        # the last 512 tokens of a 32K prompt, arriving after the rest
        dict(name="attend-1x32k-512", op="attend", seqs=1, longest=32768, least=1.0, rows=512, lse=False, **wide),
        # a small fp32 layer
        dict(name="attend-4x1k-f32", op="attend", seqs=4, longest=1025, least=0.5, rows=1, lse=True, dtype="f32", hq=8, hkv=8, d=64),
        # the next token's keys and values of a decoding batch
        dict(name="store-64x1", op="store", seqs=64, longest=8191, least=0.1, rows=1, spread=False, **wide),
        # a finished 32K context goes into the cache
        dict(name="store-32k", op="store", seqs=1, longest=32768, least=1.0, rows=32768, spread=False, **wide),
        # queries and keys of a decoding batch, and of a whole prompt of images and text
        dict(name="rope-64", op="rope", rows=64, axes="sections", pairing="half", **vlm),
        dict(name="rope-20k", op="rope", rows=20480, axes="cyclic", pairing="half", **vlm),
        # the last, partly filled page of 32 sequences forked; a pool compacted
        dict(name="copy-32", op="copy", pages=32, pool=512, **wide),
        dict(name="copy-2000", op="copy", pages=2000, pool=4200, **wide),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, most of them odd."""
    shapes = [("bf16", 32, 8, 128), ("bf16", 32, 8, 128), ("bf16", 28, 4, 128), ("bf16", 40, 8, 128), ("bf16", 16, 16, 128),
              ("bf16", 16, 2, 128), ("bf16", 64, 8, 128), ("bf16", 32, 8, 64), ("f32", 8, 8, 64), ("f32", 16, 4, 128)]
    dtype, hq, hkv, d = rng.choice(shapes)
    shape = dict(dtype=dtype, hq=hq, hkv=hkv, d=d)
    op = rng.choice(["attend", "attend", "attend", "store", "store", "rope", "copy"])
    if op == "rope":
        return dict(op=op, rows=_log_int(rng, 1, 20000), axes=rng.choice(["sections", "cyclic"]),
                    pairing=rng.choice(["half", "half", "interleaved"]), **shape)
    if op == "copy":
        n = _log_int(rng, 1, 1500)
        return dict(op=op, pages=n, pool=2 * n + rng.randint(1, 99), **shape)
    if op == "store":
        seqs = _log_int(rng, 1, 128)
        rows = 1 if rng.random() < 0.4 else _log_int(rng, 1, 32000 // seqs)
        longest = rows + _log_int(rng, 1, 8000)
        return dict(op=op, seqs=seqs, longest=longest, least=1.0 if seqs == 1 else round(rng.uniform(rows / longest, 1.0), 4), rows=rows,
                    spread=rng.random() < 0.3, **shape)
    kind = rng.random()
    if kind < 0.2:          # a piece of a prompt
        longest, seqs = _log_int(rng, 600, 30000), 1
        rows = _log_int(rng, 17, min(512, longest, 512 * 32768 // longest))
        if dtype == "f32":
            rows = min(rows, 96)
    else:
        longest = _log_int(rng, 16, 130000)
        seqs = _log_int(rng, 1, max(1, min(256, 260000 // longest)))
        rows = 1 if kind < 0.7 else rng.randint(2, 12)
    return dict(op=op, seqs=seqs, longest=longest, least=1.0 if seqs == 1 else round(rng.uniform(0.1, 1.0), 4), rows=rows,
                lse=rng.random() < 0.4, **shape)


# ---------------------------------------------------------------------------------------------------------------
# Inputs, made on the GPU from the seed.
# ---------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens of each sequence: the longest, and others spread evenly down to a share of it."""
    n, longest, least = case["seqs"], case["longest"], case["least"]
    return [longest] + [max(case["rows"], round(longest * (least + (1.0 - least) * (i - 0.5) / (n - 1)))) for i in range(1, n)]


def _exponents(amax):
    """The smallest e >= -100 with amax <= 448 * 2^e, for float32 amax >= 0."""
    m, e = torch.frexp(amax)                          # amax = m * 2^e, m in [0.5, 1): 448 = 0.875 * 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, -100)).clamp(min=-100)


def _power(e):
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


def _filled(g, n_pages, hkv, rows, cols):
    """A pool of pages with Gaussian contents whose size differs from page to page and head to head."""
    page = torch.empty(n_pages, hkv, rows, cols, dtype=F8, device=DEV)
    scale = torch.empty(n_pages, hkv, dtype=torch.float32, device=DEV)
    step = max(1, (1 << 28) // (hkv * rows * cols))
    for a in range(0, n_pages, step):
        b = min(n_pages, a + step)
        x = torch.randn(b - a, hkv, rows, cols, generator=g, device=DEV)
        x *= 0.7 + 0.6 * torch.rand(b - a, hkv, 1, 1, generator=g, device=DEV)
        s = _power(_exponents(x.abs().amax(dim=(2, 3))))
        page[a:b] = (x / s[:, :, None, None]).to(F8)
        scale[a:b] = s
    return page, scale


def _axes_of_pairs(case):
    """Which of the three axes turns each pair: stretches of pairs, or the axes in turn."""
    half = case["d"] // 2
    if case["axes"] == "cyclic":
        return [j % 3 if j < 3 * (half // 4) else 0 for j in range(half)]
    return [0 if j < half // 4 else 1 if j < half // 4 + 3 * half // 8 else 2 for j in range(half)]


def prepare(case, seed):
    op = case["op"]
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt, hq, hkv, d = DTYPES[case["dtype"]], case["hq"], case["hkv"], case["d"]
    s = dict(case=case, op=op)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    if op == "rope":
        rows = case["rows"]
        s["qkv"] = normal(rows, hq + 2 * hkv, d).to(dt)
        # images of 32 x 32 places with a stretch of text after every second one
        i = torch.arange(rows, device=DEV) + torch.randint(0, 30000, (1,), generator=g, device=DEV)
        block, at = i // 1024, i % 1024
        text = block % 3 == 2
        t = torch.where(text, i, 1024 * block)
        s["pos"] = torch.stack([t, torch.where(text, i, t + at // 32), torch.where(text, i, t + at % 32)], 1).to(torch.int32)
        s["axes"] = torch.tensor(_axes_of_pairs(case), dtype=torch.int32)
        longest = 1
    elif op == "copy":
        s["k"], s["k_scale"] = _filled(g, case["pool"], hkv, PAGE, d)
        s["v"], s["v_scale"] = _filled(g, case["pool"], hkv, d, PAGE)
        # page lists are the scheduler's, on the host
        pick = torch.randperm(case["pool"], generator=torch.Generator().manual_seed(int(seed) + 1))[: 2 * case["pages"]]
        s["src"], s["dst"] = pick[: case["pages"]].to(torch.int32), pick[case["pages"]:].to(torch.int32)
        longest = 1
    else:
        lens = torch.tensor(_lengths(case))
        lens = lens[torch.randperm(case["seqs"], generator=torch.Generator().manual_seed(int(seed) + 3))]
        longest = case["longest"]
        need = (lens + PAGE - 1) // PAGE
        total = int(need.sum())
        pool = total + 5
        order = torch.randperm(pool, generator=g, device=DEV)[:total].to(torch.int32)
        table = torch.full((case["seqs"], int(need.max())), -1, dtype=torch.int32, device=DEV)
        col = torch.arange(table.shape[1], device=DEV)[None, :]
        table[col < need.to(DEV)[:, None]] = order
        s["table"] = table
        s["k"], s["k_scale"] = _filled(g, pool, hkv, PAGE, d)
        s["v"], s["v_scale"] = _filled(g, pool, hkv, d, PAGE)
        rows = case["rows"]
        n = case["seqs"] * rows
        lens = lens.to(DEV)
        if op == "store" and case["spread"]:      # rows all over a sequence that is there already: recomputed tokens
            pick = torch.rand(case["seqs"], longest, generator=g, device=DEV)
            pick[torch.arange(longest, device=DEV)[None, :] >= lens[:, None]] = 2.0
            pos = torch.sort(torch.topk(pick, rows, dim=1, largest=False)[1], dim=1)[0]
            s["kv_len"] = lens.to(torch.int32)
        else:                                      # the last rows
            pos = lens[:, None] - rows + torch.arange(rows, device=DEV)[None, :]
            s["kv_len"] = (lens - rows).to(torch.int32)
        s["row_pos"] = pos.reshape(-1).to(torch.int32)
        s["row_start"] = None if rows == 1 else torch.arange(0, n + 1, rows, dtype=torch.int32, device=DEV)
        if op == "attend":
            s["q"] = normal(n, hq, d).to(dt)
            s["out"] = torch.empty_like(s["q"])
        else:
            s["k_new"] = (1.3 * normal(n, hkv, d)).to(dt)
            s["v_new"] = (1.3 * normal(n, hkv, d)).to(dt)
    if own:
        from paper_2603_05353_amd import Layer, PageCache
        s["layer"] = Layer(case["dtype"], hq, hkv, d, THETA, max_ctx=max(PAGE, -(-longest // PAGE) * PAGE), max_prompt=1,
                           pairing=case.get("pairing", "half"))
        if op != "rope":
            s["pages"] = PageCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    return s


def run(s):
    op, case = s["op"], s["case"]
    if own:
        layer, nq, nk = s["layer"], case["hq"], case["hkv"]
        if op == "rope":
            layer.rope_rows_axes(s["qkv"][:, : nq + nk], s["pos"], s["axes"])
            return {"qkv": s["qkv"]}
        if op == "copy":
            layer.copy_pages(s["pages"], s["src"], s["dst"])
        elif op == "store":
            layer.store_pages(s["pages"], s["table"], s["kv_len"], s["k_new"], s["v_new"], s["row_pos"], row_start=s["row_start"])
        else:
            got = layer.attend_pages(s["q"], s["row_pos"], s["pages"], s["table"], row_start=s["row_start"], max_rows=case["rows"],
                                     out=s["out"], return_lse=case["lse"])
            return {"out": got[0], "lse": got[1]} if case["lse"] else {"out": got}
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return {"rope": _plain_rope, "copy": _plain_copy, "store": _plain_store, "attend": _plain_attend}[op](s)


# ---------------------------------------------------------------------------------------------------------------
# The plain forms.
# ---------------------------------------------------------------------------------------------------------------
def _plain_rope(s):
    case = s["case"]
    d, heads = case["d"], case["hq"] + case["hkv"]
    freq = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    ang = s["pos"].double()[:, s["axes"].to(DEV).long()] * freq
    c, n = ang.cos().float()[:, None, :], ang.sin().float()[:, None, :]
    x = s["qkv"][:, :heads].float()
    if case["pairing"] == "half":
        a, b = x[..., : d // 2], x[..., d // 2:]
        turned = torch.cat([a * c - b * n, a * n + b * c], -1)
    else:
        a, b = x[..., 0::2], x[..., 1::2]
        turned = torch.stack([a * c - b * n, a * n + b * c], -1).flatten(-2)
    s["qkv"][:, :heads] = turned.to(s["qkv"].dtype)
    return {"qkv": s["qkv"]}


def _plain_copy(s):
    src, dst = s["src"].to(DEV).long(), s["dst"].to(DEV).long()
    for_bytes = (s["k"].view(torch.uint8), s["v"].view(torch.uint8))
    for_bytes[0][dst] = for_bytes[0][src]
    for_bytes[1][dst] = for_bytes[1][src]
    s["k_scale"][dst] = s["k_scale"][src]
    s["v_scale"][dst] = s["v_scale"][src]
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_put(pool, scale, x, page, at, touched, kept):
    """Rows x [n, Hkv, d] into slots `at` of pages `page`; pool is viewed as [page, head, token, d]."""
    x = x.float()
    amax = torch.zeros_like(scale).scatter_reduce_(0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
    need = _power(_exponents(amax))
    new = torch.where(kept[:, None], torch.maximum(scale, need), need)
    new = torch.where(touched[:, None], new, scale)
    shrink = torch.where(touched[:, None], torch.where(kept[:, None], scale / new, torch.zeros_like(scale)), torch.ones_like(scale))
    scale.copy_(new)
    # no more pages than rows are touched: those first, some that stay as they are behind them
    ids = torch.sort(touched, descending=True, stable=True)[1][: page.numel()]
    place = torch.zeros_like(touched, dtype=torch.int64).index_copy_(0, ids, torch.arange(ids.numel(), device=DEV))
    pool = pool.view(torch.uint8)
    by = shrink[ids][:, :, None, None]
    values = pool[ids].view(F8).float()
    values = torch.where(by == 0, torch.zeros_like(values), values * by)
    values[place[page][:, None], torch.arange(x.shape[1], device=DEV)[None, :], at[:, None]] = x / new[page][:, :, None]
    pool[ids] = values.to(F8).view(torch.uint8)


def _plain_store(s):
    rows = s["case"]["rows"]
    pos = s["row_pos"].long()
    seq = torch.arange(pos.numel(), device=DEV) // rows
    page = s["table"][seq, pos // PAGE].long()
    # how many tokens of its page are kept: those below kv_len which are not among the rows
    count = torch.zeros(s["k"].shape[0], dtype=torch.int64, device=DEV)
    again = count.clone().index_add_(0, page, (pos < s["kv_len"][seq]).long())
    there = (s["kv_len"][seq].long() - pos // PAGE * PAGE).clamp(0, PAGE)
    before = count.clone().index_copy_(0, page, there)
    touched = count.clone().index_fill_(0, page, 1) > 0
    kept = before > again
    byte = torch.tensor(ORDER, device=DEV)
    _plain_put(s["k"], s["k_scale"], s["k_new"], page, pos % PAGE, touched, kept)
    _plain_put(s["v"].transpose(2, 3), s["v_scale"], s["v_new"], page, byte[pos % PAGE], touched, kept)
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attend(s):
    case, table = s["case"], s["table"]
    n, rows, hq, hkv, d = case["seqs"], case["rows"], case["hq"], case["hkv"], case["d"]
    width = table.shape[1]
    page = table.clamp(min=0).long().reshape(-1)

    def sequence(pool, scale):                         # [sequence, kv head, token, d] in 32 bits
        x = pool.view(torch.uint8)[page].view(F8).float() * scale[page][:, :, None, None]
        return x.view(n, width, hkv, PAGE, d).transpose(1, 2).reshape(n, hkv, width * PAGE, d)

    k = sequence(s["k"], s["k_scale"])
    v = sequence(s["v"].view(torch.uint8)[..., torch.tensor(ORDER, device=DEV)].transpose(2, 3).contiguous().view(F8), s["v_scale"])
    q = s["q"].float().view(n, rows, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d)
    logits = torch.matmul(q, k.transpose(2, 3)) * d ** -0.5
    hidden = torch.arange(width * PAGE, device=DEV)[None, None, :] > s["row_pos"].view(n, rows, 1)
    logits = logits.view(n, hkv, rows, hq // hkv, -1).masked_fill(hidden[:, None, :, None, :], -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - top)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, hkv, -1, width * PAGE), v).view(n, hkv, rows, hq // hkv, d) / z
    out = {"out": o.permute(0, 2, 1, 3, 4).reshape(n * rows, hq, d).to(s["q"].dtype)}
    if case["lse"]:
        out["lse"] = (top + torch.log(z)).permute(0, 2, 1, 3, 4).reshape(n * rows, hq)
    return out


# ---------------------------------------------------------------------------------------------------------------
# What a pass cannot do without.
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if op == "rope":
        x = case["rows"] * (hq + hkv) * d
        return {"bytes": 2.0 * x * e + 12.0 * case["rows"], "flops": 3.0 * x}
    if op == "copy":
        return {"bytes": 2.0 * case["pages"] * (2 * hkv * PAGE * d + 8 * hkv), "flops": 0.0}
    total, n = sum(_lengths(case)), case["seqs"] * case["rows"]
    if op == "store":
        return {"bytes": 2.0 * n * hkv * d * (e + 1) + 8.0 * n, "flops": 0.0}
    keys = case["rows"] * (total - case["seqs"] * (case["rows"] - 1) / 2.0)
    return {"bytes": 2.0 * total * hkv * d + 2.0 * n * hq * d * e, "flops": 4.0 * d * hq * keys}


# ---------------------------------------------------------------------------------------------------------------
# The same results in 64 bits, from the definitions.
# ---------------------------------------------------------------------------------------------------------------
def _to_e4m3(x):
    """float64 values of at most 448, rounded to the nearest that e4m3 has, ties to the even one."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_rope(case, s):
    d = case["d"]
    out = s["qkv"].double()
    for j, axis in enumerate(s["axes"].tolist()):
        ang = s["pos"][:, axis].double() * THETA ** (-2.0 * j / d)
        c, n = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        i0, i1 = (j, j + d // 2) if case["pairing"] == "half" else (2 * j, 2 * j + 1)
        a, b = out[:, : case["hq"] + case["hkv"], i0].clone(), out[:, : case["hq"] + case["hkv"], i1].clone()
        out[:, : case["hq"] + case["hkv"], i0], out[:, : case["hq"] + case["hkv"], i1] = a * c - b * n, a * n + b * c
    return {"qkv": out}


def _exact_store(case, s):
    """Page by page as the definition goes; values as e4m3 numbers beside their scales."""
    rows, hkv = case["rows"], case["hkv"]
    pos = s["row_pos"].view(case["seqs"], rows).tolist()
    table, lens = s["table"].tolist(), s["kv_len"].tolist()
    got = {"k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double()}
    for name in ("k", "v"):
        pool, scale, x = s[name].double(), got[name + "_scale"], s[name + "_new"].double()
        if name == "v":                                # tokens in their own order, as keys have them
            pool = pool[..., torch.tensor(ORDER, device=DEV)].transpose(2, 3).contiguous()
        for q in range(case["seqs"]):
            first = 0
            while first < rows:
                logical = pos[q][first] // PAGE
                last = first
                while last < rows and pos[q][last] // PAGE == logical:
                    last += 1
                page, slots = table[q][logical], [p % PAGE for p in pos[q][first:last]]
                kept = set(range(max(0, min(PAGE, lens[q] - logical * PAGE)))) - set(slots)
                new = x[q * rows + first: q * rows + last]
                top = new.abs().amax(dim=(0, 2))
                need = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(min=-100.0))
                after = torch.maximum(need, scale[page]) if kept else need
                pool[page] = _to_e4m3(pool[page] * (scale[page] / after)[:, None, None]) if kept else 0.0
                pool[page][:, torch.tensor(slots, device=DEV)] = _to_e4m3(new / after[None, :, None]).transpose(0, 1)
                scale[page] = after
                first = last
        if name == "v":
            back = torch.empty_like(pool).transpose(2, 3).contiguous()
            back[..., torch.tensor(ORDER, device=DEV)] = pool.transpose(2, 3)
            pool = back
        got[name] = pool
    return got


def _exact_attend(case, s):
    n, rows, hq, hkv, d = case["seqs"], case["rows"], case["hq"], case["hkv"], case["d"]
    grp = hq // hkv
    out = torch.empty(n * rows, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.empty(n * rows, hq, dtype=torch.float64, device=DEV)
    order = torch.tensor(ORDER, device=DEV)
    kb, vb = s["k"].view(torch.uint8), s["v"].view(torch.uint8)
    pos = s["row_pos"].view(n, rows).long()
    for i in range(n):
        last = int(pos[i, -1])
        pages = s["table"][i, : last // PAGE + 1].long()
        for h in range(hkv):
            k = kb[pages, h].view(F8).double() * s["k_scale"][pages, h].double()[:, None, None]
            v = vb[pages, h].view(F8).double() * s["v_scale"][pages, h].double()[:, None, None]
            k = k.reshape(-1, d)[: last + 1]
            v = v[..., order].transpose(1, 2).reshape(-1, d)[: last + 1]
            q = s["q"][i * rows:(i + 1) * rows, h * grp:(h + 1) * grp].double().reshape(rows * grp, d)
            logits = (torch.mm(q, k.t().contiguous()) * d ** -0.5).view(rows, grp, -1)
            logits.masked_fill_((torch.arange(last + 1, device=DEV)[None, :] > pos[i][:, None])[:, None, :], -math.inf)
            z = torch.logsumexp(logits, 2)
            o = torch.mm(torch.exp(logits - z[..., None]).view(rows * grp, -1), v.contiguous())
            out[i * rows:(i + 1) * rows, h * grp:(h + 1) * grp] = o.view(rows, grp, d)
            lse[i * rows:(i + 1) * rows, h * grp:(h + 1) * grp] = z
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    if case["op"] == "attend":
        return _exact_attend(case, s)
    if case["op"] == "store":
        return _exact_store(case, s)
    got = {name: s[name].double() for name in ("k", "v", "k_scale", "v_scale")}
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        for name in got:
            got[name][b] = got[name][a]
    return got
