"""The operators around a paged cache of keys and values held in the 8-bit types, as cases that can be timed and compared.

  append     what a layer does between its projection and its attention: queries and keys normed per head (where the model has
             such norms) and turned by their position, keys and values compressed, one scale per row of `dim` values, into the
             cache rows that their slots name.  The pass ends with the expansion of the cache: codes are compared as the values
             they stand for.
  attention  new tokens of a batch of sequences (one each, a few, a prompt's chunk, whole prompts) against their cached keys
             and values, causal, several query heads per cached head.

`run` makes the framework's calls where `own` is true and computes the same from elementary torch operations where it is
false; `exact` says what the operators are in binary64.

A case is a dict of plain values:
  op       "append" or "attention"
  kind     data type of the cache: 0 dynamic tree, 1 linear, 2 static tree, 3 mantissa
  heads    query heads (append: 0 where the call has no queries)
  kv_heads cached heads
  dim      elements of a head
  page     tokens of a page
  dtype    "bfloat16", "float16" or "float32" (append only)
and for append
  tokens, padded   tokens of the call, and how many of them at its end are padding (no slot)
  norm     whether queries and keys are normed
  rot      elements of a head that are turned (0: none)
  interleaved      whether the pairs that are turned lie side by side instead of half of `rot` apart
for attention
  batch    sequences
  chunk    new tokens of a sequence: every sequence's where ragged is false, else the largest
  longest  cached tokens of the longest sequence (its new ones among them)
  ragged   whether the sequences differ in their numbers of tokens
  window   tokens that a query sees at most (0: all up to its own)
"""
import math

import torch

own = False

#: the bfloat16, float16 and float32 of a case
DTYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}

POSITIONS = 16384  # rows of the angle tables
EPS = 1e-6


def listed():
    return [
        # One token of one sequence: the smallest call of decoding, once per layer and token.  Latency counts.
        {"name": "append_one", "op": "append", "kind": 0, "tokens": 1, "padded": 0, "heads": 32, "kv_heads": 8, "dim": 128, "page": 16,
         "dtype": "bfloat16", "norm": True, "rot": 128, "interleaved": False},
        # One token each of a batch of 61 sequences, padded to 64, small heads, half of a head turned.
        {"name": "append_batch", "op": "append", "kind": 1, "tokens": 64, "padded": 3, "heads": 16, "kv_heads": 4, "dim": 64, "page": 32,
         "dtype": "float16", "norm": False, "rot": 32, "interleaved": True},
        # A long prompt at once.
        {"name": "append_prompt", "op": "append", "kind": 0, "tokens": 8191, "padded": 0, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64,
         "dtype": "bfloat16", "norm": True, "rot": 128, "interleaved": False},
        # Keys and values in 32 bits without queries, an odd head length: a cache filled from another program's activations.
        {"name": "append_f32", "op": "append", "kind": 2, "tokens": 2077, "padded": 0, "heads": 0, "kv_heads": 12, "dim": 80, "page": 16,
         "dtype": "float32", "norm": False, "rot": 80, "interleaved": False},
        # Decoding for one user with a short history: latency again.
        {"name": "decode_one", "op": "attention", "kind": 0, "batch": 1, "chunk": 1, "longest": 1337, "ragged": False, "window": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "dtype": "bfloat16"},
        # Decoding for a batch of 64 sequences of unequal age.
        {"name": "decode_batch", "op": "attention", "kind": 0, "batch": 64, "chunk": 1, "longest": 4096, "ragged": True, "window": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bfloat16"},
        # Two very long documents.
        {"name": "decode_long", "op": "attention", "kind": 0, "batch": 2, "chunk": 1, "longest": 131072, "ragged": True, "window": 0,
         "heads": 64, "kv_heads": 8, "dim": 128, "page": 128, "dtype": "bfloat16"},
        # A cached head for every query head, small heads, the mantissa type.
        {"name": "decode_heads", "op": "attention", "kind": 3, "batch": 32, "chunk": 1, "longest": 2001, "ragged": True, "window": 0,
         "heads": 16, "kv_heads": 16, "dim": 64, "page": 16, "dtype": "float16"},
        # Five drafted tokens of each of sixteen sequences are verified at once.
        {"name": "chunk_draft", "op": "attention", "kind": 0, "batch": 16, "chunk": 5, "longest": 8192, "ragged": True, "window": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bfloat16"},
        # A chunk of a long prompt behind what is cached of it.
        {"name": "chunk_prompt", "op": "attention", "kind": 0, "batch": 1, "chunk": 2048, "longest": 10240, "ragged": False, "window": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bfloat16"},
        # Chunks of unequal length under a sliding window, an odd head length.
        {"name": "chunk_window", "op": "attention", "kind": 2, "batch": 7, "chunk": 701, "longest": 3001, "ragged": True, "window": 512,
         "heads": 12, "kv_heads": 12, "dim": 80, "page": 32, "dtype": "float16"},
        # Whole prompts from an empty cache.
        {"name": "chunk_whole", "op": "attention", "kind": 0, "batch": 4, "chunk": 4096, "longest": 4096, "ragged": True, "window": 0,
         "heads": 16, "kv_heads": 2, "dim": 128, "page": 64, "dtype": "bfloat16"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    """What a case may cost at most goes by: bytes, operations, and elements that the plain form holds at once."""
    w = work(case)
    if case["op"] == "append":
        return w["bytes"], w["flops"], case["tokens"] * case["dim"] * (case["heads"] + 2 * case["kv_heads"])
    held = case["batch"] * case["longest"] * (case["kv_heads"] * case["dim"] + case["heads"] * case["chunk"])
    return w["bytes"], w["flops"], held


def draw(rng):
    most = [max(c) for c in zip(*(_cost(c) for c in listed()))]
    while True:
        heads, kv_heads = rng.choice([(32, 8), (16, 2), (12, 12), (8, 1), (64, 8), (24, 8), (20, 4), (16, 16)])
        case = {"kind": rng.randrange(4), "heads": heads, "kv_heads": kv_heads, "dim": rng.choice([64, 64, 80, 96, 128, 128, 128, 256]),
                "page": rng.choice([16, 32, 64, 128])}
        if rng.random() < 0.4:
            tokens = _log(rng, 1, 8192)
            case |= {"op": "append", "tokens": tokens, "padded": rng.choice([0, 0, tokens // 7]), "dtype": rng.choice(["bfloat16", "bfloat16", "float16", "float32"]),
                     "norm": rng.random() < 0.5, "rot": rng.choice([0, case["dim"] // 2, case["dim"], case["dim"]]),
                     "interleaved": rng.random() < 0.3, "heads": rng.choice([0, heads, heads])}
        else:
            chunk = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 4096)])
            case |= {"op": "attention", "batch": _log(rng, 1, 64), "chunk": chunk, "longest": _log(rng, chunk, 131072),
                     "ragged": rng.random() < 0.7, "window": rng.choice([0, 0, 0, rng.randint(1, 4096)]), "dtype": rng.choice(["bfloat16", "bfloat16", "float16"])}
        if all(a <= b for a, b in zip(_cost(case), most)):
            return case


def sizes(case):
    """(new tokens, cached tokens) of each sequence: spread evenly over their ranges where the case is ragged."""
    got = []
    for b in range(case["batch"]):
        f = (b * 0.6180339887498949) % 1.0 if case["ragged"] else 0.0  # sequence 0 has the most of both
        long = max(1, round(case["longest"] * (1.0 - 0.95 * f)))
        got.append((min(long, max(1, round(case["chunk"] * (1.0 - 0.9 * f)))), long))
    return got


def work(case):
    d, size = case["dim"], {"float32": 4}.get(case["dtype"], 2)
    if case["op"] == "append":
        t, kept = case["tokens"], case["tokens"] - case["padded"]
        rows = _pages(case) * case["page"] * 2 * case["kv_heads"]  # expanded at the end
        read = t * d * size * (case["heads"] + 2 * case["kv_heads"]) + t * (8 + 8 + 4 * case["rot"])
        written = t * d * size * case["heads"] + kept * 2 * case["kv_heads"] * (d + 4)
        return {"bytes": read + written + rows * (d + 4 + 4 * d), "flops": 8 * t * d * (case["heads"] + 2 * case["kv_heads"]) + rows * d}
    pairs = tokens = new = 0
    for n, long in sizes(case):
        w = case["window"] or long
        first = long - n  # of the new tokens
        pairs += sum(min(p + 1, w) for p in range(first, long))
        tokens += long - max(0, first + 1 - w)
        new += n
    return {"bytes": 2 * case["kv_heads"] * tokens * (d + 4) + 2 * new * case["heads"] * d * size, "flops": 4 * d * case["heads"] * pairs}


def _pages(case):
    """Pages of the cache that an append case writes to: a fifth of it stays as it was."""
    return -(-max(case["tokens"] - case["padded"], 1) * 5 // (4 * case["page"])) + 1


# ---------------------------------------------------------------- the data types, from their formulas


def _magnitudes(kind):
    """The 128 magnitudes of a type as float64 of the nearest binary32, by 7-bit field."""
    got = []
    for j in range(128):
        if kind == 1:
            v = j / 127
        elif kind == 0:
            zeros = 7 - j.bit_length()
            t = 6 - zeros
            v = (0.1 + 0.9 * (j - (1 << t) + 0.5) / (1 << t)) * 10.0 ** -zeros if j else 0.0
        elif kind == 2:
            v = (0.1 + 0.9 * (j % 16 + 0.5) / 16) * 10.0 ** (j // 16 - 7)
        else:
            v = (j % 16) * 10.0 ** (j // 16 - 8)
        got.append(v)
    return torch.tensor(got, dtype=torch.float64).float()


def _tables(kind, device):
    """(value of every code, the borders between neighbouring magnitudes in binary64, code of each magnitude by rank)"""
    m = _magnitudes(kind)
    ranks, code = torch.unique(m, return_inverse=True)
    first = torch.full((ranks.numel(),), 127, dtype=torch.int64).scatter_reduce(0, code, torch.arange(128), "amin")
    borders = (ranks.double()[1:] + ranks.double()[:-1]) / 2
    return torch.cat([m, -m]).to(device), borders.to(device), first.to(torch.uint8).to(device)


def _compress(y, tables):
    """Codes and scales of the rows of y (float32, the last axis one row each)."""
    _, borders, code = tables
    s = y.abs().amax(-1)
    d = torch.where(s == 0, torch.ones_like(s), s).unsqueeze(-1)
    x = (y.double() / d.double()).float()  # the quotient of two float32, rounded once
    rank = torch.bucketize(x.abs().double(), borders, out_int32=True)  # a value on a border goes to the smaller magnitude
    return code[rank] + torch.signbit(y).to(torch.uint8) * 128, s


def _fill(shape, tables, g, device):
    """Codes and scales of rows of normal values, row by row of another size."""
    codes = torch.empty(shape, dtype=torch.uint8, device=device)
    scales = torch.empty(shape[:-1], dtype=torch.float32, device=device)
    borders = tables[1].float()
    step = max(1, (1 << 26) // (shape[-1] * shape[-2] * shape[-3]))
    for part in range(shape[0]):
        for at in range(0, shape[1], step):
            y = torch.randn(codes[part, at : at + step].shape, generator=g, device=device)
            s = y.abs().amax(-1)
            rank = torch.bucketize((y / s.unsqueeze(-1)).abs(), borders, out_int32=True)
            codes[part, at : at + step] = tables[2][rank] + torch.signbit(y).to(torch.uint8) * 128
            scales[part, at : at + step] = s * torch.exp(0.3 * torch.randn(s.shape, generator=g, device=device))
    return codes, scales


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    dev, dt, d = torch.device("cuda"), DTYPES[case["dtype"]], case["dim"]
    g = torch.Generator(device=dev).manual_seed(seed)
    tables = _tables(case["kind"], dev)
    state = {"case": case, "tables": tables}
    if case["op"] == "append":
        t, kept, pages = case["tokens"], case["tokens"] - case["padded"], _pages(case)
        # queries, keys and values are parts of the projection's output
        both = torch.randn(t, case["heads"] + 2 * case["kv_heads"], d, generator=g, device=dev).mul_(torch.exp(torch.randn(d, generator=g, device=dev) * 0.5)).to(dt)
        q, k, v = both.split([case["heads"], case["kv_heads"], case["kv_heads"]], 1)
        slots = torch.full((t,), -1, dtype=torch.int64, device=dev)
        if t >= 512:  # a prompt: whole pages in any order
            order = torch.randperm(pages, generator=g, device=dev).unsqueeze(1) * case["page"] + torch.arange(case["page"], device=dev)
            slots[:kept] = order.reshape(-1)[:kept]
            start = int(torch.randint(0, POSITIONS - t, (1,), generator=g, device=dev))
            positions = torch.arange(start, start + t, device=dev)
        else:  # one token each of many sequences
            slots[:kept] = torch.randperm(pages * case["page"], generator=g, device=dev)[:kept]
            positions = torch.randint(0, POSITIONS, (t,), generator=g, device=dev)
        codes, scales = _fill((2, pages, case["kv_heads"], case["page"], d), tables, g, dev)
        state |= {"k": k, "v": v, "slots": slots, "kept": kept, "codes": codes, "scales": scales, "q": q if case["heads"] else None,
                  "positions": positions if case["rot"] else None, "rotation": None, "q_weight": None, "k_weight": None}
        if case["rot"]:
            half = case["rot"] // 2
            angle = torch.arange(POSITIONS, dtype=torch.float64, device=dev).unsqueeze(1) * 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
            state["rotation"] = torch.stack([angle.cos(), angle.sin()], 1).float()
        if case["norm"]:
            state["k_weight"] = torch.rand(d, generator=g, device=dev) + 0.5
            if case["heads"]:
                state["q_weight"] = torch.rand(d, generator=g, device=dev) + 0.5
        return state
    each = sizes(case)
    new, lens = [n for n, _ in each], [m for _, m in each]
    per = [-(-m // case["page"]) for m in lens]
    pool = sum(per) + 3
    codes, scales = _fill((2, pool, case["kv_heads"], case["page"], d), tables, g, dev)
    order = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    pages = torch.zeros((case["batch"], max(per)), dtype=torch.int32, device=dev)
    at = 0
    for b, p in enumerate(per):
        pages[b, :p] = order[at : at + p]
        at += p
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    q = (torch.randn(starts[-1], case["heads"], d, generator=g, device=dev) * 1.5).to(dt)
    return state | {"q": q, "codes": codes, "scales": scales, "pages": pages, "lens": torch.tensor(lens, dtype=torch.int32, device=dev),
                    "starts": torch.tensor(starts, dtype=torch.int32, device=dev), "longest": max(lens), "most": max(new),
                    "even": len(set(new)) == 1}


# ---------------------------------------------------------------- one pass


def run(state):
    return _append(state) if state["case"]["op"] == "append" else _attention(state)


def _append(st):
    case = st["case"]
    if own:
        from paper_1511_04561_amd import dq8
        q = dq8.cache_append(case["kind"], st["k"], st["v"], st["slots"], st["codes"], st["scales"], positions=st["positions"],
                             rotation=st["rotation"], interleaved=case["interleaved"], q=st["q"], q_weight=st["q_weight"],
                             k_weight=st["k_weight"], eps=EPS)
        values = dq8.decode(case["kind"], st["codes"], st["scales"], case["dim"])
        return {"values": values.view(st["codes"].shape), "scales": st["scales"], "q": q}
    kept, page = st["kept"], case["page"]
    k = _turn(_norm(st["k"].double(), st["k_weight"]), st, case).float()
    slots = st["slots"][:kept]
    for part, rows in enumerate((k, st["v"].float())):
        codes, scales = _compress(rows[:kept], st["tables"])
        st["codes"][part][slots // page, :, slots % page] = codes
        st["scales"][part][slots // page, :, slots % page] = scales
    q = None if st["q"] is None else _turn(_norm(st["q"].float(), st["q_weight"]), st, case).to(st["q"].dtype)
    return {"values": st["tables"][0][st["codes"].int()] * st["scales"].unsqueeze(-1), "scales": st["scales"], "q": q}


def _norm(x, weight):
    if weight is None:
        return x
    return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight.to(x.dtype)


def _turn(x, st, case):
    rot = case["rot"]
    if not rot:
        return x
    c, s = st["rotation"][st["positions"]].to(x.dtype).unsqueeze(1).unbind(2)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., : rot // 2], x[..., rot // 2 : rot])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _attention(st):
    case, q = st["case"], st["q"]
    if own:
        from paper_1511_04561_amd import dq8
        return dq8.cache_attention(case["kind"], q, st["codes"], st["scales"], st["pages"], st["lens"], starts=None if st["even"] else st["starts"],
                                   max_new=st["most"], window=case["window"])
    batch, kv, d, most, longest = case["batch"], case["kv_heads"], case["dim"], st["most"], st["longest"]
    group = case["heads"] // kv
    begin, new, lens = st["starts"][:-1].long(), (st["starts"][1:] - st["starts"][:-1]).long(), st["lens"].long()
    cb, pages = st["tables"][0], st["pages"].long()
    j = torch.arange(longest, device=q.device)
    i = torch.arange(most, device=q.device)
    k, v = ((cb[st["codes"][part][pages].int()] * st["scales"][part][pages].unsqueeze(-1)).transpose(1, 2).reshape(batch, kv, -1, d)[:, :, :longest]
            for part in (0, 1))
    rows = q[(begin[:, None] + i).clamp(max=q.shape[0] - 1)].float()  # batch, most, heads, d
    rows = rows.view(batch, most, kv, group, d).permute(0, 2, 3, 1, 4).reshape(batch, kv, group * most, d)
    s = torch.matmul(rows, k.transpose(-1, -2)).view(batch, kv, group, most, longest) * d**-0.5
    at = (lens - new)[:, None] + i  # position of each query
    seen = j <= at[:, :, None]
    if case["window"]:
        seen &= j > at[:, :, None] - case["window"]
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(s - top)
    out = torch.matmul(p.view(batch, kv, group * most, longest), v).view(batch, kv, group, most, d) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = out.permute(0, 3, 1, 2, 4).reshape(batch, most, case["heads"], d)
    token = torch.arange(q.shape[0], device=q.device)
    b = torch.searchsorted(st["starts"][1:].long(), token, right=True)
    return out[b, token - begin[b]].to(q.dtype)


# ---------------------------------------------------------------- the operators in binary64


def exact(case, seed):
    st = prepare(case, seed)
    cb = _magnitudes(case["kind"]).double().to(st["codes"].device)
    full = torch.cat([cb, -cb])
    if case["op"] == "append":
        values = torch.empty(st["codes"].shape, dtype=torch.float64, device=cb.device)
        for part in range(2):
            values[part] = full[st["codes"][part].long()] * st["scales"][part].double().unsqueeze(-1)
        scales = st["scales"].double()
        for t in range(0, st["kept"], 256):
            piece = slice(t, min(t + 256, st["kept"]))
            slot = st["slots"][piece]
            for part, x in enumerate((_row64(st, case, "k", piece), st["v"][piece].double())):
                x = x.float().double()  # what is compressed is a binary32 value
                s = x.abs().amax(-1, keepdim=True)
                u = (x / s.masked_fill(s == 0, 1.0)).float().double()
                # the nearest of all magnitudes, the smaller of two that are as near
                order = cb.sort().values
                far = (u.abs().unsqueeze(-1) - order).abs()
                near = order[far.argmin(-1)]
                lower = order[(torch.searchsorted(order, near.contiguous()) - 1).clamp(min=0)]
                near = torch.where((u.abs() - lower).abs() <= (u.abs() - near).abs(), lower, near)
                values[part][slot // case["page"], :, slot % case["page"]] = torch.copysign(near, u) * s
                scales[part][slot // case["page"], :, slot % case["page"]] = s.squeeze(-1)
        q = None if st["q"] is None else _row64(st, case, "q", slice(0, case["tokens"]))
        return {"values": values, "scales": scales, "q": q}
    q, d = st["q"], case["dim"]
    group = case["heads"] // case["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    at = 0
    for b, (n, long) in enumerate(sizes(case)):
        page = st["pages"][b, : -(-long // case["page"])].long()
        pos = torch.arange(long - n, long, device=q.device)
        j = torch.arange(long, device=q.device)
        hidden = j[None, :] > pos[:, None]
        if case["window"]:
            hidden |= pos[:, None] - j[None, :] >= case["window"]
        for h in range(case["kv_heads"]):
            k, v = (full[st["codes"][part, page, h].reshape(-1, d)[:long].long()] * st["scales"][part, page, h].reshape(-1)[:long].double().unsqueeze(1)
                    for part in (0, 1))
            for x in range(h * group, (h + 1) * group):
                score = (q[at : at + n, x].double() @ k.T) / math.sqrt(d)
                weight = torch.softmax(score.masked_fill(hidden, -math.inf), 1)
                out[at : at + n, x] = weight @ v
        at += n
    return out


def _row64(st, case, which, piece):
    """Queries or keys of some tokens, normed and turned, in binary64."""
    x, weight = st[which][piece].double(), st[which + "_weight"]
    if weight is not None:
        x = x * torch.rsqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * weight.double()
    if case["rot"]:
        half = case["rot"] // 2
        table = st["rotation"][st["positions"][piece]].double()
        z = torch.complex(table[:, 0], table[:, 1]).unsqueeze(1)
        if case["interleaved"]:
            turned = torch.view_as_real(torch.view_as_complex(x[..., : 2 * half].reshape(*x.shape[:-1], half, 2).contiguous()) * z).reshape(*x.shape[:-1], 2 * half)
        else:
            y = torch.complex(x[..., :half].contiguous(), x[..., half : 2 * half].contiguous()) * z
            turned = torch.cat([y.real, y.imag], -1)
        x = torch.cat([turned, x[..., 2 * half :]], -1)
    return x
