"""The operators of a decoding step with drafted tokens, on both sides of the paged cache, as cases that can be timed and compared.

  encode   weights of a linear layer [rows, cols] compressed to 4 bits, one bfloat16 scale per `group` neighbours of a row, and expanded again:
           codes are compared as the values they stand for.
  product  activations of a few tokens (or a prompt's) times such weights: out[m, n] = sum_k x[m, k] w[n, k] + bias[n].
  verify   drafted tokens judged by the target model's probabilities with given random numbers: the drafts that stay, and one token drawn
           behind them.
  plan     block tables, slots and positions of a step from the lengths of its requests: rejected drafts dropped, pages taken from and
           given back to a stack of free ones.

`run` makes the framework's calls where `own` is true and computes the same from elementary torch operations where it is
false; `exact` says what `encode` and `product` are in binary64 (the other two return whole numbers only).

A case is a dict of plain values:
  op       "encode", "product", "verify" or "plan"
and for encode and product
  rows, cols, group   of the weights
  dtype    of the weights (encode) or the activations: "bfloat16", "float16" or "float32" (encode only)
and for product
  tokens   rows of the activations
  out      dtype of the result
  bias     whether a bias is added
for verify
  batch, chunk   sequences, and rows of a sequence (its last accepted token and its drafts): every sequence's where ragged is false, else
           the largest
  ragged   whether the sequences differ in their numbers of rows
  vocab    probabilities of a row
  dtype    of the probabilities
  draft    whether the draft has probabilities too (else it is taken as sure of what it proposed)
for plan
  batch, page   sequences, and tokens of a page
  new, drop     new tokens of a sequence and tokens taken back from its end, at most
  longest  cached tokens of the longest sequence before the step (0: none has any)
  finished share of the sequences that end with this step and give back all their pages
"""
import math

import torch

own = False

#: the bfloat16, float16 and float32 of a case
DTYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}

#: the magnitudes of a code, in units of the group's scale, and the borders between them
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
#: the largest scale: the largest bfloat16 number whose sixfold still is a binary32 number
TOP = 170 * 2.0 ** 118


def listed():
    return [
        # One token through a square projection: the smallest call of a decoding layer.  Latency counts.
        {"name": "product_one", "op": "product", "rows": 4096, "cols": 4096, "group": 32, "tokens": 1, "dtype": "bfloat16", "out": "bfloat16", "bias": False},
        # One token through a wide layer of a large network: the rate at which weights are read.
        {"name": "product_wide", "op": "product", "rows": 28672, "cols": 8192, "group": 128, "tokens": 1, "dtype": "bfloat16", "out": "bfloat16", "bias": False},
        # Five rows each of four sequences (drafts that are verified) through a narrow long layer with a bias.
        {"name": "product_draft", "op": "product", "rows": 4096, "cols": 14336, "group": 64, "tokens": 20, "dtype": "float16", "out": "float16", "bias": True},
        # Logits in 32 bits of thirteen tokens over a vocabulary of an odd size.
        {"name": "product_head", "op": "product", "rows": 50021, "cols": 4096, "group": 32, "tokens": 13, "dtype": "bfloat16", "out": "float32", "bias": False},
        # A prompt of 500 tokens through a layer: bound by products, not by weights.
        {"name": "product_prompt", "op": "product", "rows": 8192, "cols": 4096, "group": 32, "tokens": 500, "dtype": "bfloat16", "out": "bfloat16", "bias": False},
        # A layer's weights when a model is loaded.
        {"name": "encode_layer", "op": "encode", "rows": 14336, "cols": 4096, "group": 32, "dtype": "bfloat16"},
        # Odd sizes: rows and columns that fill no tile.
        {"name": "encode_odd", "op": "encode", "rows": 1001, "cols": 777, "group": 64, "dtype": "float32"},
        # Four drafts of one user's sequence: latency again.
        {"name": "verify_one", "op": "verify", "batch": 1, "chunk": 5, "ragged": False, "vocab": 32000, "dtype": "float32", "draft": True},
        # A batch of 64 sequences with up to eight drafts each, a large vocabulary.
        {"name": "verify_batch", "op": "verify", "batch": 64, "chunk": 9, "ragged": True, "vocab": 131072, "dtype": "float32", "draft": True},
        # Drafts without probabilities (found in the text before), an odd vocabulary, 16 bits.
        {"name": "verify_sure", "op": "verify", "batch": 33, "chunk": 6, "ragged": True, "vocab": 50021, "dtype": "bfloat16", "draft": False},
        # A decoding step of 256 sequences with five rows each, after the last step's rejections.
        {"name": "plan_step", "op": "plan", "batch": 256, "page": 16, "new": 5, "drop": 4, "longest": 4096, "finished": 0.02},
        # Prompts of unequal length that start together.
        {"name": "plan_prompts", "op": "plan", "batch": 24, "page": 64, "new": 8192, "drop": 0, "longest": 0, "finished": 0.0},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    """What a case may cost at most goes by: bytes, operations, and elements that the plain form or its inputs hold at once."""
    w = work(case)
    held = {"encode": lambda: case["rows"] * case["cols"], "product": lambda: case["rows"] * (case["cols"] + case["tokens"]),
            "verify": lambda: case["batch"] * case["chunk"] * case["vocab"], "plan": lambda: case["batch"] * (case["longest"] + case["new"])}[case["op"]]()
    return w["bytes"], w["flops"], held


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = [max(a, b) for a, b in zip(most.get(c["op"], (0, 0, 0)), _cost(c))]
    while True:
        op = rng.choice(["encode", "product", "product", "product", "verify", "verify", "plan"])
        case = {"op": op}
        if op in ("encode", "product"):
            case |= {"rows": _log(rng, 16, 32768), "cols": _log(rng, 64, 28672), "group": rng.choice([32, 32, 64, 128])}
            if rng.random() < 0.5:  # most layers have sizes of this kind
                case |= {"rows": -(-case["rows"] // 256) * 256, "cols": -(-case["cols"] // 256) * 256}
        if op == "encode":
            case["dtype"] = rng.choice(["bfloat16", "float16", "float32"])
        elif op == "product":
            dtype = rng.choice(["bfloat16", "bfloat16", "float16"])
            case |= {"tokens": rng.choice([1, rng.randint(2, 8), rng.randint(9, 64), _log(rng, 65, 512)]), "dtype": dtype, "out": rng.choice([dtype, dtype, "float32"]),
                     "bias": rng.random() < 0.3}
        elif op == "verify":
            case |= {"batch": _log(rng, 1, 128), "chunk": rng.randint(1, 17), "ragged": rng.random() < 0.7, "vocab": _log(rng, 1000, 262144),
                     "dtype": rng.choice(["float32", "float32", "bfloat16", "float16"]), "draft": rng.random() < 0.7}
        else:
            new = rng.choice([1, rng.randint(2, 9), _log(rng, 10, 8192)])
            longest = rng.choice([0, _log(rng, 1, 32768)])
            case |= {"batch": _log(rng, 1, 1024), "page": rng.choice([16, 32, 64, 128]), "new": new, "drop": rng.choice([0, new - 1 if new < 10 else 0]) if longest else 0,
                     "longest": longest, "finished": rng.choice([0.0, 0.0, 0.05])}
        if all(a <= b for a, b in zip(_cost(case), most[op])):
            return case


def sizes(case):
    """Rows of each sequence: spread evenly over their range where the case is ragged."""
    return [max(1, round(case["chunk"] * (1.0 - 0.95 * ((b * 0.6180339887498949) % 1.0)))) if case["ragged"] else case["chunk"] for b in range(case["batch"])]


def requests(case):
    """(cached, dropped, new) tokens of each sequence of a plan."""
    got = []
    for b in range(case["batch"]):
        f, h = (b * 0.6180339887498949) % 1.0, (b * 0.7548776662466927) % 1.0
        long = round(case["longest"] * (1.0 - 0.95 * f))
        if h < case["finished"]:
            got.append((long, long, 0))
        else:
            got.append((long, min(long, round(case["drop"] * h)), case["new"] if case["new"] < 10 else max(1, round(case["new"] * (1.0 - 0.9 * f)))))
    return got


def work(case):
    size = {"float32": 4}.get(case.get("dtype"), 2)
    if case["op"] in ("encode", "product"):
        n = case["rows"] * case["cols"]
        packed = n // 2 + 2 * case["rows"] * -(-case["cols"] // case["group"])
        if case["op"] == "encode":  # and expanded to the same type
            return {"bytes": n * size + 2 * packed + n * size, "flops": 10 * n}
        m = case["tokens"]
        return {"bytes": packed + m * case["cols"] * size + m * case["rows"] * (4 if case["out"] == "float32" else 2) + 4 * case["rows"] * case["bias"], "flops": 2 * m * n}
    if case["op"] == "verify":  # one row of probabilities per sequence, and the draft's
        rows, n = sum(sizes(case)), case["batch"] * case["vocab"]
        return {"bytes": n * size * (1 + case["draft"]) + rows * (8 + 4 + 8 + 2 * size) + case["batch"] * 16, "flops": 2 * n}
    moved = new = 0
    for long, drop, n in requests(case):
        had, wanted = -(-long // case["page"]), -(-(long - drop + n) // case["page"])
        moved += abs(wanted - had)
        new += n
    return {"bytes": 16 * new + 8 * moved + 24 * case["batch"], "flops": 4 * new + 8 * case["batch"]}


# ---------------------------------------------------------------- the 4-bit format, from its definition


def _compress(w, group):
    """Codes [row tiles, column tiles, 1024] and scales [row tiles, column tiles, 16, 128 / group] of w [rows, cols] (any type).

    A tile has 16 rows and 128 columns, 16 bytes at a time: piece 16 g + n holds of row n four words, word s the columns 32 s + 8 g .. + 7,
    four bits each from the lowest on: sign, index of the magnitude."""
    rows, cols = w.shape
    nt, kt = -(-rows // 16), -(-cols // 128)
    full = torch.zeros((nt * 16, kt * 128), dtype=torch.float32, device=w.device)
    full[:rows, :cols] = w.float()
    x = full.view(nt * 16, -1, group)
    most = x.abs().amax(-1)
    s = (most / torch.full_like(most, 6.0)).to(torch.bfloat16).float().clamp(max=TOP).unsqueeze(-1)  # (a tensor: a quotient, not a product)
    code = torch.zeros(x.shape, dtype=torch.uint8, device=w.device)
    for t in BORDERS:
        code += x.abs() > s * t
    code = torch.where(s > 0, code, 0) + torch.signbit(x).to(torch.uint8) * 8
    bad = ~torch.isfinite(most).unsqueeze(-1)
    code = torch.where(bad, 0, code).to(torch.uint8)
    s = torch.where(bad, math.nan, s).squeeze(-1)
    c = code.view(nt, 16, kt, 4, 4, 4, 2)  # row tile, n, column tile, s, g, byte, half
    c = (c[..., 0] + c[..., 1] * 16).permute(0, 2, 4, 1, 3, 5).contiguous()
    return c.view(nt, kt, 1024), s.to(torch.bfloat16).view(nt, 16, kt, 128 // group).transpose(1, 2).contiguous()


def _expand(codes, scales, rows, cols):
    """The values, in float32."""
    nt, kt = codes.shape[:2]
    table = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], dtype=torch.float32, device=codes.device)
    c = codes.view(nt, kt, 4, 16, 4, 4).permute(0, 3, 1, 4, 2, 5)
    v = table[torch.stack([c & 15, c >> 4], -1).reshape(nt * 16, -1).int()]
    s = scales.float().transpose(1, 2).reshape(nt * 16, -1)
    return (v.view(s.shape[0], s.shape[1], -1) * s.unsqueeze(-1)).view(nt * 16, -1)[:rows, :cols]


# ---------------------------------------------------------------- inputs


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    state = {"case": case}
    if case["op"] in ("encode", "product"):
        rows, cols = case["rows"], case["cols"]

        def weights(n):  # rows of unequal size, some large ones among them
            return torch.randn(n, cols, generator=g, device=dev).mul_(torch.exp(0.3 * torch.randn(n, 1, generator=g, device=dev)) * cols ** -0.5)

        if case["op"] == "encode":
            return state | {"w": weights(rows).to(DTYPES[case["dtype"]])}
        step = max(16, (1 << 25) // cols // 16 * 16)
        parts = [_compress(weights(min(step, rows - at)), case["group"]) for at in range(0, rows, step)]
        x = torch.randn(case["tokens"], cols, generator=g, device=dev).mul_(torch.exp(0.5 * torch.randn(cols, generator=g, device=dev)))
        return state | {"codes": torch.cat([c for c, _ in parts]), "scales": torch.cat([s for _, s in parts]), "x": x.to(DTYPES[case["dtype"]]),
                        "bias": torch.randn(rows, generator=g, device=dev) if case["bias"] else None}
    if case["op"] == "verify":
        each = sizes(case)
        rows, vocab, dt = sum(each), case["vocab"], DTYPES[case["dtype"]]
        target = torch.empty((rows, vocab), dtype=dt, device=dev)
        draft = torch.empty((rows, vocab), dtype=dt, device=dev) if case["draft"] else None
        tokens = torch.empty(rows, dtype=torch.int64, device=dev)
        tokens[0] = 0
        step = max(1, (1 << 26) // vocab)
        for at in range(0, rows, step):
            logits = 3.0 * torch.randn(min(step, rows - at), vocab, generator=g, device=dev)
            p = torch.softmax(logits, 1)
            q = torch.softmax(logits + 0.7 * torch.randn(logits.shape, generator=g, device=dev), 1)
            target[at : at + step] = p.to(dt)
            if draft is not None:
                draft[at : at + step] = q.to(dt)
            # what row j proposes stands in row j + 1
            proposed = torch.multinomial(q, 1, generator=g).squeeze(1) if draft is not None else q.argmax(1)
            n = min(proposed.shape[0], rows - 1 - at)
            tokens[at + 1 : at + 1 + n] = proposed[:n]
        starts = [0]
        for n in each:
            starts.append(starts[-1] + n)
        return state | {"target": target, "draft": draft, "tokens": tokens, "uniform": torch.rand(rows, generator=g, device=dev),
                        "sample": torch.rand(case["batch"], generator=g, device=dev), "starts": torch.tensor(starts, dtype=torch.int32, device=dev),
                        "even": not case["ragged"]}
    page = case["page"]
    lens, drop, new = (list(v) for v in zip(*requests(case)))
    had = [-(-n // page) for n in lens]
    wanted = [-(-(n - d + m) // page) for n, d, m in zip(lens, drop, new)]
    wide, pool = max(max(had), max(wanted)) + 2, sum(max(h, w) for h, w in zip(had, wanted)) + 5
    order = torch.randperm(pool, generator=g, device=dev).to(torch.int32)
    pages = torch.zeros((case["batch"], wide), dtype=torch.int32, device=dev)
    index = torch.arange(wide, device=dev)
    count = torch.tensor(had, device=dev)
    pages[index < count[:, None]] = order[: sum(had)]
    free = torch.zeros(pool, dtype=torch.int32, device=dev)
    free[: pool - sum(had)] = order[sum(had) :]
    t32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    return state | {"lens": t32(lens), "drop": t32(drop) if any(drop) else None, "new": t32(new), "pages": pages, "free": free,
                    "n_free": t32([pool - sum(had)]), "total": sum(new) + (sum(new) % 3)}


# ---------------------------------------------------------------- one pass


def run(state):
    return {"encode": _encode, "product": _product, "verify": _verify, "plan": _plan}[state["case"]["op"]](state)


def _encode(st):
    case, w = st["case"], st["w"]
    if own:
        from paper_1511_04561_amd import dq8
        codes, scales = dq8.weights_encode(w, group=case["group"])
        return {"values": dq8.weights_decode(codes, scales, rows=case["rows"], cols=case["cols"], dtype=w.dtype), "scales": scales}
    codes, scales = _compress(w, case["group"])
    return {"values": _expand(codes, scales, case["rows"], case["cols"]).to(w.dtype), "scales": scales}


def _product(st):
    case, x = st["case"], st["x"]
    if own:
        from paper_1511_04561_amd import dq8
        return dq8.weights_product(x, st["codes"], st["scales"], rows=case["rows"], bias=st["bias"], dtype=DTYPES[case["out"]])
    w = _expand(st["codes"], st["scales"], case["rows"], case["cols"])
    y = torch.matmul(x.float(), w.T)
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(DTYPES[case["out"]])


def _verify(st):
    case, p, q, tokens = st["case"], st["target"], st["draft"], st["tokens"]
    if own:
        from paper_1511_04561_amd import dq8
        out, accepted, rejected = dq8.draft_verify(p, tokens, st["uniform"], st["sample"], starts=None if st["even"] else st["starts"], draft=q)
        return {"out": out, "accepted": accepted, "rejected": rejected}
    rows, vocab, dev = p.shape[0], case["vocab"], p.device
    begin, end = st["starts"][:-1].long(), st["starts"][1:].long()
    # row j: whether the token of row j + 1 is accepted
    following = torch.cat([tokens[1:], tokens[:1]])
    known = (following >= 0) & (following < vocab)
    at = following.clamp(0, vocab - 1).unsqueeze(1)
    pd = _weight(p.gather(1, at)).squeeze(1)
    qd = _weight(q.gather(1, at)).squeeze(1) if q is not None else torch.ones(rows, dtype=torch.float64, device=dev)
    accept = known & (st["uniform"].double() * qd < pd)
    row = torch.arange(rows, device=dev)
    owner = torch.searchsorted(end, row, right=True)
    stop = torch.where(accept & (row + 1 < end[owner]), rows, row)  # rows at which a sequence may end
    first = torch.full((case["batch"],), rows, dtype=torch.int64, device=dev).scatter_reduce(0, owner, stop, "amin")
    refused = first + 1 < end
    w = _weight(p[first])
    if q is not None:
        less = torch.where(refused[:, None], (w - _weight(q[first])).clamp(min=0.0), w)
    else:
        t = following[first]
        less = torch.where(refused[:, None] & (torch.arange(vocab, device=dev) == t[:, None]), 0.0, w)
    w = torch.where(less.sum(1, keepdim=True) > 0, less, w)
    r = torch.nan_to_num(st["sample"].double(), nan=0.0).clamp(min=0.0)
    total = w.sum(1, keepdim=True)
    over = (w.cumsum(1) > r[:, None] * total) & (w > 0)
    last = vocab - 1 - (w > 0).flip(1).to(torch.uint8).argmax(1)
    token = torch.where(over.any(1), over.to(torch.uint8).argmax(1), last)
    token = torch.where(total.squeeze(1) > 0, token, -1)
    out = torch.where(row < first[owner], following, torch.where(row == first[owner], token[owner], -1))
    accepted = first - begin
    return {"out": out, "accepted": accepted.int(), "rejected": (end - 1 - first).int()}


def _weight(v):
    """Probabilities in binary64; what is no positive number counts as none."""
    v = v.double()
    return torch.where((v > 0) & torch.isfinite(v), v, 0.0)


def _plan(st):
    case, page, total = st["case"], st["case"]["page"], st["total"]
    lens, new, drop, pages, free, n_free = (st[k] for k in ("lens", "new", "drop", "pages", "free", "n_free"))
    if own:
        from paper_1511_04561_amd import dq8
        slots, positions, starts, lens_out, granted, left = dq8.cache_plan(lens, new, pages, free, n_free, page, total, drop=drop)
        return {"slots": slots, "positions": positions, "starts": starts, "lens": lens_out, "granted": granted, "n_free": left, "pages": pages, "free": free}
    dev, batch, wide = lens.device, case["batch"], pages.shape[1]
    had_len = lens.long().clamp(0, wide * page)
    n = new.long().clamp(min=0)
    kept = had_len if drop is None else (had_len - drop.long().clamp(min=0)).clamp(min=0)
    ends = n.cumsum(0)
    fits = (kept + n <= wide * page) & (ends <= total)
    had = (had_len + page - 1) // page
    wanted = torch.where(fits, (kept + n + page - 1) // page, had)
    gone, needs = (had - wanted).clamp(min=0), (wanted - had).clamp(min=0)
    have = n_free.long().clamp(0, free.shape[0])
    room = free.shape[0]
    index = torch.arange(wide, device=dev)
    # pages given back, behind the free ones in the order of the sequences
    back = (index >= wanted[:, None]) & (index < had[:, None])
    place = have + (gone.cumsum(0) - gone)[:, None] + index - wanted[:, None]
    more = torch.cat([free, free.new_zeros(1)])  # the last place is for what is not stored
    more.scatter_(0, torch.where(back, place, room).clamp(max=room).view(-1), pages.reshape(-1))
    free.copy_(more[:room])
    stock = (have + gone.sum()).clamp(max=room)
    # pages taken, from the last one on
    upto = needs.cumsum(0)
    ok = fits & ((needs == 0) | (upto <= stock))
    take = (index >= had[:, None]) & (index < wanted[:, None]) & ok[:, None]
    place = stock - 1 - (upto - needs)[:, None] - index + had[:, None]
    pages.copy_(torch.where(take, free[place.clamp(0, room - 1)], pages))
    granted = torch.where(ok, n, -1)
    lens_out = torch.where(ok, kept + n, had_len)
    t = torch.arange(total, device=dev)
    b = torch.searchsorted(ends, t, right=True)
    inside = b < batch
    b = b.clamp(max=batch - 1)
    position = kept[b] + t - (ends - n)[b]
    inside &= ok[b]
    position = torch.where(inside, position, -1)
    entry = position.clamp(min=0)
    slot = pages[b, entry // page].long() * page + entry % page
    starts = torch.cat([ends.new_zeros(1), ends]).clamp(max=total)
    return {"slots": torch.where(inside, slot, -1), "positions": position, "starts": starts.int(), "lens": lens_out.int(), "granted": granted.int(),
            "n_free": (stock - take.sum()).int(), "pages": pages, "free": free}


# ---------------------------------------------------------------- the operators in binary64


def exact(case, seed):
    if case["op"] in ("verify", "plan"):
        return None  # whole numbers
    st = prepare(case, seed)
    if case["op"] == "product":
        y = torch.empty((case["tokens"], case["rows"]), dtype=torch.float64, device=st["x"].device)
        x = st["x"].double()
        for at in range(0, case["rows"], 2048):
            upto = min(at + 2048, case["rows"])
            y[:, at:upto] = x @ _rows64(st["codes"], st["scales"], at // 16, -(-upto // 16), case["group"])[: upto - at, : case["cols"]].T.contiguous()
        return y if st["bias"] is None else y + st["bias"].double()
    w, group = st["w"], case["group"]
    rows, cols = w.shape
    nt, kt = -(-rows // 16), -(-cols // 128)
    values = torch.empty((rows, cols), dtype=torch.float64, device=w.device)
    scales = torch.zeros((nt * 16, kt * 128 // group), dtype=torch.float64, device=w.device)
    for at in range(0, cols, group):
        x = w[:, at : at + group].double()
        most = x.abs().amax(1)
        s = (most / torch.full_like(most, 6.0)).float().bfloat16().double()
        far = torch.stack([(x.abs() - m * s[:, None]).abs() for m in MAGNITUDES], -1)
        near = torch.tensor(MAGNITUDES, dtype=torch.float64, device=w.device)[far.argmin(-1)]  # of two as near the first, the smaller
        values[:, at : at + group] = torch.sign(x) * near * s[:, None]
        scales[:rows, at // group] = s
    return {"values": values, "scales": scales.view(nt, 16, kt, -1).transpose(1, 2).contiguous()}


def _rows64(codes, scales, first, last, group):
    """Rows of tiles first .. last - 1 in binary64: sign, two bits of exponent, one of mantissa."""
    c = codes[first:last].to(torch.int64)
    nt, kt = c.shape[:2]
    got = torch.empty((nt, 16, kt, 128), dtype=torch.float64, device=c.device)
    for half in range(2):
        bits = (c >> (4 * half)) & 15
        exponent, mantissa = (bits >> 1) & 3, (bits & 1).double() / 2
        v = torch.where(exponent == 0, mantissa, (1 + mantissa) * torch.exp2((exponent - 1).double()))
        v = torch.where(bits >= 8, -v, v).view(nt, kt, 4, 16, 4, 4)
        for piece in range(4):
            for word in range(4):
                k = 32 * word + 8 * piece + half
                got[..., k : k + 8 : 2] = v[:, :, piece, :, word].transpose(1, 2)
    s = scales[first:last].double().transpose(1, 2)  # row tile, n, column tile, group
    return (got.view(nt, 16, kt, -1, group) * s.unsqueeze(-1)).view(nt * 16, kt * 128)
