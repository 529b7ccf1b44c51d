"""The operators over a paged key/value cache: their plain forms in torch, the cases they are measured on, and their values in
64 bits.

A cache holds, for every page of `page` tokens and every key/value head, the keys and values of those tokens, in 16 bits or in 8
bits with one scale for each token and head, and bounds of the page's keys (the largest and the smallest value of every channel, in
8 bits with one scale).  Sequences reach their pages through a table.  The passes:

  append  new tokens' keys and values are written into their pages, and read back with the bounds of the pages that they touched
  read    the tokens of a batch are read back
  attend  the new tokens' queries attend to their sequence's keys up to their own position
  sparse  every query picks the blocks (pages) whose bounds promise the largest scores, and attends to those alone
"""
import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LARGEST = {"i8": 127.0, "f8": 448.0}  # codes are scaled to it
SLACK = 2.0 ** -10  # of a step: a bound that 32 bits put this little beyond a whole number is that number
SIDES = {"i8": 1, "f8": 1, "f16": 2, "bf16": 2}


def listed():
    return [
        # One step of a decoding batch: every sequence writes one token, mostly into a page that holds others.
        _case("append: a token each", "append", storage="i8", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=64, new=1, length=8192),
        # Prompts cut into chunks by a scheduler: three sequences, chunks that begin and end inside pages.
        _case("append: ragged chunks", "append", storage="f8", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=3, new=4001, length=9001),
        # A long document that an agent reads at once.
        _case("append: a long prompt", "append", storage="i8", dtype="f16", heads=8, group=4, dim=128, page=64, seqs=1, new=65536, length=65536),
        # A short memory is taken out of the cache, to be moved into another one.
        _case("read: one short sequence", "read", storage="i8", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=1, new=1000, length=1000),
        # A long context leaves the cache whole.
        _case("read: a long context", "read", storage="f8", dtype="f16", heads=8, group=4, dim=128, page=64, seqs=1, new=131071, length=131071),
        # One agent answers alone: the smallest call, where latency is what counts.
        _case("attend: one token", "attend", storage="bf16", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=1, new=1, length=1025),
        # A decoding batch over contexts of all lengths.
        _case("attend: a token each", "attend", storage="i8", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=48, new=1, length=32768),
        # A step that mixes a prompt's chunk with short drafts of other sequences; odd heads, small pages.
        _case("attend: mixed chunks", "attend", storage="f8", dtype="f16", heads=3, group=5, dim=64, page=16, seqs=16, new=777, length=8191),
        # A chunk of a long prompt over what came before it.
        _case("attend: a long chunk", "attend", storage="bf16", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=1, new=4096, length=32768),
        # One agent with a long memory answers alone.
        _case("sparse: one token", "sparse", storage="f16", dtype="f16", heads=8, group=4, dim=128, page=64, seqs=1, new=1, length=20001, blocks=16),
        # A decoding batch over very long contexts, of which every query reads a small part.
        _case("sparse: a token each", "sparse", storage="i8", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=16, new=1, length=131072, blocks=64),
        # A chunk of a long prompt, every token with blocks of its own.
        _case("sparse: a chunk", "sparse", storage="i8", dtype="bf16", heads=8, group=4, dim=128, page=64, seqs=1, new=1024, length=32768, blocks=32),
    ]


def _case(name, op, *, storage, dtype, heads, group, dim, page, seqs, new, length, window=0, blocks=0):
    c = {"op": op, "storage": storage, "dtype": dtype, "heads": heads, "group": group, "dim": dim, "page": page, "seqs": seqs,
         "new": new, "length": length, "window": window, "blocks": blocks}
    return {"name": name, **c} if name else c


def draw(rng):
    def spread(low, high):
        return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))

    while True:
        op = rng.choice(["append", "read", "attend", "attend", "sparse", "sparse"])
        storage = rng.choice(["f16", "bf16", "i8", "i8", "f8"])
        dtype = storage if storage in TYPES else rng.choice(["f16", "bf16"])
        tokens = rng.random() < 0.5 and op != "read"
        length = spread(1, 131072)
        c = _case("", op, storage=storage, dtype=dtype, heads=rng.choice([1, 2, 3, 4, 5, 8, 8, 16]), group=rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16]),
                  dim=rng.choice([64, 64, 80, 96, 128, 128, 128, 256]), page=rng.choice([16, 32, 64, 64, 128]), seqs=spread(1, 64), new=1 if tokens else spread(1, min(length, 16384)),
                  length=length, window=rng.choice([0, 0, 0, spread(16, 8192)]) if op == "attend" else 0, blocks=spread(4, 64) if op == "sparse" else 0)
        news, lens = _lengths(c)
        w = work(c)
        # what the plain form holds: the padded scores, or the rows that the queries gather; and the cache itself
        rows = sum(news) * c["blocks"] * c["page"] if op == "sparse" else c["seqs"] * max(lens)
        scores = c["heads"] * c["group"] * (sum(news) * c["blocks"] * c["page"] if op == "sparse" else c["seqs"] * max(news) * max(lens) if op == "attend" else 0)
        rows = max(rows, sum(m * -(-max(lens) // c["page"]) for m in news) if op == "sparse" else 0)  # the bounds that they gather
        held = sum(lens) * c["heads"] * c["dim"]
        if scores <= 2 ** 31 and rows * c["heads"] * c["dim"] <= 2 ** 31 and held <= 2 ** 31 and w["bytes"] <= 8e8 and w["flops"] <= 1.5e12:
            return c


def _lengths(case):
    """New tokens and length (the new ones included) of every sequence: the first has the most of both, the others less, evenly over the logarithm."""
    r = random.Random("%(seqs)d %(new)d %(length)d %(page)d" % case)
    news = [case["new"]] + [max(1, int(case["new"] ** r.random())) for _ in range(case["seqs"] - 1)]
    lens = [case["length"]] + [max(n, int(case["length"] * 16 ** -r.random())) for n in news[1:]]
    return [min(n, case["length"]) for n in news], lens


def work(case):
    news, lens = _lengths(case)
    h, g, d, p = case["heads"], case["group"], case["dim"], case["page"]
    row = 2 * h * (d * SIDES[case["storage"]] + (4 if case["storage"] in LARGEST else 0))  # a token's keys and values
    n, side, bound = sum(news), 2 * h * d * 2, h * (2 * d + 4)
    if case["op"] == "append":
        touched = sum((l - 1) // p - (l - m) // p + 1 for m, l in zip(news, lens))
        return {"bytes": n * (2 * side + 2 * row) + touched * (bound + 2 * h * d * 4), "flops": 8 * n * h * d}
    if case["op"] == "read":
        return {"bytes": n * (row + side), "flops": 2 * n * h * d}
    if case["op"] == "attend":
        w = case["window"] or case["length"]
        # keys that a query at position l - m + i sees: min(l - m + i + 1, w)
        full = [max(0, min(m, l - w + 1)) for m, l in zip(news, lens)]
        pairs = sum(f * w + (m - f) * (2 * (l - m) + (m - f) + 1) // 2 for f, m, l in zip(full, news, lens))
        return {"bytes": sum(min(l, m + w - 1) for m, l in zip(news, lens)) * row + 2 * n * h * g * d * 2, "flops": 4 * d * h * g * pairs}
    kept = [min(case["blocks"], -(-l // p)) for l in lens]  # blocks of a query at most
    pages = sum(-(-l // p) for l in lens)
    seen = sum(min(l * h, m * h * b * p) for b, m, l in zip(kept, news, lens)) * row // h
    pairs = sum(m * b * p for b, m in zip(kept, news))
    return {"bytes": seen + pages * bound + 2 * n * h * g * d * 2 + n * h * case["blocks"] * 4,
            "flops": 4 * d * h * g * (pairs + sum(m * -(-l // p) for m, l in zip(news, lens)))}


def _rows(case, seed, count, lens):
    """Keys and values of `count` tokens: channels of unequal size, runs of tokens that resemble one another, and a few large ones."""
    gen = torch.Generator("cuda").manual_seed(seed)
    h, d, kind = case["heads"], case["dim"], TYPES[case["dtype"]]
    size = torch.exp(0.5 * torch.randn(h, d, device="cuda", generator=gen))
    run = torch.arange(count, device="cuda") // 96
    topics = torch.randn(count // 96 + 1, h, d, device="cuda", generator=gen) * size
    k, v = torch.empty(count, h, d, device="cuda", dtype=kind), torch.empty(count, h, d, device="cuda", dtype=kind)
    for at in range(0, count, 1 << 18):
        part = slice(at, min(count, at + (1 << 18)))
        k[part] = topics[run[part]] + 0.7 * torch.randn(k[part].shape, device="cuda", generator=gen)
        v[part] = torch.randn(k[part].shape, device="cuda", generator=gen) * torch.exp(0.3 * torch.randn(k[part].shape[0], h, 1, device="cuda", generator=gen))
    return k, v, topics, gen


def prepare(case, seed):
    """The cache with everything but the new tokens in it (for reading and attending: with them), the batch's plan, and the step's rows."""
    news, lens = _lengths(case)
    h, g, d, p, kind = case["heads"], case["group"], case["dim"], case["page"], TYPES[case["dtype"]]
    n, count = sum(news), sum(lens)
    k, v, topics, gen = _rows(case, seed, count, lens)
    pages = [-(-l // p) for l in lens]
    tables = torch.zeros(len(lens), max(pages), dtype=torch.int32)
    order = torch.randperm(sum(pages), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    for i, (m, part) in enumerate(zip(pages, torch.split(order, pages))):
        tables[i, :m] = part
    s = {"op": case["op"], "window": case["window"], "blocks": case["blocks"], "scale": d ** -0.5, "kind": kind}
    whole = torch.tensor([0] + lens).cumsum(0).to("cuda", torch.int32)
    s["batch"] = b = {"tables": tables.cuda(), "offsets": torch.tensor([0] + news).cumsum(0).to("cuda", torch.int32), "lens": torch.tensor(lens, dtype=torch.int32).cuda(),
                      "n_tokens": n, "max_new": max(news), "max_len": max(lens)}
    new = _tokens(b)  # where the new tokens lie among all of them
    at = whole[new["seq"]].long() + new["pos"]
    # the step's rows are parts of one product, as a model's layer gives them
    near = topics[torch.randint(0, topics.shape[0], (n,), device="cuda", generator=gen)].repeat_interleave(g, 1)
    fused = torch.empty(n, h * (g + 2), d, dtype=kind, device="cuda")
    fused[:, :h * g] = 0.6 * near + torch.randn(n, h * g, d, device="cuda", generator=gen)
    fused[:, h * g:h * (g + 1)], fused[:, h * (g + 1):] = k[at], v[at]
    s["q"], s["k"], s["v"] = fused[:, :h * g], fused[:, h * g:h * (g + 1)], fused[:, h * (g + 1):]
    held = {**b, "offsets": whole, "n_tokens": count, "max_new": max(lens)}
    if case["op"] == "append":  # the tokens before the new ones
        before = [l - m for l, m in zip(lens, news)]
        keep = torch.ones(count, dtype=torch.bool, device="cuda")
        keep[at] = False
        k, v = k[keep], v[keep]
        held = {**b, "offsets": torch.tensor([0] + before).cumsum(0).to("cuda", torch.int32), "lens": torch.tensor(before, dtype=torch.int32).cuda(), "n_tokens": count - n, "max_new": max(before)}
        first, last = (b["lens"] - b["offsets"].diff()) // p, (b["lens"] - 1) // p
        column = torch.arange(max(pages), device="cuda")
        s["touched"] = b["tables"][(column >= first[:, None]) & (column <= last[:, None])]
    if own:
        from paper_2602_21477_amd import binding as B
        s["batch"] = B.KVBatch(**b)
        s["cache"] = B.KVCache(sum(pages), h, d, storage={"f16": B.PK_F16, "bf16": B.PK_BF16, "i8": B.PK_I8, "f8": B.PK_F8}[case["storage"]], page_tokens=p)
        if held["n_tokens"]:
            s["cache"].append(k, v, B.KVBatch(**held))
        return s
    s["cache"] = c = {"storage": case["storage"], "k": torch.zeros(sum(pages), p, h, d, device="cuda", dtype=_held(case)), "hi": torch.zeros(sum(pages), h, d, device="cuda", dtype=torch.int8)}
    c["v"], c["lo"] = torch.zeros_like(c["k"]), torch.zeros_like(c["hi"])
    c["ks"], c["vs"] = (torch.ones(sum(pages), p, h, 1, device="cuda") for _ in range(2))
    c["bs"], c["fill"] = torch.zeros(sum(pages), h, 1, device="cuda"), torch.zeros(sum(pages), device="cuda", dtype=torch.long)
    if held["n_tokens"]:
        _append(c, k, v, held)
        for part in torch.split(torch.arange(sum(pages), device="cuda"), 4096):
            _bound(c, part)
    return s


def _held(case):
    return {"i8": torch.int8, "f8": torch.float8_e4m3fn}.get(case["storage"], TYPES[case["dtype"]])


def run(s):
    if own:
        c, b = s["cache"], s["batch"]
        if s["op"] == "append":
            c.append(s["k"], s["v"], b)
            return {"kv": c.read(b, s["kind"]), "bounds": c.bounds(s["touched"])}
        if s["op"] == "read":
            return {"kv": c.read(b, s["kind"])}
        if s["op"] == "attend":
            return c.attend(s["q"], b, s["scale"], window=s["window"], want_lse=True)
        blocks = c.select(s["q"], b, s["blocks"])
        return {"blocks": blocks, "out": c.attend_blocks(s["q"], blocks, b, s["scale"])}
    c, b = s["cache"], s["batch"]
    if s["op"] == "append":
        _append(c, s["k"], s["v"], b)
        _bound(c, s["touched"].long())
        return {"kv": _read(c, b, s["kind"]), "bounds": (c["hi"][s["touched"]] * c["bs"][s["touched"]], c["lo"][s["touched"]] * c["bs"][s["touched"]])}
    if s["op"] == "read":
        return {"kv": _read(c, b, s["kind"])}
    if s["op"] == "attend":
        return _attend(c, s["q"], b, s["scale"], s["window"])
    blocks = _select(c, s["q"], b, s["blocks"])
    return {"blocks": blocks, "out": _attend_blocks(c, s["q"], blocks, b, s["scale"])}


def _tokens(b):
    """Sequence and position of every new token of a batch."""
    news = b["offsets"].diff().long()
    seq = torch.repeat_interleave(torch.arange(news.shape[0], device="cuda"), news, output_size=b["n_tokens"])
    index = torch.arange(b["n_tokens"], device="cuda") - b["offsets"][seq]
    return {"seq": seq, "index": index, "pos": b["lens"][seq].long() - news[seq] + index}


def _quantised(x, storage, kind):
    """Codes and scales: one scale for each token and head."""
    x = x.float()
    if storage not in LARGEST:
        return x.to(kind), torch.ones_like(x[..., :1])
    most = x.abs().amax(-1, keepdim=True)
    up = torch.where(most > 0, torch.full_like(most, LARGEST[storage]) / most, torch.zeros_like(most)).clamp(max=3.0e38)
    y = (x * up).clamp(-LARGEST[storage], LARGEST[storage])
    return (y.round() if storage == "i8" else y).to(kind), most * (1.0 / LARGEST[storage])


def _append(c, k, v, b):
    t = _tokens(b)
    page = c["k"].shape[1]
    at = b["tables"][t["seq"], t["pos"] // page].long(), t["pos"] % page
    for x, codes, scales in ((k, "k", "ks"), (v, "v", "vs")):
        c[codes][at], c[scales][at] = _quantised(x, c["storage"], c["k"].dtype)
    c["fill"].index_reduce_(0, at[0], at[1] + 1, "amax")


def _bound(c, pages):
    """The bounds of pages, from the rows that they hold."""
    rows = c["k"][pages].float() * c["ks"][pages]
    out = (torch.arange(rows.shape[1], device="cuda") >= c["fill"][pages][:, None])[:, :, None, None]
    hi, lo = rows.masked_fill(out, -math.inf).amax(1), rows.masked_fill(out, math.inf).amin(1)
    none = torch.isinf(hi)
    hi, lo = hi.masked_fill(none, 0.0), lo.masked_fill(none, 0.0)
    most = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
    up = torch.where(most > 0, torch.full_like(most, 127.0) / most, torch.zeros_like(most)).clamp(max=3.0e38)
    c["hi"][pages], c["lo"][pages] = (hi * up - SLACK).ceil().clamp(-127, 127).to(torch.int8), (lo * up + SLACK).floor().clamp(-127, 127).to(torch.int8)
    c["bs"][pages] = most * (1.0 / 127.0)


def _read(c, b, kind):
    t = _tokens(b)
    page = c["k"].shape[1]
    at = b["tables"][t["seq"], t["pos"] // page].long(), t["pos"] % page
    return (c["k"][at].float() * c["ks"][at]).to(kind), (c["v"][at].float() * c["vs"][at]).to(kind)


def _softmax(scores, mask):
    """Weights, and the logarithm of what they were divided by: none and -inf for a row without keys."""
    scores = scores.masked_fill(~mask, -math.inf)
    most = scores.amax(-1, keepdim=True).clamp(min=-3.0e38)
    weights = torch.exp(scores - most)
    total = weights.sum(-1, keepdim=True)
    return weights / total.clamp(min=1e-37), (most + torch.log(total)).squeeze(-1)


def _attend(c, q, b, scale, window):
    """Every sequence padded to the longest, its pages side by side."""
    t, (n, hq, d) = _tokens(b), q.shape
    seqs, page, h = b["lens"].shape[0], c["k"].shape[1], c["k"].shape[2]
    keys, values = ((c[x][b["tables"].long()].float() * c[y][b["tables"].long()]).flatten(1, 2).permute(0, 2, 3, 1) for x, y in (("k", "ks"), ("v", "vs")))
    rows = torch.zeros(seqs, b["max_new"], hq, d, device="cuda")
    rows[t["seq"], t["index"]] = q.float()
    rows = rows.view(seqs, b["max_new"], h, hq // h, d).permute(0, 2, 3, 1, 4).reshape(seqs, h, -1, d)
    scores = torch.matmul(rows, keys.contiguous()).mul_(scale).view(seqs, h, hq // h, b["max_new"], -1)
    pos = (b["lens"] - b["offsets"].diff())[:, None] + torch.arange(b["max_new"], device="cuda")
    key = torch.arange(scores.shape[-1], device="cuda")
    mask = (key <= pos[:, :, None]) & (key > pos[:, :, None] - (window or 1 << 30))
    weights, lse = _softmax(scores, mask[:, None, None])
    out = torch.matmul(weights.view(seqs, h, -1, weights.shape[-1]), values.transpose(2, 3).contiguous()).view(seqs, h, hq // h, b["max_new"], d)
    out, lse = out.permute(0, 3, 1, 2, 4)[t["seq"], t["index"]], lse.permute(0, 3, 1, 2)[t["seq"], t["index"]]
    return out.reshape(n, hq, d).to(q.dtype), lse.reshape(n, hq)


def _select(c, q, b, blocks):
    t, (n, hq, d) = _tokens(b), q.shape
    h = c["k"].shape[2]
    codes, scales = _quantised(q, "i8", torch.int8)
    codes, table = codes.float().view(n, h, hq // h, d), b["tables"].long()
    hi, lo = (c[x][table][t["seq"]].float().permute(0, 2, 3, 1).contiguous() for x in ("hi", "lo"))  # [token, head, channel, block]
    bound = torch.matmul(codes.clamp(min=0), hi) + torch.matmul(codes.clamp(max=0), lo)  # whole numbers below 2^24
    score = (bound * scales.view(n, h, -1, 1)).amax(2) * c["bs"][table][t["seq"]].squeeze(-1).transpose(1, 2)
    block, mine = torch.arange(table.shape[1], device="cuda"), (t["pos"] // c["k"].shape[1])[:, None, None]
    score = score.masked_fill((block < 1) | (block > mine - 2), math.inf).masked_fill(block > mine, -math.inf)  # the first block and the last two always
    score, order = torch.sort(score, dim=-1, descending=True, stable=True)
    order = order.masked_fill(torch.isneginf(score), 1 << 30)[..., :blocks].sort(-1).values
    order = torch.nn.functional.pad(order, (0, blocks - order.shape[-1]), value=1 << 30)
    return order.masked_fill(order == 1 << 30, -1).to(torch.int32)


def _attend_blocks(c, q, blocks, b, scale):
    t, (n, hq, d) = _tokens(b), q.shape
    page, h = c["k"].shape[1], c["k"].shape[2]
    pages, head = b["tables"][t["seq"][:, None, None], blocks.clamp(min=0).long()].long(), torch.arange(h, device="cuda")[:, None]
    keys, values = ((c[x].transpose(1, 2)[pages, head].float() * c[y].transpose(1, 2)[pages, head]).flatten(2, 3) for x, y in (("k", "ks"), ("v", "vs")))
    scores = torch.matmul(q.float().view(n, h, hq // h, d), keys.transpose(2, 3).contiguous()).mul_(scale)
    key = (blocks[..., None] * page + torch.arange(page, device="cuda")).flatten(2)
    mask = (key <= t["pos"][:, None, None]) & (blocks >= 0).repeat_interleave(page, -1)
    weights, _ = _softmax(scores, mask[:, :, None])
    return torch.matmul(weights, values).reshape(n, hq, d).to(q.dtype)


def exact(case, seed):
    """The same from the definitions, in 64 bits: a row's stored values are what its codes and its 32-bit scale stand for."""
    global own
    news, lens = _lengths(case)
    h, g, d, p, st = case["heads"], case["group"], case["dim"], case["page"], case["storage"]
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c, b, table = s["cache"], s["batch"], s["batch"]["tables"].long()

    def stored(x):  # [token, head, channel] as it is held
        x = x.double()
        if st not in LARGEST:
            return x
        most = x.abs().amax(-1, keepdim=True)
        y = torch.where(most > 0, x / most * LARGEST[st], torch.zeros_like(x))
        y = y.round() if st == "i8" else y.to(torch.float8_e4m3fn).double()
        return y * (most.float() * (1.0 / LARGEST[st])).double()

    def sequence(name, i):  # all rows of sequence i that the cache holds, [head, token, channel]
        m = -(-lens[i] // p)
        return (c[name][table[i, :m]].double() * c[name + "s"][table[i, :m]].double()).flatten(0, 1)[:lens[i]].transpose(0, 1)

    if case["op"] == "append":
        k, v = stored(s["k"]), stored(s["v"])
        his, los, at = [], [], 0
        for i, (m, l) in enumerate(zip(news, lens)):
            kept = sequence("k", i)
            kept[:, l - m:] = k[at:at + m].transpose(0, 1)
            at += m
            for j in range((l - m) // p, (l - 1) // p + 1):
                rows = kept[:, j * p:min(l, (j + 1) * p)]
                hi, lo = rows.amax(1), rows.amin(1)
                most = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
                unit = torch.where(most > 0, most / 127, torch.ones_like(most))
                his.append(torch.ceil(hi / unit - SLACK).clamp(-127, 127) * unit)  # the next whole number outwards
                los.append(torch.floor(lo / unit + SLACK).clamp(-127, 127) * unit)
        return {"kv": (k, v), "bounds": (torch.stack(his), torch.stack(los))}
    if case["op"] == "read":
        return {"kv": tuple(torch.cat([sequence(x, i)[:, l - m:].transpose(0, 1) for i, (m, l) in enumerate(zip(news, lens))]) for x in ("k", "v"))}
    q = s["q"].double().view(-1, h, g, d)
    out = torch.zeros(sum(news), h, g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(news), h, g), -math.inf, dtype=torch.float64, device="cuda")
    blocks = _select(c, s["q"], b, case["blocks"]) if case["op"] == "sparse" else None  # whole numbers: the definition is what they are by
    at = 0
    for i, (m, l) in enumerate(zip(news, lens)):
        keys, values = sequence("k", i), sequence("v", i)
        for j in range(0, m, 512):
            part = slice(at + j, at + min(m, j + 512))
            pos = torch.arange(l - m + j, l - m + min(m, j + 512), device="cuda")[:, None]
            for head in range(h):
                seen = torch.arange(l, device="cuda")[None] <= pos
                if case["window"]:
                    seen &= torch.arange(l, device="cuda")[None] > pos - case["window"]
                if blocks is not None:
                    chosen = torch.zeros(pos.shape[0], table.shape[1] + 1, dtype=torch.bool, device="cuda")
                    chosen.scatter_(1, blocks[part, head].long() % (table.shape[1] + 1), True)  # -1: a column beyond the table
                    seen &= chosen[:, :-1].repeat_interleave(p, 1)[:, :l]
                for member in range(g):
                    x = (q[part, head, member] @ keys[head].T) * s["scale"]
                    x = torch.where(seen, x, torch.full_like(x, -math.inf))
                    lse[part, head, member] = torch.logsumexp(x, 1)
                    out[part, head, member] = torch.exp(x - lse[part, head, member, None]) @ values[head]
        at += m
    if blocks is not None:
        return {"blocks": None, "out": out.flatten(1, 2)}
    return out.flatten(1, 2), lse.flatten(1, 2)
