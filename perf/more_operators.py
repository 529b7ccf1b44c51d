"""More operators over a paged key/value cache: their plain forms in torch, the cases they are measured on, and their values in 64 bits.

A cache holds, for every page of `page` tokens and every key/value head, the keys and values of those tokens; sequences reach their
pages through a table.  The passes:

  branch   sequences are forked: the branches share their parents' pages, get pages of their own for new tokens (a page that they
           share and write into is copied first), write those tokens, read their own pages back and are given up again
  compact  the pages in use are moved into another cache, side by side and in their order, and every sequence goes on there
  append   a cache held in 4 bits: new tokens are written, and read back with the bounds of the pages that they touched
  attend   the new tokens' queries attend to the keys, in 4 bits, of their sequence up to their own position
  sparse   every query picks the blocks (pages) whose bounds promise the largest scores, and attends to those alone, in 4 bits
  scored   attention whose scores are capped by a hyperbolic tangent or get a bias by distance, and whose masks know documents and
           a prefix that all queries see, over any storage
"""
import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LARGEST = {"i8": 127.0, "f8": 448.0, "f4": 6.0}  # codes are scaled to it
SLACK = 2.0 ** -10  # of a step: a bound that 32 bits put this little beyond a whole number is that number
BITS = {"i8": 8, "f8": 8, "f4": 4, "f16": 16, "bf16": 16}


def listed():
    return [
        # One agent tries four continuations of what it has read: the smallest call, where latency is what counts.
        _case("branch: one answer in four", "branch", storage="bf16", dtype="bf16", seqs=1, ways=4, new=5, length=1000),
        # A search over answers: every agent's context branches, each branch goes on by a token.
        _case("branch: all agents in four", "branch", storage="i8", dtype="bf16", seqs=64, ways=4, new=1, length=16384),
        # Agents have come and gone; those that are left move into a cache without holes and decode on.
        _case("compact: what is left", "compact", storage="i8", dtype="bf16", seqs=48, new=1, length=32768),
        # One step of a decoding batch over 4 bits: every sequence writes one token, mostly into a page that holds others.
        _case("append: a token each", "append", storage="f4", dtype="bf16", seqs=64, new=1, length=8192),
        # A long document that an agent reads at once.
        _case("append: a long prompt", "append", storage="f4", dtype="f16", seqs=1, new=65536, length=65536),
        # A decoding batch over contexts that need 4 bits to fit.
        _case("attend: a token each", "attend", storage="f4", dtype="bf16", seqs=48, new=1, length=65536),
        # A chunk of a long prompt over what came before it.
        _case("attend: a long chunk", "attend", storage="f4", dtype="bf16", seqs=1, new=2048, length=32768),
        # A decoding batch over very long contexts, of which every query reads a small part; odd heads.
        _case("sparse: a token each", "sparse", storage="f4", dtype="f16", heads=5, group=3, seqs=16, new=1, length=131072, blocks=64),
        # One agent answers alone with a capped model.
        _case("scored: one token", "scored", storage="bf16", dtype="bf16", seqs=1, new=1, length=4097, cap=50.0),
        # A decoding batch of a model that knows positions by distance alone.
        _case("scored: a token each", "scored", storage="i8", dtype="bf16", seqs=48, new=1, length=32768, slopes=1),
        # What a search found, read at once: documents that do not see one another, behind instructions that all see.
        _case("scored: documents", "scored", storage="bf16", dtype="bf16", seqs=1, new=16381, length=16381, docs=700, prefix=301),
        # A chunk of a long prompt with capped scores.
        _case("scored: a long chunk", "scored", storage="bf16", dtype="bf16", seqs=1, new=4096, length=32768, cap=30.0),
    ]


def _case(name, op, *, storage, dtype, seqs, new, length, heads=8, group=4, dim=128, page=64, ways=0, window=0, blocks=0, cap=0.0, slopes=0, docs=0, prefix=0):
    c = {"op": op, "storage": storage, "dtype": dtype, "heads": heads, "group": group, "dim": dim, "page": page, "seqs": seqs, "new": new, "length": length,
         "ways": ways, "window": window, "blocks": blocks, "cap": cap, "slopes": slopes, "docs": docs, "prefix": prefix}
    return {"name": name, **c} if name else c


def draw(rng):
    def spread(low, high):
        return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))

    while True:
        op = rng.choice(["branch", "branch", "compact", "append", "attend", "attend", "sparse", "scored", "scored", "scored"])
        storage = "f4" if op in ("append", "attend", "sparse") else rng.choice(["f16", "bf16", "i8", "f8", "f4"])
        dtype = storage if storage in TYPES else rng.choice(["f16", "bf16"])
        length = spread(1, 131072)
        most = {"branch": 300, "compact": 8}.get(op, 16384)
        new = 1 if rng.random() < 0.5 else spread(1, min(length, most))
        masks = op == "scored"
        c = _case("", op, storage=storage, dtype=dtype, heads=rng.choice([1, 2, 3, 4, 5, 8, 8, 16]), group=rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16]),
                  dim=rng.choice([64, 64, 80, 96, 128, 128, 128, 256]), page=rng.choice([16, 32, 64, 64, 128]), seqs=spread(1, 64), new=new, length=length,
                  ways=rng.choice([1, 2, 3, 4, 8]) if op == "branch" else 0, window=rng.choice([0, 0, 0, spread(16, 8192)]) if op in ("attend", "scored") else 0,
                  blocks=spread(4, 64) if op == "sparse" else 0, cap=rng.choice([0.0, 5.0, 30.0, 50.0, 1000.0]) if masks else 0.0, slopes=rng.choice([0, 0, 1]) if masks else 0,
                  docs=rng.choice([0, 0, spread(3, 4096)]) if masks else 0, prefix=rng.choice([0, 0, spread(1, 4096)]) if masks else 0)
        news, lens = _lengths(c)
        w = work(c)
        # what the plain form holds: the padded scores, or the rows that the queries gather; and the cache itself
        rows = sum(news) * c["blocks"] * c["page"] if op == "sparse" else c["seqs"] * max(lens)
        scores = c["heads"] * c["group"] * (sum(news) * c["blocks"] * c["page"] if op == "sparse" else c["seqs"] * max(news) * max(lens) if op in ("attend", "scored", "compact") else 0)
        rows = max(rows, sum(m * -(-max(lens) // c["page"]) for m in news) if op == "sparse" else 0)  # the bounds that they gather
        held = sum(lens) * c["heads"] * c["dim"]
        if scores <= 2 ** 31 and rows * c["heads"] * c["dim"] <= 2 ** 31 and held <= 2 ** 31 and w["bytes"] <= 1.5e9 and w["flops"] <= 1.5e12:
            return c


def _lengths(case):
    """New tokens and length (the new ones included) of every sequence: the first has the most of both, the others less, evenly over the
    logarithm.  (A branch has new tokens beyond the length of its parent.)"""
    r = random.Random("%(seqs)d %(new)d %(length)d %(page)d" % case)
    news = [case["new"]] + [max(1, int(case["new"] ** r.random())) for _ in range(case["seqs"] - 1)]
    lens = [case["length"]] + [max(n, int(case["length"] * 16 ** -r.random())) for n in news[1:]]
    return [min(n, case["length"]) for n in news], lens


def _masks(case):
    """Of every sequence the first position of its new tokens' documents, and its prefix."""
    news, lens = _lengths(case)
    r = random.Random("%(seqs)d %(length)d %(docs)d %(prefix)d" % case)
    starts, prefixes = [], []
    for m, l in zip(news, lens):
        prefixes.append(min(l, max(1, int(case["prefix"] * r.uniform(0.3, 1.0)))) if case["prefix"] else 0)
        begins, at = [], prefixes[-1]
        while case["docs"] and at < l:
            begins.append(at)
            at += max(1, int(case["docs"] * r.uniform(0.1, 1.9)))
        mine, j = [], 0
        for p in range(l - m, l):
            while j + 1 < len(begins) and begins[j + 1] <= p:
                j += 1
            mine.append(begins[j] if begins and begins[j] <= p else 0)
        starts.append(mine)
    return starts, prefixes


def _row_bytes(case):
    """A token's keys and values as they are stored, with their scales (4 bits: half a byte more for each 32 channels of the key)."""
    h, d, st = case["heads"], case["dim"], case["storage"]
    return 2 * h * (d * BITS[st] // 8 + (4 if st in LARGEST else 0)) + (h * -(-d // 32) // 2 if st == "f4" else 0)


def work(case):
    news, lens = _lengths(case)
    h, g, d, p = case["heads"], case["group"], case["dim"], case["page"]
    row, n, side, bound = _row_bytes(case), sum(news), 2 * h * d * 2, h * (2 * d + 4)
    if case["op"] == "branch":
        w = case["ways"]
        pages = sum(-(-l // p) for l in lens)  # entries of the parents' tables; shared pages that are copied, and what is read back
        copied = w * sum(1 for l in lens if l % p)
        back = w * sum(m + l % p for m, l in zip(news, lens))
        return {"bytes": w * pages * 8 + copied * 2 * (p * row + bound) + w * n * (side + row) + back * (row + side), "flops": 8 * w * n * h * d}
    if case["op"] == "compact":
        live, total = len(set().union(*map(set, _shared(case)))), sum(lens)
        return {"bytes": 2 * live * (p * row + bound) + total * row + 2 * n * h * g * d * 2, "flops": 4 * d * h * g * sum(m * (2 * l - m + 1) // 2 for m, l in zip(news, lens))}
    if case["op"] == "append":
        touched = sum((l - 1) // p - (l - m) // p + 1 for m, l in zip(news, lens))
        return {"bytes": n * (2 * side + 2 * row) + touched * (bound + 2 * h * d * 4), "flops": 8 * n * h * d}
    if case["op"] in ("attend", "scored"):
        starts, prefixes = _masks(case)
        w, pairs, seen = case["window"] or 1 << 30, 0, 0
        for m, l, begin, prefix in zip(news, lens, starts, prefixes):
            first = l
            for q, s in zip(range(l - m, l), begin):
                low = max(0, s, q - w + 1, prefix)
                pairs += min(prefix, l) + max(0, q - low + 1)
                first = min(first, low)
            seen += prefix + max(0, l - first)
        return {"bytes": seen * row + 2 * n * h * g * d * 2, "flops": 4 * d * h * g * pairs}
    kept = [min(case["blocks"], -(-l // p)) for l in lens]  # blocks of a query at most
    pages = sum(-(-l // p) for l in lens)
    seen = sum(min(l * h, m * h * b * p) for b, m, l in zip(kept, news, lens)) * row // h
    pairs = sum(m * b * p for b, m in zip(kept, news))
    return {"bytes": seen + pages * bound + 2 * n * h * g * d * 2 + n * h * case["blocks"] * 4,
            "flops": 4 * d * h * g * (pairs + sum(m * -(-l // p) for m, l in zip(news, lens)))}


def _shared(case):
    """Pages of the sequences of a cache that is about to be compacted, numbered by first use: every third sequence shares the first half of the
    pages of the one before it."""
    _, lens = _lengths(case)
    out, at = [], 0
    for i, l in enumerate(lens):
        m = -(-l // case["page"])
        # (full pages alone: a page that is not full is written into, and has one owner)
        common = out[-1][:min(m // 2, lens[i - 1] // case["page"])] if i % 3 == 2 else []
        out.append(common + list(range(at, at + m - len(common))))
        at += m - len(common)
    return out


def _rows(case, gen, count):
    """Keys and values of `count` tokens: channels of unequal size, runs of tokens that resemble one another, and a few large ones."""
    h, d, kind = case["heads"], case["dim"], TYPES[case["dtype"]]
    size = torch.exp(0.5 * torch.randn(h, d, device="cuda", generator=gen))
    run = torch.arange(count, device="cuda") // 96
    topics = torch.randn(count // 96 + 1, h, d, device="cuda", generator=gen) * size
    k, v = torch.empty(count, h, d, device="cuda", dtype=kind), torch.empty(count, h, d, device="cuda", dtype=kind)
    for at in range(0, count, 1 << 18):
        part = slice(at, min(count, at + (1 << 18)))
        k[part] = topics[run[part]] + 0.7 * torch.randn(k[part].shape, device="cuda", generator=gen)
        v[part] = torch.randn(k[part].shape, device="cuda", generator=gen) * torch.exp(0.3 * torch.randn(k[part].shape[0], h, 1, device="cuda", generator=gen))
    return k, v, topics


def _batch(tables, news, lens):
    return {"tables": tables, "offsets": torch.tensor([0] + news).cumsum(0).to("cuda", torch.int32), "lens": torch.tensor(lens, dtype=torch.int32).cuda(),
            "n_tokens": sum(news), "max_new": max(news), "max_len": max(lens)}


def prepare(case, seed):
    """The cache with everything but the new tokens in it (where they are not written: with them), the batch's plan, and the step's rows."""
    news, lens = _lengths(case)
    op, h, g, d, p, kind = case["op"], case["heads"], case["group"], case["dim"], case["page"], TYPES[case["dtype"]]
    gen, host = torch.Generator("cuda").manual_seed(seed), torch.Generator().manual_seed(seed)
    n, count = sum(news), sum(lens)
    k, v, topics = _rows(case, gen, count)
    # pages in a random order out of what the cache has: of one that is left or branches, a part of it
    held = _shared(case) if op == "compact" else None
    pages = [-(-l // p) for l in lens]
    used = max(map(max, held)) + 1 if held else sum(pages)
    more = sum(-(-(l + m) // p) - l // p for m, l in zip(news, lens)) * case["ways"]
    n_pages = 2 * used if held else used + more + used // 8
    order = torch.randperm(n_pages, generator=host, dtype=torch.int32)
    cols = max(-(-(l + (m if case["ways"] else 0)) // p) for m, l in zip(news, lens))
    tables = torch.full((len(lens) * (1 + case["ways"]), cols), -1, dtype=torch.int32)
    at = 0
    for i, m in enumerate(pages):
        tables[i, :m] = order[torch.tensor(held[i])] if held else order[at:at + m]
        at += m
    tables = tables.cuda()
    s = {"op": op, "window": case["window"], "blocks": case["blocks"], "scale": d ** -0.5, "kind": kind, "tables": tables}
    whole = torch.tensor([0] + lens).cumsum(0).to("cuda", torch.int32)
    parents = _batch(tables[:len(lens)], lens, lens)
    if op == "branch":
        w, size = case["ways"], len(lens)
        s["lens"], s["from"] = parents["lens"].repeat(1 + w), torch.arange(size, dtype=torch.int32).repeat(w).cuda()
        s["to"] = torch.arange(size, size * (1 + w), dtype=torch.int32).cuda()
        s["batch"] = b = _batch(tables[size:], news * w, [l + m for m, l in zip(news, lens)] * w)
        s["own"] = _batch(tables[size:], [m + l % p for m, l in zip(news, lens)] * w, [l + m for m, l in zip(news, lens)] * w)
        n *= w
        at = torch.randint(0, count, (n,), device="cuda", generator=gen)  # a branch's tokens resemble some that were before
    else:
        s["batch"] = b = _batch(tables, news, lens)
        new = _tokens(b)
        at = whole[new["seq"]].long() + new["pos"]
    # the step's rows are parts of one product, as a model's layer gives them
    near = topics[torch.randint(0, topics.shape[0], (n,), device="cuda", generator=gen)].repeat_interleave(g, 1)
    fused = torch.empty(n, h * (g + 2), d, dtype=kind, device="cuda")
    fused[:, :h * g] = 0.6 * near + torch.randn(n, h * g, d, device="cuda", generator=gen)
    fused[:, h * g:h * (g + 1)], fused[:, h * (g + 1):] = k[at], v[at]
    s["q"], s["k"], s["v"] = fused[:, :h * g], fused[:, h * g:h * (g + 1)], fused[:, h * (g + 1):]
    if op == "append":  # the tokens before the new ones
        before = [l - m for l, m in zip(lens, news)]
        keep = torch.ones(count, dtype=torch.bool, device="cuda")
        keep[at] = False
        k, v, parents = k[keep], v[keep], _batch(tables, before, before)
        first, last = (b["lens"] - b["offsets"].diff()) // p, (b["lens"] - 1) // p
        column = torch.arange(cols, device="cuda")
        s["touched"] = tables[(column >= first[:, None]) & (column <= last[:, None])]
    if op == "scored":
        starts, prefixes = _masks(case)
        s["how"] = {"cap": case["cap"], "slopes": torch.exp2(-8.0 * torch.arange(1, h * g + 1, device="cuda") / (h * g)) if case["slopes"] else None,
                    "starts": torch.tensor(sum(starts, []), dtype=torch.int32).cuda() if case["docs"] else None,
                    "prefix": torch.tensor(prefixes, dtype=torch.int32).cuda() if case["prefix"] else None}
    if own:
        from paper_2602_21477_amd import binding as B
        kinds = {"f16": B.PK_F16, "bf16": B.PK_BF16, "i8": B.PK_I8, "f8": B.PK_F8, "f4": B.PK_F4}
        s["cache"] = B.KVCache(n_pages, h, d, storage=kinds[case["storage"]], page_tokens=p)
        s["batch"] = B.KVBatch(**b)
        _fill(case, held, lambda b, rows: s["cache"].append(k[rows], v[rows], B.KVBatch(**b)), parents)
        if op in ("branch", "compact"):
            s["pool"] = B.KVPool(s["cache"])
            s["pool"].adopt(tables)
        if op == "branch":
            s["own"] = B.KVBatch(**s["own"])
        if op == "compact":
            s["into"] = B.KVPool(B.KVCache(used + used // 8 + 1, h, d, storage=kinds[case["storage"]], page_tokens=p))
        return s
    s["cache"] = c = _cache(case, n_pages)
    _fill(case, held, lambda b, rows: _append(c, k[rows], v[rows], b), parents)
    for part in torch.split(torch.arange(n_pages, device="cuda"), 4096):
        _bound(c, part)
    if op in ("branch", "compact"):
        s["refs"] = torch.bincount(tables[tables >= 0].long(), minlength=n_pages)
    if op == "compact":
        s["into"] = _cache(case, used + used // 8 + 1)
    return s


def _fill(case, held, append, parents):
    """All tokens, a sequence after the other where they share pages (the rows of the later one stay)."""
    if not parents["n_tokens"]:
        return
    if not held:
        return append(parents, slice(None))
    o = parents["offsets"].tolist()
    for i in range(len(o) - 1):
        m = o[i + 1] - o[i]
        append(_batch(parents["tables"][i:i + 1], [m], [m]), slice(o[i], o[i + 1]))


def _cache(case, n_pages):
    h, d, p = case["heads"], case["dim"], case["page"]
    held = {"i8": torch.int8, "f8": torch.float8_e4m3fn, "f4": torch.float16}.get(case["storage"], TYPES[case["dtype"]])  # (4 bits: code times the group's power of two)
    c = {"storage": case["storage"], "k": torch.zeros(n_pages, p, h, d, device="cuda", dtype=held), "hi": torch.zeros(n_pages, h, d, device="cuda", dtype=torch.int8)}
    c["v"], c["lo"] = torch.zeros_like(c["k"]), torch.zeros_like(c["hi"])
    c["ks"], c["vs"] = (torch.ones(n_pages, p, h, 1, device="cuda") for _ in range(2))
    c["bs"], c["fill"] = torch.zeros(n_pages, h, 1, device="cuda"), torch.zeros(n_pages, device="cuda", dtype=torch.long)
    return c


def run(s):
    op, c, b = s["op"], s["cache"], s["batch"]
    if own:
        if op == "branch":
            s["pool"].fork(s["tables"], s["lens"], s["from"], s["to"])
            missing = s["pool"].grant(b)
            c.append(s["k"], s["v"], b)
            out = {"tables": s["tables"].clone(), "missing": missing, "kv": c.read(s["own"], s["kind"])}
            s["pool"].release(s["tables"], s["to"])
            return {**out, "refs": s["pool"].counts()}
        if op == "compact":
            from paper_2602_21477_amd import binding as B
            tables, missing = s["pool"].compact(s["into"], s["tables"])
            moved = B.KVBatch(tables, b.offsets, b.lens, b.c.n_tokens, b.c.max_new, b.c.max_len)
            return {"tables": tables, "missing": missing, "refs": s["into"].counts(), "out": s["into"].cache.attend(s["q"], moved, s["scale"])}
        if op == "append":
            c.append(s["k"], s["v"], b)
            return {"kv": c.read(b, s["kind"]), "bounds": c.bounds(s["touched"])}
        if op == "attend":
            return c.attend(s["q"], b, s["scale"], window=s["window"], want_lse=True)
        if op == "scored":
            return c.attend(s["q"], b, s["scale"], window=s["window"], want_lse=True, **s["how"])
        blocks = c.select(s["q"], b, s["blocks"])
        return {"blocks": blocks, "out": c.attend_blocks(s["q"], blocks, b, s["scale"])}
    if op == "branch":
        _fork(s)
        missing = _grant(s)
        _append(c, s["k"], s["v"], b)
        out = {"tables": s["tables"].clone(), "missing": missing, "kv": _read(c, s["own"], s["kind"])}
        _release(s)
        return {**out, "refs": s["refs"].to(torch.int32)}
    if op == "compact":
        tables, missing, refs = _compact(s)
        return {"tables": tables, "missing": missing, "refs": refs, "out": _attend(s["into"], s["q"], {**b, "tables": tables}, s["scale"], 0, {})[0]}
    if op == "append":
        _append(c, s["k"], s["v"], b)
        _bound(c, s["touched"].long())
        return {"kv": _read(c, b, s["kind"]), "bounds": (c["hi"][s["touched"]] * c["bs"][s["touched"]], c["lo"][s["touched"]] * c["bs"][s["touched"]])}
    if op in ("attend", "scored"):
        return _attend(c, s["q"], b, s["scale"], s["window"], s.get("how", {}))
    blocks = _select(c, s["q"], b, s["blocks"])
    return {"blocks": blocks, "out": _attend_blocks(c, s["q"], blocks, b, s["scale"])}


def _tokens(b):
    """Sequence and position of every new token of a batch."""
    news = b["offsets"].diff().long()
    seq = torch.repeat_interleave(torch.arange(news.shape[0], device="cuda"), news, output_size=b["n_tokens"])
    index = torch.arange(b["n_tokens"], device="cuda") - b["offsets"][seq]
    return {"seq": seq, "index": index, "pos": b["lens"][seq].long() - news[seq] + index}


# ------------------------------------------------------------------ pages

def _fork(s):
    """Row to[i] of the tables gets the pages of row from[i], which then have one owner more."""
    page, t = s["cache"]["k"].shape[1], s["tables"]
    rows = t[s["from"].long()]
    rows = rows.masked_fill(torch.arange(t.shape[1], device="cuda") >= ((s["lens"][s["from"].long()] + page - 1) // page)[:, None], -1)
    t[s["to"].long()] = rows
    s["refs"] += torch.bincount(rows[rows >= 0].long(), minlength=s["refs"].shape[0])


def _grant(s):
    """Every page that the batch's new tokens go into becomes its sequence's own: one that is not there, or that others have too, is replaced
    by the lowest free one, in the order of sequences and positions, and what a shared one held is copied.  A page that only sequences of this
    batch have, and all of them write into, is kept by the last of them."""
    b, refs, c = s["batch"], s["refs"], s["cache"]
    page, t = c["k"].shape[1], b["tables"]
    begin = (b["lens"] - b["offsets"].diff()).long()
    column = torch.arange(t.shape[1], device="cuda")
    touched = (column >= (begin // page)[:, None]) & (column <= ((b["lens"].long() - 1) // page)[:, None])
    seq, col = touched.nonzero(as_tuple=True)
    entry = t[seq, col].long()
    there = entry >= 0
    users = torch.bincount(entry[there], minlength=refs.shape[0])
    last = torch.full_like(refs, -1).index_reduce_(0, entry[there], seq[there], "amax")
    at = entry.clamp(min=0)
    keeps = there & (users[at] == refs[at]) & (last[at] == seq)
    need = (~keeps).nonzero().squeeze(1)
    free = (refs == 0).nonzero().squeeze(1)
    got = torch.full((need.shape[0],), -1, device="cuda")
    m = min(need.shape[0], free.shape[0])
    got[:m] = free[:m]
    before = entry[need]
    refs -= torch.bincount(before[before >= 0], minlength=refs.shape[0])
    refs[got[:m]] = 1
    t[seq[need], col[need]] = got.to(torch.int32)
    old = (before >= 0) & (got >= 0) & (begin[seq[need]] > col[need] * page)  # (it holds older tokens)
    for x in c:
        if x != "storage":
            c[x][got[old]] = c[x][before[old]]
    return torch.tensor([need.shape[0] - m], dtype=torch.int32, device="cuda")


def _release(s):
    rows = s["tables"][s["to"].long()]
    s["refs"] -= torch.bincount(rows[rows >= 0].long(), minlength=s["refs"].shape[0])
    s["tables"][s["to"].long()] = -1


def _compact(s):
    """Pages in use, in their order, become the first ones of another cache."""
    refs, t = s["refs"], s["tables"]
    live = (refs > 0).nonzero().squeeze(1)
    there = s["into"]["k"].shape[0]
    m = min(live.shape[0], there)
    for x in s["into"]:
        if x != "storage":
            s["into"][x][:m] = s["cache"][x][live[:m]]
    names = torch.full((refs.shape[0] + 1,), -1, device="cuda", dtype=torch.int32)
    names[live[:m]] = torch.arange(m, device="cuda", dtype=torch.int32)
    counts = torch.zeros(there, device="cuda", dtype=torch.int32)
    counts[:m] = refs[live[:m]].to(torch.int32)
    tables = names[torch.where(t >= 0, t, torch.full_like(t, refs.shape[0])).long()]
    return tables, torch.tensor([live.shape[0] - m], dtype=torch.int32, device="cuda"), counts


# ------------------------------------------------------------------ storage

def _e2m1(y):
    """To nearest even of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives."""
    a = y.abs()
    r = torch.where(a < 2, (a * 2).round() / 2, torch.where(a < 4, a.round(), (a / 2).round() * 2))
    return torch.where(y < 0, -r, r)


def _quantised(x, storage, kind, grouped=False):
    """Codes and scales: one scale for each token and head; keys in 4 bits also have a power of two for each 32 channels."""
    x = x.float()
    if storage not in LARGEST:
        return x.to(kind), torch.ones_like(x[..., :1])
    most = x.abs().amax(-1, keepdim=True)
    up = torch.where(most > 0, torch.full_like(most, LARGEST[storage]) / most, torch.zeros_like(most)).clamp(max=3.0e38)
    power = torch.ones_like(most)
    if grouped and storage == "f4":
        pad = -x.shape[-1] % 32
        groups = torch.nn.functional.pad(x.abs(), (0, pad)).unflatten(-1, (-1, 32)).amax(-1)
        shift = ((most.view(torch.int32) - groups.view(torch.int32)) >> 23).clamp(max=15)  # whole powers of two that the group's largest is below the row's
        power = torch.exp2(shift.float()).repeat_interleave(32, -1)[..., :x.shape[-1]]
    y = ((x * power) * up).clamp(-LARGEST[storage], LARGEST[storage])
    if storage == "f4":
        return (_e2m1(y) / power).to(kind), most * torch.tensor(1.0 / 6.0, dtype=torch.float32)
    return (y.round() if storage == "i8" else y).to(kind), most * (1.0 / LARGEST[storage])


def _append(c, k, v, b):
    t = _tokens(b)
    page = c["k"].shape[1]
    entry = b["tables"][t["seq"], t["pos"] // page].long()
    if (entry < 0).any():  # (tokens of pages that the sequence has not are written nowhere)
        ok = entry >= 0
        k, v, entry, t = k[ok], v[ok], entry[ok], {x: y[ok] for x, y in t.items()}
    at = entry, t["pos"] % page
    for x, codes, scales in ((k, "k", "ks"), (v, "v", "vs")):
        c[codes][at], c[scales][at] = _quantised(x, c["storage"], c["k"].dtype, grouped=codes == "k")
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


# ------------------------------------------------------------------ attention

def _softmax(scores, mask):
    """Weights, and the logarithm of what they were divided by: none and -inf for a row without keys."""
    scores = scores.masked_fill(~mask, -math.inf)
    most = scores.amax(-1, keepdim=True).clamp(min=-3.0e38)
    weights = torch.exp(scores - most)
    total = weights.sum(-1, keepdim=True)
    return weights / total.clamp(min=1e-37), (most + torch.log(total)).squeeze(-1)


def _attend(c, q, b, scale, window, how):
    """Every sequence padded to the longest, its pages side by side, a key/value head after the other."""
    t, (n, hq, d) = _tokens(b), q.shape
    seqs, m, h, table = b["lens"].shape[0], b["max_new"], c["k"].shape[2], b["tables"].clamp(min=0).long()
    g, length = hq // h, b["tables"].shape[1] * c["k"].shape[1]
    pos = (b["lens"] - b["offsets"].diff())[:, None] + torch.arange(m, device="cuda")
    key = torch.arange(length, device="cuda")
    mask = (key <= pos[:, :, None]) & (key > pos[:, :, None] - (window or 1 << 30))
    if how.get("starts") is not None:
        begin = torch.zeros(seqs, m, device="cuda", dtype=torch.int32)
        begin[t["seq"], t["index"]] = how["starts"]
        mask &= key >= begin[:, :, None]
    if how.get("prefix") is not None:
        mask |= key < how["prefix"][:, None, None]
    mask &= key < b["lens"][:, None, None]
    far = (pos[:, :, None] - key).abs().float() if how.get("slopes") is not None else None
    out, lse = torch.empty(n, hq, d, device="cuda", dtype=q.dtype), torch.empty(n, hq, device="cuda")
    for head in range(h):
        keys, values = ((c[x][:, :, head][table].float() * c[y][:, :, head][table]).flatten(1, 2) for x, y in (("k", "ks"), ("v", "vs")))
        rows = torch.zeros(seqs, g, m, d, device="cuda")
        rows[t["seq"], :, t["index"]] = q[:, head * g:(head + 1) * g].float()
        scores = torch.matmul(rows.flatten(1, 2), keys.transpose(1, 2).contiguous()).mul_(scale).view(seqs, g, m, length)
        if how.get("cap"):
            scores = torch.tanh(scores / how["cap"]) * how["cap"]
        if far is not None:
            scores -= how["slopes"][head * g:(head + 1) * g, None, None] * far[:, None]
        weights, part = _softmax(scores, mask[:, None])
        seen = torch.matmul(weights.flatten(1, 2), values.masked_fill((key >= b["lens"][:, None])[:, :, None], 0.0)).view(seqs, g, m, d)
        out[:, head * g:(head + 1) * g] = seen[t["seq"], :, t["index"]].to(q.dtype)
        lse[:, head * g:(head + 1) * g] = part[t["seq"], :, t["index"]]
    return out, lse


def _select(c, q, b, blocks):
    t, (n, hq, d) = _tokens(b), q.shape
    h = c["k"].shape[2]
    codes, scales = _quantised(q, "i8", torch.int8)
    codes, table = codes.float().view(n, h, hq // h, d), b["tables"].clamp(min=0).long()
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


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    """A row's stored values are what its codes and its 32-bit scale stand for."""
    global own
    news, lens = _lengths(case)
    op, h, g, d, p, st = case["op"], case["heads"], case["group"], case["dim"], case["page"], case["storage"]
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c, b, table = s["cache"], s["batch"], s["batch"]["tables"].long()

    def stored(x, key):  # [token, head, channel] as it is held
        x = x.double()
        if st not in LARGEST:
            return x
        most = x.abs().amax(-1, keepdim=True)
        ones = torch.ones_like(most)
        y = torch.where(most > 0, x / torch.where(most > 0, most, ones) * LARGEST[st], torch.zeros_like(x))
        if st == "i8":
            y = y.round()
        elif st == "f8":
            y = y.to(torch.float8_e4m3fn).double()
        else:
            # (the definition is in 32 bits: 6 / largest, and its product with an element, are rounded to them; rows of 16 bits have ties in plenty)
            values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
            middle = (values[1:] + values[:-1]) / 2
            up = torch.ones_like(y)
            for at in range(0, d, 32) if key else []:
                part = x[..., at:at + 32].abs().amax(-1, keepdim=True)
                up[..., at:at + 32] = 2.0 ** torch.floor(torch.log2(most / torch.where(part > 0, part, ones * 1e-300))).clamp(0, 15)
            z = (x * up * torch.where(most > 0, 6.0 / torch.where(most > 0, most, ones), torch.zeros_like(most)).float().double()).float().double().abs()
            code = torch.bucketize(z, middle)  # a value in the middle goes down here
            tie = z == middle[code.clamp(max=6)]
            code = torch.where(tie & (code % 2 == 1) & (code < 7), code + 1, code)  # and to the even one
            y = values[code] * torch.sign(x) / up
        return y * (most.float() * torch.tensor(1.0 / LARGEST[st], dtype=torch.float32)).double()

    def sequence(name, i):  # all rows of sequence i that the cache holds, [head, token, channel]
        m = -(-lens[i] // p)
        return (c[name][table[i, :m]].double() * c[name + "s"][table[i, :m]].double()).flatten(0, 1)[:lens[i]].transpose(0, 1)

    if op == "branch":
        k, v, at, out = stored(s["k"], True), stored(s["v"], False), 0, ([], [])
        parents = s["tables"].long()
        for m, l, i in [(m, l, i) for _ in range(case["ways"]) for i, (m, l) in enumerate(zip(news, lens))]:
            page = parents[i, l // p] if l % p else 0
            for name, rows, to in (("k", k, out[0]), ("v", v, out[1])):
                to += [(c[name][page].double() * c[name + "s"][page].double())[:l % p], rows[at:at + m]]
            at += m
        return {"tables": None, "missing": None, "kv": tuple(torch.cat(x) for x in out), "refs": None}
    if op == "append":
        k, v = stored(s["k"], True), stored(s["v"], False)
        his, los, at = [], [], 0
        for i, (m, l) in enumerate(zip(news, lens)):
            kept = sequence("k", i)
            kept[:, l - m:] = k[at:at + m].transpose(0, 1)
            at += m
            for j in range((l - m) // p, (l - 1) // p + 1):
                rows = kept[:, j * p:min(l, (j + 1) * p)]
                hi, lo = (x.float().double() for x in (rows.amax(1), rows.amin(1)))
                most = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
                unit = torch.where(most > 0, most / 127, torch.ones_like(most))
                # the next whole number outwards (steps are defined in 32 bits: values of 4 bits meet the slack exactly)
                up = (1 / unit).float().double()
                his.append(torch.ceil((hi * up).float().double() - SLACK).clamp(-127, 127) * unit)
                los.append(torch.floor((lo * up).float().double() + SLACK).clamp(-127, 127) * unit)
        return {"kv": (k, v), "bounds": (torch.stack(his), torch.stack(los))}
    q = s["q"].double().view(-1, h, g, d)
    out = torch.zeros(sum(news), h, g, d, dtype=torch.float64, device="cuda")
    lse = torch.full((sum(news), h, g), -math.inf, dtype=torch.float64, device="cuda")
    blocks = _select(c, s["q"], b, case["blocks"]) if op == "sparse" else None  # whole numbers: the definition is what they are by
    starts, prefixes = _masks(case)
    slope = torch.exp2(-8.0 * torch.arange(1, h * g + 1, device="cuda") / (h * g)).double().view(h, g) if case["slopes"] else None
    at = 0
    for i, (m, l) in enumerate(zip(news, lens)):
        keys, values = sequence("k", i), sequence("v", i)
        begin, key = torch.tensor(starts[i], device="cuda")[:, None], torch.arange(l, device="cuda")[None]
        for j in range(0, m, 512):
            part = slice(at + j, at + min(m, j + 512))
            pos = torch.arange(l - m + j, l - m + min(m, j + 512), device="cuda")[:, None]
            mask = (key <= pos) & (key >= begin[j:j + 512])
            if case["window"]:
                mask &= key > pos - case["window"]
            mask |= key < prefixes[i]
            for head in range(h):
                seen = mask
                if blocks is not None:
                    chosen = torch.zeros(pos.shape[0], table.shape[1] + 1, dtype=torch.bool, device="cuda")
                    chosen.scatter_(1, blocks[part, head].long() % (table.shape[1] + 1), True)  # -1: a column beyond the table
                    seen = seen & chosen[:, :-1].repeat_interleave(p, 1)[:, :l]
                for member in range(g):
                    x = (q[part, head, member] @ keys[head].T) * s["scale"]
                    if case["cap"]:
                        x = case["cap"] * torch.tanh(x / case["cap"])
                    if slope is not None:
                        x = x - slope[head, member] * (pos - key).abs()
                    x = torch.where(seen, x, torch.full_like(x, -math.inf))
                    lse[part, head, member] = torch.logsumexp(x, 1)
                    out[part, head, member] = torch.nan_to_num(torch.exp(x - lse[part, head, member, None])) @ values[head]
        at += m
    if op == "compact":
        return {"tables": None, "missing": None, "refs": None, "out": out.flatten(1, 2)}
    if blocks is not None:
        return {"blocks": None, "out": out.flatten(1, 2)}
    return out.flatten(1, 2), lse.flatten(1, 2)
