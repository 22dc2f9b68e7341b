"""The operators of the paged key-value cache that are timed: one step's page
bookkeeping, the write of new tokens' K and V, and the attention of one new
token per request over the pages.

A case is a dict of plain values with ``kind``:

* ``tables``: one step of ``requests`` sequences: pages for their new tokens,
  the slot of each, the pages of ended sequences returned. ``held`` is the
  longest sequence before the step, ``new`` the most new tokens of one, ``ends``
  how many sequences end, ``tokens`` the places in the slot map;
* ``append``: K and V ``[heads, tokens, dim]`` into the slots of a cache;
* ``attend``: one query token for each of ``requests`` sequences of up to
  ``longest`` tokens, ``heads`` query heads over ``kv_heads`` key-value heads,
  over the whole sequence or its first ``anchor`` and last ``window`` tokens.

``page`` is the tokens of a page, ``cache`` the cache's type: ``bf16``, ``f32``,
or ``e4m3``, 8-bit values with a power of two for each token and head. Lengths
are spread evenly from 1 to the longest and given to the requests in an order
that comes from the seed, as do the pages that the sequences hold.
"""
import math

import torch

own = False

DEVICE = "cuda"
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}


def listed():
    return [
        # the bookkeeping of one generation step: a token for each running sequence, mostly into a page it holds
        {"name": "tables_64_next", "kind": "tables", "requests": 64, "held": 10992, "new": 1, "ends": 0, "tokens": 64,
         "page": 16},
        # a busy server's step: sequences that end, others that go on by a few tokens, a padded slot map
        {"name": "tables_1000_mixed", "kind": "tables", "requests": 1000, "held": 10992, "new": 40, "ends": 37,
         "tokens": 24576, "page": 64},
        # a new frame of up to 1374 tokens for each of 100 streams
        {"name": "tables_100_frames", "kind": "tables", "requests": 100, "held": 5496, "new": 1374, "ends": 3,
         "tokens": 70000, "page": 64},
        # the K and V of that generation step
        {"name": "append_64_bf16", "kind": "append", "tokens": 64, "heads": 8, "dim": 128, "page": 16, "cache": "bf16"},
        # a whole sequence of 100 frames kept for later tokens
        {"name": "append_137400_bf16", "kind": "append", "tokens": 137400, "heads": 16, "dim": 64, "page": 64,
         "cache": "bf16"},
        # 32 frames into the 8-bit cache
        {"name": "append_43968_e4m3", "kind": "append", "tokens": 43968, "heads": 16, "dim": 64, "page": 64,
         "cache": "e4m3"},
        # the smallest configured sequence in full precision, one token: launches and one wave's latency
        {"name": "attend_1x1044_f32", "kind": "attend", "requests": 1, "longest": 1044, "heads": 16, "kv_heads": 16,
         "dim": 64, "page": 64, "cache": "f32", "anchor": 0, "window": 0},
        # one token over the longest configured sequence: everything hangs on splitting its length
        {"name": "attend_1x274800_bf16", "kind": "attend", "requests": 1, "longest": 274800, "heads": 16,
         "kv_heads": 16, "dim": 64, "page": 64, "cache": "bf16", "anchor": 0, "window": 0},
        # a serving batch of ragged lengths, four query heads to a key-value head, small pages
        {"name": "attend_64x10992_bf16", "kind": "attend", "requests": 64, "longest": 10992, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "cache": "bf16", "anchor": 0, "window": 0},
        # a larger batch on the 8-bit cache
        {"name": "attend_192x10992_e4m3", "kind": "attend", "requests": 192, "longest": 10992, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64, "cache": "e4m3", "anchor": 0, "window": 0},
        # many short sequences, a batch of first answers: many rows, few keys each
        {"name": "attend_256x261_bf16", "kind": "attend", "requests": 256, "longest": 261, "heads": 16, "kv_heads": 4,
         "dim": 64, "page": 16, "cache": "bf16", "anchor": 0, "window": 0},
        # streams that keep their anchor frame and the last five, all query heads on one key-value head
        {"name": "attend_48x10992_window", "kind": "attend", "requests": 48, "longest": 10992, "heads": 16,
         "kv_heads": 1, "dim": 128, "page": 16, "cache": "bf16", "anchor": 1374, "window": 6870},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"append": work(listed()[4])["bytes"], "attend": work(listed()[9])["bytes"]}
    while True:
        kind = rng.choice(["tables", "append", "attend", "attend"])
        case = {"kind": kind, "page": rng.choice([16, 32, 48, 64, 128])}
        if kind == "tables":
            n = case["requests"] = _log_int(rng, 1, 1000)
            case["held"] = _log_int(rng, 16, 10992)
            case["new"] = rng.choice([1, 1, _log_int(rng, 1, 1374)])
            case["ends"] = rng.randint(0, n // 8)
            case["tokens"] = sum(max(0, x) for x in _tables_counts(case)[1]) + rng.randint(0, n)
            if 0 < case["tokens"] <= 137400:
                return case
            continue
        case["dim"] = rng.choice([64, 128])
        case["cache"] = rng.choice(["bf16", "bf16", "f32", "e4m3"])
        if kind == "append":
            case["tokens"] = _log_int(rng, 1, 137400)
            case["heads"] = rng.choice([1, 2, 4, 8, 12, 16])
        else:
            case["requests"] = _log_int(rng, 1, 256)
            case["longest"] = _log_int(rng, 16, 274800)
            case["kv_heads"] = rng.choice([1, 2, 4, 8, 12, 16])
            case["heads"] = case["kv_heads"] * rng.choice([1, 1, 2, 4, 5, 8, 16])
            windowed = rng.random() < 0.25
            case["anchor"] = rng.randint(0, case["longest"] // 4) if windowed else 0
            case["window"] = rng.randint(1, case["longest"]) if windowed else 0
            # the plain form takes every request at the longest one's length, in 32 bits
            if case["requests"] * case["longest"] * (case["kv_heads"] * case["dim"] + case["heads"]) > 192 * 10992 * 1056:
                continue
        if work(case)["bytes"] <= most[kind]:
            return case


# ---------------------------------------------------------------- inputs


def _lengths(n, most):
    """``n`` lengths evenly spread from 1 to ``most``, the longest among them."""
    return [most - i * (most - 1) // max(1, n - 1) for i in range(n)]


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _shuffled(values, g):
    t = torch.tensor(values, dtype=torch.int32, device=DEVICE)
    return t[torch.randperm(len(values), generator=g, device=DEVICE)].contiguous()


def _paged(lengths, page, width, g, spare=0):
    """A page table ``[requests, width]`` of pages in a random order (those past a length hold 0), and the pages left."""
    need = (lengths + page - 1) // page
    pages = int(need.sum()) + spare
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    j = torch.arange(width, dtype=torch.int32, device=DEVICE)
    mine = j[None] < need[:, None]
    table = torch.zeros((len(lengths), width), dtype=torch.int32, device=DEVICE)
    table[mine] = order[: pages - spare]
    return table, order[pages - spare:], pages


def _values(shape, g, dtype):
    """N(0, 1), drawn in slices so that the 32-bit values of a large cache are never there at once."""
    t = torch.empty(shape, dtype=TYPE[dtype], device=DEVICE)
    flat = t.view(-1)
    step = 1 << 28
    for a in range(0, flat.numel(), step):
        n = min(step, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=g, device=DEVICE).to(TYPE[dtype])
    return t


def _tables_counts(case):
    """Length and new tokens of each request, -1 for one that ends."""
    n = case["requests"]
    held = _lengths(n, case["held"])
    new = _lengths(n, case["new"])[::-1]
    return held, [-1 if i < case["ends"] else x for i, x in enumerate(new)]


def prepare(case, seed):
    g = _generator(seed)
    page = case["page"]
    s = {"case": case, "kind": case["kind"]}
    if case["kind"] == "tables":
        held, new = _tables_counts(case)
        order = torch.randperm(case["requests"], generator=g, device=DEVICE)
        s["lengths"] = torch.tensor(held, dtype=torch.int32, device=DEVICE)[order].contiguous()
        s["new"] = torch.tensor(new, dtype=torch.int32, device=DEVICE)[order].contiguous()
        width = -(-(case["held"] + case["new"]) // page)
        spare = -(-case["tokens"] // page) + case["requests"]
        s["table"], left, pages = _paged(s["lengths"], page, width, g, spare)
        s["free"] = torch.zeros(pages, dtype=torch.int32, device=DEVICE)  # a stack with room for every page
        s["free"][:spare] = left
        s["count"] = torch.tensor([spare], dtype=torch.int32, device=DEVICE)
        return s
    H, D, dt = case.get("kv_heads", case["heads"]), case["dim"], case["cache"]
    wide = "f32" if dt == "f32" else "bf16"
    if case["kind"] == "append":
        T = case["tokens"]
        pages = -(-T // page) + 3
        s["k"], s["v"] = (_values((H, T, D), g, wide) for _ in range(2))
        s["k"][:, ::1374] *= 4  # a frame's camera token has large keys
        # whole pages in any order, as the slot map of one long sequence
        order = torch.randperm(pages, generator=g, device=DEVICE)
        t = torch.arange(T, device=DEVICE)
        s["slots"] = (order[t // page] * page + t % page).to(torch.int32)
        s["k_pages"], s["v_pages"] = (torch.zeros((pages, H, page, D), dtype=TYPE[dt], device=DEVICE) for _ in range(2))
        s["k_exp"], s["v_exp"] = (torch.zeros((pages, H, page), dtype=torch.uint8, device=DEVICE) if dt == "e4m3" else None
                                  for _ in range(2))
        return s
    R = case["requests"]
    s["lengths"] = _shuffled(_lengths(R, case["longest"]), g)
    s["table"], _, pages = _paged(s["lengths"], page, -(-case["longest"] // page), g)
    s["k_pages"], s["v_pages"] = (_values((pages, H, page, D), g, dt) for _ in range(2))
    s["k_exp"], s["v_exp"] = (torch.randint(125, 129, (pages, H, page), generator=g, device=DEVICE).to(torch.uint8)
                              if dt == "e4m3" else None for _ in range(2))
    s["q"] = (2 * torch.randn((case["heads"], R, D), generator=g, device=DEVICE)).to(TYPE[wide])
    return s


# ---------------------------------------------------------------- the plain forms


def _plain_tables(s):
    page, lengths, new, table, free, count = (s["case"]["page"], s["lengths"].long(), s["new"].long(), s["table"], s["free"],
                                              s["count"].long())
    T, (R, W) = s["case"]["tokens"], table.shape
    j = torch.arange(W, device=table.device)[None]
    held = (lengths + page - 1) // page
    ends = new < 0
    # ended sequences push their pages, in their order
    back = torch.where(ends, held, 0)
    at = count + torch.cumsum(back, 0) - back
    given = j < back[:, None]
    free[(at[:, None] + j)[given]] = table[given]
    top = count + back.sum()
    # the others take from the top of the stack, in their order
    grow = new.clamp(min=0)
    start = torch.cumsum(grow, 0) - grow
    after = lengths + grow
    fits = (after <= W * page) & (start + grow <= T) & ~ends
    need = torch.where(fits, (after + page - 1) // page - held, 0)
    first = torch.cumsum(need, 0) - need
    fits &= (need == 0) | (first + need <= top)
    got = (j >= held[:, None]) & (j < (held + need)[:, None]) & fits[:, None]
    table[got] = free[(top - 1 - (first[:, None] + j - held[:, None]))[got]]
    taken = torch.where(fits, first + need, 0).max()
    starts = torch.cat([start, (start + grow)[-1:]]).clamp(max=T)
    t = torch.arange(T, device=table.device)
    r = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp(max=R - 1)
    pos = lengths[r] + t - starts[r]
    slot = table[r, (pos // page).clamp(0, W - 1)].long() * page + pos % page
    slots = torch.where((t < starts[-1]) & fits[r], slot, -1)
    left = torch.where(ends, 0, torch.where(fits, after, lengths))
    return {"lengths": left.int(), "starts": starts.int(), "slots": slots.int(), "count": (top - taken).int(), "table": table,
            "free": free}


def _plain_append(s):
    case = s["case"]
    page = case["page"]
    keep = s["slots"] >= 0
    slots = s["slots"][keep].long()
    p, o = slots // page, slots % page
    out = {}
    for name in ("k", "v"):
        x, pages, exps = s[name], s[name + "_pages"], s[name + "_exp"]
        x = x[:, keep].transpose(0, 1)  # [tokens, heads, dim]
        if exps is not None:
            x = x.float()
            # the least e with max|x| <= 448 * 2^e = 1.75 * 2^(8 + e)
            bits = x.abs().amax(2).contiguous().view(torch.int32)
            e = (((bits + 0x1FFFFF) >> 23) - 135).clamp(min=-126)
            codes = torch.ldexp(x, -e[:, :, None]).to(torch.float8_e4m3fn)
            pages.view(torch.uint8)[p, :, o] = codes.view(torch.uint8)
            exps[p, :, o] = (e + 127).to(torch.uint8)
            out[name + "_exp"] = exps
        else:
            pages[p, :, o] = x
        out[name + "_pages"] = pages
    return out


def _gathered(pages, exps, table):
    """Every request's tokens ``[requests, kv_heads, tokens, dim]`` in 32 bits."""
    R, W = table.shape
    _, H, page, D = pages.shape
    x = pages.view(torch.uint8)[table].view(torch.float8_e4m3fn) if exps is not None else pages[table]
    x = x.float()
    if exps is not None:
        x *= torch.exp2(exps[table].float() - 127)[..., None]
    return x.transpose(1, 2).reshape(R, H, W * page, D)


def _plain_attend(s):
    case = s["case"]
    R, Hq, H, D = case["requests"], case["heads"], case["kv_heads"], case["dim"]
    table = s["table"].long()
    k = _gathered(s["k_pages"], s["k_exp"], table)
    n = k.shape[2]
    j = torch.arange(n, device=k.device)[None]
    length = s["lengths"].long()[:, None]
    seen = j < length
    if case["window"]:
        seen &= (j < case["anchor"]) | (j >= length - case["window"])
    q = s["q"].float().transpose(0, 1).reshape(R, H, Hq // H, D)
    z = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)
    del k
    z.masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(3, keepdim=True)
    w = torch.exp(z - top)
    total = w.sum(3, keepdim=True)
    out = torch.matmul(w, _gathered(s["v_pages"], s["v_exp"], table)) / total
    lse = (top + torch.log(total)).reshape(R, Hq)
    return {"out": out.reshape(R, Hq, D).transpose(0, 1).to(s["q"].dtype), "lse": lse.transpose(0, 1).contiguous()}


def run(s):
    if not own:
        return {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend}[s["kind"]](s)
    import paper_2607_03612_amd as P

    case = s["case"]
    if s["kind"] == "tables":
        lengths, starts, slots, count = P.page_tables(s["lengths"], s["new"], s["free"], s["count"], s["table"], case["page"],
                                                      case["tokens"])
        return {"lengths": lengths, "starts": starts, "slots": slots, "count": count, "table": s["table"], "free": s["free"]}
    if s["kind"] == "append":
        P.cache_append(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"])
        out = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
        if s["k_exp"] is not None:
            out.update(k_exp=s["k_exp"], v_exp=s["v_exp"])
        return out
    out, lse = P.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lengths"], s["k_exp"], s["v_exp"],
                                 anchor=case["anchor"], window=case["window"], want_lse=True)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------- counts


def work(case):
    page = case["page"]
    if case["kind"] == "tables":
        held, new = _tables_counts(case)
        pages = lambda n: -(-n // page)  # noqa: E731
        moved = sum(pages(a) if b < 0 else pages(a + b) - pages(a) for a, b in zip(held, new))
        # both counts in, length and start out; the slots; a page moved is read and written; a page that holds
        # the first of the new tokens is looked up
        return {"bytes": 16 * case["requests"] + 4 * case["tokens"] + 8 * moved + 4 * sum(b >= 0 for b in new), "flops": 0}
    D, size = case["dim"], SIZE[case["cache"]]
    exps = 1 if case["cache"] == "e4m3" else 0
    wide = 4 if case["cache"] == "f32" else 2
    if case["kind"] == "append":
        rows = 2 * case["tokens"] * case["heads"]
        return {"bytes": rows * (D * (wide + size) + exps) + 4 * case["tokens"], "flops": 2 * rows * D * exps}
    keys = sum(min(n, min(case["anchor"], n) + case["window"]) if case["window"] else n
               for n in _lengths(case["requests"], case["longest"]))
    queries = case["requests"] * case["heads"]
    return {"bytes": 2 * keys * case["kv_heads"] * (D * size + exps) + queries * (2 * D * wide + 4)
            + 4 * (case["requests"] + keys // page), "flops": 4 * keys * case["heads"] * D}


# ---------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    page = case["page"]
    if case["kind"] == "tables":
        return None  # whole numbers only
    if case["kind"] == "append":
        out = {}
        for name in ("k", "v"):
            x, pages, exps = s[name].double(), s[name + "_pages"].double(), s[name + "_exp"]
            if exps is not None:
                # the values before their rounding to 8 bits
                largest = x.abs().amax(2, keepdim=True)
                e = torch.ceil(torch.log2(largest / 448)).clamp(min=-126)
                e = torch.where(largest > 448 * torch.exp2(e), e + 1, e)
                e = torch.where(largest <= 224 * torch.exp2(e), e - 1, e)
                x = x * torch.exp2(-e)
                out[name + "_exp"] = None
            flat = pages.transpose(1, 2).reshape(-1, case["heads"], case["dim"])
            flat[s["slots"].long()] = x.transpose(0, 1)
            out[name + "_pages"] = flat.view(-1, page, case["heads"], case["dim"]).transpose(1, 2).contiguous()
        return out
    R, Hq, H, D = case["requests"], case["heads"], case["kv_heads"], case["dim"]
    out = torch.empty((Hq, R, D), dtype=torch.float64, device=DEVICE)
    lse = torch.empty((Hq, R), dtype=torch.float64, device=DEVICE)
    for r, n in enumerate(s["lengths"].tolist()):
        ids = s["table"][r, : -(-n // page)].long()
        tokens = torch.arange(n, device=DEVICE)
        if case["window"]:
            tokens = tokens[(tokens < case["anchor"]) | (tokens >= n - case["window"])]
        kv = []
        for name in ("k", "v"):
            x = torch.stack([y.to(torch.float64) for y in (s[name + "_pages"][i] for i in ids.tolist())]) \
                if s[name + "_exp"] is not None else s[name + "_pages"][ids].double()
            if s[name + "_exp"] is not None:
                x = x * torch.pow(2.0, s[name + "_exp"][ids].double() - 127)[..., None]
            kv.append(x.transpose(0, 1).reshape(H, -1, D)[:, tokens])
        q = s["q"][:, r].double().view(H, Hq // H, D)
        z = (q @ kv[0].transpose(1, 2).contiguous()) * D ** -0.5
        lse[:, r] = torch.logsumexp(z, 2).view(-1)
        out[:, r] = (torch.softmax(z, 2) @ kv[1]).reshape(Hq, D)
    return {"out": out, "lse": lse}
