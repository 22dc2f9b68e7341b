"""Plain definition of the paged key-value cache in Python integers and float64:
one step's bookkeeping, the 8-bit values, and the attention of one token."""
import numpy as np

E4M3_MAX = 448.0


def _pages(tokens, page_size):
    return -(-tokens // page_size)


def page_tables(lengths, new_tokens, free_pages, free_count, table, page_size, tokens):
    """The step of ``saf3r_page_tables``, request by request. Returns a dict of
    new arrays: lengths, start, slots, count, table, free."""
    lengths, new, table, free = (np.array(x, dtype=np.int64).copy() for x in (lengths, new_tokens, table, free_pages))
    R, width = table.shape
    pages = len(free)
    capacity = width * page_size
    after = lengths.copy()
    top = min(max(int(free_count), 0), pages)
    good = [0 <= int(n) <= capacity for n in lengths]
    for r in range(R):
        if good[r] and new[r] < 0:
            for j in range(_pages(int(lengths[r]), page_size)):
                if top < pages:
                    free[top] = table[r, j]
                    top += 1
            after[r] = 0
    start = np.zeros(R + 1, dtype=np.int64)
    slots = np.full(tokens, -1, dtype=np.int64)
    out_of_pages = False
    left = top
    for r in range(R):
        grow = max(int(new[r]), 0)
        first = int(start[r])
        start[r + 1] = first + grow
        if not good[r] or new[r] < 0:
            continue
        n = int(lengths[r])
        if n + grow > capacity or first + grow > tokens:
            continue
        held, want = _pages(n, page_size), _pages(n + grow, page_size)
        if want > held and (out_of_pages or want - held > left):
            out_of_pages = True
            continue
        for j in range(held, want):
            left -= 1
            table[r, j] = free[left]
        after[r] = n + grow
        for t in range(grow):
            page, at = divmod(n + t, page_size)
            if 0 <= table[r, page] < pages:
                slots[first + t] = table[r, page] * page_size + at
    return {"lengths": after, "start": np.minimum(start, tokens), "slots": slots, "count": left, "table": table, "free": free}


def e4m3_values():
    """The 256 values of OCP e4m3 (NaN for 0x7f and 0xff)."""
    codes = np.arange(256)
    e, m = (codes >> 3) & 15, codes & 7
    x = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))
    x = np.where(codes & 128, -x, x)
    x[[0x7F, 0xFF]] = np.nan
    return x


def to_e4m3(x):
    """Codes of the nearest e4m3 values, ties to the even code; NaN for what is
    not finite. ``|x| <= 448``."""
    values = e4m3_values()[:127]
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(values, a), 1, 126)
    lo = hi - 1
    up, down = values[hi] - a, a - values[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = code | np.where(np.signbit(x), 128, 0).astype(np.uint8)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def quantise(x):
    """Rows ``[..., dim]`` as codes and exponents: the least e >= -126 with
    max|x| <= 448 * 2^e over the finite values; stored as e + 127."""
    x = np.asarray(x, dtype=np.float64)
    largest = np.abs(np.where(np.isfinite(x), x, 0.0)).max(-1)
    e = np.full(largest.shape, -126)
    while True:
        short = largest > E4M3_MAX * 2.0 ** e
        if not short.any():
            break
        e = e + short
    with np.errstate(invalid="ignore"):
        codes = to_e4m3(x * 2.0 ** -e[..., None].astype(np.float64))
    return codes, (e + 127).astype(np.uint8)


def kept_tokens(n, anchor=0, window=0):
    j = np.arange(n)
    return j if window == 0 else j[(j < anchor) | (j >= n - window)]


def attend(q, k, v, scale):
    """``q [q_heads, dim]`` over ``k``, ``v [tokens, kv_heads, dim]`` (the kept
    tokens): ``(out, lse, size, terms)`` in float64, where ``size`` is the largest
    ``scale * sum |q||k|`` of a score and ``terms`` the sum of weight times |v|."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    Hq, D = q.shape
    n, H, _ = k.shape
    if n == 0:
        zero = np.zeros((Hq, D))
        return zero, np.full(Hq, -np.inf), np.zeros(Hq), zero
    head = np.arange(Hq) // (Hq // H)
    kh, vh = k[:, head].transpose(1, 0, 2), v[:, head].transpose(1, 0, 2)  # [q_heads, n, dim]
    z = scale * (kh @ q[:, :, None])[:, :, 0]
    size = scale * (np.abs(kh) @ np.abs(q)[:, :, None])[:, :, 0].max(1)
    m = z.max(1, keepdims=True)
    w = np.exp(z - m)
    total = w.sum(1, keepdims=True)
    w = w / total
    out = (w[:, None] @ vh)[:, 0]
    return out, (m + np.log(total))[:, 0], size, (w[:, None] @ np.abs(vh))[:, 0]
