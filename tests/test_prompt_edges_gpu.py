"""Attention of one and of several new tokens per request at the ends of what its arguments may be, on the GPU."""
import numpy as np
import pytest
import torch

from oracle import prompt as Q
from prompt_cases import DEV, TYPES, Cache, check, ints, quantised, queries, wide
from test_scores_gpu import slopes_of

pytestmark = pytest.mark.gpu

ALL = ["f32", "bf16", "e4m3", "e2m1"]


def held(dtype, k, v, ps=16):
    """One sequence of the tokens ``k``, ``v [n, kv_heads, dim]`` in a cache: pages, exponents, table, and what it keeps of them."""
    import paper_2607_03612_amd as P

    n, H, D = k.shape
    pages = -(-n // ps)
    raw = torch.uint8 if dtype in ("e4m3", "e2m1") else TYPES[dtype]
    kv = [torch.zeros((pages, H, ps, D // 2 if dtype == "e2m1" else D), dtype=raw, device=DEV).view(TYPES[dtype]) for _ in range(2)]
    shape = (pages, H, ps, D // 32) if dtype == "e2m1" else (pages, H, ps)
    exps = [torch.zeros(shape, dtype=torch.uint8, device=DEV) if raw == torch.uint8 else None for _ in range(2)]
    rows = [torch.from_numpy(np.ascontiguousarray(x.transpose(1, 0, 2))).to(DEV).to(wide(dtype)) for x in (k, v)]
    P.cache_append(*rows, ints(np.arange(n)), *kv, *exps)
    return kv, exps, ints(np.arange(pages)[None]), quantised(k, dtype)[0], quantised(v, dtype)[0]


@pytest.mark.parametrize("dtype", ["bf16", "f32", "e2m1"])
def test_starts_that_go_back_over_long_sequences(gpu_lib, dtype):
    """A tile may fall to a request with many more steps than were counted for it: nothing outside the rows and the
    workspace is touched, and the call ends."""
    import paper_2607_03612_amd as P

    c = Cache(1, dtype, [4096, 4096], 1, 64, 1024, spare=0)
    T = 7168
    q = queries(2, 1, T, 64, dtype)
    lengths = ints([T, 1, 1 << 20])
    table = ints(np.random.default_rng(3).integers(0, c.pages, (3, 1024)))
    need = P.prompt_attention_workspace_bytes(q, *c.kv, table, *c.exps)
    assert need > 0
    room = torch.full((need + 8192,), 0x5A, dtype=torch.uint8, device=DEV)
    ws = room[4096:4096 + need]
    out = torch.full((T + 64, 64), 7.0, dtype=wide(dtype), device=DEV)

    def run(start):
        return P.prompt_attention(q, *c.kv, table, lengths, ints(start), *c.exps, out=out[32:T + 32][None], workspace=ws, want_lse=True)

    right = [0, 2000, 2000, 3584]
    want, want_lse = (x.clone() for x in run(right))
    for start in ([0, T, 0, 3584], [0, T, 0, T], [T, 0, T, 0], [0, 5000, 100, 4000], [2 ** 31 - 1, -2 ** 31, T, 5]):
        print(f"[starts that go back] {dtype} {start}", flush=True)
        run(start)
        torch.cuda.synchronize()
        assert bool((room[:4096] == 0x5A).all()) and bool((room[4096 + need:] == 0x5A).all())
        assert bool((out[:32] == 7).all()) and bool((out[T + 32:] == 7).all())
    got, lse = run(right)
    assert torch.equal(got[:, :3584], want[:, :3584]) and torch.equal(lse[:, :3584], want_lse[:, :3584])


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale,cap", [(2.0 ** 124, 0.125), (0.125, 1e-39), (0.5, 2.0 ** -126)])
def test_a_scale_that_is_large_for_its_cap(gpu_lib, dtype, D, scale, cap):
    """scale / cap near the largest number: keys at right angles to the query have a score of 0, others one of the cap's
    size, in steps that a mask crosses and in those that it does not."""
    import paper_2607_03612_amd as P

    n, T = 600, 70
    rng = np.random.default_rng(D)
    k = np.repeat((np.arange(n) % 3 - 1.0)[:, None, None], D, 2)
    k[200:330] = 0  # whole steps of nothing but 0
    kv, exps, table, k, v = held(dtype, k, rng.standard_normal((n, 1, D)))
    q = torch.full((2, T, D), 2.0 ** -10, dtype=wide(dtype), device=DEV)
    q[1, 3] = 0
    out, lse = P.prompt_attention(q, *kv, table, ints([n]), ints([0, T]), *exps, scale=scale, cap=cap, want_lse=True)
    place = np.arange(n - T, n)
    # tanh is 0 or +-1: so it is at 40 for the oracle, whose bounds then are those of scores of the cap's size
    want = Q.attend(q.double().cpu().numpy(), place, k, v, 40 * cap / (D * 2.0 ** -10), Q.seen(n, place), cap)
    check(out, lse, want, dtype, 0 if dtype == "f32" else 8, n)


def far_scores(D, n, seed=0):
    """Keys of one value each, 3 2^(e - 1) or 2^e with e rising by one every 40 keys: exact in every type."""
    g = np.arange(n) // 20
    k = np.repeat((2.0 ** (10 + g // 2) * np.where(g % 2, 1.5, 1.0))[:, None, None], D, 2)
    return k, np.random.default_rng(seed).standard_normal((n, 1, D))


def far_want(q_value, k, v, D, scale, keep):
    """Scores that far apart leave the keys of the largest one, in equal parts; each score is off by (D + 8) u of its size."""
    z = scale * q_value * D * k[:, 0, 0]
    z = np.where(keep, z, -np.inf)
    top = z.max(1, keepdims=True)
    w = (z == top) / (z == top).sum(1, keepdims=True)
    out = w @ v[:, 0]
    lse = top[:, 0] + np.log((z == top).sum(1))
    return (out[None], lse[None], (D + 8) * 2.0 ** -24 * np.abs(top[None, :, 0]), np.zeros_like(out[None]),
            (w @ np.abs(v[:, 0]) + np.abs(out))[None])


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_value", [2.0 ** 2, 2.0 ** 8, 2.0 ** 13, 1.5 * 2.0 ** 15, -2.0 ** 16, 2.0 ** 40, -2.0 ** 60])
def test_far_scores(gpu_lib, dtype, D, q_value):
    """Scores from 1e5 on, up to 1e25: what is left of a product's rounding behind the maximum is more than an exponent
    holds. A single key, growing ones, and a split along the keys."""
    import paper_2607_03612_amd as P

    for n, T in ((1, 1), (3, 2), (170, 70), (290, 290)):
        k, v = far_scores(D, n)
        kv, exps, table, k, v = held(dtype, k, v)
        q = torch.full((1, T, D), q_value, dtype=wide(dtype), device=DEV)
        out, lse = P.prompt_attention(q, *kv, table, ints([n]), ints([0, T]), *exps, want_lse=True)
        keep = Q.seen(n, np.arange(n - T, n))
        check(out, lse, far_want(q_value, k, v, D, D ** -0.5, keep), dtype, 0 if dtype == "f32" else 8, n)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_value", [2.0 ** 2, 2.0 ** 8, 2.0 ** 13, 1.5 * 2.0 ** 15, -2.0 ** 16, 2.0 ** 40, -2.0 ** 60])
def test_far_scores_of_one_token(gpu_lib, dtype, D, q_value):
    """The same of one token per request: rows whole and shared out, beside a head whose scores are small."""
    import paper_2607_03612_amd as P

    for n in (1, 3, 170, 290):
        k, v = far_scores(D, n)
        kv, exps, table, k, v = held(dtype, k, v)
        q = torch.full((2, 1, D), q_value, dtype=wide(dtype), device=DEV)
        q[1] = 2.0 ** -14
        keep = np.ones((1, n), dtype=bool)
        near = Q.attend(q[1:].double().cpu().numpy(), [n - 1], k, v, D ** -0.5, keep)
        for width in (table.shape[1], 3000):
            wider = torch.zeros((1, width), dtype=torch.int32, device=DEV)
            wider[:, :table.shape[1]] = table
            out, lse = P.paged_attention(q, *kv, wider, ints([n]), *exps, want_lse=True)
            check(out[:1], lse[:1], far_want(q_value, k, v, D, D ** -0.5, keep), dtype, 0 if dtype == "f32" else 16, n)
            check(out[1:], lse[1:], near, dtype, 0 if dtype == "f32" else 16, n)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("q_value", [-2.0 ** 15, -1.5 * 2.0 ** 17, -2.0 ** 40])
def test_far_scores_that_end_near(gpu_lib, dtype, q_value):
    """Scores far below 0, with values of 2^100, ahead of some of 0: nothing of the former is left."""
    import paper_2607_03612_amd as P

    n, T, D = 340, 70, 64
    k, v = far_scores(D, n)
    k[n - T:] = 0
    v[:n - T] *= 2.0 ** 100
    kv, exps, table, k, v = held(dtype, k, v)
    q = torch.full((1, T, D), q_value, dtype=wide(dtype), device=DEV)
    keep = Q.seen(n, np.arange(n - T, n))
    want = far_want(q_value, k, v, D, D ** -0.5, keep)
    assert np.allclose(want[1][0], np.log(np.arange(1, T + 1)))
    out, lse = P.prompt_attention(q, *kv, table, ints([n]), ints([0, T]), *exps, want_lse=True)
    check(out, lse, want, dtype, 0 if dtype == "f32" else 8, n)
    out, lse = P.paged_attention(q[:, T - 1:], *kv, table, ints([n]), *exps, want_lse=True)
    check(out, lse, tuple(x[:, -1:] for x in want), dtype, 0 if dtype == "f32" else 16, n)


def test_far_scores_leave_other_rows(gpu_lib):
    """A row whose scores are far changes no bit of its neighbours'."""
    import paper_2607_03612_amd as P

    c = Cache(3, "bf16", [700], 2, 64, 16)
    q = queries(4, 8, 100, 64, "bf16")
    want, want_lse = P.prompt_attention(q, *c.kv, c.table, c.lengths, ints([0, 100]), want_lse=True)
    q[2, 40] *= 2.0 ** 40
    q[7, 99] *= 2.0 ** 30
    out, lse = P.prompt_attention(q, *c.kv, c.table, c.lengths, ints([0, 100]), want_lse=True)
    for h, t in ((2, 40), (7, 99)):
        top = (q[h, t].double().cpu().numpy() @ c.tokens["k"][0][: 601 + t, h // 4].T).argmax()
        v = c.tokens["v"][0][top, h // 4]
        assert np.all(np.abs(out[h, t].double().cpu().numpy() - v) <= 2.0 ** -7 * np.abs(v)) and bool(lse[h, t].isfinite())
        out[h, t], lse[h, t] = want[h, t], want_lse[h, t]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype", ALL)
def test_read_refuses_rows_in_one_place(gpu_lib, dtype):
    """k and v in one buffer: side by side they are read, on one another refused."""
    import paper_2607_03612_amd as P

    c = Cache(5, dtype, [40], 3, 64, 16)
    slots = ints(np.concatenate([c.table[0, i].item() * 16 + np.arange(16) for i in range(3)])[:40])
    want = P.cache_read(slots, *c.kv, *c.exps)
    for shape, take in (((2, 3, 40, 64), lambda t, i: t[i]), ((3, 2, 40, 64), lambda t, i: t[:, i]), ((40, 3, 2, 64), lambda t, i: t[:, :, i].transpose(0, 1)),
                        ((3, 40, 2, 64), lambda t, i: t[:, :, i])):
        both = torch.full(shape, 7.0, dtype=wide(dtype), device=DEV)
        k, v = take(both, 0), take(both, 1)
        P.cache_read(slots, *c.kv, *c.exps, k=k, v=v)
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    buffer = torch.full((4, 41, 64), 7.0, dtype=wide(dtype), device=DEV)
    for k, v in ((buffer[:3, :40], buffer[:3, :40]), (buffer[:3, :40], buffer[:3, 1:]), (buffer[:3, 1:], buffer[1:, :40]),
                 (buffer[1:, :40], buffer[:3, :40])):
        with pytest.raises(ValueError, match="share"):
            P.cache_read(slots, *c.kv, *c.exps, k=k, v=v)
    torch.cuda.synchronize()
    assert bool((buffer == 7).all())


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [1900.0, 2048.0, 2048.0 * (1 + 2.0 ** -23), 1e5, 1e9])
@pytest.mark.parametrize("size,kind", [(0.02, None), (4.0, None), (0.02, "falling"), (4.0, "falling")])
def test_large_caps(gpu_lib, dtype, D, cap, size, kind):
    """Up to a cap of 2048 a score is off by 5 2^-24 of the cap; beyond by a few roundings of its own, however large the
    cap: tanh's argument and result, both constants and the product, 6 u of the score, less than a tenth of what its sum
    of products may be off by. Steps with and without a mask, and a prefix that all see."""
    import paper_2607_03612_amd as P

    n, T = 700, 80
    c = Cache(6, dtype, [n], 2, D, 16)
    q = queries(7, 4, T, D, dtype, scale=size)
    slopes = None if kind is None else slopes_of(4, kind)
    out, lse = P.prompt_attention(q, *c.kv, c.table, c.lengths, ints([0, T]), *c.exps, prefix=ints([650]), cap=cap, slopes=slopes,
                                  want_lse=True)
    place = np.arange(n - T, n)
    args = (q.double().cpu().numpy(), place, c.tokens["k"][0], c.tokens["v"][0], D ** -0.5, Q.seen(n, place, 650))
    slopes = None if kind is None else slopes.double().cpu().numpy()
    want = Q.attend(*args, cap, slopes)
    if cap > 2048:
        uncapped = Q.attend(*args, 0.0, slopes)
        want = (*want[:2], 1.1 * uncapped[2], 1.1 * uncapped[3], want[4])
    check(out, lse, want, dtype, 0 if dtype == "f32" else 8, n)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,kind", [(0.0, None), (40.0, None), (3000.0, None), (0.0, "falling"), (40.0, "falling")])
def test_large_values_behind_growing_scores(gpu_lib, dtype, D, cap, kind):
    """A value near the largest number whose score is 7 over those before: its product with a weight is no larger than it is."""
    import paper_2607_03612_amd as P

    n, T = 200, 60
    k = np.zeros((n, 1, D))
    v = np.random.default_rng(D).standard_normal((n, 1, D))
    k[150] = 1.0
    v[150] = 1.5 * 2.0 ** 124
    kv, exps, table, k, v = held(dtype, k, v)
    q = torch.full((2, T, D), 7.0 / D, dtype=wide(dtype), device=DEV)
    q[1] = 0.5 / D
    place = np.arange(n - T, n)
    slopes = None if kind is None else slopes_of(2, kind) * 0.01
    more = dict(scale=1.0, cap=cap, slopes=slopes, want_lse=True)
    want = Q.attend(q.double().cpu().numpy(), place, k, v, 1.0, Q.seen(n, place), cap, None if kind is None else slopes.double().cpu().numpy())
    out, lse = P.prompt_attention(q, *kv, table, ints([n]), ints([0, T]), *exps, **more)
    check(out, lse, want, dtype, 0 if dtype == "f32" else 8, n)
    out, lse = P.paged_attention(q[:, T - 1:], *kv, table, ints([n]), *exps, **more)
    check(out, lse, tuple(x[:, -1:] for x in want), dtype, 0 if dtype == "f32" else 16, n)


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,kind", [(0.0, None), (9.0, None), (3000.0, None), (0.0, "falling"), (9.0, "falling")])
def test_rows_that_are_walked_again_leave_the_others(gpu_lib, dtype, D, cap, kind):
    """A query that is NaN, far scores: neither changes a bit of its neighbours', in tiles that one workgroup has whole and in
    ones that several share, with masks by prefix and window."""
    import paper_2607_03612_amd as P

    c = Cache(8, dtype, [900, 300], 2, D, 16)
    q = queries(9, 8, 150, D, dtype, scale=3.0)
    more = dict(prefix=ints([64, 5]), anchor=40, window=500, cap=cap, slopes=None if kind is None else slopes_of(8, kind), want_lse=True)
    want, want_lse = P.prompt_attention(q, *c.kv, c.table, c.lengths, ints([0, 100, 150]), *c.exps, **more)
    q[2, 40, 3], q[5, 149, 0] = float("nan"), float("inf")
    q[7, 99] *= 2.0 ** 40
    out, lse = P.prompt_attention(q, *c.kv, c.table, c.lengths, ints([0, 100, 150]), *c.exps, **more)
    assert bool(out[2, 40].isnan().all()) and bool(lse[2, 40].isnan()) and bool(out[7, 99].isfinite().all())
    for h, t in ((2, 40), (5, 149), (7, 99)):
        out[h, t], lse[h, t] = want[h, t], want_lse[h, t]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
