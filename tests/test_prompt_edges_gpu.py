"""Attention of several new tokens per request at the ends of what its arguments may be, on the GPU."""
import numpy as np
import pytest
import torch

from prompt_cases import DEV, Cache, ints, queries, wide

pytestmark = pytest.mark.gpu


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
