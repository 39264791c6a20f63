"""kv_attend where many short runs follow one another through the same warps."""
import pytest
import torch

from attention_cases import Cache, partition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,S", [(("gqa", 16, 4, 64, 0), 1_300), (("gqa", 32, 8, 128, 0), 500)])
def test_runs_that_end_inside_a_unit_one_behind_the_other(shape, S):
    """More runs than there are warps on the GPU (2,368 and 1,776), none of a multiple of 16 tokens, so that what a warp clears behind a
    run's last token lies where the next run's blocks are copied to; the same bits every time."""
    c = Cache(partition(*shape, 16, 3 * S), torch.bfloat16)
    lengths = [1 + (7 * i) % 15 + 16 * (i % 3) for i in range(S)]
    suffix = [(3 * i, n) for i, n in enumerate(lengths)]
    assert S * c.H > 2_368 and all(n % 16 for n in lengths)
    table = c.table(3 * S)
    q = (torch.randn((S, c.part.n_q_heads, c.dk), generator=c.gen, device="cuda") * 2.0).to(c.dtype)
    want = c.expect(q, table, suffix)
    first = None
    for _ in range(10):
        got = c.attend(q, table, suffix)
        if first is None:
            c.compare(*got, want)
            first = got
        for x, y in zip(first, got):
            assert torch.equal(x, y)
    assert c.pool.kv_device_status() == 0
    c.close()
