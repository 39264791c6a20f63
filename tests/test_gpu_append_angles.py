"""kv_append at angles far beyond those of a model's frequencies: their reduction, and heads as wide as they may be."""
import pytest
import torch

from test_gpu_append import cache, call, close, rotated, tensors
from paper_2604_26968_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("top", [1.0, 1_000.0, 1e5])
def test_large_angles(dtype, top):
    """Frequencies up to `top`, positions up to 2^31: angles up to 2 10^14.  The product is rounded to 64 bits by the definition too."""
    c = cache("gqa64", dtype=dtype)
    pos = torch.tensor([[0, 1, -1, 131_071, 1_000_003, -2_000_000, 2**31 - 1, -2**31, 2**31 - 12_345, 1_999_999_999]], dtype=torch.int32, device="cuda")
    inv = (top * torch.rand(32, generator=c.gen, device="cuda")).contiguous()
    inv[0] = top
    table, slots = c.table(4), torch.arange(10, device="cuda")
    q, k, v = tensors(c, 10)
    out = call(c, q, k, v, table, slots, B.kv_rope(64, 0, inv), pos)
    close(out, *rotated(q, pos, inv, [0] * 32, 0, False), c.dtype)
    e = c.entry(table[:, c.layer][slots // 16])
    close(c.slab[e // c.H, 0, e % c.H, (slots % 16)[:, None].expand_as(e)], *rotated(k, pos, inv, [0] * 32, 0, False), c.dtype)
    c.close()
