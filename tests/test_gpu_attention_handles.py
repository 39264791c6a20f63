"""The attention operators where handles are few, none, or more than one for an entry."""
import math

import pytest
import torch

from paper_2604_26968_b200 import binding as B
from paper_2604_26968_b200 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [0, 8])
def test_a_pool_without_handles(size):
    """Nothing can be admitted: every entry is FREE, attention finds nothing, tokens find no block."""
    part = W.gqa(1, 2, 2, 64, 16, 9, 16)
    pool = B.Pool([part], n_tags=0, staging_bytes=1 << 20, max_promote=16, host_meta=False)
    bf = torch.bfloat16
    w, a = torch.full((size,), 1 << 40, dtype=torch.int64, device="cuda"), torch.full((size,), 2.0, device="cuda")
    table, slot = torch.zeros((3, 1, 2), dtype=torch.int32, device="cuda"), torch.arange(5, device="cuda")
    k, out, lse = torch.ones((5, 2, 64), dtype=bf, device="cuda"), torch.full((1, 2, 64), 7.0, dtype=bf, device="cuda"), torch.zeros((1, 2), device="cuda")
    suffix = torch.tensor([[0, 40]], dtype=torch.int32, device="cuda")
    scratch = torch.empty(pool.kv_attend_scratch_bytes(0, 1, max_suffix=40), dtype=torch.uint8, device="cuda")
    pool.score.fill_(5.0)
    torch.cuda.synchronize()
    assert pool.kv_attention_score(1, 0.5, 0, w, a) == 0
    assert pool.kv_append(0, 0, k, k, table, slot) == 0
    assert pool.kv_attend(0, 0, k[:1], out, table, suffix, max_suffix=40, scale=0.1, d_scratch=scratch, d_lse=lse) == 0
    pool.sync()
    assert bool((pool.score[: part.n_entries] == math.inf).all()) and bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert w.tolist() == [1 << 40] * size and a.tolist() == [2.0] * size
    assert pool.kv_device_status() == B.KV_DEV_BLOCK_NOT_RESIDENT
    pool.close()
