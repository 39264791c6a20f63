"""What the host side of kv_append, kv_attend and kv_attention_score refuses, how it cuts the work up, and what the Python
binding refuses, all without a GPU (attention_refusals.cu)."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2604_26968_b200 import binding as B
from paper_2604_26968_b200 import workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_side(tmp_path):
    exe, csrc = str(tmp_path / "refusals"), os.path.join(ROOT, "paper_2604_26968_b200", "csrc")
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a",
                    "-diag-suppress", "186", "--cudart", "none", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", os.path.join(ROOT, "tests"),
                    os.path.join(csrc, "kvtier_host.cu"), os.path.join(csrc, "kv_attention_host.cu"),
                    os.path.join(ROOT, "tests", "attention_refusals.cu"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr


def test_packed_descriptions_are_the_structures():
    assert B._APPEND.size == C.sizeof(B.kv_append_desc) and B._ATTEND.size == C.sizeof(B.kv_attend_desc)
    d = B.kv_attend_desc.from_buffer_copy(B._ATTEND.pack(1, 2, 1, 0.5, 3, 4, 5, 6, 7, 0, 8, 9, 10, 11, 12, 13, 14, 15, 16, 17, 18, 19, 20, 21, 22))
    assert (d.partition, d.layer, d.dtype, d.scale, d.n_seqs, d.n_groups, d.max_suffix, d.max_prefix, d.max_members) == (1, 2, 1, 0.5, 3, 4, 5, 6, 7)
    assert (d.d_q, list(d.q_stride), d.d_out, list(d.out_stride), d.d_lse, d.d_table, d.n_rows) == (8, [9, 10], 11, [12, 13], 14, 15, 16)
    assert (d.d_suffix, d.d_prefix, d.d_group, d.d_weight, d.d_scratch, d.scratch_bytes) == (17, 18, 19, 20, 21, 22)
    rope = B.kv_rope(8, [0, 1, 2, 2], torch.zeros(4), first=3, interleaved=True)
    e = B.kv_append_desc.from_buffer_copy(B._APPEND.pack(1, 2, 1, 0, 3, *range(4, 16), 16, 17, 18, 19, rope.packed))
    assert (e.n_tokens, e.d_k, list(e.k_stride), e.d_v, e.d_q, e.d_q_out, list(e.q_out_stride)) == (3, 4, [5, 6], 7, 10, 13, [14, 15])
    assert (e.d_table, e.n_rows, e.d_slot, e.d_pos) == (16, 17, 18, 19)
    assert (e.rope.rot_dim, e.rope.rot_first, e.rope.interleaved, e.rope.n_axes, list(e.rope.axis[:4])) == (8, 3, 1, 3, [0, 1, 2, 2])


@pytest.fixture
def pool():
    """A binding without a pool behind it: what gets through its own checks is refused by the library."""
    p = B.Pool.__new__(B.Pool)
    p.lib, p._h, p.parts, p.n_tags = B.load(), C.c_void_p(0), [W.gqa(2, 8, 2, 64, 16, 10, 16)], 64
    p.compute = None
    return p


def test_binding_refuses_other_shapes_and_types(pool):
    bf, i32, i64 = torch.bfloat16, torch.int32, torch.int64
    n = 3
    k, q, slot = torch.zeros(n, 2, 64, dtype=bf), torch.zeros(n, 8, 64, dtype=bf), torch.zeros(n, dtype=i64)
    table, pos = torch.zeros(4, 2, 2, dtype=i32), torch.zeros(1, n, dtype=i32)
    rope = B.kv_rope(64, 0, torch.zeros(32))
    call = lambda **x: pool.kv_append(0, 1, **{**dict(d_k=k, d_v=k, d_table=table, d_slot=slot, d_q=q, d_q_out=q, rope=rope, d_pos=pos), **x})  # noqa: E731
    assert call() == B.KV_ERR_INVALID_ARG
    for x in (dict(d_k=k[:, :1]), dict(d_v=k.half()), dict(d_q=q[..., :32]), dict(d_q_out=q[:2]), dict(d_table=table[:, :1]), dict(d_pos=pos[:, :2]),
              dict(d_k=k.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**x)
    for x in (dict(d_k=k.float()), dict(d_slot=slot.int()), dict(d_table=table.long()), dict(d_pos=pos.long())):
        with pytest.raises((TypeError, ValueError)):
            call(**x)
    out, suffix, scratch = q.clone(), torch.zeros(n, 2, dtype=i32), torch.zeros(1 << 16, dtype=torch.uint8)
    prefix, group, lse, w = torch.zeros(1, 2, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(n, 8), torch.zeros(64, dtype=i64)
    call = lambda **x: pool.kv_attend(0, 1, **{**dict(d_q=q, d_out=out, d_table=table, d_suffix=suffix, max_suffix=5, scale=1.0, d_scratch=scratch,  # noqa: E731
                                                      d_prefix=prefix, d_group=group, max_prefix=5, max_members=2, d_lse=lse, d_weight=w), **x})
    assert call() == B.KV_ERR_INVALID_ARG
    for x in (dict(d_out=out[:2]), dict(d_suffix=suffix[:2]), dict(d_group=group[:1]), dict(d_group=None), dict(d_lse=lse[:2]), dict(d_weight=w[:63]),
              dict(d_prefix=prefix.expand(2, 2)), dict(d_scratch=scratch[::2])):
        with pytest.raises(ValueError):
            call(**x)
    for x in (dict(d_q=q.float()), dict(d_suffix=suffix.long()), dict(d_lse=lse.double()), dict(d_weight=w.int())):
        with pytest.raises((TypeError, ValueError)):
            call(**x)
    with pytest.raises(ValueError):
        pool.kv_attention_score(1, 0.5, 0, w[:5], lse)
    with pytest.raises(TypeError):
        pool.kv_attention_score(1, 0.5, 0, w.int(), torch.zeros(64))
