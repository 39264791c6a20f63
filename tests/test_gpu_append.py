"""kv_append against its definition in 64 bits: axes, layouts, types, slots anywhere, strides, padding, refusals."""
import pytest
import torch

from attention_cases import EPS, NONE, Cache, partition
from paper_2604_26968_b200 import binding as B

pytestmark = pytest.mark.gpu

SHAPES = {"gqa64": ("gqa", 16, 4, 64, 0), "gqa": ("gqa", 32, 8, 128, 0), "mha": ("mha", 5, 5, 80, 0), "mqa": ("mqa", 9, 1, 256, 0),
          "odd": ("gqa", 6, 3, 24, 0), "odd12": ("gqa", 4, 2, 12, 0), "mla": ("mla", 128, 1, 512, 64), "mla_small": ("mla", 3, 1, 40, 8)}
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def cache(shape, block=16, blocks=40, dtype="bf16", **kw):
    arch, qh, h, d, r = SHAPES[shape]
    return Cache(partition(arch, qh, h, d, r, block, blocks), DT[dtype], **kw)


def rotated(x, pos, inv_freq, axis, first, interleaved):
    """In 64 bits, pair by pair; and |x_i cos| + |x_j sin| of each element, for the tolerance."""
    y, size = x.double().clone(), x.double().abs()
    half = len(axis)
    for i in range(half):
        a, b = (first + 2 * i, first + 2 * i + 1) if interleaved else (first + i, first + half + i)
        ang = (pos[axis[i]].double() * inv_freq[i].double())[:, None]
        c, s = ang.cos(), ang.sin()
        u, v = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = u * c - v * s, v * c + u * s
        size[..., a] = size[..., b] = u.abs() + v.abs()
    return y, size


def close(got, want, size, dtype):
    """cos and sin are off by at most 2^-22 (reduction in 64 bits, sincosf's 2 ulp), two products and a sum in 32 bits by 2^-22 more;
    then one rounding to the type (and half its smallest step)."""
    lim = 2.0 ** -21 * size + EPS[dtype] * want.abs() * (1 + 2.0 ** -10) + 2.0 ** -25
    err = (got.double() - want).abs()
    assert bool((err <= lim).all()), float((err / lim).max())


def tensors(c, n, with_q=True):
    p, g = c.part, c.gen
    r = lambda h, d: torch.randn((n, h, d), generator=g, device="cuda").to(c.dtype)  # noqa: E731
    q = r(p.n_q_heads, c.dk) if with_q else None
    return q, r(c.H, c.dk), (r(c.H, c.dv) if c.slab.shape[1] == 2 else None)


def call(c, q, k, v, table, slot, rope, pos, q_out=None, status=0):
    out = torch.full_like(q, 9.0) if q is not None and q_out is None else q_out
    torch.cuda.synchronize()
    rc = c.pool.kv_append(c.q, c.layer, k, v, table, slot, d_q=q, d_q_out=out, rope=rope, d_pos=pos)
    assert rc == 0, rc
    c.pool.sync()
    assert c.pool.kv_device_status() == status
    return out


def check(c, n, slots, table, rot_dim, axis, interleaved=False, first=0, pos=None, with_q=True):
    half = rot_dim // 2
    inv = (10_000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(half, 1))).float()
    n_axes = max(axis) + 1 if axis else 1
    if pos is None:
        pos = torch.randint(0, 3_000, (n_axes, n), generator=c.gen, device="cuda", dtype=torch.int32)
    q, k, v = tensors(c, n, with_q)
    before = c.slab.clone()
    rope = B.kv_rope(rot_dim, axis, inv, first=first, interleaved=interleaved) if half else None
    out = call(c, q, k, v, table, slots, rope, pos if half else None)
    if with_q:
        close(out, *rotated(q, pos, inv, axis, first, interleaved), c.dtype)
    bt = c.part.block_tokens
    kw, size = rotated(k, pos, inv, axis, first, interleaved)
    e = c.entry(table[:, c.layer][slots // bt])                    # [tokens][heads]
    h = e % c.H
    at = (slots % bt)[:, None].expand_as(e)
    got = c.slab[e // c.H, 0, h, at]
    close(got, kw, size, c.dtype)
    before[e // c.H, 0, h, at] = got
    if v is not None:
        assert torch.equal(c.slab[e // c.H, 1, h, at], v)
        before[e // c.H, 1, h, at] = v
    assert torch.equal(c.slab.view(torch.int16), before.view(torch.int16)), "something else was written"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_shapes(shape, interleaved, dtype):
    c = cache(shape, dtype=dtype)
    d = {"mla": 64, "mla_small": 8}.get(shape, c.dk)
    first = c.dk - d
    for n in (1, 2, 77):
        table = c.table(20)
        slots = torch.randperm(20 * 16, generator=c.gen, device="cuda")[:n]
        check(c, n, slots, table, d, [min(2, i * 3 // (d // 2)) for i in range(d // 2)], interleaved, first)
    c.close()


@pytest.mark.parametrize("rot_dim,first", [(0, 0), (2, 0), (6, 3), (64, 0), (64, 64), (32, 8), (126, 1), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_of_a_head(rot_dim, first, interleaved):
    c = cache("gqa")
    check(c, 33, torch.arange(5, 38, device="cuda"), c.table(20), rot_dim, [i % 4 for i in range(rot_dim // 2)], interleaved, first)
    c.close()


def test_far_and_negative_positions():
    c = cache("gqa64")
    pos = torch.tensor([[0, 1, -1, 131_071, 1_000_003, -2_000_000, 2**31 - 1, -2**31]], dtype=torch.int32, device="cuda")
    check(c, 8, torch.arange(8, device="cuda"), c.table(4), 64, [0] * 32, pos=pos)
    c.close()


@pytest.mark.parametrize("block", [1, 7, 64])
def test_prompt_through_blocks(block):
    c = cache("gqa", block=block, blocks=1200 // block)
    rows = 1000 // block
    check(c, 640, torch.arange(3, 643, device="cuda"), c.table(rows), 128, [i // 22 if i < 44 else 2 for i in range(64)])
    c.close()


def test_keys_alone_and_in_place_and_strides():
    c = cache("gqa")
    check(c, 9, torch.arange(9, device="cuda"), c.table(4), 128, [0] * 64, with_q=False)
    n, inv = 12, (500_000.0 ** (-torch.arange(64, device="cuda", dtype=torch.float64) / 64)).float()
    pos = torch.randint(0, 9_000, (1, n), generator=c.gen, device="cuda", dtype=torch.int32)
    table, slots = c.table(8), torch.arange(16, 16 + n, device="cuda")
    rope = B.kv_rope(128, 0, inv)
    for shift in (0, 1, 8):
        wide = torch.zeros(shift + n * 48 * 128, dtype=c.dtype, device="cuda")
        qkv = wide[shift:].view(n, 48 * 128)
        qkv.copy_(torch.randn(qkv.shape, generator=c.gen, device="cuda"))
        q, k, v = qkv[:, :4096].view(n, 32, 128), qkv[:, 4096:5120].view(n, 8, 128), qkv[:, 5120:].view(n, 8, 128)
        want, size = rotated(q, pos, inv, [0] * 64, 0, False)
        kw, ks = rotated(k, pos, inv, [0] * 64, 0, False)
        vw = v.clone()
        call(c, q, k, v, table, slots, rope, pos, q_out=q)          # in place
        close(q, want, size, c.dtype)
        e = c.entry(table[:, c.layer][slots // 16])
        at = (slots % 16)[:, None].expand_as(e)
        close(c.slab[e // 8, 0, e % 8, at], kw, ks, c.dtype)
        assert torch.equal(c.slab[e // 8, 1, e % 8, at], vw)
    c.close()


def test_padding_missing_blocks_and_slots_beyond():
    c = cache("gqa64")
    table = c.table(6)
    table[1, c.layer, 2] = NONE
    q, k, v = tensors(c, 5)
    slots = torch.tensor([-1, 17, 6 * 16, 3, -7], device="cuda")
    pos = torch.zeros((1, 5), dtype=torch.int32, device="cuda")
    before = c.slab.clone()
    rope = B.kv_rope(64, 0, torch.ones(32, device="cuda"))
    out = call(c, q, k, v, table, slots, rope, pos, status=B.KV_DEV_BAD_INDEX | B.KV_DEV_BLOCK_NOT_RESIDENT)
    for t in (0, 2, 4):
        assert bool((out[t] == 9.0).all())
    for t in (1, 3):
        assert torch.equal(out[t], q[t])                          # (angle 0)
        for h in range(4):
            e = int(c.entry(table[int(slots[t]) // 16, c.layer, h]))
            if e >= 0:
                before[e // 4, 0, e % 4, int(slots[t]) % 16] = k[t, h]
                before[e // 4, 1, e % 4, int(slots[t]) % 16] = v[t, h]
    assert torch.equal(c.slab, before)
    c.close()


def test_refusals():
    c = cache("gqa64")
    p, table, slots = c.pool, c.table(4), torch.arange(3, device="cuda")
    q, k, v = tensors(c, 3)
    inv, pos = torch.ones(32, device="cuda"), torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    rope = B.kv_rope(64, 0, inv)
    ok = dict(d_q=q, d_q_out=q.clone(), rope=rope, d_pos=pos)
    assert p.kv_append(0, 1, k, v, table, slots, **ok) == 0
    assert p.kv_append(0, 1, k[:0], v[:0], table, slots[:0], rope=rope, d_pos=pos[:, :0]) == 0
    bad = B.KV_ERR_INVALID_ARG
    assert p.kv_append(0, 2, k, v, table, slots, **ok) == bad
    assert p.kv_append(0, -1, k, v, table, slots, **ok) == bad
    assert p.kv_append(0, 1, k, None, table, slots, **ok) == bad
    assert p.kv_append(0, 1, k, v, table, slots, d_q=q, rope=rope, d_pos=pos) == bad
    assert p.kv_append(0, 1, k, v, table, slots, rope=rope) == bad
    assert p.kv_append(0, 1, k, v, table, slots, rope=B.kv_rope(64, 0, inv, first=2), d_pos=pos) == bad
    assert p.kv_append(0, 1, k, v, table, slots, rope=B.kv_rope(64, 1, inv, n_axes=1), d_pos=pos) == bad
    assert p.kv_append(0, 1, k, v, table, slots, rope=B.kv_rope(64, 4, inv), d_pos=pos.expand(5, 3).contiguous()) == bad
    with pytest.raises(ValueError):
        p.kv_append(0, 1, k[:, :3], v, table, slots, **ok)
    with pytest.raises(TypeError):
        p.kv_append(0, 1, k, v, table, slots.int(), **ok)
    with pytest.raises(ValueError):
        B.kv_rope(64, [0] * 31, inv)
    p.sync()
    c.close()
