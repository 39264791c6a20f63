"""kv_attend through each of its kernels: strides and alignment of queries and outputs, bounds far above the lengths, many groups,
blocks beyond the first 4 GiB of a slab."""
import pytest
import torch

from attention_cases import Cache, partition

pytestmark = pytest.mark.gpu

# (shape, members of the group): which kernel takes prefix and suffixes
KERNELS = {"tiles128": (("gqa", 32, 8, 128, 0), 11, 16), "tiles64": (("gqa", 16, 4, 64, 0), 40, 16), "tiles one row tile": (("mqa", 160, 1, 128, 0), 1, 32),
           "tiles two teams": (("mqa", 71, 1, 64, 0), 1, 16), "tiles latent": (("mla", 128, 1, 512, 64), 3, 64), "streams": (("gqa", 32, 8, 128, 0), 3, 16),
           "rows 80": (("gqa", 6, 2, 80, 0), 5, 16), "rows 256": (("gqa", 8, 2, 256, 0), 20, 16), "rows, block of 8": (("gqa", 16, 4, 64, 0), 13, 8),
           "latent, few heads": (("mla", 16, 1, 512, 64), 1, 64), "latent, narrow": (("mla", 5, 1, 64, 16), 4, 16)}


class World:
    def __init__(self, name, blocks=0, lengths=None, plen=333, dtype=torch.bfloat16):
        shape, self.members, bt = KERNELS[name]
        S = self.S = self.members + 2
        self.lengths = lengths or [(31 * i + 5) % 90 for i in range(S)]
        first, self.suffix = 0, []
        for n in self.lengths:
            self.suffix.append((first, n))
            first += -(-n // bt)
        self.prefix, rows = [(first, plen)], first + -(-plen // bt)
        self.c = c = Cache(partition(*shape, bt, max(blocks, rows + 5)), dtype)
        self.table = c.table(rows)
        self.group = [0, self.members]
        self.q = (torch.randn((S, c.part.n_q_heads, c.dk), generator=c.gen, device="cuda") * 2.0).to(c.dtype)
        self.want = c.expect(self.q, self.table, self.suffix, self.prefix, self.group)

    def attend(self, q=None, **kw):
        return self.c.attend(self.q if q is None else q, self.table, self.suffix, self.prefix, self.group, **kw)


def strided(dense, shift, pad_head, pad_seq):
    """A view of other memory with these strides, `shift` elements behind its start; and that memory."""
    S, H, D = dense.shape
    wide = torch.full((shift + S * (H * (D + pad_head) + pad_seq) + 8,), 5.0, dtype=dense.dtype, device="cuda")
    return wide.as_strided((S, H, D), (H * (D + pad_head) + pad_seq, D + pad_head, 1), shift), wide


def weight_limit(c, want, members):
    """A row's weight is p_t in 32 bits: scores are off by d (as in Cache.compare), which enters p_t and lse; exp2 and log2 by 2^-22 of 1 + |lse|,
    three times.  Up to 32 threads add a block's rows up, 256 rows at a time, and each rounds to half of 2^-32."""
    d = (c.dk + 2) * 2.0 ** -24 * float(want[4].max())
    top = float(want[1][torch.isfinite(want[1])].abs().max())
    rows = members * (c.part.n_q_heads // c.H)
    return (2.0 ** -18 + 2 * d + 2.0 ** -19 * (1 + top)) * want[2] + 2.0 ** -28 * (1 + rows // 256)


@pytest.mark.parametrize("name", list(KERNELS))
def test_strides_and_alignment(name):
    w = World(name)
    c = w.c
    plain = torch.full((w.S, c.part.n_q_heads, c.dv), 5.0, dtype=c.dtype, device="cuda")
    for prefix, group in ((w.prefix, w.group), (None, None)):
        want = c.expect(w.q, w.table, w.suffix, prefix, group)
        for shift, pad_head, pad_seq in ((0, 8, 40), (1, 0, 0), (2, 4, 2), (4, 4, 4), (3, 1, 7)):
            q, _ = strided(w.q, shift, pad_head, pad_seq)
            q.copy_(w.q)
            out, back = strided(plain, shift, pad_head, pad_seq)
            got, lse = c.attend(q, w.table, w.suffix, prefix, group, out=out)
            c.compare(got, lse, want)
            inside = torch.zeros_like(back, dtype=torch.bool)
            inside.as_strided(out.shape, out.stride(), shift).fill_(True)
            assert bool((back[~inside] == 5.0).all()), "something else was written"
        # heads outermost, and one query for all sequences (stride 0)
        got, lse = c.attend(w.q.transpose(0, 1).contiguous().transpose(0, 1), w.table, w.suffix, prefix, group,
                            out=plain.transpose(0, 1).contiguous().transpose(0, 1))
        c.compare(got, lse, want)
        one = w.q[:1].expand(w.S, -1, -1)
        got, lse = c.attend(one, w.table, w.suffix, prefix, group)
        c.compare(got, lse, c.expect(one, w.table, w.suffix, prefix, group))
    assert c.pool.kv_device_status() == 0
    c.close()


@pytest.mark.parametrize("name", list(KERNELS))
def test_bounds_far_above_the_lengths(name):
    """A captured call keeps the bounds of the longest context: what is not there is neither read nor counted."""
    w = World(name)
    weight = torch.zeros(w.c.pool.n_tags, dtype=torch.int64, device="cuda")
    tight = torch.zeros_like(weight)
    w.attend(weight=tight)
    out, lse = w.attend(weight=weight, bounds=dict(max_suffix=20_000, max_prefix=30_001, max_members=w.S))
    w.c.compare(out, lse, w.want)
    lim = weight_limit(w.c, w.want, w.members)
    for x in (weight, tight):
        assert bool(((x.double() * 2.0 ** -32 - w.want[2]).abs() <= lim).all())
    assert w.c.pool.kv_device_status() == 0
    w.c.close()


@pytest.mark.parametrize("name", ["tiles128", "tiles latent", "streams", "rows 80", "latent, few heads"])
@pytest.mark.parametrize("groups", [31, 32, 33, 75])
def test_many_groups(name, groups):
    """Groups found by a warp (up to 31) and by halving; some empty, some prefixes empty, sequences before, between none, and behind."""
    shape, _, bt = KERNELS[name]
    sizes = [(5 * g) % 3 for g in range(groups)]
    sizes[groups // 2] = 6
    starts = [1]
    for n in sizes:
        starts.append(starts[-1] + n)
    S = starts[-1] + 2
    first, runs = 0, []
    for n in [(7 * i) % 40 for i in range(S)] + [(11 * g) % 50 for g in range(groups)]:
        runs.append((first, n))
        first += -(-n // bt)
    c = Cache(partition(*shape, bt, first + 5), torch.float16)
    table = c.table(first + 1)
    q = torch.randn((S, c.part.n_q_heads, c.dk), generator=c.gen, device="cuda").to(c.dtype)
    want = c.expect(q, table, runs[:S], runs[S:], starts)
    weight = torch.zeros(c.pool.n_tags, dtype=torch.int64, device="cuda")
    out, lse = c.attend(q, table, runs[:S], runs[S:], starts, weight=weight)
    c.compare(out, lse, want)
    lim = weight_limit(c, want, max(sizes))
    assert bool(((weight.double() * 2.0 ** -32 - want[2]).abs() <= lim).all())
    assert c.pool.kv_device_status() == 0
    c.close()


@pytest.mark.parametrize("name", ["tiles128", "streams", "rows 80", "tiles latent"])
def test_blocks_beyond_four_gib(name):
    """All blocks of the table lie behind the first 2^32 bytes of the slab, and are written there by kv_append."""
    shape, members, bt = KERNELS[name]
    part = partition(*shape, bt, 1_000)
    blocks = int(4.4e9 // (part.entry_bytes * part.heads * part.n_layers))
    w = World(name, blocks=blocks)
    c, behind = w.c, 2 ** 32 // w.c.part.entry_bytes + 1
    n = w.table.numel()
    assert c.part.n_entries - behind >= n
    handles = behind + torch.randperm(c.part.n_entries - behind, generator=c.gen, device="cuda")[:n]
    w.table.copy_(handles.to(torch.int32).view_as(w.table))
    k = torch.randn((40, c.H, c.dk), generator=c.gen, device="cuda").to(c.dtype)
    v = torch.randn((40, c.H, c.dv), generator=c.gen, device="cuda").to(c.dtype) if c.slab.shape[1] == 2 else None
    slots = torch.randperm(w.table.shape[0] * bt, generator=c.gen, device="cuda")[:40].contiguous()
    torch.cuda.synchronize()
    assert c.pool.kv_append(0, c.layer, k, v, w.table, slots) == 0
    c.pool.sync()
    e = c.entry(w.table[:, c.layer][slots // bt])
    at = (slots % bt)[:, None].expand_as(e)
    assert torch.equal(c.slab[e // c.H, 0, e % c.H, at], k) and (v is None or torch.equal(c.slab[e // c.H, 1, e % c.H, at], v))
    out, lse = w.attend()
    c.compare(out, lse, c.expect(w.q, w.table, w.suffix, w.prefix, w.group))
    assert c.pool.kv_device_status() == 0
    c.close()
