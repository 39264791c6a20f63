"""kv_attend against its definition in 64 bits: head layouts, types, lengths from nothing to many chunks, shared
prefixes, holes, garbage behind a run's last token, strides, weights, replays, and refusals."""
import math

import pytest
import torch

from attention_cases import NONE, Cache, partition
from paper_2604_26968_b200 import binding as B

pytestmark = pytest.mark.gpu

SHAPES = {"gqa64": ("gqa", 16, 4, 64, 0), "gqa": ("gqa", 32, 8, 128, 0), "gqa8": ("gqa", 16, 2, 128, 0), "mha": ("mha", 6, 6, 128, 0),
          "mqa": ("mqa", 32, 1, 128, 0), "mqa71": ("mqa", 71, 1, 64, 0), "mqa160": ("mqa", 160, 1, 128, 0), "wide": ("gqa", 8, 2, 256, 0), "odd80": ("gqa", 6, 2, 80, 0),
          "odd8": ("gqa", 3, 3, 8, 0), "mla": ("mla", 128, 1, 512, 64), "mla16": ("mla", 16, 1, 512, 64), "mla_small": ("mla", 5, 1, 64, 16)}
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def cache(shape, block, blocks, dtype="bf16", **kw):
    arch, qh, h, d, r = SHAPES[shape]
    return Cache(partition(arch, qh, h, d, r, block, blocks), DT[dtype], **kw)


def queries(c, S, by=2.0):
    return (torch.randn((S, c.part.n_q_heads, c.dk), generator=c.gen, device="cuda") * by).to(c.dtype)


def runs(lengths, block, first=0):
    """Runs of these lengths, one behind the other in the table; and the rows they take."""
    out = []
    for n in lengths:
        out.append((first, n))
        first += -(-n // block)
    return out, first


def check(c, q, table, suffix, prefix=None, group=None, weights=False, **kw):
    want = c.expect(q, table, suffix, prefix, group)
    w = torch.zeros(c.pool.n_tags, dtype=torch.int64, device="cuda") if weights else None
    out, lse = c.attend(q, table, suffix, prefix, group, weight=w, **kw)
    c.compare(out, lse, want)
    if weights:
        # a row's weight is p_t in 32 bits (2^-18 relative covers scores, exp2, log2 and lse as in compare);
        # each call to the accumulator rounds to 2^-32
        d = (c.dk + 2) * 2.0 ** -24 * float(want[4].max())
        got = w.double() * 2.0 ** -32
        lim = (2.0 ** -18 + 2 * d + 2.0 ** -19 * (1 + float(want[1][torch.isfinite(want[1])].abs().max()) if want[1].isfinite().any() else 1)) * want[2] + 2.0 ** -32 * (2 + q.shape[0])
        err = (got - want[2]).abs()
        assert bool((err <= lim).all()), float((err / lim).max())
    assert c.pool.kv_device_status() == 0
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_suffixes_of_many_lengths(shape, dtype):
    c = cache(shape, 16, 260, dtype)
    lengths = [1, 0, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 511, 700]
    suffix, rows = runs(lengths, 16)
    check(c, queries(c, len(lengths)), c.table(rows), suffix, weights=True)
    c.close()


@pytest.mark.parametrize("length", [0, 1, 77, 128, 129])
@pytest.mark.parametrize("shape", ["gqa64", "gqa", "mqa", "mqa160", "mla"])
def test_one_sequence(shape, length):
    c = cache(shape, 16, 32)
    suffix, rows = runs([length], 16)
    check(c, queries(c, 1), c.table(max(rows, 1)), suffix, weights=True)
    c.close()


@pytest.mark.parametrize("block", [1, 2, 7, 8, 16, 32, 48, 64, 128, 256])
@pytest.mark.parametrize("shape", ["gqa64", "gqa", "mla_small"])
def test_block_sizes(shape, block):
    if shape == "gqa64" and block == 7:
        block = 11
    c = cache(shape, block, 1700 // block + 40)
    suffix, rows = runs([1, 255, 0, 70, 513], block)
    prefix, rows = runs([331], block, rows)
    check(c, queries(c, 5), c.table(rows), suffix, prefix, [1, 4], weights=True)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("members", [1, 2, 5, 17, 40])
@pytest.mark.parametrize("shape", ["gqa64", "gqa", "mha", "mqa", "wide", "odd80", "mla"])
def test_shared_prefixes(shape, members, dtype):
    c = cache(shape, 16, 400, dtype)
    S = members + 3
    suffix, rows = runs([(37 * i) % 90 for i in range(S)], 16)
    prefix, rows = runs([1300, 45], 16, rows)
    # the first group's members, two of another, one without
    check(c, queries(c, S), c.table(rows), suffix, prefix, [0, members, members + 2], weights=True)
    c.close()


@pytest.mark.parametrize("shape", ["gqa", "gqa64", "mla"])
def test_long_prefix_in_many_chunks(shape):
    c = cache(shape, 64, 330)
    suffix, rows = runs([5, 64, 0], 64)
    prefix, rows = runs([19_003], 64, rows)
    check(c, queries(c, 3), c.table(rows), suffix, prefix, [0, 3], weights=True)
    c.close()


@pytest.mark.parametrize("shape", ["gqa64", "gqa", "mqa", "mla"])
@pytest.mark.parametrize("share", [0.3, 0.97, 1.0])
def test_holes(shape, share):
    """Blocks that are nowhere, in the host tier, beyond the handles; whole rows without any."""
    c = cache(shape, 16, 220)
    suffix, rows = runs([200, 40, 0, 333, 16], 16)
    prefix, rows = runs([900, 31], 16, rows)
    table = c.table(rows)
    hole = torch.rand(table.shape, generator=c.gen, device="cuda") < share
    kind = torch.randint(0, 3, table.shape, generator=c.gen, device="cuda")
    demoted = torch.unique(table[hole & (kind == 2)])[:60]
    with torch.cuda.stream(c.pool.compute):
        c.pool.compute.wait_stream(torch.cuda.default_stream())
        victims = demoted.to(torch.int32).clone()
    if victims.numel():
        assert c.pool.kv_demote(victims, victims.numel(), 1 << 19) == 0
    c.pool.sync()
    table[hole & (kind == 0)] = NONE
    table[hole & (kind == 1)] = c.pool.n_tags + 5
    if share == 1.0:
        table[hole & (kind == 2)] = NONE
    check(c, queries(c, 5), table, suffix, prefix, [0, 2, 3], weights=True)
    c.close()


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("shape", ["gqa64", "gqa", "mqa", "odd80", "mla"])
def test_garbage_where_nothing_is(shape, value):
    """What lies behind a run's last token, or in blocks that no handle names, reaches nothing."""
    c = cache(shape, 16, 160)
    suffix, rows = runs([1, 70, 130, 3], 16)
    prefix, rows = runs([333], 16, rows)
    table = c.table(rows)
    used = torch.zeros(c.slab.shape[0] * c.H, dtype=torch.bool, device="cuda")
    used[c.entry(table[:, c.layer]).flatten()] = True
    hole = torch.rand(table.shape, generator=c.gen, device="cuda") < 0.2
    bad = torch.where(used.view(-1, c.H), False, True)
    keep = c.slab.clone()
    c.slab[:] = torch.where(bad[:, None, :, None, None], torch.tensor(value, dtype=c.dtype, device="cuda"), c.slab)
    for row, n in suffix + prefix:
        if n % 16:
            for h in range(c.H):
                e = int(c.entry(table[row + n // 16, c.layer, h]))
                c.slab[e // c.H, :, e % c.H, n % 16:] = value
    e = c.entry(table)[hole].flatten()
    c.slab[e // c.H, :, e % c.H] = value
    table[hole] = NONE
    del keep
    out, lse = check(c, queries(c, 4), table, suffix, prefix, [0, 3], weights=True)
    assert bool(out.isfinite().all())
    c.close()


def test_blocks_named_twice_and_overlapping_runs():
    """Drafts of one sequence: four query tokens, a common prefix, one run of different lengths; and repeated handles."""
    c = cache("gqa", 16, 90)
    table = c.table(60, distinct=False)
    suffix = [(40, 3), (40, 4), (40, 5), (40, 6), (0, 640)]
    check(c, queries(c, 5), table, suffix, [(0, 640)], [0, 4], weights=True)
    c.close()


def test_strides_and_alignment():
    c = cache("gqa", 16, 60)
    S, QH, D = 5, 32, 128
    suffix, rows = runs([90, 1, 64, 200, 33], 16)
    table = c.table(rows)
    dense = queries(c, S)
    want = c.expect(dense, table, suffix)
    for shift, pad_head, pad_seq in ((0, 0, 0), (1, 0, 0), (0, 8, 40), (3, 1, 7)):
        wide = torch.zeros(shift + S * (QH * (D + pad_head) + pad_seq), dtype=c.dtype, device="cuda")
        q = wide[shift:].as_strided((S, QH, D), (QH * (D + pad_head) + pad_seq, D + pad_head, 1), shift)
        q.copy_(dense)
        back = torch.full_like(wide, 5.0)
        out = back.as_strided((S, QH, D), (QH * (D + pad_head) + pad_seq, D + pad_head, 1), shift)
        got, lse = c.attend(q, table, suffix, out=out)
        c.compare(got, lse, want)
        inside = torch.zeros_like(back, dtype=torch.bool)
        inside.as_strided((S, QH, D), out.stride(), shift).fill_(True)
        assert bool((back[~inside] == 5.0).all())
    heads_first = dense.transpose(0, 1).contiguous().transpose(0, 1)
    got, lse = c.attend(heads_first, table, suffix)
    c.compare(got, lse, want)
    c.close()


def test_second_partition_and_foreign_blocks():
    """The second partition of a pool; a handle of the other one is passed over and flagged."""
    other = partition("gqa", 16, 4, 64, 0, 16, 24)
    arch, qh, h, d, r = SHAPES["gqa"]
    c = Cache(partition(arch, qh, h, d, r, 16, 40), torch.bfloat16, before=[other])
    suffix, rows = runs([100, 333], 16)
    table = c.table(rows)
    check(c, queries(c, 2), table, suffix)
    table[3, c.layer, 2] = 5
    q = queries(c, 2)
    out, lse = c.attend(q, table, suffix)
    table[3, c.layer, 2] = NONE
    c.compare(out, lse, c.expect(q, table, suffix))
    assert c.pool.kv_device_status() == B.KV_DEV_BAD_INDEX
    c.close()


def test_bad_runs_count_as_empty():
    c = cache("gqa64", 16, 60)
    good, rows = runs([100, 50, 20], 16)
    table = c.table(rows)
    q = queries(c, 3)
    for bad in ((rows - 1, 17), (rows, 1), (0xFFFFFF, 5), (0, 101)):
        suffix = torch.tensor([good[0], bad, good[2]], dtype=torch.int64).to(torch.int32)
        out, lse = c.attend(q, table, suffix, bounds=dict(max_suffix=100))
        c.compare(out, lse, c.expect(q, table, [good[0], (0, 0), good[2]]))
        assert c.pool.kv_device_status() == B.KV_DEV_BAD_INDEX
    # groups that do not ascend, reach behind the sequences, have too many members
    for group in ([2, 1], [0, 4], [0, 3]):
        out, lse = c.attend(q, table, good, [(0, 60)], group, bounds=dict(max_members=2, max_prefix=60))
        c.compare(out, lse, c.expect(q, table, good))
        assert c.pool.kv_device_status() == B.KV_DEV_BAD_INDEX
    c.close()


def test_large_values():
    """Scores of many hundreds: sums stay finite, the largest wins."""
    c = cache("gqa", 16, 60, spread=8.0)
    suffix, rows = runs([200, 77], 16)
    q = queries(c, 2, by=8.0)
    table = c.table(rows)
    want = c.expect(q, table, suffix)
    out, lse = c.attend(q, table, suffix)
    c.compare(out, lse, want)
    c.close()


@pytest.mark.parametrize("shape", ["gqa", "mla"])
def test_same_results_every_time_and_in_a_graph(shape):
    """A captured call: replayed on other lengths, tables, queries, it gives what a fresh call gives, bit for bit."""
    c = cache(shape, 16, 300)
    lengths = [[200, 1, 90, 333], [17, 333, 0, 64]]
    prefixes = [[700], [650]]
    q, table = queries(c, 4), c.table(140)
    suffix = torch.tensor(runs(lengths[0], 16, 50)[0], dtype=torch.int32, device="cuda")
    prefix = torch.tensor([(0, 700)], dtype=torch.int32, device="cuda")
    group = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    bounds = dict(max_suffix=333, max_prefix=700, max_members=4)
    scratch = c.scratch(4, 1, weights=True, **bounds)
    weight = torch.zeros(c.pool.n_tags, dtype=torch.int64, device="cuda")
    out = torch.empty((4, c.part.n_q_heads, c.dv), dtype=c.dtype, device="cuda")
    lse = torch.empty((4, c.part.n_q_heads), device="cuda")
    s = c.pool.compute
    s.wait_stream(torch.cuda.current_stream())

    def call():
        rc = c.pool.kv_attend(c.q, c.layer, q, out, table, suffix, scale=0.1, d_scratch=scratch, d_prefix=prefix, d_group=group, d_lse=lse,
                              d_weight=weight, **bounds)
        assert rc == 0

    call()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for i in (1, 0, 1):
        first = runs(lengths[i], 16, 50)[0]
        suffix.copy_(torch.tensor(first, dtype=torch.int32))
        prefix.copy_(torch.tensor([(0, prefixes[i][0])], dtype=torch.int32))
        q.copy_(queries(c, 4))
        weight.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a = (out.clone(), lse.clone(), weight.clone())
        scratch.fill_(0x5A)
        weight.zero_()
        torch.cuda.synchronize()
        call()
        c.pool.sync()
        for x, y in zip(a, (out, lse, weight)):
            assert torch.equal(x, y)
        c.compare(out, lse, c.expect(q, table, first, [(0, prefixes[i][0])], [0, 3], scale=0.1))
    del graph
    c.close()


def test_sequences_behind_the_last_are_left_alone():
    c = cache("gqa", 16, 40)
    suffix, rows = runs([30, 200], 16)
    table = c.table(rows)
    q = queries(c, 5)
    back = torch.full((5, 32, 128), 3.0, dtype=c.dtype, device="cuda")
    out, lse = c.attend(q[:2], table, suffix, out=back[:2])
    c.compare(out, lse, c.expect(q[:2], table, suffix))
    assert bool((back[2:] == 3.0).all())
    c.close()


def test_no_sequences_and_refusals():
    c = cache("gqa", 16, 40)
    p = c.pool
    table = c.table(8)
    q, out = queries(c, 2), torch.empty((2, 32, 128), dtype=c.dtype, device="cuda")
    suffix = torch.tensor([(0, 20), (2, 90)], dtype=torch.int32, device="cuda")
    scratch = c.scratch(2, max_suffix=90)
    call = dict(scale=0.1, d_scratch=scratch, max_suffix=90)
    assert p.kv_attend(0, 1, q, out, table, suffix, **call) == 0
    assert p.kv_attend(0, 1, q[:0], out[:0], table, suffix[:0], **call) == 0
    assert p.kv_attend(0, -1, q, out, table, suffix, **call) == B.KV_ERR_INVALID_ARG
    assert p.kv_attend(0, 2, q, out, table, suffix, **call) == B.KV_ERR_INVALID_ARG
    assert p.kv_attend(0, 1, q, out, table, suffix, **{**call, "scale": math.nan}) == B.KV_ERR_INVALID_ARG
    assert p.kv_attend(0, 1, q, out, table, suffix, **{**call, "max_suffix": 50_000}) == B.KV_ERR_INVALID_ARG      # (scratch too small)
    assert p.kv_attend(0, 1, q, out, table, suffix, **{**call, "max_suffix": 0x40000000}) == B.KV_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        p.kv_attend(0, 1, q, out[:1], table, suffix, **call)
    with pytest.raises(ValueError):
        p.kv_attend(0, 1, q, out, table[:, :1], suffix, **call)
    with pytest.raises(TypeError):
        p.kv_attend(0, 1, q.float(), out, table, suffix, **call)
    with pytest.raises(ValueError):
        p.kv_attend(0, 1, q, out.half(), table, suffix, **call)
    p.sync()
    c.close()


@pytest.mark.parametrize("shape,members,plen,block", [("gqa", 64, 9_000, 16), ("gqa", 20, 5_000, 32), ("gqa64", 70, 6_001, 16), ("mqa", 3, 4_000, 64),
                                                      ("mla", 6, 3_000, 64), ("mla", 3, 1_500, 16), ("gqa", 4, 7_000, 16)])
def test_long_runs_give_the_same_bits_every_time(shape, members, plen, block):
    """Many tiles and chunks on all SMs: ten calls, scratch filled with NaN before each."""
    c = cache(shape, block, plen // block + 20 * members + 50)
    S = members + 1
    suffix, rows = runs([(53 * i) % 300 for i in range(S)], block)
    prefix, rows = runs([plen], block, rows)
    table, q = c.table(rows), queries(c, S)
    want = c.expect(q, table, suffix, prefix, [0, members])
    first = None
    for _ in range(10):
        w = torch.zeros(c.pool.n_tags, dtype=torch.int64, device="cuda")
        got = (*c.attend(q, table, suffix, prefix, [0, members], weight=w), w)
        if first is None:
            c.compare(got[0], got[1], want)
            first = got
        for x, y in zip(first, got):
            assert torch.equal(x, y)
    assert c.pool.kv_device_status() == 0
    c.close()


@pytest.mark.parametrize("shape", ["gqa", "gqa64", "mqa71", "mla"])
def test_groups_of_many_and_few_members(shape):
    """One launch for groups on both sides of a row tile; a group of none; prefixes of nothing, one token, many."""
    c = cache(shape, 16, 420)
    sizes = [1, 40, 0, 3, 20, 5]
    starts = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    S = starts[-1] + 2
    suffix, rows = runs([(29 * i) % 70 for i in range(S)], 16)
    prefix, rows = runs([700, 1_111, 5, 0, 64, 1], 16, rows)
    check(c, queries(c, S), c.table(rows), suffix, prefix, starts, weights=True)
    c.close()


@pytest.mark.parametrize("scale", [-0.11, 0.0, 1e-3, 3.0])
@pytest.mark.parametrize("shape,members", [("gqa", 3), ("gqa", 12), ("odd80", 3), ("mla", 2)])
def test_scales(shape, members, scale):
    c = cache(shape, 16, 90)
    suffix, rows = runs([70, 0, 33] + [5] * members, 16)
    prefix, rows = runs([321], 16, rows)
    table, q = c.table(rows), queries(c, members + 3, by=0.5)
    table[2, c.layer, 0] = NONE
    want = c.expect(q, table, suffix, prefix, [0, members], scale=scale)
    out, lse = c.attend(q, table, suffix, prefix, [0, members], scale=scale)
    c.compare(out, lse, want)
    c.close()


def test_two_streams_at_once():
    """Two calls on two streams, each with its own scratch, while the other runs."""
    c = cache("gqa", 16, 500)
    suffix, rows = runs([300] * 12, 16)
    prefix, rows = runs([3_000], 16, rows)
    table = c.table(rows)
    work = []
    for i in range(2):
        q = queries(c, 12)
        want = c.expect(q, table, suffix, prefix, [0, 10 + i])
        b = dict(max_suffix=300, max_prefix=3_000, max_members=11)
        work.append(dict(q=q, want=want, out=torch.empty((12, 32, 128), dtype=c.dtype, device="cuda"), lse=torch.empty((12, 32), device="cuda"),
                         scratch=c.scratch(12, 1, **b), stream=torch.cuda.Stream(), group=torch.tensor([0, 10 + i], dtype=torch.int32, device="cuda"), b=b))
    d_s = torch.tensor(suffix, dtype=torch.int32, device="cuda")
    d_p = torch.tensor(prefix, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for _ in range(8):
        for w in work:
            assert c.pool.kv_attend(0, 1, w["q"], w["out"], table, d_s, scale=128 ** -0.5, d_scratch=w["scratch"], d_prefix=d_p, d_group=w["group"],
                                    d_lse=w["lse"], stream=w["stream"], **w["b"]) == 0
    torch.cuda.synchronize()
    for w in work:
        c.compare(w["out"], w["lse"], w["want"])
    c.close()


def test_infinite_and_nan_queries_stay_in_their_rows():
    c = cache("gqa", 16, 120)
    suffix, rows = runs([64] * 20, 16)
    prefix, rows = runs([500], 16, rows)
    table, q = c.table(rows), queries(c, 20)
    want = c.expect(q, table, suffix, prefix, [0, 18])
    q[3, 5] = math.nan
    q[19, 7] = math.inf
    out, lse = c.attend(q, table, suffix, prefix, [0, 18])
    keep = torch.ones((20, 32), dtype=torch.bool, device="cuda")
    keep[3, 5] = keep[19, 7] = False
    assert bool(out[3, 5].isnan().all()) and bool(lse[3, 5].isnan())
    out, lse = torch.where(keep[..., None], out, want[0].to(c.dtype)), torch.where(keep, lse, want[1].float())
    c.compare(out, lse, want)
    c.close()


@pytest.mark.parametrize("block", [16, 32, 48, 64, 96, 128, 256])
@pytest.mark.parametrize("shape,members", [("gqa", 11), ("gqa64", 40), ("mqa160", 1), ("mla", 2)])
def test_tiles_of_any_block_size(shape, members, block):
    """Runs that end inside a tile, a block, a block longer than a tile; garbage behind their last token."""
    c = cache(shape, block, 3_000 // block + 4 * members + 30)
    S = members + 2
    suffix, rows = runs([(block * i + 7 * i + 1) % 200 for i in range(S)], block)
    prefix, rows = runs([2 * block + 1_017, 65], block, rows)
    table = c.table(rows)
    for row, n in suffix + prefix:
        if n % block:
            for h in range(c.H):
                e = int(c.entry(table[row + n // block, c.layer, h]))
                c.slab[e // c.H, :, e % c.H, n % block:] = math.nan
    table[1, c.layer, 0] = NONE
    check(c, queries(c, S), table, suffix, prefix, [0, members, members + 1], weights=True)
    c.close()
