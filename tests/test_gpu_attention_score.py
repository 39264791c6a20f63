"""kv_attention_score bit for bit against its definition, its victims, and a run of the operators together."""
import numpy as np
import pytest
import torch

from attention_cases import Cache, partition
from paper_2604_26968_b200 import binding as B
from paper_2604_26968_b200 import workloads as W

pytestmark = pytest.mark.gpu


def definition(acc, weight, tag, state, last, epoch, decay, protect):
    """float32, each operation rounded once."""
    acc, weight = acc.copy(), weight.copy()
    score = np.full(len(tag), np.inf, np.float32)
    live = np.flatnonzero(state == 1)
    g = tag[live]
    acc[g] = np.float32(decay) * acc[g] + weight[g].astype(np.float32) * np.float32(2.0 ** -32)
    weight[g] = 0
    young = (epoch - last[live].astype(np.int64) < protect) & (protect > 0)
    score[live] = np.where(young, np.float32(np.inf), acc[g])
    return acc, weight, score


@pytest.mark.parametrize("decay,protect", [(0.875, 2), (0.0, 0), (1.0, 1), (0.9, 1000)])
@pytest.mark.parametrize("blocks,heads", [(1, 1), (3, 1), (257, 3), (1023, 8), (40_001, 1)])
def test_scores_and_victims(blocks, heads, decay, protect):
    part = W.gqa(1, heads, heads, 8, 16, blocks, max(16, blocks * heads))
    n = part.n_entries
    pool = B.Pool([part], n_tags=2 * n + 8, staging_bytes=1 << 20, max_promote=16, host_meta=False)
    r = np.random.default_rng(blocks * 7 + heads)
    with torch.cuda.stream(pool.compute):
        pool.compute.wait_stream(torch.cuda.default_stream())
        assert pool.kv_admit(0, 0.9, torch.zeros(n, dtype=torch.uint8, device="cuda"), False) == (0, n)
        gone = np.sort(r.permutation(n)[: n // 5]).astype(np.int32)
        if len(gone):
            assert pool.kv_demote(torch.from_numpy(gone).cuda(), len(gone), 1 << 19) == 0
        pool.sync()
        state = pool.state[:n].cpu().numpy()
        tag = np.where(state == 1, r.permutation(2 * n + 8)[:n], 0xFFFFFFFF)
        last = r.integers(0, 12, n)
        pool.tag[:n] = torch.from_numpy(tag.astype(np.uint32).view(np.int32)).cuda()
        pool.loc.fill_(-1)
        pool.loc[torch.from_numpy(tag[state == 1].astype(np.int64)).cuda()] = torch.from_numpy(np.flatnonzero(state == 1).astype(np.int32)).cuda()
        pool.last_epoch[:n] = torch.from_numpy(last.astype(np.int32)).cuda()
        weight = np.where(r.random(2 * n + 8) < 0.2, 0, r.integers(0, 2 ** 44, 2 * n + 8))
        acc = r.random(2 * n + 8, dtype=np.float32)
        d_w, d_a = torch.from_numpy(weight).cuda(), torch.from_numpy(acc).cuda()
        for epoch in (10, 11):
            assert pool.kv_attention_score(epoch, decay, protect, d_w, d_a) == 0
            pool.sync()
            acc, weight, score = definition(acc, weight, tag, state, last, epoch, decay, protect)
            assert np.array_equal(d_a.cpu().numpy().view(np.uint32), acc.view(np.uint32))
            assert np.array_equal(d_w.cpu().numpy(), weight)
            assert np.array_equal(pool.score[:n].cpu().numpy().view(np.uint32), score.view(np.uint32))
        live = int((state == 1).sum())
        for k in {1, live // 3, live} - {0}:
            out = torch.full((max(4, k),), -1, dtype=torch.int32, device="cuda")
            assert pool.kv_select_victims(k, out) == 0
            pool.sync()
            ids = np.flatnonzero(state == 1)
            want = np.sort(ids[np.argsort(score[ids], kind="stable")[:k]])
            assert np.array_equal(out[:k].cpu().numpy(), want)
        assert pool.kv_device_status() == 0
    pool.close()


def test_refusals():
    part = W.gqa(1, 2, 2, 8, 16, 9, 16)
    pool = B.Pool([part], n_tags=18, staging_bytes=1 << 20, max_promote=16, host_meta=False)
    w, a = torch.zeros(20, dtype=torch.int64, device="cuda"), torch.zeros(20, device="cuda")
    torch.cuda.synchronize()
    assert pool.kv_admit(0, 0.9, torch.zeros(18, dtype=torch.uint8, device="cuda"), False) == (0, 18)
    bad = B.KV_ERR_INVALID_ARG
    assert pool.kv_attention_score(1, -0.1, 0, w, a) == bad
    assert pool.kv_attention_score(1, 1.5, 0, w, a) == bad
    assert pool.kv_attention_score(1, float("nan"), 0, w, a) == bad
    assert pool.kv_attention_score(1, 0.5, 2 ** 31, w, a) == bad
    assert pool.kv_attention_score(1, 0.5, 0, w[1:], a) == bad
    with pytest.raises(ValueError):
        pool.kv_attention_score(1, 0.5, 0, w[:17], a)
    with pytest.raises(TypeError):
        pool.kv_attention_score(1, 0.5, 0, w.int(), a)
    pool.close()


def test_handles_that_lead_nowhere_keep_what_they_have():
    part = W.gqa(1, 2, 2, 8, 16, 9, 16)
    pool = B.Pool([part], n_tags=21, staging_bytes=1 << 20, max_promote=16, host_meta=False)
    assert pool.kv_admit(0, 0.9, torch.zeros(18, dtype=torch.uint8, device="cuda"), False) == (0, 18)
    pool.sync()
    w = (torch.arange(1, 22, device="cuda") << 32).contiguous()
    a = torch.full((21,), 2.0, device="cuda")
    pool.loc[19] = -2 ** 31 + 3                      # in the host tier
    torch.cuda.synchronize()
    assert pool.kv_attention_score(1, 0.5, 0, w, a) == 0
    pool.sync()
    assert torch.equal(pool.score[:18], torch.arange(2.0, 20.0, device="cuda"))
    assert w.tolist() == [0] * 18 + [19 << 32, 20 << 32, 21 << 32] and a[18:].tolist() == [2.0] * 3
    assert pool.kv_device_status() == 0
    pool.close()


def test_append_attend_evict_and_promote():
    """A prompt and decoding steps of sequences with a common prefix: tokens enter the cache, attend, the
    blocks with the least weight leave, attention goes on without them, and they come back with what they had gathered."""
    part = partition("gqa", 16, 4, 64, 0, 16, 80, ring=512)
    c = Cache(part, torch.bfloat16, n_tags=2000)
    p, S, L = c.pool, 3, c.layer
    inv = (10_000.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)).float()
    rope = B.kv_rope(64, [0] * 12 + [1] * 10 + [2] * 10, inv)
    table = c.table(40)
    prompt, n_new = 300, 20
    with torch.cuda.stream(p.compute):
        def add(slots, at):
            n = len(slots)
            r = lambda h: torch.randn((n, h, 64), generator=c.gen, device="cuda").to(c.dtype)  # noqa: E731
            q, k, v = r(16), r(4), r(4)
            out = torch.empty_like(q)
            pos = torch.tensor([[a, a // 3, a % 3] for a in at], dtype=torch.int32, device="cuda").t().contiguous()
            assert p.kv_append(0, L, k, v, table, torch.tensor(slots, device="cuda"), d_q=q, d_q_out=out, rope=rope, d_pos=pos) == 0
            return out

        add(list(range(prompt)), list(range(prompt)))
        weight = torch.zeros(p.n_tags, dtype=torch.int64, device="cuda")
        acc = torch.zeros(p.n_tags, device="cuda")
        first = [19 + 2 * s for s in range(S)]                       # two rows for each sequence's own tokens
        scratch = c.scratch(S, 1, max_suffix=32, max_prefix=prompt, max_members=S, weights=True)
        group = torch.tensor([0, S], dtype=torch.int32, device="cuda")
        prefix = torch.tensor([(0, prompt)], dtype=torch.int32, device="cuda")
        total = torch.zeros(p.n_tags, dtype=torch.float64, device="cuda")
        out = torch.empty((S, 16, 64), dtype=c.dtype, device="cuda")
        lse = torch.empty((S, 16), device="cuda")

        def step(i):
            q = add([first[s] * 16 + i for s in range(S)], [prompt + i] * S)
            suffix = [(first[s], i + 1) for s in range(S)]
            assert p.kv_attend(0, L, q, out, table, torch.tensor(suffix, dtype=torch.int32, device="cuda"), max_suffix=32, scale=0.125,
                               d_scratch=scratch, d_prefix=prefix, d_group=group, max_prefix=prompt, max_members=S, d_lse=lse,
                               d_weight=weight) == 0
            p.sync()
            want = c.expect(q, table, suffix, [(0, prompt)], [0, S], scale=0.125)
            c.compare(out, lse, want)
            return want[2]

        for i in range(n_new):
            total += step(i)
        got = weight.double() * 2.0 ** -32
        assert float((got - total).abs().max()) <= 2.0 ** -16 * float(total.max())
        assert p.kv_attention_score(5, 0.5, 0, weight, acc) == 0
        victims = torch.empty(100, dtype=torch.int32, device="cuda")
        assert p.kv_select_victims(100, victims) == 0
        p.sync()
        score = acc[p.tag[: part.n_entries].long()]
        assert set(victims.tolist()) == set(torch.sort(score, stable=True).indices[:100].tolist())
        tags = p.tag[victims.long()].clone()
        kept = acc[tags.long()].clone()
        used = c.entry(table[:19, L])
        assert p.kv_demote(victims, 100, 1 << 19) == 0
        p.sync()
        # blocks with the least weight of the table's are gone; attention passes over them
        again = step(n_new)
        assert bool((again[tags.long()] == 0).all())
        cur, live, mask = p.kv_ring_query(0)
        assert p.kv_promote(0, np.flatnonzero(mask), 1 << 19) == 0
        p.sync()
        assert torch.equal(c.entry(table[:19, L]) >= 0, used >= 0)
        assert torch.equal(acc[tags.long()], kept)
        step(n_new + 1)
        assert p.kv_device_status() == 0
    c.close()


def test_a_captured_step_replayed():
    """Tokens in, attention with weights, score and victims in one graph: its replays do what the calls do."""
    part = partition("gqa", 32, 8, 128, 0, 16, 60, ring=64)
    S, n = 5, 9
    inv = (10_000.0 ** (-torch.arange(64, device="cuda", dtype=torch.float64) / 64)).float()
    rope = B.kv_rope(128, [0] * 20 + [1] * 22 + [2] * 22, inv)

    def world():
        c = Cache(part, torch.bfloat16, seed=3)
        g = c.gen
        r = lambda *x: torch.randn(x, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        table = c.table(40)
        w = dict(c=c, table=table, k=r(n, 8, 128), v=r(n, 8, 128), q=r(n, 32, 128), slot=torch.arange(3, 3 + n, device="cuda"),
                 pos=torch.arange(3 * n, dtype=torch.int32, device="cuda").view(3, n), qs=r(S, 32, 128), out=torch.zeros(S, 32, 128, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros(S, 32, device="cuda"), suffix=torch.tensor([(30 + s, 3 * s) for s in range(S)], dtype=torch.int32, device="cuda"),
                 prefix=torch.tensor([(0, 400)], dtype=torch.int32, device="cuda"), group=torch.tensor([0, 4], dtype=torch.int32, device="cuda"),
                 weight=torch.zeros(c.pool.n_tags, dtype=torch.int64, device="cuda"), acc=torch.zeros(c.pool.n_tags, device="cuda"),
                 victims=torch.zeros(100, dtype=torch.int32, device="cuda"), scratch=c.scratch(S, 1, max_suffix=20, max_prefix=500, max_members=5, weights=True))
        torch.cuda.synchronize()
        return w

    def step(w):
        p = w["c"].pool
        assert p.kv_append(0, 1, w["k"], w["v"], w["table"], w["slot"], d_q=w["q"], d_q_out=w["q"], rope=rope, d_pos=w["pos"]) == 0
        assert p.kv_attend(0, 1, w["qs"], w["out"], w["table"], w["suffix"], max_suffix=20, scale=0.09, d_scratch=w["scratch"], d_prefix=w["prefix"],
                           d_group=w["group"], max_prefix=500, max_members=5, d_lse=w["lse"], d_weight=w["weight"]) == 0
        assert p.kv_attention_score(7, 0.5, 1, w["weight"], w["acc"]) == 0
        assert p.kv_select_victims(100, w["victims"]) == 0

    a, b = world(), world()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=b["c"].pool.compute):
        step(b)
    for _ in range(3):
        step(a)
        a["c"].pool.sync()
        graph.replay()
        torch.cuda.synchronize()
        for x in ("q", "out", "lse", "weight", "acc", "victims"):
            assert torch.equal(a[x], b[x]), x
        assert torch.equal(a["c"].slab.view(torch.int16), b["c"].slab.view(torch.int16))
        assert torch.equal(a["c"].pool.score, b["c"].pool.score)
    del graph
    a["c"].close()
    b["c"].close()
