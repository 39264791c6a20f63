"""kv_attend beside promotions: on two streams, in a graph that is replayed behind one, in a capture that begins with one open."""
import numpy as np
import pytest
import torch

from attention_cases import Cache, partition
from paper_2604_26968_b200 import binding as B

pytestmark = pytest.mark.gpu


class World:
    """Six runs of 400 tokens, a third of whose blocks are in the host tier."""

    def __init__(self):
        part = partition("gqa", 32, 8, 128, 0, 16, 170, ring=2_000)
        self.c = c = Cache(part, torch.bfloat16)
        self.table = c.table(150)
        self.suffix = [(25 * i, 400) for i in range(6)]
        self.q = (torch.randn((6, 32, 128), generator=c.gen, device="cuda") * 2.0).to(c.dtype)
        self.before = c.expect(self.q, self.table, self.suffix)
        here = c.entry(self.table[:, c.layer].flatten())
        self.victims = torch.sort(here[torch.randperm(len(here), generator=c.gen, device="cuda")[:400]]).values.to(torch.int32)
        self.d_suffix = torch.tensor(self.suffix, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()

    def demote(self):
        p = self.c.pool
        assert p.kv_demote(self.victims, len(self.victims), 1 << 19) == 0
        p.sync()
        torch.cuda.synchronize()
        return self.c.expect(self.q, self.table, self.suffix)

    def promote(self):
        p = self.c.pool
        _, _, live = p.kv_ring_query(0)
        assert p.kv_promote(0, np.flatnonzero(live), 1 << 19) == 0

    def buffers(self):
        return dict(out=torch.full((6, 32, 128), 7.0, dtype=self.c.dtype, device="cuda"), lse=torch.full((6, 32), 7.0, device="cuda"),
                    scratch=self.c.scratch(6, max_suffix=400))

    def attend(self, b, stream=None):
        return self.c.pool.kv_attend(0, 1, self.q, b["out"], self.table, self.d_suffix, max_suffix=400, scale=128 ** -0.5, d_scratch=b["scratch"],
                                     d_lse=b["lse"], stream=stream)


def test_two_streams_behind_one_promotion():
    w = World()
    streams = [w.c.pool.compute, torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        w.demote()
        work = [(s, w.buffers()) for s in streams[turn:] + streams[:turn]]
        torch.cuda.synchronize()
        w.promote()
        for s, b in work:
            assert w.attend(b, s) == 0
        torch.cuda.synchronize()
        for _, b in work:
            w.c.compare(b["out"], b["lse"], w.before)
    assert w.c.pool.kv_device_status() == 0
    w.c.close()


def test_replays_behind_promotions():
    w = World()
    p, b = w.c.pool, w.buffers()
    assert w.attend(b) == 0
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        assert w.attend(b, stream) == 0
    for _ in range(3):
        without = w.demote()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        w.c.compare(b["out"], b["lse"], without)
        w.promote()
        assert p.kv_join_promotions(stream) == 0
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        w.c.compare(b["out"], b["lse"], w.before)
    assert p.kv_device_status() == 0
    del graph
    w.c.close()


def test_a_capture_while_a_promotion_is_open():
    """The call is refused, the capture goes on; joined, it is taken, on the pool's stream and on another."""
    w = World()
    p, b = w.c.pool, w.buffers()
    w.demote()
    w.promote()
    graph, stream, x = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.zeros(4, device="cuda")
    with torch.cuda.graph(graph, stream=stream):
        assert w.attend(b, stream) == B.KV_ERR_CUDA
        x += 1
    graph.replay()
    assert p.kv_join_promotions() == 0
    for s in (stream, p.compute):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            assert w.attend(b, s) == 0
        p.sync()
        b["out"].zero_()
        g.replay()
        torch.cuda.synchronize()
        w.c.compare(b["out"], b["lse"], w.before)
        del g
    assert x.tolist() == [1.0] * 4
    del graph
    w.c.close()
