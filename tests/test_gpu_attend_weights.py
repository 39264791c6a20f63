"""What kv_attend adds to its accumulator."""
import math

import pytest
import torch

from attention_cases import Cache, partition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("arch,members,block", [(("gqa", 32, 8, 128, 0), 18, 16), (("gqa", 16, 4, 64, 0), 40, 16), (("mqa", 71, 1, 64, 0), 3, 8),
                                                (("mla", 128, 1, 512, 64), 5, 64), (("gqa", 8, 2, 128, 0), 4, 16)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_no_numbers_take_nothing_from_the_others(arch, members, block, bad):
    """A query of NaN or infinities in a group: the blocks of the prefix get what the other rows give them.

    Each row's weight is p_t in 32 bits: the scores' error d (dk products added in 32 bits, as in Cache.compare) enters p_t and lse, exp2 and
    log2 are good to 2^-22 of 1 + |lse|, and each addition to the accumulator rounds to 2^-32."""
    S = members + 2
    c = Cache(partition(*arch, block, 700 // block + 10 * S + 10), torch.bfloat16)
    suffix, first = [], 0
    for i in range(S):
        suffix.append((first, 1 + 37 * i % 90))
        first += -(-suffix[-1][1] // block)
    prefix = [(first, 500)]
    table = c.table(first + -(-500 // block))
    q = (torch.randn((S, c.part.n_q_heads, c.dk), generator=c.gen, device="cuda") * 2.0).to(c.dtype)
    clean = c.expect(q, table, suffix, prefix, [0, members])
    G = c.part.n_q_heads // c.H
    places = [(0, 0), (members // 2, c.part.n_q_heads - 1), (members - 1, G // 2), (members, 1)]
    want = torch.zeros_like(clean[2])
    # the weight of the rows that stay: the definition without the bad rows, row by row
    for s in range(S):
        segs = ([prefix[0]] if s < members else []) + [suffix[s]]
        for h in range(c.H):
            keep = [j for j in range(h * G, (h + 1) * G) if (s, j) not in places]
            hs = torch.cat([table[row + torch.arange(n, device="cuda") // block, c.layer, h].long() for row, n in segs])
            at = torch.cat([torch.arange(n, device="cuda") % block for _, n in segs])
            e = c.entry(hs)
            k = c.slab[e // c.H, 0, e % c.H, at].double()
            p = (q[s, keep].double() @ k.t() * c.dk ** -0.5).softmax(1)
            want.index_add_(0, hs, p.sum(0))
    for s, j in places:
        q[s, j] = bad
        if bad == math.inf:
            q[s, j, ::2] = -bad
    w = torch.zeros(c.pool.n_tags, dtype=torch.int64, device="cuda")
    out, lse = c.attend(q, table, suffix, prefix, [0, members], weight=w)
    for s, j in places:
        assert bool(lse[s, j].isnan()) and bool(out[s, j].isnan().all())
        out[s, j], lse[s, j] = clean[0][s, j].to(c.dtype), clean[1][s, j].float()
    c.compare(out, lse, clean)
    d = (c.dk + 2) * 2.0 ** -24 * float(clean[4].max())
    lim = (2.0 ** -18 + 2 * d + 2.0 ** -19 * (1 + float(clean[1].abs().max()))) * want + 2.0 ** -32 * (2 + S)
    err = (w.double() * 2.0 ** -32 - want).abs()
    assert bool((err <= lim).all()), float((err / lim).max())
    c.close()
