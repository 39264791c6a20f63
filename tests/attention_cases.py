"""Pools with known K/V for the attention operators' tests, and the operators' definitions in 64 bits.

A pool is filled by the library (handle = entry), its slab and block table are the test's own, so that a table may
name blocks anywhere, twice, or not at all."""
import math

import numpy as np
import torch

from paper_2604_26968_b200 import binding as B
from paper_2604_26968_b200 import workloads as W

NONE = -1
EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative


def partition(arch, q_heads, heads, dim, rope, block, blocks, layers=2, ring=64):
    if arch == "mla":
        p = W.mla(layers, dim, rope, block, blocks, ring)
        p.n_q_heads = p.n_kv_heads = q_heads
        return p
    make = {"gqa": lambda: W.gqa(layers, q_heads, heads, dim, block, blocks, ring),
            "mha": lambda: W.mha(layers, heads, dim, block, blocks, ring),
            "mqa": lambda: W.mqa(layers, q_heads, dim, block, blocks, ring)}
    return make[arch]()


class Cache:
    """One pool, its partition q under test filled with random (or given) elements."""

    def __init__(self, part, dtype=torch.bfloat16, seed=0, before=(), layer=1, spread=1.0, n_tags=None):
        self.parts = list(before) + [part]
        self.part, self.q, self.layer, self.dtype = part, len(before), layer, dtype
        n = sum(p.n_entries for p in self.parts)
        biggest = max(p.entry_bytes for p in self.parts)
        self.pool = B.Pool(self.parts, n_tags=n_tags or 2 * n, staging_bytes=max(1 << 20, 4 * biggest + 4096), max_promote=4096,
                           host_meta=False, stream=torch.cuda.Stream())
        self.pool.compute.wait_stream(torch.cuda.current_stream())
        rc, k = self.pool.kv_admit(0, 0.9, torch.zeros(n, dtype=torch.uint8, device="cuda"), False)
        assert rc == 0 and k == n
        self.base = sum(p.n_entries for p in before)
        self.H = part.heads
        self.dk = part.d_latent + part.d_rope if part.variant == W.MLA else part.head_dim
        self.dv = part.d_latent if part.variant == W.MLA else part.head_dim
        chunks = 1 if part.variant == W.MLA else 2
        self.pool.sync()
        g = torch.Generator(device="cuda").manual_seed(seed)
        slab = self.pool.slabs[self.q].view(dtype)
        slab.copy_((torch.randn(slab.numel(), generator=g, device="cuda") * spread).to(dtype))
        # [layer x block][chunk][head][token][element]
        self.slab = slab.view(part.n_layers * part.blocks_per_layer, chunks, self.H, part.block_tokens, self.dk)
        self.gen = g
        torch.cuda.synchronize()

    def close(self):
        self.pool.close()

    def table(self, rows, distinct=True):
        """Handles [rows][layers][heads] of this partition's entries in random order."""
        n = rows * self.part.n_layers * self.H
        e = self.part.n_entries
        r = (torch.randperm(e, generator=self.gen, device="cuda")[:n] if distinct
             else torch.randint(0, e, (n,), generator=self.gen, device="cuda"))
        assert r.numel() == n
        return (r + self.base).to(torch.int32).view(rows, self.part.n_layers, self.H).contiguous()

    def entry(self, handles):
        """Local entry of each handle, -1 where its block is not in HBM."""
        loc = self.pool.loc.long() & 0xFFFFFFFF
        h = handles.long() & 0xFFFFFFFF
        e = torch.where(h < self.pool.n_tags, loc[h.clamp(max=self.pool.n_tags - 1)], 0xFFFFFFFF)
        return torch.where(e >= 0x80000000, -1, e - self.base)

    def rows_of(self, entries, chunk):
        return self.slab[entries // self.H, chunk, entries % self.H]

    def scratch(self, *a, **k):
        n = self.pool.kv_attend_scratch_bytes(self.q, *a, **k)
        assert n > 0
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    def attend(self, q, table, suffix, prefix=None, group=None, scale=None, weight=None, out=None, bounds=None, scratch=None, lse=True,
               stream=None):
        """The call, with bounds as tight as the lengths; returns (out, lse) after waiting."""
        S = q.shape[0]
        suffix = torch.as_tensor(suffix, dtype=torch.int32, device="cuda").view(-1, 2)
        kw = {}
        b = dict(max_suffix=int(suffix[:, 1].max()) if S else 0, max_prefix=0, max_members=0)
        if prefix is not None:
            prefix = torch.as_tensor(prefix, dtype=torch.int32, device="cuda").view(-1, 2)
            group = torch.as_tensor(group, dtype=torch.int32, device="cuda")
            kw = dict(d_prefix=prefix, d_group=group)
            b["max_prefix"] = int(prefix[:, 1].max()) if len(prefix) else 0
            b["max_members"] = int((group[1:] - group[:-1]).max()) if len(prefix) else 0
        b.update(bounds or {})
        if scratch is None:
            scratch = self.scratch(S, 0 if prefix is None else len(prefix), weights=weight is not None, **b)
            scratch.fill_(0xFF)                    # (NaN wherever a kernel were to read what none has written)
        if out is None:
            out = torch.full((S, self.part.n_q_heads, self.dv), 7.0, dtype=self.dtype, device="cuda")
        lse = torch.full((S, self.part.n_q_heads), 7.0, device="cuda") if lse else None
        torch.cuda.synchronize()
        rc = self.pool.kv_attend(self.q, self.layer, q, out, table, suffix, scale=self.dk ** -0.5 if scale is None else scale,
                                 d_scratch=scratch, d_lse=lse, d_weight=weight, **b, **kw)
        assert rc == 0, rc
        self.pool.sync()
        self.scratch_used = scratch
        return out, lse

    def expect(self, q, table, suffix, prefix=None, group=None, scale=None):
        """(out, lse, weight by handle) in 64 bits, and sum_t p_t |v_t| and sqrt(sum_t p_t^2 v_t^2) for the tolerances."""
        S, QH = q.shape[:2]
        G, bt = QH // self.H, self.part.block_tokens
        scale = self.dk ** -0.5 if scale is None else scale
        out = torch.zeros((S, QH, self.dv), dtype=torch.float64, device="cuda")
        mag = torch.zeros_like(out)
        lse = torch.full((S, QH), -math.inf, dtype=torch.float64, device="cuda")
        weight = torch.zeros(self.pool.n_tags, dtype=torch.float64, device="cuda")
        group = list(group) if group is not None else [0]
        top = torch.zeros((S, QH), dtype=torch.float64, device="cuda")      # largest sum of |q_i k_i| * scale
        for s in range(S):
            segs = [tuple(suffix[s])]
            for g in range(len(group) - 1):
                if group[g] <= s < group[g + 1]:
                    segs.insert(0, tuple(prefix[g]))
            for h in range(self.H):
                hs, at = [], []
                for row, n in segs:
                    t = torch.arange(n, device="cuda")
                    hs.append(table[row + t // bt, self.layer, h].long() & 0xFFFFFFFF)
                    at.append(t % bt)
                hs, at = torch.cat(hs), torch.cat(at)
                e = self.entry(hs)
                hs, at, e = hs[e >= 0], at[e >= 0], e[e >= 0]
                if not e.numel():
                    continue
                k = self.slab[e // self.H, 0, e % self.H, at].double()
                v = k[:, : self.dv] if self.part.variant == W.MLA else self.slab[e // self.H, 1, e % self.H, at].double()
                x = q[s, h * G:(h + 1) * G].double()
                z = x @ k.t() * scale
                p = z.softmax(1)
                out[s, h * G:(h + 1) * G] = p @ v
                mag[s, h * G:(h + 1) * G] = p @ v.abs()
                lse[s, h * G:(h + 1) * G] = z.logsumexp(1)
                top[s, h * G:(h + 1) * G] = (x.abs() @ k.abs().t() * abs(scale)).amax(1)
                weight.index_add_(0, hs, p.sum(0))
        return out, lse, weight, mag, top

    def compare(self, got, lse, want):
        """out and lse against expect().

        Scores: dk products added in 32 bits, and a multiplication: an error of at most (dk + 2) 2^-24 sum|q_i k_i| scale, called d.
        It enters every p_t as a factor exp(+-d) and so does lse (plus the 32-bit rounding of the result, exp2 and log2 approximations
        of 2^-22, and a join of parts): lse is off by d + 2^-20 (1 + |lse|).
        out: p_t is rounded to the elements' type (EPS: half a step, relative) and scores shift it by at most 2 d + 2^-20, so it is
        off by (EPS + 2 d + 2^-19) sum p|v|, and its own rounding adds EPS |out| -- and, for fp16, half the smallest step 2^-25,
        of the output and, as p_t may be below the normal range, of every p_t (at most n 2^-25 max|v|, kept below by spread values)."""
        out, l, _, mag, top = want
        d = (self.dk + 2) * 2.0 ** -24 * top
        empty = torch.isinf(l)
        assert torch.equal(torch.isneginf(lse), empty), "lse of empty rows"
        some = ~empty
        err = (lse.double() - l).abs()[some]
        lim = (d + 2.0 ** -20 * (1 + l.abs()))[some]
        assert bool((err <= lim).all()), ("lse", float((err / lim).max()))
        e = EPS[self.dtype]
        lim = (e + 2 * d[..., None] + 2.0 ** -19) * mag + e * out.abs() + 2.0 ** -24
        if self.dtype == torch.float16:
            lim = lim + 2.0 ** -14 * mag
        err = (got.double() - out).abs()
        assert bool((err <= lim).all()), ("out", float((err / lim).max()))
        assert bool((got[empty] == 0).all())
