"""Attention over the pool's blocks, what writes them, and eviction by what it weighs, as measurable cases.

Three operators of a decoding engine whose cache is the pool:

append   new tokens' queries and keys get rotary positions (one axis for text, three for images and
         video: time, height, width), and keys and values are written into the pool's blocks through the
         sequences' block tables
attend   one query token a sequence attends over the pool's blocks; sequences of a group share a prefix.
         With `weights` each block's attention weight is added up by its handle, and the accumulators are
         brought up to date behind it (decay 0: they then hold this step's weights)
evict    the epoch's accumulated attention weight becomes the score of every entry, and the k lowest leave

Blocks lie anywhere: every (position-block, layer, head) of a sequence has a handle of its own, and handles
name entries in random order, as after many demotions and promotions.  Entries that were evicted are holes
(handle KV_NONE) that attention passes over.

Lengths are drawn from a case's plain values alone; contents, tables and positions from the seed.
"""
import math
import random

import torch

own = False

NONE = -1                      # KV_NONE in a table of int32
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- the cases -----------------------------------------------------------------------

def _append(arch, tokens, q_heads, heads, dim, **more):
    c = {"kind": "append", "arch": arch, "tokens": tokens, "q_heads": q_heads, "heads": heads, "dim": dim, "rope": dim,
         "block": 16, "axes": 3, "interleaved": False, "dtype": "bf16", "start": 0}
    c.update(more)
    return c


def _attend(arch, seqs, groups, prefix, suffix, q_heads, heads, dim, **more):
    c = {"kind": "attend", "arch": arch, "seqs": seqs, "groups": groups, "prefix": prefix, "suffix": suffix,
         "q_heads": q_heads, "heads": heads, "dim": dim, "rope": 0, "block": 16, "dtype": "bf16", "holes": 0.0,
         "loose": 0, "weights": False}
    c.update(more)
    return c


def listed():
    return [
        # a decoding step of 64 chats: one token each, text positions far into a long context
        _append("gqa", 64, 32, 8, 128, name="append-decode", axes=1, start=120_000),
        # a video prompt: frames of patches, three axes; an odd number of tokens
        _append("gqa", 16_411, 32, 8, 128, name="append-video"),
        # a prompt of an MLA model: the shared rope part of the latent rows, interleaved pairs
        _append("mla", 4_096, 128, 1, 512, name="append-mla", rope=64, block=64, axes=1, interleaved=True, start=3_000),
        # one short sequence of the tiny test model: the smallest call
        _attend("gqa", 1, 0, 0, 77, 16, 4, 64, name="attend-tiny"),
        # chats in four groups with a system prompt each, ragged; some without; what eviction goes by is added up
        _attend("gqa", 64, 4, 613, 1_500, 32, 8, 128, name="attend-chat", loose=7, weights=True),
        # many samples of one long document (80-layer GQA model): the prefix is most of the work
        _attend("gqa", 64, 1, 32_749, 512, 64, 8, 128, name="attend-document"),
        # a long prefix of an MHA model, fp16, a third of its head-blocks evicted
        _attend("mha", 24, 2, 4_090, 700, 32, 32, 128, name="attend-holes", dtype="fp16", holes=0.33, weights=True),
        # long sequences that share nothing, one KV head for all 32 query heads
        _attend("mqa", 32, 0, 0, 9_001, 32, 1, 128, name="attend-mqa"),
        # agentic sessions of an MLA model over one set of tools
        _attend("mla", 16, 1, 8_200, 1_024, 128, 1, 512, name="attend-mla", rope=64, block=64),
        # the test pool
        {"kind": "evict", "name": "evict-tiny", "heads": 4, "entries": 4_096, "evict": 0.05, "free": 0.0, "protect": 1},
        # a chat pool of 24 GiB, some of it free
        {"kind": "evict", "name": "evict-chat", "heads": 8, "entries": 3_145_728, "evict": 0.10, "free": 0.02, "protect": 2},
        # four models' pool of 150 GiB; an odd number of entries
        {"kind": "evict", "name": "evict-fleet", "heads": 1, "entries": 18_835_041, "evict": 0.10, "free": 0.0, "protect": 2},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


ARCHS = (("gqa", 16, 4, 64, 0), ("gqa", 32, 8, 128, 0), ("gqa", 64, 8, 128, 0), ("mha", 32, 32, 128, 0),
         ("mqa", 32, 1, 128, 0), ("mla", 128, 1, 512, 64))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "evict"])
    if kind == "evict":
        return {"kind": "evict", "heads": rng.choice([1, 4, 8, 32]), "entries": _log_uniform(rng, 2_000, 12_000_000),
                "evict": rng.uniform(0.01, 0.3), "free": rng.choice([0.0, rng.uniform(0.0, 0.3)]), "protect": rng.choice([0, 1, 2, 5])}
    arch, q_heads, heads, dim, rope = rng.choice(ARCHS)
    block = rng.choice([16, 64]) if arch == "mla" else rng.choice([16, 16, 16, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if kind == "append":
        return _append(arch, _log_uniform(rng, 1, 3_500 if arch == "mla" else 9_000), q_heads, heads, dim, rope=rope or rng.choice([dim, dim, dim // 2]),
                       block=block, axes=rng.choice([1, 2, 3, 3]), interleaved=rng.random() < 0.4, dtype=dtype,
                       start=_log_uniform(rng, 1, 1_000_000))
    seqs = _log_uniform(rng, 1, 64)
    groups = rng.choice([0, 1, 1, rng.randint(1, max(1, min(8, seqs // 2)))])
    # (a token of an MHA model has four times the bytes; each of an MLA model's query heads works on all of a row)
    prefix = min(_log_uniform(rng, 1, {"mha": 4_000, "mla": 8_000}.get(arch, 16_000)), 120_000 // seqs if arch == "mla" else 16_000) if groups else 0
    suffix = min(_log_uniform(rng, 1, 4_000), (25_000 if arch in ("mha", "mla") else 100_000) // seqs)
    return _attend(arch, seqs, groups, prefix, suffix, q_heads, heads, dim, rope=rope, block=block, dtype=dtype,
                   holes=rng.choice([0.0, 0.0, rng.uniform(0.0, 0.6)]), loose=rng.randint(0, seqs // 3) if groups else 0,
                   weights=rng.random() < 0.5)


# ---- lengths (from the plain values alone) -------------------------------------------

def _plan(c):
    """(members of each group, prefix tokens of each group, suffix tokens of each sequence); sequences are in the
    groups' order, those without a prefix last."""
    r = random.Random("%d %d %d %d" % (c["seqs"], c["groups"], c["prefix"], c["suffix"]))
    members, left = [], c["seqs"] - c["loose"]
    for g in range(c["groups"]):
        rest = c["groups"] - 1 - g
        n = left if not rest else min(max(1, int(round(left / (rest + 1) * r.uniform(0.6, 1.4)))), left - rest)
        members.append(n)
        left -= n
    prefix = [c["prefix"] if g == 0 else int(c["prefix"] * r.uniform(0.4, 1.0)) for g in range(c["groups"])]
    suffix = [c["suffix"] if s == 0 else max(1, int(c["suffix"] * r.uniform(0.1, 1.0))) for s in range(c["seqs"])]
    if c["groups"] and c["seqs"] > 3:
        suffix[2] = 0                            # a sequence that is its prefix and nothing else
    return members, prefix, suffix


def _blocks(tokens, block):
    return -(-tokens // block)


def _row(c):
    """(elements of a key row, of a value row, chunks of an entry)"""
    return (c["dim"] + c["rope"], c["dim"], 1) if c["arch"] == "mla" else (c["dim"], c["dim"], 2)


def work(c):
    if c["kind"] == "evict":
        # state, handle, last epoch, weight, accumulator read; weight, accumulator, score written; victims
        return {"bytes": c["entries"] * (1 + 4 + 4 + 8 + 4 + 8 + 4 + 4) + 4 * int(c["entries"] * (1 - c["free"]) * c["evict"]),
                "flops": 2 * c["entries"]}
    dk, dv, chunks = _row(c)
    if c["kind"] == "append":
        per = c["q_heads"] * dk * 2 * 2 + c["heads"] * (dk + (dv if chunks == 2 else 0)) * 2 * 2
        return {"bytes": c["tokens"] * (per + 8 + 4 * c["axes"] + 4 * c["heads"] // c["block"]),
                "flops": c["tokens"] * (c["q_heads"] + c["heads"]) * c["rope"] * 3}
    members, prefix, suffix = _plan(c)
    keep = 1 - c["holes"]
    tokens = sum(prefix) + sum(suffix)
    pairs = sum(m * p for m, p in zip(members, prefix)) + sum(suffix)
    kv = tokens * c["heads"] * (dk + (dv if chunks == 2 else 0)) * 2 * keep
    table = 8 * c["heads"] * tokens / c["block"]
    sums = 16 * c["heads"] * tokens / c["block"] if c["weights"] else 0
    return {"bytes": kv + table + sums + c["seqs"] * c["q_heads"] * (2 * dk + 2 * dv + 4),
            "flops": 2 * (dk + dv) * pairs * c["q_heads"] * keep}


# ---- inputs --------------------------------------------------------------------------

LAYERS, LAYER = 2, 1             # a pool of two layers, the second of which is at work


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    return g


def _randn(shape, g, dtype, by=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(by).to(dtype)


def _slab(c, blocks, g):
    """A pool's slab: [layer x block][K, V][head][token][dim], or [layer x block][token][latent + rope]."""
    dk, dv, chunks = _row(c)
    shape = (LAYERS * blocks, 2, c["heads"], c["block"], dk) if chunks == 2 else (LAYERS * blocks, 1, 1, c["block"], dk)
    out = torch.empty(shape, dtype=DTYPES[c["dtype"]], device="cuda")
    step = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3] * shape[4]))
    for at in range(0, shape[0], step):
        out[at:at + step] = _randn((min(step, shape[0] - at),) + shape[1:], g, out.dtype)
    return out


def _table(c, rows, blocks, g):
    """Handles [row][layer][head], each naming another of the pool's entries."""
    n = LAYERS * blocks * c["heads"]
    return torch.randperm(n, generator=g, device="cuda")[: rows * LAYERS * c["heads"]].to(torch.int32).view(rows, LAYERS, c["heads"])


def _pool(s):
    """The framework's pool over a state's inputs: every entry resident, handle = entry."""
    from paper_2604_26968_b200 import binding as B
    from paper_2604_26968_b200 import workloads as W
    c = s["case"]
    if c["kind"] == "evict":
        part = W.gqa(1, c["heads"], c["heads"], 1, 16, s["blocks"], max(16, s["n"] - s["resident"]))
    elif c["arch"] == "mla":
        part = W.mla(LAYERS, c["dim"], c["rope"], c["block"], s["blocks"], 16)
    else:
        make = {"gqa": W.gqa, "mha": lambda L, q, h, d, *a: W.mha(L, h, d, *a), "mqa": lambda L, q, h, d, *a: W.mqa(L, q, d, *a)}[c["arch"]]
        part = make(LAYERS, c["q_heads"], c["heads"], c["dim"], c["block"], s["blocks"], 16)
    pool = B.Pool([part], n_tags=part.n_entries, staging_bytes=max(1 << 20, 2 * part.entry_bytes + 4096), max_promote=16,
                  host_meta=False, stream=torch.cuda.current_stream())
    pairs = torch.zeros(part.n_entries, dtype=torch.uint8, device="cuda")
    rc, n = pool.kv_admit(0, 0.9, pairs, False)
    if rc or n != part.n_entries:
        raise RuntimeError("kv_admit: %d, %d" % (rc, n))
    if c["kind"] == "evict":
        if s["resident"] < s["n"]:      # the free ones have been demoted
            _ok(pool.kv_demote(torch.arange(s["resident"], s["n"], dtype=torch.int32, device="cuda"), s["n"] - s["resident"], 1 << 19))
            pool.sync()
        pool.tag[: s["resident"]] = s["tag"][: s["resident"]]
        pool.loc.fill_(NONE)            # (handles of other entries are nowhere)
        pool.loc[s["tag"][: s["resident"]].long()] = torch.arange(s["resident"], dtype=torch.int32, device="cuda")
        pool.last_epoch[: s["n"]] = s["last_epoch"]
        s["victims"] = torch.empty(max(4, s["k"]), dtype=torch.int32, device="cuda")
    else:
        pool.slabs[0].copy_(s["slab"].view(-1).view(torch.uint8))
        s["slab"] = pool.slabs[0].view(DTYPES[c["dtype"]]).view(s["slab"].shape)   # (one copy of it)
    if c["kind"] == "append":
        s["rope"] = B.kv_rope(c["rope"], s["axis"], s["inv_freq"], first=c["dim"] if c["arch"] == "mla" else 0,
                              interleaved=c["interleaved"])
    if c["kind"] == "attend":
        s["bounds"] = dict(max_suffix=max(s["suffix_len"]), max_prefix=max(s["prefix_len"], default=0), max_members=max(s["members"], default=0))
        s["scratch"] = torch.empty(pool.kv_attend_scratch_bytes(0, c["seqs"], c["groups"], weights=c["weights"], **s["bounds"]),
                                   dtype=torch.uint8, device="cuda")
        if c["weights"]:
            s["weight"] = torch.zeros(pool.n_tags, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    s["pool"] = pool


def prepare(c, seed):
    g = _gen(seed)
    s = {"case": c}
    if c["kind"] == "evict":
        H, n = c["heads"], c["entries"]
        s["blocks"] = n // H
        n = s["n"] = s["blocks"] * H
        s["resident"] = n - int(n * c["free"])
        s["k"] = int(s["resident"] * c["evict"])
        # handles: a block's heads were admitted one after the other, blocks lie anywhere
        s["tag"] = (torch.randperm(s["blocks"], generator=g, device="cuda").to(torch.int32).view(-1, 1) * H
                    + torch.arange(H, device="cuda", dtype=torch.int32)).view(-1)
        # attention weight of an epoch, in units of 2^-32: log-normal, many blocks hardly looked at
        w = torch.randn(n, generator=g, device="cuda").mul_(2.0).sub_(3.0).exp_().clamp_(max=1e5)
        s["weight"] = w.double().mul_(2.0 ** 32).to(torch.int64)
        del w
        s["acc"] = torch.randn(n, generator=g, device="cuda").mul_(1.5).sub_(2.0).exp_()
        s["epoch"] = 40
        s["last_epoch"] = torch.randint(0, s["epoch"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        s["state"] = (torch.arange(n, device="cuda") < s["resident"]).to(torch.uint8)
        s["score"] = torch.empty(n, device="cuda")
    elif c["kind"] == "append":
        dk, dv, chunks = _row(c)
        n, dt = c["tokens"], DTYPES[c["dtype"]]
        need = _blocks(n, c["block"]) + 3
        s["blocks"] = max(8, need + need // 4)
        s["resident"] = LAYERS * s["blocks"] * c["heads"]
        s["slab"] = _slab(c, s["blocks"], g)
        s["table"] = _table(c, need, s["blocks"], g)
        if n <= 256:      # a decoding step: tokens anywhere in the table
            s["slot"] = torch.randperm(need * c["block"], generator=g, device="cuda")[:n].contiguous()
        else:             # a prompt that begins inside a block
            s["slot"] = torch.arange(n, device="cuda") + 5
        # q, k and v side by side, as a projection writes them
        wide = c["q_heads"] * dk + c["heads"] * (dk + (dv if chunks == 2 else 0))
        qkv = _randn((n, wide), g, dt)
        q, k = c["q_heads"] * dk, c["heads"] * dk
        s["q"] = qkv[:, :q].view(n, c["q_heads"], dk)
        s["k"] = qkv[:, q:q + k].view(n, c["heads"], dk)
        s["v"] = qkv[:, q + k:].view(n, c["heads"], dv) if chunks == 2 else None
        s["q_out"] = torch.empty((n, c["q_heads"], dk), dtype=dt, device="cuda")
        # frames of patches behind the text: time, height, width; text: one axis
        at = torch.arange(n, device="cuda", dtype=torch.int32)
        if n <= 256:
            at = torch.randint(0, 4_000, (n,), generator=g, device="cuda", dtype=torch.int32)
        width = max(1, int(math.sqrt(min(n, 1_024)) * 1.3))
        axes = [at if c["axes"] == 1 else at // (width * width), at // width % width, at % width][: c["axes"]]
        s["pos"] = torch.stack(axes) + c["start"]
        half = c["rope"] // 2
        s["axis"] = [min(c["axes"] - 1, i * c["axes"] // half) for i in range(half)]
        s["d_axis"] = torch.tensor(s["axis"], device="cuda")
        s["inv_freq"] = (10_000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)).float()
    else:
        dk, dv, chunks = _row(c)
        dt, bt = DTYPES[c["dtype"]], c["block"]
        s["members"], s["prefix_len"], s["suffix_len"] = _plan(c)
        rows = [_blocks(t, bt) for t in s["prefix_len"] + s["suffix_len"]]
        first = [sum(rows[:i]) for i in range(len(rows))]
        need = sum(rows)
        s["blocks"] = max(8, need + need // 8)
        s["resident"] = LAYERS * s["blocks"] * c["heads"]
        s["slab"] = _slab(c, s["blocks"], g)
        s["table"] = _table(c, need, s["blocks"], g)
        if c["holes"]:
            s["table"][torch.rand(s["table"].shape, generator=g, device="cuda") < c["holes"]] = NONE
        G = c["groups"]
        seg = torch.tensor(list(zip(first, s["prefix_len"] + s["suffix_len"])), dtype=torch.int32, device="cuda").view(-1, 2)
        s["prefix"], s["suffix"] = seg[:G].contiguous(), seg[G:].contiguous()
        starts = [sum(s["members"][:i]) for i in range(G + 1)]
        s["group"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["group_of"] = torch.tensor([g_ for g_, m in enumerate(s["members"]) for _ in range(m)] + [0] * (c["seqs"] - starts[-1]), device="cuda")
        s["place"] = torch.tensor([i for m in s["members"] for i in range(m)] + [0] * (c["seqs"] - starts[-1]), device="cuda")
        s["grouped"] = torch.arange(c["seqs"], device="cuda") < starts[-1]
        s["scale"] = dk ** -0.5
        s["q"] = _randn((c["seqs"], c["q_heads"], dk), g, dt, 2.5)
        s["out"] = torch.empty((c["seqs"], c["q_heads"], dv), dtype=dt, device="cuda")
        s["lse"] = torch.empty((c["seqs"], c["q_heads"]), device="cuda")
        if c["weights"]:
            s["acc"] = torch.zeros(s["resident"], device="cuda")
    if own:
        _pool(s)
    return s


# ---- the operators in their plain form -----------------------------------------------

def _rotate(s, x):
    """x [tokens][heads][dim] with its rotary part turned, in 32 bits; angles in 64."""
    c = s["case"]
    first, half = (c["dim"] if c["arch"] == "mla" else 0), c["rope"] // 2
    angle = s["pos"].double()[s["d_axis"]].t() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    y = x.clone()
    if c["interleaved"]:
        i = torch.arange(half, device="cuda") * 2 + first
        j = i + 1
    else:
        i = torch.arange(half, device="cuda") + first
        j = i + half
    y[..., i] = x[..., i] * cos - x[..., j] * sin
    y[..., j] = x[..., j] * cos + x[..., i] * sin
    return y


def _plain_append(s):
    c, slab = s["case"], s["slab"]
    H, bt = c["heads"], c["block"]
    entry = s["table"][s["slot"] // bt, LAYER].long()                 # [tokens][heads]; handle = entry
    at = (s["slot"] % bt)[:, None].expand(-1, H)
    s["q_out"].copy_(_rotate(s, s["q"]))
    slab[entry // H, 0, entry % H, at] = _rotate(s, s["k"]).to(slab.dtype)
    if s["v"] is not None:
        slab[entry // H, 1, entry % H, at] = s["v"]
    return {"q": s["q_out"], "slab": slab}


def _segment(s, seg):
    """Keys, values [segment][head][token][dim] in 32 bits, which tokens are there, and their handles; the segments padded
    to the longest."""
    c, slab = s["case"], s["slab"]
    H, bt = c["heads"], c["block"]
    longest = max(s["prefix_len"] if seg is s["prefix"] else s["suffix_len"])
    n = max(1, -(-longest // bt))
    row = torch.arange(n, device="cuda")
    inside = row[None] * bt < seg[:, 1:2]
    rows = torch.where(inside, seg[:, :1] + row[None], 0).long()
    handle = torch.where(inside[..., None], s["table"][rows, LAYER], NONE).permute(0, 2, 1).long()   # [seg][head][block]
    e = handle.clamp(min=0)
    k = slab[e // H, 0, e % H].float().flatten(2, 3)
    v = k[..., : c["dim"]] if c["arch"] == "mla" else slab[e // H, 1, e % H].float().flatten(2, 3)
    token = torch.arange(n * bt, device="cuda")
    there = (token < seg[:, 1:2])[:, None] & (handle >= 0).repeat_interleave(bt, 2)
    return k, v, there, handle


def _plain_attend(s):
    c = s["case"]
    S, H, G, bt = c["seqs"], c["heads"], c["q_heads"] // c["heads"], c["block"]
    q = s["q"].float().view(S, H, G, -1)
    k, v, there, handle = _segment(s, s["suffix"])
    score = (q @ k.transpose(2, 3) * s["scale"]).masked_fill_(~there[:, :, None], -math.inf)
    top = score.amax(3)
    shared = c["groups"] > 0 and max(s["prefix_len"]) > 0
    if shared:
        M = max(s["members"])
        kp, vp, there_p, handle_p = _segment(s, s["prefix"])
        qg = torch.zeros((c["groups"], M) + q.shape[1:], device="cuda")
        of, place = s["group_of"][s["grouped"]], s["place"][s["grouped"]]
        qg[of, place] = q[s["grouped"]]
        score_p = (qg.permute(0, 2, 1, 3, 4).flatten(2, 3) @ kp.transpose(2, 3) * s["scale"]).masked_fill_(~there_p[:, :, None], -math.inf)
        score_p = score_p.unflatten(2, (M, G))                           # [group][head][member][query head][token]
        top_p = score_p.amax(4)
        top[s["grouped"]] = torch.maximum(top[s["grouped"]], top_p[of, :, place])
    base = top.masked_fill(top == -math.inf, 0.0)
    p = (score - base[..., None]).exp_()
    total = p.sum(3)
    out = p @ v
    if shared:
        base_g = torch.zeros((c["groups"], M, H, G), device="cuda")
        base_g[of, place] = base[s["grouped"]]
        mine = torch.zeros((c["groups"], M), device="cuda")
        mine[of, place] = 1.0
        p_p = (score_p - base_g.permute(0, 2, 1, 3)[..., None]).exp_() * mine[:, None, :, None, None]
        total[s["grouped"]] += p_p.sum(4)[of, :, place]
        out_p = (p_p.flatten(2, 3) @ vp).unflatten(2, (M, G))
        out[s["grouped"]] += out_p[of, :, place]
    some = total > 0
    out = torch.where(some[..., None], out / total.clamp(min=1e-38)[..., None], 0.0)
    s["out"].copy_(out.view(S, c["q_heads"], -1))
    s["lse"].copy_((base + total.log()).view(S, -1))
    got = {"out": s["out"], "lse": s["lse"]}
    if c["weights"]:
        share = torch.where(some, 1.0 / total, 0.0)
        acc = s["acc"].zero_()
        w = (p * share[..., None]).sum(2).unflatten(2, (-1, bt)).sum(3)
        acc.index_add_(0, handle.clamp(min=0).flatten(), w.flatten())
        if shared:
            share_g = torch.zeros((c["groups"], M, H, G), device="cuda")
            share_g[of, place] = share[s["grouped"]]
            w = (p_p * share_g.permute(0, 2, 1, 3)[..., None]).sum((2, 3)).unflatten(2, (-1, bt)).sum(3)
            acc.index_add_(0, handle_p.clamp(min=0).flatten(), w.flatten())
        got["weight"] = acc
    return got


DECAY = 0.875


def _plain_evict(s):
    tag, here = s["tag"].long(), s["state"] == 1
    new = s["acc"][tag] * DECAY + s["weight"][tag].float() * 2.0 ** -32
    s["acc"][tag] = torch.where(here, new, s["acc"][tag])
    s["weight"][tag] = torch.where(here, 0, s["weight"][tag])
    young = s["epoch"] - s["last_epoch"] < s["case"]["protect"]
    score = torch.where(here & ~young, new, math.inf)
    s["score"].copy_(score)
    order = torch.sort(score, stable=True).indices[: s["k"]]
    return {"acc": s["acc"], "score": s["score"], "victims": order.sort().values.to(torch.int32)}


# ---- one pass ------------------------------------------------------------------------

def _ok(rc):
    if rc:
        raise RuntimeError("kvtier: %d" % rc)


def _own(s):
    c, pool = s["case"], s["pool"]
    if c["kind"] == "append":
        _ok(pool.kv_append(0, LAYER, s["k"], s["v"], s["table"], s["slot"], d_q=s["q"], d_q_out=s["q_out"], rope=s["rope"], d_pos=s["pos"]))
        return {"q": s["q_out"], "slab": s["slab"]}
    if c["kind"] == "attend":
        shared = dict(d_prefix=s["prefix"], d_group=s["group"]) if c["groups"] else {}
        _ok(pool.kv_attend(0, LAYER, s["q"], s["out"], s["table"], s["suffix"], scale=s["scale"], d_scratch=s["scratch"], d_lse=s["lse"],
                           d_weight=s["weight"] if c["weights"] else None, **shared, **s["bounds"]))
        if not c["weights"]:
            return {"out": s["out"], "lse": s["lse"]}
        _ok(pool.kv_attention_score(1, 0.0, 0, s["weight"], s["acc"]))
        return {"out": s["out"], "lse": s["lse"], "weight": s["acc"]}
    _ok(pool.kv_attention_score(s["epoch"], DECAY, c["protect"], s["weight"], s["acc"]))
    _ok(pool.kv_select_victims(s["k"], s["victims"]))
    return {"acc": s["acc"], "score": pool.score[: s["n"]], "victims": s["victims"][: s["k"]]}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[s["case"]["kind"]](s)


# ---- the definitions in 64 bits ------------------------------------------------------

def _exact_append(s):
    c = s["case"]
    first, half = (c["dim"] if c["arch"] == "mla" else 0), c["rope"] // 2
    turn = torch.stack([s["pos"][a].double() * s["inv_freq"][i].double() for i, a in enumerate(s["axis"])], 1)
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]

    def rotated(x):
        x = x.double().clone()
        part = x[..., first:first + 2 * half]
        if c["interleaved"]:
            z = torch.view_as_complex(part.unflatten(2, (half, 2)).contiguous()) * turn
            part.copy_(torch.view_as_real(z).flatten(2))
        else:
            z = torch.complex(part[..., :half], part[..., half:]) * turn
            part[..., :half], part[..., half:] = z.real, z.imag
        return x

    slab = s["slab"].double()
    flat = slab.view(-1, slab.shape[-1])
    k = rotated(s["k"])
    for h in range(c["heads"]):
        e = s["table"][:, LAYER, h].long()[s["slot"] // c["block"]]
        row = ((e // c["heads"]) * slab.shape[1] * slab.shape[2] + e % c["heads"]) * c["block"] + s["slot"] % c["block"]
        flat[row] = k[:, h]
        if s["v"] is not None:
            flat[row + c["heads"] * c["block"]] = s["v"][:, h].double()
    return {"q": rotated(s["q"]), "slab": slab}


def _exact_attend(s):
    c = s["case"]
    H, G, bt = c["heads"], c["q_heads"] // c["heads"], c["block"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    weight = torch.zeros(s["resident"], dtype=torch.float64, device="cuda")
    prefix, suffix = s["prefix"].tolist(), s["suffix"].tolist()
    for i in range(c["seqs"]):
        segs = [suffix[i]]
        if bool(s["grouped"][i]):
            segs.insert(0, prefix[int(s["group_of"][i])])
        for h in range(H):
            handles = torch.cat([s["table"][a:a + -(-n // bt), LAYER, h].long().repeat_interleave(bt)[:n] for a, n in segs])
            where = torch.cat([torch.arange(n, device="cuda") % bt for _, n in segs])
            where, handles = where[handles >= 0], handles[handles >= 0]
            if not len(handles):
                continue
            keys = s["slab"][handles // H, 0, handles % H, where].double()
            values = keys[:, : c["dim"]] if c["arch"] == "mla" else s["slab"][handles // H, 1, handles % H, where].double()
            logits = s["q"][i, h * G:(h + 1) * G].double() @ keys.t() * s["scale"]
            lse[i, h * G:(h + 1) * G] = logits.logsumexp(1)
            prob = logits.softmax(1)
            out[i, h * G:(h + 1) * G] = prob @ values
            weight.index_add_(0, handles, prob.sum(0))
    got = {"out": out, "lse": lse}
    if c["weights"]:
        got["weight"] = weight
    return got


def _exact_evict(s):
    acc, score = s["acc"].double(), torch.full((s["n"],), math.inf, dtype=torch.float64, device="cuda")
    live = torch.nonzero(s["state"]).view(-1)
    tags = s["tag"][live].long()
    acc[tags] = DECAY * acc[tags] + s["weight"][tags].double() / 2 ** 32
    old = s["epoch"] - s["last_epoch"][live] >= s["case"]["protect"]
    score[live[old]] = acc[tags[old]]
    return {"acc": acc, "score": score, "victims": None}


def exact(c, seed):
    s = prepare(c, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[c["kind"]](s)
