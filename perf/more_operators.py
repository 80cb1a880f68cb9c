"""Operators of a serving loop over an 8-bit cache and over shared prefixes, as cases whose time and outputs can be measured.

Five operators on a paged cache, all methods of ``kvec.KvecSelector``:

* ``append``: ``rotate_append`` into a cache of 8 bits: norms and rotation of queries and keys, then keys and values
  as e4m3 numbers with a scale for each token and head, written as they are quantised.
* ``decode``: ``paged_decode`` over that cache: one new token per sequence, optionally a sliding window, first slots in
  sight and accumulated attention weights.
* ``evict``: ``paged_evict`` of that cache by the accumulated weights; numbers and scales move to new pages.
* ``read``: ``paged_read`` brings a cache's slots back as packed 16-bit rows, as the attention of a prompt's next chunk takes
  them.
* ``shared``: ``shared_decode``, one new token per sequence where groups of sequences share a long prefix, whose keys
  and values are read once for all of them; each sequence's own slots come after it.

``run`` computes them from elementary torch operations in 32 bits, or with ``own`` by the framework's calls.
"""
import math

import torch

own = False   # set from outside: True runs the framework's operators

D = 128
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
E4M3 = torch.float8_e4m3fn
MOST = 448.0             # the largest e4m3 number
LEAST = 2.0 ** -126      # the least scale
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _text(lens):
    return ",".join(str(int(n)) for n in lens)


def _lens(case, key="lens"):
    return [int(n) for n in case[key].split(",")]


# Eight ragged prompts of 4096 to 16384 tokens: the lengths that bench.py's default batch has.
RAGGED8 = "14535,5460,4453,11131,6806,12840,12578,14873"
# Sixty-four conversations of 1024 to 2048 tokens.
BATCH64 = _text(1024 + (389 * i) % 1025 for i in range(64))
# Thirty-two caches of 1000 to 4096 slots; the shortest are within the budget and are kept whole.
BATCH32 = _text(1000 + (997 * i) % 3097 for i in range(32))
# What conversations of 16 to 527 tokens have of their own behind a shared prefix.
TURNS64 = _text(16 + (211 * i) % 512 for i in range(64))
# The same with 1 to 1000 tokens, in three groups of 101, 42 and 17.
TURNS160 = _text(1 + (619 * i) % 1000 for i in range(160))


def _append(name, dtype, q_heads, kv_heads, new, held, page, rot, interleaved, norm):
    return {"name": name, "op": "append", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "new": new,
            "held": held, "page": page, "rot": rot, "interleaved": interleaved, "norm": norm}


def _decode(name, dtype, q_heads, kv_heads, lens, page, window, sinks, weights):
    return {"name": name, "op": "decode", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "lens": lens,
            "page": page, "window": window, "sinks": sinks, "weights": weights}


def _evict(name, dtype, q_heads, kv_heads, lens, page, budget, sinks, recent):
    return {"name": name, "op": "evict", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads,
            "lens": lens, "page": page, "budget": budget, "sinks": sinks, "recent": recent}


def _read(name, dtype, q_heads, kv_heads, lens, first, page, eight):
    return {"name": name, "op": "read", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "lens": lens,
            "first": first, "page": page, "eight": eight}


def _shared(name, dtype, q_heads, kv_heads, prefixes, groups, lens, page, weights):
    return {"name": name, "op": "shared", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "prefixes": prefixes,
            "groups": groups, "lens": lens, "page": page, "weights": weights}


def listed():
    return [
        # One token of one conversation: launch latency is all there is.
        _append("append_one", "bf16", 32, 8, "1", "700", 16, 128, False, True),
        # The prefill of eight ragged prompts, one layer.
        _append("append_prefill", "bf16", 32, 8, RAGGED8, _text([0] * 8), 64, 128, False, True),
        # A decoding step over one compacted cache: the smallest call.
        _decode("decode_short", "bf16", 32, 8, "512", 16, 0, 0, True),
        # A batch of conversations, seven query heads a KV head, weights accumulated for the eviction.
        _decode("decode_batch", "fp16", 28, 4, BATCH64, 64, 0, 0, True),
        # One very long conversation: the cache's length has to be split over the device.
        _decode("decode_long", "bf16", 32, 8, "131072", 128, 0, 0, False),
        # One cache that has grown past its budget by a few dozen tokens.
        _evict("evict_one", "bf16", 32, 8, "576", 16, 512, 4, 32),
        # A batch of caches of different lengths.
        _evict("evict_batch", "fp16", 28, 4, BATCH32, 64, 1024, 4, 128),
        # What the last odd chunk of a chunked prefill attends to.
        _read("read_chunk", "fp16", 28, 4, "1057", "0", 64, True),
        # The caches of eight ragged prompts, whole.
        _read("read_prompts", "bf16", 32, 8, RAGGED8, _text([0] * 8), 64, True),
        # Four answers to one short prompt, sampled side by side.
        _shared("shared_short", "bf16", 32, 8, "500", "4", "1,17,40,23", 16, False),
        # Sixty-four conversations behind one instruction; the own slots' weights are kept for the eviction.
        _shared("shared_batch", "fp16", 28, 4, "4096", "64", TURNS64, 64, True),
        # Three documents that many questions are asked about, the longest by a hundred at once.
        _shared("shared_groups", "bf16", 32, 8, "32768,8001,20000", "101,42,17", TURNS160, 128, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "evict", "read", "shared"])
    dtype = rng.choice(["bf16", "fp16"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (8, 8), (16, 8), (16, 2)])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "append":
        batch = _log(rng, 1, 64)
        top = max(2, 60_000 // batch)
        new = [_log(rng, 1, top) if rng.random() < 0.5 else 1 for _ in range(batch)]
        held = [_log(rng, 1, 4000) for _ in range(batch)]
        return _append("drawn", dtype, q_heads, kv_heads, _text(new), _text(held), page, rng.choice([16, 64, 96, 128]),
                       rng.random() < 0.5, rng.random() < 0.5)
    if op == "decode":
        batch = _log(rng, 1, 64)
        top = 131072 // batch
        lens = [_log(rng, max(1, top // 64), top) for _ in range(batch)]
        window, sinks = (_log(rng, 16, 8192), rng.randrange(0, 17)) if rng.random() < 0.4 else (0, 0)
        return _decode("drawn", dtype, q_heads, kv_heads, _text(lens), page, window, sinks, rng.random() < 0.6)
    if op == "evict":
        batch = _log(rng, 1, 32)
        top = min(32768, 40_000 // batch)
        lens = [_log(rng, max(1, top // 16), top) for _ in range(batch)]
        budget = max(1, int(max(lens) * rng.uniform(0.05, 0.9)))
        sinks = rng.randrange(0, min(8, budget) + 1)
        return _evict("drawn", dtype, q_heads, kv_heads, _text(lens), page, budget, sinks,
                      rng.randrange(0, (budget - sinks) // 2 + 1))
    if op == "read":
        batch = _log(rng, 1, 32)
        top = 80_000 // batch
        lens = [_log(rng, max(1, top // 64), top) for _ in range(batch)]
        # Whole caches, or what a sequence holds from some slot on.
        first = [rng.randrange(0, n) if rng.random() < 0.4 else 0 for n in lens]
        return _read("drawn", dtype, q_heads, kv_heads, _text(lens), _text(first), page, rng.random() < 0.8)
    groups = [_log(rng, 1, 100) for _ in range(rng.randrange(1, 5))]
    while sum(groups) > 160:
        groups.pop()
    prefixes = [_log(rng, 64, 32768 // len(groups)) for _ in groups]
    top = max(2, min(4000, 60_000 // sum(groups)))
    lens = [_log(rng, 1, top) for _ in range(sum(groups))]
    return _shared("drawn", dtype, q_heads, kv_heads, _text(prefixes), _text(groups), _text(lens), page, rng.random() < 0.5)


# ---------------------------------------------------------------- inputs

def _pages_of(lens, page):
    return [(n + page - 1) // page for n in lens]


def _table(counts, gen, first=0):
    """Pages first .. first + sum(counts) - 1 in a shuffled order, one row per sequence; -1 past its pages."""
    perm = (torch.randperm(sum(counts), generator=gen) + first).to(torch.int32)
    table = torch.full((len(counts), max(1, max(counts))), -1, dtype=torch.int32)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = perm[at:at + c]
        at += c
    return table


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cu(lens):
    return torch.tensor([0] + list(lens), dtype=torch.int64).cumsum(0).to(torch.int32)


def prepare(case, seed):
    dev, dt = "cuda", DTYPES[case["dtype"]]
    Hq, Hkv, page, op = case["q_heads"], case["kv_heads"], case["page"], case["op"]
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * std).to(dt)

    def rows(pages):
        """Pages of rows whose sizes differ by token and head: 16-bit ones, or e4m3 numbers and scales."""
        x = torch.randn((pages, Hkv, page, D), generator=gen, device=dev)
        x = x.mul_(torch.randn((pages, Hkv, page, 1), generator=gen, device=dev).mul_(0.4).exp_())
        if not st["eight"]:
            return x.to(dt), None
        scale = (x.abs().amax(-1) / MOST).clamp_(min=LEAST)
        return x.div_(scale[..., None]).to(E4M3), scale

    st = {"case": case, "Hq": Hq, "Hkv": Hkv, "dtype": dt, "eight": op in ("append", "decode", "evict") or case.get("eight", False)}
    counts_before = 0
    if op == "append":
        new, held = _lens(case, "new"), _lens(case, "held")
        lens = [a + b for a, b in zip(new, held)]      # with the new tokens counted
        T, rot = sum(new), case["rot"]
        # One projection's output: queries, keys and values of a token side by side.
        qkv = normal(T, Hq + 2 * Hkv, D)
        inv = 1.0 / 10000.0 ** (torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot)
        angle = torch.arange(max(lens), dtype=torch.float64, device=dev)[:, None] * inv
        st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], new=new,
                  cu=_cu(new).to(dev), positions=_ints([h + i for n, h in zip(new, held) for i in range(n)]),
                  rot_table=torch.cat([angle.cos(), angle.sin()], 1).float())
        st["norms"] = (normal(D, std=0.2) + 1, normal(D, std=0.2) + 1) if case["norm"] else (None, None)
    else:
        lens = _lens(case)
    if op == "shared":
        prefixes, groups = _lens(case, "prefixes"), _lens(case, "groups")
        held = _pages_of(prefixes, page)
        counts_before = sum(held)
        st.update(prefix_table=_table(held, host).to(dev), prefix_lens=_ints(prefixes), cu_seqs=_cu(groups).to(dev),
                  max_prefix=max(prefixes), max_group=max(groups))
    counts = _pages_of(lens, page)
    spare = _pages_of([min(n, case["budget"]) for n in lens], page) if op == "evict" else []
    pages = counts_before + sum(counts) + sum(spare)
    st.update(lens=_ints(lens), max_len=max(lens), page_table=_table(counts, host, first=counts_before).to(dev))
    st["k_pages"], st["k_scales"] = rows(pages)
    st["v_pages"], st["v_scales"] = rows(pages)
    if op in ("decode", "shared"):
        # Queries of trained models look at some keys far more than at others: a wider spread than the keys'.
        st["q"] = normal(len(lens), Hq, D, std=2.0)
    if op == "evict":
        st["new_table"] = _table(spare, host, first=sum(counts)).to(dev)
    if op == "read":
        first = _lens(case, "first")
        cu = _cu([n - f for n, f in zip(lens, first)])
        st.update(first=_ints(first), cu=cu.to(dev), rows=int(cu[-1]))
    if op == "evict" or case.get("weights"):
        # Accumulated weights span decades: a few slots hold most of the attention.
        st["weights"] = torch.randn((pages, Hkv, page), generator=gen, device=dev).mul_(2.0).exp_()
    else:
        st["weights"] = None
    return st


# ---------------------------------------------------------------- the plain forms

def _slot_rows(table, slots, Hkv, page):
    """Row numbers, in the pages seen as rows, of slots [..., n] of the tables [batch, pages]: [batch, Hkv, n]."""
    at = table.long().clamp(min=0).gather(1, (slots // page).clamp(max=table.shape[1] - 1)) * Hkv
    heads = torch.arange(Hkv, device=table.device)
    return (at[:, None, :] + heads[None, :, None]) * page + (slots % page)[:, None, :]


def _values(pages, scales, rows):
    """The numbers, in 32 bits, that rows of a cache stand for."""
    if scales is None:
        return pages.view(-1, D)[rows].float()
    return pages.view(torch.uint8).view(-1, D)[rows].view(E4M3).float() * scales.view(-1)[rows][..., None]


def _rotated(x, norm, cos, sin, rot, interleaved):
    x = x.float()
    if norm is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * norm.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _store(pages, scales, rows, x):
    scale = (x.abs().amax(-1) / MOST).clamp(min=LEAST)
    pages.view(torch.uint8).view(-1, D)[rows] = (x / scale[..., None]).to(E4M3).view(torch.uint8)
    scales.view(-1)[rows] = scale


def _plain_append(st):
    case, dt, Hkv = st["case"], st["dtype"], st["Hkv"]
    page, rot = case["page"], case["rot"]
    at = st["rot_table"][st["positions"].long()][:, None, :]
    cos, sin = at[..., :rot // 2], at[..., rot // 2:]
    q = _rotated(st["q"], st["norms"][0], cos, sin, rot, case["interleaved"]).to(dt)
    k = _rotated(st["k"], st["norms"][1], cos, sin, rot, case["interleaved"])
    cu, token = st["cu"].long(), torch.arange(q.shape[0], device=q.device)
    seq = torch.searchsorted(cu[1:], token, right=True)
    slot = st["lens"].long()[seq] - (cu[seq + 1] - token)
    rows = (st["page_table"].long()[seq, slot // page] * Hkv)[:, None] + torch.arange(Hkv, device=q.device)
    rows = rows * page + (slot % page)[:, None]
    _store(st["k_pages"], st["k_scales"], rows, k)
    _store(st["v_pages"], st["v_scales"], rows, st["v"].float())
    return q, st["k_pages"], st["k_scales"], st["v_pages"], st["v_scales"]


def _visible(j, n, case):
    seen = j < n
    if case.get("window"):
        seen = seen & ((j >= n - case["window"]) | (j < case["sinks"]))
    return seen


def _own_logits(st):
    """Every sequence's own slots: rows [batch, Hkv, n], values, logits [batch, Hkv, g, n], which of them are seen."""
    case, Hkv, page = st["case"], st["Hkv"], st["case"]["page"]
    batch = st["q"].shape[0]
    j = torch.arange(st["max_len"], device="cuda")
    rows = _slot_rows(st["page_table"], j[None, :].expand(batch, -1), Hkv, page)
    k, v = _values(st["k_pages"], st["k_scales"], rows), _values(st["v_pages"], st["v_scales"], rows)
    seen = _visible(j[None, :], st["lens"].long()[:, None], case)[:, None, None, :]
    x = (st["q"].float().view(batch, Hkv, -1, D) @ k.transpose(-1, -2)) * SCALE
    return rows, v, x.masked_fill(~seen, -math.inf), seen


def _add_weights(st, rows, p, seen):
    here = seen.expand(-1, st["Hkv"], -1, -1).squeeze(2)
    st["weights"].view(-1).index_put_((rows[here],), p.sum(2)[here], accumulate=True)


def _plain_decode(st):
    rows, v, x, seen = _own_logits(st)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = (p @ v).reshape(st["q"].shape).to(st["dtype"])
    if st["weights"] is None:
        return (out,)
    _add_weights(st, rows, p, seen)
    return out, st["weights"]


def _plain_evict(st):
    case, Hkv, page, B = st["case"], st["Hkv"], st["case"]["page"], st["case"]["budget"]
    n = st["lens"].long()
    batch = n.shape[0]
    j = torch.arange(st["max_len"], device="cuda")[None, :]
    rows = _slot_rows(st["page_table"], j.expand(batch, -1), Hkv, page)
    w = st["weights"].view(-1)[rows]
    w = w.masked_fill(w.isnan(), -math.inf)
    always = (j < case["sinks"]) | (j >= n[:, None] - case["recent"])
    w = w.masked_fill(always[:, None, :], math.inf).masked_fill((j >= n[:, None])[:, None, :], -math.inf)
    held = (j < n[:, None])[:, None, :].expand(-1, Hkv, -1)
    # By weight, then by slot; slots past the end behind all others.
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(held.gather(-1, order).int(), dim=-1, descending=True, stable=True).indices)
    kept = order[..., :B]
    new_lens = n.clamp(max=B)
    valid = torch.arange(kept.shape[-1], device="cuda") < new_lens[:, None, None]
    kept = kept.masked_fill(~valid, st["max_len"]).sort(-1).values
    valid = kept < st["max_len"]
    src = rows.gather(-1, kept.clamp(max=st["max_len"] - 1))
    to = torch.arange(kept.shape[-1], device="cuda")[None, :].expand(batch, -1)
    dst = _slot_rows(st["new_table"], to, Hkv, page)
    src, dst = src[valid], dst[valid]
    flat = [st[x].view(torch.uint8).view(-1, D) for x in ("k_pages", "v_pages")]
    flat += [st[x].view(-1) for x in ("k_scales", "v_scales", "weights")]
    moved = [x[src] for x in flat]
    _ = [x.index_copy_(0, dst, y) for x, y in zip(flat, moved)]
    out = torch.full((batch, Hkv, B), -1, dtype=torch.int32, device="cuda")
    out[..., :kept.shape[-1]] = kept.masked_fill(~valid, -1).int()
    return new_lens.int(), out, st["k_pages"], st["k_scales"], st["v_pages"], st["v_scales"], st["weights"]


def _plain_read(st):
    page, Hkv = st["case"]["page"], st["Hkv"]
    cu, token = st["cu"].long(), torch.arange(st["rows"], device="cuda")
    seq = torch.searchsorted(cu[1:], token, right=True)
    slot = st["first"].long()[seq] + token - cu[seq]
    rows = (st["page_table"].long()[seq, slot // page] * Hkv)[:, None] + torch.arange(Hkv, device="cuda")
    rows = rows * page + (slot % page)[:, None]
    return (_values(st["k_pages"], st["k_scales"], rows).to(st["dtype"]),
            _values(st["v_pages"], st["v_scales"], rows).to(st["dtype"]))


def _plain_shared(st):
    case, Hkv, page = st["case"], st["Hkv"], st["case"]["page"]
    q = st["q"].float()
    batch = q.shape[0]
    g = st["Hq"] // Hkv
    rows, v, x, seen = _own_logits(st)
    # The prefixes' keys and values once a group, for the queries of all its sequences: [group, Hkv, seat * g + j, D].
    cu = st["cu_seqs"].long()
    s = torch.arange(batch, device="cuda")
    group = torch.searchsorted(cu[1:], s, right=True)
    seat = s - cu[group]
    G, N = cu.shape[0] - 1, st["max_group"]
    qs = q.new_zeros((G, N, Hkv, g, D))
    qs[group, seat] = q.view(batch, Hkv, g, D)
    j = torch.arange(st["max_prefix"], device="cuda")
    at = _slot_rows(st["prefix_table"], j[None, :].expand(G, -1), Hkv, page)
    pk, pv = _values(st["k_pages"], None, at), _values(st["v_pages"], None, at)
    y = (qs.transpose(1, 2).reshape(G, Hkv, N * g, D) @ pk.transpose(-1, -2)) * SCALE
    y = y.masked_fill((j[None, :] >= st["prefix_lens"].long()[:, None])[:, None, None, :], -math.inf)
    top = y.amax(-1, keepdim=True)
    y = y.sub_(top).exp_()

    def seats(t):
        return t.view(G, Hkv, N, g, -1)[group, :, seat]          # [batch, Hkv, g, ...]

    pm, pl, po = seats(top), seats(y.sum(-1, keepdim=True)), seats(y @ pv)
    m = torch.maximum(pm, x.amax(-1, keepdim=True))
    p, before = torch.exp(x - m), torch.exp(pm - m)
    total = p.sum(-1, keepdim=True) + before * pl
    out = ((p @ v + before * po) / total).reshape(st["q"].shape).to(st["dtype"])
    if st["weights"] is None:
        return (out,)
    _add_weights(st, rows, p / total, seen)
    return out, st["weights"]


# ---------------------------------------------------------------- the framework's calls

_selectors = {}   # a serving program's handle: one for the model's heads, whatever the inputs


def _own(st):
    from paper_2606_29563_gb300 import kvec
    case, op = st["case"], st["case"]["op"]
    heads = (st["Hq"], st["Hkv"])
    if heads not in _selectors:
        _selectors[heads] = kvec.KvecSelector(kvec.make_params(*heads, num_ext_heads=min(3, heads[1]), max_batch=256,
                                                               max_seqlen=1024, max_layers=1))
    sel = _selectors[heads]
    if "cache" not in st:
        st["cache"] = kvec.PagedCache(st["k_pages"], st["v_pages"], st["page_table"], st["lens"], st["weights"],
                                      k_scales=st["k_scales"], v_scales=st["v_scales"], dtype=st["dtype"])
    cache = st["cache"]
    if op == "append":
        q = sel.rotate_append(st["q"], st["k"], st["v"], st["positions"], st["rot_table"], cache, st["cu"],
                              q_norm=st["norms"][0], k_norm=st["norms"][1], eps=EPS, interleaved=case["interleaved"])
        return q, st["k_pages"], st["k_scales"], st["v_pages"], st["v_scales"]
    if op == "decode":
        out = sel.paged_decode(st["q"], cache, st["max_len"], window=case["window"], sinks=case["sinks"])
        return (out,) if st["weights"] is None else (out, st["weights"])
    if op == "evict":
        new_lens, kept = sel.paged_evict(cache, st["new_table"], case["budget"], sinks=case["sinks"],
                                         recent=case["recent"], max_len=st["max_len"])
        return new_lens, kept, st["k_pages"], st["k_scales"], st["v_pages"], st["v_scales"], st["weights"]
    if op == "read":
        return sel.paged_read(cache, st["cu"], st["rows"], first=st["first"])
    if "prefix" not in st:
        st["prefix"] = kvec.SharedPrefix(st["prefix_table"], st["prefix_lens"], st["cu_seqs"])
    out = sel.shared_decode(st["q"], cache, st["prefix"], st["max_len"], max_prefix=st["max_prefix"])
    return (out,) if st["weights"] is None else (out, st["weights"])


_PLAIN = {"append": _plain_append, "decode": _plain_decode, "evict": _plain_evict, "read": _plain_read, "shared": _plain_shared}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op, Hq, Hkv = case["op"], case["q_heads"], case["kv_heads"]
    row, eight = D * 2, D + 4
    if op == "append":
        T = sum(_lens(case, "new"))
        return {"bytes": T * ((2 * Hq + 2 * Hkv) * row + 2 * Hkv * eight + case["rot"] * 4 + 8), "flops": T * (Hq + 2 * Hkv) * D * 6}
    if op == "decode":
        seen = sum(min(n, case["window"] + min(case["sinks"], max(0, n - case["window"]))) if case["window"] else n
                   for n in _lens(case))
        return {"bytes": seen * Hkv * (2 * eight + (8 if case["weights"] else 0)) + len(_lens(case)) * Hq * row * 2,
                "flops": 4 * seen * Hq * D}
    if op == "evict":
        lens = _lens(case)
        kept = sum(min(n, case["budget"]) for n in lens)
        return {"bytes": Hkv * (4 * sum(lens) + kept * (4 * eight + 12)), "flops": 0}
    if op == "read":
        T = sum(_lens(case)) - sum(_lens(case, "first"))
        return {"bytes": T * Hkv * 2 * ((eight if case["eight"] else row) + row), "flops": 0}
    lens, prefixes, groups = _lens(case), _lens(case, "prefixes"), _lens(case, "groups")
    return {"bytes": Hkv * (2 * row * (sum(prefixes) + sum(lens)) + (8 * sum(lens) if case["weights"] else 0)) + len(lens) * Hq * row * 2,
            "flops": 4 * D * Hq * (sum(p * n for p, n in zip(prefixes, groups)) + sum(lens))}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_turn(x, norm, table, case):
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS) * norm.double()
    half = case["rot"] // 2
    c, s = table[:, None, :half].double(), table[:, None, half:].double()
    y = x.clone()
    first = slice(0, 2 * half, 2) if case["interleaved"] else slice(0, half)
    second = slice(1, 2 * half, 2) if case["interleaved"] else slice(half, 2 * half)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def _held(st, table_row, slots):
    """Keys and values [n, Hkv, D] in 64 bits of a sequence's slots, and where they are."""
    page = st["case"]["page"]
    slots = torch.as_tensor(slots, device="cuda", dtype=torch.int64)
    at, ofs = table_row.long()[slots // page], slots % page
    found = []
    for name in ("k", "v"):
        x = st[name + "_pages"]
        x = x.view(torch.uint8)[at, :, ofs].view(E4M3) if st["eight"] else x[at, :, ofs]
        x = x.double()
        found.append(x * st[name + "_scales"][at, :, ofs].double()[..., None] if st["eight"] else x)
    return found[0], found[1], at, ofs


def exact(case, seed):
    st = prepare(case, seed)
    op, Hq, Hkv, page = case["op"], st["Hq"], st["Hkv"], case["page"]
    g, lens, table = Hq // Hkv, st["lens"].tolist(), st["page_table"]
    W = None if st["weights"] is None else st["weights"].double()
    if op == "append":
        turn = st["rot_table"][st["positions"].long()]
        q, k = (_exact_turn(x, w, turn, case) for x, w in zip((st["q"], st["k"]), st["norms"]))
        rows = table.tolist()
        pages, slots = [], []
        for s, (n, c) in enumerate(zip(lens, st["new"])):
            pages += [rows[s][j // page] for j in range(n - c, n)]
            slots += [j % page for j in range(n - c, n)]
        pages, slots = torch.tensor(pages, device="cuda"), torch.tensor(slots, device="cuda")
        found = [q]
        for name, x in (("k", k), ("v", st["v"].double())):
            scale = torch.clamp(x.abs().max(-1).values / MOST, min=LEAST)
            P, S = st[name + "_pages"].double(), st[name + "_scales"].double()
            P[pages, :, slots] = x / scale[..., None]      # what the stored numbers are rounded from
            S[pages, :, slots] = scale
            found += [P, S]
        return tuple(found)
    if op == "read":
        parts = [_held(st, table[s], range(f, n))[:2] for s, (f, n) in enumerate(zip(_lens(case, "first"), lens))]
        return tuple(torch.cat(x) for x in zip(*parts))
    if op == "evict":
        # Eviction moves values and changes none.
        K, V, KS, VS = (st[x].double() for x in ("k_pages", "v_pages", "k_scales", "v_scales"))
        kept = torch.full((len(lens), Hkv, case["budget"]), -1, dtype=torch.int32, device="cuda")
        for s, n in enumerate(lens):
            j = torch.arange(n, device="cuda")
            at, ofs = table[s].long()[j // page], j % page
            b = min(n, case["budget"])
            score = W[at, :, ofs].T.clone()                               # [Hkv, n]
            score[:, :case["sinks"]] = math.inf
            score[:, max(0, n - case["recent"]):] = math.inf
            best = torch.argsort(score, dim=-1, descending=True, stable=True)[:, :b].sort(-1).values
            kept[s, :, :b] = best.int()
            j = torch.arange(b, device="cuda")
            to, ofs_to = st["new_table"][s].long()[j // page], j % page
            h = torch.arange(Hkv, device="cuda")[:, None]
            for X in (K, V, KS, VS, W):
                X[to[None, :], h, ofs_to[None, :]] = X[at[best], h, ofs[best]]
        return torch.tensor([min(n, case["budget"]) for n in lens], dtype=torch.int32, device="cuda"), kept, K, KS, V, VS, W
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    group_of, prefix = [], []
    if op == "shared":
        group_of = [r for r, n in enumerate(_lens(case, "groups")) for _ in range(n)]
        prefix = [_held(st, st["prefix_table"][r], range(n))[:2] for r, n in enumerate(_lens(case, "prefixes"))]
    for s, n in enumerate(lens):
        seen = [i for i in range(n) if not case.get("window") or i >= n - case["window"] or i < case["sinks"]]
        k, v, at, ofs = _held(st, table[s], seen)
        if op == "shared":
            pk, pv = prefix[group_of[s]]
            k, v = torch.cat([pk, k]), torch.cat([pv, v])
        # [Hkv, g, n]
        x = st["q"][s].double().view(Hkv, g, D) @ k.permute(1, 2, 0) / math.sqrt(D)
        e = torch.exp(x - x.max(-1, keepdim=True).values)
        p = e / e.sum(-1, keepdim=True)
        out[s] = (p @ v.transpose(0, 1)).reshape(Hq, D)
        if W is not None:
            W[at, :, ofs] += p.sum(1)[:, k.shape[0] - len(seen):].T
    return (out,) if W is None else (out, W)
