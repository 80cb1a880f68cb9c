"""The operators around the eviction that a serving loop runs, as cases whose time and outputs can be measured.

Four operators on one cache, all methods of ``kvec.KvecSelector``:

* ``rotate_append``: norms of queries and keys for each head, their rotation by position, and the store of keys
  and values into a paged cache.
* ``paged_decode``: attention of one new token over the paged cache, optionally with a sliding window and a few
  first slots that stay visible; adds each slot's attention weight to the cache's accumulated weights.
* ``paged_evict``: eviction by the accumulated weight; the kept rows move to new pages.
* ``prefill_attention``: causal attention of packed sequences with an optional sliding window and first tokens
  that stay visible, and each row's log-sum-exp (what the eviction's ``lse`` entry points take).

``run`` computes them from elementary torch operations in 32 bits, or with ``own`` by the framework's calls.
"""
import math

import torch

own = False   # set from outside: True runs the framework's operators

D = 128
SCALE = 1.0 / math.sqrt(D)
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _text(lens):
    return ",".join(str(int(n)) for n in lens)


def _lens(case, key="lens"):
    return [int(n) for n in case[key].split(",")]


# Eight ragged prompts of 4096 to 16384 tokens: the lengths that bench.py's default batch has.
RAGGED8 = "14535,5460,4453,11131,6806,12840,12578,14873"
# Sixteen conversations of up to 32768 tokens, of which a sliding window reads the last part.
CHATS16 = "32768,20011,9001,32000,15555,28111,3071,32767,11111,24064,30000,4095,18000,26001,31313,12345"
# Sixty-four conversations of 1024 to 2048 tokens.
BATCH64 = _text(1024 + (389 * i) % 1025 for i in range(64))
# Thirty-two caches of 1000 to 4096 slots; the shortest are within the budget and are kept whole.
BATCH32 = _text(1000 + (997 * i) % 3097 for i in range(32))


def _append(name, dtype, q_heads, kv_heads, new, held, page, rot, interleaved, norm):
    return {"name": name, "op": "rotate_append", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "new": new,
            "held": held, "page": page, "rot": rot, "interleaved": interleaved, "norm": norm}


def _decode(name, dtype, q_heads, kv_heads, lens, page, window, sinks, weights):
    return {"name": name, "op": "paged_decode", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "lens": lens,
            "page": page, "window": window, "sinks": sinks, "weights": weights}


def _evict(name, dtype, kv_heads, lens, page, budget, sinks, recent):
    return {"name": name, "op": "paged_evict", "dtype": dtype, "q_heads": kv_heads * 4, "kv_heads": kv_heads,
            "lens": lens, "page": page, "budget": budget, "sinks": sinks, "recent": recent}


def _prefill(name, dtype, q_heads, kv_heads, q_lens, k_lens, window, sinks):
    return {"name": name, "op": "prefill_attention", "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads,
            "q_lens": q_lens, "k_lens": k_lens, "window": window, "sinks": sinks}


def listed():
    return [
        # One token of one conversation: launch latency is all there is.
        _append("append_one", "bf16", 32, 8, "1", "700", 16, 128, False, True),
        # A decoding step of 64 conversations, rotation of a part of each head, in interleaved pairs, no norms.
        _append("append_batch", "fp16", 28, 4, _text([1] * 64), BATCH64, 64, 64, True, False),
        # The prefill of eight ragged prompts, one layer.
        _append("append_prefill", "bf16", 32, 8, RAGGED8, _text([0] * 8), 64, 128, False, True),
        # A decoding step over one compacted cache: the smallest call.
        _decode("decode_short", "bf16", 32, 8, "512", 16, 0, 0, True),
        # A batch of conversations, seven query heads a KV head, weights accumulated for the eviction.
        _decode("decode_batch", "fp16", 28, 4, BATCH64, 64, 0, 0, True),
        # One very long conversation: the cache's length has to be split over the device.
        _decode("decode_long", "bf16", 32, 8, "131072", 128, 0, 0, False),
        # Long conversations of which only the first slots and a window are visible.
        _decode("decode_window", "bf16", 32, 8, CHATS16, 32, 4096, 4, True),
        # One cache that has grown past its budget by a few dozen tokens.
        _evict("evict_one", "bf16", 8, "576", 16, 512, 4, 32),
        # A batch of caches of different lengths.
        _evict("evict_batch", "fp16", 4, BATCH32, 64, 1024, 4, 128),
        # The last odd chunk of a chunked prefill: few query rows, seven query heads a KV head.
        _prefill("prefill_chunk", "fp16", 28, 4, "33", "1057", 0, 0),
        # Two causal prompts, one of an odd length.
        _prefill("prefill_causal", "bf16", 32, 8, "8192,5001", "8192,5001", 0, 0),
        # One long prompt under a sliding window with four first tokens in sight.
        _prefill("prefill_window", "bf16", 32, 8, "16384", "16384", 2048, 4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate_append", "paged_decode", "paged_evict", "prefill_attention"])
    dtype = rng.choice(["bf16", "fp16"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (8, 8), (16, 8), (16, 2)])
    page = rng.choice([16, 32, 64, 128, 256])
    if op == "rotate_append":
        batch = _log(rng, 1, 64)
        top = max(2, 60_000 // batch)
        new = [_log(rng, 1, top) if rng.random() < 0.5 else 1 for _ in range(batch)]
        held = [_log(rng, 1, 4000) for _ in range(batch)]
        return _append("drawn", dtype, q_heads, kv_heads, _text(new), _text(held), page, rng.choice([16, 64, 96, 128]),
                       rng.random() < 0.5, rng.random() < 0.5)
    if op == "paged_decode":
        batch = _log(rng, 1, 64)
        top = 131072 // batch
        lens = [_log(rng, max(1, top // 64), top) for _ in range(batch)]
        window, sinks = (_log(rng, 16, 8192), rng.randrange(0, 17)) if rng.random() < 0.4 else (0, 0)
        return _decode("drawn", dtype, q_heads, kv_heads, _text(lens), page, window, sinks, rng.random() < 0.6)
    if op == "paged_evict":
        batch = _log(rng, 1, 32)
        top = min(32768, 40_000 // batch)
        lens = [_log(rng, max(1, top // 16), top) for _ in range(batch)]
        budget = max(1, int(max(lens) * rng.uniform(0.05, 0.9)))
        sinks = rng.randrange(0, min(8, budget) + 1)
        return _evict("drawn", dtype, kv_heads, _text(lens), page, budget, sinks, rng.randrange(0, (budget - sinks) // 2 + 1))
    batch = _log(rng, 1, 4)
    k_lens = [_log(rng, 16, 8192 // batch) for _ in range(batch)]
    q_lens = k_lens if rng.random() < 0.5 else [_log(rng, 1, n) for n in k_lens]
    window, sinks = (_log(rng, 16, 4096), rng.randrange(0, 9)) if rng.random() < 0.5 else (0, 0)
    return _prefill("drawn", dtype, q_heads, kv_heads, _text(q_lens), _text(k_lens), window, sinks)


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
    Hq, Hkv = case["q_heads"], case["kv_heads"]
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=dev, dtype=torch.float32) * std).to(dt)

    st = {"case": case, "Hq": Hq, "Hkv": Hkv, "dtype": dt}
    if case["op"] == "prefill_attention":
        q_lens, k_lens = _lens(case, "q_lens"), _lens(case, "k_lens")
        cu_q, cu_k = _cu(q_lens).pin_memory(), _cu(k_lens).pin_memory()
        # Queries of trained models look at some keys far more than at others: a wider spread than the keys'.
        st.update(q=normal(sum(q_lens), Hq, D, std=2.0), k=normal(sum(k_lens), Hkv, D), v=normal(sum(k_lens), Hkv, D),
                  q_lens=q_lens, k_lens=k_lens, cu_q=cu_q, cu_k=cu_k, cu_q_dev=cu_q.to(dev), cu_k_dev=cu_k.to(dev))
        return st
    page = case["page"]
    if case["op"] == "rotate_append":
        new, held = _lens(case, "new"), _lens(case, "held")
        lens = [a + b for a, b in zip(new, held)]      # with the new tokens counted
        T, rot = sum(new), case["rot"]
        # One projection's output: queries, keys and values of a token side by side.
        qkv = normal(T, Hq + 2 * Hkv, D)
        most = max(lens)
        inv = 1.0 / 10000.0 ** (torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot)
        angle = torch.arange(most, dtype=torch.float64, device=dev)[:, None] * inv
        st.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], new=new,
                  cu=_cu(new).to(dev), positions=_ints([h + i for n, h in zip(new, held) for i in range(n)]),
                  rot_table=torch.cat([angle.cos(), angle.sin()], 1).float())
        st["norms"] = (normal(D, std=0.2) + 1, normal(D, std=0.2) + 1) if case["norm"] else (None, None)
    else:
        lens = _lens(case)
    counts = _pages_of(lens, page)
    spare = _pages_of([min(n, case["budget"]) for n in lens], page) if case["op"] == "paged_evict" else []
    pages = sum(counts) + sum(spare)
    st.update(lens=_ints(lens), max_len=max(lens), page_table=_table(counts, host).to(dev),
              k_pages=normal(pages, Hkv, page, D), v_pages=normal(pages, Hkv, page, D))
    if case["op"] == "paged_decode":
        st["q"] = normal(len(lens), Hq, D, std=2.0)
    if case["op"] == "paged_evict":
        st["new_table"] = _table(spare, host, first=sum(counts)).to(dev)
    if case["op"] == "paged_evict" or case.get("weights"):
        # Accumulated weights span decades: a few slots hold most of the attention.
        st["weights"] = torch.randn((pages, Hkv, page), generator=gen, device=dev).mul_(2.0).exp_()
    else:
        st["weights"] = None
    return st


# ---------------------------------------------------------------- the plain forms

def _slot_rows(table, slots, Hkv, page):
    """Row numbers, in the pages seen as rows, of slots [..., n] of the tables [batch, pages]: [batch, Hkv, n]."""
    at = table.long().gather(1, (slots // page).clamp(max=table.shape[1] - 1)) * Hkv
    heads = torch.arange(Hkv, device=table.device)
    return (at[:, None, :] + heads[None, :, None]) * page + (slots % page)[:, None, :]


def _rotated(x, norm, cos, sin, rot, interleaved):
    x = x.float()
    if norm is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * norm.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y, z = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([y, z], -1).flatten(-2) if interleaved else torch.cat([y, z], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(st):
    case, dt, Hkv = st["case"], st["dtype"], st["Hkv"]
    page, rot = case["page"], case["rot"]
    at = st["rot_table"][st["positions"].long()][:, None, :]
    cos, sin = at[..., :rot // 2], at[..., rot // 2:]
    q = _rotated(st["q"], st["norms"][0], cos, sin, rot, case["interleaved"]).to(dt)
    k = _rotated(st["k"], st["norms"][1], cos, sin, rot, case["interleaved"]).to(dt)
    cu, token = st["cu"].long(), torch.arange(q.shape[0], device=q.device)
    seq = torch.searchsorted(cu[1:], token, right=True)
    slot = st["lens"].long()[seq] - (cu[seq + 1] - token)
    rows = (st["page_table"].long()[seq, slot // page] * Hkv)[:, None] + torch.arange(Hkv, device=q.device)
    rows = rows * page + (slot % page)[:, None]
    st["k_pages"].view(-1, D)[rows] = k
    st["v_pages"].view(-1, D)[rows] = st["v"]
    return q, st["k_pages"], st["v_pages"]


def _visible(j, n, case):
    seen = j < n
    if case["window"]:
        seen = seen & ((j >= n - case["window"]) | (j < case["sinks"]))
    return seen


def _plain_decode(st):
    case, Hkv, page = st["case"], st["Hkv"], st["case"]["page"]
    batch, g = st["q"].shape[0], st["Hq"] // Hkv
    j = torch.arange(st["max_len"], device="cuda")
    table = st["page_table"].clamp(min=0)
    rows = _slot_rows(table, j[None, :].expand(batch, -1), Hkv, page)
    k, v = st["k_pages"].view(-1, D)[rows].float(), st["v_pages"].view(-1, D)[rows].float()
    seen = _visible(j[None, :], st["lens"].long()[:, None], case)[:, None, None, :]
    x = (st["q"].float().view(batch, Hkv, g, D) @ k.transpose(-1, -2)) * SCALE
    x = x.masked_fill(~seen, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = (p @ v).reshape(batch, st["Hq"], D).to(st["dtype"])
    if st["weights"] is None:
        return (out,)
    here = seen.expand(-1, Hkv, -1, -1).squeeze(2)
    st["weights"].view(-1).index_put_((rows[here],), p.sum(2)[here], accumulate=True)
    return out, st["weights"]


def _plain_evict(st):
    case, Hkv, page, B = st["case"], st["Hkv"], st["case"]["page"], st["case"]["budget"]
    n = st["lens"].long()
    batch = n.shape[0]
    j = torch.arange(st["max_len"], device="cuda")[None, :]
    rows = _slot_rows(st["page_table"].clamp(min=0), j.expand(batch, -1), Hkv, page)
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
    dst = _slot_rows(st["new_table"].clamp(min=0), to, Hkv, page)
    src, dst = src[valid], dst[valid]
    for name in ("k_pages", "v_pages"):
        flat = st[name].view(-1, D)
        flat[dst] = flat[src]
    flat = st["weights"].view(-1)
    flat[dst] = flat[src]
    out = torch.full((batch, Hkv, B), -1, dtype=torch.int32, device="cuda")
    out[..., :kept.shape[-1]] = kept.masked_fill(~valid, -1).int()
    return new_lens.int(), out, st["k_pages"], st["v_pages"], st["weights"]


def _padded(x, lens, most, at_end):
    """Packed rows [sum lens, H, D] as [batch, H, most, D] in 32 bits, zeros around them."""
    parts = [torch.nn.functional.pad(p, (0, 0, 0, 0, most - p.shape[0], 0) if at_end else (0, 0, 0, 0, 0, most - p.shape[0]))
             for p in x.split(lens)]
    return torch.stack(parts).transpose(1, 2).float()


def _plain_prefill(st):
    case, g = st["case"], st["Hq"] // st["Hkv"]
    q_lens, k_lens = st["q_lens"], st["k_lens"]
    batch, nq, nk = len(q_lens), max(q_lens), max(k_lens)
    # Every sequence ends at the last row and the last key of the padded ones.
    q, k, v = _padded(st["q"], q_lens, nq, True), _padded(st["k"], k_lens, nk, True), _padded(st["v"], k_lens, nk, True)
    x = (q.view(batch, st["Hkv"], g, nq, D) @ k.transpose(-1, -2)[:, :, None]) * SCALE
    first = (nk - st["cu_k_dev"].diff())[:, None, None]
    p = torch.arange(nk - nq, nk, device="cuda")[None, :, None]
    t = torch.arange(nk, device="cuda")[None, None, :]
    seen = (t <= p) & (t >= first)
    if case["window"]:
        seen = seen & ((t > p - case["window"]) | (t < first + case["sinks"]))
    x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    base = top.masked_fill(top == -math.inf, 0.0)
    x = x.sub_(base).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x @ v[:, :, None]) / total.masked_fill(total == 0, 1.0)
    lse = (base + total.log()).squeeze(-1)
    rows = torch.arange(nq, device="cuda") >= (nq - st["cu_q_dev"].diff())[:, None]
    out = out.reshape(batch, st["Hq"], nq, D).transpose(1, 2)[rows]
    return out.to(st["dtype"]), lse.reshape(batch, st["Hq"], nq).transpose(1, 2)[rows]


# ---------------------------------------------------------------- the framework's calls

_selectors = {}   # a serving program's handle: one for the model's heads, whatever the inputs


def _own(st):
    from paper_2606_29563_gb300 import kvec
    case = st["case"]
    heads = (st["Hq"], st["Hkv"])
    if heads not in _selectors:
        _selectors[heads] = kvec.KvecSelector(kvec.make_params(*heads, num_ext_heads=min(3, heads[1]), max_batch=64,
                                                               max_seqlen=1024, max_layers=1))
    sel = _selectors[heads]
    if case["op"] == "prefill_attention":
        return sel.prefill_attention(st["q"], st["k"], st["v"], st["cu_q"], st["cu_q_dev"], st["cu_k"], st["cu_k_dev"],
                                     window=case["window"], sinks=case["sinks"])
    if "cache" not in st:
        st["cache"] = kvec.PagedCache(st["k_pages"], st["v_pages"], st["page_table"], st["lens"], st["weights"])
    cache = st["cache"]
    if case["op"] == "rotate_append":
        q = sel.rotate_append(st["q"], st["k"], st["v"], st["positions"], st["rot_table"], cache, st["cu"],
                              q_norm=st["norms"][0], k_norm=st["norms"][1], eps=EPS, interleaved=case["interleaved"])
        return q, st["k_pages"], st["v_pages"]
    if case["op"] == "paged_decode":
        out = sel.paged_decode(st["q"], cache, st["max_len"], window=case["window"], sinks=case["sinks"])
        return (out,) if st["weights"] is None else (out, st["weights"])
    new_lens, kept = sel.paged_evict(cache, st["new_table"], case["budget"], sinks=case["sinks"], recent=case["recent"],
                                     max_len=st["max_len"])
    return new_lens, kept, st["k_pages"], st["v_pages"], st["weights"]


_PLAIN = {"rotate_append": _plain_append, "paged_decode": _plain_decode, "paged_evict": _plain_evict,
          "prefill_attention": _plain_prefill}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    Hq, Hkv = case["q_heads"], case["kv_heads"]
    row = D * 2
    if case["op"] == "rotate_append":
        T = sum(_lens(case, "new"))
        return {"bytes": T * ((Hq + 2 * Hkv) * row * 2 + case["rot"] * 4 + 8), "flops": T * (Hq + Hkv) * D * 6}
    if case["op"] == "paged_decode":
        seen = sum(min(n, case["window"] + min(case["sinks"], max(0, n - case["window"]))) if case["window"] else n
                   for n in _lens(case))
        return {"bytes": seen * Hkv * (2 * row + (8 if case["weights"] else 0)) + len(_lens(case)) * Hq * row * 2,
                "flops": 4 * seen * Hq * D}
    if case["op"] == "paged_evict":
        lens = _lens(case)
        kept = sum(min(n, case["budget"]) for n in lens)
        return {"bytes": Hkv * (4 * sum(lens) + kept * (4 * row + 12)), "flops": 0}
    pairs = 0
    for nq, nk in zip(_lens(case, "q_lens"), _lens(case, "k_lens")):
        W, S = case["window"], case["sinks"]
        for p in range(nk - nq, nk):
            if p >= 0:
                near = min(p + 1, W) if W else p + 1
                pairs += near + min(S, p + 1 - near)
    Tq, Tk = sum(_lens(case, "q_lens")), sum(_lens(case, "k_lens"))
    return {"bytes": Tq * Hq * (2 * row + 4) + Tk * Hkv * 2 * row, "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_softmax(x):
    m = x.max(-1, keepdim=True).values
    e = torch.exp(x - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
    z = e.sum(-1, keepdim=True)
    return e / torch.where(z > 0, z, torch.ones_like(z)), (m + torch.log(z)).squeeze(-1)


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


def exact(case, seed):
    st = prepare(case, seed)
    Hq, Hkv = st["Hq"], st["Hkv"]
    g = Hq // Hkv
    if case["op"] == "prefill_attention":
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(st["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        q0 = k0 = 0
        for nq, nk in zip(st["q_lens"], st["k_lens"]):
            i = torch.arange(nk - nq, nk, device="cuda")[:, None]
            t = torch.arange(nk, device="cuda")[None, :]
            mask = t > i
            if case["window"]:
                mask = mask | ((i - t >= case["window"]) & (t >= case["sinks"]))
            for h in range(Hq):
                x = st["q"][q0:q0 + nq, h].double() @ st["k"][k0:k0 + nk, h // g].double().T / math.sqrt(D)
                x[mask] = -math.inf
                p, lse[q0:q0 + nq, h] = _exact_softmax(x)
                out[q0:q0 + nq, h] = p @ st["v"][k0:k0 + nk, h // g].double()
            q0, k0 = q0 + nq, k0 + nk
        return out, lse
    page = case["page"]
    K, V = st["k_pages"].double(), st["v_pages"].double()
    lens = st["lens"].tolist()
    table = st["page_table"].tolist()
    if case["op"] == "rotate_append":
        turn = st["rot_table"][st["positions"].long()]
        q, k = (_exact_turn(x, w, turn, case) for x, w in zip((st["q"], st["k"]), st["norms"]))
        pages, slots = [], []
        for s, (n, c) in enumerate(zip(lens, st["new"])):
            pages += [table[s][j // page] for j in range(n - c, n)]
            slots += [j % page for j in range(n - c, n)]
        pages, slots = torch.tensor(pages, device="cuda"), torch.tensor(slots, device="cuda")
        K[pages, :, slots] = k
        V[pages, :, slots] = st["v"].double()
        return q, K, V
    W = None if st["weights"] is None else st["weights"].double()
    if case["op"] == "paged_decode":
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        for s, n in enumerate(lens):
            j = [i for i in range(n) if not case["window"] or i >= n - case["window"] or i < case["sinks"]]
            at = torch.tensor([table[s][i // page] for i in j], device="cuda")
            ofs = torch.tensor(j, device="cuda") % page
            k, v = K[at, :, ofs], V[at, :, ofs]                       # [visible, Hkv, D]
            x = torch.einsum("hgd,nhd->hgn", st["q"][s].double().view(Hkv, g, D), k) / math.sqrt(D)
            p, _ = _exact_softmax(x)
            out[s] = torch.einsum("hgn,nhd->hgd", p, v).reshape(Hq, D)
            if W is not None:
                W[at, :, ofs] += p.sum(1).T
        return (out,) if W is None else (out, W)
    # Eviction moves values and changes none.
    kept = torch.full((len(lens), Hkv, case["budget"]), -1, dtype=torch.int32, device="cuda")
    fresh = st["new_table"].tolist()
    for s, n in enumerate(lens):
        at = torch.tensor([table[s][i // page] for i in range(n)], device="cuda")
        ofs = torch.arange(n, device="cuda") % page
        b = min(n, case["budget"])
        score = W[at, :, ofs].T.clone()                               # [Hkv, n]
        score[:, :case["sinks"]] = math.inf
        score[:, max(0, n - case["recent"]):] = math.inf
        best = torch.argsort(score, dim=-1, descending=True, stable=True)[:, :b].sort(-1).values
        kept[s, :, :b] = best.int()
        to = torch.tensor([fresh[s][i // page] for i in range(b)], device="cuda")
        ofs_to = torch.arange(b, device="cuda") % page
        h = torch.arange(Hkv, device="cuda")[:, None]
        for X in (K, V, W):
            X[to[None, :], h, ofs_to[None, :]] = X[at[best], h, ofs[best]]
    return torch.tensor([min(n, case["budget"]) for n in lens], dtype=torch.int32, device="cuda"), kept, K, V, W
