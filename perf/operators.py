"""The paged key/value cache of a causal decoder and what is done with it, as cases that can be timed one by one.

Three kinds of case:

* ``append``  the keys and values of new tokens are stored in the pages of their sequences;
* ``attend``  the new tokens of every sequence (one each when decoding, a chunk each when a prompt is read) attend over
              all tokens of their sequence in the cache, optionally with scores capped by a tanh, a bias that falls with
              distance, a sliding window, and with the attention weight that every cached token receives added up;
* ``evict``   sequences over their budget lose the tokens of least accumulated weight; tokens from the end of the
              sequence fill the holes.

Layout: pages of keys and of values are [n_pages, n_kv_heads, page, dh]; ``table`` [n_seqs, max_pages] names the pages of a
sequence in order; slot j of sequence b is place j % page of page table[b, j // page].  ``length`` counts the tokens of a
sequence in the cache with the new ones, which take the last slots.  ``pos`` and ``weight`` [n_seqs, max_pages * page] hold
position and accumulated weight of the token in each slot.
"""
import math

import torch

own = False
DEV = "cuda"


def _attend(name, dtype, n_seqs, heads, kv_heads, dh, page, max_len, new, ragged=False, softcap=0.0, window=0,
            slopes=False, weights=False, moved=False):
    return {"name": name, "kind": "attend", "dtype": dtype, "n_seqs": n_seqs, "heads": heads, "kv_heads": kv_heads,
            "dh": dh, "page": page, "max_len": max_len, "new": new, "ragged": ragged, "softcap": softcap,
            "window": window, "slopes": slopes, "weights": weights, "moved": moved}


def _append(name, dtype, n_seqs, kv_heads, dh, page, max_len, new, ragged=False):
    return {"name": name, "kind": "append", "dtype": dtype, "n_seqs": n_seqs, "kv_heads": kv_heads, "dh": dh,
            "page": page, "max_len": max_len, "new": new, "ragged": ragged}


def _evict(name, dtype, n_seqs, kv_heads, dh, page, max_len, over, ragged=False):
    return {"name": name, "kind": "evict", "dtype": dtype, "n_seqs": n_seqs, "kv_heads": kv_heads, "dh": dh,
            "page": page, "max_len": max_len, "over": over, "ragged": ragged}


def listed():
    return [
        # one token of one GPT-2-small-shaped sequence: what an interactive user waits for at every layer and token
        _attend("decode_one", "bf16", 1, 12, 12, 64, 16, 777, 1),
        # a serving batch of the same decoder, sequences of all ages
        _attend("decode_batch", "bf16", 64, 12, 12, 64, 16, 2048, 1, ragged=True),
        # long contexts, heads that share keys, the weights of the cached tokens added up for a later eviction
        _attend("decode_long_weights", "bf16", 6, 32, 8, 128, 64, 32768, 1, ragged=True, weights=True),
        # the other element type, after evictions (positions are not slots), with a bias by distance
        _attend("decode_f32_bias", "f32", 8, 12, 12, 64, 16, 1000, 1, ragged=True, slopes=True, moved=True),
        # whole prompts of the GPT-2-small shape at once
        _attend("prompts", "bf16", 16, 12, 12, 64, 16, 1024, 1024),
        # a chunk of one long prompt over what is already cached, capped scores
        _attend("chunk_long_capped", "bf16", 1, 32, 8, 128, 64, 16384, 512, softcap=30.0),
        # ragged chunks in a sliding window, weights added up
        _attend("chunks_window_weights", "bf16", 12, 12, 12, 64, 32, 3000, 333, ragged=True, window=1024, weights=True),
        # the other element type
        _attend("chunk_f32", "f32", 4, 12, 12, 64, 16, 1024, 256, ragged=True),
        # one token of each of a batch's sequences, and whole prompts
        _append("append_tokens", "bf16", 64, 12, 64, 16, 2048, 1, ragged=True),
        _append("append_prompts", "bf16", 16, 12, 64, 16, 1024, 1024, ragged=True),
        # decoding within a budget: a few tokens over; and a prompt's cache cut to a quarter
        _evict("evict_few", "bf16", 64, 12, 64, 16, 1040, 16, ragged=False),
        _evict("evict_prompt", "bf16", 8, 8, 128, 64, 8192, 6144, ragged=True),
    ]


# ---- drawn cases ---------------------------------------------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    return kv * (1 if kv in (12, 16) else rng.choice([1, 1, 2, 3, 4, 8])), kv


_MAX_FLOPS = 70e9                # the chunk of the listed long prompt
_MAX_BYTES = 1.2e9
_F32_COST = 16                   # fp32 products against bf16 ones


def _draw_attend(rng):
    heads, kv = _heads(rng)
    decode = rng.random() < 0.5
    c = {"kind": "attend", "dtype": "f32" if rng.random() < 0.25 else "bf16", "n_seqs": _log(rng, 1, 96), "heads": heads,
         "kv_heads": kv, "dh": rng.choice([64, 64, 128]), "page": rng.choice([16, 16, 32, 64, 128]),
         "max_len": _log(rng, 17, 32768), "new": 1 if decode else _log(rng, 2, 1024), "ragged": rng.random() < 0.7,
         "softcap": 30.0 if rng.random() < 0.25 else 0.0, "window": 0, "slopes": rng.random() < 0.25,
         "weights": rng.random() < 0.3, "moved": decode and rng.random() < 0.3}
    c["new"] = min(c["new"], c["max_len"])
    if rng.random() < 0.25:
        c["window"] = _log(rng, 1, c["max_len"])
    while True:
        w = work(c)
        pool = 2.0 * c["n_seqs"] * c["max_len"] * kv * c["dh"] * _size(c)
        scores = 4.0 * c["n_seqs"] * c["new"] * c["max_len"] * heads
        if (w["flops"] * (_F32_COST if c["dtype"] == "f32" else 1) <= _MAX_FLOPS and pool <= _MAX_BYTES and
                scores <= _MAX_BYTES):
            return c
        if c["n_seqs"] > 1:
            c["n_seqs"] = (3 * c["n_seqs"]) // 4
        else:
            c["max_len"] = max(17, (3 * c["max_len"]) // 4)
            c["new"] = min(max(1, (3 * c["new"]) // 4), c["max_len"])
            c["window"] = min(c["window"], c["max_len"])


def draw(rng):
    p = rng.random()
    if p < 0.7:
        return _draw_attend(rng)
    _, kv = _heads(rng)
    c = {"kind": "append" if p < 0.85 else "evict", "dtype": "f32" if rng.random() < 0.25 else "bf16",
         "n_seqs": _log(rng, 1, 96), "kv_heads": kv, "dh": rng.choice([64, 64, 128]),
         "page": rng.choice([16, 16, 32, 64, 128]), "max_len": _log(rng, 17, 16384), "ragged": rng.random() < 0.7}
    while 2.0 * c["n_seqs"] * c["max_len"] * kv * c["dh"] * _size(c) > 0.5 * _MAX_BYTES:
        c["n_seqs"] = max(1, (3 * c["n_seqs"]) // 4)
        if c["n_seqs"] == 1:
            c["max_len"] = (3 * c["max_len"]) // 4
    if c["kind"] == "append":
        c["new"] = 1 if rng.random() < 0.5 else min(c["max_len"], _log(rng, 2, 1024))
        while c["n_seqs"] * c["new"] > 16384:
            c["new"] = max(1, (3 * c["new"]) // 4)
    else:
        c["over"] = _log(rng, 1, c["max_len"] - 1)
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------

def _size(c):
    return 4 if c["dtype"] == "f32" else 2


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lengths(c):
    """(length, new) of every sequence: ragged ones spread from one token on; a case's lengths are its own, not the seed's."""
    n, most, new = c["n_seqs"], c["max_len"], c.get("new", 1)
    lens, news = [], []
    for b in range(n):
        f = ((b * 0.6180339887498949) % 1.0) if c["ragged"] and b else 1.0
        g = ((b * 0.7548776662466927) % 1.0) if c["ragged"] and b else 1.0
        q = max(1, int(round(new * g)))
        lens.append(max(q, int(round(most * f)), 1))
        news.append(q)
    return lens, news


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    B, kv, dh, page, dt = c["n_seqs"], c["kv_heads"], c["dh"], c["page"], _dtype(c)
    lens, news = _lengths(c)
    mp = (c["max_len"] + page - 1) // page + 1
    n_pages = sum((n + page - 1) // page for n in lens) + 3
    s = {"case": c, "k": _randn(g, (n_pages, kv, page, dh), dt), "v": _randn(g, (n_pages, kv, page, dh), dt)}
    # the pages of a pool that has been in use for a while are in no order; -1 where a sequence has no page yet
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    first = [0]
    for n in lens:
        first.append(first[-1] + (n + page - 1) // page)
    col = torch.arange(mp, device=DEV)
    first_t = torch.tensor(first, device=DEV)
    at = first_t[:-1, None] + col[None, :]
    s["table"] = torch.where(at < first_t[1:, None], order[at.clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    s["length"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    slots = mp * page
    pos = torch.arange(slots, dtype=torch.int32, device=DEV).repeat(B, 1)
    if c["kind"] == "evict" or c.get("moved"):
        # tokens have been evicted before: positions rise in steps of one to three, and old tokens stand in no order
        step = torch.randint(1, 4, (B, slots), generator=g, device=DEV)
        pos = (step.cumsum(1) - 1).to(torch.int32)
        old = torch.arange(slots, device=DEV)[None, :] < (s["length"][:, None] * 3) // 4
        mix = torch.where(old, torch.rand((B, slots), generator=g, device=DEV), 2.0)
        pos = torch.gather(pos, 1, torch.sort(mix, dim=1, stable=True)[1]).contiguous()
    if c["kind"] == "evict":
        # accumulated weights are spread over orders of magnitude; positions and weights share one buffer
        weight = torch.exp(2.0 * torch.randn((B, slots), generator=g, device=DEV)) * 0.1
        s["marks_before"] = torch.stack([pos, weight.view(torch.int32)]).contiguous()
        s["marks"] = s["marks_before"].clone()
        s["keep"] = torch.clamp(s["length"] - c["over"], min=1).to(torch.int32)
        s["length_out"] = torch.zeros_like(s["length"])
        return s
    start = [0]
    for q in news:
        start.append(start[-1] + q)
    s["start"] = torch.tensor(start, dtype=torch.int32, device=DEV)
    rows = start[-1]
    s["pos"] = pos
    if c["kind"] == "append":
        qkv = _randn(g, (rows, 3 * kv, dh), dt)             # what a block's projection leaves: queries, keys, values
        s["k_new"], s["v_new"] = qkv[:, kv:2 * kv], qkv[:, 2 * kv:]
        at_row = s["start"][:-1, None] + torch.arange(c["new"], device=DEV)[None, :]
        slot = s["length"][:, None] - (s["start"][1:] - s["start"][:-1])[:, None] + torch.arange(c["new"], device=DEV)[None, :]
        ok = at_row < s["start"][1:, None]
        s["pos_new"] = torch.zeros((rows,), dtype=torch.int32, device=DEV)
        s["pos_new"][at_row[ok].long()] = 2 * slot[ok].to(torch.int32)
        s["weight"] = torch.rand((B, slots), generator=g, device=DEV)
        return s
    s["q"] = 1.5 * _randn(g, (rows, c["heads"], dh), dt)
    s["out"] = torch.zeros((rows, c["heads"], dh), dtype=dt, device=DEV)
    if c["slopes"]:
        s["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, c["heads"] + 1, device=DEV) / c["heads"]).float()
    if c["weights"]:
        # as much as a few earlier calls have left: a token of a sequence gets heads * new / length of a call on average
        s["weight"] = torch.rand((B, slots), generator=g, device=DEV) * (4.0 * c["heads"] * c["new"] / c["max_len"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if kind == "append":
        return _run_append(state)
    if kind == "evict":
        return _run_evict(state)
    return _run_attend(state)


def _places(s, slot):
    """Page and place of the slots [n_seqs, n] of each sequence."""
    page = s["case"]["page"]
    return torch.gather(s["table"].long(), 1, slot // page).clamp(min=0), slot % page


def _new_rows(s):
    """Rows [n_seqs, new] of the new tokens, their slots, and which of them there are."""
    i = torch.arange(s["case"]["new"], device=DEV)[None, :]
    first, last = s["start"][:-1, None].long(), s["start"][1:, None].long()
    ok = first + i < last
    slot = s["length"][:, None].long() - (last - first) + i
    return torch.where(ok, first + i, 0), torch.where(ok, slot, 0), ok


def _run_append(s):
    c = s["case"]
    if own:
        from paper_2512_16843_amd import llmc
        llmc.llmc_kv_append(s["k_new"], s["v_new"], s["k"], s["v"], s["table"], s["length"],
                            new_start=None if c["new"] == 1 else s["start"], max_new=c["new"], pos_new=s["pos_new"],
                            pos=s["pos"], weight=s["weight"])
    else:
        rows, slot, ok = _new_rows(s)
        page, place = _places(s, slot)
        seq = torch.arange(c["n_seqs"], device=DEV)[:, None].expand_as(slot)[ok]
        rows, slot, page, place = rows[ok], slot[ok], page[ok], place[ok]
        s["k"][page, :, place] = s["k_new"][rows]
        s["v"][page, :, place] = s["v_new"][rows]
        s["pos"][seq, slot] = s["pos_new"][rows]
        s["weight"][seq, slot] = 0.0
    return {"k": s["k"], "v": s["v"], "pos": s["pos"], "weight": s["weight"]}


def _run_attend(s):
    c = s["case"]
    if own:
        from paper_2512_16843_amd import llmc
        if "workspace" not in s:
            need = llmc.llmc_attention_paged_workspace_bytes(s["q"], s["k"], s["table"], max_new=c["new"],
                                                             max_len=c["max_len"], weights=c["weights"])
            s["workspace"] = torch.empty((need,), dtype=torch.uint8, device=DEV)
        llmc.llmc_attention_paged(s["q"], s["k"], s["v"], s["table"], s["length"], s["out"], s["workspace"],
                                  new_start=None if c["new"] == 1 else s["start"], max_new=c["new"],
                                  max_len=c["max_len"], pos=s["pos"] if c["moved"] else None, weight=s.get("weight"),
                                  softcap=c["softcap"], window=c["window"], slopes=s.get("slopes"))
        return {"out": s["out"], "weight": s.get("weight")}
    B, kv, dh, H, new = c["n_seqs"], c["kv_heads"], c["dh"], c["heads"], c["new"]
    G, n = H // kv, c["max_len"]
    rows, slot, ok = _new_rows(s)
    every = torch.arange(n, device=DEV)[None, :].expand(B, n)
    page, place = _places(s, every)
    there = every < s["length"][:, None]
    k = torch.where(there[:, :, None, None], s["k"][page, :, place].float(), 0.0).permute(0, 2, 3, 1).contiguous()
    v = torch.where(there[:, :, None, None], s["v"][page, :, place].float(), 0.0).permute(0, 2, 1, 3).contiguous()
    q = s["q"][rows].float().reshape(B, new, kv, G, dh).permute(0, 2, 1, 3, 4).reshape(B, kv, new * G, dh)
    x = torch.matmul(q, k).reshape(B, kv, new, G, n) * (1.0 / math.sqrt(dh))
    if c["softcap"] > 0:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    pos = s["pos"][:, :n] if c["moved"] else every.to(torch.int32)
    away = torch.gather(pos, 1, slot.clamp(max=n - 1))[:, :, None] - pos[:, None, :]            # [B, new, n]
    if c["slopes"]:
        x = x - s["slopes"].reshape(1, kv, 1, G, 1) * away[:, None, :, None, :].float()
    seen = (every[:, None, :] <= slot[:, :, None]) & ok[:, :, None]
    if c["window"] > 0:
        seen = seen & (away < c["window"])
    seen = seen[:, None, :, None, :]
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
    p = e / e.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(p.reshape(B, kv, new * G, n), v).reshape(B, kv, new, G, dh).permute(0, 2, 1, 3, 4)
    s["out"][rows[ok]] = o.reshape(B, new, H, dh)[ok].to(s["out"].dtype)
    if c["weights"]:
        s["weight"][:, :n] += p.sum(dim=(1, 2, 3))
    return {"out": s["out"], "weight": s.get("weight")}


def _run_evict(s):
    c = s["case"]
    sink, recent = _protected(c)
    s["marks"].copy_(s["marks_before"])                # as they stand when the sequences have grown over their budgets
    pos, weight = s["marks"][0], s["marks"][1].view(torch.float32)
    if own:
        from paper_2512_16843_amd import llmc
        if "workspace" not in s:
            need = llmc.llmc_kv_evict_workspace_bytes(s["table"], max_len=c["max_len"])
            s["workspace"] = torch.empty((need,), dtype=torch.uint8, device=DEV)
        llmc.llmc_kv_evict(s["k"], s["v"], s["table"], s["length"], pos, weight, s["keep"], s["length_out"],
                           s["workspace"], max_len=c["max_len"], sink=sink, recent=recent)
    else:
        n = c["max_len"]
        slot = torch.arange(n, device=DEV)[None, :].expand(c["n_seqs"], n)
        there = slot < s["length"][:, None]
        p, w, keep = pos[:, :n], weight[:, :n], torch.minimum(s["keep"], s["length"])[:, None]
        last = torch.where(there, p, -1).amax(1, keepdim=True)
        safe = (p < sink) | (p > last - recent)
        order = torch.sort(p, dim=1, stable=True)[1]
        order = torch.gather(order, 1, torch.sort(torch.gather(w, 1, order), dim=1, stable=True)[1])
        group = torch.where(there, safe.to(torch.int32), 2)
        order = torch.gather(order, 1, torch.sort(torch.gather(group, 1, order), dim=1, stable=True)[1])
        rank = torch.empty_like(order).scatter_(1, order, slot)
        gone = rank < s["length"][:, None] - keep
        holes = gone & (slot < keep)
        movers = there & ~gone & (slot >= keep)
        to = torch.sort(holes.to(torch.int32), dim=1, descending=True, stable=True)[1]
        src = torch.sort(movers.to(torch.int32), dim=1, descending=True, stable=True)[1]
        ok = slot < holes.sum(1, keepdim=True)
        seq = torch.arange(c["n_seqs"], device=DEV)[:, None].expand_as(slot)[ok]
        (pt, ot), (ps, os_) = _places(s, to), _places(s, src)
        s["k"][pt[ok], :, ot[ok]] = s["k"][ps[ok], :, os_[ok]]
        s["v"][pt[ok], :, ot[ok]] = s["v"][ps[ok], :, os_[ok]]
        pos[seq, to[ok]] = pos[seq, src[ok]]
        weight[seq, to[ok]] = weight[seq, src[ok]]
        s["length_out"].copy_(torch.minimum(s["length"], s["keep"]))
    return {"k": s["k"], "v": s["v"], "pos": pos, "weight": weight, "length": s["length_out"]}


def _protected(c):
    """The first and the last positions, which are kept whatever weight they have gathered."""
    return 4, min(32, c["max_len"] // 4)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["kind"] != "attend":
        return None                                          # copies: nothing is computed
    s = prepare(c, seed)
    lens, news = _lengths(c)
    H, kv, dh, page = c["heads"], c["kv_heads"], c["dh"], c["page"]
    G = H // kv
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    weight = s["weight"].double() if c["weights"] else None
    row = 0
    for b in range(c["n_seqs"]):
        n, q = lens[b], news[b]
        ids = s["table"][b, :(n + page - 1) // page].long()
        pos = (s["pos"][b, :n] if c["moved"] else torch.arange(n, device=DEV)).double()
        slot = torch.arange(n - q, n, device=DEV)
        away = pos[slot][:, None] - pos[None, :]
        hidden = torch.arange(n, device=DEV)[None, :] > slot[:, None]
        if c["window"] > 0:
            hidden |= away >= c["window"]
        for h in range(H):
            kh = s["k"][ids, h // G].reshape(-1, dh)[:n].double()
            vh = s["v"][ids, h // G].reshape(-1, dh)[:n].double()
            x = torch.mm(s["q"][row:row + q, h].double(), kh.t()) / math.sqrt(dh)
            if c["softcap"] > 0:
                x = torch.tanh(x / c["softcap"]) * c["softcap"]
            if c["slopes"]:
                x = x - s["slopes"][h].double() * away
            p = torch.softmax(x.masked_fill(hidden, -math.inf), dim=-1)
            out[row:row + q, h] = torch.mm(p, vh)
            if weight is not None:
                weight[b, :n] += p.sum(0)
        row += q
    return {"out": out, "weight": weight}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    c = case
    e, kv, dh = _size(c), c["kv_heads"], c["dh"]
    lens, news = _lengths(c)
    rows = sum(news)
    if c["kind"] == "append":
        return {"bytes": rows * (4.0 * kv * dh * e + 12.0), "flops": 0.0}
    if c["kind"] == "evict":
        read = moved = 0.0
        for n in lens:
            keep = max(1, n - c["over"])
            read += 8.0 * n
            # a token of the end is kept as often as any other: (n - keep) * keep / n tokens move on average
            moved += (n - keep) * keep / float(n)
        return {"bytes": read + moved * (4.0 * kv * dh * e + 16.0), "flops": 0.0}
    pairs = keys = 0.0
    for n, q in zip(lens, news):
        w = c["window"] if c["window"] > 0 and not c["moved"] else n
        first = n - q + 1                                    # keys that the first and the last new token could see
        pairs += sum(min(w, first + i) for i in (0, q - 1)) * 0.5 * q if w >= n or w <= first else \
            0.5 * (first + w) * (w - first) + w * (n - w + 1.0)
        keys += min(n, w + q - 1)
    bytes_ = keys * 2.0 * kv * dh * e + 2.0 * rows * c["heads"] * dh * e
    if c["weights"]:
        bytes_ += 8.0 * keys
    if c["slopes"] and c["moved"]:
        bytes_ += 4.0 * keys
    return {"bytes": bytes_, "flops": 4.0 * dh * c["heads"] * pairs}
