"""What the paged-cache operators are measured on: cases, their inputs, a plain form of each operator in elementary
torch operations, and the operator from its definition in 64 bits.

Three operators over a key/value cache kept in pages (a page table per sequence), for batches of sequences that each
bring a chunk of new tokens (one token: decoding; many: prefill):
  append  rotate the new keys (and queries) by their positions and write keys and values into the cache's pages,
          with the per-page key bounds kept up to date
  attend  attention of the new tokens over the whole cache of their sequence
  block   attention over the pages whose key bounds promise the largest scores, chosen for each new token
Geometries, lengths and batch shapes are those of the package's workloads: 32 query / 8 KV heads of 64, 24 / 8 heads of
128, contexts of 4096 to 131072 (one of 1048576), 32 ragged sequences of 8192 to 65536 tokens.
"""
import math
import random

import torch

own = False

CHUNK = 1 << 30            # most scores held at once by the plain forms


# ---------------------------------------------------------------------------------------------- cases
def _case(name, op, dtype, hq, hkv, d, page, batch, q, kv, **more):
    c = {"name": name, "op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "page": page, "batch": batch,
         "q_lo": q[0], "q_hi": q[1], "kv_lo": kv[0], "kv_hi": kv[1], "lens": 11, "tokens_first": False}
    c.update(more)
    return c


def listed():
    rot = {"rot": 128, "pairs": False, "bounds": True}
    return [
        # one sequence decodes one token: the smallest write of a serving loop, all latency
        _case("append_one_1b", "append", "bf16", 32, 8, 64, 64, 1, (1, 1), (4096, 4096), rot=64, pairs=False, bounds=True),
        # a decode batch: one row per sequence, each into a page that is partly filled
        _case("append_batch_3b", "append", "bf16", 24, 8, 128, 64, 32, (1, 1), (1000, 4096), **rot),
        # prefill chunks of odd lengths behind existing prefixes, token-major pages, adjacent pairs, half of the dims rotated
        _case("append_chunk_3b", "append", "fp16", 24, 8, 128, 16, 4, (3000, 4096), (4097, 9000), tokens_first=True, rot=64, pairs=True, bounds=True),
        # one sequence decodes one token over a short context
        _case("attend_one_1b", "attend", "bf16", 32, 8, 64, 64, 1, (1, 1), (4096, 4096), causal=True),
        # a decode batch of ragged long sequences: the cache is read once
        _case("attend_batch_3b", "attend", "bf16", 24, 8, 128, 64, 32, (1, 1), (8192, 65536), causal=True),
        # whole prompts without a prefix
        _case("attend_prompts_1b", "attend", "fp16", 32, 8, 64, 64, 4, (5000, 8192), (0, 0), causal=True),
        # a chunk of a prompt at the end of a 128K context: matrix products
        _case("attend_chunk_3b_128k", "attend", "bf16", 24, 8, 128, 64, 1, (4096, 4096), (131072, 131072), causal=True),
        # a mixed step: decoding sequences and chunks of every length in one call, small pages, token-major
        _case("attend_mixed_3b", "attend", "bf16", 24, 8, 128, 16, 24, (1, 600), (700, 20000), causal=True, tokens_first=True),
        # one sequence decodes over 128K tokens, 35 of 2048 pages read
        _case("block_one_3b_128k", "block", "bf16", 24, 8, 128, 64, 1, (1, 1), (131072, 131072), sink=1, tail=2, topk=32),
        # the ragged decode batch
        _case("block_batch_3b", "block", "bf16", 24, 8, 128, 64, 32, (1, 1), (8192, 65536), sink=1, tail=2, topk=32),
        # one sequence decodes over a million tokens
        _case("block_one_3b_1m", "block", "bf16", 24, 8, 128, 64, 1, (1, 1), (1048576, 1048576), sink=1, tail=4, topk=128),
        # short chunks (several drafted tokens to check per sequence), each token with pages of its own
        _case("block_chunk_1b", "block", "fp16", 32, 8, 64, 32, 8, (3, 40), (20000, 32768), sink=1, tail=4, topk=60),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed kinds with other sizes; it costs no more than the largest listed one of its operator."""
    most = {}
    for c in listed():
        w = work(c)
        m = most.setdefault(c["op"], {"bytes": 0, "flops": 0})
        for k in m:
            m[k] = max(m[k], w[k])
    while True:
        op = rng.choice(["append", "attend", "block"])
        hq, hkv, d = rng.choice([(32, 8, 64), (24, 8, 128), (8, 2, 64), (6, 6, 128), (16, 2, 128)])
        decode = rng.random() < 0.5
        batch = _spread(rng, 1, 48)
        q_hi = 1 if decode else _spread(rng, 2, {"append": 8192, "attend": 8192, "block": 96}[op])
        q_lo = 1 if decode else _spread(rng, 1, q_hi)
        kv_hi = max(q_hi, _spread(rng, 1, {"append": 16384, "attend": 131072, "block": 131072}[op]))
        kv_lo = _spread(rng, 1, kv_hi)
        c = _case("", op, rng.choice(["bf16", "fp16"]), hq, hkv, d, rng.choice([16, 32, 64, 128]), batch,
                  (q_lo, q_hi), (kv_lo, kv_hi), lens=rng.randrange(1 << 20), tokens_first=rng.random() < 0.5)
        if op == "append":
            c.update(rot=rng.choice([0, d // 2, d, d]), pairs=rng.random() < 0.3, bounds=rng.random() < 0.6)
        elif op == "attend":
            c.update(causal=rng.random() < 0.8)
        else:
            c.update(sink=rng.randrange(0, 4), tail=rng.randrange(1, 6), topk=_spread(rng, 1, 160))
        del c["name"]
        w = work(c)
        q_lens, kv_lens = _lengths(c)
        state = sum(kv_lens) * c["hkv"] * c["d"] * 4
        if w["bytes"] <= most[op]["bytes"] and w["flops"] <= most[op]["flops"] and state <= 5 << 30:
            return c


def _lengths(c):
    """New tokens and cache length (the new tokens included) of each sequence."""
    r = random.Random(c["lens"])
    q_lens = [r.randint(c["q_lo"], c["q_hi"]) for _ in range(c["batch"])]
    return q_lens, [max(n, r.randint(c["kv_lo"], c["kv_hi"])) for n in q_lens]


def _selected(c, pos):
    """Keys that the token at position `pos` reads in a block call: all of its pages but the last are full."""
    pages = pos // c["page"] + 1
    taken = min(pages, c["sink"] + c["tail"] + c["topk"])
    return (taken - 1) * c["page"] + pos % c["page"] + 1


def work(case):
    c = case
    q_lens, kv_lens = _lengths(c)
    new = sum(q_lens)
    row = c["d"] * 2
    if c["op"] == "append":
        touched = sum((n - 1) // c["page"] - (n - m) // c["page"] + 1 for m, n in zip(q_lens, kv_lens))
        moved = 2 * new * row * (c["hq"] + 2 * c["hkv"]) + (touched * c["hkv"] * 2 * row if c["bounds"] else 0)
        return {"bytes": moved, "flops": 3 * new * c["rot"] * (c["hq"] + c["hkv"])}
    out = new * c["hq"] * (2 * row + 4)
    if c["op"] == "attend":
        seen = sum(m * n - (m * (m - 1) // 2 if c["causal"] else 0) for m, n in zip(q_lens, kv_lens))
        return {"bytes": sum(kv_lens) * c["hkv"] * 2 * row + out, "flops": 4 * c["d"] * c["hq"] * seen}
    # every page's bounds once per sequence, and each new token's selected rows (a chunk's tokens may share them: at
    # least those of one token)
    pages = sum((n + c["page"] - 1) // c["page"] for n in kv_lens)
    seen = [_selected(c, n - m + i) for m, n in zip(q_lens, kv_lens) for i in range(m)]
    first = [_selected(c, n - 1) for n in kv_lens]
    scored = sum(m * ((n + c["page"] - 1) // c["page"]) for m, n in zip(q_lens, kv_lens))
    kept = c["sink"] + c["tail"] + c["topk"]
    return {"bytes": pages * c["hkv"] * 2 * row + sum(first) * c["hkv"] * 2 * row + out + new * c["hkv"] * kept * 4,
            "flops": (4 * sum(seen) + 2 * scored) * c["d"] * c["hq"]}


# ---------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    """A filled paged cache (pages in random order, some keys along the queries' topic so that attention is peaked) and
    the step's inputs."""
    c, dev = case, torch.device("cuda")
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    hq, hkv, d, ps = c["hq"], c["hkv"], c["d"], c["page"]
    q_lens, kv_lens = _lengths(c)
    new, batch = sum(q_lens), c["batch"]
    n_seq = [(n + ps - 1) // ps for n in kv_lens]
    n_pages = sum(n_seq) + 3
    shape = (n_pages, ps, hkv, d) if c["tokens_first"] else (n_pages, hkv, ps, d)
    k = torch.randn(shape, dtype=dt, device=dev, generator=g)
    v = torch.randn(shape, dtype=dt, device=dev, generator=g)
    if c["tokens_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)           # [page, head, slot, dim], whatever the storage
    order = torch.randperm(n_pages, device=dev, generator=g).int()
    table = torch.full((batch, max(n_seq)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(n_seq):
        table[b, :n] = order[at:at + n]
        at += n
    topic = torch.randn(batch, hkv, d, device=dev, generator=g)
    seq_of = torch.repeat_interleave(torch.arange(batch, device=dev), torch.tensor(q_lens, device=dev))
    # a key in about 500 is three times its sequence's topic
    far = torch.tensor(kv_lens, device=dev)
    pick = torch.repeat_interleave(torch.arange(batch, device=dev), far // 500 + 1)
    pos = (torch.rand(pick.numel(), device=dev, generator=g) * far[pick]).long().clamp_max(far[pick] - 1)
    k[table[pick, pos // ps].long(), :, pos % ps] = (3 * topic[pick]).to(dt)
    first = torch.tensor([n - m for m, n in zip(q_lens, kv_lens)], device=dev)
    cu_q = [0]
    for m in q_lens:
        cu_q.append(cu_q[-1] + m)
    start = torch.tensor(cu_q[:-1], device=dev)
    s = {"c": c, "k": k, "v": v, "table": table, "q_lens": q_lens, "kv_lens": kv_lens, "cu_q": cu_q, "seq_of": seq_of,
         "pos": torch.arange(new, device=dev) - start[seq_of] + first[seq_of]}
    mixed = torch.randn(new, hkv, hq // hkv, d, device=dev, generator=g)
    q = (0.25 * topic[seq_of][:, :, None] + math.sqrt(1 - 0.25 ** 2) * mixed).reshape(new, hq, d).to(dt)
    s["bounds"] = None
    if c["op"] == "append":
        # the projections' output: query, key and value heads of a token beside each other
        qkv = torch.randn(new, hq + 2 * hkv, d, dtype=dt, device=dev, generator=g)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_out"] = torch.empty(new, hq, d, dtype=dt, device=dev)
        s["inv_freq"] = None
        if c["rot"]:
            s["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().to(dev)
        if c["bounds"]:
            s["bounds"] = torch.zeros(n_pages, hkv, 2, d, dtype=dt, device=dev)
    else:
        s["q"] = q
        s["y"] = torch.empty(new, hq, d, dtype=dt, device=dev)
        s["lse"] = torch.empty(new, hq, dtype=torch.float32, device=dev)
        if c["op"] == "block":
            s["bounds"] = torch.stack([k.amin(2), k.amax(2)], 2).contiguous()
            s["idx"] = torch.empty(new, hkv, c["sink"] + c["tail"] + c["topk"], dtype=torch.int32, device=dev)
    if own:
        import numpy as np

        import paper_2604_05438_b200 as T
        s["kv"] = T.PagedKVCache(k, v, table, np.array(kv_lens, np.int64), np.array(cu_q, np.int64), hq, s["bounds"])
        if c["op"] == "append":
            s["rotary"] = T.RotaryMap(s["inv_freq"], c["pairs"]) if c["rot"] else None
        elif c["op"] == "attend":
            n = T.paged_workspace_bytes(s["kv"], T.WS_PAGED_ATTENTION)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=dev)
        else:
            s["sel"] = T.PageSelection(c["sink"], c["tail"], c["topk"])
            n = T.paged_workspace_bytes(s["kv"], T.WS_PAGED_BLOCK_ATTENTION, s["sel"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["c"]
    if own:
        import paper_2604_05438_b200 as T
        if c["op"] == "append":
            T.paged_append(s["kv"], s["k_new"], s["v_new"], s["rotary"], s["q"], s["q_out"])
            return {"k": s["k"], "v": s["v"], "q": s["q_out"], "bounds": s["bounds"]}
        if c["op"] == "attend":
            flags = 0 if c["causal"] else T.FLAG_FULL_CONTEXT
            T.paged_attention(s["kv"], s["q"], s["y"], s["lse"], None, flags, s["ws"])
            return {"y": s["y"], "lse": s["lse"]}
        T.paged_block_attention(s["kv"], s["sel"], s["q"], s["y"], s["lse"], s["idx"], None, s["ws"])
        return {"y": s["y"], "lse": s["lse"], "pages": s["idx"]}
    return {"append": _plain_append, "attend": _plain_attend, "block": _plain_block}[c["op"]](s)


def _rotated(x, angle, pairs):
    """x [rows, heads, d] in 32 bits, the first 2 * angle.shape[1] dims of each head rotated."""
    n = angle.shape[1]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if pairs else (x[..., :n], x[..., n:2 * n])
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if pairs else torch.cat(turned, -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _plain_append(s):
    c = s["c"]
    ps, dt = c["page"], s["k"].dtype
    k_new, q = s["k_new"].float(), s["q"].float()
    if c["rot"]:
        angle = s["pos"].double()[:, None] * s["inv_freq"].double()      # far positions: 32 bits lose the angle
        k_new, q = _rotated(k_new, angle, c["pairs"]), _rotated(q, angle, c["pairs"])
    page = s["table"][s["seq_of"], s["pos"] // ps].long()
    s["k"][page, :, s["pos"] % ps] = k_new.to(dt)
    s["v"][page, :, s["pos"] % ps] = s["v_new"]
    s["q_out"].copy_(q)
    if s["bounds"] is not None:
        # the touched pages, once each, and how many of their slots hold a row now
        b_of, page_of = torch.unique(torch.stack([s["seq_of"], s["pos"] // ps], 1), dim=0).unbind(1)
        filled = torch.tensor(s["kv_lens"], device=page.device)[b_of] - page_of * ps
        empty = torch.arange(ps, device=page.device) >= filled[:, None]
        phys = s["table"][b_of, page_of].long()
        rows = s["k"][phys].float()
        low = rows.masked_fill(empty[:, None, :, None], math.inf).amin(2)
        high = rows.masked_fill(empty[:, None, :, None], -math.inf).amax(2)
        s["bounds"][phys] = torch.stack([low, high], 2).to(dt)
    return {"k": s["k"], "v": s["v"], "q": s["q_out"], "bounds": s["bounds"]}


def _plain_attend(s):
    c = s["c"]
    hkv, group, d, dt = c["hkv"], c["hq"] // c["hkv"], c["d"], s["k"].dtype
    ys, lses = [], []
    for b, (m, n) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        pages = s["table"][b, :(n + c["page"] - 1) // c["page"]].long()
        key = s["k"][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :n].float()
        val = s["v"][pages].transpose(0, 1).reshape(hkv, -1, d)[:, :n].float()
        q = s["q"][s["cu_q"][b]:s["cu_q"][b] + m].float().view(m, hkv, group, d).permute(1, 0, 2, 3)
        at = torch.arange(n, device=key.device)
        for rows in torch.arange(m, device=key.device).split(max(1, CHUNK // (c["hq"] * n))):
            score = q[:, rows].flatten(1, 2) @ key.transpose(1, 2) / math.sqrt(d)
            if c["causal"]:
                later = at > (rows + n - m).repeat_interleave(group)[:, None]
                score.masked_fill_(later, -math.inf)
            top = score.amax(2, keepdim=True)
            score.sub_(top).exp_()
            total = score.sum(2, keepdim=True)
            y = (score @ val / total).view(hkv, -1, group, d)
            ys.append(y.transpose(0, 1).flatten(1, 2).to(dt))
            lses.append((top + total.log()).view(hkv, -1, group).transpose(0, 1).flatten(1, 2))
    return {"y": torch.cat(ys), "lse": torch.cat(lses)}


def _plain_block(s):
    c = s["c"]
    hkv, group, d, ps, dt = c["hkv"], c["hq"] // c["hkv"], c["d"], c["page"], s["k"].dtype
    kept = c["sink"] + c["tail"] + c["topk"]
    dev = s["k"].device
    heads = torch.arange(hkv, device=dev)[None, :, None]
    ys, lses, ids = [], [], []
    for b, (m, n) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        n_pages = (n + ps - 1) // ps
        table = s["table"][b, :n_pages].long()
        low, high = s["bounds"][table].double().permute(2, 1, 3, 0)      # [2][head][dim][page]
        q_all = s["q"][s["cu_q"][b]:s["cu_q"][b] + m].view(m, hkv, group, d)
        page = torch.arange(n_pages, device=dev)
        for rows in torch.arange(m, device=dev).split(max(1, CHUNK // (hkv * min(kept, n_pages) * ps * d))):
            # the largest score that a key within a page's bounds could have, in 64 bits: neighbours in the order may be
            # closer than 32 bits tell apart; the group's heads share their pages
            q = q_all[rows].double().transpose(0, 1)                         # [head][row][group][dim]
            bound = (q.clamp_min(0).flatten(1, 2) @ high + q.clamp_max(0).flatten(1, 2) @ low)
            bound = bound.view(hkv, -1, group, n_pages).amax(2).transpose(0, 1)
            pos = (rows + n - m)[:, None]
            seen = page <= pos // ps
            always = (page < c["sink"]) | (page > pos // ps - c["tail"])
            bound = bound.masked_fill((always | ~seen)[:, None], -math.inf)
            order = bound.sort(dim=2, descending=True, stable=True).indices[:, :, :c["topk"]]
            free = (seen & ~always).sum(1)[:, None, None]
            taken = torch.zeros_like(bound, dtype=torch.bool)
            taken.scatter_(2, order, torch.arange(order.shape[2], device=dev) < free.expand(-1, hkv, 1))
            taken |= (always & seen)[:, None]
            idx = page.expand_as(taken).masked_fill(~taken, n_pages).sort(2).values[:, :, :kept]
            idx = torch.nn.functional.pad(idx, (0, kept - idx.shape[2]), value=n_pages)
            none = idx == n_pages
            use = idx[:, :, :min(kept, n_pages)]
            phys = table[use.clamp_max(n_pages - 1)]
            where = use[..., None] * ps + torch.arange(ps, device=dev)
            masked = ((use == n_pages)[..., None] | (where > pos[..., None, None])).flatten(2)[:, :, None]
            key = s["k"][phys, heads].flatten(2, 3).float()                  # [row][head][key][dim]
            score = q_all[rows].float() @ key.transpose(2, 3) / math.sqrt(d)
            score.masked_fill_(masked, -math.inf)
            del key
            top = score.amax(3, keepdim=True)
            score.sub_(top).exp_()
            total = score.sum(3, keepdim=True)
            val = s["v"][phys, heads].flatten(2, 3).float()
            ys.append((score @ val / total).flatten(1, 2).to(dt))
            lses.append((top + total.log()).flatten(1))
            ids.append(idx.masked_fill(none, -1).int())
    return {"y": torch.cat(ys), "lse": torch.cat(lses), "pages": torch.cat(ids)}


# ---------------------------------------------------------------------------------------------- from the definition
def exact(case, seed):
    """The outputs of `run` from the operators' definitions in 64 bits."""
    global own
    kept_own, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept_own
    return {"append": _exact_append, "attend": _exact_attend, "block": _exact_block}[case["op"]](s)


def _exact_append(s):
    c = s["c"]
    ps, n = c["page"], c["rot"] // 2
    if s["k"].numel() > 1 << 28:
        return None
    key, val, q = s["k"].double(), s["v"].double(), s["q"].double().clone()
    row = s["k_new"].double().clone()
    for x in (row, q):
        if n:
            # each pair as a complex number, times e^(i angle)
            turn = torch.polar(torch.ones_like(s["pos"], dtype=torch.float64)[:, None],
                               s["pos"].double()[:, None] * s["inv_freq"].double())[:, None]
            first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["pairs"] else (slice(0, n), slice(n, 2 * n))
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
    bounds = None if s["bounds"] is None else s["bounds"].double()
    for b, (m, length) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        begin, lo = length - m, s["cu_q"][b]
        for p in range(begin // ps, (length - 1) // ps + 1):
            phys = int(s["table"][b, p])
            t0, t1 = max(begin, p * ps), min(length, (p + 1) * ps)
            at = slice(t0 - p * ps, t1 - p * ps)
            key[phys, :, at] = row[lo + t0 - begin:lo + t1 - begin].transpose(0, 1)
            val[phys, :, at] = s["v_new"][lo + t0 - begin:lo + t1 - begin].double().transpose(0, 1)
            if bounds is not None:
                have = key[phys, :, :t1 - p * ps]
                bounds[phys, :, 0], bounds[phys, :, 1] = have.min(1).values, have.max(1).values
    return {"k": key, "v": val, "q": q, "bounds": bounds}


def _rows_of(x, table, n):
    """Rows 0 .. n-1 of a sequence, [head, row, dim] in 64 bits."""
    rows = x.permute(0, 2, 1, 3)[table.long()].reshape(-1, x.shape[1], x.shape[3])[:n]
    return rows.permute(1, 0, 2).double()


def _exact_attend(s):
    c = s["c"]
    group, d = c["hq"] // c["hkv"], c["d"]
    y = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    for b, (m, n) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        table = s["table"][b, :-(-n // c["page"])]
        key, val = _rows_of(s["k"], table, n), _rows_of(s["v"], table, n)
        step = max(1, (CHUNK // 4) // n)
        for h in range(c["hq"]):
            for i in range(0, m, step):
                at = slice(s["cu_q"][b] + i, s["cu_q"][b] + min(m, i + step))
                score = s["q"][at, h].double().mul(d ** -0.5) @ key[h // group].T
                if c["causal"]:
                    score += torch.full_like(score, -math.inf).triu(n - m + i + 1)
                lse[at, h] = score.logsumexp(1)
                y[at, h] = (score - lse[at, h, None]).exp() @ val[h // group]
    return {"y": y, "lse": lse}


def _exact_block(s):
    c = s["c"]
    hkv, group, d, ps = c["hkv"], c["hq"] // c["hkv"], c["d"], c["page"]
    kept = c["sink"] + c["tail"] + c["topk"]
    y = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    pages = torch.full((len(s["pos"]), hkv, kept), -1, dtype=torch.int32)
    where = s["pos"].tolist()
    if len(where) * hkv > 2048:
        return None
    for t, b in enumerate(s["seq_of"].tolist()):
        last = where[t] // ps
        table = s["table"][b, :last + 1].long()
        for h in range(hkv):
            q = s["q"][t, h * group:(h + 1) * group].double()
            low, high = s["bounds"][table, h, 0].double(), s["bounds"][table, h, 1].double()
            best = torch.where(q[:, None] >= 0, q[:, None] * high, q[:, None] * low).sum(2).amax(0).tolist()
            middle = range(c["sink"], last + 1 - c["tail"])
            take = set(sorted(middle, key=lambda j: (-best[j], j))[:c["topk"]])
            take = sorted(take | set(range(min(c["sink"], last + 1))) | set(range(max(0, last + 1 - c["tail"]), last + 1)))
            pages[t, h, :len(take)] = torch.tensor(take, dtype=torch.int32)
            at = torch.tensor([j * ps + i for j in take for i in range(ps) if j * ps + i <= where[t]], device=q.device)
            key, val = s["k"][table[at // ps], h, at % ps].double(), s["v"][table[at // ps], h, at % ps].double()
            score = q @ key.T / math.sqrt(d)
            lse[t, h * group:(h + 1) * group] = score.logsumexp(1)
            y[t, h * group:(h + 1) * group] = torch.softmax(score, 1) @ val
    return {"y": y, "lse": lse, "pages": pages}
