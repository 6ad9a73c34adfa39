"""What the operators around an 8-bit paged cache are measured on: cases, their inputs, a plain form of each operator in
elementary torch operations, and the operator from its definition in 64 bits.

An 8-bit cache holds a row x (one token, one KV head) as e4m3 codes c and one power of two s, x ~ c s, where s is the
smallest power of two (2^-126 at least) with max |x| <= 448 s and c = x / s rounded.  Operators:
  norm    append to a 16-bit cache: root-mean-square norm of each query and key head with weights, then the rotation by the
          position, written into the cache's pages with the per-page key bounds kept up to date
  write   append to an 8-bit cache, with or without the norms
  read    an 8-bit cache's rows back as 16-bit rows
  attend  attention of the new tokens over an 8-bit cache
  block   attention over the pages of an 8-bit cache whose key bounds promise the largest scores
Geometries, lengths and batch shapes are those of the package's workloads: 32 query / 8 KV heads of 64, 24 / 8 heads of
128, contexts of 4096 to 131072, 32 ragged sequences of 8192 to 65536 tokens.
"""
import math
import random

import torch

own = False

CHUNK = 1 << 30            # most scores held at once by the plain forms
EPS = 1e-6                 # of the norms


# ---------------------------------------------------------------------------------------------- cases
def _case(name, op, dtype, hq, hkv, d, page, batch, q, kv, **more):
    c = {"name": name, "op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "page": page, "batch": batch,
         "q_lo": q[0], "q_hi": q[1], "kv_lo": kv[0], "kv_hi": kv[1], "lens": 11, "tokens_first": False}
    c.update(more)
    return c


def listed():
    return [
        # one sequence decodes one token: the smallest write of a serving loop, all latency
        _case("norm_one_1b", "norm", "bf16", 32, 8, 64, 64, 1, (1, 1), (4096, 4096), rot=64, pairs=False, bounds=True, norm=True),
        # prefill chunks of odd lengths behind prefixes, token-major pages, adjacent pairs, half of the dims rotated
        _case("norm_chunk_3b", "norm", "fp16", 24, 8, 128, 16, 4, (3000, 4096), (4097, 9000), tokens_first=True, rot=64, pairs=True,
              bounds=True, norm=True),
        # a decode batch: one row per sequence, each into a page that is partly filled
        _case("write_batch_3b", "write", "bf16", 24, 8, 128, 64, 32, (1, 1), (1000, 4096), rot=128, pairs=False, bounds=True, norm=True),
        # prefill chunks of every length, no norms and no bounds
        _case("write_chunk_1b", "write", "bf16", 32, 8, 64, 32, 6, (900, 5000), (900, 12000), rot=64, pairs=False, bounds=False, norm=False),
        # a few short prefixes handed on
        _case("read_some_1b", "read", "fp16", 32, 8, 64, 16, 3, (1, 1), (200, 700), tokens_first=True),
        # long sequences' whole caches, for a pass that reads 16 bits
        _case("read_batch_3b", "read", "bf16", 24, 8, 128, 64, 8, (1, 1), (8192, 65536)),
        # one sequence decodes one token over a short context
        _case("attend_one_1b", "attend", "bf16", 32, 8, 64, 64, 1, (1, 1), (4096, 4096), causal=True),
        # a decode batch of ragged long sequences: the cache is read once
        _case("attend_batch_3b", "attend", "bf16", 24, 8, 128, 64, 32, (1, 1), (8192, 65536), causal=True),
        # a chunk of a prompt at the end of a 64K context: matrix products
        _case("attend_chunk_3b_64k", "attend", "bf16", 24, 8, 128, 64, 1, (2048, 2048), (65536, 65536), causal=True),
        # a mixed step: decoding sequences and chunks of every length in one call, small pages, token-major
        _case("attend_mixed_1b", "attend", "fp16", 32, 8, 64, 16, 24, (1, 400), (700, 20000), causal=True, tokens_first=True),
        # one sequence decodes over 128K tokens, 35 of 2048 pages read
        _case("block_one_3b_128k", "block", "bf16", 24, 8, 128, 64, 1, (1, 1), (131072, 131072), sink=1, tail=2, topk=32),
        # the ragged decode batch
        _case("block_batch_3b", "block", "bf16", 24, 8, 128, 64, 32, (1, 1), (8192, 65536), sink=1, tail=2, topk=32),
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
        op = rng.choice(["norm", "write", "read", "attend", "attend", "block"])
        hq, hkv, d = rng.choice([(32, 8, 64), (24, 8, 128), (8, 2, 64), (6, 6, 128), (16, 2, 128)])
        decode = rng.random() < 0.5
        batch = _spread(rng, 1, 48)
        q_hi = 1 if decode or op == "read" else _spread(rng, 2, {"norm": 8192, "write": 8192, "attend": 8192, "block": 96}[op])
        q_lo = 1 if decode or op == "read" else _spread(rng, 1, q_hi)
        kv_hi = max(q_hi, _spread(rng, 1, {"norm": 16384, "write": 16384, "read": 65536, "attend": 131072, "block": 131072}[op]))
        kv_lo = _spread(rng, 1, kv_hi)
        c = _case("", op, rng.choice(["bf16", "fp16"]), hq, hkv, d, rng.choice([16, 32, 64, 128]), batch,
                  (q_lo, q_hi), (kv_lo, kv_hi), lens=rng.randrange(1 << 20), tokens_first=rng.random() < 0.5)
        if op in ("norm", "write"):
            c.update(rot=rng.choice([0, d // 2, d, d]), pairs=rng.random() < 0.3, bounds=rng.random() < 0.6,
                     norm=op == "norm" or rng.random() < 0.5)
        elif op == "attend":
            c.update(causal=rng.random() < 0.8)
        elif op == "block":
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
    row = c["d"] * 2                                        # a 16-bit row; an 8-bit one is c["d"] + 1
    held = c["d"] + 1
    if c["op"] in ("norm", "write"):
        touched = sum((n - 1) // c["page"] - (n - m) // c["page"] + 1 for m, n in zip(q_lens, kv_lens))
        moved = new * row * 2 * c["hq"] + new * 2 * c["hkv"] * (row + (row if c["op"] == "norm" else held))
        moved += touched * c["hkv"] * 2 * row if c["bounds"] else 0
        return {"bytes": moved, "flops": new * (c["hq"] + c["hkv"]) * (3 * c["rot"] + (4 * c["d"] if c["norm"] else 0))}
    if c["op"] == "read":
        return {"bytes": sum(kv_lens) * 2 * c["hkv"] * (held + row), "flops": sum(kv_lens) * 2 * c["hkv"] * c["d"]}
    out = new * c["hq"] * (2 * row + 4)
    if c["op"] == "attend":
        seen = sum(m * n - (m * (m - 1) // 2 if c["causal"] else 0) for m, n in zip(q_lens, kv_lens))
        return {"bytes": sum(kv_lens) * c["hkv"] * 2 * held + out, "flops": 4 * c["d"] * c["hq"] * seen}
    # every page's bounds once per sequence, and each new token's selected rows (a chunk's tokens may share them: at
    # least those of one token)
    pages = sum((n + c["page"] - 1) // c["page"] for n in kv_lens)
    seen = [_selected(c, n - m + i) for m, n in zip(q_lens, kv_lens) for i in range(m)]
    first = [_selected(c, n - 1) for n in kv_lens]
    scored = sum(m * ((n + c["page"] - 1) // c["page"]) for m, n in zip(q_lens, kv_lens))
    kept = c["sink"] + c["tail"] + c["topk"]
    return {"bytes": pages * c["hkv"] * 2 * row + sum(first) * c["hkv"] * 2 * held + out + new * c["hkv"] * kept * 4,
            "flops": (4 * sum(seen) + 2 * scored) * c["d"] * c["hq"]}


# ---------------------------------------------------------------------------------------------- inputs
def _held(x):
    """Codes and scales that rows x [.., dim] are held as: the scale's exponent from the largest magnitude m 2^e,
    1/2 <= m < 1, of which 448 = 0.875 * 2^9 is the most that a code can say."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(-126, 127)
    codes = (x * torch.exp2(-e.to(x.dtype))).float().to(torch.float8_e4m3fn)
    return codes, (e[..., 0] + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(codes, scales):
    return codes.float() * scales.float()[..., None]


def prepare(case, seed):
    """A filled paged cache (pages in random order, rows of different sizes, some keys along the queries' topic so that
    attention is peaked) and the step's inputs."""
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
    v.mul_(torch.exp2(torch.randn(shape[:3], dtype=dt, device=dev, generator=g))[..., None])
    if c["tokens_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)           # [page, head, slot, dim], whatever the storage
    order = torch.randperm(n_pages, device=dev, generator=g).int()
    table = torch.full((batch, max(n_seq)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(n_seq):
        table[b, :n] = order[at:at + n]
        at += n
    topic = torch.randn(batch, hkv, d, device=dev, generator=g)
    lens = torch.tensor(kv_lens, device=dev)
    seq_of = torch.repeat_interleave(torch.arange(batch, device=dev), torch.tensor(q_lens, device=dev))
    # a key in about 500 is three times its sequence's topic
    pick = torch.repeat_interleave(torch.arange(batch, device=dev), lens // 500 + 1)
    pos = (torch.rand(pick.numel(), device=dev, generator=g) * lens[pick]).long().clamp_max(lens[pick] - 1)
    k[table[pick, pos // ps].long(), :, pos % ps] = (3 * topic[pick]).to(dt)
    first = torch.tensor([n - m for m, n in zip(q_lens, kv_lens)], device=dev)
    cu_q = [0]
    for m in q_lens:
        cu_q.append(cu_q[-1] + m)
    start = torch.tensor(cu_q[:-1], device=dev)
    s = {"c": c, "dt": dt, "k": k, "v": v, "table": table, "q_lens": q_lens, "kv_lens": kv_lens, "cu_q": cu_q, "seq_of": seq_of,
         "lens": lens, "pos": torch.arange(new, device=dev) - start[seq_of] + first[seq_of], "bounds": None}
    if c["op"] != "norm":
        s["k"], s["k_scales"] = _held(k.float())
        s["v"], s["v_scales"] = _held(v.float())
        if c["tokens_first"]:                                  # codes as they were stored, scales by head
            s["k"], s["v"] = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (s["k"], s["v"]))
        s["k_scales"], s["v_scales"] = s["k_scales"].contiguous(), s["v_scales"].contiguous()
    if c["op"] in ("norm", "write"):
        # the projections' output: query, key and value heads of a token beside each other
        qkv = torch.randn(new, hq + 2 * hkv, d, dtype=dt, device=dev, generator=g)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_out"] = torch.empty(new, hq, d, dtype=dt, device=dev)
        s["inv_freq"] = None
        if c["rot"]:
            s["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().to(dev)
        if c["norm"]:
            s["q_weight"] = 1 + 0.2 * torch.randn(d, device=dev, generator=g)
            s["k_weight"] = 1 + 0.2 * torch.randn(d, device=dev, generator=g)
        if c["bounds"]:
            s["bounds"] = torch.zeros(n_pages, hkv, 2, d, dtype=dt, device=dev)
    elif c["op"] == "read":
        # [head][row][dim], as the summary build takes a cache
        s["seq_of_row"] = torch.repeat_interleave(torch.arange(batch, device=dev), lens)
        s["pos_of_row"] = torch.arange(sum(kv_lens), device=dev) - (lens.cumsum(0) - lens)[s["seq_of_row"]]
        s["k_out"] = torch.empty(hkv, sum(kv_lens), d, dtype=dt, device=dev)
        s["v_out"] = torch.empty_like(s["k_out"])
    else:
        mixed = torch.randn(new, hkv, hq // hkv, d, device=dev, generator=g)
        s["q"] = (0.25 * topic[seq_of][:, :, None] + math.sqrt(1 - 0.25 ** 2) * mixed).reshape(new, hq, d).to(dt)
        s["y"] = torch.empty(new, hq, d, dtype=dt, device=dev)
        s["lse"] = torch.empty(new, hq, dtype=torch.float32, device=dev)
        if c["op"] == "block":
            held = _values(s["k"], s["k_scales"])
            s["bounds"] = torch.stack([held.amin(2), held.amax(2)], 2).to(dt)
            s["idx"] = torch.empty(new, hkv, c["sink"] + c["tail"] + c["topk"], dtype=torch.int32, device=dev)
    if own:
        import numpy as np

        import paper_2604_05438_b200 as T
        step = (table, np.array(kv_lens, np.int64), np.array(cu_q, np.int64), hq)
        if c["op"] == "norm":
            s["kv"] = T.PagedKVCache(s["k"], s["v"], *step, s["bounds"])
        else:
            s["kv"] = T.PagedKVCache8(s["k"], s["v"], s["k_scales"], s["v_scales"], *step, dt, s["bounds"])
        if c["op"] in ("norm", "write"):
            s["rotary"] = T.RotaryMap(s["inv_freq"], c["pairs"]) if c["rot"] else None
            s["norms"] = T.HeadNorms(s["q_weight"], s["k_weight"], EPS) if c["norm"] else None
        elif c["op"] == "read":
            s["rows"] = T.CacheRows(np.concatenate([[0], np.cumsum(kv_lens)]), device=dev)
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
        if c["op"] in ("norm", "write"):
            T.paged_append(s["kv"], s["k_new"], s["v_new"], s["rotary"], s["q"], s["q_out"], norms=s["norms"])
            return _written(s)
        if c["op"] == "read":
            T.paged_read(s["kv"], s["rows"], s["k_out"].transpose(0, 1), s["v_out"].transpose(0, 1))
            return {"k": s["k_out"], "v": s["v_out"]}
        if c["op"] == "attend":
            flags = 0 if c["causal"] else T.FLAG_FULL_CONTEXT
            T.paged_attention(s["kv"], s["q"], s["y"], s["lse"], None, flags, s["ws"])
            return {"y": s["y"], "lse": s["lse"]}
        T.paged_block_attention(s["kv"], s["sel"], s["q"], s["y"], s["lse"], s["idx"], None, s["ws"])
        return {"y": s["y"], "lse": s["lse"], "pages": s["idx"]}
    plain = {"norm": _plain_append, "write": _plain_append, "read": _plain_read, "attend": _plain_attend, "block": _plain_block}
    return plain[c["op"]](s)


def _written(s):
    out = {"k": s["k"], "v": s["v"], "q": s["q_out"], "bounds": s["bounds"]}
    if s["c"]["op"] == "write":
        out["k_scales"], out["v_scales"] = s["k_scales"], s["v_scales"]
    return out


def _rotated(x, angle, pairs):
    """x [rows, heads, d] in 32 bits, the first 2 * angle.shape[1] dims of each head rotated."""
    n = angle.shape[1]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if pairs else (x[..., :n], x[..., n:2 * n])
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if pairs else torch.cat(turned, -1)
    return torch.cat([turned, x[..., 2 * n:]], -1)


def _normed(x, weight):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight


def _plain_append(s):
    c = s["c"]
    ps = c["page"]
    k_new, v_new, q = s["k_new"].float(), s["v_new"].float(), s["q"].float()
    if c["norm"]:
        k_new, q = _normed(k_new, s["k_weight"]), _normed(q, s["q_weight"])
    if c["rot"]:
        angle = s["pos"].double()[:, None] * s["inv_freq"].double()      # far positions: 32 bits lose the angle
        k_new, q = _rotated(k_new, angle, c["pairs"]), _rotated(q, angle, c["pairs"])
    page, slot = s["table"][s["seq_of"], s["pos"] // ps].long(), s["pos"] % ps
    if c["op"] == "write":
        for x, codes, scales in ((k_new, s["k"], s["k_scales"]), (v_new, s["v"], s["v_scales"])):
            new_codes, new_scales = _held(x)
            codes.view(torch.uint8)[page, :, slot] = new_codes.view(torch.uint8)
            scales.view(torch.uint8)[page, :, slot] = new_scales.view(torch.uint8)
    else:
        s["k"][page, :, slot] = k_new.to(s["dt"])
        s["v"][page, :, slot] = s["v_new"]
    s["q_out"].copy_(q)
    if s["bounds"] is not None:
        # the touched pages, once each, and how many of their slots hold a row now
        b_of, page_of = torch.unique(torch.stack([s["seq_of"], s["pos"] // ps], 1), dim=0).unbind(1)
        empty = torch.arange(ps, device=page.device) >= (s["lens"][b_of] - page_of * ps)[:, None]
        phys = s["table"][b_of, page_of].long()
        if c["op"] == "write":
            rows = s["k"].view(torch.uint8)[phys].view(torch.float8_e4m3fn)
            rows = _values(rows, s["k_scales"].view(torch.uint8)[phys].view(torch.float8_e8m0fnu))
        else:
            rows = s["k"][phys].float()
        low = rows.masked_fill(empty[:, None, :, None], math.inf).amin(2)
        high = rows.masked_fill(empty[:, None, :, None], -math.inf).amax(2)
        s["bounds"][phys] = torch.stack([low, high], 2).to(s["dt"])
    return _written(s)


def _plain_read(s):
    ps = s["c"]["page"]
    page, slot = s["table"][s["seq_of_row"], s["pos_of_row"] // ps].long(), s["pos_of_row"] % ps
    for name in ("k", "v"):
        codes = s[name].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn)                 # [row, head, dim]
        scales = s[name + "_scales"].view(torch.uint8)[page, :, slot].view(torch.float8_e8m0fnu)
        s[name + "_out"].copy_(_values(codes, scales).transpose(0, 1))
    return {"k": s["k_out"], "v": s["v_out"]}


def _rows(s, name, pages):
    """Held values of the given pages [.., page, head, slot, dim]."""
    codes = s[name].view(torch.uint8)[pages].view(torch.float8_e4m3fn)
    return _values(codes, s[name + "_scales"].view(torch.uint8)[pages].view(torch.float8_e8m0fnu))


def _plain_attend(s):
    c = s["c"]
    hkv, group, d = c["hkv"], c["hq"] // c["hkv"], c["d"]
    ys, lses = [], []
    for b, (m, n) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        pages = s["table"][b, :(n + c["page"] - 1) // c["page"]].long()
        key = _rows(s, "k", pages).transpose(0, 1).reshape(hkv, -1, d)[:, :n]
        val = _rows(s, "v", pages).transpose(0, 1).reshape(hkv, -1, d)[:, :n]
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
            ys.append(y.transpose(0, 1).flatten(1, 2).to(s["dt"]))
            lses.append((top + total.log()).view(hkv, -1, group).transpose(0, 1).flatten(1, 2))
    return {"y": torch.cat(ys), "lse": torch.cat(lses)}


def _plain_block(s):
    c = s["c"]
    hkv, group, d, ps = c["hkv"], c["hq"] // c["hkv"], c["d"], c["page"]
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
            at = (table[use.clamp_max(n_pages - 1)], heads)
            where = use[..., None] * ps + torch.arange(ps, device=dev)
            masked = ((use == n_pages)[..., None] | (where > pos[..., None, None])).flatten(2)[:, :, None]
            key = _rows(s, "k", at).flatten(2, 3)                            # [row][head][key][dim]
            score = q_all[rows].float() @ key.transpose(2, 3) / math.sqrt(d)
            score.masked_fill_(masked, -math.inf)
            del key
            top = score.amax(3, keepdim=True)
            score.sub_(top).exp_()
            total = score.sum(3, keepdim=True)
            ys.append((score @ _rows(s, "v", at).flatten(2, 3) / total).flatten(1, 2).to(s["dt"]))
            lses.append((top + total.log()).flatten(1))
            ids.append(idx.masked_fill(none, -1).int())
    return {"y": torch.cat(ys), "lse": torch.cat(lses), "pages": torch.cat(ids)}


# ---------------------------------------------------------------------------------------------- from the definition
def exact(case, seed):
    """The outputs of `run` from the operators' definitions in 64 bits (codes before their rounding)."""
    global own
    kept_own, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept_own
    parts = {"norm": _exact_append, "write": _exact_append, "read": _exact_read, "attend": _exact_attend, "block": _exact_block}
    return parts[case["op"]](s)


def _power(scales):
    return torch.pow(2.0, scales.view(torch.uint8).double() - 127)


def _exact_append(s):
    c = s["c"]
    ps, n = c["page"], c["rot"] // 2
    if s["k"].numel() > 1 << 28:
        return None
    key, val, q = s["k"].double(), s["v"].double(), s["q"].double().clone()
    row, vrow = s["k_new"].double().clone(), s["v_new"].double().clone()
    if c["norm"]:
        for x, w in ((row, s["k_weight"]), (q, s["q_weight"])):
            x /= ((x * x).sum(-1, keepdim=True) / c["d"] + EPS).sqrt()
            x *= w.double()
    for x in (row, q):
        if n:
            # each pair as a complex number, times e^(i angle)
            turn = torch.polar(torch.ones_like(s["pos"], dtype=torch.float64)[:, None],
                               s["pos"].double()[:, None] * s["inv_freq"].double())[:, None]
            first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["pairs"] else (slice(0, n), slice(n, 2 * n))
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
    scales = {}
    if c["op"] == "write":
        scales = {"k_scales": _power(s["k_scales"]), "v_scales": _power(s["v_scales"])}
        size = []
        for x in (row, vrow):
            # the smallest power of two of which 448 reach the largest magnitude
            size.append(torch.pow(2.0, torch.ceil(torch.log2(x.abs().max(-1).values / 448)).clamp_min(-126)))
            x /= size[-1][..., None]
    # (the bounds of an 8-bit cache are those of rounded codes: there is no value of theirs before the rounding)
    bounds = None if s["bounds"] is None or c["op"] == "write" else s["bounds"].double()
    for b, (m, length) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        begin, lo = length - m, s["cu_q"][b]
        for p in range(begin // ps, (length - 1) // ps + 1):
            phys = int(s["table"][b, p])
            t0, t1 = max(begin, p * ps), min(length, (p + 1) * ps)
            at, of = slice(t0 - p * ps, t1 - p * ps), slice(lo + t0 - begin, lo + t1 - begin)
            key[phys, :, at] = row[of].transpose(0, 1)
            val[phys, :, at] = vrow[of].transpose(0, 1)
            if scales:
                scales["k_scales"][phys, :, at] = size[0][of].T
                scales["v_scales"][phys, :, at] = size[1][of].T
            if bounds is not None:
                have = key[phys, :, :t1 - p * ps]
                bounds[phys, :, 0], bounds[phys, :, 1] = have.min(1).values, have.max(1).values
    return {"k": key, "v": val, "q": q, "bounds": bounds, **scales}


def _rows_of(s, name, table, n):
    """Rows 0 .. n-1 of a sequence, [head, row, dim] in 64 bits."""
    pages = table.long()
    x = s[name].permute(0, 2, 1, 3).view(torch.uint8)[pages].view(torch.float8_e4m3fn).double()
    x *= _power(s[name + "_scales"].view(torch.uint8)[pages]).transpose(1, 2)[..., None]
    return x.reshape(-1, x.shape[2], x.shape[3])[:n].permute(1, 0, 2)


def _exact_read(s):
    if s["k_out"].numel() > 1 << 29:
        return None
    out = {"k": [], "v": []}
    for b, n in enumerate(s["kv_lens"]):
        for name in out:
            out[name].append(_rows_of(s, name, s["table"][b, :-(-n // s["c"]["page"])], n))
    return {name: torch.cat(x, 1) for name, x in out.items()}


def _exact_attend(s):
    c = s["c"]
    group, d = c["hq"] // c["hkv"], c["d"]
    y = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=s["q"].device)
    for b, (m, n) in enumerate(zip(s["q_lens"], s["kv_lens"])):
        table = s["table"][b, :-(-n // c["page"])]
        key, val = _rows_of(s, "k", table, n), _rows_of(s, "v", table, n)
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

    def held(name, phys, h, slot):
        codes = s[name].view(torch.uint8)[phys, h, slot].view(torch.float8_e4m3fn).double()
        return codes * _power(s[name + "_scales"].view(torch.uint8)[phys, h, slot])[:, None]

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
            key, val = held("k", table[at // ps], h, at % ps), held("v", table[at // ps], h, at % ps)
            score = q @ key.T / math.sqrt(d)
            lse[t, h * group:(h + 1) * group] = score.logsumexp(1)
            y[t, h * group:(h + 1) * group] = torch.softmax(score, 1) @ val
    return {"y": y, "lse": lse, "pages": pages}
