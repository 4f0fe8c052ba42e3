"""Operators of the paged key/value cache: what is measured, and their plain forms in elementary torch operations.

Three operators share one cache of pages: `write` stores (and quantises) the keys and values of new tokens, `read`
brings a range of positions back as numbers, `attend` is causal grouped-query attention of a chunk of new tokens (one
token per sequence in a decode step) over everything the cache holds for their sequences.

Pools are [n_pages][n_kv_heads][page_size][head_dim] in bf16, e4m3 or int8; 8-bit pools have one float32 scale per
(token, kv head).  Sequence b owns the packed rows cu_rows[b] .. cu_rows[b+1], row i being position
kv_len[b] - n_b + i; position p lies in row p % page_size of page page_table[b][p // page_size].
"""
import math
import random

import torch

own = False

QMAX = {"e4m3": 448.0, "int8": 127.0}
POOL = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
MIN_AMAX = 2.0 ** -110  # smaller row maxima are treated as this one (its reciprocal still fits in float32)


def _case(op, dtype, heads, kv_heads, head_dim, page, batch, rows, kv, spread, out="bf16", name=None):
    c = {"op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
         "batch": batch, "rows": rows, "kv": kv, "spread": spread, "out": out}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of 64 sequences: a token each goes into the cache (latency)
        _case("write", "e4m3", 32, 8, 128, 16, 64, 1, 2000, 0.9, name="write_step_e4m3"),
        # ragged prompts of a small model
        _case("write", "int8", 16, 4, 64, 32, 5, 300, 700, 0.8, name="write_ragged_int8"),
        # the prompts of a whole batch after its prefill pass
        _case("write", "e4m3", 32, 8, 128, 16, 8, 4096, 4096, 0.0, name="write_prompts_e4m3"),
        # a short context read back in float32 for inspection
        _case("read", "int8", 16, 4, 64, 32, 3, 211, 333, 0.5, "f32", name="read_ragged_int8"),
        # long contexts read back as bf16, e.g. to move them to a pass that wants plain keys and values
        _case("read", "e4m3", 32, 8, 128, 64, 4, 16384, 16384, 0.3, name="read_long_e4m3"),
        # a single user's decode step on a small model (latency)
        _case("attend", "bf16", 16, 4, 64, 16, 1, 1, 500, 0.0, name="attend_step_one_bf16"),
        # decode step of a served batch
        _case("attend", "bf16", 32, 8, 128, 16, 64, 1, 4096, 0.7, name="attend_step_batch_bf16"),
        # decode step over two very long contexts, many query heads
        _case("attend", "e4m3", 64, 8, 128, 64, 2, 1, 131072, 0.1, name="attend_step_long_e4m3"),
        # checking five drafted tokens per sequence
        _case("attend", "int8", 32, 8, 128, 16, 16, 5, 8192, 0.6, name="attend_drafts_int8"),
        # chunked prefill of a batch, half-way through its prompts
        _case("attend", "bf16", 32, 8, 128, 16, 8, 512, 4096, 0.2, name="attend_chunk_bf16"),
        # one chunk of a long document over an 8-bit cache
        _case("attend", "e4m3", 32, 8, 128, 64, 1, 1024, 32768, 0.0, name="attend_chunk_e4m3"),
        # ragged chunks of a small model
        _case("attend", "int8", 16, 4, 64, 32, 6, 200, 1500, 0.9, name="attend_ragged_int8"),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    heads = [(32, 8, 128), (64, 8, 128), (16, 4, 64), (4, 4, 64), (28, 4, 128), (12, 4, 64), (8, 1, 128), (32, 32, 128)]
    while True:
        op = rng.choice(["write", "read", "attend", "attend", "attend"])
        dtype = rng.choice(["bf16", "e4m3", "int8"])
        h, kvh, dh = rng.choice(heads)
        batch, page, spread = log(1, 128), rng.choice([16, 32, 64, 128]), rng.choice([0.0, 0.3, 0.9])
        kv = log(1, 131072)
        rows = min(kv, 1 if op == "attend" and rng.random() < 0.4 else log(1, 4096))
        c = _case(op, dtype, h, kvh, dh, page, batch, rows, kv, spread, rng.choice(["bf16", "f32"]) if op == "read" else "bf16")
        w = work(c)
        plain_scores = 4.0 * batch * h * rows * kv  # bytes of the plain form's score matrix
        if w["flops"] <= 5.3e11 and w["bytes"] <= 4e8 and 8.0 * batch * kv * kvh * dh <= 2.2e9 and (op != "attend" or plain_scores <= 4.3e9):
            return c


def _lengths(c):
    """Rows and cached positions of each sequence: part of the case, not of the seed."""
    r = random.Random("%d %d %d %s" % (c["batch"], c["rows"], c["kv"], c["spread"]))
    kv, rows = [], []
    for b in range(c["batch"]):
        first = b == 0  # the first sequence has the largest sizes
        k = c["kv"] if first else max(1, int(round(c["kv"] * (1 - c["spread"] * r.random()))))
        n = c["rows"] if first else max(1, int(round(c["rows"] * (1 - c["spread"] * r.random()))))
        kv.append(k)
        rows.append(min(n, k))
    return rows, kv


def _quantise(x, dtype):
    """x [..., dh] float32 -> codes, scales: one scale per vector."""
    amax = x.abs().amax(-1).clamp_min(MIN_AMAX)
    scale = amax / QMAX[dtype]
    # (a number over a tensor would be torch's reciprocal times the number: two roundings)
    y = x * torch.full_like(amax, QMAX[dtype]).div(amax).unsqueeze(-1)
    if dtype == "int8":
        y = y.round().clamp(-127, 127)
    else:
        y = y.clamp(-448, 448)
    return y.to(POOL[dtype]), scale


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(int(seed) * 1000003 + 17)
    rows, kv = _lengths(c)
    KV, dh, ps = c["kv_heads"], c["head_dim"], c["page"]
    n_pages_of = [-(-k // ps) for k in kv]
    width = max(n_pages_of)
    n_pages = sum(n_pages_of) + 3  # a few pages belong to nobody
    perm = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).cpu().tolist()
    table = torch.zeros(c["batch"], width, dtype=torch.int32)
    at = 0
    for b, n in enumerate(n_pages_of):
        table[b, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
        at += n
    # keys have a few loud channels, as trained models do
    loud = 1.0 + 3.0 * (torch.rand(KV, 1, dh, generator=g, device=dev) > 0.95)

    def pool(is_key):
        x = torch.randn(n_pages, KV, ps, dh, generator=g, device=dev, dtype=torch.bfloat16)
        if is_key:
            x = x * loud.to(torch.bfloat16)
        if c["dtype"] == "bf16":
            return x, None
        return _quantise(x.float(), c["dtype"])

    k_pool, k_scale = pool(True)
    v_pool, v_scale = pool(False)
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    qkv = torch.randn(cu[-1], (c["heads"] + 2 * KV) * dh, generator=g, device=dev, dtype=torch.bfloat16)
    dq, dkv = c["heads"] * dh, KV * dh
    return {
        "case": c, "k_pool": k_pool, "v_pool": v_pool, "k_scale": k_scale, "v_scale": v_scale,
        "page_table": table.to(dev), "cu_rows": torch.tensor(cu, dtype=torch.int32, device=dev),
        "kv_len": torch.tensor(kv, dtype=torch.int32, device=dev), "n_rows": cu[-1], "max_rows": max(rows), "max_kv": max(kv),
        # slices of the projection's output, as the framework lays it out: q heads, k heads, v heads
        "q": qkv[:, :dq], "k": qkv[:, dq:dq + dkv], "v": qkv[:, dq + dkv:],
    }


def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state, op)
    if op == "write":
        return _plain_write(state)
    if op == "read":
        return _plain_read(state)
    return _plain_attend(state)


def _run_own(s, op):
    from paper_2509_24257_b200 import binding as vb

    cache = vb.KVCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    rows = vb.PagedRows(s["page_table"], s["cu_rows"], s["kv_len"], s["max_rows"])
    if op == "write":
        vb.kv_write(cache, rows, s["k"], s["v"])
        return _pools(s)
    if op == "read":
        k, v = vb.kv_read(cache, rows, s["n_rows"], torch.float32 if s["case"]["out"] == "f32" else torch.bfloat16)
        return {"k": k, "v": v}
    return vb.op_attention_paged(s["q"], cache, rows)


def _pools(s):
    out = {"k": s["k_pool"], "v": s["v_pool"]}
    if s["k_scale"] is not None:
        out["k_scale"], out["v_scale"] = s["k_scale"], s["v_scale"]
    return out


def _places(s):
    """(sequence, position, page, row inside the page) of every packed row."""
    cu, kv, n = s["cu_rows"].long(), s["kv_len"].long(), s["n_rows"]
    counts = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(counts.shape[0], device=cu.device), counts, output_size=n)
    pos = kv[seq] - counts[seq] + torch.arange(n, device=cu.device) - cu[seq]
    ps = s["case"]["page"]
    return seq, pos, s["page_table"][seq, pos // ps].long(), pos % ps


def _plain_write(s):
    c = s["case"]
    _, _, page, off = _places(s)
    k, v = s["k"].reshape(-1, c["kv_heads"], c["head_dim"]), s["v"].reshape(-1, c["kv_heads"], c["head_dim"])
    if c["dtype"] == "bf16":
        s["k_pool"][page, :, off] = k
        s["v_pool"][page, :, off] = v
        return _pools(s)
    kc, ks = _quantise(k.float(), c["dtype"])
    vc, vs = _quantise(v.float(), c["dtype"])
    # indexed stores are made on the bytes: torch has none for 8-bit floats
    s["k_pool"].view(torch.uint8)[page, :, off] = kc.view(torch.uint8)
    s["v_pool"].view(torch.uint8)[page, :, off] = vc.view(torch.uint8)
    s["k_scale"][page, :, off] = ks
    s["v_scale"][page, :, off] = vs
    return _pools(s)


def _gather(pool, page, off):
    x = pool.view(torch.uint8)[page, :, off].view(pool.dtype) if pool.element_size() == 1 else pool[page, :, off]
    return x.float()


def _plain_read(s):
    c = s["case"]
    _, _, page, off = _places(s)
    k, v = _gather(s["k_pool"], page, off), _gather(s["v_pool"], page, off)
    if s["k_scale"] is not None:
        k, v = k * s["k_scale"][page, :, off].unsqueeze(-1), v * s["v_scale"][page, :, off].unsqueeze(-1)
    dt = torch.float32 if c["out"] == "f32" else torch.bfloat16
    return {"k": k.to(dt), "v": v.to(dt)}


def _context(s, pool, scale):
    """The sequences' pages side by side in float32: [batch][kv heads][positions][head_dim]."""
    pages = s["page_table"].long()
    x = pool.view(torch.uint8)[pages].view(pool.dtype) if pool.element_size() == 1 else pool[pages]
    x = x.float()
    if scale is not None:
        x = x * scale[pages].unsqueeze(-1)
    b, w, kvh, ps, dh = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(b, kvh, w * ps, dh)


def _plain_attend(s):
    c = s["case"]
    H, KV, dh, B, R = c["heads"], c["kv_heads"], c["head_dim"], c["batch"], s["max_rows"]
    G = H // KV
    seq, pos, _, _ = _places(s)
    i = torch.arange(s["n_rows"], device=seq.device) - s["cu_rows"].long()[seq]
    q = torch.zeros(B, R, KV, G, dh, device=seq.device)
    q[seq, i] = s["q"].reshape(-1, KV, G, dh).float()
    at = torch.full((B, R), -1, dtype=torch.long, device=seq.device)  # position of each row; padding sees key 0 only
    at[seq, i] = pos
    q = q.permute(0, 2, 3, 1, 4).reshape(B, KV, G * R, dh)
    k = _context(s, s["k_pool"], s["k_scale"])
    scores = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(dh)).view(B, KV, G, R, -1)
    del k
    hidden = torch.arange(scores.shape[-1], device=seq.device) > at.clamp_min(0).unsqueeze(-1)
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    p = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    v = _context(s, s["v_pool"], s["v_scale"])
    o = torch.matmul(p.view(B, KV, G * R, -1), v).view(B, KV, G, R, dh).div_(total)
    return o.permute(0, 3, 1, 2, 4)[seq, i].reshape(s["n_rows"], H * dh).to(torch.bfloat16)


def work(case):
    c = case
    rows, kv = _lengths(c)
    n, KV, dh = sum(rows), c["kv_heads"], c["head_dim"]
    stored = 2.0 * KV * (dh * 2 if c["dtype"] == "bf16" else dh + 4)  # bytes of one position, keys and values
    if c["op"] == "write":
        return {"bytes": n * (2.0 * KV * dh * 2 + stored), "flops": 0.0 if c["dtype"] == "bf16" else n * 2.0 * KV * dh * 2}
    if c["op"] == "read":
        return {"bytes": n * (2.0 * KV * dh * (4 if c["out"] == "f32" else 2) + stored), "flops": n * 2.0 * KV * dh}
    pairs = sum(r * (k - r) + r * (r + 1) / 2.0 for r, k in zip(rows, kv))
    return {"bytes": sum(kv) * stored + 2.0 * n * c["heads"] * dh * 2, "flops": 4.0 * c["heads"] * dh * pairs}


def exact(case, seed):
    """The definitions in float64, one sequence at a time."""
    c = case
    s = prepare(case, seed)
    rows, kv = _lengths(c)
    H, KV, dh, ps = c["heads"], c["kv_heads"], c["head_dim"], c["page"]

    if c["op"] == "write":
        if c["dtype"] == "bf16":
            return None  # a copy: no computed number
        out = {"k": None, "v": None}  # codes are compared with the plain form's
        table = s["page_table"].cpu().tolist()
        for name, x, scale in (("k_scale", s["k"], s["k_scale"]), ("v_scale", s["v"], s["v_scale"])):
            a = x.double().reshape(-1, KV, dh).abs().max(dim=-1).values.clamp(min=MIN_AMAX) / QMAX[c["dtype"]]
            full = scale.double()
            r0 = 0
            for b in range(c["batch"]):
                p = torch.arange(kv[b] - rows[b], kv[b])
                pg = torch.tensor(table[b])[p // ps].to(full.device)
                full[pg, :, (p % ps).to(full.device)] = a[r0:r0 + rows[b]]
                r0 += rows[b]
            out[name] = full
        return out

    def sequence(b, pool, scale):  # [kv][KV][dh] float64
        n = -(-kv[b] // ps)
        pg = s["page_table"][b, :n].long()
        x = (pool.view(torch.uint8)[pg].view(pool.dtype) if pool.element_size() == 1 else pool[pg]).double()
        if scale is not None:
            x = x * scale[pg].double()[..., None]
        return x.transpose(1, 2).reshape(n * ps, KV, dh)[:kv[b]]

    ks, vs, outs = [], [], []
    r0 = 0
    for b in range(c["batch"]):
        k, v = sequence(b, s["k_pool"], s["k_scale"]), sequence(b, s["v_pool"], s["v_scale"])
        n = rows[b]
        if c["op"] == "read":
            ks.append(k[kv[b] - n:])
            vs.append(v[kv[b] - n:])
        else:
            q = s["q"][r0:r0 + n].double().reshape(n, H, dh)
            last = torch.arange(kv[b] - n, kv[b], device=q.device)
            hide = torch.arange(kv[b], device=q.device)[None, :] > last[:, None]
            o = torch.empty(n, H, dh, dtype=torch.float64, device=q.device)
            for h in range(H):
                kh = h * KV // H
                t = (q[:, h] @ k[:, kh].T) / dh ** 0.5
                t[hide] = -torch.inf
                o[:, h] = torch.softmax(t, dim=-1) @ v[:, kh]
            outs.append(o.reshape(n, H * dh))
        r0 += n
    if c["op"] == "read":
        return {"k": torch.cat(ks), "v": torch.cat(vs)}
    return torch.cat(outs)
