"""Operators of a prover that serves: what is measured, and their plain forms in elementary torch operations.

`w4`: products with 4-bit weights, y[r][n] = sum_g scale[g][n] * sum_{k in g} x[r][k] * c[n][k] (+ y).  Codes c in -7 .. 7 lie as
c + 8 in uint8 [n][k / 2], the even k in the low half; one bf16 scale per group of 32, 64 or 128 inputs and output, [k / group][n].

`drafts`: the drafted tokens of a batch against the target's logits, with given random numbers.  Sequence b owns the rows
cu_rows[b] .. cu_rows[b+1]; row i has the input token tokens[i] and the logits of what follows it.  p = softmax(target / T), q =
softmax(draft / T), or one at the drafted token where there are no draft logits.  The token x of row i + 1 is accepted iff
accept_u[i + 1] * q(x) < p(x); the first one that is not is replaced by the first v at which the running sum of max(0, p - q) exceeds
sample_u[b] times its total; if all are accepted one more is taken from the last row's p in the same way.  T = 0: p is one at
the largest logit (lowest index) and a token is accepted iff it is that one.

`pages`: what happens to a paged cache's pages between attention calls.  refs counts the table entries that name a page (0: free).  reserve
grows sequences to given lengths, lowest free pages first, sequences in order; a sequence that would write into a shared page gets a
copy of it, unless all the others that hold it got theirs.  free shortens, fork lets an empty sequence share another's pages, copy brings
pages from another pool, compact moves the highest pages in use into the lowest holes.
"""
import math
import random

import torch

own = False

QMAX = {"e4m3": 448.0, "int8": 127.0}
POOL = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _w4(rows, n, k, group, out, add, name=None):
    c = {"op": "w4", "rows": rows, "n": n, "k": k, "group": group, "out": out, "add": add}
    return dict(c, name=name) if name else c


def _drafts(batch, rows, vocab, dtype, draft, spread, greedy, name=None):
    c = {"op": "drafts", "batch": batch, "rows": rows, "vocab": vocab, "dtype": dtype, "draft": draft, "spread": spread, "greedy": greedy}
    return dict(c, name=name) if name else c


def _pages(kind, dtype, layers, kv_heads, head_dim, page, batch, kv, rows, fan, name=None):
    c = {"op": "pages", "kind": kind, "dtype": dtype, "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
         "batch": batch, "kv": kv, "rows": rows, "fan": fan}
    return dict(c, name=name) if name else c


def listed():
    return [
        # output projection of one user's token (latency)
        _w4(1, 4096, 4096, 128, "bf16", False, name="w4_one_row"),
        # gate and up projections of one user's token
        _w4(1, 28672, 4096, 128, "bf16", False, name="w4_one_row_wide"),
        # down projection of five drafted tokens, added to the residual stream
        _w4(5, 4096, 14336, 64, "f32", True, name="w4_drafts_down"),
        # gate and up projections of a decode step of 64 sequences
        _w4(64, 28672, 4096, 128, "bf16", False, name="w4_batch_wide"),
        # one user's four drafted tokens (latency)
        _drafts(1, 5, 32000, "f32", True, 0.0, 0.0, name="drafts_one"),
        # tokens proposed by looking them up in the prompt (no draft distribution), odd vocabulary, some users greedy
        _drafts(17, 9, 50257, "f32", False, 0.8, 0.3, name="drafts_lookup_ragged"),
        # five drafted tokens of each of 64 sequences
        _drafts(64, 6, 128256, "bf16", True, 0.3, 0.1, name="drafts_batch"),
        # a decode step's pages: room for six rows each, and back to what was accepted (latency)
        _pages("step", "bf16", 2, 8, 128, 16, 64, 2000, 6, 2, name="pages_step"),
        # four samples of one prompt, small model (latency)
        _pages("fork", "int8", 4, 4, 64, 32, 1, 777, 1, 4, name="pages_fork_one"),
        # eight samples of each of eight prompts
        _pages("fork", "e4m3", 8, 8, 128, 64, 8, 4000, 1, 8, name="pages_fork_samples"),
        # a parked sequence comes back, others leave, the rest moves together; small model
        _pages("swap", "int8", 2, 4, 64, 32, 9, 1500, 1, 3, name="pages_swap_ragged"),
        # the same on a served batch
        _pages("swap", "bf16", 4, 8, 128, 16, 24, 6000, 1, 3, name="pages_swap_batch"),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        op = rng.choice(["w4", "drafts", "pages"])
        if op == "w4":
            group = rng.choice([32, 64, 128, 128])
            c = _w4(log(1, 64), 8 * log(8, 16032), group * log(1, 28672 // group), group, *rng.choice([("bf16", False), ("f32", False), ("f32", True)]))
            if c["n"] * c["k"] <= 28672 * 4096:
                return c
        elif op == "drafts":
            c = _drafts(log(1, 128), log(1, 16), log(100, 151936), rng.choice(["bf16", "f32"]), rng.random() < 0.6, rng.choice([0.0, 0.3, 0.9]),
                        rng.choice([0.0, 0.3, 1.0]))
            if c["batch"] * c["rows"] * c["vocab"] <= 64 * 6 * 128256:
                return c
        else:
            heads, dim = rng.choice([(8, 128), (4, 64), (1, 128), (16, 64), (2, 128)])
            kind = rng.choice(["step", "fork", "swap"])
            c = _pages(kind, rng.choice(["bf16", "e4m3", "int8"]), rng.choice([1, 2, 3, 5, 8]), heads, dim, rng.choice([16, 32, 64, 128]),
                       log(1, 16) if kind == "fork" else log(1, 256), log(1, 16384), log(1, 32), rng.choice([2, 3, 4, 7]))
            if work(c)["bytes"] <= 8.9e8 and _pool_bytes(c) <= 6e9:
                return c


# --------------------------------------------------------------------------- who holds which pages


def _ceil(a, b):
    return -(-a // b)


def _plan(c):
    """The lengths and sharing of a pages case, part of the case and not of the seed."""
    r = random.Random("%(kind)s %(batch)d %(kv)d %(rows)d %(fan)d %(page)d" % c)
    B, ps, kv, fan, rows = c["batch"], c["page"], c["kv"], c["fan"], c["rows"]
    p = {"parent": [], "src": [], "dst": [], "back": None}
    if c["kind"] == "step":
        # every fan-th sequence is a copy of the one before it that has not written since; a step adds `rows`, some are taken back
        p["len"] = [kv] + [max(1, int(kv * (0.1 + 0.9 * r.random()))) for _ in range(B - 1)]
        p["parent"] = [b - 1 if b and b % fan == 0 else -1 for b in range(B)]
        p["len"] = [p["len"][q] if q >= 0 else n for n, q in zip(p["len"], p["parent"])]
        p["grow"] = [n + rows for n in p["len"]]
        p["final"] = [n + 1 + int((rows - 1) * r.random()) for n in p["len"]]
    elif c["kind"] == "fork":
        p["len"] = [kv] + [max(1, int(kv * (0.3 + 0.7 * r.random()))) for _ in range(B - 1)] + [0] * (B * (fan - 1))
        p["src"] = [b for b in range(B) for _ in range(fan - 1)]
        p["dst"] = list(range(B, B * fan))
        full = p["len"][:B] + [p["len"][b] for b in p["src"]]
        p["grow"] = [n + rows for n in full]
        p["final"] = [n if i % 3 else p["len"][i] if i < B else 0 for i, n in enumerate(p["grow"])]  # every third one is dropped again
    else:
        # the last sequence was parked; every fan-th leaves
        p["len"] = [kv] + [max(1, int(kv * (0.2 + 0.8 * r.random()))) for _ in range(B - 1)] + [0]
        p["back"] = max(1, kv // 2)
        p["final"] = [0 if b % fan == fan - 1 else n for b, n in enumerate(p["len"][:B])] + [0]
        p["grow"] = [0] * B + [p["back"]]
    held = sum(_ceil(n, ps) for b, n in enumerate(p["len"]) if not p["parent"] or p["parent"][b] < 0)
    more = max(max(p["grow"]), max(p["len"]))
    p["width"] = _ceil(more, ps) + 1
    extra = sum(_ceil(g, ps) - _ceil(n, ps) + 1 for g, n in zip(p["grow"], p["len"]) if g > n)
    p["n_pages"] = held + extra + max(4, held // 4)
    return p


def _page_bytes(c):
    e = 2 if c["dtype"] == "bf16" else 1
    return 2.0 * c["kv_heads"] * c["page"] * (c["head_dim"] * e + (0 if e == 2 else 4))


def _pool_bytes(c):
    return _plan(c)["n_pages"] * _page_bytes(c) * c["layers"]


def _first_pages(c, p, seed):
    """Table, counts: pages in a random order, shared where a sequence has a parent."""
    perm = list(range(p["n_pages"]))
    random.Random(seed * 7919 + 5).shuffle(perm)
    table = [[0] * p["width"] for _ in p["len"]]
    refs = [0] * p["n_pages"]
    at = 0
    for b, n in enumerate(p["len"]):
        for j in range(_ceil(n, c["page"])):
            if p["parent"] and p["parent"][b] >= 0:
                table[b][j] = table[p["parent"][b]][j]
            else:
                table[b][j] = perm[at]
                at += 1
            refs[table[b][j]] += 1
    return table, refs


# --------------------------------------------------------------------------- inputs


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(int(seed) * 1000003 + 29)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device=dev, dtype=dtype)

    if c["op"] == "w4":
        w = normal(c["n"], c["k"] // c["group"], c["group"]) * 0.02
        scale = (w.abs().amax(-1) / 7).to(torch.bfloat16)
        codes = (w / scale.float().unsqueeze(-1)).round().clamp(-7, 7).add(8).to(torch.uint8).reshape(c["n"], c["k"] // 2, 2)
        x = normal(c["rows"], c["k"])
        x = x * (1 + 9 * (torch.rand(c["k"], generator=g, device=dev) > 0.99))  # a few loud channels, as trained models have
        return {"case": c, "codes": codes[..., 0] | (codes[..., 1] << 4), "scales": scale.t().contiguous(), "x": x.to(torch.bfloat16),
                "y": normal(c["rows"], c["n"]) if c["add"] else None}
    if c["op"] == "drafts":
        rows = _rows(c)
        cu = [sum(rows[:b]) for b in range(len(rows) + 1)]
        n, V = cu[-1], c["vocab"]
        target = normal(n, V) * 2.5
        draft = target + 0.6 * normal(n, V)
        temp = 0.5 + torch.rand(c["batch"], generator=g, device=dev)
        temp[torch.rand(c["batch"], generator=g, device=dev) < c["greedy"]] = 0.0
        seq = torch.repeat_interleave(torch.arange(c["batch"], device=dev), torch.tensor(rows, device=dev), output_size=n)
        # drafted tokens: drawn from the draft's distribution, the largest one where the user is greedy
        noise = -torch.log(torch.rand(n, V, generator=g, device=dev).clamp_min(1e-30)).clamp_min(1e-30).log()
        tokens = (draft - noise * temp[seq, None] * (1.0 if c["draft"] else 0.3)).argmax(-1)
        tokens = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), tokens[:-1]]).to(torch.int32)
        return {"case": c, "target": target.to(FLOAT[c["dtype"]]), "draft": draft.to(FLOAT[c["dtype"]]) if c["draft"] else None, "tokens": tokens,
                "cu_rows": torch.tensor(cu, dtype=torch.int32, device=dev), "max_rows": max(rows), "temperature": temp,
                "accept_u": torch.rand(n, generator=g, device=dev), "sample_u": torch.rand(c["batch"], generator=g, device=dev),
                "kv_len": torch.randint(max(rows), 5000, (c["batch"],), generator=g, device=dev, dtype=torch.int32), "seq": seq}
    p = _plan(c)
    table, refs = _first_pages(c, p, int(seed))
    B, W, N = len(p["len"]), p["width"], p["n_pages"]
    ints = torch.tensor([x for row in table for x in row] + p["len"] + refs, dtype=torch.int32).to(dev)

    def pools(n):
        shape = (c["layers"], n, c["kv_heads"], c["page"], c["head_dim"])
        if c["dtype"] == "bf16":
            return [normal(*shape, dtype=torch.bfloat16) for _ in range(2)] + [None, None]
        codes = [torch.randint(-100, 100, shape, generator=g, device=dev, dtype=torch.int8) for _ in range(2)]
        codes = [x if c["dtype"] == "int8" else (x.to(torch.bfloat16) * 4).to(torch.float8_e4m3fn) for x in codes]
        return codes + [torch.rand(*shape[:-1], generator=g, device=dev) * 0.01 + 0.001 for _ in range(2)]

    s = {"case": c, "pools": pools(N), "ints0": ints, "ints": ints.clone(), "table": None, "n_parked": 0,
         "grow": torch.tensor(p["grow"], dtype=torch.int32, device=dev), "final": torch.tensor(p["final"], dtype=torch.int32, device=dev),
         "src": torch.tensor(p["src"], dtype=torch.int32, device=dev), "dst": torch.tensor(p["dst"], dtype=torch.int32, device=dev)}
    s["table"], s["kv_len"], s["refs"] = s["ints"][:B * W].view(B, W), s["ints"][B * W:B * W + B], s["ints"][B * W + B:]
    if p["back"]:
        s["n_parked"] = _ceil(p["back"], c["page"])
        s["parked"] = pools(s["n_parked"] + 2)
        s["parked_pages"] = torch.randperm(s["n_parked"] + 2, generator=g, device=dev)[:s["n_parked"]].to(torch.int32)
    return s


def _rows(c):
    """Rows of each sequence of a drafts case: the drafted tokens and the one before them."""
    r = random.Random("%d %d %s" % (c["batch"], c["rows"], c["spread"]))
    return [c["rows"]] + [max(1, int(round(c["rows"] * (1 - c["spread"] * r.random())))) for _ in range(c["batch"] - 1)]


# --------------------------------------------------------------------------- one pass


def run(state):
    op = state["case"]["op"]
    if own:
        return {"w4": _own_w4, "drafts": _own_drafts, "pages": _own_pages}[op](state)
    return {"w4": _plain_w4, "drafts": _plain_drafts, "pages": _plain_pages}[op](state)


def _own_w4(s):
    from paper_2509_24257_b200 import binding as vb

    w = vb.W4Weights(s["codes"], s["scales"], s["case"]["group"])
    return vb.op_w4_matvec(s["x"], w, residual=s["y"], dtype=FLOAT[s["case"]["out"]])


def _plain_w4(s):
    c = s["case"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).reshape(c["n"], -1, c["group"]).float() - 8
    w = (codes * s["scales"].t().float().unsqueeze(-1)).reshape(c["n"], c["k"])
    y = torch.matmul(s["x"].float(), w.t())
    if c["add"]:
        y = y + s["y"]
    return y.to(FLOAT[c["out"]])


def _own_drafts(s):
    from paper_2509_24257_b200 import binding as vb

    r = vb.verify_drafts(s["target"], s["tokens"], s["cu_rows"], s["max_rows"], s["accept_u"], s["sample_u"], draft=s["draft"],
                         temperature=s["temperature"], kv_len=s["kv_len"])
    return {"tokens": r.tokens, "n_emitted": r.n_emitted, "logp": r.logp, "new_len": r.new_len}


def _probabilities(logits, temp):
    """Unnormalised probabilities of rows in float64 (they come from differences next to borders), the largest one being 1."""
    x = logits.double()
    top = x.amax(-1, keepdim=True)
    e = ((x - top) / torch.where(temp > 0, temp, 1.0).double().unsqueeze(-1)).exp_()
    first = (x == top).to(torch.uint8).argmax(-1)
    at = torch.arange(x.shape[-1], device=x.device)
    return torch.where((temp > 0).unsqueeze(-1), e, (at == first.unsqueeze(-1)).double())


def _plain_drafts(s):
    c, n, seq = s["case"], s["target"].shape[0], s["seq"]
    dev = seq.device
    cu = s["cu_rows"].long()
    first, count = cu[:-1], cu[1:] - cu[:-1]
    row = torch.arange(n, device=dev)
    i = row - first[seq]
    temp = s["temperature"][seq]
    p = _probabilities(s["target"], temp)
    p = p / p.sum(-1, keepdim=True)
    follows = s["tokens"].long()[(row + 1).clamp(max=n - 1)]  # the drafted token that row's logits are about
    drafted = i < count[seq] - 1
    px = p.gather(1, follows.unsqueeze(1)).squeeze(1)
    greedy = temp == 0
    if s["draft"] is not None:
        q = _probabilities(s["draft"], temp)
        q = q / q.sum(-1, keepdim=True)
        qx = q.gather(1, follows.unsqueeze(1)).squeeze(1)
    else:
        q, qx = None, torch.ones_like(px)
    u = s["accept_u"][(row + 1).clamp(max=n - 1)].double()
    ok = torch.where(greedy, px > 0, u * qx < px)
    # the first row of each sequence at which no drafted token was accepted
    stop = torch.where(drafted & ok, c["rows"], i)
    last = torch.full((c["batch"],), c["rows"], device=dev).scatter_reduce(0, seq, stop, "amin")
    at = first + last
    r = p[at]
    if q is None:
        left = r.scatter(1, follows[at].unsqueeze(1), 0.0)
    else:
        left = (r - q[at]).clamp_min(0.0)
    left = torch.where((drafted[at] & ~greedy[at]).unsqueeze(1), left, r)
    left = torch.where(left.sum(-1, keepdim=True) > 0, left, r)
    run_sum = left.cumsum(-1)
    over = run_sum > s["sample_u"].double().unsqueeze(1) * run_sum[:, -1:]
    v = torch.arange(left.shape[1], device=dev)
    taken = torch.where(over.any(-1), over.to(torch.uint8).argmax(-1), torch.where(left > 0, v, -1).amax(-1))
    emitted = torch.where(i < last[seq], follows, torch.where(i == last[seq], taken[seq], -1))
    logp = p.gather(1, emitted.clamp_min(0).unsqueeze(1)).squeeze(1).log()
    return {"tokens": emitted.to(torch.int32), "n_emitted": (last + 1).to(torch.int32), "logp": torch.where(emitted >= 0, logp, 0.0).float(),
            "new_len": (s["kv_len"] - count + last + 1).to(torch.int32)}


def _pages_out(s, n_used=None):
    out = {"table": s["table"], "kv_len": s["kv_len"], "refs": s["refs"], "pools": [x for x in s["pools"] if x is not None]}
    if n_used is not None:
        out["n_used"] = n_used
    return out


def _caches(vb, pools):
    """The pools' layers as the framework's caches."""
    k, v, ks, vs = pools
    return [vb.KVCache(k[l], v[l], None if ks is None else ks[l], None if vs is None else vs[l]) for l in range(k.shape[0])]


def _own_pages(s):
    from paper_2509_24257_b200 import binding as vb

    if "handle" not in s:  # what a program keeps beside its pools
        s["handle"] = vb.KVPages(_caches(vb, s["pools"]), s["table"], s["kv_len"], s["refs"])
        s["parking"] = _caches(vb, s["parked"]) if s["n_parked"] else None
    h, kind = s["handle"], s["case"]["kind"]
    s["ints"].copy_(s["ints0"])  # every pass starts from the same tables
    if kind == "step":
        vb.kv_reserve(h, s["grow"])
        vb.kv_free(h, s["final"])
        return _pages_out(s)
    if kind == "fork":
        vb.kv_fork(h, s["src"], s["dst"])
        vb.kv_reserve(h, s["grow"])
        vb.kv_free(h, s["final"])
        return _pages_out(s)
    vb.kv_free(h, s["final"])
    vb.kv_reserve(h, s["grow"])
    vb.kv_copy(s["parking"], h.caches, s["parked_pages"], s["table"][-1, :s["n_parked"]])
    return _pages_out(s, vb.kv_compact(h))


def _plain_pages(s):
    kind, n = s["case"]["kind"], s["n_parked"]
    s["ints"].copy_(s["ints0"])
    if kind == "step":
        _plain_reserve(s, s["grow"].long())
        _plain_free(s, s["final"].long())
        return _pages_out(s)
    if kind == "fork":
        _plain_fork(s)
        _plain_reserve(s, s["grow"].long())
        _plain_free(s, s["final"].long())
        return _pages_out(s)
    _plain_free(s, s["final"].long())
    _plain_reserve(s, s["grow"].long())
    dst = s["table"][-1, :n].long()
    _set(s["pools"], dst, s["parked"], s["parked_pages"].long())
    return _pages_out(s, _plain_compact(s))


def _set(to, dst, source, src):
    """Pages src of the pools `source` into pages dst of the pools `to`, all layers."""
    def bits(x):
        return x.view(torch.uint8) if x.element_size() == 1 else x  # (no indexed stores of 8-bit floats)

    bits(to[0])[:, dst] = bits(source[0])[:, src]
    bits(to[1])[:, dst] = bits(source[1])[:, src]
    if to[2] is not None:
        to[2][:, dst] = source[2][:, src]
        to[3][:, dst] = source[3][:, src]


def _count(s, entries, mask, by):
    """refs[entry] += by for the masked entries."""
    s["refs"].index_add_(0, entries[mask], torch.full_like(entries[mask], by, dtype=torch.int32))


def _plain_free(s, new_len):
    ps, n = s["case"]["page"], s["kv_len"].long()
    new = torch.minimum(new_len, n)
    j = torch.arange(s["table"].shape[1], device=n.device)
    drop = (j >= ((new + ps - 1) // ps).unsqueeze(1)) & (j < ((n + ps - 1) // ps).unsqueeze(1))
    _count(s, s["table"].long(), drop, -1)
    s["kv_len"].copy_(new)


def _plain_fork(s):
    ps, src, dst = s["case"]["page"], s["src"].long(), s["dst"].long()
    n = s["kv_len"].long()[src]
    entries = s["table"][src]
    shared = torch.arange(entries.shape[1], device=n.device) < ((n + ps - 1) // ps).unsqueeze(1)
    s["table"][dst] = torch.where(shared, entries, s["table"][dst])
    _count(s, entries.long(), shared, 1)
    s["kv_len"][dst] = n.to(torch.int32)


def _plain_reserve(s, new_len):
    ps, n, refs = s["case"]["page"], s["kv_len"].long(), s["refs"]
    B, W = s["table"].shape
    grows = (new_len > n) & (new_len <= W * ps)
    have, want = (n + ps - 1) // ps, (new_len + ps - 1) // ps
    last = s["table"].long().gather(1, (have - 1).clamp_min(0).unsqueeze(1)).squeeze(1)
    partly = grows & (n % ps != 0) & (refs[last] > 1)
    same = partly.unsqueeze(0) & partly.unsqueeze(1) & (last.unsqueeze(0) == last.unsqueeze(1))
    b = torch.arange(B, device=n.device)
    keeps = (same.sum(1) == refs[last]) & ~(same & (b.unsqueeze(0) > b.unsqueeze(1))).any(1)  # the last of all its holders
    copies = partly & ~keeps
    need = torch.where(grows, want - have + copies.long(), 0)
    upto = need.cumsum(0)
    free = torch.nonzero(refs == 0).squeeze(1)
    served = grows & (upto <= free.shape[0])
    need, copies = torch.where(served, need, 0), copies & served
    # page `k` of a sequence's need goes to its table at: the copied page first, then the new ones
    k = torch.arange(W + 1, device=n.device)
    take = k < need.unsqueeze(1)
    page = free[((upto - need).unsqueeze(1) + k)[take]]
    to = (have.unsqueeze(1) + k - copies.long().unsqueeze(1))[take]
    s["table"][b.unsqueeze(1).expand(-1, W + 1)[take], to] = page.to(torch.int32)
    refs[page] = 1
    old = last[copies]
    _count(s, old, torch.ones_like(old, dtype=torch.bool), -1)
    fresh = s["table"].long().gather(1, (have - 1).clamp_min(0).unsqueeze(1)).squeeze(1)[copies]
    _set(s["pools"], fresh, s["pools"], old)
    s["kv_len"].copy_(torch.where(served, new_len, n))


def _plain_compact(s):
    ps, n, refs = s["case"]["page"], s["kv_len"].long(), s["refs"]
    used = refs > 0
    n_used = used.sum()
    at = torch.arange(refs.shape[0], device=n.device)
    src, dst = torch.nonzero(used & (at >= n_used)).squeeze(1), torch.nonzero(~used & (at < n_used)).squeeze(1)
    _set(s["pools"], dst, s["pools"], src)
    refs[dst] = refs[src]
    refs[src] = 0
    now = at.clone()
    now[src] = dst
    held = torch.arange(s["table"].shape[1], device=n.device) < ((n + ps - 1) // ps).unsqueeze(1)
    s["table"].copy_(torch.where(held, now[s["table"].long()], s["table"].long()))
    return n_used.to(torch.int32).reshape(1)


# --------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    c = case
    if c["op"] == "w4":
        out = c["rows"] * c["n"] * (2.0 if c["out"] == "bf16" else 4.0) * (2 if c["add"] else 1)
        return {"bytes": c["n"] * c["k"] / 2.0 + 2.0 * c["n"] * c["k"] / c["group"] + 2.0 * c["rows"] * c["k"] + out,
                "flops": 2.0 * c["rows"] * c["n"] * c["k"]}
    if c["op"] == "drafts":
        rows, e = _rows(c), 2.0 if c["dtype"] == "bf16" else 4.0
        read = sum(rows) + (sum(rows) - len(rows) if c["draft"] else 0)
        return {"bytes": read * e * c["vocab"] + 16.0 * sum(rows) + 20.0 * len(rows), "flops": 4.0 * read * c["vocab"]}
    p = _plan(c)
    ps, moved = c["page"], 0
    table, refs = _first_pages(c, p, 1)
    n = list(p["len"])
    entries = sum(_ceil(x, ps) for x in n)
    if c["kind"] == "swap":
        # moved: the pages that come back, and those in use behind the new end
        left = [x for x, f in zip(n, p["final"]) if f]
        used = sum(_ceil(x, ps) for x in left) + _ceil(p["back"], ps)
        moved = _ceil(p["back"], ps) + int(used * (1 - used / p["n_pages"]))
    elif c["kind"] == "step":
        moved = sum(1 for b, x in enumerate(n) if x % ps and p["parent"][b] >= 0)
    else:
        moved = sum(1 for b in p["src"] if n[b] % ps)
        entries += 2 * sum(_ceil(n[b], ps) for b in p["src"])
    return {"bytes": 2.0 * moved * c["layers"] * _page_bytes(c) + 4.0 * (entries + 2 * len(refs) + 4 * len(table)), "flops": 0.0}


# --------------------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None  # copies and whole numbers
    s = prepare(case, seed)
    if c["op"] == "w4":
        y = torch.zeros(c["rows"], c["n"], dtype=torch.float64, device=s["x"].device) if s["y"] is None else s["y"].double()
        step = max(1, (1 << 26) // c["k"])
        for n0 in range(0, c["n"], step):
            packed = s["codes"][n0:n0 + step].to(torch.int32)
            w = torch.empty(packed.shape[0], c["k"], dtype=torch.float64, device=packed.device)
            w[:, 0::2], w[:, 1::2] = packed % 16 - 8, packed // 16 - 8
            w *= s["scales"][:, n0:n0 + step].double().repeat_interleave(c["group"], 0).T
            y[:, n0:n0 + step] += s["x"].double() @ w.T
        return y
    rows, cu, V = _rows(c), s["cu_rows"].tolist(), c["vocab"]
    temps, toks, ua, us = s["temperature"].tolist(), s["tokens"].tolist(), s["accept_u"].tolist(), s["sample_u"].tolist()
    logp = torch.zeros(cu[-1], dtype=torch.float64, device=s["target"].device)

    def log_softmax(row, t):
        x = row.double()
        if t == 0:
            y = torch.full_like(x, -math.inf)
            y[int(torch.argmax((x == x.max()).int()))] = 0.0
            return y
        return x / t - torch.logsumexp(x / t, 0)

    for b in range(c["batch"]):
        for i in range(rows[b]):
            r = cu[b] + i
            lp = log_softmax(s["target"][r], temps[b])
            res = lp.exp()
            if i < rows[b] - 1:
                x = toks[r + 1]
                if s["draft"] is not None and temps[b] > 0:
                    q = log_softmax(s["draft"][r], temps[b]).exp()
                else:
                    q = torch.zeros_like(res)
                    q[x] = 1.0
                good = float(lp[x]) == 0.0 if temps[b] == 0 else ua[r + 1] * float(q[x]) < math.exp(float(lp[x]))
                if good:
                    logp[r] = lp[x]
                    continue
                if temps[b] > 0:
                    d = torch.clamp(res - q, min=0)
                    res = d if float(d.sum()) > 0 else res
            total = torch.cumsum(res, 0)
            over = torch.nonzero(total > us[b] * total[-1])
            v = int(over[0]) if over.numel() else int(torch.nonzero(res > 0)[-1])
            logp[r] = lp[v]
            break
    return {"tokens": None, "n_emitted": None, "logp": logp, "new_len": None}
