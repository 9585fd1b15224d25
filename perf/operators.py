"""The calls the paged key/value cache is measured on: appending rows to it, the
attention that reads it, and that attention for a batch with a common prefix.

Head layouts are those of the presets in ``paper_2509_01190_amd/workloads.py``
(12 heads of 64, 32 of 64, 32 of 128 on 8, 4 of 32) or generic. Where a case is
ragged, its lengths are spread evenly between the shortest and the longest by
its own numbers, so that they do not depend on the seed; pages are dealt to the
sequences in a shuffled order, as a pool that has served others hands them out.
Queries and keys share one direction per head which a few rows carry, as a
trained model's attention singles out some positions.
"""
import math

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # one new token for each of a few small sequences: launches and latency
        {"name": "append one token", "op": "append", "dtype": "bf16", "heads": 12, "kv": 12, "hd": 64, "page": 16,
         "batch": 8, "new": 1, "new_min": 1, "cached": 200, "cached_min": 5, "theta": 10000.0, "q": True},
        # the rows of a prefill of four prompts
        {"name": "append prompts", "op": "append", "dtype": "bf16", "heads": 32, "kv": 8, "hd": 128, "page": 64,
         "batch": 4, "new": 4096, "new_min": 4096, "cached": 0, "cached_min": 0, "theta": 500000.0, "q": True},
        # fp32 rows of a ragged batch, keys and values alone
        {"name": "append ragged f32", "op": "append", "dtype": "f32", "heads": 12, "kv": 12, "hd": 64, "page": 32,
         "batch": 13, "new": 701, "new_min": 1, "cached": 1000, "cached_min": 0, "theta": 10000.0, "q": False},
        # one token of a few short sequences, as a pruned prefill leaves them
        {"name": "decode short", "op": "attend", "dtype": "bf16", "heads": 12, "kv": 12, "hd": 64, "page": 16,
         "batch": 4, "new": 1, "new_min": 1, "cached": 299, "cached_min": 9, "causal": True},
        # one token of a served batch of ragged lengths, grouped heads
        {"name": "decode batch", "op": "attend", "dtype": "bf16", "heads": 32, "kv": 8, "hd": 128, "page": 64,
         "batch": 64, "new": 1, "new_min": 1, "cached": 4095, "cached_min": 100, "causal": True},
        # one token of a few very long sequences
        {"name": "decode long", "op": "attend", "dtype": "bf16", "heads": 32, "kv": 8, "hd": 128, "page": 128,
         "batch": 4, "new": 1, "new_min": 1, "cached": 65535, "cached_min": 50001, "causal": True},
        # fp32 decoding
        {"name": "decode f32", "op": "attend", "dtype": "f32", "heads": 12, "kv": 12, "hd": 64, "page": 32,
         "batch": 16, "new": 1, "new_min": 1, "cached": 1023, "cached_min": 33, "causal": True},
        # the next piece of long prompts, most of whose rows are cached
        {"name": "prompt pieces", "op": "attend", "dtype": "bf16", "heads": 32, "kv": 8, "hd": 128, "page": 64,
         "batch": 4, "new": 1024, "new_min": 1024, "cached": 7000, "cached_min": 3001, "causal": True},
        # a batch in which a few sequences bring prompts and the others one token
        {"name": "mixed batch", "op": "attend", "dtype": "bf16", "heads": 32, "kv": 32, "hd": 64, "page": 32,
         "batch": 24, "new": 509, "new_min": 1, "cached": 2047, "cached_min": 17, "causal": True, "few_long": True},
        # one token of a batch behind a long common prompt
        {"name": "prefix decode", "op": "prefix", "dtype": "bf16", "heads": 32, "kv": 8, "hd": 128, "page": 64,
         "batch": 64, "new": 1, "new_min": 1, "cached": 511, "cached_min": 3, "causal": True, "prefix": 8192},
        # the same, small
        {"name": "prefix decode short", "op": "prefix", "dtype": "bf16", "heads": 12, "kv": 12, "hd": 64, "page": 16,
         "batch": 8, "new": 1, "new_min": 1, "cached": 40, "cached_min": 0, "causal": True, "prefix": 501},
        # questions on one common document
        {"name": "prefix pieces", "op": "prefix", "dtype": "bf16", "heads": 32, "kv": 32, "hd": 64, "page": 64,
         "batch": 16, "new": 97, "new_min": 20, "cached": 0, "cached_min": 0, "causal": True, "prefix": 4097},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "prefix", "prefix"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, kv, hd = rng.choice([(12, 12, 64), (32, 32, 64), (32, 8, 128), (32, 8, 128), (32, 32, 128), (16, 2, 64),
                                (8, 1, 128), (24, 8, 64), (20, 4, 128), (4, 4, 32), (8, 2, 16)])
    page = rng.choice([16, 32, 64, 128, 256])
    width = kv * hd * (2 if dtype == "bf16" else 4)  # bytes of a row's keys
    case = {"op": op, "dtype": dtype, "heads": heads, "kv": kv, "hd": hd, "page": page}
    if op == "append":
        new = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
        batch = max(1, min(_log(rng, 1, 256), 16384 // new))
        cached = _log(rng, 1, 2048)
        case.update(batch=batch, new=new, new_min=new if rng.random() < 0.5 else 1, cached=cached,
                    cached_min=rng.randint(0, cached), theta=rng.choice([10000.0, 500000.0]), q=rng.random() < 0.7)
        return case
    few = dtype == "f32" or hd < 64  # the vector types' rates: less work
    pieces = rng.random() < 0.35
    new = _log(rng, 2, 256 if few else 1024) if pieces else 1
    cached = _log(rng, 1, 4000 if few else 8000 if pieces else 40000)
    batch = _log(rng, 1, 64)
    rows = 100000 if few else 260000
    batch = max(1, min(batch, int(rows * 2048 // (max(cached, 256) * width)), 4096 // new))
    case.update(batch=batch, new=new, new_min=rng.randint(1, new), cached=cached, cached_min=rng.randint(0, cached),
                causal=rng.random() < 0.8)
    if op == "prefix":
        case["cached"] = min(cached, 1000)
        case["cached_min"] = min(case["cached_min"], case["cached"])
        case["prefix"] = _log(rng, 20, 4000 if few else 20000)
    return case


def _lengths(case):
    """(new rows, cached rows with the new ones) of every sequence."""
    at = [math.modf((b + 1) * 0.6180339887498949)[0] for b in range(case["batch"])]
    cached = [case["cached_min"] + int(round((case["cached"] - case["cached_min"]) * a)) for a in at]
    new = [case["new_min"] + int(round((case["new"] - case["new_min"]) * math.modf(7 * a)[0])) for a in at]
    if case.get("few_long"):  # every eighth brings a prompt, the others one row
        new = [case["new"] if b % 8 == 3 else 1 for b in range(case["batch"])]
    return new, [n + c for n, c in zip(new, cached)]


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dt, H, kv, hd, ps, B = _type(case), case["heads"], case["kv"], case["hd"], case["page"], case["batch"]
    new, lens = _lengths(case)
    T, kvd = sum(new), kv * hd

    def normal(*shape):
        return torch.randn(*shape, device=DEV, dtype=dt, generator=g)

    prefix = case.get("prefix", 0)
    need = [-(-n // ps) for n in lens]
    most, first = max(max(need), 1), -(-prefix // ps)
    pages = first + sum(need) + 3
    order = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
    # a table row's unused entries name some page of the pool, as a reused table's do
    table = order[torch.randint(0, pages, (B, most), device=DEV, generator=g)]
    at = first
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    state = {"case": dict(case), "table": table, "cu_host": cu, "max_len": max(lens),
             "cu": torch.tensor(cu, dtype=torch.int32, device=DEV),
             "len": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    if case["op"] == "append":
        # the projection's rows q | k | v, not rotated yet; positions with the gaps that pruning leaves
        state["qkv"] = normal(T, (H + 2 * kv) * hd)
        step = torch.randint(1, 4, (T,), device=DEV, generator=g)
        state["pos"] = torch.cumsum(step, 0).remainder(100000).to(torch.int32)
        state["pool"] = torch.zeros(pages, ps, 2 * kvd, dtype=dt, device=DEV)
        state["pool"].normal_(generator=g)
        return state
    direction = torch.randn(kv, hd, device=DEV, generator=g)
    direction *= math.sqrt(3.0 * math.sqrt(hd)) / direction.norm(dim=1, keepdim=True)
    pool = normal(pages, ps, 2 * kvd)
    marked = (torch.rand(pages, ps, 1, 1, device=DEV, generator=g) < 0.02).to(dt)
    pool.view(pages, ps, 2, kv, hd)[:, :, 0] += marked * direction.to(dt)
    state["pool"] = pool
    q = normal(T, H * hd)
    q.view(T, kv, H // kv, hd).add_(direction.to(dt)[:, None])
    state["q"] = q
    if prefix:
        state["prefix_pages"], state["prefix"] = order[:first].contiguous(), prefix
    return state


# ---------------------------------------------------------------------------- the framework's calls
def _handles(state):
    """What a serving program makes once and keeps beside its tensors."""
    from paper_2509_01190_amd import zsa
    if "handles" not in state:
        state["handles"] = (zsa.PagedKV(state["pool"], state["table"], state["case"]["kv"]),
                            zsa.Seqs.wrap(state["cu_host"], state["cu"]))
    return zsa, *state["handles"]


def _own(state):
    case = state["case"]
    zsa, kv, seqs = _handles(state)
    H = case["heads"]
    if case["op"] == "append":
        d, kvd = H * case["hd"], case["kv"] * case["hd"]
        qkv = state["qkv"]
        q = zsa.paged_append(kv, qkv[:, d:d + kvd], qkv[:, d + kvd:], seqs, state["len"], pos=state["pos"],
                             rope_theta=case["theta"], q=qkv[:, :d] if case["q"] else None, n_heads=H)
        return {"q": q, "pool": state["pool"]} if case["q"] else {"pool": state["pool"]}
    if case["op"] == "attend":
        out, lse = zsa.paged_attention(state["q"], kv, H, seqs, state["len"], max_kv_len=state["max_len"],
                                       causal=case["causal"], want_lse=True)
    else:
        out, lse = zsa.prefix_attention(state["q"], kv, H, seqs, state["len"], state["prefix_pages"], state["prefix"],
                                        max_kv_len=state["max_len"], causal=case["causal"], want_lse=True)
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------- the plain form
def _sequence_of(state):
    """(sequence, row in it) of every new row."""
    cu = state["cu"].long()
    t = torch.arange(state["cu_host"][-1], device=DEV)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    return b, t - cu[b]


def _rotate(x, pos, theta):
    """x [T, heads, hd], pairs (i, i + hd/2) by pos theta^(-2i/hd)."""
    half = x.shape[2] // 2
    i = torch.arange(half, device=DEV, dtype=torch.float64)
    angle = pos.double()[:, None] * torch.pow(torch.tensor(theta, dtype=torch.float64, device=DEV), -i / half)
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[..., :half].float(), x[..., half:].float()
    return torch.cat([a * c - b * s, b * c + a * s], dim=2)


def _append(state):
    case = state["case"]
    H, kv, hd, ps = case["heads"], case["kv"], case["hd"], case["page"]
    qkv, pool, dt = state["qkv"], state["pool"], _type(case)
    T, d, kvd = qkv.shape[0], H * hd, kv * hd
    b, r = _sequence_of(state)
    new = (state["cu"][1:] - state["cu"][:-1]).long()
    row = (state["len"].long() - new)[b] + r
    at = state["table"].long()[b, row // ps] * ps + row % ps
    k = _rotate(qkv[:, d:d + kvd].view(T, kv, hd), state["pos"], case["theta"]).reshape(T, kvd).to(dt)
    pool.view(-1, 2 * kvd)[at] = torch.cat([k, qkv[:, d + kvd:]], dim=1)
    if not case["q"]:
        return {"pool": pool}
    return {"q": _rotate(qkv[:, :d].view(T, H, hd), state["pos"], case["theta"]).reshape(T, d).to(dt), "pool": pool}


def _part(q, k, v, seen):
    """Maximum, sum and sum of values of q [.., n, hd] over k, v [.., L, hd]; seen: which keys count, or None."""
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(q.shape[-1])
    if seen is not None:
        s = s.masked_fill(~seen, -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    return m, p.sum(dim=-1, keepdim=True), torch.matmul(p, v)


def _attend(state):
    case = state["case"]
    H, kv, hd, ps, dt = case["heads"], case["kv"], case["hd"], case["page"], _type(case)
    G, B, T = H // kv, case["batch"], state["q"].shape[0]
    cu, lens, pool = state["cu"].long(), state["len"].long(), state["pool"]
    n = max(1, max(y - x for x, y in zip(state["cu_host"], state["cu_host"][1:])))
    # the sequences' own rows, padded to the longest
    pages = -(-state["max_len"] // ps)
    rows = pool[state["table"][:, :pages].long()].view(B, pages * ps, 2, kv, hd)[:, :state["max_len"]].float()
    k, v = rows[:, :, 0].permute(0, 2, 1, 3).contiguous(), rows[:, :, 1].permute(0, 2, 1, 3).contiguous()
    t = torch.minimum(cu[:-1, None] + torch.arange(n, device=DEV), torch.tensor(T - 1, device=DEV))
    q = state["q"][t].view(B, n, kv, G, hd).permute(0, 2, 3, 1, 4).float().reshape(B, kv, G * n, hd)
    j, r = torch.arange(k.shape[2], device=DEV), torch.arange(n, device=DEV)
    most = lens[:, None].expand(B, n)
    if case["causal"]:
        most = most - (cu[1:] - cu[:-1])[:, None] + r[None] + 1
    seen = (j[None, None] < most[:, :, None])[:, None, None].expand(B, 1, G, n, j.numel()).reshape(B, 1, G * n, j.numel())
    m, l, o = _part(q, k, v, seen)
    # back to the new rows: [T, kv, G]
    b, r = _sequence_of(state)
    m, l, o = (x.view(B, kv, G, n, -1)[b, :, :, r] for x in (m, l, o))
    if case["op"] == "prefix":
        rows = pool[state["prefix_pages"].long()].view(-1, 2, kv, hd)[:state["prefix"]].float()
        k, v = rows[:, 0].permute(1, 0, 2).contiguous(), rows[:, 1].permute(1, 0, 2).contiguous()
        q = state["q"].view(T, kv, G, hd).permute(1, 0, 2, 3).float().reshape(kv, T * G, hd)
        m2, l2, o2 = (x.view(kv, T, G, -1).permute(1, 0, 2, 3) for x in _part(q, k, v, None))
        both = torch.maximum(m, m2)
        a, a2 = torch.exp(m - both), torch.exp(m2 - both)
        m, l, o = both, l * a + l2 * a2, o * a + o2 * a2
    out = torch.where(l > 0, o / l, torch.zeros_like(o))
    lse = (m + torch.log(l)).view(T, H).t().contiguous()
    return {"out": out.reshape(T, H * hd).to(dt), "lse": lse}


def run(state):
    if own:
        return _own(state)
    return _append(state) if state["case"]["op"] == "append" else _attend(state)


def work(case):
    new, lens = _lengths(case)
    e = 2 if case["dtype"] == "bf16" else 4
    H, kv, hd, T = case["heads"], case["kv"], case["hd"], sum(new)
    if case["op"] == "append":
        heads = (H if case["q"] else 0) + 2 * kv
        return {"bytes": 2 * T * heads * hd * e + 4 * T, "flops": 3 * T * (heads - kv) * hd}
    P = case.get("prefix", 0)
    pairs = P * T
    for n, m in zip(new, lens):
        pairs += n * m - (n * (n - 1) // 2 if case["causal"] else 0)
    rows = P + sum(lens)
    return {"bytes": rows * 2 * kv * hd * e + 2 * T * H * hd * e + 4 * T * H, "flops": 4 * hd * H * pairs}


# ---------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    H, kv, hd, ps = case["heads"], case["kv"], case["hd"], case["page"]
    new, lens = _lengths(case)
    flat = state["pool"].view(-1, 2 * kv * hd)
    table = state["table"].cpu()
    cu = state["cu_host"]

    def places(pages, n):
        r = torch.arange(n)
        return (pages[r // ps].long() * ps + r % ps).to(DEV)

    if case["op"] == "append":
        w = torch.tensor([case["theta"] ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=torch.float64, device=DEV)

        def turned(x, heads, pos):
            z = x.double().view(x.shape[0], heads, 2, hd // 2)
            z = torch.complex(z[:, :, 0], z[:, :, 1]) * torch.polar(
                torch.ones((), dtype=torch.float64, device=DEV), pos.double()[:, None] * w)[:, None]
            return torch.stack([z.real, z.imag], dim=2).reshape(x.shape[0], heads * hd)

        d, kvd = H * hd, kv * hd
        pool = flat.double()
        for b, n in enumerate(lens):
            at = places(table[b], n)[n - new[b]:]
            x = state["qkv"][cu[b]:cu[b + 1]]
            pool[at, :kvd] = turned(x[:, d:d + kvd], kv, state["pos"][cu[b]:cu[b + 1]])
            pool[at, kvd:] = x[:, d + kvd:].double()
        pool = pool.view(state["pool"].shape)
        return {"q": turned(state["qkv"][:, :d], H, state["pos"]), "pool": pool} if case["q"] else {"pool": pool}
    T, G = sum(new), H // kv
    out = torch.zeros(T, H, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((H, T), -math.inf, dtype=torch.float64, device=DEV)
    before = state["prefix"] if "prefix" in state else 0
    head = places(state["prefix_pages"].cpu(), before) if before else torch.zeros(0, dtype=torch.long, device=DEV)
    for b, n in enumerate(lens):
        rows = flat[torch.cat([head, places(table[b], n)])].view(-1, 2, kv, hd)
        q = state["q"][cu[b]:cu[b + 1]].view(new[b], H, hd)
        i = torch.arange(new[b], device=DEV)
        hidden = torch.arange(rows.shape[0], device=DEV)[None] > (before + n - new[b] + i)[:, None]
        for h in range(H):
            s = q[:, h].double() @ rows[:, 0, h // G].double().T * hd ** -0.5
            if case["causal"]:
                s[hidden] = -math.inf
            out[cu[b]:cu[b + 1], h] = torch.softmax(s, dim=1) @ rows[:, 1, h // G].double()
            lse[h, cu[b]:cu[b + 1]] = torch.logsumexp(s, dim=1)
    return {"out": out.view(T, H * hd), "lse": lse}
