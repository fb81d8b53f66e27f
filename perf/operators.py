"""Cases of the paged key-value cache: append to it, attention of new tokens over it, eviction from it.

Three kinds of case, each one call of paper_2603_05454_b200.PagedKVCache:

  attention   one new token (or a short block) per sequence over the cached keys and values; with `weights` also the attention
              weight that every cached key has gathered
  append      the keys and values of new tokens written behind the cached ones; weight and position of the new slots started
  evict       per KV head the `budget` slots with the largest gathered weight kept (the first `sink` and last `recent`
              positions in any case), kept slots behind the budget moved into the freed ones

Head layouts are those of the benchmark's two large shapes (32/32 and 28/4 heads of 128) and of the small test models.  The
lengths of a batch follow from the case alone: the first sequence has `len` slots, the others down to `spread` fewer (half of them).

The plain form of each operator is elementary torch operations in 32 bits.
"""
import math

import torch

own = False          # the tools set it: run() makes the framework's calls

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# query heads, KV heads, head_dim
HEADS = {"llada": (32, 32, 128), "dream": (28, 4, 128), "small": (4, 2, 128), "small64": (8, 4, 64), "tiny": (4, 4, 64)}


def listed():
    return [
        # one sequence in the last steps of a short decode: latency is everything
        dict(name="token_short", op="attention", heads="llada", dtype="bf16", batch=1, len=301, rows=1, ragged=0, page=16, weights=0),
        # a small model's batch, blocks of up to five tokens, weights gathered for the eviction
        dict(name="block_small", op="attention", heads="small64", dtype="bf16", batch=3, len=715, rows=5, ragged=1, page=16, weights=1),
        # a tiny fp32 model, a batch of short sequences
        dict(name="token_fp32", op="attention", heads="tiny", dtype="fp32", batch=5, len=2003, rows=1, ragged=0, page=32, weights=0),
        # a few sequences with long documents in front of them, grouped-query heads
        dict(name="token_dream_long", op="attention", heads="dream", dtype="bf16", batch=6, len=30011, rows=1, ragged=0, page=64, weights=0),
        # a serving batch of sixteen at two thousand positions, a key head per query head: half a gigabyte of keys and values
        dict(name="token_llada_batch", op="attention", heads="llada", dtype="bf16", batch=16, len=2047, rows=1, ragged=0, page=64, weights=0),
        # a step of a batch whose cache is about to be thinned
        dict(name="token_llada_weights", op="attention", heads="llada", dtype="bf16", batch=8, len=4001, rows=1, ragged=0, page=64, weights=1),
        # one new token for each of sixteen sequences
        dict(name="append_token", op="append", heads="llada", dtype="bf16", batch=16, len=1500, rows=1, ragged=0, page=16),
        # four prompts of up to 1023 tokens into fresh pages
        dict(name="append_prompts", op="append", heads="llada", dtype="bf16", batch=4, len=0, rows=1023, ragged=1, page=64),
        # every sequence a few tokens over its budget
        dict(name="evict_step", op="evict", heads="llada", dtype="bf16", batch=16, len=1032, spread=8, budget=1024, sink=4, recent=64, page=64),
        # four prompts thinned to a quarter, grouped-query heads
        dict(name="evict_dream", op="evict", heads="dream", dtype="bf16", batch=4, len=4093, budget=1024, sink=4, recent=128, page=64),
        # one long document: four KV heads of 65 thousand slots each
        dict(name="evict_long", op="evict", heads="dream", dtype="bf16", batch=1, len=65521, budget=8192, sink=16, recent=1024, page=64),
        # the serving batch thinned from two thousand slots to 512
        dict(name="evict_llada", op="evict", heads="llada", dtype="bf16", batch=16, len=2047, budget=512, sink=4, recent=64, page=64),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "append", "evict", "evict"])
    heads = rng.choice(["llada", "dream", "dream", "small", "small64", "tiny"])
    dtype = "fp32" if heads == "tiny" or rng.random() < 0.15 else "bf16"
    hq, hkv, dh = HEADS[heads]
    row = hkv * dh * (2 if dtype == "bf16" else 4)          # bytes of a key row
    batch = _logint(rng, 1, 32)
    page = rng.choice([16, 32, 48, 64, 128])
    case = dict(op=op, heads=heads, dtype=dtype, batch=batch, page=page)
    if op == "append":
        rows = 1 if rng.random() < 0.4 else _logint(rng, 2, max(2, min(2048, 32_000_000 // (row * batch))))
        case.update(len=rng.choice([0, _logint(rng, 1, 2000)]), rows=rows, ragged=int(rows > 1 and rng.random() < 0.7))
        return case
    case["len"] = _logint(rng, 1 if op == "attention" else 40, max(64, min(60000, 250_000_000 // (row * batch))))
    if op == "attention":
        rows = 1 if rng.random() < 0.6 else rng.randint(2, 8)
        case.update(rows=rows, ragged=int(rows > 1 and rng.random() < 0.5), weights=int(rng.random() < 0.4))
    else:
        budget = max(8, int(case["len"] * rng.uniform(0.1, 1.1)))
        case.update(budget=budget, sink=rng.randint(0, budget // 8), recent=rng.randint(0, budget // 4))
    return case


def _lens(case):
    n = case["len"]
    spread = case.get("spread", n // 2)
    return [n - (b * (37 * n // 100 + 1)) % (spread + 1) for b in range(case["batch"])]


def _rows(case):
    r = case["rows"]
    return [r - (b * (r // 3 + 1)) % r if case["ragged"] else r for b in range(case["batch"])]


def _pages(case):
    """Pages of a sequence: enough for the longest, and one more."""
    return -(-(case["len"] + case.get("rows", 0)) // case["page"]) + 1


def prepare(case, seed):
    hq, hkv, dh = HEADS[case["heads"]]
    dt, batch, page = TYPES[case["dtype"]], case["batch"], case["page"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 2654435761 % (1 << 62) + 7)
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    per_seq = _pages(case)
    n_pages = batch * per_seq + 3
    # pages in the order in which a server's free list hands them out after a while: none in particular
    table = torch.randperm(n_pages, generator=g, device=DEV)[: batch * per_seq].to(torch.int32).view(batch, per_seq).contiguous()
    st = dict(case=case, table=table, lens=ints(_lens(case)))
    for name in ("k", "v"):
        st[name] = torch.empty(n_pages, page, hkv, dh, dtype=dt, device=DEV)
        for at in range(0, n_pages, 1024):
            st[name][at:at + 1024] = normal(min(1024, n_pages - at), page, hkv, dh).to(dt)
    cap = per_seq * page
    if case["op"] in ("attention", "append"):
        rows = _rows(case)
        n = sum(rows)
        st["row_off"] = ints([sum(rows[:b]) for b in range(batch + 1)]) if case["ragged"] else None
        st["n_rows"] = n
    if case["op"] == "attention":
        # queries of twice unit size: a head's weight gathers on a few dozen keys; a slice of the fused projection's result
        st["qkv"] = (2.0 * normal(n, (hq + 2 * hkv) * dh)).to(dt)
        st["q"] = st["qkv"][:, : hq * dh]
        st["out"] = torch.zeros(n, hq * dh, dtype=dt, device=DEV)
        st["lse"] = torch.zeros(n, hq, device=DEV)
        if case["weights"]:
            st["weights_in"] = torch.rand(batch, hkv, cap, generator=g, device=DEV) ** 4
            st["weights_out"] = torch.zeros(batch, hkv, cap, device=DEV)
    elif case["op"] == "append":
        st["kv_new"] = normal(n, 2 * hkv * dh).to(dt)          # the key and value part of the fused projection's result
        st["seen"] = st["lens"] + 5                            # five positions were evicted earlier
        st["lens_out"], st["seen_out"] = torch.zeros_like(st["lens"]), torch.zeros_like(st["lens"])
        st["weights"] = torch.ones(batch, hkv, cap, device=DEV)
        st["pos"] = torch.full((batch, hkv, cap), -1, dtype=torch.int32, device=DEV)
    else:
        # weights with a heavy tail; one slot in eight was never attended to (exact ties).  Slots hold their positions out of order,
        # as an earlier eviction leaves them.
        w = torch.exp(2.0 * normal(batch, hkv, cap)) * 1e-3
        st["weights"] = torch.where(torch.rand(batch, hkv, cap, generator=g, device=DEV) < 0.125, torch.zeros_like(w), w)
        lens = st["lens"].view(batch, 1, 1)
        key = torch.rand(batch, hkv, cap, generator=g, device=DEV).masked_fill_(torch.arange(cap, device=DEV) >= lens, 2.0)
        st["pos"] = torch.argsort(key, dim=-1).to(torch.int32)
        st["seen"] = st["lens"].clone()
        st["weights_out"] = torch.zeros(batch, hkv, cap, device=DEV)
        st["pos_out"] = torch.full((batch, hkv, cap), -1, dtype=torch.int32, device=DEV)
        st["lens_out"] = torch.zeros_like(st["lens"])
    if own:
        from paper_2603_05454_b200 import PagedKVCache
        st["cache"] = PagedKVCache(st["k"], st["v"], st["table"], n_heads=hq, max_rows=case.get("rows", 1), weights=bool(case.get("weights")))
    return st


def run(st):
    if own:
        return _run_own(st)
    return {"attention": _plain_attention, "append": _plain_append, "evict": _plain_evict}[st["case"]["op"]](st)


def _run_own(st):
    c, case = st["cache"], st["case"]
    if case["op"] == "attention":
        if not case["weights"]:
            c.attention(st["q"], st["lens"], st["out"], row_off=st["row_off"], lse=st["lse"])
            return st["out"], st["lse"]
        c.attention(st["q"], st["lens"], st["out"], row_off=st["row_off"], lse=st["lse"], weights_in=st["weights_in"], weights_out=st["weights_out"])
        return st["out"], st["lse"], st["weights_out"]
    if case["op"] == "append":
        half = st["kv_new"].shape[1] // 2
        c.append(st["kv_new"][:, :half], st["kv_new"][:, half:], st["lens"], st["lens_out"], row_off=st["row_off"], weights=st["weights"],
                 pos=st["pos"], seen=st["seen"], seen_out=st["seen_out"])
        return st["k"], st["v"], st["weights"], st["pos"], st["lens_out"], st["seen_out"]
    c.evict(st["weights"], st["lens"], case["budget"], st["weights_out"], st["lens_out"], n_sink=case["sink"], n_recent=case["recent"],
            pos=st["pos"], pos_out=st["pos_out"], seen=st["seen"])
    return st["k"], st["v"], st["weights_out"], st["pos_out"], st["lens_out"]


def _slots(st, n):
    """Row of the flattened pool that holds slot j of every sequence, j < n: [batch, n]."""
    page = st["case"]["page"]
    j = torch.arange(n, device=DEV)
    return st["table"][:, j // page].long() * page + j % page


def _row_places(st):
    """Sequence and index within the sequence of every packed row."""
    case = st["case"]
    r = torch.arange(st["n_rows"], device=DEV)
    if st["row_off"] is None:
        return r // case["rows"], r % case["rows"]
    seq = torch.searchsorted(st["row_off"][1:].long(), r, right=True)
    return seq, r - st["row_off"].long()[seq]


def _plain_attention(st):
    case = st["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    batch, n, group = case["batch"], case["len"], hq // hkv
    slots = _slots(st, n)
    k = st["k"].view(-1, hkv, dh)[slots].float()             # [batch, n, hkv, dh]
    v = st["v"].view(-1, hkv, dh)[slots].float()
    seq, idx = _row_places(st)
    q = torch.zeros(batch, case["rows"], hkv, group, dh, device=DEV)
    q[seq, idx] = st["q"].float().reshape(-1, hkv, group, dh)
    q = q.permute(0, 2, 1, 3, 4).reshape(batch, hkv, case["rows"] * group, dh)
    s = q @ k.permute(0, 2, 3, 1) * (1.0 / math.sqrt(dh))    # [batch, hkv, rows * group, n]
    live = (torch.arange(n, device=DEV) < st["lens"].view(-1, 1))[:, None, None, :]
    s = s.masked_fill(~live, float("-inf"))
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m)
    total = e.sum(-1, keepdim=True)
    p = e / total
    o = p @ v.permute(0, 2, 1, 3)
    back = lambda t: t.view(batch, hkv, case["rows"], group, -1).permute(0, 2, 1, 3, 4)[seq, idx].reshape(st["n_rows"], -1)  # noqa: E731
    st["out"].copy_(back(o))
    st["lse"].copy_(back(m + torch.log(total)))
    if not case["weights"]:
        return st["out"], st["lse"]
    real = torch.zeros(batch, case["rows"], dtype=torch.bool, device=DEV)
    real[seq, idx] = True
    p = p.view(batch, hkv, case["rows"], group, n) * real.view(batch, 1, -1, 1, 1)
    st["weights_out"][:, :, :n] = torch.where(live[:, 0], st["weights_in"][:, :, :n] + p.sum((2, 3)), st["weights_out"][:, :, :n])
    return st["out"], st["lse"], st["weights_out"]


def _plain_append(st):
    case = st["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    seq, idx = _row_places(st)
    slot = st["lens"].long()[seq] + idx
    at = st["table"].long()[seq, slot // case["page"]] * case["page"] + slot % case["page"]
    new = st["kv_new"].view(-1, 2, hkv, dh)
    st["k"].view(-1, hkv, dh)[at] = new[:, 0]
    st["v"].view(-1, hkv, dh)[at] = new[:, 1]
    st["weights"][seq, :, slot] = 0.0
    st["pos"][seq, :, slot] = (st["seen"][seq] + idx.to(torch.int32)).view(-1, 1).expand(-1, hkv)
    n = torch.zeros_like(st["lens"]).index_add_(0, seq, torch.ones_like(seq, dtype=torch.int32))
    st["lens_out"].copy_(st["lens"] + n)
    st["seen_out"].copy_(st["seen"] + n)
    return st["k"], st["v"], st["weights"], st["pos"], st["lens_out"], st["seen_out"]


def _plain_evict(st):
    case = st["case"]
    hq, hkv, dh = HEADS[case["heads"]]
    batch, n, budget = case["batch"], case["len"], case["budget"]
    w, pos = st["weights"][:, :, :n], st["pos"][:, :, :n].long()
    lens, seen = st["lens"].view(-1, 1, 1).long(), st["seen"].view(-1, 1, 1).long()
    j = torch.arange(n, device=DEV).expand(batch, hkv, n)
    live = j < lens
    first = (pos < case["sink"]) | (pos >= seen - case["recent"])
    # an order of the slots: unused ones last, protected ones first, then by falling weight, then by position
    order = torch.argsort(pos, dim=-1, stable=True)
    key = torch.where(live, torch.where(first, torch.full_like(w, float("inf")), w), torch.full_like(w, float("-inf")))
    order = order.gather(-1, torch.argsort(key.gather(-1, order), dim=-1, descending=True, stable=True))
    keep = torch.zeros_like(live).scatter_(-1, order, (torch.arange(n, device=DEV) < budget).expand(batch, hkv, n)) & live
    hole = live & ~keep & (j < budget)
    mover = keep & (j >= budget)
    # the i-th mover goes to the i-th hole
    src = torch.argsort((~mover).to(torch.int8), dim=-1, stable=True)
    rank = hole.long().cumsum(-1) - 1
    take = torch.where(hole, src.gather(-1, rank.clamp(min=0)), j)
    b, h, s = hole.nonzero(as_tuple=True)
    t = take[b, h, s]
    page, table = case["page"], st["table"].long()
    to, at = table[b, s // page] * page + s % page, table[b, t // page] * page + t % page
    for pool in (st["k"], st["v"]):
        flat = pool.view(-1, hkv, dh)
        flat[to, h] = flat[at, h]
    used = (j < lens.clamp(max=budget))
    st["weights_out"][:, :, :n] = torch.where(used, w.gather(-1, take), st["weights_out"][:, :, :n])
    st["pos_out"][:, :, :n] = torch.where(used, pos.gather(-1, take).to(torch.int32), st["pos_out"][:, :, :n])
    st["lens_out"].copy_(st["lens"].clamp(max=budget))
    return st["k"], st["v"], st["weights_out"], st["pos_out"], st["lens_out"]


def exact(case, seed):
    """The definition, a sequence (and, for an eviction, a head) at a time, sums and exponentials in 64 bits."""
    if case["op"] == "evict" and case["batch"] * HEADS[case["heads"]][1] > 600:
        return None
    global own
    keep, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = keep
    return {"attention": _exact_attention, "append": _exact_append, "evict": _exact_evict}[case["op"]](st, case)


def _sequence(st, case, b, name):
    """Pool rows of sequence b, slot by slot."""
    page, n = case["page"], _lens(case)[b]
    hkv, dh = HEADS[case["heads"]][1:]
    pages = st[name].index_select(0, st["table"][b].long())
    return pages.reshape(-1, hkv, dh)[:n]


def _exact_attention(st, case):
    hq, hkv, dh = HEADS[case["heads"]]
    out, lse = st["out"].double(), st["lse"].double()
    weights = st["weights_out"].double() if case["weights"] else None
    at = 0
    for b, rows in enumerate(_rows(case)):
        k, v = (_sequence(st, case, b, name).double() for name in ("k", "v"))
        for h in range(hq):
            g = h * hkv // hq
            q = st["q"][at:at + rows, h * dh:(h + 1) * dh].double()
            s = torch.einsum("rd,nd->rn", q, k[:, g]) / dh ** 0.5
            z = torch.logsumexp(s, -1)
            p = torch.exp(s - z[:, None])
            out[at:at + rows, h * dh:(h + 1) * dh] = torch.einsum("rn,nd->rd", p, v[:, g])
            lse[at:at + rows, h] = z
            if weights is not None:
                n = p.shape[1]
                if h % (hq // hkv) == 0:
                    weights[b, g, :n] = st["weights_in"][b, g, :n].double()
                weights[b, g, :n] += p.sum(0)
        at += rows
    return (out, lse) if weights is None else (out, lse, weights)


def _exact_append(st, case):
    hq, hkv, dh = HEADS[case["heads"]]
    k, v, weights, pos = (st[name].double() for name in ("k", "v", "weights", "pos"))
    at, lens_out, seen_out = 0, [], []
    for b, (n, rows) in enumerate(zip(_lens(case), _rows(case))):
        slots = torch.arange(n, n + rows, device=DEV)
        pages = st["table"][b].long()[torch.div(slots, case["page"], rounding_mode="floor")]
        new = st["kv_new"][at:at + rows].double()
        k[pages, slots % case["page"]] = new[:, : hkv * dh].reshape(rows, hkv, dh)
        v[pages, slots % case["page"]] = new[:, hkv * dh:].reshape(rows, hkv, dh)
        weights[b, :, n:n + rows] = 0
        pos[b, :, n:n + rows] = torch.arange(n + 5, n + 5 + rows, device=DEV, dtype=torch.float64)
        lens_out.append(n + rows)
        seen_out.append(n + 5 + rows)
        at += rows
    whole = lambda x: torch.tensor(x, dtype=torch.int64)  # noqa: E731
    return k, v, weights, pos.long(), whole(lens_out), whole(seen_out)


def _exact_evict(st, case):
    hkv = HEADS[case["heads"]][1]
    k, v, weights, pos = st["k"].double(), st["v"].double(), st["weights_out"].double(), st["pos_out"].long()
    page, budget = case["page"], case["budget"]
    for b, n in enumerate(_lens(case)):
        table = st["table"][b].long()
        for h in range(hkv):
            w, p = st["weights"][b, h, :n].double(), st["pos"][b, h, :n].long()
            w = w.masked_fill((p < case["sink"]) | (p >= n - case["recent"]), float("inf"))
            by_position = torch.argsort(p)
            heaviest = by_position[torch.sort(w[by_position], descending=True, stable=True).indices]
            kept = torch.sort(heaviest[:budget]).values
            movers = kept[kept >= budget]
            stay = torch.arange(min(n, budget), device=DEV)
            holes = stay[~torch.isin(stay, kept)]
            place = stay.clone()
            place[holes] = movers
            weights[b, h, : len(place)] = st["weights"][b, h, place].double()
            pos[b, h, : len(place)] = st["pos"][b, h, place].long()
            for new, pool in ((k, st["k"]), (v, st["v"])):
                new[table[holes // page], holes % page, h] = pool[table[movers // page], movers % page, h].double()
    return k, v, weights, pos, torch.tensor([min(n, budget) for n in _lens(case)], dtype=torch.int64)


def work(case):
    hq, hkv, dh = HEADS[case["heads"]]
    e = 2 if case["dtype"] == "bf16" else 4
    lens = _lens(case)
    total = sum(lens)
    if case["op"] == "evict":
        # slots whose weight and position are read; of the kept ones the share that lies behind the budget has to move
        moved = sum(case["budget"] * (n - case["budget"]) / n for n in lens if n > case["budget"])
        kept = sum(min(n, case["budget"]) for n in lens)
        return {"bytes": hkv * (8.0 * total + 8.0 * kept + 4.0 * dh * e * moved), "flops": 0.0}
    rows = _rows(case)
    if case["op"] == "append":
        return {"bytes": sum(rows) * hkv * (4.0 * dh * e + 8.0), "flops": 0.0}
    b = 2.0 * total * hkv * dh * e + sum(rows) * hq * (2.0 * dh * e + 4.0) + (8.0 * total * hkv if case["weights"] else 0.0)
    return {"bytes": b, "flops": 4.0 * hq * dh * sum(n * r for n, r in zip(lens, rows))}
