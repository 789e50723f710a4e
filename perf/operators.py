"""The paged K/V cache behind a pruned prompt: its calls, for measuring them.

A case is one call on a cache of a batch of sequences through KvCache of
paper_2608_02134_amd.binding:

  append   new K/V rows into the cache's pages: one token a sequence, or the
           rows of a prompt at the positions that pruning kept
  prefill  attention of a sequence's new tokens over its cache, causal, with an
           optional sliding window and first tokens that stay visible
  decode   the same for one new token a sequence; optionally the attention
           weights are added to the cache's
  evict    the rows of least accumulated attention weight leave the cache

Head layouts and lengths are those of this repository's workloads (the
Qwen2.5-VL-7B boundary, 28/4 heads of 128, prompts of 1375 positions compacted
to 335; document pages; clips of 16384 visual tokens) and generic ones.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
QWEN = {"hq": 28, "hkv": 4, "dh": 128}
HEADS = [QWEN, {"hq": 32, "hkv": 8, "dh": 128}, {"hq": 8, "hkv": 2, "dh": 64}, {"hq": 16, "hkv": 2, "dh": 128},
         {"hq": 12, "hkv": 12, "dh": 96}, {"hq": 16, "hkv": 1, "dh": 256}, {"hq": 4, "hkv": 4, "dh": 32}]


def _case(op, name=None, *, heads=QWEN, dtype="bf16", page=16, batch=1, **more):
    """lo, hi: the shortest and longest cache of the batch (rows held with the
    new ones); new: the most new tokens of a sequence."""
    c = dict(heads, op=op, dtype=dtype, page=page, batch=batch, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of a serving batch writes one row a sequence: latency
        _case("append", "append_step", batch=16, lo=300, hi=420, new=1, src=0, positions=True),
        # 16 pruned prompts: a prefix layer's K/V at the 335 positions of 1375 that were kept
        _case("append", "append_pruned_prompts", batch=16, lo=335, hi=335, new=335, src=1375, positions=False),
        # one pruned chat request, first answer token: the smallest attention call
        _case("decode", "decode_one", lo=336, hi=336, window=0, sinks=0, weigh=False, positions=False),
        # a serving batch of unlike lengths whose caches are kept bounded: weights added up
        _case("decode", "decode_batch", batch=64, page=64, lo=200, hi=4096, window=0, sinks=0, weigh=True,
              positions=True),
        # long documents, 8 at a time: the cache's bytes, offsets beyond 32 bits
        _case("decode", "decode_long", heads=HEADS[1], batch=8, page=64, lo=100000, hi=131072, window=0, sinks=0,
              weigh=False, positions=False),
        # fp32, caches that evictions have reordered, windowed by the rows' positions
        _case("decode", "decode_window_f32", heads=HEADS[2], dtype="f32", batch=5, page=32, lo=900, hi=5001,
              window=1024, sinks=4, weigh=True, positions=True),
        # the boundary sequence of one pruned request through a later block
        _case("prefill", "prefill_pruned", lo=335, hi=335, new=335, window=0, sinks=0, positions=False),
        # ragged prompts, short window
        _case("prefill", "prefill_ragged_window", batch=16, page=64, lo=100, hi=1375, new=1375, window=512, sinks=4,
              positions=False),
        # a clip of four frames of 64 x 64 tokens before the boundary, long window: the largest call
        _case("prefill", "prefill_clip_window", page=64, lo=16448, hi=16448, new=16448, window=4096, sinks=4,
              positions=False),
        # fp32, the next question of a chat over a cache that is there already
        _case("prefill", "prefill_question_f32", heads=HEADS[2], dtype="f32", batch=3, page=32, lo=2100, hi=4100,
              new=77, window=0, sinks=0, positions=False),
        # 16 sequences whose caches are brought back to 4096 rows after 64 more
        _case("evict", "evict_step", batch=16, page=64, lo=4160, hi=4160, budget=4096, sinks=4, recent=64),
        # long documents cut to an eighth at once
        _case("evict", "evict_document", heads=HEADS[1], batch=2, page=64, lo=60001, hi=65536, budget=8192, sinks=4,
              recent=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prefill", "prefill", "evict"])
    heads = QWEN if rng.random() < 0.4 else rng.choice(HEADS)
    base = dict(heads=heads, dtype="f32" if rng.random() < 0.25 else "bf16", page=rng.choice([16, 32, 64, 128, 256]))
    window, sinks = (_log(rng, 16, 4096), rng.choice([0, 1, 4, 17])) if rng.random() < 0.5 else (0, 0)
    if op == "append":
        batch = _log(rng, 1, 48)
        if rng.random() < 0.5:
            new = _log(rng, 2, 700)
            return _case(op, batch=batch, lo=new, hi=new, new=new, src=new + _log(rng, 1, 1500), positions=False, **base)
        new = _log(rng, 1, 600)
        return _case(op, batch=batch, lo=new, hi=new + _log(rng, 1, 2000), new=new, src=0, positions=rng.random() < 0.5,
                     **base)
    if op == "decode":
        hi = _log(rng, 1, 60000)
        batch = _log(rng, 1, max(1, min(96, 400000 // hi)))
        return _case(op, batch=batch, lo=_log(rng, 1, hi), hi=hi, window=window, sinks=sinks, weigh=rng.random() < 0.4,
                     positions=rng.random() < 0.4, **base)
    if op == "prefill":
        f32 = base["dtype"] == "f32"
        hi = _log(rng, 2, 3000 if f32 else 9000)
        new = hi if rng.random() < 0.6 else _log(rng, 1, hi)
        batch = _log(rng, 1, max(1, min(24, 9000 // hi)))
        return _case(op, batch=batch, lo=_log(rng, 1, hi), hi=hi, new=new, window=window, sinks=sinks,
                     positions=rng.random() < 0.2, **base)
    hi = _log(rng, 64, 40000)
    batch = _log(rng, 1, max(1, min(32, 300000 // hi)))
    budget = max(40, int(hi * rng.choice([0.98, 0.75, 0.5, 0.2])))
    return _case(op, batch=batch, lo=max(1, int(hi * rng.uniform(0.3, 1))), hi=hi, budget=min(budget, hi - 1),
                 sinks=rng.choice([0, 4]), recent=rng.randint(0, 32), **base)


# --- inputs -------------------------------------------------------------------
def _lengths(case):
    """Rows held by each sequence after the call's new ones, spread evenly from lo to hi."""
    b, lo, hi = case["batch"], case["lo"], case["hi"]
    return [hi - (hi - lo) * i // max(b - 1, 1) for i in range(b)]


def _new(case):
    return [min(case["new"], n) for n in _lengths(case)]


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    dev, dt = "cuda", DTYPES[case["dtype"]]
    b, hq, hkv, dh, page = (case[x] for x in ("batch", "hq", "hkv", "dh", "page"))
    lens = _lengths(case)
    per = -(-case["hi"] // page)           # pages a sequence may have
    n_pages = b * per + 3                  # some are not in use
    randn = lambda *s: torch.randn(s, generator=g, device=dev, dtype=dt)  # noqa: E731
    s = {"case": case}
    s["k_pages"], s["v_pages"] = randn(n_pages, hkv, page, dh), randn(n_pages, hkv, page, dh)
    s["page_table"] = torch.randperm(n_pages, generator=g, device=dev)[: b * per].to(torch.int32).view(b, per)
    op, cap = case["op"], per * page
    held = torch.tensor(lens, dtype=torch.int32, device=dev)
    if op == "append":
        held = held - torch.tensor(_new(case), dtype=torch.int32, device=dev)
    # a cache that evictions have gone over has seen more positions than it holds, in any order
    seen, slot_pos = held.clone(), None
    if op == "evict" or case["positions"]:
        old = held - (torch.tensor(_new(case), dtype=torch.int32, device=dev) if op == "prefill" else 0)
        past = (old + old // 3).long()                       # positions that went by before the new ones
        r = torch.rand((b, hkv, cap + cap // 3), generator=g, device=dev)
        r = torch.where(torch.arange(r.shape[2], device=dev) < past[:, None, None], r, 2.0)
        pick = torch.argsort(r, dim=2)[..., :cap]            # a random choice of `old` of the past ones, then any
        at = torch.arange(cap, device=dev)
        new_pos = past[:, None, None] + (at - old[:, None, None])
        slot_pos = torch.where(at < old[:, None, None], pick, new_pos).to(torch.int32)
        if op == "decode":                                   # the new token's row is the last one
            last = held[:, None, None].long() - 1
            slot_pos = torch.where(at == last, past[:, None, None].to(torch.int32), slot_pos)
            past = past + 1
        elif op == "prefill":
            past = past + torch.tensor(_new(case), device=dev)
        seen = past.to(torch.int32)
    weights = None
    if op == "evict" or case.get("weigh"):
        # attention weights that many steps have added up: many small, a few large
        u = torch.rand((b, hkv, cap), generator=g, device=dev)
        weights = torch.exp(6 * u - 10) * torch.rand((b, hkv, cap), generator=g, device=dev)
    # one buffer for what a call counts and adds up, as KvCache.create lays it out
    parts = [held, seen] + [x.reshape(-1) for x in (slot_pos,) if x is not None]
    parts += [weights.reshape(-1).view(torch.int32)] if weights is not None else []
    s["start"] = torch.cat(parts)
    s["book"] = s["start"].clone()
    s["lens"], s["seen"], rest = s["book"][:b], s["book"][b:2 * b], s["book"][2 * b:]
    s["slot_pos"] = s["weights"] = None
    if slot_pos is not None:
        s["slot_pos"], rest = rest[: b * hkv * cap].view(b, hkv, cap), rest[b * hkv * cap:]
    if weights is not None:
        s["weights"] = rest.view(torch.float32).view(b, hkv, cap)
    if op in ("append", "prefill"):
        new = _new(case)
        s["max_new"] = max(new)
        s["starts"] = torch.tensor([sum(new[:i]) for i in range(b + 1)], dtype=torch.int32, device=dev)
        s["total"] = sum(new)
    if op == "append":
        # K and V of the tokens as a projection leaves them: side by side in one row
        rows = b * case["src"] if case["src"] else s["total"]
        kv = randn(rows, 2, hkv, dh)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        s["src"] = None
        if case["src"]:
            r = torch.rand((b, case["src"]), generator=g, device=dev)
            s["src"] = torch.argsort(r, dim=1)[:, : case["new"]].sort(dim=1).values.to(torch.int32)
    elif op == "decode":
        s["q"] = 2 * randn(b, hq, dh)      # logits of deviation 2: some keys stand out
    elif op == "prefill":
        s["q"] = 2 * randn(s["total"], hq, dh)
    return s


def _cache(s):
    """The handle a program keeps beside its tensors."""
    if "cache" not in s:
        from paper_2608_02134_amd import binding
        s["cache"] = binding.KvCache(s["k_pages"], s["v_pages"], s["page_table"], s["lens"], n_q_heads=s["case"]["hq"],
                                     slot_pos=s["slot_pos"], seen=s["seen"], weights=s["weights"])
    return s["cache"]


# --- the plain forms ------------------------------------------------------------
def _rows(s, pages):
    """The cache's rows as [B][Hkv][slots][dh] in fp32."""
    x = pages[s["page_table"].long()]                        # [B][per][Hkv][page][dh]
    b, per, hkv, page, dh = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(b, hkv, per * page, dh).float()


def _plain_attend(s, q, own_slot, weigh=False):
    """q [B][Hkv][M][dh] fp32 (M: tokens x group), own_slot [B][M] of each row's token (-1: no token)."""
    c, k, v = s["case"], _rows(s, s["k_pages"]), _rows(s, s["v_pages"])
    slot = torch.arange(k.shape[2], device=k.device, dtype=torch.int32)
    seen = slot <= own_slot[:, None, :, None]                # [B][1][M][slots]
    if c["window"]:
        pos = slot.expand(k.shape[0], 1, -1) if s["slot_pos"] is None else s["slot_pos"]
        mine = torch.gather(pos, 2, own_slot.clamp(min=0).long()[:, None].expand(-1, pos.shape[1], -1))
        near = mine[..., None] - pos[:, :, None] < c["window"]
        seen = seen & (near | (pos < c["sinks"])[:, :, None])
    x = torch.matmul(q * c["dh"] ** -0.5, k.transpose(-1, -2)).masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v) / total
    return out, (m + torch.log(total))[..., 0], x.div_(total).sum(2) if weigh else None


def _plain_append(s):
    c, n = s["case"], s["max_new"]
    lens, page, b = s["lens"].long(), s["case"]["page"], s["case"]["batch"]
    i = torch.arange(n, device=lens.device).expand(b, n)
    first = s["starts"].long()
    live = i < (first[1:] - first[:-1])[:, None]
    row = s["src"].long() + torch.arange(b, device=lens.device)[:, None] * c["src"] if c["src"] else first[:-1, None] + i
    slot = (lens[:, None] + i)[live]
    seq = torch.arange(b, device=lens.device)[:, None].expand(b, n)[live]
    to = s["page_table"][seq, slot // page].long()
    s["k_pages"][to, :, slot % page] = s["k"][row[live]]
    s["v_pages"][to, :, slot % page] = s["v"][row[live]]
    if s["slot_pos"] is not None:
        s["slot_pos"][seq, :, slot] = (s["seen"].long()[:, None] + i)[live][:, None].to(torch.int32)
    s["seen"] += (first[1:] - first[:-1]).to(torch.int32)
    s["lens"] += (first[1:] - first[:-1]).to(torch.int32)


def _plain_evict(s):
    c = s["case"]
    w, pos, lens, keep = s["weights"], s["slot_pos"], s["lens"][:, None, None], c["budget"]
    slot = torch.arange(w.shape[2], device=w.device)
    held = slot < lens
    safe = (pos < c["sinks"]) | (pos >= s["seen"][:, None, None] - c["recent"])
    rank = torch.where(held, torch.where(safe, math.inf, w), -math.inf)
    order = torch.argsort(rank, dim=2, descending=True, stable=True)
    kept = torch.zeros_like(held.expand_as(w)).scatter_(2, order[..., :keep], True) & held
    full = lens > keep
    to = (~kept & held & (slot < keep) & full).nonzero()
    at = (kept & (slot >= keep) & full).nonzero()
    page = lambda x: (s["page_table"][x[:, 0], x[:, 2] // c["page"]].long(), x[:, 1], x[:, 2] % c["page"])  # noqa: E731
    for x, f, t in ((s["k_pages"], page(at), page(to)), (s["v_pages"], page(at), page(to)),
                    (w, at.unbind(1), to.unbind(1)), (pos, at.unbind(1), to.unbind(1))):
        x[t] = x[f]
    s["lens"].clamp_(max=keep)


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if op != "prefill":
        s["book"].copy_(s["start"])        # the same pass again: what the last one counted is taken back
    if op == "append":
        if own:
            _cache(s).append(s["k"], s["v"], starts=None if c["src"] else s["starts"], max_new=s["max_new"], src=s["src"])
        else:
            _plain_append(s)
        return {"k": s["k_pages"], "v": s["v_pages"], "book": s["book"]}
    if op == "evict":
        if own:
            _cache(s).evict(c["budget"], sinks=c["sinks"], recent=c["recent"])
        else:
            _plain_evict(s)
        # rows past the budget are free: what they hold is nobody's
        live = s["weights"][..., : c["budget"]], s["slot_pos"][..., : c["budget"]]
        return {"k": s["k_pages"], "v": s["v_pages"], "lens": s["lens"], "weights": live[0], "pos": live[1]}
    b, hq, hkv, dh = s["lens"].shape[0], c["hq"], c["hkv"], c["dh"]
    if op == "decode":
        if own:
            out, lse = _cache(s).decode(s["q"], window=c["window"], sinks=c["sinks"], accumulate=c["weigh"], lse=True)
        else:
            own_slot = (s["lens"] - 1)[:, None].expand(b, hq // hkv)
            out, lse, p = _plain_attend(s, s["q"].float().view(b, hkv, hq // hkv, dh), own_slot, c["weigh"])
            out, lse = out.reshape(b, hq, dh).to(s["q"].dtype), lse.reshape(b, hq)
            if c["weigh"]:
                s["weights"] += p
        return {"out": out, "lse": lse, "weights": s["weights"]} if c["weigh"] else {"out": out, "lse": lse}
    if own:
        out, lse = _cache(s).prefill(s["q"], starts=s["starts"], max_new=s["max_new"], window=c["window"],
                                      sinks=c["sinks"], lse=True)
        return {"out": out, "lse": lse}
    n, hg, first = s["max_new"], hq // hkv, s["starts"].long()
    i = torch.arange(n, device=first.device).expand(b, n)
    live = i < (first[1:] - first[:-1])[:, None]
    row = torch.where(live, first[:-1, None] + i, 0)
    q = s["q"].float()[row].view(b, n, hkv, hg, dh).permute(0, 2, 3, 1, 4).reshape(b, hkv, hg * n, dh)
    own_slot = torch.where(live, s["lens"][:, None] - (first[1:] - first[:-1])[:, None] + i, -1).to(torch.int32)
    out, lse, _ = _plain_attend(s, q, own_slot.repeat(1, hg))
    out = out.view(b, hkv, hg, n, dh).permute(0, 3, 1, 2, 4).reshape(b, n, hq, dh)[live]
    lse = lse.view(b, hkv, hg, n).permute(0, 3, 1, 2).reshape(b, n, hq)[live]
    return {"out": out.to(s["q"].dtype), "lse": lse}


# --- what a pass cannot do without ------------------------------------------------
def _visible(n, t, window, sinks):
    """Keys that the query of slot t sees in a cache in order."""
    lo = max(0, t + 1 - window) if window else 0
    return t + 1 - lo + min(sinks, lo)


def work(case):
    e, hkv, hq, dh = DTYPES[case["dtype"]].itemsize, case["hkv"], case["hq"], case["dh"]
    op, lens = case["op"], _lengths(case)
    if op == "append":
        rows = sum(_new(case))
        return {"bytes": 4.0 * rows * hkv * dh * e, "flops": 0.0}
    if op == "evict":
        over = [n for n in lens if n > case["budget"]]
        moved = sum((n - case["budget"]) * case["budget"] / n for n in over)   # holes among the first `budget` slots
        return {"bytes": hkv * (8.0 * sum(over) + moved * (4 * dh * e + 8)), "flops": 0.0}
    if op == "decode":
        # where positions are out of order the same number of keys is in the window, about
        seen = sum(_visible(n, n - 1, case["window"], case["sinks"]) for n in lens)
        more = hkv * sum(lens) * (8 * bool(case["weigh"]) + 4 * bool(case["positions"] and case["window"]))
        return {"bytes": 2.0 * seen * hkv * dh * e + more + len(lens) * hq * (2 * dh * e + 4), "flops": 4.0 * hq * dh * seen}
    new, pairs, keys = _new(case), 0, 0
    for n, m in zip(lens, new):
        w = case["window"] if case["window"] else n
        sink = case["sinks"] if case["window"] else 0
        # sum over t = n - m .. n - 1 of min(t + 1, w) + min(sinks, max(0, t + 1 - w))
        upto = lambda x, cap: x * (x + 1) / 2 if x <= cap else cap * (cap + 1) / 2 + (x - cap) * cap  # noqa: E731
        pairs += upto(n, w) - upto(n - m, w) + upto(max(0, n - w), sink) - upto(max(0, n - m - w), sink)
        keys += min(n, m + w + sink)
    return {"bytes": 2.0 * keys * hkv * dh * e + sum(new) * hq * (2 * dh * e + 4), "flops": 4.0 * hq * dh * pairs}


# --- the definition in 64 bits ------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("append", "evict"):
        return None                        # rows are moved, nothing is computed
    f64 = torch.float64
    lens, table, hg = s["lens"].tolist(), s["page_table"].long(), case["hq"] // case["hkv"]
    first = s["starts"].tolist() if case["op"] == "prefill" else list(range(len(lens) + 1))
    if sum(n * (first[b + 1] - first[b]) for b, n in enumerate(lens)) * case["hq"] > 2e10:
        return None
    out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=f64, device="cuda")
    add = torch.zeros((len(lens), case["hkv"], table.shape[1] * case["page"]), dtype=f64, device="cuda")
    for b, n in enumerate(lens):
        m = first[b + 1] - first[b]
        t = torch.arange(n - m, n, device="cuda")
        for h in range(case["hkv"]):
            k = s["k_pages"][table[b], h].reshape(-1, case["dh"])[:n].to(f64)
            v = s["v_pages"][table[b], h].reshape(-1, case["dh"])[:n].to(f64)
            p = torch.arange(n, device="cuda") if s["slot_pos"] is None else s["slot_pos"][b, h, :n].long()
            hidden = torch.arange(n, device="cuda")[None] > t[:, None]
            if case["window"]:
                hidden |= (p[None] <= p[t][:, None] - case["window"]) & (p[None] >= case["sinks"])
            for j in range(h * hg, (h + 1) * hg):
                x = s["q"][first[b]:first[b + 1], j].to(f64) @ k.T / math.sqrt(case["dh"])
                x[hidden] = -math.inf
                lse[first[b]:first[b + 1], j] = torch.logsumexp(x, 1)
                a = torch.softmax(x, 1)
                out[first[b]:first[b + 1], j] = a @ v
                add[b, h, :n] += a.sum(0)
    got = {"out": out, "lse": lse}
    return dict(got, weights=s["weights"].to(f64) + add) if case.get("weigh") else got
