"""Rotation on the way into the paged K/V cache, and caches held in 4 bits: their calls, for measuring them.

A case is one call on a cache of a batch of sequences through KvCache or KvCache4 of
paper_2608_02134_amd.binding:

  rotary    new K/V rows into the cache's pages, keys and queries rotated by their positions on the way
  append4   the same into a cache held in 4 bits, and the rows that it then holds
  decode4   attention of one new token a sequence over a cache held in 4 bits, with an optional window
            and first tokens that stay visible
  prefill4  the same for a sequence's new tokens, causal

A cache of 4 bits holds, for each row and 32 channels of a head, one power of two (a byte e: 2^(e - 127), the least
for which no magnitude is above 7) and 32 signed codes of 0, 0.5, 1, 1.5, 2, 3, 4, 6, the nearest, ties to the
even code; a byte holds the codes of two neighbouring channels, the first one low.

Head layouts and lengths are those of this repository's workloads (the Qwen2.5-VL-7B boundary, 28/4 heads of
128, prompts of 1375 positions compacted to 335; document pages; clips of 16384 visual tokens) and generic ones.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
QWEN = {"hq": 28, "hkv": 4, "dh": 128}
HEADS = [QWEN, {"hq": 32, "hkv": 8, "dh": 128}, {"hq": 8, "hkv": 2, "dh": 64}, {"hq": 16, "hkv": 2, "dh": 128},
         {"hq": 12, "hkv": 12, "dh": 96}, {"hq": 16, "hkv": 1, "dh": 256}, {"hq": 4, "hkv": 4, "dh": 32}]
N_POS = 32768          # rows of the tables of cosines and sines


def _case(op, name=None, *, heads=QWEN, dtype="bf16", page=64, batch=1, **more):
    """lo, hi: the shortest and longest cache of the batch (rows held with the new ones); new: the most new tokens
    of a sequence; src: rows that `new` are taken from, 0 for all; pos: "slot" (none given), "one" or "thw" numbers
    a token; rot: rotated dimensions of a head; pairs: "halves" or "neighbours"; q: queries are rotated too."""
    c = dict(heads, op=op, dtype=dtype, page=page, batch=batch, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of a serving batch behind a multimodal prompt: one row a sequence, latency
        _case("rotary", "rotary_step", page=16, batch=16, lo=300, hi=420, new=1, src=0, pos="thw", rot=128,
              pairs="halves", q=True),
        # a clip of four frames of 64 x 64 tokens before the boundary: the most bytes
        _case("rotary", "rotary_clip", lo=16448, hi=16448, new=16448, src=0, pos="thw", rot=128, pairs="halves", q=True),
        # ragged text prompts in fp32, half of each head rotated, neighbouring pairs
        _case("rotary", "rotary_ragged_f32", heads=HEADS[2], dtype="f32", page=32, batch=5, lo=100, hi=1375, new=1375,
              src=0, pos="slot", rot=32, pairs="neighbours", q=True),
        # a decode step of a larger batch into 4 bits
        _case("append4", "append4_step", batch=64, lo=200, hi=4096, new=1, src=0, pos="one", rot=128, pairs="halves",
              q=True),
        # 16 pruned prompts: a prefix layer's unrotated K and V at the 335 positions of 1375 that were kept
        _case("append4", "append4_pruned_prompts", batch=16, lo=335, hi=335, new=335, src=1375, pos="thw", rot=128,
              pairs="halves", q=False),
        # one pruned chat request, first answer token: the smallest attention call
        _case("decode4", "decode4_one", page=16, lo=336, hi=336, window=0, sinks=0),
        # a serving batch of unlike lengths
        _case("decode4", "decode4_batch", batch=64, lo=200, hi=4096, window=0, sinks=0),
        # long documents, 8 at a time, what 4 bits are for: the cache's bytes
        _case("decode4", "decode4_long", heads=HEADS[1], batch=8, lo=100000, hi=131072, window=0, sinks=0),
        # fp32 queries, windowed
        _case("decode4", "decode4_window_f32", heads=HEADS[2], dtype="f32", batch=5, page=32, lo=900, hi=5001,
              window=1024, sinks=4),
        # ragged prompts, short window
        _case("prefill4", "prefill4_ragged_window", batch=16, lo=100, hi=1375, new=1375, window=512, sinks=4),
        # the next question of a chat over documents that are there already
        _case("prefill4", "prefill4_question", batch=3, lo=2100, hi=4100, new=77, window=0, sinks=0),
        # a clip of four frames of 64 x 64 tokens before the boundary, long window: the largest call
        _case("prefill4", "prefill4_clip_window", lo=16448, hi=16448, new=16448, window=4096, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "append4", "decode4", "decode4", "prefill4", "prefill4"])
    heads = QWEN if rng.random() < 0.4 else rng.choice(HEADS)
    base = dict(heads=heads, dtype="f32" if rng.random() < 0.25 else "bf16", page=rng.choice([16, 32, 64, 128, 256]))
    window, sinks = (_log(rng, 16, 4096), rng.choice([0, 1, 4, 17])) if rng.random() < 0.5 else (0, 0)
    if op in ("rotary", "append4"):
        batch, new = _log(rng, 1, 48), _log(rng, 1, 600)
        src = new + _log(rng, 1, 1000) if rng.random() < 0.4 else 0
        return _case(op, batch=batch, lo=new, hi=new if src else new + _log(rng, 1, 2000), new=new, src=src,
                     pos=rng.choice(["slot", "one", "thw"]), rot=rng.choice([heads["dh"], heads["dh"] // 2]),
                     pairs=rng.choice(["halves", "halves", "neighbours"]), q=rng.random() < 0.7, **base)
    if op == "decode4":
        hi = _log(rng, 1, 60000)
        batch = _log(rng, 1, max(1, min(96, 400000 // hi)))
        return _case(op, batch=batch, lo=_log(rng, 1, hi), hi=hi, window=window, sinks=sinks, **base)
    hi = _log(rng, 2, 3000 if base["dtype"] == "f32" else 9000)
    new = hi if rng.random() < 0.6 else _log(rng, 1, hi)
    batch = _log(rng, 1, max(1, min(24, 9000 // hi)))
    return _case(op, batch=batch, lo=_log(rng, 1, hi), hi=hi, new=new, window=window, sinks=sinks, **base)


# --- 4 bits -----------------------------------------------------------------------
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _scale_bytes(dh):
    """Bytes of a row's scales: a power of two, the last ones unused."""
    return 1 << (dh // 32 - 1).bit_length()


def _quantise(x):
    """[..., dh] fp32 -> codes [..., dh / 2] and scales [..., _scale_bytes] as bytes; blocks with an infinity or NaN have scale 255."""
    y = x.unflatten(-1, (-1, 32))
    size = y.abs()
    top = size.amax(-1)
    e = ((((top.view(torch.int32) + 0x1FFFFF) >> 23) - 2).clamp(1, 254))
    size = size / (e << 23).view(torch.float32)[..., None]
    code = torch.signbit(y).to(torch.uint8) * 8
    for at, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (size >= at) if up else (size > at)
    e = torch.where(torch.isfinite(top), e, 255).to(torch.uint8)
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    room = _scale_bytes(x.shape[-1]) - e.shape[-1]
    return code[..., 0] | (code[..., 1] << 4), torch.nn.functional.pad(e, (0, room))


def _values(codes, scales):
    """fp32 values of codes and scales as _quantise gives them."""
    table = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], device=codes.device)
    x = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()].unflatten(-1, (-1, 32))
    scales = scales[..., : x.shape[-2]]
    s = torch.where(scales == 255, math.nan, (scales.int() << 23).view(torch.float32))
    return (x * s[..., None]).flatten(-2)


# --- inputs -------------------------------------------------------------------
def _lengths(case):
    """Rows held by each sequence after the call's new ones, spread evenly from lo to hi."""
    b, lo, hi = case["batch"], case["lo"], case["hi"]
    return [hi - (hi - lo) * i // max(b - 1, 1) for i in range(b)]


def _new(case):
    return [min(case["new"], n) for n in _lengths(case)]


def _sections(rot):
    """Pairs that turn by t, h and w: a quarter and three eighths each, in fours."""
    side = rot // 2 * 3 // 8 // 4 * 4
    return (rot // 2 - 2 * side, side, side)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 7919 + 29)
    dev, dt, op = "cuda", DTYPES[case["dtype"]], case["op"]
    b, hq, hkv, dh, page = (case[x] for x in ("batch", "hq", "hkv", "dh", "page"))
    lens = _lengths(case)
    per = -(-case["hi"] // page)           # pages a sequence may have
    n_pages = b * per + 3                  # some are not in use
    randn = lambda *s: torch.randn(s, generator=g, device=dev, dtype=dt)  # noqa: E731
    s = {"case": case}
    s["page_table"] = torch.randperm(n_pages, generator=g, device=dev)[: b * per].to(torch.int32).view(b, per)
    held = torch.tensor(lens, dtype=torch.int32, device=dev)
    if op in ("rotary", "append4", "prefill4"):
        new = _new(case)
        s["max_new"], s["total"] = max(new), sum(new)
        s["starts"] = torch.tensor([sum(new[:i]) for i in range(b + 1)], dtype=torch.int32, device=dev)
    if op == "rotary":
        s["k_pages"], s["v_pages"] = randn(n_pages, hkv, page, dh), randn(n_pages, hkv, page, dh)
    else:
        # rows as an earlier call left them: quantised from normal ones (a new cache's for append4)
        for x in "kv":
            s[x + "_codes"] = torch.zeros((n_pages, hkv, page, dh // 2), dtype=torch.uint8, device=dev)
            s[x + "_scales"] = torch.zeros((n_pages, hkv, page, _scale_bytes(dh)), dtype=torch.uint8, device=dev)
            step = max(1, 2 ** 27 // (hkv * page * dh))
            for p in range(0, 0 if op == "append4" else n_pages, step):
                at = slice(p, min(p + step, n_pages))
                rows = torch.randn((at.stop - p, hkv, page, dh), generator=g, device=dev)
                s[x + "_codes"][at], s[x + "_scales"][at] = _quantise(rows)
    if op in ("rotary", "append4"):
        s["start"] = held - torch.tensor(new, dtype=torch.int32, device=dev)
        s["lens"] = s["start"].clone()
        # K and V of the tokens as a projection leaves them, behind their queries in one row
        heads = (hq if case["q"] else 0) + 2 * hkv
        rows = b * case["src"] if case["src"] else s["total"]
        qkv = randn(rows, heads, dh)
        s["q"] = qkv[:, :hq] if case["q"] else None
        s["k"], s["v"] = qkv[:, heads - 2 * hkv:heads - hkv], qkv[:, heads - hkv:]
        s["src"] = None
        if case["src"]:
            r = torch.rand((b, case["src"]), generator=g, device=dev)
            s["src"] = torch.argsort(r, dim=1)[:, : case["new"]].sort(dim=1).values.to(torch.int32)
        # the table of a model's rotation; angles in 64 bits
        half = case["rot"] // 2
        angle = torch.arange(N_POS, device=dev, dtype=torch.float64)[:, None] * \
            1e6 ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
        s["pos"] = None
        if case["pos"] == "one":
            s["pos"] = torch.randint(0, N_POS, (rows,), generator=g, device=dev, dtype=torch.int32)
        elif case["pos"] == "thw":
            # frames of 64 x 64 tokens behind a text of its own length
            i = torch.arange(rows, device=dev)
            at = int(torch.randint(0, 1000, (1,), generator=g, device=dev))
            s["pos"] = torch.stack([at + i // 4096, at + i // 64 % 64, at + i % 64], 1).to(torch.int32)
    else:
        s["lens"] = held
        s["q"] = 2 * randn(b if op == "decode4" else s["total"], hq, dh)   # some keys stand out
    return s


def _cache(s):
    """The handles a program keeps beside its tensors."""
    if "cache" not in s:
        from paper_2608_02134_amd import binding
        c = s["case"]
        if c["op"] == "rotary":
            s["cache"] = binding.KvCache(s["k_pages"], s["v_pages"], s["page_table"], s["lens"], n_q_heads=c["hq"])
        else:
            s["cache"] = binding.KvCache4(s["k_codes"], s["v_codes"], s["k_scales"], s["v_scales"], s["page_table"],
                                          s["lens"], n_q_heads=c["hq"], dtype=DTYPES[c["dtype"]])
        if c["op"] in ("rotary", "append4"):
            s["rotary"] = binding.Rotary(s["cos"], s["sin"], interleaved=c["pairs"] == "neighbours",
                                         sections=_sections(c["rot"]) if c["pos"] == "thw" else None)
    return s["cache"]


# --- the plain forms ------------------------------------------------------------
def _turn(c, x, cos, sin):
    """x [n][heads][dh] by cos, sin [n][rot / 2], in their type."""
    rot, half = c["rot"], c["rot"] // 2
    x = x.to(cos.dtype)
    if c["pairs"] == "halves":
        a, b = x[..., :half], x[..., half:rot]
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    cos, sin = cos[:, None], sin[:, None]
    a, b = a * cos - b * sin, b * cos + a * sin
    both = torch.cat([a, b], -1) if c["pairs"] == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([both, x[..., rot:]], -1)


def _angles(s, row, slot):
    """cos, sin [n][rot / 2] of the tokens: of row `row` of pos, or in slot `slot`."""
    c = s["case"]
    if s["pos"] is None:
        at = slot[:, None].expand(-1, c["rot"] // 2)
    elif c["pos"] == "one":
        at = s["pos"][row][:, None].expand(-1, c["rot"] // 2)
    else:
        at = torch.repeat_interleave(s["pos"][row], torch.tensor(_sections(c["rot"]), device=row.device), dim=1,
                                     output_size=c["rot"] // 2)
    at = at.long().clamp(0, N_POS - 1)
    return torch.gather(s["cos"], 0, at), torch.gather(s["sin"], 0, at)


def _tokens(s):
    """Of each new token: its sequence, its slot and its row of k, v, q and pos."""
    c, n, b = s["case"], s["max_new"], s["case"]["batch"]
    lens, first = s["lens"].long(), s["starts"].long()
    i = torch.arange(n, device=lens.device).expand(b, n)
    live = i < (first[1:] - first[:-1])[:, None]
    seq = torch.arange(b, device=lens.device)[:, None].expand(b, n)
    row = s["src"].long() + seq * c["src"] if c["src"] else first[:-1, None] + i
    return seq[live], (lens[:, None] + i)[live], row[live]


def _plain_append(s):
    c = s["case"]
    seq, slot, row = _tokens(s)
    to, at = s["page_table"][seq, slot // c["page"]].long(), slot % c["page"]
    cos, sin = _angles(s, row, slot)
    k, v = _turn(c, s["k"][row], cos, sin), s["v"][row]
    q = None if s["q"] is None else _turn(c, s["q"][row], cos, sin).to(v.dtype)
    s["lens"] += s["starts"][1:] - s["starts"][:-1]
    if c["op"] == "rotary":
        s["k_pages"][to, :, at], s["v_pages"][to, :, at] = k.to(v.dtype), v
        return {"k": s["k_pages"], "v": s["v_pages"], "q": q, "lens": s["lens"]}
    got = {}
    for x, y in (("k", k), ("v", v.float())):
        codes, scales = _quantise(y)
        s[x + "_codes"][to, :, at], s[x + "_scales"][to, :, at] = codes, scales
        got[x] = _values(codes, scales).to(v.dtype)
    return dict(got, q=q, lens=s["lens"])


def _rows(s, x):
    """The cache's rows as [B][Hkv][slots][dh] in fp32."""
    codes, scales = (s[x + y][s["page_table"].long()].transpose(1, 2).flatten(2, 3) for y in ("_codes", "_scales"))
    return _values(codes, scales)


def _plain_attend(s, q, own_slot):
    """q [B][Hkv][M][dh] fp32 (M: tokens x group), own_slot [B][M] of each row's token (-1: no token)."""
    c, k = s["case"], _rows(s, "k")
    slot = torch.arange(k.shape[2], device=k.device, dtype=torch.int32)
    mine = own_slot[:, None, :, None]
    seen = slot <= mine                                      # [B][1][M][slots]
    if c["window"]:
        seen = seen & ((mine - slot < c["window"]) | (slot < c["sinks"]))
    x = torch.matmul(q * c["dh"] ** -0.5, k.transpose(-1, -2)).masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    return torch.matmul(x, _rows(s, "v")) / total, (m + torch.log(total))[..., 0]


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if op in ("rotary", "append4"):
        s["lens"].copy_(s["start"])        # the same pass again: what the last one counted is taken back
        if not own:
            return _plain_append(s)
        cache, starts = _cache(s), None if c["src"] else s["starts"]
        q = cache.append_rotary(s["k"], s["v"], s["rotary"], pos=s["pos"], q=s["q"], starts=starts,
                                max_new=s["max_new"], src=s["src"])
        if op == "rotary":
            return {"k": s["k_pages"], "v": s["v_pages"], "q": q, "lens": s["lens"]}
        k, v = cache.read(s["total"], starts=starts, max_new=s["max_new"])
        return {"k": k, "v": v, "q": q, "lens": s["lens"]}
    b, hq, hkv, dh = s["lens"].shape[0], c["hq"], c["hkv"], c["dh"]
    if op == "decode4":
        if own:
            out, lse = _cache(s).decode(s["q"], window=c["window"], sinks=c["sinks"], lse=True)
        else:
            own_slot = (s["lens"] - 1)[:, None].expand(b, hq // hkv)
            out, lse = _plain_attend(s, s["q"].float().view(b, hkv, hq // hkv, dh), own_slot)
            out, lse = out.reshape(b, hq, dh).to(s["q"].dtype), lse.reshape(b, hq)
        return {"out": out, "lse": lse}
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
    out, lse = _plain_attend(s, q, own_slot.repeat(1, hg))
    out = out.view(b, hkv, hg, n, dh).permute(0, 3, 1, 2, 4).reshape(b, n, hq, dh)[live]
    lse = lse.view(b, hkv, hg, n).permute(0, 3, 1, 2).reshape(b, n, hq)[live]
    return {"out": out.to(s["q"].dtype), "lse": lse}


# --- what a pass cannot do without ------------------------------------------------
def _visible(n, t, window, sinks):
    """Keys that the query of slot t sees."""
    lo = max(0, t + 1 - window) if window else 0
    return t + 1 - lo + min(sinks, lo)


def work(case):
    e, hkv, hq, dh = DTYPES[case["dtype"]].itemsize, case["hkv"], case["hq"], case["dh"]
    op, lens = case["op"], _lengths(case)
    held = dh / 2 + dh / 32                # bytes of a row in 4 bits
    if op in ("rotary", "append4"):
        rows, q = sum(_new(case)), hq if case["q"] else 0
        # K, V and q read and q written; rows written as they are, or in 4 bits and their values
        kept = 2 * hkv * (dh * e if op == "rotary" else held + dh * e)
        return {"bytes": rows * ((2 * hkv + 2 * q) * dh * e + kept), "flops": 3.0 * rows * (hkv + q) * case["rot"]}
    if op == "decode4":
        seen = sum(_visible(n, n - 1, case["window"], case["sinks"]) for n in lens)
        return {"bytes": 2.0 * seen * hkv * held + len(lens) * hq * (2 * dh * e + 4), "flops": 4.0 * hq * dh * seen}
    new, pairs, keys = _new(case), 0, 0
    for n, m in zip(lens, new):
        w = case["window"] if case["window"] else n
        sink = case["sinks"] if case["window"] else 0
        # sum over t = n - m .. n - 1 of min(t + 1, w) + min(sinks, max(0, t + 1 - w))
        upto = lambda x, cap: x * (x + 1) / 2 if x <= cap else cap * (cap + 1) / 2 + (x - cap) * cap  # noqa: E731
        pairs += upto(n, w) - upto(n - m, w) + upto(max(0, n - w), sink) - upto(max(0, n - m - w), sink)
        keys += min(n, m + w + sink)
    return {"bytes": 2.0 * keys * hkv * held + sum(new) * hq * (2 * dh * e + 4), "flops": 4.0 * hq * dh * pairs}


# --- the definition in 64 bits ------------------------------------------------------
def _exact_values(x):
    """The values nearest to x [..., dh] that 4 bits and a power of two for 32 channels hold."""
    y = x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True).clamp(min=1e-36)
    scale = torch.exp2(torch.ceil(torch.log2(top / 7)))
    y = y / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
    return ((torch.round(y / step) * step).clamp(-6, 6) * scale).flatten(-2)


def _exact_append(case, s):
    """Token by token's row: complex numbers times exp of their angles' cosine and sine."""
    half, rot = case["rot"] // 2, case["rot"]
    lens, new = s["lens"].tolist(), _new(case)
    take = [(i * case["src"] + s["src"][i].long() if case["src"] else s["starts"][i].long() + torch.arange(m, device="cuda"))
            for i, m in enumerate(new)]
    row = torch.cat(take)
    slot = torch.cat([torch.arange(n, n + m, device="cuda") for n, m in zip(lens, new)])
    seq = torch.cat([torch.full((m,), i, device="cuda") for i, m in enumerate(new)])
    axis = torch.zeros(half, dtype=torch.long, device="cuda")
    if case["pos"] == "thw":
        t, h, _ = _sections(rot)
        axis[t:], axis[t + h:] = 1, 2
    pos = slot[:, None] if s["pos"] is None else s["pos"][row].long().view(len(row), -1)
    at = pos[:, axis].clamp(max=N_POS - 1)
    z = torch.complex(torch.gather(s["cos"], 0, at).double(), torch.gather(s["sin"], 0, at).double())[:, None]

    def turn(x):
        x = x[row].double().clone()
        first, second = (slice(0, half), slice(half, rot)) if case["pairs"] == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
        y = torch.complex(x[..., first], x[..., second]) * z
        x[..., first], x[..., second] = y.real, y.imag
        return x

    k, q = turn(s["k"]), None if s["q"] is None else turn(s["q"])
    if case["op"] == "append4":
        return {"k": _exact_values(k), "v": _exact_values(s["v"][row].double()), "q": q, "lens": None}
    pages = s["k_pages"].double()
    pages[s["page_table"][seq, slot // case["page"]].long(), :, slot % case["page"]] = k
    return {"k": pages, "v": None, "q": q, "lens": None}   # V is moved, not computed


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rotary", "append4"):
        return _exact_append(case, s)
    f64 = torch.float64
    lens, table, hg, dh = s["lens"].tolist(), s["page_table"].long(), case["hq"] // case["hkv"], case["dh"]
    first = s["starts"].tolist() if case["op"] == "prefill4" else list(range(len(lens) + 1))
    if sum(n * (first[b + 1] - first[b]) for b, n in enumerate(lens)) * case["hq"] > 2e10:
        return None
    signed = torch.tensor(MAGNITUDES, dtype=f64, device="cuda")

    def rows(x, b, h, n):
        codes = s[x + "_codes"][table[b], h].reshape(-1, dh // 2)[:n].int()
        power = s[x + "_scales"][table[b], h].reshape(codes.shape[0] if n == 0 else -1, _scale_bytes(dh))[:n, : dh // 32]
        y = torch.empty((n, dh), dtype=f64, device="cuda")
        for odd in (0, 1):
            c = codes >> 4 if odd else codes & 15
            y[:, odd::2] = signed[c & 7] * (1 - 2 * (c >> 3))
        return y * torch.exp2(power.to(f64) - 127).repeat_interleave(32, 1)

    out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=f64, device="cuda")
    for b, n in enumerate(lens):
        t = torch.arange(n - (first[b + 1] - first[b]), n, device="cuda")
        p = torch.arange(n, device="cuda")
        hidden = p[None] > t[:, None]
        if case["window"]:
            hidden |= (p[None] <= t[:, None] - case["window"]) & (p[None] >= case["sinks"])
        for h in range(case["hkv"]):
            k, v = rows("k", b, h, n), rows("v", b, h, n)
            for j in range(h * hg, (h + 1) * hg):
                x = s["q"][first[b]:first[b + 1], j].to(f64) @ k.T / math.sqrt(dh)
                x[hidden] = -math.inf
                lse[first[b]:first[b + 1], j] = torch.logsumexp(x, 1)
                out[first[b]:first[b + 1], j] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}
