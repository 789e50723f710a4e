"""The paged K/V cache on the GPU against its oracle: appended rows and
evictions bit-exact, attention within bounds derived from its roundings."""
import copy

import numpy as np
import pytest

from oracle import cache_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from . import cache_cases as C  # noqa: E402


def _say(what):
    print(f"\n[case] {what}", flush=True)


# --- append ------------------------------------------------------------------------
APPENDS = {
    "step": dict(dtype="bf16", hq=28, hkv=4, dh=128, page=16, lens=[15, 16, 0, 100], slots=128, new=[1, 1, 1, 1]),
    "ragged": dict(dtype="bf16", hq=4, hkv=2, dh=96, page=32, lens=[3, 31, 64], slots=160, new=[70, 0, 33]),
    "fills_up": dict(dtype="f32", hq=3, hkv=3, dh=32, page=16, lens=[30, 5], slots=32, new=[9, 32]),
    "wide": dict(dtype="f32", hq=2, hkv=1, dh=256, page=64, lens=[0], slots=300, new=[300]),
}


@pytest.mark.parametrize("case", list(APPENDS))
@pytest.mark.parametrize("positions", [False, True])
def test_append(case, positions):
    a = dict(APPENDS[case])
    _say(f"append {case} positions={positions} {a}")
    new = a.pop("new")
    rng = np.random.default_rng(3)
    c = C.make(rng, positions=positions, weights=positions, **a)
    kv = C.rounded(rng.standard_normal((sum(new), 2, a["hkv"], a["dh"])), a["dtype"])
    first = np.concatenate([[0], np.cumsum(new)])
    dev = C.on_gpu(c)
    x = C.to_gpu(kv, a["dtype"])
    dev.append(x[:, 0], x[:, 1], starts=torch.tensor(first, dtype=torch.int32).cuda(), max_new=max(new))
    O.append(c, kv[:, 0], kv[:, 1], new, [np.arange(first[b], first[b + 1]) for b in range(len(new))])
    _compare_caches(c, dev)


def _compare_caches(c, dev):
    assert np.array_equal(dev.lens.cpu().numpy(), c["lens"])
    assert C.same(C.host(dev.k_pages), c["k"]) and C.same(C.host(dev.v_pages), c["v"])
    if c.get("slot_pos") is not None:
        assert np.array_equal(dev.seen.cpu().numpy(), c["seen"])
        for b in range(len(c["lens"])):
            n = c["lens"][b]
            assert np.array_equal(dev.slot_pos[b, :, :n].cpu().numpy(), c["slot_pos"][b, :, :n])
    if c.get("weights") is not None:
        for b in range(len(c["lens"])):
            n = c["lens"][b]
            assert C.same(C.host(dev.weights[b, :, :n]), c["weights"][b, :, :n])


@pytest.mark.parametrize("n,per", [(335, 1375), (1, 1), (40, 97)])
def test_append_of_kept_rows(n, per):
    _say(f"append src n={n} of {per}")
    rng = np.random.default_rng(n)
    c = C.make(rng, dtype="bf16", hq=28, hkv=4, dh=128, page=16, lens=[0, 7], slots=400)
    kv = C.rounded(rng.standard_normal((2 * per, 2, 4, 128)), "bf16")
    src = np.stack([np.sort(rng.choice(per, n, replace=False)) for _ in range(2)]).astype(np.int32)
    dev, x = C.on_gpu(c), C.to_gpu(kv, "bf16")
    dev.append(x[:, 0], x[:, 1], src=torch.from_numpy(src).cuda())
    O.append(c, kv[:, 0], kv[:, 1], [n, n], [src[0], per + src[1]])
    _compare_caches(c, dev)


def test_append_clamps_and_leaves_out():
    """Source rows out of range are clamped, rows on pages that are none left
    out, starts out of range clipped to the rows there are."""
    _say("append bad indices")
    rng = np.random.default_rng(5)
    c = C.make(rng, dtype="bf16", hq=2, hkv=2, dh=64, page=16, lens=[10, 3], slots=64)
    c["table"][0, 1], c["table"][1, 0] = -1, 10 ** 6
    kv = C.rounded(rng.standard_normal((24, 2, 2, 64)), "bf16")
    src = np.array([[-5, 0, 11, 12, 2 ** 31 - 1] * 4, [3, 2, 1, 0, -2 ** 31] * 4], np.int32)
    dev, x = C.on_gpu(c), C.to_gpu(kv, "bf16")
    dev.append(x[:, 0], x[:, 1], src=torch.from_numpy(src).cuda())
    rows = np.clip(src.astype(np.int64), 0, 11) + np.array([[0], [12]])
    O.append(c, kv[:, 0], kv[:, 1], [20, 20], rows)
    _compare_caches(c, dev)
    starts = torch.tensor([20, 2 ** 31 - 1, -4], dtype=torch.int32).cuda()   # 4 rows, then none
    dev.append(x[:, 0], x[:, 1], starts=starts, max_new=6)
    O.append(c, kv[:, 0], kv[:, 1], [4, 0], [np.arange(20, 24), []])
    _compare_caches(c, dev)


# --- attention ----------------------------------------------------------------------
HEADS = [(28, 4, 128), (8, 2, 64), (6, 6, 96), (16, 1, 256), (4, 4, 32), (32, 1, 128), (5, 1, 160), (40, 2, 64),
         (3, 1, 192), (2, 2, 224)]
WINDOWS = [(0, 0), (1, 0), (37, 4), (64, 0), (5, 100)]


def _decode(rng, c, window, sinks, accumulate=False, stride=0):
    b, hq, dh = len(c["lens"]), c["hq"], c["k"].shape[3]
    q = C.queries(rng, c, b)
    dev, x = C.on_gpu(c), C.to_gpu(q, c["dtype"])
    if stride:
        wide = torch.full((b, hq + 3, dh), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, 1:hq + 1] = x
        x = wide[:, 1:hq + 1]
    out, lse = dev.decode(x, window=window, sinks=sinks, accumulate=accumulate, lse=True)
    ref = O.attend(c, q, list(range(b)), [1] * b, dh ** -0.5, window, sinks)
    C.check_attention(ref, C.host(out), C.host(lse), c["dtype"], dh)
    if accumulate:
        C.check_weights(ref, c["weights"], C.host(dev.weights), dh)


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_heads(heads, dtype):
    hq, hkv, dh = heads
    _say(f"decode {dtype} {heads}")
    rng = np.random.default_rng(hq * dh)
    c = C.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[1, 200, 33], slots=208, weights=True)
    _decode(rng, c, 0, 0, accumulate=True, stride=1)


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("positions", [False, True])
def test_decode_lengths(window, page, positions):
    _say(f"decode lengths window={window} page={page} positions={positions}")
    rng = np.random.default_rng(page)
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 300]
    c = C.make(rng, dtype="bf16", hq=14, hkv=2, dh=64, page=page, lens=lens, slots=300, positions=positions,
               weights=True)
    _decode(rng, c, *window, accumulate=True)


@pytest.mark.parametrize("dtype,n", [("bf16", 4999), ("f32", 3001), ("bf16", 9000)])
@pytest.mark.parametrize("window", [(0, 0), (700, 5)], ids=str)
def test_decode_long(dtype, n, window):
    _say(f"decode long {dtype} {n} {window}")
    rng = np.random.default_rng(n)
    c = C.make(rng, dtype=dtype, hq=7, hkv=1, dh=128, page=32, lens=[n, 1], slots=n, weights=True)
    _decode(rng, c, *window, accumulate=True)


def test_decode_length_past_the_table_and_below_zero():
    _say("decode lens out of range")
    rng = np.random.default_rng(8)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[48, 20], slots=48, weights=True)
    c["lens"][:] = 2 ** 31 - 1, -7
    _decode(rng, c, 0, 0, accumulate=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [(0, 0), (9, 2)], ids=str)
def test_decode_pages_that_are_none(dtype, window):
    _say(f"decode bad pages {dtype} {window}")
    rng = np.random.default_rng(9)
    c = C.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[60, 40, 16], slots=64, weights=True)
    c["table"][0, 1], c["table"][0, 3], c["table"][1, 0], c["table"][2, 0] = -1, 2 ** 31 - 1, 10 ** 6, -2 ** 31
    _decode(rng, c, *window, accumulate=True)


def _prefill(rng, c, new, window, sinks, gap=2, stride=0):
    b, hq, dh = len(c["lens"]), c["hq"], c["k"].shape[3]
    first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    rows = int(first[-1]) + gap
    q = C.queries(rng, c, rows)
    dev, x = C.on_gpu(c), C.to_gpu(q, c["dtype"])
    if stride:
        wide = torch.full((rows, hq + 3, dh), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, 1:hq + 1] = x
        x = wide[:, 1:hq + 1]
    out = torch.full((rows, hq, dh), 7.0, dtype=x.dtype, device="cuda")
    lse = torch.full((rows, hq), 7.0, device="cuda")
    dev.prefill(x, starts=torch.from_numpy(first).cuda(), max_new=max(new), window=window, sinks=sinks, out=out, lse=lse)
    ref = O.attend(c, q, first[:-1], new, dh ** -0.5, window, sinks)
    assert (out[first[-1]:] == 7).all() and (lse[first[-1]:] == 7).all(), "rows behind the last sequence"
    live = np.arange(rows) < first[-1]
    C.check_attention(ref, C.host(out), C.host(lse), c["dtype"], dh, rows=live)
    return ref, C.host(out), C.host(lse)


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_heads(heads, dtype):
    hq, hkv, dh = heads
    _say(f"prefill {dtype} {heads}")
    rng = np.random.default_rng(hq + dh)
    c = C.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[70, 1, 90], slots=96)
    _prefill(rng, c, [70, 1, 21], 0, 0, stride=1)


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("positions", [False, True])
def test_prefill_lengths(window, page, positions):
    _say(f"prefill lengths window={window} page={page} positions={positions}")
    rng = np.random.default_rng(page + 1)
    lens = [1, 17, 64, 65, 129, 200, 200, 40]
    new = [1, 17, 64, 30, 129, 1, 150, 0]
    c = C.make(rng, dtype="bf16", hq=6, hkv=2, dh=64, page=page, lens=lens, slots=208, positions=positions)
    _prefill(rng, c, new, *window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [(0, 0), (300, 3)], ids=str)
def test_prefill_long(dtype, window):
    _say(f"prefill long {dtype} {window}")
    rng = np.random.default_rng(77)
    c = C.make(rng, dtype=dtype, hq=2, hkv=1, dh=128, page=64, lens=[1100], slots=1100)
    _prefill(rng, c, [1037], *window)


def test_prefill_few_tokens_on_a_long_cache():
    _say("prefill 3 tokens over 6000 slots")
    rng = np.random.default_rng(78)
    c = C.make(rng, dtype="bf16", hq=7, hkv=1, dh=128, page=64, lens=[6001, 50], slots=6016)
    _prefill(rng, c, [3, 5], 0, 0)


def test_prefill_more_rows_than_slots_held():
    """Rows whose own slot lies before the cache's first see nothing."""
    _say("prefill more rows than slots")
    rng = np.random.default_rng(79)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[5, 0], slots=32)
    _prefill(rng, c, [9, 4], 0, 0)
    _prefill(rng, c, [9, 4], 2, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_pages_that_are_none(dtype):
    _say(f"prefill bad pages {dtype}")
    rng = np.random.default_rng(80)
    c = C.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[60, 40, 16], slots=64)
    c["table"][0, 1], c["table"][0, 3], c["table"][1, 0], c["table"][2, 0] = -1, 2 ** 31 - 1, 10 ** 6, -2 ** 31
    _prefill(rng, c, [60, 20, 16], 0, 0)
    _prefill(rng, c, [60, 20, 16], 9, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("window", [(0, 0), (20, 2)], ids=str)
def test_what_is_not_seen_changes_nothing(dtype, bad, window):
    """A row of infinities or NaN in K and V changes the queries that see it and
    no other."""
    _say(f"unseen {bad} {dtype} {window}")
    args = dict(dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[150], slots=160)
    c = C.make(np.random.default_rng(81), **args)
    _, clean, clean_lse = _prefill(np.random.default_rng(1), c, [150], *window)
    for slot in (90, 149):
        d = copy.deepcopy(c)
        p, r = O.row_of(d, 0, 0, slot)
        d["v"][p, :, r] = bad
        if slot == 90:
            d["k"][p, :, r] = bad
        q = C.queries(np.random.default_rng(1), d, 152)[:150]
        out, lse = C.on_gpu(d).prefill(C.to_gpu(q, dtype), window=window[0], sinks=window[1], lse=True)
        out, lse = C.host(out), C.host(lse)
        t = np.arange(150)
        sees = (t >= slot) & ((window[0] == 0) | (t - slot < window[0]))
        assert np.array_equal(out[~sees], clean[:150][~sees]) and np.array_equal(lse[~sees], clean_lse[:150][~sees])
        assert not np.isfinite(out[sees]).any()


def test_decode_sees_infinities_as_the_formula_does():
    _say("decode infinities")
    rng = np.random.default_rng(82)
    for dtype in ("bf16", "f32"):
        c = C.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[60, 60], slots=64)
        p, r = O.row_of(c, 0, 0, 50)
        c["v"][p, 0, r] = np.inf
        q = C.queries(rng, c, 2)
        out, lse = C.on_gpu(c).decode(C.to_gpu(q, dtype), lse=True)
        out = C.host(out)
        assert np.isposinf(out[0, :2]).all() and np.isfinite(out[0, 2:]).all() and np.isfinite(out[1]).all()
        assert np.isfinite(C.host(lse)).all()
        c["k"][p, 0, r] = np.nan
        out, lse = C.on_gpu(c).decode(C.to_gpu(q, dtype), lse=True)
        assert np.isnan(C.host(out)[0, :2]).all() and np.isnan(C.host(lse)[0, :2]).all()
        assert np.isfinite(C.host(out)[0, 2:]).all()


# --- eviction -----------------------------------------------------------------------
EVICTS = {
    "one_over": dict(lens=[65, 64, 3], slots=80, budget=64, sinks=4, recent=8),
    "half": dict(lens=[300, 151, 150], slots=304, budget=150, sinks=0, recent=0),
    "most": dict(lens=[300, 1000], slots=1008, budget=17, sinks=9, recent=8),
    "one_left": dict(lens=[50, 2, 1, 0], slots=64, budget=1, sinks=0, recent=0),
    "long": dict(lens=[5000, 4100], slots=5008, budget=4096, sinks=4, recent=100),
}


@pytest.mark.parametrize("case", list(EVICTS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
def test_evict(case, dtype, kind):
    a = dict(EVICTS[case])
    _say(f"evict {case} {dtype} {kind} {a}")
    budget, sinks, recent = a.pop("budget"), a.pop("sinks"), a.pop("recent")
    rng = np.random.default_rng(17)
    c = C.make(rng, dtype=dtype, hq=6, hkv=3, dh=32, page=16, positions=True, weights=True, **a)
    w = c["weights"]
    if kind == "ties":
        w[:] = rng.integers(0, 3, w.shape) * 0.5
    if kind == "odd":
        w[:] = rng.choice([0.0, -0.0, np.inf, -np.inf, np.nan, -1.0, 1e-40, 3.0], w.shape).astype(np.float32)
    dev = C.on_gpu(c)
    dev.evict(budget, sinks=sinks, recent=recent)
    O.evict(c, budget, sinks, recent)
    # (rows past the budget keep what they held in both)
    _compare_caches(c, dev)


@pytest.mark.parametrize("n,slots", [(8193, 8208), (30000, 65536), (66000, 66016)])
@pytest.mark.parametrize("kind", ["random", "ties", "near"])
def test_evict_long(n, slots, kind):
    """Caches longer than one block keeps keys for; weights that agree in their
    upper halves."""
    _say(f"evict long {n} of {slots} {kind}")
    rng = np.random.default_rng(n)
    c = C.make(rng, dtype="bf16", hq=2, hkv=1, dh=32, page=16, lens=[n], slots=slots, positions=True, weights=True)
    w = c["weights"]
    if kind == "ties":
        w[:] = np.where(rng.random(w.shape) < 0.7, 0.25, rng.random(w.shape).astype(np.float32))
    if kind == "near":
        w[:] = (1 + rng.integers(0, 1 << 15, w.shape) * 2.0 ** -23).astype(np.float32)
    dev = C.on_gpu(c)
    dev.evict(n // 3, sinks=4, recent=100)
    O.evict(c, n // 3, 4, 100)
    _compare_caches(c, dev)


def test_evict_pages_that_are_none():
    _say("evict bad pages")
    rng = np.random.default_rng(18)
    c = C.make(rng, dtype="bf16", hq=2, hkv=2, dh=64, page=16, lens=[60, 64], slots=64, positions=True, weights=True)
    c["table"][0, 1], c["table"][1, 3] = -1, 10 ** 6
    dev = C.on_gpu(c)
    dev.evict(30, sinks=1, recent=5)
    O.evict(c, 30, 1, 5)
    _compare_caches(c, dev)


# --- together -------------------------------------------------------------------------
def test_prompt_decode_and_eviction_together():
    """A prompt, then tokens one by one with weights added up and the cache cut
    back every few steps: what a bounded deployment runs."""
    _say("together")
    rng = np.random.default_rng(19)
    hq, hkv, dh, b, n = 8, 2, 64, 2, 45
    dev = C.B.KvCache.create(n_seq=b, slots=70, n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, dtype=torch.bfloat16,
                             page_size=16, evicts=True)
    c = {"dtype": "bf16", "hq": hq, "q_scale": 2.0, "k": np.zeros(tuple(dev.k_pages.shape)),
         "v": np.zeros(tuple(dev.v_pages.shape)), "table": dev.page_table.cpu().numpy(), "lens": np.zeros(b, np.int32),
         "seen": np.zeros(b, np.int32), "slot_pos": np.zeros(tuple(dev.slot_pos.shape), np.int32),
         "weights": np.zeros(tuple(dev.weights.shape))}
    for step in range(40):
        m = n if step == 0 else 1
        kv = C.rounded(rng.standard_normal((b * m, 2, hkv, dh)), "bf16")
        q = C.queries(rng, c, b * m)
        x, y = C.to_gpu(kv, "bf16"), C.to_gpu(q, "bf16")
        dev.append(x[:, 0], x[:, 1])
        O.append(c, kv[:, 0], kv[:, 1], [m] * b, [np.arange(i * m, (i + 1) * m) for i in range(b)])
        if step == 0:
            out, lse = dev.prefill(y, window=30, sinks=3, lse=True)
            ref = O.attend(c, q, [0, m], [m] * b, dh ** -0.5, 30, 3)
        else:
            out, lse = dev.decode(y, window=30, sinks=3, accumulate=True, lse=True)
            ref = O.attend(c, q, list(range(b)), [1] * b, dh ** -0.5, 30, 3)
            C.check_weights(ref, c["weights"], C.host(dev.weights), dh)
            c["weights"] = C.host(dev.weights)     # (their roundings would add up)
        C.check_attention(ref, C.host(out), C.host(lse), "bf16", dh)
        if step % 7 == 6:
            dev.evict(40, sinks=3, recent=5)
            O.evict(c, 40, 3, 5)
            _compare_caches(c, dev)
    assert c["lens"].max() <= 47 and c["seen"][0] == n + 39


def test_captured_steps_replay():
    """Append, decode with accumulation and eviction in one graph, replayed with
    eager work between, against the same calls made eagerly."""
    _say("graph")
    rng = np.random.default_rng(20)
    args = dict(dtype="bf16", hq=14, hkv=2, dh=128, page=16, lens=[300, 60], slots=320, positions=True, weights=True)
    a, b = C.on_gpu(C.make(np.random.default_rng(21), **args)), C.on_gpu(C.make(np.random.default_rng(21), **args))
    kv = torch.zeros((2, 2, 2, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 14, 128), dtype=torch.bfloat16, device="cuda")

    def step(cache):
        cache.append(kv[:, 0], kv[:, 1])
        out, lse = cache.decode(q, accumulate=True, lse=True)
        cache.evict(200, sinks=2, recent=9)
        return out, lse

    keep = [t.clone() for t in (a.lens, a.seen, a.slot_pos, a.weights, a.k_pages, a.v_pages)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a)
    for t, s in zip((a.lens, a.seen, a.slot_pos, a.weights, a.k_pages, a.v_pages), keep):
        t.copy_(s)
    for i in range(4):
        kv.copy_(torch.from_numpy(rng.standard_normal(kv.shape)).cuda())
        q.copy_(torch.from_numpy(rng.standard_normal(q.shape)).cuda())
        graph.replay()
        want = step(b)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
        for x, y in ((a.lens, b.lens), (a.seen, b.seen)):
            assert torch.equal(x, y), i
        n = int(b.lens.max())
        assert torch.equal(a.weights[..., :60], b.weights[..., :60]) and n == 200


def test_repeats_bit_for_bit_on_another_stream():
    _say("another stream")
    rng = np.random.default_rng(22)
    c = C.make(rng, dtype="bf16", hq=28, hkv=4, dh=128, page=64, lens=[2000, 700], slots=2048, weights=True)
    q = C.to_gpu(C.queries(rng, c, 2), "bf16")
    dev = C.on_gpu(c)
    w0 = dev.weights.clone()
    out, lse = dev.decode(q, accumulate=True, lse=True)
    w1 = dev.weights.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dev.weights.copy_(w0)
        out2, lse2 = dev.decode(q, accumulate=True, lse=True)
    side.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(w1, dev.weights)


# --- calls that a program may make and the cases above do not ---------------------------
def _unaligned(t):
    """The same values at an address that is a multiple of 4 bytes only."""
    x = torch.empty(t.numel() + 5, dtype=t.dtype, device=t.device)
    for skip in (1, 2, 3, 5):
        y = x[skip: skip + t.numel()]
        if y.data_ptr() % 8:
            break
    y.copy_(t.reshape(-1))
    return y.view(t.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_and_weights_at_any_address(dtype):
    """Prefill, decode, append and eviction with slot_pos and weights that are not
    16-byte aligned give what they give with aligned ones, bit for bit."""
    _say(f"unaligned {dtype}")
    rng = np.random.default_rng(30)
    c = C.make(rng, dtype=dtype, hq=6, hkv=3, dh=64, page=16, lens=[150, 33], slots=176, positions=True, weights=True)
    a, b = C.on_gpu(c), C.on_gpu(c)
    b = C.B.KvCache(b.k_pages, b.v_pages, b.page_table, b.lens, n_q_heads=6, seen=b.seen,
                    slot_pos=_unaligned(b.slot_pos), weights=_unaligned(b.weights))
    q = C.to_gpu(C.queries(rng, c, 40), dtype)
    kv = C.to_gpu(C.rounded(rng.standard_normal((2, 2, 3, 64)), dtype), dtype)
    got = []
    for x in (a, b):
        x.append(kv[:, 0], kv[:, 1])
        p = x.prefill(q, window=37, sinks=3, lse=True)
        d = x.decode(q[:2], window=37, sinks=3, accumulate=True, lse=True)
        x.evict(100, sinks=3, recent=20)
        got.append([*p, *d, x.slot_pos[0, :, :100], x.weights[0, :, :100], x.lens, x.seen])
    assert got[1][4].data_ptr() % 16 != 0
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [128, 256, 512, 1024])
def test_large_pages(dtype, page):
    _say(f"page {page} {dtype}")
    rng = np.random.default_rng(page)
    c = C.make(rng, dtype=dtype, hq=6, hkv=2, dh=64, page=page, lens=[1100, 2, page], slots=1100, weights=True)
    _decode(rng, c, 0, 0, accumulate=True)
    _prefill(rng, c, [130, 2, 5], 200, 3)


@pytest.mark.parametrize("scale", [0.0, -0.11, 0.5])
def test_scales(scale):
    """A scale of zero weighs every visible key alike; a negative one is a sign."""
    _say(f"scale {scale}")
    for dtype in ("bf16", "f32"):
        rng = np.random.default_rng(31)
        c = C.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[70, 20], slots=80)
        q = C.queries(rng, c, 10)
        dev, x = C.on_gpu(c), C.to_gpu(q, dtype)
        out, lse = dev.prefill(x, scale=scale, lse=True)
        C.check_attention(O.attend(c, q, [0, 5], [5, 5], scale), C.host(out), C.host(lse), dtype, 64)
        out, lse = dev.decode(x[:2], scale=scale, lse=True)
        C.check_attention(O.attend(c, q[:2], [0, 1], [1, 1], scale), C.host(out), C.host(lse), dtype, 64)


def test_most_heads():
    """256 query heads on one kv head and on 256."""
    for hq, hkv in ((256, 1), (256, 256)):
        _say(f"heads {hq} on {hkv}")
        rng = np.random.default_rng(hkv)
        c = C.make(rng, dtype="bf16", hq=hq, hkv=hkv, dh=32, page=16, lens=[40, 17], slots=48, weights=True)
        _decode(rng, c, 0, 0, accumulate=True)
        _prefill(rng, c, [3, 17], 9, 1)


@pytest.mark.parametrize("dtype,cap", [("bf16", 512), ("bf16", 528), ("f32", 256), ("f32", 272)])
@pytest.mark.parametrize("window", [(0, 0), (100, 3)], ids=str)
def test_decode_where_one_block_takes_a_sequence_and_just_past(dtype, cap, window):
    _say(f"decode {dtype} slots {cap} {window}")
    rng = np.random.default_rng(cap)
    c = C.make(rng, dtype=dtype, hq=6, hkv=2, dh=96, page=16, lens=[cap, cap - 1, cap - 16, 240, 1], slots=cap)
    _decode(rng, c, *window)


def test_prefill_of_many_blocks():
    """More blocks than are split over keys, in runs over heads and unlike sequences."""
    _say("prefill many blocks")
    rng = np.random.default_rng(32)
    lens = [700, 3, 650, 1, 333]
    c = C.make(rng, dtype="bf16", hq=28, hkv=4, dh=64, page=16, lens=lens, slots=704)
    _prefill(rng, c, lens, 0, 0)
    _prefill(rng, c, [600, 3, 649, 1, 0], 130, 4)


def test_append_of_few_and_many_tokens():
    for n in (15, 16, 17, 18):
        _say(f"append {n}")
        rng = np.random.default_rng(n)
        c = C.make(rng, dtype="bf16", hq=6, hkv=2, dh=32, page=16, lens=[10, 0, 60], slots=64, positions=True, weights=True)
        kv = C.rounded(rng.standard_normal((3 * n, 2, 2, 32)), "bf16")
        dev, x = C.on_gpu(c), C.to_gpu(kv, "bf16")
        dev.append(x[:, 0], x[:, 1])
        O.append(c, kv[:, 0], kv[:, 1], [n] * 3, [np.arange(i * n, (i + 1) * n) for i in range(3)])
        _compare_caches(c, dev)


def test_rows_past_max_new_are_not_taken():
    _say("rows past max_new")
    rng = np.random.default_rng(33)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[30, 40], slots=64)
    q = C.queries(rng, c, 20)
    starts = torch.tensor([2, 12, 20], dtype=torch.int32).cuda()      # 10 and 8 rows, of which 5 each
    dev, x = C.on_gpu(c), C.to_gpu(q, "bf16")
    out, lse = torch.full_like(x, 7.0), torch.full((20, 4), 7.0, device="cuda")
    dev.prefill(x, starts=starts, max_new=5, out=out, lse=lse)
    took = np.r_[2:7, 12:17]
    left = np.setdiff1d(np.arange(20), took)
    C.check_attention(O.attend(c, q, [2, 12], [5, 5], 0.125), C.host(out), C.host(lse), "bf16", 64,
                      rows=np.isin(np.arange(20), took))
    assert (out[left] == 7).all() and (lse[left] == 7).all()


def test_offsets_past_32_bits():
    """Pages beyond 2^31 elements: every call gives what it gives on low pages."""
    _say("far pages")
    hkv, page, dh, b, per = 8, 64, 128, 2, 5
    far = (1 << 31) // (hkv * page * dh) + 7             # the first of the far pages
    shape = (hkv, page, dh)
    big = [torch.empty((far + b * per, *shape), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    low = [torch.randn((b * per, *shape), device="cuda").bfloat16() for _ in "kv"]
    for x, y in zip(big, low):
        x[far:] = y
    got = []
    g = torch.Generator("cuda").manual_seed(5)
    q = 2 * torch.randn((20, 32, dh), generator=g, device="cuda").bfloat16()
    kv = torch.randn((20, 2, hkv, dh), generator=g, device="cuda").bfloat16()
    w = torch.rand((b, hkv, per * page), generator=g, device="cuda")
    for pages, base in ((low, 0), (big, far)):
        table = (base + torch.arange(b * per, device="cuda", dtype=torch.int32)).view(b, per)
        pos = torch.arange(per * page, device="cuda", dtype=torch.int32).expand(b, hkv, -1).contiguous()
        lens = torch.tensor([300, 130], dtype=torch.int32, device="cuda")
        dev = C.B.KvCache(*pages, table, lens, n_q_heads=32, seen=lens.clone(), slot_pos=pos, weights=w.clone())
        dev.append(kv[:, 0], kv[:, 1])
        p = dev.prefill(q, lse=True)
        d = dev.decode(q[:2], accumulate=True, lse=True)
        dev.evict(150, sinks=2, recent=5)
        e = dev.decode(q[:2], lse=True)
        got.append([*p, *d, *e, dev.weights[..., :140], dev.slot_pos[..., :140], dev.lens,
                    pages[0][base:base + b * per], pages[1][base:base + b * per]])
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_prefill_replays(dtype):
    """A prefill split over keys and joined, and one that is not, in one graph with
    the appending of their rows."""
    _say(f"graph prefill {dtype}")
    rng = np.random.default_rng(34)
    c = C.make(rng, dtype=dtype, hq=14, hkv=2, dh=64, page=16, lens=[700, 90], slots=720)
    dev = C.on_gpu(c)
    kv = torch.zeros((6, 2, 2, 64), dtype=C.DT[dtype], device="cuda")
    q = torch.zeros((6, 14, 64), dtype=C.DT[dtype], device="cuda")
    keep = dev.lens.clone()

    def step():
        dev.lens.copy_(keep)
        dev.append(kv[:, 0], kv[:, 1])
        return [*dev.prefill(q, lse=True), *dev.prefill(q[:2], window=9, sinks=1, lse=True)]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        kv.copy_(torch.from_numpy(rng.standard_normal(kv.shape)).cuda())
        q.copy_(torch.from_numpy(rng.standard_normal(q.shape)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in got]
        for x, y in zip(held, step()):
            assert torch.equal(x, y), i


def test_two_calls_at_once():
    """Attention calls on one cache on two streams, each with scratch memory of its own."""
    _say("two streams")
    rng = np.random.default_rng(35)
    c = C.make(rng, dtype="bf16", hq=28, hkv=4, dh=128, page=64, lens=[3000, 2500], slots=3008)
    dev = C.on_gpu(c)
    q = [C.to_gpu(C.queries(rng, c, 12), "bf16") for _ in range(2)]
    want = [[*dev.prefill(x, lse=True), *dev.decode(x[:2], lse=True)] for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in q]
    for _ in range(5):
        got = []
        for x, s in zip(q, streams):
            with torch.cuda.stream(s):
                got.append([*dev.prefill(x, lse=True), *dev.decode(x[:2], lse=True)])
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert all(torch.equal(u, v) for u, v in zip(x, y))


def test_a_query_does_not_depend_on_its_neighbours():
    """Bit for bit: large logits of other queries of a block change nothing."""
    _say("neighbours")
    rng = np.random.default_rng(36)
    for dtype in ("bf16", "f32"):
        c = C.make(rng, dtype=dtype, hq=4, hkv=1, dh=64, page=16, lens=[400], slots=400)
        dev, q = C.on_gpu(c), C.queries(rng, c, 60)
        out, lse = dev.prefill(C.to_gpu(q, dtype), lse=True)
        loud = q.copy()
        loud[1::2] *= 40 * np.linspace(0, 1, 30)[:, None, None]
        loud = C.rounded(loud, dtype)
        out2, lse2 = dev.prefill(C.to_gpu(loud, dtype), lse=True)
        assert torch.equal(out[::2], out2[::2]) and torch.equal(lse[::2], lse2[::2])
        assert not torch.equal(lse[1::2], lse2[1::2])


def test_wrapper_refusals_on_the_device():
    _say("refusals")
    rng = np.random.default_rng(37)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[30, 40], slots=64)
    dev = C.on_gpu(c)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = q[:, :2].contiguous()
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    for call, what in (
            (lambda: dev.decode(q.float()), "torch.bfloat16"),
            (lambda: dev.decode(q[:1]), "one token for each"),
            (lambda: dev.decode(q.cpu()), "device"),
            (lambda: dev.decode(q.transpose(0, 1).contiguous().transpose(0, 1)), "in one run"),
            (lambda: dev.decode(q[:1].expand(2, 4, 64)), "in one run"),
            (lambda: dev.decode(q, out=torch.empty_like(q, dtype=torch.float32)), "out must"),
            (lambda: dev.decode(q, lse=torch.empty((2, 4), device="cuda").bfloat16()), "lse must"),
            (lambda: dev.prefill(q, starts=starts), "max_new"),
            (lambda: dev.prefill(q, starts=starts.long(), max_new=1), "starts"),
            (lambda: dev.prefill(q[:, :2]), "tokens"),
            (lambda: dev.append(k, k[:1]), "tokens"),
            (lambda: dev.append(k, k, src=starts[None]), "src"),
            (lambda: dev.append(k, k, starts=starts, max_new=1, src=starts[:2, None].contiguous()), "both"),
            (lambda: dev.append(torch.cat([k, k[:1]]), torch.cat([k, k[:1]])), "same number")):
        with pytest.raises(ValueError, match=what):
            call()
    for call, what in ((lambda: dev.decode(q, accumulate=True), "weights"),
                       (lambda: dev.evict(20), "needs"),
                       (lambda: dev.decode(q, window=-1), "window"),
                       (lambda: dev.prefill(q, starts=starts, max_new=65), "max_new")):
        with pytest.raises(RuntimeError, match=what):
            call()
    assert dev.lens.tolist() == [30, 40]


@pytest.mark.parametrize("kind", ["odd", "one_value", "protected"])
def test_evict_of_long_caches_of_unlike_lengths(kind):
    """Sequences below the budget, of one slice and of many in one call; infinities
    and NaN; one weight for all; more protected rows than the budget."""
    _say(f"evict unlike {kind}")
    rng = np.random.default_rng(38)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=32, page=16, lens=[100, 4097, 12300, 3000, 0], slots=12304,
               positions=True, weights=True)
    w = c["weights"]
    if kind == "odd":
        w[:] = rng.choice([0.0, -0.0, np.inf, -np.inf, np.nan, -1.0, 1e-40, 3.0], w.shape).astype(np.float32)
    if kind == "one_value":
        w[:] = 0.125
    if kind == "protected":
        c["slot_pos"][2, 1, ::2] = 0
    dev = C.on_gpu(c)
    dev.evict(3000, sinks=2, recent=900)
    O.evict(c, 3000, 2, 900)
    _compare_caches(c, dev)


def test_pruned_prompt_into_the_cache():
    """prune, compact, the prefix layer's rows at the kept positions into the cache,
    attention over them and one answer token: what a deployment runs."""
    from paper_2608_02134_amd import binding as B
    from paper_2608_02134_amd import synth

    from .gpu_run import run
    _say("prune, compact, append, prefill, decode")
    prob = synth.make_problem("tiny", grid=(1, 8, 8), t=4, k=16)
    outs, pr = run(prob, torch, trace=False)
    before, n, after, hq, hkv, dh = 5, 64, 9, 8, 2, 64
    length = before + n + after
    idx = torch.from_numpy(np.ascontiguousarray(outs[0]["out_idx"].astype(np.int32)[None])).cuda()
    pos = torch.zeros((1, length, 3), dtype=torch.int32, device="cuda")
    _, keep, _, _ = B.compact_sequence(idx, before, n, seq_pos=pos)
    rng = np.random.default_rng(39)
    kv = C.rounded(rng.standard_normal((2, length, hkv, dh)), "bf16")
    k, v = C.to_gpu(kv, "bf16")
    cache = B.KvCache.create(n_seq=1, slots=64, n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, dtype=torch.bfloat16,
                             page_size=16)
    cache.append(k, v, src=keep)
    kept = keep.shape[1]
    assert cache.lens.tolist() == [kept]
    for x, pages in zip(B.gather_rows([k[None], v[None]], keep), (cache.k_pages, cache.v_pages)):
        held = pages.permute(0, 2, 1, 3).reshape(-1, hkv, dh)[:kept]
        assert torch.equal(held, x[0])
    c = {"dtype": "bf16", "hq": hq, "q_scale": 2.0, "k": C.host(cache.k_pages), "v": C.host(cache.v_pages),
         "table": cache.page_table.cpu().numpy(), "lens": np.array([kept], np.int32)}
    q = C.queries(rng, c, kept)
    out, lse = cache.prefill(C.to_gpu(q, "bf16"), lse=True)
    C.check_attention(O.attend(c, q, [0], [kept], dh ** -0.5), C.host(out), C.host(lse), "bf16", dh)
    new = C.rounded(rng.standard_normal((2, 1, hkv, dh)), "bf16")
    cache.append(*C.to_gpu(new, "bf16"))
    O.append(c, new[0], new[1], [1], [np.arange(1)])
    out, lse = cache.decode(C.to_gpu(q[:1], "bf16"), lse=True)
    C.check_attention(O.attend(c, q[:1], [0], [1], dh ** -0.5), C.host(out), C.host(lse), "bf16", dh)
    pr.close()


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 3), (2 ** 31 - 1, 2 ** 31 - 1), (70, 2 ** 31 - 1), (1, 64), (1, 0)])
@pytest.mark.parametrize("positions", [False, True])
def test_windows_and_first_tokens_of_any_size(window, sinks, positions):
    """Also with queries whose own slot lies before the cache's first."""
    _say(f"window {window} sinks {sinks} positions {positions}")
    for dtype in ("bf16", "f32"):
        rng = np.random.default_rng(40)
        c = C.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[5, 300, 64], slots=304, positions=positions)
        _prefill(rng, c, [9, 200, 64], window, sinks)
        _decode(rng, c, window, sinks)


# --- infinities and NaN at every head size ------------------------------------------------
def _bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


@pytest.mark.parametrize("dh", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("held,new,window", [(200, 200, (0, 0)), (200, 200, (20, 2)), (607, 37, (0, 0)), (607, 37, (300, 2))],
                         ids=str)
def test_unseen_infinities_at_every_head_size(dh, dtype, held, new, window):
    """A value row of infinities or NaN at the first, a late and the last row of a
    key tile (of 32 or 64), in the first, the last or all dims: queries that do
    not see it keep their bits, the others those of the other dims.  A whole
    prompt, and a few tokens over a longer cache (keys split and joined)."""
    _say(f"unseen at {dh} {dtype} {held} {new} {window}")
    rng = np.random.default_rng(dh)
    c = C.make(rng, dtype=dtype, hq=6, hkv=2, dh=dh, page=16, lens=[held], slots=608)
    dev, q = C.on_gpu(c), C.to_gpu(C.queries(rng, c, new), dtype)
    clean, clean_lse = dev.prefill(q, window=window[0], sinks=window[1], lse=True)
    assert torch.isfinite(clean).all()
    t = np.arange(held - new, held)
    edge = held - new if new < held else 96       # a tile that some queries see in part
    slots = [edge // 32 * 32 + x for x in (0, 26, 30, 31, 32)] + [held - 1]
    if window[0] and new < held:
        slots += [t[0] - window[0] + 1 + x for x in (0, 16, 17)]      # 271, 287 and 288: the windows begin here
    for i, slot in enumerate(slots):
        p, r = O.row_of(c, 0, 0, slot)
        dims = [slice(0, 8), slice(dh - 8, dh), slice(0, dh)][i % 3]
        keep = dev.v_pages[p, :, r].clone()
        dev.v_pages[p, :, r, dims] = (np.nan, np.inf, -np.inf)[i // 2 % 3]
        out, lse = dev.prefill(q, window=window[0], sinks=window[1], lse=True)
        dev.v_pages[p, :, r] = keep
        sees = torch.from_numpy((t >= slot) & ((window[0] == 0) | (t - slot < window[0]))).cuda()
        assert torch.equal(lse, clean_lse), slot
        assert torch.equal(_bits(out[~sees]), _bits(clean[~sees])), (slot, dims)
        other = torch.ones(dh, dtype=torch.bool, device="cuda")
        other[dims] = False
        assert torch.equal(_bits(out[..., other]), _bits(clean[..., other])), (slot, dims)
        assert not torch.isfinite(out[sees][..., ~other]).any(), (slot, dims)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("slots", [48, 1600])
def test_weights_of_unseen_slots_stay_where_a_seen_key_is_nan(dtype, slots):
    """The query's own weights are NaN then; slots outside the window, on pages that
    are none and in other sequences gain nothing."""
    _say(f"weights beside NaN {dtype} {slots}")
    rng = np.random.default_rng(41)
    n = slots - 5
    c = C.make(rng, dtype=dtype, hq=6, hkv=2, dh=64, page=16, lens=[n, n, 20], slots=slots, weights=True)
    window, sinks = 21, 3
    p, r = O.row_of(c, 0, 1, n - 2)
    c["k"][p, 1, r] = np.nan                     # kv head 1 of sequence 0, seen
    p, r = O.row_of(c, 1, 0, n - 24)
    c["k"][p, :, r] = np.nan                     # sequence 1, outside the window
    c["table"][0, (n - 20) // 16] = -1           # some of the window's slots
    q = C.queries(rng, c, 3)
    dev = C.on_gpu(c)
    _, lse = dev.decode(C.to_gpu(q, dtype), window=window, sinks=sinks, accumulate=True, lse=True)
    ref = O.attend(c, q, [0, 1, 2], [1, 1, 1], 0.125, window, sinks)
    got, seen = C.host(dev.weights), np.zeros(c["weights"].shape, bool)
    for b, m in enumerate(c["lens"]):
        s = np.arange(m)
        held = np.array([O.row_of(c, b, 0, x) is not None for x in s])
        seen[b, :, :m] = held & ((m - 1 - s < window) | (s < sinks))
    assert np.array_equal(got[~seen], c["weights"][~seen])
    assert np.isnan(got[0, 1][seen[0, 1]]).all() and np.isnan(C.host(lse)[0, 3:]).all()
    ok = np.ones(3 * 2, bool)
    ok[1] = False                                # (every other sequence and kv head)
    rel = C.weight_error(ref, 64).reshape(3, 2, -1).max(2)
    want = c["weights"] + ref["probs"]
    for b, h in np.argwhere(ok.reshape(3, 2)):
        assert (np.abs(got[b, h] - want[b, h]) <= ref["probs"][b, h] * rel[b, h] + 40 * C.U32 * np.abs(want[b, h])).all(), (b, h)


@pytest.mark.parametrize("scale", [0.0, 2e-32, -2e-32, 1e-44])
def test_scales_far_below_one(scale):
    """Products far above one: only the scale makes logits of them, and a scale of
    zero still weighs every visible key alike."""
    _say(f"scale {scale}")
    for dtype in ("bf16", "f32"):
        rng = np.random.default_rng(42)
        c = C.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[300, 20], slots=304)
        used = np.isfinite(c["k"])
        c["k"][used] = C.rounded(c["k"][used] * 1e15, dtype)
        c["q_scale"] = 1e15
        q = C.queries(rng, c, 10)
        scale32 = float(np.float32(scale))
        dev, x = C.on_gpu(c), C.to_gpu(q, dtype)
        for window, sinks in ((0, 0), (9, 2)):
            out, lse = dev.prefill(x, scale=scale, window=window, sinks=sinks, lse=True)
            ref = O.attend(c, q, [0, 5], [5, 5], scale32, window, sinks)
            C.check_attention(ref, C.host(out), C.host(lse), dtype, 64)
            out, lse = dev.decode(x[:2], scale=scale, window=window, sinks=sinks, lse=True)
            C.check_attention(O.attend(c, q[:2], [0, 1], [1, 1], scale32, window, sinks), C.host(out), C.host(lse), dtype, 64)


@pytest.mark.parametrize("n_seq,hkv,new", [(65535, 16, 1), (2048, 8, 4), (257, 24, 2)])
def test_prefill_of_many_short_sequences(n_seq, hkv, new):
    """More heads than row blocks by far: 2^20 of them, and a few thousand.  The
    sequences' pages are shared, which reading allows."""
    _say(f"prefill of {n_seq} sequences, {hkv} heads, {new} tokens")
    g = torch.Generator("cuda").manual_seed(47)
    n_pages, page, dh = 40, 16, 32
    k, v = (torch.randn((n_pages, hkv, page, dh), generator=g, device="cuda").bfloat16() for _ in "kv")
    table = torch.randint(0, n_pages, (n_seq, 1), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.randint(0, page + 1, (n_seq,), generator=g, device="cuda", dtype=torch.int32)
    q = (2 * torch.randn((n_seq * new, hkv, dh), generator=g, device="cuda")).bfloat16()
    dev = C.B.KvCache(k, v, table, lens, n_q_heads=hkv)
    out, lse = dev.prefill(q, lse=True)
    slot, f64 = torch.arange(page, device="cuda"), torch.float64
    for b0 in range(0, n_seq, 4096):
        ids, n = table[b0:b0 + 4096, 0].long(), lens[b0:b0 + 4096]
        rows = slice(b0 * new, (b0 + len(ids)) * new)
        kk, vv = (x[ids].to(f64) for x in (k, v))                       # [b][h][slot][d]
        qq = q[rows].view(len(ids), new, hkv, dh).to(f64)
        ref = {x: [] for x in ("out", "lse", "mass", "size", "most")}
        for i in range(new):
            prod = qq[:, i, :, None] * kk                               # [b][h][slot][d]
            see = (slot <= (n - new + i)[:, None])[:, None].expand(-1, hkv, -1)
            x = torch.where(see, prod.sum(-1) * dh ** -0.5, -np.inf)
            m = x.amax(-1, keepdim=True).clamp(min=-1e300)
            e = torch.exp(x - m)
            total = e.sum(-1, keepdim=True)
            a = e / total.clamp(min=1e-300)
            ref["lse"].append((m + torch.log(total))[..., 0])
            ref["out"].append((a[..., None] * vv).sum(2))
            ref["mass"].append((a[..., None] * vv.abs()).sum(2))
            ref["size"].append(torch.where(see, prod.abs().sum(-1) * dh ** -0.5, 0).amax(-1))
            ref["most"].append(see.sum(-1).double())
        ref = {x: torch.stack(y, 1).flatten(0, 1).cpu().numpy() for x, y in ref.items()}
        ref["lse"][ref["most"] == 0] = -np.inf
        C.check_attention(ref, C.host(out[rows]), C.host(lse[rows]), "bf16", dh)


def test_sequences_that_share_the_pages_of_a_common_prefix():
    """Three sequences begin with the same two whole pages; what is appended to is
    each one's own."""
    _say("shared prefix")
    rng = np.random.default_rng(45)
    c = C.make(rng, dtype="bf16", hq=8, hkv=2, dh=64, page=16, lens=[32, 32, 32], slots=80)
    c["table"][1, :2] = c["table"][2, :2] = c["table"][0, :2]
    q, m = C.queries(rng, c, 3 * 21), 21
    kv = C.rounded(rng.standard_normal((3 * m, 2, 2, 64)), "bf16")
    dev, x = C.on_gpu(c), C.to_gpu(kv, "bf16")
    shared = dev.k_pages[dev.page_table[0, :2].long()].clone()
    dev.append(x[:, 0], x[:, 1])
    O.append(c, kv[:, 0], kv[:, 1], [m] * 3, [np.arange(i * m, (i + 1) * m) for i in range(3)])
    _compare_caches(c, dev)
    assert torch.equal(shared, dev.k_pages[dev.page_table[0, :2].long()])
    out, lse = dev.prefill(C.to_gpu(q, "bf16"), lse=True)
    C.check_attention(O.attend(c, q, [0, m, 2 * m], [m] * 3, 0.125), C.host(out), C.host(lse), "bf16", 64)
    out, lse = dev.decode(C.to_gpu(q[:3], "bf16"), lse=True)
    C.check_attention(O.attend(c, q[:3], [0, 1, 2], [1] * 3, 0.125), C.host(out), C.host(lse), "bf16", 64)


def test_captured_steps_replay_the_whole_state():
    """Append, windowed decode with accumulation and eviction in one graph: after
    each replay every weight, position and row of the live slots and all pages are
    those of the same calls made eagerly."""
    _say("graph, whole state")
    rng = np.random.default_rng(43)
    args = dict(dtype="bf16", hq=14, hkv=2, dh=128, page=16, lens=[300, 60], slots=320, positions=True, weights=True)
    a, b = C.on_gpu(C.make(np.random.default_rng(44), **args)), C.on_gpu(C.make(np.random.default_rng(44), **args))
    kv = torch.zeros((2, 2, 2, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 14, 128), dtype=torch.bfloat16, device="cuda")

    def step(cache):
        cache.append(kv[:, 0], kv[:, 1])
        out, lse = cache.decode(q, window=150, sinks=2, accumulate=True, lse=True)
        cache.evict(200, sinks=2, recent=9)
        return out, lse

    state = lambda x: (x.lens, x.seen, x.slot_pos, x.weights, x.k_pages, x.v_pages)  # noqa: E731
    keep = [t.clone() for t in state(a)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a)
    for t, s in zip(state(a), keep):
        t.copy_(s)
    for i in range(5):
        kv.copy_(torch.from_numpy(rng.standard_normal(kv.shape)).cuda())
        q.copy_(torch.from_numpy(rng.standard_normal(q.shape)).cuda())
        graph.replay()
        want = step(b)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
        assert torch.equal(a.lens, b.lens) and torch.equal(a.seen, b.seen), i
        assert a.lens.tolist() == [200, 61 + i]
        for seq, n in enumerate(a.lens.tolist()):
            assert torch.equal(a.weights[seq, :, :n], b.weights[seq, :, :n]), (i, seq)
            assert torch.equal(a.slot_pos[seq, :, :n], b.slot_pos[seq, :, :n]), (i, seq)
        for x, y in ((a.k_pages, b.k_pages), (a.v_pages, b.v_pages)):
            assert torch.equal(_bits(x), _bits(y)), i     # (slots that hold nothing are NaN in both)


@pytest.mark.parametrize("bits", [0x7FFF, -1, 0x7F81, -127, 0x7FC0, -64])
@pytest.mark.parametrize("where", ["q", "k", "v"])
def test_a_nan_of_any_payload_stays_one(bits, where):
    """bf16 NaN with all, one and the usual mantissa bits, of either sign, quiet or
    not: the outputs that it reaches are NaN, in one block and joined from splits."""
    _say(f"NaN {bits & 0xFFFF:#x} in {where}")
    nan = torch.tensor(bits, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    assert torch.isnan(nan)
    for slots in (64, 3008):
        rng = np.random.default_rng(48)
        c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[slots, slots - 7], slots=slots)
        q = C.to_gpu(C.queries(rng, c, 2), "bf16")
        dev = C.on_gpu(c)
        if where == "q":
            q[0, 1] = nan
            hit = [(0, 1)]
        else:
            p, r = O.row_of(c, 0, 0, slots // 2)
            {"k": dev.k_pages, "v": dev.v_pages}[where][p, 0, r] = nan
            hit = [(0, 0), (0, 1)]
        for out, lse in (dev.prefill(q, lse=True), dev.decode(q, lse=True)):
            for b in range(2):
                for h in range(4):
                    bad = torch.isnan(out[b, h])
                    assert bad.all() if (b, h) in hit else not bad.any(), (slots, b, h)
                    assert torch.isnan(lse[b, h]).item() == ((b, h) in hit and where != "v"), (slots, b, h)


def test_max_new_beside_src():
    """It was taken for the columns of src whatever it said."""
    _say("max_new beside src")
    c = C.make(np.random.default_rng(49), dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[30, 40], slots=64)
    dev = C.on_gpu(c)
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    src = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    for n in (0, 1, 3):
        with pytest.raises(ValueError, match="max_new"):
            dev.append(k, k, src=src, max_new=n)
    assert dev.lens.tolist() == [30, 40]
    dev.append(k, k, src=src, max_new=2)
    assert dev.lens.tolist() == [32, 42]


@pytest.mark.parametrize("seed", range(16))
def test_infinities_and_nan_where_the_formula_has_them(seed):
    """Random layouts with a few value rows of infinities and NaN: each output is
    the infinity or NaN of the formula or within the bounds, in prefill and decode."""
    rng = np.random.default_rng(1000 + seed)
    dtype, dh, page = ("bf16", "f32")[seed % 2], 32 * (seed // 2 + 1), int(2 ** rng.integers(4, 8))
    hkv, b, slots = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(40, 500))
    hq, lens = hkv * int(rng.integers(1, 9)), [int(n) for n in rng.integers(1, slots + 1, b)]
    window, sinks = (0, 0) if rng.random() < 0.3 else (int(rng.integers(1, slots)), int(rng.integers(0, 9)))
    c = C.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=page, lens=lens, slots=slots, positions=bool(rng.integers(2)),
               q_scale=1.0)
    _say(f"infinities {dtype} {hq} on {hkv} of {dh}, {lens}, window {window}")
    for bad in (np.nan, np.inf, -np.inf, np.inf):
        seq, d = int(rng.integers(b)), int(rng.integers(dh))
        p, r = O.row_of(c, seq, 0, int(rng.integers(lens[seq])))
        c["v"][p, int(rng.integers(hkv)), r, d:d + 20] = bad
    new = [min(n, 50) for n in lens]
    first = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q, dev = C.queries(rng, c, int(first[-1])), C.on_gpu(c)
    x = C.to_gpu(q, dtype)
    calls = [(dev.prefill(x, starts=torch.from_numpy(first).cuda(), max_new=max(new), window=window, sinks=sinks, lse=True),
              O.attend(c, q, first[:-1], new, dh ** -0.5, window, sinks)),
             (dev.decode(x[:b], window=window, sinks=sinks, lse=True),
              O.attend(c, q[:b], list(range(b)), [1] * b, dh ** -0.5, window, sinks))]
    for (out, lse), ref in calls:
        out, odd = C.host(out), ~np.isfinite(ref["out"])
        assert np.array_equal(out[odd], ref["out"][odd], equal_nan=True)
        ref["out"][odd] = ref["mass"][odd] = out[odd] = 0
        C.check_attention(ref, out, C.host(lse), dtype, dh)
