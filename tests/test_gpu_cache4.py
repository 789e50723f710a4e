"""Caches of 4 bits on the GPU against their oracle: appended codes and scales
bit for bit, values exactly, attention within bounds derived from its roundings."""
import numpy as np
import pytest

from oracle import cache4_oracle as O4
from oracle import cache_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2608_02134_amd import binding as B  # noqa: E402

from . import cache4_cases as C4  # noqa: E402
from . import cache_cases as C  # noqa: E402

DIMS = [32, 64, 96, 128, 160, 192, 224, 256]


def _say(what):
    print(f"\n[case] {what}", flush=True)


def _starts(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()


# --- append and read -----------------------------------------------------------------
def odd_rows(rng, shape, dtype):
    """Blocks of many sizes: normal ones, of all zeros, with ties, below and at the
    least scale, near the largest numbers, with infinities and NaN."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-20, 20, shape[:-1] + (1,))
    blocks = x.reshape(-1, 32)
    kind = rng.integers(0, 12, len(blocks))
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 0.0, 0.5, -0.0])
    for i, k in enumerate(kind):
        if k == 0:
            blocks[i] = 0
        elif k == 1:
            blocks[i] = grid[rng.integers(0, 12, 32)] * rng.choice([-1, 1], 32) * 2.0 ** rng.integers(-30, 30)
        elif k == 2:
            blocks[i] *= 2.0 ** -126 / np.abs(blocks[i]).max()
        elif k == 3:
            blocks[i] *= 2.0 ** -130 / np.abs(blocks[i]).max()
        elif k == 4:
            blocks[i] *= 3.38e38 / np.abs(blocks[i]).max()
        elif k == 5:
            blocks[i, rng.integers(0, 32)] = rng.choice([np.inf, -np.inf, np.nan])
    return C.rounded(blocks.reshape(shape), dtype)


@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("few", [True, False])
def test_append(dh, dtype, few):
    """Ragged rows of strided tensors; every other byte of the cache stays."""
    _say(f"append4 dh={dh} {dtype} few={few}")
    rng = np.random.default_rng(dh)
    new = [1, 0, 7] if few else [18, 0, 25]
    c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[15, 3, 20], slots=48)
    kv = odd_rows(rng, (sum(new), 5, dh), dtype)
    dev, x = C4.on_gpu(c), C.to_gpu(kv, dtype)
    dev.append(x[:, 0:2], x[:, 3:5], starts=_starts(new), max_new=max(new))
    first = np.concatenate([[0], np.cumsum(new)])
    O4.append4(c, kv[:, 0:2].astype(np.float32), kv[:, 3:5].astype(np.float32), new,
               [np.arange(first[b], first[b + 1]) for b in range(3)])
    C4.compare(c, dev)
    k, v = dev.read(sum(new), starts=_starts(new), max_new=max(new))
    seq = np.repeat(np.arange(3), new)
    slot = np.concatenate([np.arange(c["lens"][b] - new[b], c["lens"][b]) for b in range(3)])
    for got, name in ((k, "k"), (v, "v")):
        want = np.array([c[name][c["table"][b][s // 16], :, s % 16] for b, s in zip(seq, slot)])
        assert C.same(C.host(got), want)


@pytest.mark.parametrize("dh,rot,interleaved,sections", [(128, 128, False, (16, 24, 24)), (64, 32, True, None),
                                                         (96, 48, False, None), (160, 160, True, (40, 20, 20)),
                                                         (256, 128, False, None), (32, 16, True, None)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 21])
def test_append_turned(dh, rot, interleaved, sections, dtype, n):
    """Keys are turned in fp32 and quantised without a rounding between; rows
    picked by src, with queries."""
    _say(f"append4 rotary dh={dh} rot={rot} {dtype} n={n}")
    rng = np.random.default_rng(dh + rot + n)
    c = C4.make(rng, dtype=dtype, hq=6, hkv=2, dh=dh, page=32, lens=[9, 40], slots=64)
    r = C4.rotary(rng, 70, rot, interleaved=interleaved, sections=sections)
    per = n + 11
    qkv = C.rounded(rng.standard_normal((2 * per, 10, dh)), dtype)
    pos = rng.integers(0, 70, (2 * per, 3) if sections else 2 * per).astype(np.int32)
    src = np.stack([rng.permutation(per)[:n] for _ in range(2)]).astype(np.int32)
    dev, x = C4.on_gpu(c), C.to_gpu(qkv, dtype)
    got = dev.append_rotary(x[:, 6:8], x[:, 8:], C4.rotary_on_gpu(r), pos=torch.from_numpy(pos).cuda(), q=x[:, :6],
                            src=torch.from_numpy(src).cuda())
    turned = O4.turn(qkv[:, :8], r, pos)
    rows = [src[0].astype(int), per + src[1].astype(int)]
    O4.append4(c, turned[:, 6:], qkv[:, 8:].astype(np.float32), [n, n], rows)
    C4.compare(c, dev)
    assert C.same(C.host(got), C.rounded(turned[:, :6], dtype)[np.concatenate(rows)])


@pytest.mark.parametrize("n", [5, 30])
def test_append_without_pos_and_past_the_capacity(n):
    _say(f"append4 past the capacity n={n}")
    rng = np.random.default_rng(n)
    c = C4.make(rng, dtype="bf16", hq=2, hkv=2, dh=64, page=16, lens=[46, 20, 48], slots=48)
    c["table"][1, 1] = -1
    r = C4.rotary(rng, 200, 64)
    qkv = C.rounded(rng.standard_normal((3 * n, 6, 64)), "bf16")
    dev, x = C4.on_gpu(c), C.to_gpu(qkv, "bf16")
    got = dev.append_rotary(x[:, 2:4], x[:, 4:], C4.rotary_on_gpu(r), q=x[:, :2])
    pos = np.concatenate([first + np.arange(n) for first in (46, 20, 48)])
    turned = O4.turn(qkv[:, :4], r, pos)
    rows = [b * n + np.arange(n) for b in range(3)]
    O4.append4(c, turned[:, 2:], qkv[:, 4:].astype(np.float32), [n] * 3, rows)
    C4.compare(c, dev)
    assert C.same(C.host(got), C.rounded(turned[:, :2], "bf16"))


def test_read_where_there_are_no_rows():
    """Slots before the first and on pages that are none read as zeros; rows of no
    sequence stay; blocks of NaN read as NaN, the least scale as it is."""
    _say("read4")
    rng = np.random.default_rng(8)
    c = C4.make(rng, dtype="f32", hq=2, hkv=2, dh=96, page=16, lens=[5, 40, 0], slots=48)
    c["table"][1, 1] = 10 ** 6
    c["k_scales"][c["table"][1, 2], :, 3] = [255, 0, 254]
    C4.refresh(c)
    dev = C4.on_gpu(c)
    starts = torch.tensor([0, 20, 50, 51], dtype=torch.int32).cuda()
    k, v = (torch.full((60, 2, 96), 9.0, device="cuda") for _ in "kv")
    B._check(B.gmc_cache4_read(dev.desc, 60, starts.data_ptr(), 30, k.data_ptr(), v.data_ptr(),
                               torch.cuda.current_stream().cuda_stream), "read")
    for got, name in ((k, "k"), (v, "v")):
        want = np.full((60, 2, 96), 9.0)
        for b, (lo, n) in enumerate(((0, 20), (20, 30), (50, 1))):
            for i in range(n):
                s = c["lens"][b] - n + i
                at = None if s < 0 else O.row_of(c, b, 0, s)
                want[lo + i] = 0 if at is None else c[name][at[0], :, at[1]]
        assert C.same(C.host(got), C.rounded(want, "f32"))   # 2 to 6 times 2^127 are above the largest number: infinite


# --- attention --------------------------------------------------------------------------
HEADS = [(28, 4, 128), (8, 2, 64), (6, 6, 96), (16, 1, 256), (4, 4, 32), (32, 1, 128), (5, 1, 160), (40, 2, 64),
         (3, 1, 192), (2, 2, 224)]
WINDOWS = [(0, 0), (1, 0), (37, 4), (64, 0), (5, 100), (2 ** 31 - 1, 3), (70, 2 ** 31 - 1)]


def _decode(rng, c, window, sinks, stride=0, scale=None):
    b, hq, dh = len(c["lens"]), c["hq"], c["k"].shape[3]
    q = C.queries(rng, c, b)
    dev, x = C4.on_gpu(c), C.to_gpu(q, c["dtype"])
    if stride:
        wide = torch.full((b, hq + 3, dh), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, 1:hq + 1] = x
        x = wide[:, 1:hq + 1]
    out, lse = dev.decode(x, window=window, sinks=sinks, lse=True, scale=scale)
    ref = O.attend(c, q, list(range(b)), [1] * b, dh ** -0.5 if scale is None else scale, window, sinks)
    C4.check_attention(ref, C.host(out), C.host(lse), c["dtype"], dh, True)


def _prefill(rng, c, new, window, sinks, stride=0, scale=None, extra=0):
    hq, dh, total = c["hq"], c["k"].shape[3], sum(new)
    q = C.queries(rng, c, total + extra)
    dev, x = C4.on_gpu(c), C.to_gpu(q, c["dtype"])
    if stride:
        wide = torch.full((total + extra, hq + 3, dh), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, 1:hq + 1] = x
        x = wide[:, 1:hq + 1]
    out = torch.full((total + extra, hq, dh), 5.0, dtype=C.DT[c["dtype"]], device="cuda")
    lse = torch.full((total + extra, hq), 5.0, device="cuda")
    dev.prefill(x, starts=_starts(new), max_new=max(new), window=window, sinks=sinks, scale=scale, out=out, lse=lse)
    first = np.concatenate([[0], np.cumsum(new)])
    ref = O.attend(c, q, first, new, dh ** -0.5 if scale is None else scale, window, sinks)
    C4.check_attention(ref, C.host(out), C.host(lse), c["dtype"], dh, False)
    assert (out[total:] == 5).all() and (lse[total:] == 5).all()


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_heads(heads, dtype):
    hq, hkv, dh = heads
    _say(f"decode4 {dtype} {heads}")
    rng = np.random.default_rng(hq * dh)
    c = C4.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[1, 200, 33], slots=208)
    _decode(rng, c, 0, 0, stride=1)
    c = C4.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[1300, 600], slots=1328)   # split and joined
    _decode(rng, c, 0, 0)


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("page", [16, 64])
def test_decode_lengths(window, page):
    _say(f"decode4 lengths window={window} page={page}")
    rng = np.random.default_rng(page)
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 300]
    _decode(rng, C4.make(rng, dtype="bf16", hq=14, hkv=2, dh=64, page=page, lens=lens, slots=300), *window)
    _decode(rng, C4.make(rng, dtype="f32", hq=2, hkv=2, dh=96, page=page, lens=lens, slots=700), *window)


@pytest.mark.parametrize("dtype,n", [("bf16", 4999), ("f32", 3001), ("bf16", 9000)])
@pytest.mark.parametrize("window", [(0, 0), (700, 5), (100, 7), (1, 640), (4000, 2 ** 31 - 1)], ids=str)
def test_decode_long(dtype, n, window):
    _say(f"decode4 long {dtype} n={n} window={window}")
    rng = np.random.default_rng(n)
    _decode(rng, C4.make(rng, dtype=dtype, hq=7, hkv=1, dh=128, page=128, lens=[n, n // 3], slots=n), *window)


@pytest.mark.parametrize("n_seq,hkv,slots", [(16, 4, 1040), (64, 4, 330), (200, 4, 300), (256, 3, 160)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_many_sequences(n_seq, hkv, slots, dtype):
    """One block a head, of eight waves or four, and split ones, by the heads there are."""
    _say(f"decode4 of {n_seq} sequences, {hkv} heads, {slots} slots {dtype}")
    rng = np.random.default_rng(n_seq)
    lens = rng.integers(0, slots + 1, n_seq).tolist()
    _decode(rng, C4.make(rng, dtype=dtype, hq=hkv, hkv=hkv, dh=32, page=16, lens=lens, slots=slots), 0, 0)
    _decode(rng, C4.make(rng, dtype=dtype, hq=hkv, hkv=hkv, dh=32, page=16, lens=lens, slots=slots), 70, 3)


def test_decode_length_past_the_table_and_below_zero():
    _say("decode4 odd lengths")
    rng = np.random.default_rng(11)
    c = C4.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[64, 64], slots=64)
    c["lens"] = np.array([10 ** 9, -5], np.int32)
    _decode(rng, c, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [(0, 0), (9, 2)], ids=str)
def test_pages_that_are_none(dtype, window):
    _say(f"4 bits, pages that are none {dtype} {window}")
    rng = np.random.default_rng(6)
    c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[100, 90, 32], slots=112)
    c["table"][0, 2], c["table"][0, 3], c["table"][1, :], c["table"][2, 1] = -1, 10 ** 6, -7, 2 ** 31 - 1
    _decode(rng, c, *window)
    _prefill(rng, c, [40, 3, 17], *window)


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_heads(heads, dtype):
    hq, hkv, dh = heads
    _say(f"prefill4 {dtype} {heads}")
    rng = np.random.default_rng(hq * dh + 1)
    c = C4.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[1, 150, 70], slots=160)
    _prefill(rng, c, [1, 40, 70], 0, 0, stride=1, extra=3)
    c = C4.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[700], slots=704)      # split and joined
    _prefill(rng, c, [5], 0, 0)


@pytest.mark.parametrize("window", WINDOWS, ids=str)
@pytest.mark.parametrize("page", [16, 64])
def test_prefill_lengths(window, page):
    _say(f"prefill4 lengths window={window} page={page}")
    rng = np.random.default_rng(page + 1)
    lens, new = [0, 1, 17, 64, 65, 129, 200], [0, 1, 17, 3, 65, 64, 1]
    c = C4.make(rng, dtype="bf16", hq=14, hkv=2, dh=64, page=page, lens=lens, slots=208)
    _prefill(rng, c, new, *window)
    c = C4.make(rng, dtype="f32", hq=3, hkv=1, dh=96, page=page, lens=lens, slots=208)
    _prefill(rng, c, new, *window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [(0, 0), (300, 3)], ids=str)
def test_prefill_long(dtype, window):
    _say(f"prefill4 long {dtype} {window}")
    rng = np.random.default_rng(31)
    c = C4.make(rng, dtype=dtype, hq=2, hkv=1, dh=128, page=64, lens=[900, 611], slots=900)
    _prefill(rng, c, [900, 333], *window)


@pytest.mark.parametrize("window", [(1, 0), (130, 4), (700, 1), (3900, 9), (9, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)], ids=str)
def test_prefill_window_of_long_caches(window):
    """Windows far below the capacity: fewer splits than the scratch memory is for."""
    _say(f"prefill4 windows of long caches {window}")
    rng = np.random.default_rng(32)
    c = C4.make(rng, dtype="bf16", hq=7, hkv=1, dh=64, page=64, lens=[4100, 2055], slots=5000)
    _prefill(rng, c, [43, 9], *window)


def test_prefill_more_rows_than_slots_held():
    """Queries that stand before the first slot see nothing."""
    _say("prefill4 before the first slot")
    rng = np.random.default_rng(33)
    c = C4.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[3, 0], slots=48)
    _prefill(rng, c, [9, 5], 0, 0)
    _prefill(rng, c, [9, 5], 2, 1)


@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [(0, 0), (20, 2)], ids=str)
def test_blocks_of_nan(dh, dtype, window):
    """A block that reads as NaN reaches the queries that see it, in all elements
    where it is K's and in its 32 where it is V's, and no other."""
    _say(f"4 bits, blocks of NaN dh={dh} {dtype} {window}")
    rng = np.random.default_rng(dh)
    c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[100, 77], slots=112)
    last = dh // 32 - 1
    for b, h, s, blk, x in ((0, 0, 70, 0, "v"), (0, 1, 90, last, "v"), (1, 0, 60, last, "k"), (1, 1, 5, 0, "v")):
        c[x + "_scales"][c["table"][b][s // 16], h, s % 16, blk] = 255
    C4.refresh(c)
    new = [60, 77]
    q = C.queries(rng, c, sum(new))
    dev = C4.on_gpu(c)
    out, lse = dev.prefill(C.to_gpu(q, dtype), starts=_starts(new), max_new=77, window=window[0], sinks=window[1],
                           lse=True)
    _nan_as_formula(c, q, [0, 60], new, out, lse, window, dtype)
    out, lse = dev.decode(C.to_gpu(q[:2], dtype), window=window[0], sinks=window[1], lse=True)
    _nan_as_formula(c, q[:2], [0, 1], [1, 1], out, lse, window, dtype, decode=True)


def _nan_as_formula(c, q, first, new, out, lse, window, dtype, decode=False):
    dh = c["k"].shape[3]
    with np.errstate(invalid="ignore"):
        ref = O.attend(c, q, first, new, dh ** -0.5, *window)
    out, lse = C.host(out), C.host(lse)
    assert np.array_equal(np.isnan(out), np.isnan(ref["out"])) and np.array_equal(np.isnan(lse), np.isnan(ref["lse"]))
    assert np.isnan(ref["out"]).any() or window[0]
    # rows without NaN among their keys: as without
    clean = ~np.isnan(ref["out"]).any((1, 2)) & ~np.isnan(ref["lse"]).any(1)
    if clean.any():
        C4.check_attention(ref, out, lse, dtype, dh, decode) if clean.all() else \
            C4.check_attention({k: (v[clean] if k != "probs" else v) for k, v in ref.items()}, out[clean], lse[clean],
                               dtype, dh, decode)


@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [(0, 0), (20, 2)], ids=str)
def test_values_that_overflow(dh, dtype, window):
    """Scales that nothing appends, whose larger codes are infinite: an infinity
    among V's values reaches the queries that see it with its sign, and no other."""
    _say(f"4 bits, infinite values dh={dh} {dtype} {window}")
    rng = np.random.default_rng(dh + 1)
    c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[100, 77], slots=112)
    where = [(0, 0, 70, 0, 5), (0, 1, 90, dh - 1, 14), (1, 0, 60, dh // 2, 7), (1, 1, 5, 3, 12)]
    for b, h, s, d, code in where:
        at = c["table"][b][s // 16], h, s % 16
        c["v_codes"][at][32 * (d // 32):32 * (d // 32) + 32] = 0
        c["v_codes"][at + (d,)] = code
        c["v_scales"][at + (d // 32,)] = 254
    C4.refresh(c)
    with np.errstate(over="ignore"):
        c["v"] = c["v"].astype(np.float32).astype(np.float64)    # infinite where the type has no such number
    assert np.isinf(c["v"]).sum() == 4
    new = [60, 77]
    q = C.queries(rng, c, sum(new))
    dev = C4.on_gpu(c)
    got = (dev.prefill(C.to_gpu(q, dtype), starts=_starts(new), max_new=77, window=window[0], sinks=window[1]),
           dev.decode(C.to_gpu(q[:2], dtype), window=window[0], sinks=window[1]))
    for out, first, n in zip(got, ([0, 60], [0, 1]), (new, [1, 1])):
        with np.errstate(invalid="ignore"):
            want = O.attend(c, q[: sum(n)], first, n, dh ** -0.5, *window)["out"]
        out = C.host(out)
        assert np.array_equal(np.isfinite(out), np.isfinite(want))
        assert C.same(out[~np.isfinite(want)], want[~np.isfinite(want)])


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_that_are_not_finite(bad, dtype):
    """They change no other row; their own rows are NaN."""
    _say(f"4 bits, query of {bad} {dtype}")
    rng = np.random.default_rng(3)
    c = C4.make(rng, dtype=dtype, hq=6, hkv=2, dh=64, page=16, lens=[90, 40], slots=96)
    q = C.queries(rng, c, 2)
    dev, x = C4.on_gpu(c), C.to_gpu(q, dtype)
    want = dev.decode(x), dev.prefill(x)
    x[0, 1, 7], x[1, 3, 9] = bad, bad
    for got, w in zip((dev.decode(x), dev.prefill(x)), want):
        other = torch.ones(2, 6, dtype=torch.bool, device="cuda")
        other[0, 1], other[1, 3] = False, False
        assert torch.equal(got[other], w[other]) and torch.isnan(got[~other]).all()


@pytest.mark.parametrize("scale", [0.0, -0.11, 0.5, 2e-32])
def test_scales(scale):
    _say(f"4 bits, scale {scale}")
    rng = np.random.default_rng(4)
    for dtype in ("bf16", "f32"):
        c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[100, 40], slots=112)
        _decode(rng, c, 0, 0, scale=scale)
        _prefill(rng, c, [30, 40], 0, 0, scale=scale)


@pytest.mark.parametrize("page", [128, 256, 512, 1024])
def test_large_pages(page):
    _say(f"4 bits, pages of {page}")
    rng = np.random.default_rng(page)
    for dtype in ("bf16", "f32"):
        c = C4.make(rng, dtype=dtype, hq=3, hkv=1, dh=32, page=page, lens=[page + 40, page - 1, 2 * page], slots=2 * page,
                    spare=1)
        _decode(rng, c, 0, 0)
        _prefill(rng, c, [50, 7, 1], 100, 3)


@pytest.mark.parametrize("cap", [512, 528])
@pytest.mark.parametrize("window", [(0, 0), (100, 3)], ids=str)
def test_decode_where_one_block_takes_a_sequence_and_just_past(cap, window):
    _say(f"decode4 cap={cap}")
    rng = np.random.default_rng(cap)
    for dtype in ("bf16", "f32"):
        c = C4.make(rng, dtype=dtype, hq=7, hkv=1, dh=128, page=16, lens=[cap, cap - 17, 1, 0], slots=cap)
        _decode(rng, c, *window)


def test_scales_of_every_size():
    """Scales from the least to the largest that sums of fp32 hold."""
    _say("4 bits, scales of every size")
    rng = np.random.default_rng(14)
    for low, high in ((0, 30), (1, 254), (100, 150)):
        for dtype in ("bf16", "f32"):
            c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=64, page=16, lens=[60, 33], slots=64)
            c["k_scales"][c["k_scales"] != 255] = 125
            live = c["v_scales"] != 255
            c["v_scales"][live] = rng.integers(low, high, live.sum())
            C4.refresh(c)
            if high == 254:     # products and sums stay finite
                c["v_codes"][(c["v_scales"] > 240).repeat(32, -1)] = 0
                C4.refresh(c)
            _decode(rng, c, 0, 0) if low else _decode_tiny(rng, c)


def _decode_tiny(rng, c):
    """Values below the least normal number: the weights times them, and their
    rounding, fall out of the type's range by up to its least step."""
    q = C.queries(rng, c, 2)
    out = C.host(C4.on_gpu(c).decode(C.to_gpu(q, c["dtype"])))
    ref = O.attend(c, q, [0, 1], [1, 1], 64 ** -0.5)["out"]
    assert (np.abs(out - ref) <= 2.0 ** -7 * np.abs(ref).max() + 2.0 ** -126).all()


# --- together and beside each other -----------------------------------------------------------
def test_prompt_and_answer_together():
    """A kept prompt's rows turned into 4 bits, attended over, then tokens one by
    one: each call as the oracle has it over the values that the cache holds."""
    _say("4 bits, prompt and answer")
    rng = np.random.default_rng(50)
    hq, hkv, dh, per, n = 14, 2, 128, 60, 35
    r = C4.rotary(rng, 200, dh, sections=(16, 24, 24))
    dev, rot = B.KvCache4.create(n_seq=2, slots=60, n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, dtype=torch.bfloat16,
                                 page_size=16), C4.rotary_on_gpu(r)
    c = {"dtype": "bf16", "hq": hq, "table": dev.page_table.cpu().numpy(), "lens": np.zeros(2, np.int32)}
    for x in "kv":
        c[x + "_codes"] = np.zeros((8, hkv, 16, dh), np.uint8)
        c[x + "_scales"] = np.zeros((8, hkv, 16, dh // 32), np.uint8)
    C4.refresh(c)
    qkv = C.rounded(rng.standard_normal((2 * per, hq + 2 * hkv, dh)), "bf16")
    pos = rng.integers(0, 200, (2 * per, 3)).astype(np.int32)
    src = np.stack([np.sort(rng.permutation(per)[:n]) for _ in range(2)]).astype(np.int32)
    x = C.to_gpu(qkv, "bf16")
    q = dev.append_rotary(x[:, hq:hq + hkv], x[:, hq + hkv:], rot, pos=torch.from_numpy(pos).cuda(), q=x[:, :hq],
                          src=torch.from_numpy(src).cuda())
    out, lse = dev.prefill(q, window=20, sinks=2, lse=True)
    turned = O4.turn(qkv[:, :hq + hkv], r, pos)
    rows = [src[0].astype(int), per + src[1].astype(int)]
    O4.append4(c, turned[:, hq:], qkv[:, hq + hkv:].astype(np.float32), [n, n], rows)
    C4.compare(c, dev, fill=0)
    tq = C.rounded(turned[:, :hq], "bf16")[np.concatenate(rows)]
    assert C.same(C.host(q), tq)
    C4.check_attention(O.attend(c, tq, [0, n], [n, n], dh ** -0.5, 20, 2), C.host(out), C.host(lse), "bf16", dh, False)
    for step in range(3):
        qkv = C.rounded(rng.standard_normal((2, hq + 2 * hkv, dh)), "bf16")
        x = C.to_gpu(qkv, "bf16")
        q = dev.append_rotary(x[:, hq:hq + hkv], x[:, hq + hkv:], rot, q=x[:, :hq])
        out, lse = dev.decode(q, lse=True)
        turned = O4.turn(qkv[:, :hq + hkv], r, c["lens"].astype(int))
        O4.append4(c, turned[:, hq:], qkv[:, hq + hkv:].astype(np.float32), [1, 1], [[0], [1]])
        C4.compare(c, dev, fill=0)
        tq = C.rounded(turned[:, :hq], "bf16")
        C4.check_attention(O.attend(c, tq, [0, 1], [1, 1], dh ** -0.5), C.host(out), C.host(lse), "bf16", dh, True)
    k, v = dev.read(max_new=n + 3)
    full = B.KvCache.create(n_seq=2, slots=60, n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, dtype=torch.bfloat16)
    full.append(k, v)
    a, b = full.decode(q, lse=True), (out, lse)
    # the same values in pages of the type: the same products, differently ordered sums
    assert torch.allclose(a[1], b[1], rtol=0, atol=1e-4) and (a[0].float() - b[0].float()).abs().max() <= 2 ** -6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps_replay(dtype):
    """Append with rotation, decode and prefill, split and not, in one graph,
    replayed on another stream with eager work between."""
    _say(f"4 bits graph {dtype}")
    rng = np.random.default_rng(60)
    args = dict(dtype=dtype, hq=14, hkv=2, dh=64, page=16, lens=[700, 90], slots=720)
    a, b = (C4.on_gpu(C4.make(np.random.default_rng(61), **args)) for _ in range(2))
    rot = C4.rotary_on_gpu(C4.rotary(rng, 800, 64))
    qkv = torch.zeros((6, 18, 64), dtype=C.DT[dtype], device="cuda")
    keep = a.lens.clone()

    def step(cache):
        cache.lens.copy_(keep)
        q = cache.append_rotary(qkv[:, 14:16], qkv[:, 16:], rot, q=qkv[:, :14])
        return [q, *cache.prefill(q, lse=True), *cache.prefill(q[:2], window=9, sinks=1, lse=True),
                *cache.decode(q[:2], lse=True), *cache.read(max_new=3)]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a)
    for i in range(4):
        qkv.copy_(torch.from_numpy(rng.standard_normal(qkv.shape)).cuda())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        want = step(b)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), i
        for name in ("k_codes", "v_codes", "k_scales", "v_scales", "lens"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (name, i)


def test_two_calls_at_once():
    """Calls on one cache on two streams, each with scratch memory of its own."""
    _say("4 bits, two streams")
    rng = np.random.default_rng(35)
    c = C4.make(rng, dtype="bf16", hq=28, hkv=4, dh=128, page=64, lens=[3000, 2500], slots=3008)
    dev = C4.on_gpu(c)
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
        for g, w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))


def test_a_query_does_not_depend_on_its_neighbours():
    _say("4 bits, neighbours")
    rng = np.random.default_rng(36)
    c = C4.make(rng, dtype="bf16", hq=28, hkv=4, dh=128, page=64, lens=[300, 300], slots=320)
    dev = C4.on_gpu(c)
    q = C.to_gpu(C.queries(rng, c, 40), "bf16")
    want = dev.prefill(q)
    q2 = q * 3
    q2[7], q2[31] = q[7], q[31]
    got = dev.prefill(q2)
    assert torch.equal(got[7], want[7]) and torch.equal(got[31], want[31])


def test_offsets_past_32_bits():
    """Pages whose codes lie beyond 2^32 bytes."""
    _say("4 bits, far pages")
    rng = np.random.default_rng(70)
    hkv, page, dh = 2, 64, 128
    n_pages = (1 << 32) // (hkv * page * dh // 2) + 40
    dev = [torch.zeros((n_pages, hkv, page, n), dtype=torch.uint8, device="cuda") for n in (64, 64, 4, 4)]
    table = torch.tensor([[n_pages - 1, n_pages - 2, n_pages - 3, 0]], dtype=torch.int32, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    far = B.KvCache4(*dev, table, lens, n_q_heads=4, dtype=torch.bfloat16)
    near = B.KvCache4.create(n_seq=1, slots=256, n_q_heads=4, n_kv_heads=hkv, head_dim=dh, dtype=torch.bfloat16)
    x = C.to_gpu(C.rounded(rng.standard_normal((150, 8, dh)), "bf16"), "bf16")
    for cache in (far, near):
        cache.append(x[:, 4:6], x[:, 6:])
    got, want = ([*c.prefill(x[:, :4], lse=True), *c.decode(x[-1:, :4], lse=True), *c.read(max_new=150)] for c in (far, near))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not far.k_codes[1: n_pages - 3].any() and not far.v_codes[1: n_pages - 3].any()


def test_sequences_that_share_pages():
    _say("4 bits, shared pages")
    rng = np.random.default_rng(71)
    c = C4.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[48, 48, 48], slots=64)
    c["table"][1, :2], c["table"][2, :3] = c["table"][0, :2], c["table"][0, :3]
    for x in "kv":
        c[x + "_scales"][c[x + "_scales"] == 255] = 125
    C4.refresh(c)
    c["lens"] = np.array([48, 40, 48], np.int32)
    _decode(rng, c, 0, 0)
    _prefill(rng, c, [10, 30, 48], 0, 0)


@pytest.mark.parametrize("n_seq,hkv,new", [(65535, 8, 1), (300, 24, 2), (65535, 1, 11)])
def test_many_sequences(n_seq, hkv, new):
    """As many sequences as a call takes: every one's rows as one sequence alone has them."""
    _say(f"4 bits, {n_seq} sequences")
    rng = np.random.default_rng(n_seq)
    rows = C.to_gpu(C.rounded(rng.standard_normal((new, 3 * hkv, 32)), "bf16"), "bf16")
    made = lambda n: B.KvCache4.create(n_seq=n, slots=16, n_q_heads=hkv, n_kv_heads=hkv, head_dim=32,  # noqa: E731
                                       dtype=torch.bfloat16, page_size=16)
    rot = C4.rotary_on_gpu(C4.rotary(rng, 16, 32))
    got = []
    for n in (1, n_seq):
        cache, x = made(n), rows.repeat(n, 1, 1)
        q = cache.append_rotary(x[:, hkv:2 * hkv], x[:, 2 * hkv:], rot, q=x[:, :hkv])
        out = [q, cache.prefill(q), *cache.read(max_new=new)]
        got.append([y.view(n, new, hkv, 32) for y in out] + [cache.decode(q.view(n, new, hkv, 32)[:, 0].contiguous())])
    for one, many in zip(*got):
        assert torch.equal(many, one.expand_as(many))


def test_wrapper_on_the_device():
    _say("4 bits, refusals")
    rng = np.random.default_rng(1)
    c = C4.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[20, 5], slots=32)
    dev = C4.on_gpu(c)
    x = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError, match="keeps its rows"):
        dev.evict(10)
    with pytest.raises(ValueError, match="one token"):
        dev.decode(x[:3])
    with pytest.raises(ValueError, match="q must"):
        dev.prefill(x.float())
    with pytest.raises(ValueError, match="max_new"):
        dev.read()
    with pytest.raises(ValueError, match="rows"):
        dev.read(5, max_new=2)
    with pytest.raises(ValueError, match="rows"):
        dev.read(starts=_starts([1, 1]), max_new=1)
    with pytest.raises(ValueError, match="at least 1"):
        dev.read(0, starts=_starts([1, 1]), max_new=1)
    with pytest.raises(Exception, match="max_new"):
        dev.append(x.repeat(20, 1, 1)[:, :2], x.repeat(20, 1, 1)[:, 2:])
    before = dev.lens.clone()
    assert torch.equal(dev.lens, before)
    f32 = C4.on_gpu({**c, "dtype": "f32"})
    out = f32.decode(x[:2].float())
    assert out.dtype == torch.float32


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("below", [70, 75, 80, 87])
@pytest.mark.parametrize("slots,one,other", [(208, 3, 5), (208, 3, 150), (1328, 40, 1100), (1328, 900, 700)])
def test_infinite_values_of_small_weights(dtype, below, slots, one, other):
    """An infinite value on a key whose logit is `below` under the largest, so that its
    weight is small but no less than 2^-126: no part of that weight may vanish."""
    _say(f"4 bits, infinite values of small weights {dtype} {below} {slots} {one} {other}")
    rng = np.random.default_rng(below)
    n, dh = slots - 8, 96
    c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[n], slots=slots)
    row = lambda s: (c["table"][0][s // 16], slice(None), s % 16)  # noqa: E731
    for s in range(n):
        c["k_codes"][row(s)] = 0
    # products with queries of one: `below` for the other key, 0 for all besides
    c["k_codes"][row(other)][:, :below] = 2
    c["k_scales"][row(other)] = 127
    d = {0: (5, 7, np.inf), 1: (70, 15, -np.inf)}       # of each kv head: dimension, code, what it reads as
    for h, (at, code, _) in d.items():
        page, _, r = row(one)
        c["v_codes"][page, h, r, 32 * (at // 32):32 * (at // 32) + 32] = 0
        c["v_codes"][page, h, r, at] = code
        c["v_scales"][page, h, r, at // 32] = 254
    C4.refresh(c)
    q = C.to_gpu(np.ones((1, 4, dh)), dtype)
    dev = C4.on_gpu(c)
    want = np.repeat(c["v"][row(other)], 2, 0)[None]
    for what, out in (("decode", dev.decode(q, scale=1.0)), ("prefill", dev.prefill(q, scale=1.0))):
        out = C.host(out)
        for h in range(4):
            at, _, inf = d[h // 2]
            assert out[0, h, at] == inf, (what, h, out[0, h, at])
            rest = np.arange(dh) != at
            # the weight of `other` is 1 but for roundings of weight, product, quotient and
            # output; what the rest add is below 1400 e^-70 6
            tol = (3 * C.UBF if dtype == "bf16" else 16 * C.U32) * np.abs(want[0, h]) + 1e-26
            assert (np.abs(out[0, h] - want[0, h]) <= tol)[rest].all(), (what, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 160, 224])
def test_keys_that_overflow(dh, dtype):
    """An infinity among K's values makes an infinite logit with the product's sign:
    the key is not seen where that is negative, the row is NaN where it is positive."""
    _say(f"4 bits, infinite keys dh={dh} {dtype}")
    rng = np.random.default_rng(dh + 2)
    c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[100, 77], slots=112)
    for b, h, s, at, code in ((0, 0, 70, 5, 15), (1, 1, 50, dh - 1, 7)):
        page, r = c["table"][b][s // 16], s % 16
        c["k_codes"][page, h, r, 32 * (at // 32):32 * (at // 32) + 32] = 0
        c["k_codes"][page, h, r, at] = code
        c["k_scales"][page, h, r, at // 32] = 254
    C4.refresh(c)
    with np.errstate(over="ignore"):
        c["k"] = c["k"].astype(np.float32).astype(np.float64)
    new = [60, 60]
    # few bits, so that an fp32 query is one bf16 alone; no zeros
    q = rng.choice([-2.0, -1.5, -0.5, 0.5, 1.0, 1.75], (sum(new), 4, dh))
    dev = C4.on_gpu(c)
    x = C.to_gpu(q, dtype)
    for (out, lse), first, n, decode in ((dev.prefill(x, lse=True), [0, 60], new, False),
                                         (dev.decode(x[[59, 119]], lse=True), [0, 1], [1, 1], True)):
        rows = q if not decode else q[[59, 119]]
        with np.errstate(invalid="ignore"):
            ref = O.attend(c, rows, first, n, dh ** -0.5)
        _finite_as_formula(ref, C.host(out), C.host(lse), dtype, dh, decode)


def _finite_as_formula(ref, out, lse, dtype, dh, decode):
    """NaN where the formula has it and the other elements within C4.check_attention's
    bounds, element by element.  (Sizes of infinite products bound nothing: as of the others.)"""
    assert np.array_equal(np.isnan(out), np.isnan(ref["out"])) and np.array_equal(np.isnan(lse), np.isnan(ref["lse"]))
    assert np.isfinite(ref["out"]).any() and np.isnan(ref["out"]).any()
    _elements(ref, out, lse, dtype, dh, decode)


def _elements(ref, out, lse, dtype, dh, decode, lost=0.0):
    """C4.check_attention's bounds for each element that is finite, `lost` beside them."""
    terms = 3 if dtype == "f32" else 2 if decode else 1
    size = np.where(np.isfinite(ref["size"]), ref["size"], np.nanmax(ref["size"][np.isfinite(ref["size"])]))
    rel = C.weight_error({"size": size, "most": ref["most"] * terms}, dh if dtype == "bf16" else dh * terms)
    live, seen = np.isfinite(ref["out"]), np.isfinite(ref["lse"])
    step = C.UBF * 1.01 if dtype == "bf16" else 0.0
    with np.errstate(invalid="ignore"):
        tol = ref["mass"] * (rel[..., None] + step) + (step + C.U32) * np.abs(ref["out"]) + lost
        assert (np.abs(out - ref["out"]) <= tol)[live].all()
        assert (np.abs(lse - ref["lse"]) <= rel + 2 * C.U32 * np.abs(ref["lse"]))[seen].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 96, 160, 256])
def test_elements_beside_blocks_of_nan(dh, dtype):
    """What is beside a NaN - other blocks of its row, other heads, other tokens - is
    as the formula has it, element by element."""
    _say(f"4 bits, beside blocks of NaN dh={dh} {dtype}")
    rng = np.random.default_rng(dh + 3)
    c = C4.make(rng, dtype=dtype, hq=6, hkv=3, dh=dh, page=16, lens=[100, 77], slots=112)
    for b, h, s, blk, x in ((0, 0, 70, 0, "v"), (0, 1, 90, dh // 32 - 1, "v"), (1, 0, 60, 1, "k"), (1, 2, 5, 0, "v")):
        c[x + "_scales"][c["table"][b][s // 16], h, s % 16, blk] = 255
    C4.refresh(c)
    new = [60, 77]
    q = C.queries(rng, c, sum(new))
    dev, x = C4.on_gpu(c), C.to_gpu(q, dtype)
    for window in ((0, 0), (20, 2)):
        for (out, lse), first, n, rows in ((dev.prefill(x, starts=_starts(new), max_new=77, window=window[0],
                                                        sinks=window[1], lse=True), [0, 60], new, q),
                                           (dev.decode(x[:2], window=window[0], sinks=window[1], lse=True), [0, 1],
                                            [1, 1], q[:2])):
            with np.errstate(invalid="ignore"):
                ref = O.attend(c, rows, first, n, dh ** -0.5, *window)
            _finite_as_formula(ref, C.host(out), C.host(lse), dtype, dh, len(rows) == 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 96, 256])
def test_prefill_over_scales_of_every_size(dh, dtype):
    """Scales of K and V from the least on; products and sums of fp32 hold the largest."""
    _say(f"prefill4, scales of every size dh={dh} {dtype}")
    rng = np.random.default_rng(15)
    new = [20, 33]
    for low, high in ((30, 240), (100, 150), (0, 30)):
        c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[60, 33], slots=64)
        live = c["v_scales"] != 255
        c["v_scales"][live] = rng.integers(low, high, live.sum())
        C4.refresh(c)
        if low:
            _prefill(rng, c, new, 0, 0)
            continue
        # below the least normal number: each of up to 60 keys' three products, the
        # quotient and the output may lose what is below 2^-126
        _both(rng, c, new, None, 182 * 2.0 ** -126, decode=False)
    for low, high, scale in ((0, 30, 1.0), (215, 222, 2.0 ** -95)):
        c = C4.make(rng, dtype=dtype, hq=4, hkv=2, dh=dh, page=16, lens=[60, 33], slots=64)
        live = c["k_scales"] != 255
        c["k_scales"][live] = rng.integers(low, high, live.sum())
        C4.refresh(c)
        # (logits lie up to 200 apart: a weight below 2^-126 of the largest is zero in 32
        # bits, so each of 60 keys may lose 2^-126 of a value of up to 6 / 2.  With heads of 256
        # all keys whose value is not zero are such ones for a query, whose element is 1e-39)
        _both(rng, c, new, scale, 180 * 2.0 ** -126)


def _both(rng, c, new, scale, lost, decode=True):
    """Prefill of the new tokens, and decode of other queries, within _elements' bounds."""
    dtype, dh = c["dtype"], c["k"].shape[3]
    scale = dh ** -0.5 if scale is None else scale
    first = np.concatenate([[0], np.cumsum(new)])
    q = C.queries(rng, c, first[-1])
    dev, x = C4.on_gpu(c), C.to_gpu(q, dtype)
    out, lse = dev.prefill(x, starts=_starts(new), max_new=max(new), scale=scale, lse=True)
    _elements(O.attend(c, q, first, new, scale), C.host(out), C.host(lse), dtype, dh, False, lost)
    if decode:
        q = C.queries(rng, c, 2)
        out, lse = dev.decode(C.to_gpu(q, dtype), scale=scale, lse=True)
        _elements(O.attend(c, q, [0, 1], [1, 1], scale), C.host(out), C.host(lse), dtype, dh, True, lost)


def test_refused_calls_leave_the_cache():
    _say("4 bits, what refused calls leave")
    rng = np.random.default_rng(16)
    c = C4.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[20, 5], slots=32)
    dev, full = C4.on_gpu(c), C.on_gpu(C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[20, 5], slots=32,
                                              positions=True, weights=True))
    held = ("lens", "page_table", "k_codes", "v_codes", "k_scales", "v_scales", "k_pages", "v_pages", "seen",
            "slot_pos", "weights")
    bits = lambda t: t.clone().view(torch.uint8)  # noqa: E731
    before = [{x: bits(getattr(cache, x)) for x in held if getattr(cache, x, None) is not None} for cache in (dev, full)]
    x = torch.ones((4, 8, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    r = C4.rotary_on_gpu(C4.rotary(rng, 8, 64))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    for cache in (dev, full):
        big = x.repeat(20, 1, 1)
        for refused in (lambda: cache.append(big[:, 4:6], big[:, 6:]), lambda: cache.append(k, v[:3]),
                        lambda: cache.append(k.float(), v), lambda: cache.append(k, v, starts=i32(3)),
                        lambda: cache.append(k, v, src=i32(2, 40)), lambda: cache.append(k, v, src=i32(3, 1)),
                        lambda: cache.append_rotary(k, v, r, pos=i32(3)),
                        lambda: cache.append_rotary(k, v, r, q=q[:3]),
                        lambda: cache.append_rotary(k, v, r, q=q, out=torch.empty_like(q)[:3]),
                        lambda: cache.append_rotary(k, v, B.Rotary.create(4, 128)),
                        lambda: cache.append_rotary(big[:, 4:6], big[:, 6:], r),
                        lambda: cache.decode(x[:3, :4]), lambda: cache.prefill(q.float()),
                        lambda: cache.evict(1, sinks=1, recent=1)):
            with pytest.raises((ValueError, TypeError, RuntimeError)):
                refused()
    torch.cuda.synchronize()
    for cache, was in zip((dev, full), before):
        for name, t in was.items():
            assert torch.equal(bits(getattr(cache, name)), t), name
