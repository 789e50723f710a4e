"""Appending with rotation on the GPU against the oracle, bit for bit, into pages
of the type; queries rotated by the same call."""
import copy

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


def _say(what):
    print(f"\n[case] {what}", flush=True)


def _compare(c, dev, what=("k_pages", "v_pages")):
    assert np.array_equal(dev.lens.cpu().numpy(), c["lens"])
    for x, name in zip("kv", what):
        assert C.same(C.host(getattr(dev, name)), c[x]), name
    if c.get("slot_pos") is not None:
        assert np.array_equal(dev.seen.cpu().numpy(), c["seen"])
        assert np.array_equal(dev.slot_pos.cpu().numpy(), c["slot_pos"])
    if c.get("weights") is not None:
        assert C.same(C.host(dev.weights), c["weights"])


def _starts(counts):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32).cuda()


def default_pos(c, counts, rows_of):
    """Each row's position where none are given: that of the slot it comes to."""
    pos = np.zeros(max(int(r.max()) for r in rows_of if len(r)) + 1, np.int64)
    for b, rows in enumerate(rows_of):
        first = c["seen"][b] if c.get("seen") is not None else O.held(c, b)
        pos[rows] = first + np.arange(len(rows))
    return pos


# heads, head_dim, rot_dim, pairs, sections
SHAPES = [((28, 4, 128), 128, False, (16, 24, 24)), ((28, 4, 128), 128, True, None), ((8, 2, 64), 32, True, (8, 4, 4)),
          ((4, 4, 32), 16, False, None), ((12, 12, 96), 48, False, (0, 16, 8)), ((12, 12, 96), 96, True, None),
          ((16, 1, 256), 256, False, (64, 32, 32)), ((5, 1, 160), 80, False, None), ((3, 1, 192), 64, False, None),
          ((2, 2, 224), 224, False, (4, 52, 56)), ((7, 7, 32), 32, False, None)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("few", [True, False])
def test_heads_and_tables(shape, dtype, few):
    """Ragged new tokens of strided rows, with positions, some out of the table."""
    (hq, hkv, dh), rot, interleaved, sections = shape
    _say(f"append_rotary {shape} {dtype} few={few}")
    rng = np.random.default_rng(hq * dh + rot)
    new = [1, 0, 5] if few else [19, 0, 33]
    c = C.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[15, 4, 30], slots=70, positions=True, weights=True)
    r = C4.rotary(rng, 50, rot, interleaved=interleaved, sections=sections)
    total = sum(new)
    qkv = C.rounded(rng.standard_normal((total, hq + 2 * hkv + 1, dh)), dtype)
    pos = rng.integers(-3, 60, (total, 3) if sections else total).astype(np.int32)
    dev, x = C.on_gpu(c), C.to_gpu(qkv, dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:hq + 2 * hkv]
    got = dev.append_rotary(k, v, C4.rotary_on_gpu(r), pos=torch.from_numpy(pos).cuda(), q=q, starts=_starts(new),
                            max_new=max(new))
    turned = C.rounded(O4.turn(qkv[:, :hq + hkv], r, pos), dtype)
    first = np.concatenate([[0], np.cumsum(new)])
    O.append(c, turned[:, hq:], qkv[:, hq + hkv:hq + 2 * hkv], new, [np.arange(first[b], first[b + 1]) for b in range(3)])
    _compare(c, dev)
    assert C.same(C.host(got), turned[:, :hq])


@pytest.mark.parametrize("positions", [False, True])
@pytest.mark.parametrize("n", [1, 3, 8, 9, 40])
@pytest.mark.parametrize("sections", [None, (8, 16, 8)])
def test_positions_of_the_slots(positions, n, sections):
    """Without pos a token turns by the position that its slot gets."""
    _say(f"append_rotary without pos, positions={positions} n={n}")
    rng = np.random.default_rng(n)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[0, 21], slots=64, positions=positions)
    r = C4.rotary(rng, 200, 64, sections=sections)
    qkv = C.rounded(rng.standard_normal((2 * n, 8, 64)), "bf16")
    dev, x = C.on_gpu(c), C.to_gpu(qkv, "bf16")
    got = dev.append_rotary(x[:, 4:6], x[:, 6:], C4.rotary_on_gpu(r), q=x[:, :4])
    rows = [np.arange(n), n + np.arange(n)]
    turned = C.rounded(O4.turn(qkv[:, :6], r, default_pos(c, [n, n], rows)), "bf16")
    O.append(c, turned[:, 4:], qkv[:, 6:], [n, n], rows)
    _compare(c, dev)
    assert C.same(C.host(got), turned[:, :4])


@pytest.mark.parametrize("n,per", [(335, 700), (1, 1), (7, 97)])
def test_kept_rows_with_their_positions(n, per):
    """Rows picked from a prompt, in any order and twice, each with its own
    position; the queries come out in the order of the slots."""
    _say(f"append_rotary src n={n} of {per}")
    rng = np.random.default_rng(n)
    c = C.make(rng, dtype="bf16", hq=6, hkv=2, dh=128, page=16, lens=[0, 7], slots=400)
    r = C4.rotary(rng, 900, 128, sections=(16, 24, 24))
    qkv = C.rounded(rng.standard_normal((2 * per, 10, 128)), "bf16")
    pos = rng.integers(0, 900, (2 * per, 3)).astype(np.int32)
    src = rng.integers(0, per, (2, n)).astype(np.int32)
    dev, x = C.on_gpu(c), C.to_gpu(qkv, "bf16")
    got = dev.append_rotary(x[:, 6:8], x[:, 8:], C4.rotary_on_gpu(r), pos=torch.from_numpy(pos).cuda(), q=x[:, :6],
                            src=torch.from_numpy(src).cuda())
    turned = C.rounded(O4.turn(qkv[:, :8], r, pos), "bf16")
    rows = [src[0].astype(int), per + src[1].astype(int)]
    O.append(c, turned[:, 6:], qkv[:, 8:], [n, n], rows)
    _compare(c, dev)
    assert C.same(C.host(got), turned[:, :6][np.concatenate(rows)])


@pytest.mark.parametrize("n", [3, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_in_place(n, dtype):
    _say(f"append_rotary in place n={n} {dtype}")
    rng = np.random.default_rng(n)
    for shape in SHAPES:
        (hq, hkv, dh), rot, interleaved, _ = shape
        c = C.make(rng, dtype=dtype, hq=hq, hkv=hkv, dh=dh, page=16, lens=[2], slots=48)
        r = C4.rotary(rng, 64, rot, interleaved=interleaved)
        q, kv = (C.rounded(rng.standard_normal((n, h, dh)), dtype) for h in (hq, 2 * hkv))
        dev, x, y = C.on_gpu(c), C.to_gpu(q, dtype), C.to_gpu(kv, dtype)
        got = dev.append_rotary(y[:, :hkv], y[:, hkv:], C4.rotary_on_gpu(r), q=x, out=x)
        assert got is x
        assert C.same(C.host(x), C.rounded(O4.turn(q, r, 2 + np.arange(n)), dtype)), shape


@pytest.mark.parametrize("n", [4, 5, 8, 9, 256, 257])
def test_few_and_many_tokens(n):
    """Tokens that one block takes, those whose heads four waves share and those that a
    wave has to itself: as one token at a time."""
    _say(f"append_rotary of {n} tokens")
    rng = np.random.default_rng(n)
    args = dict(dtype="bf16", hq=12, hkv=4, dh=96, page=32, lens=[3, 40], slots=304)
    a, b = (C.on_gpu(C.make(np.random.default_rng(5), **args)) for _ in range(2))
    r = C4.rotary_on_gpu(C4.rotary(rng, 400, 96))
    x = C.to_gpu(C.rounded(rng.standard_normal((2, n, 20, 96)), "bf16"), "bf16")
    y = x.view(2 * n, 20, 96).clone()
    q = y[:, :12].contiguous()
    got = a.append_rotary(y[:, 12:16], y[:, 16:], r, q=q, out=q).view(2, n, 12, 96)
    for i in range(n):
        one = x[:, i].contiguous()
        want = b.append_rotary(one[:, 12:16], one[:, 16:], r, q=one[:, :12])
        assert torch.equal(got[:, i], want), i
    for name in ("k_pages", "v_pages", "lens"):
        assert torch.equal(torch.nan_to_num(getattr(a, name).float()), torch.nan_to_num(getattr(b, name).float())), name


@pytest.mark.parametrize("n", [6, 26])
def test_full_caches_and_bad_indices(n):
    """Tokens past the capacity are not stored, rows on pages that are none left
    out, and their queries turned all the same; rows of no sequence stay."""
    _say(f"append_rotary past the capacity n={n}")
    rng = np.random.default_rng(n)
    c = C.make(rng, dtype="bf16", hq=2, hkv=2, dh=64, page=16, lens=[46, 20, 48], slots=48, positions=True, weights=True)
    c["table"][1, 1] = 10 ** 6
    r = C4.rotary(rng, 80, 64)
    rows = 3 * n + 5
    qkv = C.rounded(rng.standard_normal((rows, 6, 64)), "bf16")
    pos = rng.integers(0, 80, rows).astype(np.int32)
    first = [0, n, 2 * n, 3 * n]
    dev, x = C.on_gpu(c), C.to_gpu(qkv, "bf16")
    out = torch.full((rows, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    dev.append_rotary(x[:, 2:4], x[:, 4:], C4.rotary_on_gpu(r), pos=torch.from_numpy(pos).cuda(), q=x[:, :2], out=out,
                      starts=torch.tensor(first, dtype=torch.int32).cuda(), max_new=n)
    turned = C.rounded(O4.turn(qkv[:, :4], r, pos), "bf16")
    O.append(c, turned[:, 2:], qkv[:, 4:], [n] * 3, [np.arange(first[b], first[b + 1]) for b in range(3)])
    _compare(c, dev)
    assert C.same(C.host(out)[: 3 * n], turned[: 3 * n, :2]) and (out[3 * n:] == 7).all()
    # rows past max_new are not taken, starts are clipped to the rows there are
    c = C.make(rng, dtype="bf16", hq=2, hkv=2, dh=64, page=16, lens=[0, 3], slots=64)
    dev = C.on_gpu(c)
    out.fill_(7.0)
    starts = torch.tensor([rows - 2, 2 ** 31 - 1, -4], dtype=torch.int32).cuda()
    dev.append_rotary(x[:, 2:4], x[:, 4:], C4.rotary_on_gpu(r), pos=torch.from_numpy(pos).cuda(), q=x[:, :2], out=out,
                      starts=starts, max_new=n)
    O.append(c, turned[:, 2:], qkv[:, 4:], [2, 0], [np.arange(rows - 2, rows), []])
    _compare(c, dev)
    assert C.same(C.host(out)[-2:], turned[-2:, :2]) and (out[:-2] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan(dtype):
    """They go where the formula has them: both elements of their pair."""
    _say(f"append_rotary infinities {dtype}")
    rng = np.random.default_rng(2)
    x = C.rounded(rng.standard_normal((12, 3, 64)), dtype)
    for i, bad in enumerate([np.inf, -np.inf, np.nan] * 3):
        x[i, i % 2, 5 * i] = bad
    c = C.make(rng, dtype=dtype, hq=1, hkv=1, dh=64, page=16, lens=[0], slots=16)
    r = C4.rotary(rng, 20, 64)
    r["cos"][3], r["sin"][3] = 1.0, 0.0      # infinity times a sine of zero
    dev, y = C.on_gpu(c), C.to_gpu(x, dtype)
    got = dev.append_rotary(y[:, 1:2], y[:, 2:], C4.rotary_on_gpu(r), q=y[:, :1])
    with np.errstate(invalid="ignore"):
        turned = C.rounded(O4.turn(x[:, :2], r, np.arange(12)), dtype)
    O.append(c, turned[:, 1:], x[:, 2:], [12], [np.arange(12)])
    _compare(c, dev)
    assert C.same(C.host(got), turned[:, :1])


def test_captured_and_on_another_stream():
    """A step in a graph, replayed on a side stream with eager work between,
    against the same calls made eagerly."""
    _say("append_rotary graph")
    rng = np.random.default_rng(9)
    args = dict(dtype="bf16", hq=28, hkv=4, dh=128, page=16, lens=[300, 60], slots=400, positions=True, weights=True)
    a, b = (C.on_gpu(C.make(np.random.default_rng(4), **args)) for _ in range(2))
    rot = C4.rotary_on_gpu(C4.rotary(rng, 600, 128, sections=(16, 24, 24)))
    for n in (2, 20):
        qkv = torch.zeros((2 * n, 36, 128), dtype=torch.bfloat16, device="cuda")
        pos = torch.zeros((2 * n, 3), dtype=torch.int32, device="cuda")
        start = [t.clone() for t in (a.lens, a.seen)]

        def step(cache):
            cache.lens.copy_(start[0])
            cache.seen.copy_(start[1])
            q = cache.append_rotary(qkv[:, 28:32], qkv[:, 32:], rot, pos=pos, q=qkv[:, :28])
            return [q, *cache.prefill(q, lse=True)]

        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step(a)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(a)
        for i in range(4):
            qkv.copy_(torch.from_numpy(rng.standard_normal(qkv.shape)).cuda())
            pos.copy_(torch.from_numpy(rng.integers(0, 600, pos.shape)).cuda())
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                graph.replay()
            want = step(b)
            torch.cuda.synchronize()
            for x, y in zip(got, want):
                assert torch.equal(x, y), i
            for name in ("k_pages", "v_pages", "lens", "seen", "slot_pos", "weights"):
                x, y = getattr(a, name), getattr(b, name)
                assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float())), (name, i)


def test_a_table_of_far_positions():
    """Rotary.create against angles in 64 bits: each entry rounded once, after an
    angle of up to 2e5 whose own rounding in 64 bits is 2^-36 at most."""
    _say("Rotary.create")
    r = B.Rotary.create(200000, 32, base=5e5)
    p = np.array([0, 1, 131071, 199999])
    angle = p[:, None] * 5e5 ** (-np.arange(16) / 16)
    for got, want in ((r.cos, np.cos(angle)), (r.sin, np.sin(angle))):
        got = got[torch.from_numpy(p).cuda()].double().cpu().numpy()
        assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -34).all()
    assert r.desc.rot_dim == 32 and r.desc.n_pos == 200000


def test_offsets_past_32_bits():
    """The last pages of a cache of more than 2^32 elements, and rows of q far apart."""
    _say("append_rotary far pages")
    rng = np.random.default_rng(12)
    n_pages = (1 << 31) // (2 * 64 * 128) + 70      # K alone: over 2^31 elements, 2^32 bytes
    pages = [torch.zeros((n_pages, 2, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([60], dtype=torch.int32, device="cuda")
    dev = B.KvCache(*pages, table, lens, n_q_heads=4)
    r = C4.rotary(rng, 128, 128)
    wide = torch.zeros((10, 1 << 20), dtype=torch.bfloat16, device="cuda")
    qkv = C.rounded(rng.standard_normal((10, 8, 128)), "bf16")
    wide[:, : 8 * 128] = C.to_gpu(qkv, "bf16").view(10, -1)
    x = wide[:, : 8 * 128].unflatten(1, (8, 128))
    q = dev.append_rotary(x[:, 4:6], x[:, 6:], C4.rotary_on_gpu(r), q=x[:, :4])
    turned = C.rounded(O4.turn(qkv[:, :6], r, 60 + np.arange(10)), "bf16")
    got = torch.cat([pages[0][n_pages - 1, :, 60:], pages[0][n_pages - 2, :, :6]], 1)
    assert C.same(C.host(got), turned[:, 4:].transpose(1, 0, 2)) and C.same(C.host(q), turned[:, :4])
    got = torch.cat([pages[1][n_pages - 1, :, 60:], pages[1][n_pages - 2, :, :6]], 1)
    assert C.same(C.host(got), qkv[:, 6:].transpose(1, 0, 2))
    assert not pages[0][: n_pages - 2].any() and not pages[1][: n_pages - 2].any()


def test_wrapper_refusals_on_the_device():
    _say("append_rotary refusals")
    rng = np.random.default_rng(1)
    c = C.make(rng, dtype="bf16", hq=4, hkv=2, dh=64, page=16, lens=[0, 0], slots=32)
    dev, r = C.on_gpu(c), C4.rotary_on_gpu(C4.rotary(rng, 8, 64))
    r3 = C4.rotary_on_gpu(C4.rotary(rng, 8, 64, sections=(8, 12, 12)))
    x = torch.zeros((4, 8, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    for kw, what in ((dict(pos=i32(3)), "pos"), (dict(pos=i32(4, 3)), "pos"), (dict(pos=i32(4).long()), "pos"),
                     (dict(pos=i32(4).cpu()), "pos"), (dict(q=q[:2]), "q and k"), (dict(q=q[:, :2]), "q must"),
                     (dict(out=torch.empty(4, 4, 64)), "out needs q"), (dict(q=q, out=torch.empty(4, 4, 64)), "out must"),
                     (dict(starts=i32(3)), "max_new"), (dict(starts=i32(3), src=i32(2, 1)), "src and starts")):
        with pytest.raises(ValueError, match=what):
            dev.append_rotary(k, v, r, **kw)
    with pytest.raises(ValueError, match="pos"):
        dev.append_rotary(k, v, r3, pos=i32(4))
    big = B.Rotary.create(4, 128)
    with pytest.raises(Exception, match="rot_dim"):
        dev.append_rotary(k, v, big)
    with pytest.raises(Exception, match="q_out may be q"):
        y = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
        dev.append_rotary(k, v, r, q=y, out=y, src=i32(2, 2))
    assert not dev.lens.any()
