"""Argument checks of rotated appends and caches of 4 bits, on the CPU: nothing
reaches a device."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2608_02134_amd import binding as B

torch = pytest.importorskip("torch")

P = 0x10000    # an aligned address that is never read
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    B.lib()


def _cache(**over):
    c = dict(dtype=B.GMC_BF16, n_q_heads=28, n_kv_heads=4, head_dim=128, page_size=16, max_pages=8, n_pages=20, n_seq=2,
             k_pages=P, v_pages=P, page_table=P, lens=P)
    return B.GmcCache(**{**c, **over})


def _cache4(**over):
    c = dict(dtype=B.GMC_BF16, n_q_heads=28, n_kv_heads=4, head_dim=128, page_size=16, max_pages=8, n_pages=20, n_seq=2,
             k_codes=P, v_codes=P, k_scales=P, v_scales=P, page_table=P, lens=P)
    return B.GmcCache4(**{**c, **over})


def _rotary(**over):
    r = dict(cos=P, sin=P, n_pos=100, rot_dim=128, interleaved=0, sections=(0, 0, 0))
    r.update(over)
    r["sections"] = (ctypes.c_int32 * 3)(*r["sections"])
    return B.GmcRotary(**r)


def _refused(code, what, want=B.GMC_ERR_ARG):
    assert code == want, B.gmc_last_error()
    assert what in B.gmc_last_error(), B.gmc_last_error()


def _append(c, r, k=P, v=P, sk=512, sv=512, rows=2, starts=None, src=None, n=1, pos=None, q=None, sq=3584, out=None):
    call = B.gmc_cache4_append if isinstance(c, B.GmcCache4) else B.gmc_cache_append_rotary
    return call(c, r, k, v, sk, sv, rows, starts, src, n, pos, q, sq, out)


BAD4 = [("dtype", 2, "dtype"), ("n_q_heads", 30, "divide"), ("n_q_heads", 260, "n_q_heads"), ("head_dim", 48, "head_dim"),
        ("head_dim", 288, "head_dim"), ("page_size", 8, "page_size"), ("page_size", 48, "page_size"),
        ("max_pages", 0, "max_pages"), ("max_pages", (1 << 20) + 1, "max_pages"), ("n_pages", 0, "n_pages"),
        ("n_seq", 0, "n_seq"), ("n_seq", 65536, "n_seq"), ("k_codes", None, "null"), ("v_codes", None, "null"),
        ("page_table", None, "null"), ("lens", None, "null"), ("k_codes", P + 8, "aligned"), ("v_codes", P + 2, "aligned"),
        ("k_scales", None, "scales"), ("v_scales", None, "scales"), ("k_scales", P + 4, "scales"),
        ("v_scales", P + 1, "scales")]


@pytest.mark.parametrize("field,value,what", BAD4)
def test_bad_descriptors(field, value, what):
    c = _cache4(**{field: value})
    _refused(_append(c, None), what)
    _refused(_append(c, _rotary()), what)
    _refused(B.gmc_cache4_read(c, 2, None, 1, P, P), what)
    _refused(B.gmc_cache4_prefill(c, P, 3584, 2, None, 1, 0.1, 0, 0, P, None, P, BIG), what)
    _refused(B.gmc_cache4_decode(c, P, 3584, 0.1, 0, 0, P, None, P, BIG), what)
    _refused(B.gmc_cache4_decode_bytes(c), what)
    _refused(B.gmc_cache4_prefill_bytes(c, 1), what)


def test_null_descriptors():
    _refused(B.lib().gmc_cache4_append(None, None, P, P, 512, 512, 2, None, None, 1, None, None, 0, None, None), "NULL")
    _refused(B.lib().gmc_cache_append_rotary(ctypes.byref(_cache()), None, P, P, 512, 512, 2, None, None, 1, None, None,
                                             0, None, None), "rotary is NULL")
    _refused(B.lib().gmc_cache_append_rotary(None, ctypes.byref(_rotary()), P, P, 512, 512, 2, None, None, 1, None,
                                             None, 0, None, None), "NULL")


BAD_ROTARY = [(dict(cos=None), "tables"), (dict(sin=None), "tables"), (dict(cos=P + 8), "tables"), (dict(sin=P + 4), "tables"),
              (dict(n_pos=0), "n_pos"), (dict(n_pos=1 << 31), "n_pos"), (dict(rot_dim=0), "rot_dim"),
              (dict(rot_dim=8), "rot_dim"), (dict(rot_dim=24), "rot_dim"), (dict(rot_dim=144), "rot_dim"),
              (dict(rot_dim=-16), "rot_dim"), (dict(interleaved=2), "interleaved"), (dict(interleaved=-1), "interleaved"),
              (dict(sections=(16, 24, 20)), "pairs"), (dict(sections=(16, 22, 26)), "multiple of 4"),
              (dict(sections=(-4, 40, 28)), "negative"), (dict(sections=(2 ** 31 - 4, 4, 64)), "multiple of 4")]


@pytest.mark.parametrize("over,what", BAD_ROTARY, ids=str)
def test_bad_tables(over, what):
    _refused(_append(_cache(), _rotary(**over)), what)
    _refused(_append(_cache4(), _rotary(**over)), what)


@pytest.mark.parametrize("kind", ["pages", "codes"])
def test_append_refusals(kind):
    c, r = (_cache() if kind == "pages" else _cache4()), _rotary()
    _refused(_append(c, r, k=None), "k is NULL")
    _refused(_append(c, r, v=P + 4), "v must be 16-byte aligned")
    _refused(_append(c, r, sk=511), "k must")
    _refused(_append(c, r, sv=(1 << 24) + 8), "2^24")
    _refused(_append(c, r, n=0), "max_new")
    _refused(_append(c, r, n=129, rows=258), "max_new")
    _refused(_append(c, r, rows=3), "rows=3")
    _refused(_append(c, r, starts=P, src=P), "src and starts")
    _refused(_append(c, r, src=P, rows=3), "multiple of n_seq")
    _refused(_append(c, r, q=P), "q and q_out")
    _refused(_append(c, r, out=P), "q and q_out")
    _refused(_append(c, r, q=P + 8, out=P + 4096), "q must")
    _refused(_append(c, r, q=P, sq=3576, out=P + 4096), "q must")
    _refused(_append(c, r, q=P, out=P + 8), "q_out is not")
    _refused(_append(c, r, q=P, sq=3592, out=P), "q_out may be q")
    _refused(_append(c, r, q=P, out=P, src=P, rows=4), "q_out may be q")


def test_what_a_cache_of_4_bits_needs_a_table_for():
    c = _cache4()
    _refused(_append(c, None, pos=P), "need rotary")
    _refused(_append(c, None, q=P, out=P), "need rotary")
    _refused(_append(c, None, out=P), "need rotary")


def test_attention_and_read_refusals():
    c = _cache4()
    pre = lambda q=P, s=3584, rows=2, starts=None, n=1, scale=0.1, w=0, k=0, out=P: B.gmc_cache4_prefill(  # noqa: E731
        c, q, s, rows, starts, n, scale, w, k, out, None, P, BIG)
    dec = lambda q=P, s=3584, scale=0.1, w=0, k=0, out=P: B.gmc_cache4_decode(c, q, s, scale, w, k, out, None, P, BIG)  # noqa: E731
    for call in (pre, dec):
        _refused(call(q=None), "q is NULL")
        _refused(call(q=P + 8), "q must")
        _refused(call(s=3588), "q must")
        _refused(call(w=-1), "window")
        _refused(call(k=1 << 31), "sinks")
        _refused(call(out=None), "out")
        _refused(call(out=P + 8), "out")
        for scale in (float("nan"), float("inf"), 1e39):
            _refused(call(scale=scale), "scale")
    _refused(pre(n=0), "max_new")
    _refused(pre(n=129, starts=P), "max_new")
    _refused(pre(rows=5), "rows=5")
    _refused(B.gmc_cache4_prefill_bytes(c, 0), "max_new")
    read = lambda rows=2, starts=None, n=1, k=P, v=P: B.gmc_cache4_read(c, rows, starts, n, k, v)  # noqa: E731
    _refused(read(k=None), "k_out")
    _refused(read(v=P + 8), "v_out")
    _refused(read(rows=3), "rows=3")
    _refused(read(n=0), "max_new")
    _refused(read(rows=0, starts=P), "rows=0")


def test_workspaces_and_grids():
    c = _cache4(max_pages=512, n_pages=2000)
    need = B.gmc_cache4_decode_bytes(c)
    assert need > 0
    _refused(B.gmc_cache4_decode(c, P, 3584, 0.1, 0, 0, P, None, P, need - 1), "workspace", B.GMC_ERR_CAPACITY)
    _refused(B.gmc_cache4_decode(c, P, 3584, 0.1, 0, 0, P, None, None, need), "workspace")
    _refused(B.gmc_cache4_decode(c, P, 3584, 0.1, 0, 0, P, None, P + 16, need), "workspace")
    need = B.gmc_cache4_prefill_bytes(c, 3)
    assert need > 0
    _refused(B.gmc_cache4_prefill(c, P, 3584, 6, None, 3, 0.1, 0, 0, P, None, P, need - 1), "workspace",
             B.GMC_ERR_CAPACITY)
    many = _cache4(n_seq=65535, n_q_heads=256, n_kv_heads=256, head_dim=32, max_pages=1 << 20, n_pages=1 << 20)
    _refused(B.gmc_cache4_prefill(many, P, 8192, 1, P, 1, 0.1, 0, 0, P, None, P, 1 << 62), "2^23 blocks")


def test_checked_calls_reach_the_device():
    """What passes the checks fails here for want of a device, not before."""
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for c in (_cache(), _cache4()):
        assert _append(c, _rotary()) == B.GMC_ERR_HIP
        assert _append(c, _rotary(sections=(0, 64, 0)), pos=P, q=P, sq=3584, out=P) == B.GMC_ERR_HIP
        assert _append(c, _rotary(rot_dim=16, interleaved=1), rows=9, starts=P, n=128, q=P, sq=7168, out=P + 512) == B.GMC_ERR_HIP
        assert _append(c, _rotary(), src=P, rows=6, n=4) == B.GMC_ERR_HIP
    c = _cache4()
    assert _append(c, None) == B.GMC_ERR_HIP
    assert B.gmc_cache4_read(c, 9, P, 128, P, P) == B.GMC_ERR_HIP
    assert B.gmc_cache4_prefill(c, P, 3584, 9, P, 128, 0.1, 5, 4, P, P, P, BIG) == B.GMC_ERR_HIP
    assert B.gmc_cache4_decode(c, P, 7168, 0.1, 0, 0, P, None, P, BIG) == B.GMC_ERR_HIP
    assert "device" in B.gmc_last_error()


def _tensors(**over):
    u8, i32 = torch.uint8, torch.int32
    t = dict(k_codes=torch.zeros((6, 2, 16, 48), dtype=u8), v_codes=torch.zeros((6, 2, 16, 48), dtype=u8),
             k_scales=torch.zeros((6, 2, 16, 4), dtype=u8), v_scales=torch.zeros((6, 2, 16, 4), dtype=u8),
             page_table=torch.zeros((2, 3), dtype=i32), lens=torch.zeros(2, dtype=i32), n_q_heads=4, dtype=torch.bfloat16)
    t.update(over)
    return t


@pytest.mark.parametrize("over,what", [
    (dict(dtype=torch.float16), "dtype"),
    (dict(k_codes=torch.zeros((6, 2, 16, 48), dtype=torch.int8)), "k_codes"),
    (dict(k_codes=torch.zeros((6, 2, 16, 40), dtype=torch.uint8)), "k_codes"),
    (dict(k_codes=torch.zeros((6, 2, 48), dtype=torch.uint8)), "k_codes"),
    (dict(v_codes=torch.zeros((6, 2, 16, 32), dtype=torch.uint8)), "v_codes"),
    (dict(k_scales=torch.zeros((6, 2, 16, 3), dtype=torch.uint8)), "k_scales"),
    (dict(v_scales=torch.zeros((6, 2, 16, 4))), "v_scales"),
    (dict(page_table=torch.zeros((2, 3))), "page_table"),
    (dict(page_table=torch.zeros((2, 0), dtype=torch.int32)), "empty"),
    (dict(lens=torch.zeros(3, dtype=torch.int32)), "lens"),
    (dict(n_q_heads=3), "n_q_heads"),
    (dict(v_codes=torch.zeros((6, 2, 48, 16), dtype=torch.uint8).transpose(2, 3)), "contiguous"),
    (dict(), "GPU")])
def test_wrapper_rejects_mismatched_tensors(over, what):
    with pytest.raises(ValueError, match=what):
        B.KvCache4(**_tensors(**over))


@pytest.mark.parametrize("over", [dict(n_seq=0), dict(slots=0), dict(page_size=0), dict(head_dim=48), dict(head_dim=0)])
def test_wrapper_creates_no_empty_caches(over):
    args = dict(n_seq=2, slots=40, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, device="cpu")
    with pytest.raises(ValueError, match="must be"):
        B.KvCache4.create(**{**args, **over})


@pytest.mark.parametrize("cos,sin,more,what", [
    (torch.zeros(4, 16), torch.zeros(4, 8), {}, "one shape"), (torch.zeros(4, 16).double(), torch.zeros(4, 16), {}, "float32"),
    (torch.zeros(64), torch.zeros(64), {}, "float32"), (torch.zeros(4, 12), torch.zeros(4, 12), {}, "rot_dim"),
    (torch.zeros(0, 16), torch.zeros(0, 16), {}, "rot_dim"), (torch.zeros(16, 4).T, torch.zeros(16, 4).T, {}, "contiguous"),
    (torch.zeros(4, 16), torch.zeros(4, 16), {}, "GPU")])
def test_wrapper_rejects_tables(cos, sin, more, what):
    with pytest.raises(ValueError, match=what):
        B.Rotary(cos, sin, **more)


def test_wrapper_creates_no_bad_tables():
    for n_pos, rot in ((0, 64), (5, 24), (5, 0)):
        with pytest.raises(ValueError, match="must be"):
            B.Rotary.create(n_pos, rot, device="cpu")


@pytest.mark.parametrize("mirror,name", [(B.GmcCache4, "gmc_cache4"), (B.GmcRotary, "gmc_rotary")])
def test_struct_layout_matches_the_c_compiler(tmp_path, mirror, name):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in mirror._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gmc.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", offsetof({name}, {n}));\n' for n in names) +
                   f'  printf("%zu\\n", sizeof({name}));\n  return 0;\n}}\n')
    exe = tmp_path / "layout"
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-std=c99", "-I", include, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [getattr(mirror, n).offset for n in names] + [ctypes.sizeof(mirror)]


def test_every_new_entry_point_is_declared_and_bound():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gmc.h")).read()
    names = [n for n in B.SIGNATURES if n.startswith("gmc_cache4_") or n.endswith("_rotary")]
    assert len(names) == 7
    for n in names:
        assert n + "(" in header and hasattr(B.lib(), n), n
