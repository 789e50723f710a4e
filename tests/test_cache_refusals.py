"""The paged cache's argument checks, on the CPU: nothing reaches a device."""
import pytest

from paper_2608_02134_amd import binding as B

torch = pytest.importorskip("torch")

P = 0x10000    # an aligned address that is never read


@pytest.fixture(scope="module", autouse=True)
def built():
    B.lib()


def _cache(**over):
    c = dict(dtype=B.GMC_BF16, n_q_heads=28, n_kv_heads=4, head_dim=128, page_size=16, max_pages=8, n_pages=20,
             n_seq=2, k_pages=P, v_pages=P, page_table=P, lens=P, seen=P, slot_pos=P, weights=P)
    c.update(over)
    return B.GmcCache(**c)


def _refused(code, what, want=B.GMC_ERR_ARG):
    assert code == want, B.gmc_last_error()
    assert what in B.gmc_last_error(), B.gmc_last_error()


BAD = [("dtype", 2, "dtype"), ("n_q_heads", 0, "n_q_heads"), ("n_q_heads", 30, "divide"), ("n_kv_heads", 0, "divide"),
       ("n_q_heads", 260, "n_q_heads"), ("head_dim", 48, "head_dim"), ("head_dim", 288, "head_dim"),
       ("head_dim", 0, "head_dim"), ("page_size", 8, "page_size"), ("page_size", 48, "page_size"),
       ("page_size", 2048, "page_size"), ("max_pages", 0, "max_pages"), ("max_pages", (1 << 20) + 1, "max_pages"),
       ("n_pages", 0, "n_pages"), ("n_pages", 1 << 31, "n_pages"), ("n_seq", 0, "n_seq"), ("n_seq", 65536, "n_seq"),
       ("k_pages", None, "null"), ("v_pages", None, "null"), ("page_table", None, "null"), ("lens", None, "null"),
       ("k_pages", P + 8, "aligned"), ("v_pages", P + 2, "aligned"), ("seen", None, "seen")]


@pytest.mark.parametrize("field,value,what", BAD)
def test_bad_descriptors(field, value, what):
    c = _cache(**{field: value})
    _refused(B.gmc_cache_append(c, P, P, 512, 512, 2, None, None, 1), what)
    _refused(B.gmc_cache_prefill(c, P, 3584, 2, None, 1, 0.1, 0, 0, P, None, P, 1 << 40), what)
    _refused(B.gmc_cache_decode(c, P, 3584, 0.1, 0, 0, 0, P, None, P, 1 << 40), what)
    _refused(B.gmc_cache_evict(c, 50, 4, 4, P, 1 << 40), what)
    _refused(B.gmc_cache_decode_bytes(c, 1), what)
    _refused(B.gmc_cache_prefill_bytes(c, 1), what)
    _refused(B.gmc_cache_evict_bytes(c, 50), what)


def test_null_cache():
    _refused(B.lib().gmc_cache_append(None, P, P, 512, 512, 2, None, None, 1, None), "NULL")


def test_append_refusals():
    c = _cache()
    call = lambda k=P, v=P, sk=512, sv=512, rows=2, starts=None, src=None, n=1: B.gmc_cache_append(  # noqa: E731
        c, k, v, sk, sv, rows, starts, src, n)
    _refused(call(k=None), "k is NULL")
    _refused(call(v=None), "v is NULL")
    _refused(call(k=P + 4), "k must be 16-byte aligned")
    _refused(call(sk=511), "k must")
    _refused(call(sv=514), "v must")
    _refused(call(n=0), "max_new")
    _refused(call(n=129, rows=258), "max_new")
    _refused(call(rows=3), "rows=3")
    _refused(call(rows=0, starts=P), "rows=0")
    _refused(call(starts=P, src=P), "src and starts")
    _refused(call(src=P, rows=3), "multiple of n_seq")
    _refused(call(src=P, rows=0), "multiple of n_seq")


def test_attention_refusals():
    c = _cache()
    call = lambda q=P, s=3584, rows=2, starts=None, n=1, w=0, k=0, out=P: B.gmc_cache_prefill(  # noqa: E731
        c, q, s, rows, starts, n, 0.1, w, k, out, None, P, 1 << 40)
    _refused(call(q=None), "q is NULL")
    _refused(call(q=P + 8), "q must")
    _refused(call(s=3583), "q must")
    _refused(call(s=3588), "q must")
    _refused(call(w=-1), "window")
    _refused(call(k=-1), "sinks")
    _refused(call(w=1 << 31), "window")
    _refused(call(out=None), "out")
    _refused(call(out=P + 8), "out")
    _refused(call(n=0), "max_new")
    _refused(call(n=129, starts=P), "max_new")
    _refused(call(rows=5), "rows=5")
    _refused(B.gmc_cache_prefill_bytes(c, 0), "max_new")
    _refused(B.gmc_cache_decode(_cache(weights=None), P, 3584, 0.1, 0, 0, 1, P, None, P, 1 << 40), "weights")


def test_workspaces_too_small():
    c = _cache()
    need = B.gmc_cache_decode_bytes(c, True)
    assert need > 0
    _refused(B.gmc_cache_decode(c, P, 3584, 0.1, 0, 0, 1, P, None, P, need - 1), "workspace", B.GMC_ERR_CAPACITY)
    _refused(B.gmc_cache_decode(c, P, 3584, 0.1, 0, 0, 1, P, None, None, need), "workspace")
    _refused(B.gmc_cache_decode(c, P, 3584, 0.1, 0, 0, 1, P, None, P + 16, need), "workspace")
    need = B.gmc_cache_evict_bytes(c, 50)
    assert need > 0
    _refused(B.gmc_cache_evict(c, 50, 4, 4, P, need - 1), "workspace", B.GMC_ERR_CAPACITY)


def test_evict_refusals():
    c = _cache()
    _refused(B.gmc_cache_evict(c, 0, 0, 0, P, 1 << 40), "budget")
    _refused(B.gmc_cache_evict(c, 10, 6, 5, P, 1 << 40), "sinks + recent")
    _refused(B.gmc_cache_evict(c, 10, -1, 5, P, 1 << 40), "none negative")
    _refused(B.gmc_cache_evict(c, 10, 1 << 62, 1 << 62, P, 1 << 40), "sinks + recent")
    for missing in ("weights", "slot_pos"):
        _refused(B.gmc_cache_evict(_cache(**{missing: None}), 50, 4, 4, P, 1 << 40), "needs")
    assert B.gmc_cache_evict_bytes(c, 128) == 0      # a budget of every slot: nothing can leave
    assert B.gmc_cache_evict(c, 128, 4, 4, None, 0) == B.GMC_OK


def test_checked_calls_reach_the_device():
    """What passes the checks fails here for want of a device, not before."""
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    c = _cache()
    assert B.gmc_cache_append(c, P, P, 512, 1024, 2, None, None, 1) == B.GMC_ERR_HIP
    assert B.gmc_cache_append(c, P, P, 512, 512, 7, P, None, 100) == B.GMC_ERR_HIP
    assert B.gmc_cache_prefill(c, P, 3584, 9, P, 128, 0.1, 5, 4, P, P, P, 1 << 40) == B.GMC_ERR_HIP
    assert B.gmc_cache_decode(c, P, 7168, 0.1, 0, 0, 1, P, None, P, 1 << 40) == B.GMC_ERR_HIP
    assert B.gmc_cache_evict(c, 50, 4, 46, P, 1 << 40) == B.GMC_ERR_HIP
    assert "device" in B.gmc_last_error()


def _tensors(**over):
    i32 = torch.int32
    t = dict(k_pages=torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16), v_pages=torch.zeros((6, 2, 16, 64), dtype=torch.bfloat16),
             page_table=torch.zeros((2, 3), dtype=i32), lens=torch.zeros(2, dtype=i32), n_q_heads=4,
             slot_pos=torch.zeros((2, 2, 48), dtype=i32), seen=torch.zeros(2, dtype=i32), weights=torch.zeros((2, 2, 48)))
    t.update(over)
    return t


@pytest.mark.parametrize("over,what", [
    (dict(k_pages=torch.zeros((6, 2, 16, 64), dtype=torch.float16)), "k_pages"),
    (dict(k_pages=torch.zeros((6, 2, 64), dtype=torch.bfloat16)), "k_pages"),
    (dict(v_pages=torch.zeros((6, 2, 16, 32), dtype=torch.bfloat16)), "v_pages"),
    (dict(page_table=torch.zeros((2, 3))), "page_table"),
    (dict(lens=torch.zeros(3, dtype=torch.int32)), "lens"),
    (dict(lens=torch.zeros(2, dtype=torch.int64)), "lens"),
    (dict(seen=torch.zeros(2)), "seen"),
    (dict(seen=None), "seen"),
    (dict(slot_pos=torch.zeros((2, 2, 47), dtype=torch.int32)), "slot_pos"),
    (dict(weights=torch.zeros((2, 2, 48), dtype=torch.float64)), "weights"),
    (dict(n_q_heads=3), "n_q_heads"),
    (dict(v_pages=torch.zeros((6, 2, 64, 16), dtype=torch.bfloat16).transpose(2, 3)), "contiguous"),
    (dict(), "GPU"),
])
def test_wrapper_rejects_mismatched_tensors(over, what):
    with pytest.raises(ValueError, match=what):
        B.KvCache(**_tensors(**over))


def test_struct_layout_matches_the_c_compiler(tmp_path):
    import ctypes
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in B.GmcCache._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "gmc.h"\nint main(void) {\n' +
                   "".join(f'  printf("%zu\\n", offsetof(gmc_cache, {n}));\n' for n in names) +
                   '  printf("%zu %d\\n", sizeof(gmc_cache), GMC_CACHE_MAX_HEADS);\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([cc, "-std=c99", "-I", include, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [getattr(B.GmcCache, n).offset for n in names] + [ctypes.sizeof(B.GmcCache),
                                                                                     B.GMC_CACHE_MAX_HEADS]


def test_prefill_of_more_blocks_than_a_grid_holds():
    """2^23 blocks of 128 (token, head) queries: more are refused before anything
    is launched, also where one sequence's count alone passes 32 bits."""
    big = dict(max_pages=1 << 20, n_pages=1 << 20)
    call = lambda c, n: B.gmc_cache_prefill(c, P, c.n_q_heads * c.head_dim, 1, P, n, 0.1, 0, 0, P, None, P, 1 << 62)  # noqa: E731
    _refused(call(_cache(n_seq=1, n_q_heads=256, n_kv_heads=1, head_dim=32, **big), 1 << 24), "2^23 blocks")
    _refused(call(_cache(n_seq=65535, n_q_heads=256, n_kv_heads=256, head_dim=32, **big), 1), "2^23 blocks")
    _refused(call(_cache(n_seq=3000, n_q_heads=8, n_kv_heads=2, head_dim=64, **big), 100000), "2^23 blocks")


def test_rows_too_far_apart():
    c = _cache()
    _refused(B.gmc_cache_append(c, P, P, (1 << 24) + 8, 512, 2, None, None, 1), "2^24")
    _refused(B.gmc_cache_prefill(c, P, (1 << 24) + 8, 2, None, 1, 0.1, 0, 0, P, None, P, 1 << 40), "2^24")
    _refused(B.gmc_cache_decode(c, P, (1 << 24) + 8, 0.1, 0, 0, 0, P, None, P, 1 << 40), "2^24")


@pytest.mark.parametrize("scale", [float("nan"), -float("nan"), float("inf"), -float("inf"), 1e39])
def test_scales_that_are_not_finite(scale):
    """Both attention calls refuse them alike (1e39 is infinite as a float)."""
    c = _cache()
    _refused(B.gmc_cache_prefill(c, P, 3584, 2, None, 1, scale, 0, 0, P, None, P, 1 << 40), "scale")
    _refused(B.gmc_cache_decode(c, P, 3584, scale, 0, 0, 0, P, None, P, 1 << 40), "scale")


def test_eviction_of_more_caches_than_a_launch_takes():
    """Long caches take 1024 threads a head, short ones 256; a launch has fewer than
    2^32.  (What passes is not run: it would need a device.)"""
    many = dict(n_q_heads=256, n_kv_heads=256, head_dim=32)
    _refused(B.gmc_cache_evict(_cache(n_seq=16384, max_pages=513, **many), 50, 4, 4, P, 1 << 62), "4194303 caches")
    _refused(B.gmc_cache_evict(_cache(n_seq=65535, max_pages=1 << 20, **many), 50, 4, 4, P, 1 << 62), "4194303 caches")
    if not torch.cuda.is_available():
        assert B.gmc_cache_evict(_cache(n_seq=16383, max_pages=513, **many), 50, 4, 4, P, 1 << 62) == B.GMC_ERR_HIP
        assert B.gmc_cache_evict(_cache(n_seq=65535, max_pages=512, **many), 50, 4, 4, P, 1 << 62) == B.GMC_ERR_HIP


@pytest.mark.parametrize("over", [
    dict(page_table=torch.zeros((0, 3), dtype=torch.int32), lens=torch.zeros(0, dtype=torch.int32), slot_pos=None, weights=None,
         seen=None),
    dict(page_table=torch.zeros((2, 0), dtype=torch.int32), slot_pos=None, weights=None),
    dict(k_pages=torch.zeros((6, 0, 16, 64)), v_pages=torch.zeros((6, 0, 16, 64)), slot_pos=None, weights=None),
    dict(k_pages=torch.zeros((0, 2, 16, 64)), v_pages=torch.zeros((0, 2, 16, 64)))])
def test_wrapper_rejects_empty_caches(over):
    with pytest.raises(ValueError, match="must not be empty"):
        B.check_cache_tensors(**_tensors(**over))


@pytest.mark.parametrize("over", [dict(n_seq=0), dict(slots=0), dict(page_size=0), dict(slots=-5)])
def test_wrapper_creates_no_empty_caches(over):
    args = dict(n_seq=2, slots=40, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=torch.bfloat16, device="cpu")
    with pytest.raises(ValueError, match="at least 1"):
        B.KvCache.create(**{**args, **over})
