"""Seeded caches of 4 bits and rotary tables for the tests of gmc_cache4_* and
gmc_cache_append_rotary, on the host and on the GPU (test infrastructure)."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache4_oracle as O4
from paper_2608_02134_amd import binding as B

from . import cache_cases as C


def values(codes, scales):
    """float64 values of codes [..., dh] and scales [..., dh / 32]."""
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127)).repeat(32, -1)
    return np.array(O4.MAGNITUDES)[codes & 7] * np.where(codes & 8, -1.0, 1.0) * power


def make(rng, *, dtype, hq, hkv, dh, page, lens, slots, spare=3, q_scale=2.0):
    """A cache of len(lens) sequences whose pages are shuffled, of values around
    one; rows past the lengths read as NaN."""
    b, per = len(lens), -(-slots // page)
    n_pages = b * per + spare
    c = {"dtype": dtype, "hq": hq, "q_scale": q_scale}
    for x in "kv":
        c[x + "_codes"] = rng.integers(0, 16, (n_pages, hkv, page, dh)).astype(np.uint8)
        c[x + "_scales"] = rng.integers(124, 127, (n_pages, hkv, page, dh // 32)).astype(np.uint8)
    c["table"] = rng.permutation(n_pages)[: b * per].reshape(b, per).astype(np.int32)
    c["lens"] = np.array(lens, np.int32)
    used = np.zeros((n_pages, page), bool)
    for i, n in enumerate(lens):
        for s in range(min(n, per * page)):
            used[c["table"][i][s // page], s % page] = True
    for x in "kv":
        c[x + "_scales"][~used[:, None].repeat(hkv, 1)] = 255
    refresh(c)
    return c


def refresh(c):
    """The values after a change of codes or scales."""
    for x in "kv":
        c[x] = values(c[x + "_codes"], c[x + "_scales"])


def packed(codes):
    return (codes[..., ::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def padded(scales, fill=0):
    """Scales with the row's unused bytes."""
    room = B.cache4_scale_bytes(32 * scales.shape[-1]) - scales.shape[-1]
    return np.concatenate([scales, np.full(scales.shape[:-1] + (room,), fill, np.uint8)], -1)


def on_gpu(c, fill=171):
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return B.KvCache4(t(packed(c["k_codes"])), t(packed(c["v_codes"])), t(padded(c["k_scales"], fill)),
                      t(padded(c["v_scales"], fill)), t(c["table"]), t(c["lens"]), n_q_heads=c["hq"],
                      dtype=C.DT[c["dtype"]])


def compare(c, dev, fill=171):
    """Every byte of codes and scales, but the codes of blocks that read as NaN."""
    assert np.array_equal(dev.lens.cpu().numpy(), c["lens"])
    for x in "kv":
        scales = getattr(dev, x + "_scales").cpu().numpy()
        assert np.array_equal(scales, padded(c[x + "_scales"], fill)), x
        got, want = getattr(dev, x + "_codes").cpu().numpy(), packed(c[x + "_codes"])
        number = (c[x + "_scales"] != 255).repeat(16, -1)
        assert np.array_equal(got[number], want[number]), x


def rotary(rng, n_pos, rot, *, interleaved=False, sections=None, base=100.0):
    angle = np.arange(n_pos)[:, None] * base ** (-np.arange(rot // 2) / (rot // 2))
    return {"cos": np.cos(angle).astype(np.float32), "sin": np.sin(angle).astype(np.float32),
            "interleaved": interleaved, "sections": sections}


def rotary_on_gpu(r):
    return B.Rotary(torch.from_numpy(r["cos"]).cuda(), torch.from_numpy(r["sin"]).cuda(), interleaved=r["interleaved"],
                    sections=r["sections"])


def check_attention(ref, out, lse, dtype, dh, decode):
    """C.check_attention, whose sums have a term for each product: bf16 weights of
    decode enter as two terms, fp32 queries and weights as three, which are exact, and
    the sums have as many more additions."""
    terms = 3 if dtype == "f32" else 2 if decode else 1
    C.check_attention({**ref, "most": ref["most"] * terms}, out, lse, dtype, dh if dtype == "bf16" else dh * terms)
