"""Seeded paged caches for the tests of gmc_cache_*, on the host and on the
GPU, and the error bounds of attention over them (test infrastructure)."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache_oracle as O
from paper_2608_02134_amd import binding as B

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(a, dtype):
    """float64 values that the dtype holds exactly."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]).double().numpy()


def make(rng, *, dtype, hq, hkv, dh, page, lens, slots, positions=False, weights=False, spare=3, q_scale=2.0):
    """A cache of len(lens) sequences whose pages are shuffled; slots past the
    lengths hold NaN."""
    b, per = len(lens), -(-slots // page)
    n_pages = b * per + spare
    c = {"dtype": dtype, "hq": hq, "q_scale": q_scale}
    c["k"] = rounded(rng.standard_normal((n_pages, hkv, page, dh)), dtype)
    c["v"] = rounded(rng.standard_normal((n_pages, hkv, page, dh)), dtype)
    c["table"] = rng.permutation(n_pages)[: b * per].reshape(b, per).astype(np.int32)
    c["lens"] = np.array(lens, np.int32)
    used = np.zeros((n_pages, page), bool)
    for i, n in enumerate(lens):
        for s in range(min(n, per * page)):
            used[c["table"][i][s // page], s % page] = True
    c["k"][~used[:, None].repeat(hkv, 1)] = np.nan
    c["v"][~used[:, None].repeat(hkv, 1)] = np.nan
    cap = per * page
    if positions:
        past = (c["lens"] * 1.5).astype(np.int64) + 1
        c["seen"] = past.astype(np.int32)
        c["slot_pos"] = np.zeros((b, hkv, cap), np.int32)
        for i in range(b):
            for h in range(hkv):
                c["slot_pos"][i, h] = np.concatenate([rng.permutation(past[i])[: lens[i]],
                                                      np.full(max(cap - lens[i], 0), 7)])[:cap]
    if weights:
        c["weights"] = (rng.random((b, hkv, cap)) * 1e-2).astype(np.float32).astype(np.float64)
    return c


def on_gpu(c):
    """The cache as a KvCache."""
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    more = {}
    if c.get("slot_pos") is not None:
        more = dict(slot_pos=t(c["slot_pos"]), seen=t(c["seen"]))
    if c.get("weights") is not None:
        more["weights"] = t(c["weights"].astype(np.float32))
    return B.KvCache(t(c["k"]).to(DT[c["dtype"]]), t(c["v"]).to(DT[c["dtype"]]), t(c["table"]), t(c["lens"]),
                     n_q_heads=c["hq"], **more)


def queries(rng, c, rows):
    return rounded(c["q_scale"] * rng.standard_normal((rows, c["hq"], c["k"].shape[3])), c["dtype"])


def to_gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


# --- error bounds, from the roundings the kernels are allowed -------------------
U32, UBF = 2.0 ** -24, 2.0 ** -8      # half a step relative to the value


def logit_error(ref, dh):
    """|error| of a logit in fp32: dh products summed (each addition rounds the
    partial sum, at most `size`, by half a step), the scale and the change of base
    to 2 (three roundings of a value at most `size`)."""
    return (dh + 4) * U32 * np.nan_to_num(ref["size"])


def weight_error(ref, dh):
    """Relative error of an attention weight or of their sum: the logit's error
    in numerator and denominator, an exponential to 4 half steps with an
    argument as large as 2 * size rounded once, the sum of `most` terms, joined
    parts and a division."""
    return 2 * logit_error(ref, dh) + (np.nan_to_num(ref["most"]) + 16) * U32 + 4 * np.nan_to_num(ref["size"]) * U32


def check_attention(ref, out, lse, dtype, dh, rows=None):
    """bf16: the weights enter the value product as bf16 (half a step each) and
    the result is rounded once more."""
    rows = np.isfinite(ref["lse"]).any(1) | np.isneginf(ref["lse"]).any(1) if rows is None else rows
    ref = {k: (v[rows] if k != "probs" else v) for k, v in ref.items()}
    out, lse = out[rows], lse[rows]
    rel = weight_error(ref, dh)[..., None]
    tol = ref["mass"] * rel + U32 * np.abs(ref["out"])
    if dtype == "bf16":
        tol = ref["mass"] * (rel + UBF * 1.01) + UBF * 1.01 * np.abs(ref["out"])
    bad = ~(np.abs(out - ref["out"]) <= tol)
    assert not bad.any(), (f"{bad.sum()} of {bad.size} entries off, worst "
                           f"{np.nanmax(np.abs(out - ref['out']) / np.maximum(tol, 1e-300)):.3g} of the bound, "
                           f"first at {np.argwhere(bad)[0]}")
    none = np.isneginf(ref["lse"])
    assert same(lse[none], ref["lse"][none])
    ltol = (weight_error(ref, dh) + 2 * U32 * np.abs(np.where(none, 0, ref["lse"])))[~none]
    off = np.abs(lse - np.where(none, 0, ref["lse"]))[~none]
    assert (off <= ltol).all(), f"lse off by {np.max(off / np.maximum(ltol, 1e-300)):.3g} of the bound"
    assert (out[none] == 0).all()


def check_weights(ref, before, after, dh):
    """Weights after accumulating: each of the group's terms as weight_error, one
    rounded addition for each."""
    b, hkv, _ = before.shape
    rel = weight_error(ref, dh).reshape(b, hkv, -1).max(2)[..., None]
    want = before + ref["probs"]
    tol = ref["probs"] * rel + 40 * U32 * np.abs(want)
    bad = ~(np.abs(after - want) <= tol)
    assert not bad.any(), f"{bad.sum()} weights off, first at {np.argwhere(bad)[0]}"
