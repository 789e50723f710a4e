"""The README's examples of the K/V cache, run as they stand there."""
import os
import re

import numpy as np
import pytest

from oracle import cache4_oracle as O4
from oracle import cache_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from . import cache4_cases as C4  # noqa: E402
from . import cache_cases as C  # noqa: E402

B, TOKENS, KEPT, HQ, HKV, DH = 16, 60, 25, 28, 4, 128


def _example(word):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    found = [code for code in re.findall(r"```python\n(.*?)```", text, re.S) if word in code]
    assert len(found) == 1
    return found[0]


def _inputs(rng, positions):
    """What the examples' program has in hand: a prompt's projections, its kept rows
    and one more token of each request."""
    rows = lambda n, h: C.to_gpu(C.rounded(rng.standard_normal((n, h, DH)), "bf16"), "bf16")  # noqa: E731
    keep = np.stack([np.sort(rng.permutation(TOKENS)[:KEPT]) for _ in range(B)]).astype(np.int32)
    return dict(torch=torch, k=rows(B * TOKENS, HKV), v=rows(B * TOKENS, HKV), q=rows(B * TOKENS, HQ),
                keep=torch.from_numpy(keep).cuda(), positions=torch.from_numpy(positions.reshape(-1, 3)).cuda(),
                k1=rows(B, HKV), v1=rows(B, HKV), q1=rows(B, HQ))


def test_the_example_of_a_cache_runs():
    print("\n[case] README, KvCache", flush=True)
    rng = np.random.default_rng(1)
    at = _inputs(rng, np.zeros((B, TOKENS, 3), np.int32))
    at["q"] = at["q"][: B * KEPT]
    exec(_example("import KvCache\n"), at)
    assert at["out"].shape == (B, HQ, DH) and (at["cache"].lens == KEPT + 1).all()


def test_the_example_of_rotation_turns_the_answer_by_the_position_behind_its_prompt():
    """An image's tokens in the middle of a text: (t, h, w) of theirs, then text goes on
    behind the largest position.  Few rows are kept, so their number is another position."""
    print("\n[case] README, Rotary and KvCache4", flush=True)
    rng = np.random.default_rng(2)
    pos = np.zeros((B, TOKENS, 3), np.int32)
    for b in range(B):
        head, i, w = 3 + b, np.arange(36), 6 if b % 2 else 4
        pos[b, :head] = np.arange(head)[:, None]
        pos[b, head:head + 36] = head + np.stack([0 * i, i // w, i % w], 1)
        pos[b, head + 36:] = (head + 36 // w + np.arange(TOKENS - head - 36))[:, None]
    at = _inputs(rng, pos)
    given = C.host(at["q1"])
    exec(_example("import KvCache4"), at)
    rotary, cache = at["rotary"], at["cache"]
    after = pos.max((1, 2)) + 1
    assert not (after == KEPT).any() and (cache.lens == KEPT + 1).all()
    table = {"cos": rotary.cos[:200].cpu().numpy(), "sin": rotary.sin[:200].cpu().numpy(), "interleaved": False,
             "sections": rotary.sections}
    answer = np.repeat(after[:, None], 3, 1)
    assert C.same(C.host(at["q1"]), C.rounded(O4.turn(given, table, answer), "bf16"))
    turned = O4.turn(C.host(at["k1"]), table, answer)
    got = C.host(at["cache"].read(max_new=1)[0])
    for b in range(B):
        for h in range(HKV):
            for blk in range(0, DH, 32):
                codes, e = O4.quantise(turned[b, h, blk:blk + 32])
                assert got[b, h, blk:blk + 32].tolist() == [O4.value(x, e) for x in codes]
    # and its output is attention from there over all rows that the cache holds
    k, v = (C.host(x).reshape(B, KEPT + 1, HKV, DH).transpose(0, 2, 1, 3) for x in cache.read(max_new=KEPT + 1))
    held = {"k": k, "v": v, "table": np.arange(B)[:, None], "lens": np.full(B, KEPT + 1)}
    ref = O.attend(held, C.host(at["q1"]), list(range(B)), [1] * B, DH ** -0.5)
    C4.check_attention(ref, C.host(at["out"]), ref["lse"], "bf16", DH, True)
