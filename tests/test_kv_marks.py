"""The inputs of tests/kv_marks.py show the losses that they are made to show, in the tolerances that they come with (CPU only: the
mistakes are planted in the definition's answer)."""
import numpy as np
import pytest

from oracle import kv_oracle as O
from tests.kv_marks import LN2, TILE, Marks

CASES = [("bf16", 4, 1, 64, 64, 64, [40001, 70]), ("fp8", 8, 2, 128, 128, 32, [9000, 0, 33]), ("fp32", 6, 2, 96, 80, 16, [5000]),
         ("bf16", 4, 1, 128, 128, 64, [131072])]


@pytest.mark.parametrize("case", CASES[:3])
def test_answers_are_the_definition(case):
    c = Marks(*case)
    out, lse = O.attend(c.q.astype(np.float64), np.nan_to_num(c.k.astype(np.float64)), np.nan_to_num(c.v.astype(np.float64)), c.table, c.lens,
                        np.log(2.0), k_scale=np.full(c.Hkv, c.k_scale))
    ref, ref_lse = c.answers()
    some = np.isfinite(ref_lse)
    assert (np.isneginf(lse) == ~some).all()
    assert np.abs(out - ref).max() < 1e-12 and np.abs(lse[some] - ref_lse[some]).max() < 1e-12
    assert np.float32(np.float64(np.float32(LN2)) * 1.4426950408889634) == 1.0


@pytest.mark.parametrize("case", CASES)
def test_losses_show(case):
    c = Marks(*case)
    G = c.Hq // c.Hkv
    for b, n in enumerate(c.lens):
        for hk in range(c.Hkv) if n else ():
            heads = range(hk * G, hk * G + G)
            right = [c.answer(b, h) for h in heads]
            off = lambda got: [(w.any(), f) for w, f in (c.wrong(x[0], x[1], *r) for x, r in zip(got, right))]  # noqa: E731
            assert not any(w or f for w, f in off(right))
            for t in {0, n // 2 // TILE, (n - 1) // TILE - 1, n // 3 // TILE}:
                tile = np.arange(max(t, 0) * TILE, min(max(t, 0) * TILE + TILE, n))
                # a tile that nobody sees: outputs and logarithm; one whose values are not summed; a part of 128 tokens likewise
                assert any(w and f for w, f in off([c.answer(b, h, lost=tile) for h in heads]))
                assert any(w for w, _ in off([c.answer(b, h, unsummed=tile) for h in heads]))
                assert any(w for w, _ in off([c.answer(b, h, unsummed=np.arange(tile[0], min(tile[0] + 128, n))) for h in heads]))
                if G > 1:  # and one whose sums lie in another query head's row
                    assert any(w for w, _ in off([c.answer(b, h, other=np.arange(tile[0], min(tile[0] + 128, n))) for h in heads]))
