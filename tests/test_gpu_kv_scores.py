"""Page selection where scores are no numbers or infinite (oracle/kv_oracle.py)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv import Case, _choice, m  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _blocks(c, n_sel, first, last):
    """The chosen pages, which the oracle must have chosen too (the attention over them may be no numbers: it is not looked at)."""
    _, blocks = c.m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, n_sel, keep_first=first, keep_last=last, want_blocks=True)
    want = np.full(tuple(blocks.shape), -1)
    for b, heads in enumerate(_choice(c, n_sel, first, last)):
        for h, pages in enumerate(heads):
            want[b, h, :len(pages)] = pages
    got = blocks.cpu().numpy()
    assert (got == want).all()
    assert c.kv.error_flags() == 0
    return got


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("pages", [40, 700])   # one workgroup's, and several
@pytest.mark.parametrize("flip", [False, True])
def test_a_head_whose_sum_is_no_number_is_passed_over(m, dtype, pages, flip):  # noqa: F811
    # a query head with an infinite element, which meets 0 on some pages and a number on others, beside one that has numbers everywhere
    c = Case(m, dtype, 4, 2, 64, 64, 16, [16 * pages, 16 * pages - 7], seed=pages, summaries=True, max_sel=16)
    c.q[:, 1 if flip else 0, 3] = float("inf")
    at = c.table.long()[:, :pages]
    c.lo[at[:, ::3], :, 3], c.hi[at[:, ::3], :, 3] = 0.0, 0.0
    _blocks(c, 16, 1, 1)
    c.q[:, :, 3] = float("nan")  # no head has a number on any page: the lowest pages
    got = _blocks(c, 9, 1, 2)
    assert (got[0, 0] == [0, 1, 2, 3, 4, 5, 6, pages - 2, pages - 1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("value", [1.5, -1.5, 0.0])
def test_a_page_with_a_dimension_without_numbers_comes_last(m, dtype, value):  # noqa: F811
    # kv_append completes a page whose keys are no numbers in one dimension: its summary is empty there, and every other page comes before it
    page, D = 16, 32
    c = Case(m, dtype, 4, 2, D, D, page, [page * 9], seed=3, summaries=True, nan_tail=False, max_sel=8)
    c.q[:, :, 5] = value
    k = torch.randn((page, 2, D), device="cuda").to(c.kv.dtype)
    k[:, :, 5] = float("nan")
    k[7, :, 6] = 300.0  # (of large scores otherwise)
    pos = torch.arange(4 * page, 5 * page, dtype=torch.int32, device="cuda")
    zeros = torch.zeros((page, 4, D), dtype=c.kv.dtype, device="cuda")
    m.kv_append(c.kv, c.pages, c.table, pos, zeros, k, zeros[:, :2].contiguous(), None, seq=torch.zeros(page, dtype=torch.int32, device="cuda"))
    at = int(c.table[0, 4])
    assert torch.isposinf(c.lo[at, :, 5]).all() and torch.isneginf(c.hi[at, :, 5]).all()
    for n in range(3, 9):
        assert 4 not in _blocks(c, n, 1, 1)
    c.hi[int(c.table[0, 4]), :, 7] = float("inf")
    assert 4 not in _blocks(c, 8, 1, 1)


def test_infinite_summaries(m):  # noqa: F811
    # keys of +-inf are met by queries of their sign only; a zero of the query takes k_min
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [16 * 300], seed=9, summaries=True, max_sel=20)
    at = c.table[0].long()
    c.hi[at[[20, 41]], :, 3] = float("inf")
    c.lo[at[[33, 41]], :, 3] = float("-inf")
    for value in (1.0, -1.0, 0.0, -0.0):
        c.q[:, :, 3] = value
        got = _blocks(c, 12, 1, 1)
        if value == 1.0:
            assert {20, 41} <= set(got[0, 0].tolist())
        if value == -1.0:
            assert {33, 41} <= set(got[0, 0].tolist())
