"""Attention whose answer names every tile of tokens that went into it (tests/kv_marks.py; tests/test_kv_marks.py shows what it would see):
splitting and joining of long sequences, lines of many short ones, windows, selected pages."""
import numpy as np
import pytest
import torch

from tests.kv_marks import LN2, Marks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2401_14361_amd as mod
    mod.lib()
    return mod


def _on_device(m, c, **kw):
    kv = m.Kv(c.Hq, c.Hkv, c.Dk, c.Dv, c.page, c.dtype, max_batch=len(c.lens), max_pages=c.width, **kw)
    k, v = torch.from_numpy(c.k).cuda().to(kv.page_dtype), torch.from_numpy(c.v).cuda().to(kv.page_dtype)
    scales = dict(k_scale=torch.full((c.Hkv,), c.k_scale, device="cuda"), v_scale=torch.ones(c.Hkv, device="cuda")) if c.dtype == "fp8" else {}
    if kw.get("max_sel"):
        summary = torch.from_numpy(np.nan_to_num(c.k, nan=0.0)).cuda()
        scales.update(k_min=summary.amin(2).to(kv.dtype), k_max=summary.amax(2).to(kv.dtype))
    return kv, m.KvPages(kv, k, v, **scales), torch.from_numpy(c.table).cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda"), torch.from_numpy(c.q).to(kv.dtype).cuda()


def _check(c, out, lse, window=0, chosen=None):
    ref, ref_lse = c.answers(window, chosen)
    far, far_lse = c.wrong(out.double().cpu().numpy(), lse.double().cpu().numpy(), ref, ref_lse)
    assert not far.any(), (far.sum(), np.argwhere(far)[:8])
    assert not far_lse.any(), (far_lse.sum(), np.argwhere(far_lse)[:8])


def ragged(B, top, seed):
    n = np.random.default_rng(seed).integers(0, top + 1, B).tolist()
    n[B // 2] = top
    return n


MANY = [
    # dtype, Hq, Hkv, Dk, Dv, page, lens
    ("bf16", 4, 1, 64, 64, 64, [40001, 70]),              # hundreds of workgroups share an item
    ("fp8", 4, 1, 64, 64, 64, [40001, 70]),
    ("fp32", 4, 1, 64, 64, 64, [40001, 70]),
    ("bf16", 4, 1, 128, 128, 64, [131072]),
    ("bf16", 8, 2, 128, 128, 16, [20011, 300, 4999, 1]),
    ("fp8", 8, 2, 128, 128, 32, [20011, 300, 4999, 1]),
    ("fp32", 8, 2, 128, 128, 32, [7001, 300, 999]),
    ("fp32", 4, 2, 96, 96, 16, [9001, 17]),
    ("bf16", 4, 4, 192, 128, 16, [5001, 800, 16]),
    ("fp8", 4, 4, 192, 128, 16, [5001, 800, 32]),
    ("fp32", 4, 2, 192, 128, 32, [5001, 800]),
    ("bf16", 8, 2, 256, 256, 64, [9001, 127]),
    ("fp8", 8, 2, 256, 256, 64, [9001, 127]),
    ("fp32", 6, 2, 256, 256, 64, [4001, 127]),
    ("bf16", 40, 2, 64, 64, 32, [9001, 31]),              # twenty query heads a group: two blocks of heads
    ("fp8", 64, 1, 128, 128, 16, [6007, 100]),            # four
    ("bf16", 8, 4, 64, 64, 16, ragged(140, 2000, 1)),     # more items than workgroups: stretches go from one to the next
    ("fp8", 8, 4, 128, 128, 32, ragged(140, 2000, 2)),
    ("fp32", 8, 4, 64, 64, 16, ragged(140, 900, 3)),
    ("bf16", 4, 4, 128, 128, 16, ragged(160, 200, 4)),    # many short ones
    ("bf16", 4, 2, 256, 256, 16, ragged(90, 300, 5)),
    ("bf16", 4, 4, 192, 128, 16, ragged(70, 3000, 6)),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,lens", MANY)
def test_every_tile_counts_once(m, dtype, Hq, Hkv, Dk, Dv, page, lens):
    c = Marks(dtype, Hq, Hkv, Dk, Dv, page, lens, seed=Dk)
    kv, pages, table, lens_t, q = _on_device(m, c, max_sel=0)
    out, lse = m.kv_attend(kv, pages, table, lens_t, q, LN2, want_lse=True)
    _check(c, out, lse)
    assert kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("window", [1, 100, 1000, 8000])
def test_every_tile_of_a_window_counts_once(m, dtype, window):
    for lens in ([20000, 1001, 17, 0, 9000], ragged(130, 1500, window)):
        c = Marks(dtype, 8, 4, 64, 64, 16, lens, seed=window)
        kv, pages, table, lens_t, q = _on_device(m, c, max_sel=0)
        out, lse = m.kv_attend(kv, pages, table, lens_t, q, LN2, window=window, want_lse=True)
        _check(c, out, lse, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("lens,n_sel", [([30000, 500, 0, 12001], 100), (ragged(40, 6000, 9), 24)])
def test_every_tile_of_selected_pages_counts_once(m, dtype, lens, n_sel):
    c = Marks(dtype, 8, 4, 128, 128, 16, lens, seed=n_sel)
    kv, pages, table, lens_t, q = _on_device(m, c, max_sel=n_sel)
    out, lse, blocks = m.kv_attend_blocks(kv, pages, table, lens_t, q, LN2, n_sel, keep_first=1, keep_last=2, want_lse=True, want_blocks=True)
    _check(c, out, lse, chosen=blocks.cpu().numpy())
