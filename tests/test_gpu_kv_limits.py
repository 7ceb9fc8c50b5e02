"""The paged KV cache at the ends of what its calls take: heads, batches, table widths, pages that lie apart, a handle's first call in a
captured graph."""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.kv_marks import LN2, Marks
from tests.test_gpu_kv import Case, _append_inputs, _check_append, _freq, bits, m  # noqa: F401 (a fixture)
from tests.test_gpu_kv_marks import _check, _on_device

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("Hq,Hkv", [(1024, 1), (1024, 1024), (1024, 8)])
def test_the_most_heads(m, dtype, Hq, Hkv):  # noqa: F811
    c = Marks(dtype, Hq, Hkv, 16, 32, 16, [200, 17, 0], seed=Hkv)
    kv, pages, table, lens, q = _on_device(m, c, max_sel=6)
    out, lse = m.kv_attend(kv, pages, table, lens, q, LN2, want_lse=True)
    _check(c, out, lse)
    out, lse, blocks = m.kv_attend_blocks(kv, pages, table, lens, q, LN2, 6, want_lse=True, want_blocks=True)
    _check(c, out, lse, chosen=blocks.cpu().numpy())
    got, group = blocks.cpu().numpy(), Hq // Hkv
    keys = np.nan_to_num(c.k)
    for b in (0, 1):
        nb = -(-c.lens[b] // 16)
        at = c.table[b, :nb]
        for hk in {0, Hkv // 2, Hkv - 1}:
            want = O.choose(c.q[b, hk * group:hk * group + group].astype(np.float64), keys[at, hk].min(1).astype(np.float64), keys[at, hk].max(1).astype(np.float64), nb, 6, 1, 1)
            assert [x for x in got[b, hk].tolist() if x >= 0] == want
    assert kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("Hq,Hkv,layout", [(1024, 1, "dense"), (1024, 1024, "packed"), (512, 512, "odd")])
def test_append_with_the_most_heads(m, dtype, Hq, Hkv, layout):  # noqa: F811
    pos = [15, 3, -1, 31]
    c = Case(m, dtype, Hq, Hkv, 32, 16, 16, [16, 4, 0, 32], seed=Hkv, summaries=True, nan_tail=False, max_sel=0)
    q, k, v = _append_inputs(c, 4, seed=Hq, layout=layout)
    before = [t.clone() for t in (c.k, c.v)]
    q_out = torch.full((4, Hq, 32), 7.0, dtype=c.kv.dtype, device="cuda")
    q_before = q_out.clone()
    m.kv_append(c.kv, c.pages, c.table, torch.tensor(pos, dtype=torch.int32, device="cuda"), q, k, v, _freq(32), q_out=q_out)
    place = _check_append(c, q, k, v, q_out, q_before, *before, range(4), pos, _freq(32), False)
    for t in (0, 3):
        keys = c.k[place[t][0]].float()
        assert (c.lo[place[t][0]].float() == keys.amin(1)).all() and (c.hi[place[t][0]].float() == keys.amax(1)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("with_seq", [False, True])
def test_append_to_pages_that_lie_apart(m, dtype, with_seq):  # noqa: F811
    pos = [31, 3, 40, 47]
    c = Case(m, dtype, 4, 2, 64, 32, 16, [32, 4, 41, 48], seed=2, summaries=True, nan_tail=False, gap=48, max_sel=0)
    room = [bits(torch.as_strided(t, (c.n_pages - 1, 48), (t.stride(0), 1), t.storage_offset() + t[0].numel())) for t in (c.k, c.v)]
    q, k, v = _append_inputs(c, 4, seed=3)
    before = [t.clone() for t in (c.k, c.v)]
    seq = torch.arange(4, dtype=torch.int32, device="cuda") if with_seq else None
    q_out = m.kv_append(c.kv, c.pages, c.table, torch.tensor(pos, dtype=torch.int32, device="cuda"), q, k, v, _freq(64), seq=seq)
    place = _check_append(c, q, k, v, q_out, q_out, *before, range(4), pos, _freq(64), False)
    for t in (0, 3):
        keys = c.k[place[t][0]].float()
        assert (c.lo[place[t][0]].float() == keys.amin(1)).all() and (c.hi[place[t][0]].float() == keys.amax(1)).all()
    now = [bits(torch.as_strided(t, (c.n_pages - 1, 48), (t.stride(0), 1), t.storage_offset() + t[0].numel())) for t in (c.k, c.v)]
    assert all((a == b).all() for a, b in zip(now, room))
    out, lse = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, want_lse=True)
    c.check(out, lse, *c.oracle())


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("fp8", 128), ("fp32", 96), ("bf16", 256)])
def test_tables_wider_than_any_sequence(m, dtype, D):  # noqa: F811
    # as a captured step has them: room for 2^17 tokens, sequences of a few hundred
    c = Marks(dtype, 4, 2, D, D, 16, [(37 * b * b + 11 * b) % 300 for b in range(40)], seed=D)
    c.table = np.concatenate([c.table, np.full((40, 8192 - c.width), -1, np.int32)], 1)
    c.width = 8192
    kv, pages, table, lens, q = _on_device(m, c, max_sel=8)
    out, lse = m.kv_attend(kv, pages, table, lens, q, LN2, want_lse=True)
    _check(c, out, lse)
    out, lse, blocks = m.kv_attend_blocks(kv, pages, table, lens, q, LN2, 8, want_lse=True, want_blocks=True)
    _check(c, out, lse, chosen=blocks.cpu().numpy())
    assert kv.error_flags() == 0


def test_selected_pages_of_the_largest_batch(m):  # noqa: F811
    B = 4096
    lens = np.random.default_rng(1).integers(0, 200, B).tolist()
    c = Marks("bf16", 2, 1, 16, 16, 16, lens, seed=4)
    kv, pages, table, lens_t, q = _on_device(m, c, max_sel=5)
    out, lse, blocks = m.kv_attend_blocks(kv, pages, table, lens_t, q, LN2, 5, want_lse=True, want_blocks=True)
    _check(c, out, lse, chosen=blocks.cpu().numpy())


def test_the_first_calls_of_a_handle_in_a_graph(m):  # noqa: F811
    c = Case(m, "bf16", 6, 3, 112, 48, 64, [3000, 77, 1], seed=7, summaries=True, nan_tail=False, max_sel=9)
    q, k, v = _append_inputs(c, 3, seed=5)
    freq, pos, q_out = _freq(112), torch.tensor([2999, 76, 0], dtype=torch.int32, device="cuda"), torch.zeros_like(q)
    out, few = (torch.zeros((3, 6, 48), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.kv_append(c.kv, c.pages, c.table, pos, q, k, v, freq, q_out=q_out)
        m.kv_attend(c.kv, c.pages, c.table, c.len_t, q_out, c.scale, out=out)
        m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, q_out, c.scale, 9, out=few)
    for step in range(3):
        q.copy_(torch.randn_like(q))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q_out, out, few)]
        want_q = m.kv_append(c.kv, c.pages, c.table, pos, q, k, v, freq)
        want = [want_q, m.kv_attend(c.kv, c.pages, c.table, c.len_t, want_q, c.scale), m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, want_q, c.scale, 9)]
        torch.cuda.synchronize()
        assert all((bits(a) == bits(b)).all() for a, b in zip(got, want))
    assert c.kv.error_flags() == 0
