"""What calls allocate: on a stream that is not the current one it belongs to that stream and holds the same bits."""
import numpy as np
import pytest
import torch

import moei_inputs as mi
from tests.helpers import EPS, dev, pack_bank
from tests.test_gpu_kv import Case, _append_inputs, _freq, bits, m  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _owner(t):
    """The stream whose memory a tensor lies in."""
    at, = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
    return at


def _tensors(x):
    return [t for t in (x if isinstance(x, tuple) else (x,)) if isinstance(t, torch.Tensor)]


def _both_ways(call, by_handle):
    """call(stream) on the current stream and on another one, which has its outputs."""
    want = [bits(t) for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = _tensors(call(side.cuda_stream if by_handle else side))
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
    torch.cuda.synchronize()
    assert len(got) == len(want) > 0
    for t, w in zip(got, want):
        assert _owner(t) == side.cuda_stream
        assert (bits(t) == w).all()
    mine = call(torch.cuda.current_stream())
    assert all(_owner(t) == torch.cuda.current_stream().cuda_stream for t in _tensors(mine))


@pytest.mark.parametrize("by_handle", [False, True])
def test_kv_calls(m, by_handle):  # noqa: F811
    for Dv in (64, 48):
        c = Case(m, "bf16", 4, 2, 64, Dv, 16, [900, 40, 1], seed=Dv, summaries=True, nan_tail=False, max_sel=16)
        q, k, v = _append_inputs(c, 3, seed=1)
        pos = torch.tensor([899, 39, 0], dtype=torch.int32, device="cuda")
        _both_ways(lambda s: m.kv_append(c.kv, c.pages, c.table, pos, q, k, v, _freq(64), stream=s), by_handle)
        _both_ways(lambda s: m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, want_lse=True, stream=s), by_handle)
        _both_ways(lambda s: m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, 9, want_lse=True, want_blocks=True, stream=s), by_handle)


def test_kv_outputs_of_the_caller(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [900, 40, 0], seed=5, summaries=True, max_sel=16)
    out, lse, blocks = m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, 9, want_lse=True, want_blocks=True)
    side = torch.cuda.Stream()
    for s in (None, side):
        o, l, b = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(blocks)
        torch.cuda.synchronize()
        got = m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, 9, out=o, lse=l, blocks=b, stream=s)
        torch.cuda.synchronize()
        assert got[0] is o and got[1] is l and got[2] is b
        assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(b, blocks)
        l.zero_()
        torch.cuda.synchronize()
        got = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, lse=l, stream=s)
        torch.cuda.synchronize()
        want = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, want_lse=True)
        assert got[1] is l and torch.equal(got[0], want[0]) and torch.equal(l, want[1])
    for bad in (dict(lse=lse[:2].contiguous()), dict(lse=lse.bfloat16()), dict(lse=lse.t().contiguous().t()), dict(blocks=blocks[..., :8].contiguous()),
                dict(blocks=blocks.long())):
        with pytest.raises(AssertionError):
            m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, 9, **bad)


@pytest.mark.parametrize("by_handle", [False, True])
def test_calls_of_the_expert_path(m, by_handle):  # noqa: F811
    cfg = mi.get_config("C2").scaled(L=2, H=512, I=192, N=8, prompt=16)
    L, E, k = cfg.L, cfg.E, cfg.k
    T, _, _ = mi.eamc_traces(cfg, threads=2)
    bank = pack_bank(m, cfg, mi.expert_bank(cfg, 4, threads=2))
    desc = m.ModelDesc.from_config(cfg)
    eamc = m.Eamc(desc, cfg.N)
    eamc.load(T)
    cache = m.Cache(desc, L * E)
    for s in range(L * E + L * cfg.n_shared):
        t = cache.slot_tensor(s)
        t.copy_(dev(bank[s % 4]).view(t.dtype))
    cache.reset(L * E)
    reqs = [mi.make_request(cfg, b, decode=1) for b in range(3)]
    eam = dev(np.stack([r.prefill_eam for r in reqs]).astype(np.int32))
    x = dev(np.stack([r.x[0, 0] for r in reqs]))
    logits = torch.randn((3, E), device="cuda")
    idx, w = m.moe_route_topk(logits, k, bool(cfg.renorm))
    best, _, _ = m.eamc_match(eamc, eam)
    W, bias = dev(mi.router_weights(cfg, 0)), dev(reqs[0].bias[0])
    _both_ways(lambda s: m.moe_route_topk(logits, k, bool(cfg.renorm), stream=s), by_handle)
    _both_ways(lambda s: m.eamc_match(eamc, eam, want_sims=True, stream=s), by_handle)
    _both_ways(lambda s: m.eamc_match_topm(eamc, eam[0].contiguous(), 4, want_sims=True, stream=s), by_handle)
    _both_ways(lambda s: m.expert_priority(eamc, best, 0, cache.slot_table(), EPS, idx, stream=s)[:2], by_handle)  # (the orders are filled in part)
    _both_ways(lambda s: m.expert_ffn_gemv(cache, idx[0], w[0], x[0], stream=s), by_handle)
    _both_ways(lambda s: m.expert_ffn_grouped(cache, 0, idx, w, x, stream=s), by_handle)

    def prefill(s):
        counts = eam[0].clone()  # (updated in place)
        torch.cuda.synchronize()
        return m.moe_prefill_layer(cache, counts, 0, W, bias, x, want_picks=True, stream=s)

    _both_ways(prefill, by_handle)
    assert cache.error_flags() == 0
    cache.close()
    eamc.close()


def test_kv_outputs_have_the_documented_shape(m):  # noqa: F811
    # queries may be any contiguous tensor of a call's elements, as projections leave them: outputs are [B][Hq][v_dim] all the same
    for Dv in (64, 48):
        c = Case(m, "bf16", 4, 2, 64, Dv, 16, [90, 40, 1], seed=Dv, summaries=True, max_sel=6)
        want = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale)
        for q in (c.q, c.q.view(3, 256), c.q.view(3, 1, 256), c.q.view(1, 3, 4, 64), c.q.view(-1)):
            out = m.kv_attend(c.kv, c.pages, c.table, c.len_t, q, c.scale)
            few = m.kv_attend_blocks(c.kv, c.pages, c.table, c.len_t, q, c.scale, 6)
            assert torch.equal(out, want) and torch.equal(few, want) and out.shape == few.shape == (3, 4, Dv)
