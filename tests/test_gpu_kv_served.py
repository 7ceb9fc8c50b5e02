"""The calls of a served cache together, as a decode loop makes them: requests that share a prompt, keys normed and turned by their positions,
weights added up over the steps, eviction to other pages, and on from there.  Every step against the definitions in 64 bits on what the pages hold by then; tolerances are those
of the calls' own tests.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.test_gpu_kv import E, HALF, _freq, bits, host, m  # noqa: F401 (a fixture)
from tests.test_gpu_streams import _both_ways

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE = 4, 2, 64, 16


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


class Server:
    def __init__(self, m, dtype, B, width, seed):  # noqa: F811
        self.m, self.dtype, self.B, self.width = m, dtype, B, width
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.kv = m.Kv(HQ, HKV, D, D, PAGE, dtype, max_batch=B, max_pages=width, max_sel=0, shared=True, max_weight_tokens=B * width * PAGE)
        self.n_pages = 2 * B * width
        self.k, self.v = (torch.zeros((self.n_pages, HKV, PAGE, D), device="cuda").to(self.kv.page_dtype) for _ in range(2))
        self.scales = {} if dtype != "fp8" else {n: torch.full((HKV,), x, device="cuda") for n, x in (("k_scale", 0.05), ("v_scale", 0.03))}
        self.pages = m.KvPages(self.kv, self.k, self.v, **self.scales)
        self.free = torch.randperm(self.n_pages, generator=self.g, device="cuda").tolist()
        self.qw, self.kw = (1.0 + 0.3 * torch.randn(D, generator=self.g, device="cuda") for _ in range(2))
        self.freq, self.scale = _freq(D), D ** -0.5

    def take(self, n):
        got, self.free = self.free[:n], self.free[n:]
        return got

    def tokens(self, T):
        return [(2 * torch.randn((T, h, D), generator=self.g, device="cuda")).to(self.kv.dtype) for h in (HQ, HKV, HKV)]

    def append(self, table, pos, seq=None, turn=None):
        q, k, v = self.tokens(len(pos))
        out = self.m.kv_append_norm(self.kv, self.pages, table, ints(pos), q, k, v, self.qw, self.kw, self.freq,
                                    seq=None if seq is None else ints(seq), turn=None if turn is None else ints(turn))
        at = pos if turn is None else turn
        want = O.rotate(O.norm(host(q), host(self.qw), float(np.float32(1e-6))), at, host(self.freq), False)
        io = "fp32" if self.dtype == "fp32" else "bf16"
        assert (np.abs(host(out) - want) <= HALF[io] * np.abs(want) + 2.0 ** -18 * np.abs(want).max()).all()
        return out

    def oracle(self, what, q, table, lens, *args):
        scales = {n: host(t) for n, t in self.scales.items()}
        return what(host(q), host(self.k), host(self.v), table.cpu().numpy(), lens, self.scale, *args, **scales)

    def bound(self, ref, q, lens):
        k, v = np.abs(host(self.k)).sum(-1).max(), np.abs(host(self.v)).max()
        if self.scales:
            k, v = k * 0.05, v * 0.03
        dz = (D + 4) * E * np.abs(host(q)).max() * k * self.scale + 2.0 ** -21
        n = max(lens)
        return (2 * dz + 2.0 ** -16 + (2 * n + 64) * E) * v + HALF["fp32" if self.dtype == "fp32" else "bf16"] * np.abs(ref), 2 * dz + 2.0 ** -20 + (n + 8) * E


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_a_served_batch(m, dtype):  # noqa: F811
    B, prompt, shared, keep = 5, 43, 32, 24
    s = Server(m, dtype, B, 8, seed=3)
    # the prompt's whole pages belong to all, and are written once; the rest of it is each request's own
    common = s.take(shared // PAGE)
    rows = [common + s.take(8 - len(common)) for _ in range(B)]
    table = torch.tensor(rows, dtype=torch.int32, device="cuda")
    s.append(table, list(range(shared)), seq=[0] * shared)
    own = [(b, p) for b in range(B) for p in range(shared, prompt - b)]
    s.append(table, [p for _, p in own], seq=[b for b, _ in own])
    lens, gone = [prompt - b for b in range(B)], [0] * B
    weights = torch.zeros((B, HKV, 8 * PAGE), device="cuda")
    expected = np.zeros((B, HKV, 8 * PAGE))
    slack = np.zeros((B, HKV, 8 * PAGE))
    starts, prefix = ints([0, B]), ints([shared])
    for step in range(40):
        q = s.append(table, lens, turn=[n + x for n, x in zip(lens, gone)])
        lens = [n + 1 for n in lens]
        now = ints(lens)
        ref, ref_lse = s.oracle(O.attend, q, table, lens)
        tol, rel = s.bound(ref, q, lens)
        out, lse = m.kv_attend_shared(s.kv, s.pages, table, now, starts, prefix, q, s.scale, want_lse=True)
        assert (np.abs(host(out) - ref) <= tol).all() and (np.abs(host(lse) - ref_lse) <= rel).all()
        out, lse = m.kv_attend_weights(s.kv, s.pages, table, now, q, s.scale, weights, want_lse=True)
        assert (np.abs(host(out) - ref) <= tol).all() and (np.abs(host(lse) - ref_lse) <= rel).all()
        given = O.attend_weights(host(q), host(s.k), table.cpu().numpy(), lens, ref_lse, s.scale, **({"k_scale": host(s.scales["k_scale"])} if s.scales else {}))
        expected, slack = expected + given, slack + rel * given + 3 * E * (expected + given)
        assert (np.abs(host(weights) - expected) <= slack).all()
        if step == 20:  # what every head gave least to goes; the pages that were shared stay with nobody here
            w, k, v = host(weights), s.k.clone(), s.v.clone()
            fresh = torch.tensor([s.take(8) for _ in range(B)], dtype=torch.int32, device="cuda")
            to_weights = torch.zeros((B, HKV, 8 * PAGE), device="cuda")
            to_lens, kept = m.kv_evict(s.kv, s.pages, table, now, weights, keep, fresh, to_weights, keep_first=2, keep_last=5)
            assert to_lens.tolist() == [keep] * B
            new_expected, new_slack = np.zeros_like(expected), np.zeros_like(slack)
            for b in range(B):
                for hk in range(HKV):
                    chosen = O.keep(w[b, hk], lens[b], keep, 2, 5)
                    assert kept[b, hk].tolist() == chosen
                    new_expected[b, hk, :keep], new_slack[b, hk, :keep] = expected[b, hk, chosen], slack[b, hk, chosen]
                    for i, j in enumerate(chosen):
                        a, z = int(table[b, j // PAGE]), int(fresh[b, i // PAGE])
                        assert (bits(s.k[z, hk, i % PAGE]) == bits(k[a, hk, j % PAGE])).all() and (bits(s.v[z, hk, i % PAGE]) == bits(v[a, hk, j % PAGE])).all()
            gone = [g + n - keep for g, n in zip(gone, lens)]
            table, weights, lens = fresh, to_weights, [keep] * B
            expected, slack = new_expected, new_slack
            starts, prefix = ints([0]), ints([])
    assert s.kv.error_flags() == 0


def test_outputs_belong_to_the_stream_of_the_call(m):  # noqa: F811
    s = Server(m, "bf16", 3, 8, seed=1)
    table = torch.tensor([s.take(8) for _ in range(3)], dtype=torch.int32, device="cuda")
    s.append(table, [p for _ in range(3) for p in range(100)], seq=[b for b in range(3) for _ in range(100)])
    q, k, v = s.tokens(3)
    lens, pos, to_table = ints([100, 90, 1]), ints([100, 90, 1]), torch.tensor([s.take(2) for _ in range(3)], dtype=torch.int32, device="cuda")
    weights = torch.zeros((3, HKV, 8 * PAGE), device="cuda")
    starts, prefix = ints([0, 2, 3]), ints([80, 0])
    for by_handle in (False, True):
        _both_ways(lambda st: m.kv_append_norm(s.kv, s.pages, table, pos, q, k, v, s.qw, s.kw, s.freq, stream=st), by_handle)
        _both_ways(lambda st: m.kv_attend_shared(s.kv, s.pages, table, lens, starts, prefix, q, s.scale, want_lse=True, stream=st), by_handle)
        _both_ways(lambda st: m.kv_attend_weights(s.kv, s.pages, table, lens, q, s.scale, weights, want_lse=True, stream=st), by_handle)
        w = torch.rand_like(weights)
        torch.cuda.synchronize()
        _both_ways(lambda st: m.kv_evict(s.kv, s.pages, table, lens, w, 20, to_table, stream=st), by_handle)
    for out, lse in ((torch.zeros_like(q), torch.zeros((3, HQ), device="cuda")),):
        got = m.kv_attend_shared(s.kv, s.pages, table, lens, starts, prefix, q, s.scale, out=out, lse=lse)
        assert got[0] is out and got[1] is lse
        want = m.kv_attend_shared(s.kv, s.pages, table, lens, starts, prefix, q, s.scale)
        assert torch.equal(out, want)
        got = m.kv_attend_weights(s.kv, s.pages, table, lens, q, s.scale, weights, out=out, lse=lse)
        assert got[0] is out and got[1] is lse
    to_lens, kept = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((3, HKV, 20), dtype=torch.int32, device="cuda")
    got = m.kv_evict(s.kv, s.pages, table, lens, w, 20, to_table, to_lens=to_lens, kept=kept)
    assert got[0] is to_lens and got[1] is kept and to_lens.tolist() == [20, 20, 1]


def test_two_handles_on_two_streams_at_once(m):  # noqa: F811
    both = []
    for seed in (1, 2):
        s = Server(m, "bf16", 6, 64, seed=seed)
        table = torch.tensor([s.take(64) for _ in range(6)], dtype=torch.int32, device="cuda")
        s.k.copy_(torch.randn(s.k.shape, generator=s.g, device="cuda"))
        s.v.copy_(torch.randn(s.v.shape, generator=s.g, device="cuda"))
        q = s.tokens(6)[0]
        args = dict(s=s, table=table, q=q, lens=ints([1000, 700, 1024, 3, 900, 650]), starts=ints([0, 3, 6]), prefix=ints([600, 640]),
                    w=torch.zeros((6, HKV, 64 * PAGE), device="cuda"), fresh=torch.tensor([s.take(10) for _ in range(6)], dtype=torch.int32, device="cuda"))

        def steps(x=args):
            s, got = x["s"], []
            x["w"].zero_()
            got += m.kv_attend_shared(s.kv, s.pages, x["table"], x["lens"], x["starts"], x["prefix"], x["q"], s.scale, want_lse=True)
            got += m.kv_attend_weights(s.kv, s.pages, x["table"], x["lens"], x["q"], s.scale, x["w"], want_lse=True)
            got += m.kv_evict(s.kv, s.pages, x["table"], x["lens"], x["w"], 150, x["fresh"])
            return got + [x["w"].clone()]
        both.append((steps, [bits(t) for t in steps()]))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    results = [[], []]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                results[i].append(both[i][0]())
    torch.cuda.synchronize()
    for i in (0, 1):
        for got in results[i]:
            for t, w in zip(got, both[i][1]):
                assert (bits(t) == w).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages_beyond_32_bits(m, dtype):  # noqa: F811
    # a pool of more than 2^32 bytes and elements; its last pages
    n_pages = (1 << 32) // (16 * 256) // (1 if dtype == "bf16" else 2) + 40
    kv = m.Kv(2, 1, 256, 256, 16, dtype, max_batch=2, max_pages=8, max_sel=0, shared=True, max_weight_tokens=2 * 128)
    k, v = (torch.empty((n_pages, 1, 16, 256), dtype=kv.page_dtype, device="cuda") for _ in range(2))
    pages = m.KvPages(kv, k, v)
    rows = [[n_pages - 1 - 8 * b - i for i in range(8)] for b in range(2)]
    table = torch.tensor(rows, dtype=torch.int32, device="cuda")
    for r in rows:
        for p in r:
            k[p], v[p] = torch.randn((1, 16, 256), device="cuda"), torch.randn((1, 16, 256), device="cuda")
    q = torch.randn((2, 2, 256), device="cuda").to(kv.dtype)
    low = table - (n_pages - 16)                      # the same pages in a small pool
    small = m.KvPages(kv, k[n_pages - 16:].clone(), v[n_pages - 16:].clone())
    lens, starts, prefix = ints([120, 100]), ints([0, 2]), ints([64])
    w = [torch.zeros((2, 1, 128), device="cuda") for _ in range(2)]
    got = [m.kv_attend_shared(kv, p, t, lens, starts, prefix, q, 0.0625, want_lse=True) + m.kv_attend_weights(kv, p, t, lens, q, 0.0625, x, want_lse=True)
           for p, t, x in ((pages, table, w[0]), (small, low, w[1]))]
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.equal(*w)
    to = torch.tensor([[n_pages - 20, n_pages - 21], [n_pages - 22, n_pages - 23]], dtype=torch.int32, device="cuda")
    _, kept = m.kv_evict(kv, pages, table, lens, w[0], 30, to)
    for b in range(2):
        for i, j in enumerate(kept[b, 0].tolist()):
            assert torch.equal(k[int(to[b, i // 16]), 0, i % 16], k[rows[b][j // 16], 0, j % 16]) and torch.equal(v[int(to[b, i // 16]), 0, i % 16], v[rows[b][j // 16], 0, j % 16])
    x = torch.randn((2, 1, 256), device="cuda").to(kv.dtype)
    ones = torch.ones(256, device="cuda")
    m.kv_append_norm(kv, pages, table, ints([127, 111]), q, x, x, ones, ones, None)
    assert torch.equal(v[rows[0][7], 0, 15], x[0, 0]) and torch.equal(v[rows[1][6], 0, 15], x[1, 0])
    want = O.norm(host(x), np.ones(256), float(np.float32(1e-6)))
    assert (np.abs(host(k[rows[0][7], 0, 15]) - want[0, 0]) <= HALF[dtype] * np.abs(want[0, 0]) + 2.0 ** -19 * np.abs(want).max()).all()
    assert kv.error_flags() == 0


def test_scratch_that_is_there_stays_where_a_captured_graph_finds_it(m):  # noqa: F811
    s = Server(m, "bf16", 3, 20, seed=5)
    s.k.copy_(torch.randn(s.k.shape, generator=s.g, device="cuda"))
    s.v.copy_(torch.randn(s.v.shape, generator=s.g, device="cuda"))
    table, lens = ints(s.take(3 * 20)).view(3, 20), ints([300, 310, 290])
    q, starts, prefix = torch.randn((3, HQ, D), generator=s.g, device="cuda").bfloat16(), ints([0, 3]), ints([250])
    w = torch.zeros((3, HKV, 20 * PAGE), device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]

    def steps(outs):
        s.m.kv_attend_shared(s.kv, s.pages, table, lens, starts, prefix, q, s.scale, out=outs[0])
        s.m.kv_attend_weights(s.kv, s.pages, table, lens, q, s.scale, w, out=outs[1])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(outs)
    for i in range(4):
        torch.cuda.synchronize()
        s.kv.set_shared(True)
        s.kv.set_weights(3 * 20 * PAGE)
        other = torch.full((64 << 20,), 7, dtype=torch.uint8, device="cuda")  # what would lie where scratch had been
        q.copy_(torch.randn(q.shape, generator=s.g, device="cuda"))
        w.zero_()
        graph.replay()
        got, got_w = [x.clone() for x in outs], w.clone()
        w.zero_()
        want = [torch.empty_like(q) for _ in range(2)]
        steps(want)
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(got_w, w) and (other == 7).all()
