"""Attention that adds up weights, and eviction by them, against the definitions in 64 bits (oracle/kv_oracle.py).

A weight is exp(z - lse): z is off by dz (tests/test_gpu_kv.py), the maximum and the sum behind it by as much and (n + 8) e, exp2 and its argument by
2^-21: (2 dz + 2^-20 + (n + 8) e) of the weight.  A group's heads are added in fp32 to each other and to what was there: (heads + 1) e of the sum.
What is kept, and every moved row and weight, is exact.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.test_gpu_kv import E, Case, _append_inputs, _freq, bits, host, m  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def rows_of(c, spare=0, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return scale * torch.rand((len(c.lens), c.kv.k_page[0], c.width * c.page + spare), generator=g, device="cuda")


def check_weights(c, weights, before, window=0, lens=None, table=None):
    q, k = host(c.q), np.nan_to_num(host(c.k))
    scales = {} if c.ks is None else dict(k_scale=host(c.ks))
    table, lens = (c.table if table is None else table).cpu().numpy(), lens or c.lens
    _, lse = c.oracle(window=window, lens=lens)
    want = O.attend_weights(q, host(c.k), table, lens, lse, c.scale, window=window, **scales)
    if c.ks is not None:
        k = k * host(c.ks)[None, :, None, None]
    dz = (q.shape[2] + 4) * E * np.abs(q).max() * np.abs(k).sum(-1).max() * c.scale + 2.0 ** -21
    n, group = max(max(lens), 1), q.shape[1] // c.kv.k_page[0]
    got, old = host(weights), host(before)
    room = want.shape[2]
    tol = (2 * dz + 2.0 ** -20 + (n + 8) * E) * want + (group + 1) * E * (want + np.abs(old[..., :room]))
    assert (np.abs(got[..., :room] - old[..., :room] - want) <= tol).all()
    nothing = np.ones_like(got, dtype=bool)
    for b, x in enumerate(lens):
        x = min(max(x, 0), room)
        nothing[b, :, max(0, x - window) if window else 0:x] = False
    same = (bits(weights).reshape(*got.shape, 4) == bits(before).reshape(*got.shape, 4)).all(-1)
    assert same[nothing].all()
    return want


WEIGHTS = [
    # dtype, Hq, Hkv, Dk, Dv, page, lens
    ("bf16", 1, 1, 64, 64, 16, [1]),
    ("bf16", 4, 1, 128, 128, 16, [1, 15, 16, 17]),
    ("bf16", 8, 2, 128, 128, 64, [0, 63, 64, 65, 700]),
    ("bf16", 6, 2, 80, 96, 32, [33, 0, 129]),
    ("bf16", 40, 2, 64, 64, 32, [257, 31]),          # twenty query heads a group: two passes
    ("bf16", 2, 2, 256, 256, 128, [129, 1000]),
    ("fp8", 8, 1, 128, 128, 16, [1, 31, 32, 33, 500]),
    ("fp8", 6, 2, 192, 128, 64, [65, 640]),
    ("fp8", 17, 1, 80, 48, 16, [49, 48]),
    ("fp32", 4, 2, 64, 64, 16, [0, 1, 40, 333]),
    ("fp32", 3, 1, 128, 112, 32, [65, 200]),
    ("fp32", 6, 2, 96, 80, 32, [1000, 31, 0, 65]),
    ("fp32", 5, 1, 256, 240, 64, [130, 64]),
    ("bf16", 4, 2, 64, 64, 16, [5000, 3, 2100, 1024, 1025]),
]


@pytest.mark.parametrize("spare", [0, 3])
@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,lens", WEIGHTS)
def test_attend_weights(m, dtype, Hq, Hkv, Dk, Dv, page, lens, spare):  # noqa: F811
    c = Case(m, dtype, Hq, Hkv, Dk, Dv, page, lens, seed=Dk + page)
    c.kv.set_weights(len(lens) * c.width * page)
    weights = rows_of(c, spare)
    before = weights.clone()
    want = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, want_lse=True)
    out, lse = m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, weights, want_lse=True)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    check_weights(c, weights, before)
    first = weights.clone()
    for _ in range(2):  # the same bits every run, and a step's weights add up to the heads of a group
        weights.copy_(before)
        assert torch.equal(m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, weights), want[0])
        assert torch.equal(weights, first)
    got = (host(weights) - host(before)).sum(-1)
    some = np.array([n > 0 for n in lens])
    assert (np.abs(got[some] - Hq // Hkv) <= 2.0 ** -10 * (Hq // Hkv)).all() and (got[~some] == 0).all()
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("window", [1, 16, 17, 100, 5000])
def test_weights_of_a_window(m, dtype, window):  # noqa: F811
    c = Case(m, dtype, 4, 2, 64, 64, 16, [0, 1, 17, 300, 2500], seed=window)
    c.kv.set_weights(5 * c.width * 16)
    weights = rows_of(c)
    before = weights.clone()
    want = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, window=window)
    assert torch.equal(m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, weights, window=window), want)
    check_weights(c, weights, before, window=window)


@pytest.mark.parametrize("B,top", [(1, 40000), (65, 300), (300, 40)])
def test_weights_of_batches_of_any_size(m, B, top):  # noqa: F811
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, top, B)] if B > 1 else [top]
    c = Case(m, "bf16", 4, 2, 64, 64, 16, lens, seed=B)
    c.kv.set_weights(B * c.width * 16)
    weights = rows_of(c, 1)
    before = weights.clone()
    m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, weights)
    check_weights(c, weights, before)


@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,lens,window", [
    ("bf16", 16, 1, 128, 128, 32, [40000], 0),
    ("bf16", 40, 1, 64, 64, 64, [30001, 17], 0),
    ("fp8", 12, 1, 192, 128, 32, [50000], 0),
    ("fp8", 16, 2, 128, 128, 16, [40000], 33333),
    ("fp32", 16, 1, 256, 256, 32, [9000, 8875, 611], 0),
])
def test_weights_of_few_long_sequences(m, dtype, Hq, Hkv, Dk, Dv, page, lens, window):  # noqa: F811
    # fewer workgroups than fit the card, whose parts one of them joins
    c = Case(m, dtype, Hq, Hkv, Dk, Dv, page, lens, seed=Hq)
    c.kv.set_weights(len(lens) * c.width * page)
    weights = rows_of(c)
    before = weights.clone()
    out, lse = m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, weights, window=window, want_lse=True)
    c.check(out, lse, *c.oracle(window=window))
    check_weights(c, weights, before, window=window)
    first = weights.clone()
    weights.copy_(before)
    assert torch.equal(m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, weights, window=window), out)
    assert torch.equal(weights, first)


def test_weights_of_bad_pages_and_lengths(m):  # noqa: F811
    for dtype in ("bf16", "fp8", "fp32"):
        c = Case(m, dtype, 4, 2, 64, 64, 16, [200, 210, 16, 60], seed=2)
        c.kv.set_weights(4 * c.width * 16)
        c.table[0, 3], c.table[1, 13], c.table[2, 0] = -1, c.n_pages, 2 ** 31 - 1
        c.table[3] = c.table[3, 0]
        lens = [200, 210, 16, c.width * 16 + 5]
        weights = rows_of(c)
        before = weights.clone()
        m.kv_attend_weights(c.kv, c.pages, c.table, ints(lens), c.q, c.scale, weights)
        assert c.kv.error_flags() == 3
        check_weights(c, weights, before, lens=lens)
        assert torch.equal(weights[2], before[2])
        m.kv_attend_weights(c.kv, c.pages, c.table, ints([-3, 0, 0, 0]), c.q, c.scale, weights)
        assert c.kv.error_flags() == 2


def test_weights_are_refused_without_room(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [200, 60], seed=2)
    weights = rows_of(c)
    args = (c.kv, c.pages, c.table, c.len_t, c.q, c.scale)

    def refused(text, error=None, code=None, args=args, weights=weights, **more):
        with pytest.raises(error or m.MoeiError) as e:
            m.kv_attend_weights(*args, weights, **more)
        assert text in str(e.value) and code in (None, getattr(e.value, "code", None))

    refused("moei_kv_set_weights", code=-5)
    c.kv.set_weights(2 * c.width * 16 - 1)
    refused("moei_kv_set_weights", code=-5)
    c.kv.set_weights(2 * c.width * 16)
    m.kv_attend_weights(*args, weights)
    refused("", AssertionError, weights=weights[..., :-1].contiguous())
    refused("", AssertionError, weights=weights[..., :-1])
    refused("", AssertionError, weights=weights.bfloat16())
    refused("", AssertionError, weights=weights[:1])
    refused("window", window=-1)
    refused("overlaps", out=weights.view(torch.bfloat16).flatten()[8:8 + c.q.numel()].view(2, 4, 64))
    refused("overlaps", lse=weights.flatten()[:8].view(2, 4))
    refused("overlaps", args=(*args[:4], weights.view(torch.bfloat16).flatten()[-c.q.numel():].view(2, 4, 64), c.scale))
    c.kv.set_weights(0)
    refused("moei_kv_set_weights", code=-5)
    with pytest.raises(m.MoeiError):
        c.kv.set_weights(-1)
    assert c.kv.max_weight_tokens == 0


# ------------------------------------------------------------------------------------------------ eviction
def evict(m, c, weights, n_keep, first, last, seed=0, summaries=False, to_width=None, with_weights=True):  # noqa: F811
    """The call on a copy of the pools with room for what is kept; checks all it writes, and that it writes nothing else."""
    B, page, Hkv = len(c.lens), c.page, c.kv.k_page[0]
    to_width = to_width or -(-n_keep // page)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    old = c.n_pages
    n_pages = old + B * to_width
    grown = [torch.cat([x, torch.randn((n_pages - old, *x.shape[1:]), generator=g, device="cuda").to(x.dtype)]) for x in (c.k, c.v)]
    lo = hi = None
    if summaries:
        lo, hi = (torch.zeros((n_pages, Hkv, c.k.shape[3]), dtype=c.kv.dtype, device="cuda") for _ in range(2))
    pages = m.KvPages(c.kv, *grown, k_min=lo, k_max=hi, k_scale=c.ks, v_scale=c.vs)
    to_table = (old + torch.randperm(B * to_width, generator=g, device="cuda")).to(torch.int32).view(B, to_width)
    to_weights = torch.randn((B, Hkv, to_width * page + 2), generator=g, device="cuda") if with_weights else None
    before = [x.clone() for x in grown]
    w_before = None if to_weights is None else host(to_weights)
    flags = c.kv.error_flags()
    to_lens, kept = m.kv_evict(c.kv, pages, c.table, c.len_t, weights, n_keep, to_table, to_weights, keep_first=first, keep_last=last)
    assert flags == 0
    table, to, w = c.table.cpu().numpy(), to_table.cpu().numpy(), weights.cpu().numpy()
    want, full = [x.cpu() for x in before], set()
    want_kept = np.full((B, Hkv, n_keep), -1)
    room = c.width * page
    for b, n in enumerate(c.len_t.tolist()):
        n = min(max(n, 0), room)
        assert int(to_lens[b]) == min(n, n_keep)
        for hk in range(Hkv):
            chosen = np.array(O.keep(w[b, hk], n, n_keep, first, last), dtype=np.int64)
            want_kept[b, hk, :len(chosen)] = chosen
            i = np.arange(len(chosen))
            if w_before is not None:
                w_before[b, hk, :len(chosen)] = w[b, hk, chosen]
            fp, tp = table[b, chosen // page], to[b, i // page]
            ok = (fp >= 0) & (fp < n_pages) & (tp >= 0) & (tp < n_pages)
            for x, y in zip(want, before):
                y = y.cpu()
                x.view(torch.uint8)[tp[ok], hk, (i % page)[ok]] = y.view(torch.uint8)[fp[ok], hk, (chosen % page)[ok]]
            full |= {int(p) for p in tp[page - 1::page]}
    assert (kept.cpu().numpy() == want_kept).all()
    for x, y in zip(grown, want):
        assert (bits(x) == y.contiguous().view(torch.uint8).numpy()).all()
    if to_weights is not None:
        got = host(to_weights)
        assert ((got == w_before) | (np.isnan(got) & np.isnan(w_before))).all()
    if summaries:
        for p in range(n_pages):
            keys = grown[0][p].to(c.kv.dtype)
            if p in full:
                assert torch.equal(lo[p], keys.amin(1)) and torch.equal(hi[p], keys.amax(1))
            else:
                assert (lo[p] == 0).all() and (hi[p] == 0).all()
    return pages, to_table, to_weights, to_lens, kept


EVICT = [
    # dtype, Hkv, Dk, Dv, page, lens, n_keep, first, last
    ("bf16", 2, 64, 64, 16, [100, 37, 0, 1, 36, 38], 37, 4, 8),
    ("bf16", 1, 128, 128, 64, [1000], 1, 0, 1),
    ("bf16", 1, 128, 128, 64, [1000, 2], 1, 0, 0),
    ("bf16", 3, 80, 96, 32, [3000, 129, 2048], 128, 0, 0),
    ("bf16", 2, 64, 64, 256, [2000, 1999], 700, 100, 600),   # nothing is chosen
    ("fp8", 2, 128, 128, 16, [500, 333], 100, 1, 5),
    ("fp8", 8, 16, 48, 32, [5000, 65, 64], 64, 10, 10),
    ("fp32", 2, 64, 32, 16, [333, 50], 49, 4, 4),
    ("fp32", 1, 256, 256, 128, [700], 256, 0, 255),
    ("bf16", 1, 16, 16, 16, [30000], 20000, 16, 1000),
    ("bf16", 1, 16, 16, 16, [70000, 65536, 17], 999, 3, 30),
]


@pytest.mark.parametrize("summaries", [False, True])
@pytest.mark.parametrize("dtype,Hkv,Dk,Dv,page,lens,n_keep,first,last", EVICT)
def test_evict(m, dtype, Hkv, Dk, Dv, page, lens, n_keep, first, last, summaries):  # noqa: F811
    c = Case(m, dtype, 2 * Hkv, Hkv, Dk, Dv, page, lens, seed=Dk + page, nan_tail=False)
    evict(m, c, rows_of(c, 3), n_keep, first, last, summaries=summaries, to_width=min(c.width, -(-n_keep // page) + 1) if c.width * page >= n_keep else None)
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("what", ["equal", "few", "special", "zeros", "negative", "bits", "low bits"])
def test_equal_and_special_weights(m, what):  # noqa: F811
    c = Case(m, "bf16", 2, 2, 16, 16, 16, [5000, 1300, 64], seed=1, nan_tail=False)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    w = rows_of(c)
    if what == "equal":
        w.fill_(0.25)
    elif what == "few":
        w = torch.randint(0, 3, w.shape, generator=g, device="cuda").float()
    elif what == "special":
        pick = torch.randint(0, 8, w.shape, generator=g, device="cuda")
        for i, x in enumerate((float("nan"), float("inf"), -float("inf"), -float("nan"), 1e-45, -1e-45, 3e38)):
            w[pick == i] = x
    elif what == "zeros":
        w = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.5, torch.zeros_like(w), -torch.zeros_like(w))
    elif what == "negative":
        w = -torch.rand(w.shape, generator=g, device="cuda").pow(8)
    elif what == "bits":
        w = torch.randint(0, 2 ** 31 - 2 ** 24, w.shape, generator=g, device="cuda", dtype=torch.int32).view(torch.float32).contiguous()
    else:
        w = (torch.randint(0, 900, w.shape, generator=g, device="cuda", dtype=torch.int32) + 0x3f800000).view(torch.float32).contiguous()
    for n_keep, first, last in ((1, 0, 0), (333, 5, 64), (1299, 0, 1)):
        evict(m, c, w, n_keep, first, last)


@pytest.mark.parametrize("B,Hkv,top", [(3, 1, 70000), (3, 43, 20000), (2, 16, 30000), (130, 1, 16500), (2, 64, 16385)])
@pytest.mark.parametrize("what", ["spread", "equal", "few"])
def test_long_sequences(m, B, Hkv, top, what):  # noqa: F811
    # more tokens than a workgroup holds: chosen from by several workgroups, or where there are many heads by one that reads the weights again and again
    rng = np.random.default_rng(B)
    lens = [top, *(int(x) for x in rng.integers(0, top // 8, B - 1))]
    c = Case(m, "fp8", Hkv, Hkv, 16, 16, 256, lens, seed=1, nan_tail=False)
    w = rows_of(c)
    w = {"spread": w, "equal": torch.full_like(w, 0.5), "few": torch.round(w * 3)}[what]
    for _ in range(2):  # what the choice keeps in memory is as it was
        evict(m, c, w, 1999, 3, 130)


def test_evict_bad_pages_and_lengths(m):  # noqa: F811
    c = Case(m, "bf16", 2, 2, 64, 64, 16, [100, 90, 80, 70], seed=1, nan_tail=False)
    w = rows_of(c)
    c.len_t.copy_(ints([100, -4, 80, 70]))
    evict(m, c, w, 33, 2, 2)
    assert c.kv.error_flags() == 2
    c.len_t.copy_(ints([100, 90, 2 ** 31 - 1, 70]))
    c.table[2] = c.table[0]
    evict(m, c, w, 33, 2, 2)
    assert c.kv.error_flags() == 2
    c.len_t.copy_(ints([100, 90, 80, 70]))
    c.table[0, 0], c.table[1, 3], c.table[3, 4] = -1, 2 ** 31 - 1, 10 ** 6
    evict(m, c, w, 33, 2, 2)
    assert c.kv.error_flags() == 1


def test_evict_without_weights_to_keep_and_pages_that_lie_apart(m):  # noqa: F811
    c = Case(m, "bf16", 2, 2, 64, 48, 16, [100, 90], seed=1, nan_tail=False)
    evict(m, c, rows_of(c), 33, 2, 2, with_weights=False)
    for dtype in ("bf16", "fp8", "fp32"):
        c = Case(m, dtype, 2, 2, 64, 48, 16, [100, 40], seed=1, nan_tail=False, gap=48, spare=8)
        w, k, v = rows_of(c), c.k.clone(), c.v.clone()
        to_table = c.spare[:6].view(2, 3).contiguous()
        to_lens, kept = m.kv_evict(c.kv, c.pages, c.table, c.len_t, w, 35, to_table, keep_first=1, keep_last=1)
        for b, n in enumerate(c.lens):
            for hk in range(2):
                chosen = O.keep(host(w)[b, hk], n, 35, 1, 1)
                assert kept[b, hk].tolist() == chosen
                for i, j in enumerate(chosen):
                    a, z = int(c.table[b, j // 16]), int(to_table[b, i // 16])
                    assert (bits(c.k[z, hk, i % 16]) == bits(k[a, hk, j % 16])).all() and (bits(c.v[z, hk, i % 16]) == bits(v[a, hk, j % 16])).all()
                    k[z, hk, i % 16], v[z, hk, i % 16] = k[a, hk, j % 16], v[a, hk, j % 16]
        assert (bits(c.k) == bits(k)).all() and (bits(c.v) == bits(v)).all()


def test_evict_refusals(m):  # noqa: F811
    c = Case(m, "bf16", 2, 2, 64, 64, 16, [100, 90], seed=1, nan_tail=False, spare=9)
    w, to_table = rows_of(c), c.spare[:6].view(2, 3).contiguous()
    before = bits(c.k)

    def refused(text, error=None, n_keep=33, lens=c.len_t, weights=w, table=c.table, to=to_table, **more):
        with pytest.raises(error or m.MoeiError) as e:
            m.kv_evict(c.kv, c.pages, table, lens, weights, n_keep, to, **more)
        assert text in str(e.value)

    refused("keep_first", n_keep=0)
    refused("keep_first", keep_first=-1)
    refused("keep_first", keep_last=-1)
    refused("keep_first", keep_first=30, keep_last=4)
    refused("keep_first", keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1)
    refused("hold", n_keep=49)
    refused("hold", to=torch.zeros((2, c.width + 1), dtype=torch.int32, device="cuda"))
    refused("d_to_len", to_lens=c.len_t)
    refused("d_to_weights", to_weights=w)
    refused("d_to_table", to=c.table, n_keep=33)
    for other in (w, c.table, to_table, c.len_t):  # (a buffer that begins with the other's last element)
        room = torch.zeros(2 ** 16, dtype=torch.int32, device="cuda")
        moved = room[:other.numel()].view(other.dtype).view(other.shape).copy_(other)
        kept = room[other.numel() - 1:other.numel() - 1 + 2 * 2 * 33].view(2, 2, 33)
        refused("d_kept", kept=kept, **{"weights" if other is w else "table" if other is c.table else "to" if other is to_table else "lens": moved})
    both = torch.zeros(2 * 2 * 33 + 1, dtype=torch.int32, device="cuda")
    refused("d_kept", kept=both[1:].view(2, 2, 33), to_lens=both[:2])
    refused("d_kept", kept=both[:-1].view(2, 2, 33), to_weights=both[1:].view(torch.float32).view(2, 2, 33))
    refused("", AssertionError, weights=w[..., :-1].contiguous())
    refused("", AssertionError, to_weights=w[..., :32].contiguous())
    refused("", AssertionError, to=to_table[:1])
    refused("", AssertionError, lens=c.len_t.long())
    refused("", AssertionError, kept=torch.zeros((2, 2, 32), dtype=torch.int32, device="cuda"))
    refused("", AssertionError, to_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert (bits(c.k) == before).all()


def test_captured_replayed_and_on_another_stream(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [300, 40, 1500], seed=1, nan_tail=False, spare=3 * 8)
    c.kv.set_weights(3 * c.width * 16)
    w, to_table = rows_of(c, scale=0.01), c.spare[:24].view(3, 8).contiguous()
    to_w, to_lens, kept = torch.zeros((3, 2, 128), device="cuda"), ints([0, 0, 0]), torch.zeros((3, 2, 120), dtype=torch.int32, device="cuda")
    out = torch.empty_like(c.q)

    def steps():
        m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, w, out=out)
        m.kv_evict(c.kv, c.pages, c.table, c.len_t, w, 120, to_table, to_w, keep_first=2, keep_last=8, to_lens=to_lens, kept=kept)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps()
    for i in range(4):
        c.q.copy_(torch.randn_like(c.q))
        c.len_t.copy_(ints([300 - i, 40 + i, 1400 + i]))
        start = w.clone()
        graph.replay()
        got = [bits(x) for x in (w, to_w, to_lens, kept, out, c.k, c.v)]
        w.copy_(start)
        for x in (to_lens, kept, out):
            x.zero_()
        if i < 2:
            steps()
        else:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                steps()
            torch.cuda.current_stream().wait_stream(side)
        for x, y in zip((w, to_w, to_lens, kept, out, c.k, c.v), got):
            assert (bits(x) == y).all()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = m.kv_evict(c.kv, c.pages, c.table, c.len_t, w, 120, to_table, to_w, keep_first=2, keep_last=8, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], to_lens) and torch.equal(got[1], kept)


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_summaries_of_full_pages_whose_last_row_was_not_moved(m, dtype):  # noqa: F811
    # a full page's summary is that of all it holds, moved or not: the first one's first 16 have no old page, the second one's second 16, of the third one's first page the last
    c = Case(m, dtype, 2, 2, 64, 64, 16, [100, 100, 100, 40], seed=1, nan_tail=False)
    c.table[0, 0], c.table[1, 1], c.table[2, 2] = -1, 2 ** 31 - 1, 10 ** 6
    w = torch.zeros_like(rows_of(c))
    w[2, :, :15] = w[2, 0, 40] = w[2, 1, 45] = w[2, :, 48:72] = 1.0
    evict(m, c, w, 40, 0, 0, summaries=True)
    assert c.kv.error_flags() == 1


def test_evict_refuses_outputs_over_what_it_reads(m):  # noqa: F811
    c = Case(m, "bf16", 2, 2, 64, 64, 16, [100, 90], seed=1, nan_tail=False, spare=9)
    given = dict(weights=rows_of(c), table=c.table, to=c.spare[:6].view(2, 3).contiguous(), lens=c.len_t)
    before = bits(c.k), bits(c.v)

    def refused(text, weights, table, to, lens, **more):
        with pytest.raises(m.MoeiError) as e:
            m.kv_evict(c.kv, c.pages, table, lens, weights, 33, to, **more)
        assert text in str(e.value)

    for name, other in given.items():  # (an output that begins with the other's last element, or ends with its first)
        for at_end in (True, False):
            for text, n, dtype, shape in (("d_to_len", 2, torch.int32, (2,)), ("d_to_weights", 2 * 2 * 33, torch.float32, (2, 2, 33))):
                room = torch.zeros(n + other.numel() - 1, dtype=torch.int32, device="cuda")
                at, to = (0, other.numel() - 1) if at_end else (n - 1, 0)
                moved = room[at:at + other.numel()].view(other.dtype).view(other.shape).copy_(other)
                output = room[to:to + n].view(dtype).view(shape)
                refused(text, **{**given, name: moved}, **{"to_lens" if text == "d_to_len" else "to_weights": output})
    room = torch.zeros(2 * 2 * 33 + 1, device="cuda")
    refused("d_to_len", **given, to_weights=room[:-1].view(2, 2, 33), to_lens=room[-2:].view(torch.int32))
    refused("d_to_len", **given, to_weights=room[1:].view(2, 2, 33), to_lens=room[:2].view(torch.int32))
    torch.cuda.synchronize()
    assert (bits(c.k) == before[0]).all() and (bits(c.v) == before[1]).all()


@pytest.mark.parametrize("B,Hkv,width,lens,n_keep", [
    (1, 1, 5100, [1_305_000], 1999),                                                   # more tokens than so many workgroups take in the smallest stretches
    (16, 8, 430, [110_080, 3, 0, 2000, 9_999, *range(400, 1500, 100)], 333),     # as many rows as several workgroups choose from, most of them short
])
@pytest.mark.parametrize("what", ["spread", "few"])
def test_the_widest_choices_by_several_workgroups(m, B, Hkv, width, lens, n_keep, what):  # noqa: F811
    c = Case(m, "fp8", Hkv, Hkv, 16, 16, 256, lens, seed=1, nan_tail=False, width=width, max_sel=0)
    w = rows_of(c)
    w = w if what == "spread" else torch.round(w * 3)
    for _ in range(2):  # what the choice keeps in memory is as it was
        evict(m, c, w, n_keep, 3, 130)
    assert c.kv.error_flags() == 0


def test_weights_that_are_no_numbers_of_either_kind_and_sign(m):  # noqa: F811
    # quiet and signalling ones with every sign, and the numbers beside them
    c = Case(m, "bf16", 2, 2, 16, 16, 16, [3000, 20_000], seed=1, nan_tail=False)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    odd = torch.tensor([0x7f800001, 0x7fbfffff, 0x7fc00000, 0x7fffffff, 0x7f800000, 0x7f7fffff, 1, 0, 0x007fffff, 0x00800000], dtype=torch.int64, device="cuda")
    odd = torch.cat([odd, odd - 2 ** 31]).to(torch.int32)
    w = rows_of(c)
    w = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.7, odd[torch.randint(0, 20, w.shape, generator=g, device="cuda")], w.view(torch.int32)).view(torch.float32)
    for n_keep in (1, 500, 1700, 2900):
        evict(m, c, w.contiguous(), n_keep, 0, 0)


def test_weights_and_eviction_of_the_largest_batch(m):  # noqa: F811
    rng = np.random.default_rng(6)
    c = Case(m, "bf16", 2, 1, 16, 16, 16, [int(x) for x in rng.integers(0, 60, 4096)], seed=6, nan_tail=False, max_sel=0)
    c.kv.set_weights(4096 * c.width * 16)
    w = rows_of(c)
    before = w.clone()
    m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, w)
    check_weights(c, w, before)
    evict(m, c, w, 20, 2, 3)
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("dtype,Hq,Hkv", [("bf16", 1024, 1), ("fp32", 1024, 2), ("fp8", 1024, 1024)])
def test_weights_and_eviction_of_1024_heads(m, dtype, Hq, Hkv):  # noqa: F811
    c = Case(m, dtype, Hq, Hkv, 16, 16, 16, [100, 33], seed=6, nan_tail=False, max_sel=0)
    c.kv.set_weights(2 * c.width * 16)
    w = rows_of(c)
    before = w.clone()
    m.kv_attend_weights(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, w)
    check_weights(c, w, before)
    evict(m, c, w, 35, 2, 3)
