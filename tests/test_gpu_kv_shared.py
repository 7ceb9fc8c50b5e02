"""Attention of a batch whose sequences share prefixes, against the definition in 64 bits (oracle/kv_oracle.py).

Tolerances are those of tests/test_gpu_kv.py, with twice the roundings of sums: a part of a prefix is a sum of its tokens, and joining it costs three
roundings more, for 32 tokens at least, or for the whole prefix: (2 n + 64) e of the largest value.  2^-16 of a weight is allowed for products of bf16 values as there,
though weights of prefixes enter them whole: test_weights_of_prefixes_keep_24_bits does without.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.test_gpu_kv import E, Case, bits, host, m  # noqa: F401 (a fixture)
from tests.test_gpu_kv_exact import bf16, e4m3, logits_whose_weights_need_24_bits

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def check(c, out, lse, ref, ref_lse):
    n = max(max(c.lens), 1)
    tol, tol_l = c.bound(ref, n)
    tol, tol_l = tol + (n + 56) * E * np.nanmax(np.abs(host(c.v))) * (1.0 if c.vs is None else float(c.vs.max())), tol_l + (n + 56) * E
    got, got_l = host(out), host(lse)
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()
    empty = np.isneginf(ref_lse)
    assert (np.isneginf(got_l) == empty).all()
    assert (np.abs(got_l[~empty] - ref_lse[~empty]) <= tol_l).all()


def oracle(c, starts, prefix, lens=None, table=None):
    scales = {} if c.ks is None else dict(k_scale=host(c.ks), v_scale=host(c.vs))
    return O.attend_shared(host(c.q), host(c.k), host(c.v), (c.table if table is None else table).cpu().numpy(), lens or c.lens, c.scale, starts, prefix, **scales)


def attend(m, c, starts, prefix, **more):  # noqa: F811
    c.kv.set_shared(True)
    return m.kv_attend_shared(c.kv, c.pages, c.table, c.len_t, ints(starts), ints(prefix), c.q, c.scale, want_lse=True, **more)


# dtype, Hq, Hkv, Dk, Dv, page, lens, starts, prefix
SHARED = [
    ("bf16", 1, 1, 64, 64, 16, [1], [0, 1], [1]),
    ("bf16", 4, 1, 128, 128, 16, [17, 16, 33], [0, 3], [16]),
    ("bf16", 8, 2, 128, 128, 64, [700, 640, 641, 705], [0, 4], [640]),
    ("bf16", 8, 2, 128, 128, 32, [300, 290, 299, 500, 0, 77, 90, 76], [0, 4, 8], [289, 75]),     # prefixes that end inside pages, an empty slot
    ("bf16", 6, 2, 80, 96, 32, [133, 129, 200, 140, 20], [0, 5], [129]),                          # one is shorter than the prefix
    ("bf16", 16, 1, 192, 128, 16, [300, 305, 290, 280], [1, 3], [290]),                           # two lie in no group
    ("bf16", 40, 2, 64, 64, 32, [257, 250, 300], [0, 1, 3], [200, 250]),                          # twenty heads a group, a group of one
    ("bf16", 2, 2, 256, 256, 128, [1000, 900, 1024], [0, 3], [896]),
    ("bf16", 3, 3, 16, 16, 16, [50, 52], [0, 0, 2, 2], [10, 49, 5]),                              # groups of nobody
    ("fp8", 8, 1, 128, 128, 16, [500, 333, 400, 350], [0, 4], [333]),
    ("fp8", 4, 4, 64, 64, 32, [100, 97, 96], [0, 3], [96]),
    ("fp8", 6, 2, 192, 128, 64, [640, 650], [0, 2], [640]),
    ("fp8", 2, 1, 256, 256, 16, [77, 78, 79], [0, 3], [70]),
    ("fp8", 17, 1, 80, 48, 16, [149, 148], [0, 2], [140]),
    ("fp32", 4, 2, 64, 64, 16, [333, 340, 0, 335], [0, 4], [330]),
    ("fp32", 3, 1, 128, 112, 32, [265, 200, 270], [0, 3], [200]),
    ("fp32", 2, 2, 192, 128, 16, [131, 140], [0, 2], [128]),
    ("fp32", 5, 1, 256, 240, 64, [330, 264], [0, 2], [257]),
    ("fp32", 6, 2, 96, 80, 32, [1000, 999, 1010], [0, 3], [990]),
    ("bf16", 4, 2, 64, 256, 32, [200, 210], [0, 2], [150]),                                       # values wider than keys
    ("fp8", 4, 2, 16, 208, 16, [200, 210], [0, 2], [150]),
    ("fp32", 4, 2, 256, 16, 16, [200, 210], [0, 2], [150]),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,lens,starts,prefix", SHARED)
def test_attend_shared(m, dtype, Hq, Hkv, Dk, Dv, page, lens, starts, prefix):  # noqa: F811
    c = Case(m, dtype, Hq, Hkv, Dk, Dv, page, lens, seed=Dk + page)
    out, lse = attend(m, c, starts, prefix)
    check(c, out, lse, *oracle(c, starts, prefix))
    again = attend(m, c, starts, prefix)
    assert (bits(again[0]) == bits(out)).all() and (bits(again[1]) == bits(lse)).all()
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("D,Dv", [(64, 64), (128, 128), (192, 128), (256, 256)])
@pytest.mark.parametrize("B,group", [(5, 3), (9, 5), (23, 3), (40, 4), (70, 6)])
def test_rows_of_any_number(m, dtype, D, Dv, B, group):  # noqa: F811
    # 15, 45, 69, 160 and 420 query heads meet a prefix: one wavefront, two or four of 32 to a workgroup, and several workgroups; own tokens from none on
    rng = np.random.default_rng(B)
    prefix = 700 if B < 50 else 345
    lens = [prefix + int(x) for x in rng.integers(0, 40, B)]
    c = Case(m, dtype, 2 * group, 2, D, Dv, 16, lens, seed=B)
    out, lse = attend(m, c, [0, B], [prefix])
    check(c, out, lse, *oracle(c, [0, B], [prefix]))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("prefix", [20000, 19999, 8192 * 2 + 1])
def test_long_prefixes_are_split(m, dtype, prefix):  # noqa: F811
    c = Case(m, dtype, 4, 1, 64, 64, 64, [20003, 20000, 20100], seed=3)
    out, lse = attend(m, c, [0, 3], [prefix])
    check(c, out, lse, *oracle(c, [0, 3], [prefix]))


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_many_groups(m, dtype):  # noqa: F811
    # more groups than lanes, of none to four sequences, whose prefixes and lengths go from nothing to hundreds
    rng = np.random.default_rng(5)
    sizes = [int(x) for x in rng.integers(0, 5, 150)]
    starts = [2, *(2 + np.cumsum(sizes)).tolist()]
    B = starts[-1] + 3
    prefix = [int(x) for x in rng.choice([0, 1, 15, 16, 17, 100, 300], 150)]
    lens = [int(x) for x in rng.integers(0, 60, B)]
    for g, p in enumerate(prefix):
        for i, b in enumerate(range(starts[g], starts[g + 1])):
            lens[b] = p + lens[b] if i != 1 else lens[b]  # the second one may be shorter
    c = Case(m, dtype, 4, 2, 64, 64, 16, lens, seed=5)
    out, lse = attend(m, c, starts, prefix)
    check(c, out, lse, *oracle(c, starts, prefix))
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_groups_of_unlike_sizes(m, dtype):  # noqa: F811
    # one of 300 query heads a key/value head beside many of three: what is planned for small groups takes several blocks of rows for the large one
    sizes, rng = [1] * 20 + [100] + [1] * 15, np.random.default_rng(2)
    starts = [0, *np.cumsum(sizes).tolist()]
    prefix = [int(x) for x in rng.integers(1, 200, len(sizes))]
    lens = [prefix[g] + int(rng.integers(0, 30)) for g, n in enumerate(sizes) for _ in range(n)]
    c = Case(m, dtype, 6, 2, 64, 64, 16, lens, seed=6)
    check(c, *attend(m, c, starts, prefix), *oracle(c, starts, prefix))


def test_the_largest_batch(m):  # noqa: F811
    rng = np.random.default_rng(4)
    B, prefix = 4096, 40
    lens = [prefix + int(x) for x in rng.integers(-1, 20, B)]
    c = Case(m, "bf16", 2, 1, 16, 16, 16, lens, seed=4)
    check(c, *attend(m, c, [0, B], [prefix]), *oracle(c, [0, B], [prefix]))
    one = list(range(B + 1))  # a group for every sequence
    check(c, *attend(m, c, one, [prefix] * B), *oracle(c, [0], []))
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_prefixes_of_nothing(m, dtype):  # noqa: F811
    c = Case(m, dtype, 4, 2, 128, 128, 16, [100, 0, 33], seed=1)
    want = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, want_lse=True)
    out, lse = attend(m, c, [0], [])
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    check(c, *attend(m, c, [0, 3], [0]), *oracle(c, [0], []))
    check(c, *attend(m, c, [0, 1, 1, 3], [0, 50, 0]), *oracle(c, [0], []))
    # a prefix that nobody has as many tokens of, and an empty batch
    c.lens = [10, 0, 33]
    c.len_t.copy_(ints(c.lens))
    check(c, *attend(m, c, [0, 2, 3], [100, 0]), *oracle(c, [0], []))
    c.lens = [0, 0, 0]
    c.len_t.zero_()
    out, lse = attend(m, c, [0, 3], [100])
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert c.kv.error_flags() == 0


def test_what_lies_behind_a_prefix_does_not_matter(m):  # noqa: F811
    # the first sequence ends with the prefix, inside a page whose other rows hold no numbers; its own page of another sequence holds none in the prefix's rows
    for dtype in ("bf16", "fp8", "fp32"):
        c = Case(m, dtype, 8, 2, 128, 128, 64, [135, 150, 170], seed=4)
        for t in (c.k, c.v):
            for b in (1, 2):
                for p in (0, 1):
                    t[int(c.table[b, p])] = float("nan")
                t[int(c.table[b, 2]), :, :7] = float("nan")
        out, lse = attend(m, c, [0, 3], [135])
        check(c, out, lse, *oracle(c, [0, 3], [135]))


def test_bad_pages_groups_and_lengths(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [200, 210, 220, 230], seed=2)
    plain = oracle(c, [0], [])
    for starts in ([0, 5], [-1, 4], [3, 2], [0, 2 ** 31 - 1]):
        check(c, *attend(m, c, starts, [64]), *plain)
        assert c.kv.error_flags() == 2
    check(c, *attend(m, c, [0, 3, 1, 4], [64, 64, 64]), *plain)
    assert c.kv.error_flags() == 2
    c.table[2] = c.table[3]
    plain = oracle(c, [0], [])
    check(c, *attend(m, c, [0, 2, 4], [-5, 2 ** 31 - 1]), *plain)   # nothing, and as many as the table holds, which nobody has
    assert c.kv.error_flags() == 2
    # pages outside the pool are masked, in a prefix for all of its group
    for dtype in ("bf16", "fp8", "fp32"):
        c = Case(m, dtype, 4, 2, 64, 64, 16, [200, 210, 220, 230], seed=2)
        c.table[0, 3], c.table[0, 11], c.table[2, 12] = -1, c.n_pages, 2 ** 31 - 1
        out, lse = attend(m, c, [0, 4], [190])
        check(c, out, lse, *oracle(c, [0, 4], [190]))
        assert c.kv.error_flags() == 1
    c.table[0, :12] = -1
    out, lse = attend(m, c, [0, 4], [190])
    check(c, out, lse, *oracle(c, [0, 4], [190]))
    assert c.kv.error_flags() == 1
    c.len_t[1] = 2 ** 31 - 1   # longer than the table: as long as that
    c.lens[1] = c.width * 16
    c.table[1] = c.table[3]
    out, lse = attend(m, c, [0, 1, 4], [0, 0])
    assert c.kv.error_flags() & 2


def test_extreme_logits(m):  # noqa: F811
    # one token outweighs all others, in the prefix, at its end and behind it; equal ones; huge ones of both signs
    for at in (0, 63, 64, 127, 128, 140):
        c = Case(m, "fp32", 2, 1, 64, 64, 16, [141, 141], seed=at)
        c.k.zero_()
        for b in (0, 1):
            c.k[int(c.table[b, at // 16]), :, at % 16] = 3e3
        c.q.fill_(1.0)
        c.q[:, 1] = -1.0
        out, lse = attend(m, c, [0, 2], [128])
        ref, ref_lse = oracle(c, [0, 2], [128])
        assert (np.abs(host(out) - ref) <= 2.0 ** -18).all() and (np.abs(host(lse) - ref_lse) <= 2.0 ** -18 * np.maximum(1, np.abs(ref_lse))).all()


def test_shared_pages_of_a_real_table(m):  # noqa: F811
    # as a server has it: the rows name the same pages for the prefix's whole pages; the plain attention gives the same up to rounding
    for dtype in ("bf16", "fp8", "fp32"):
        c = Case(m, dtype, 8, 2, 128, 128, 32, [515, 530, 600, 512], seed=9)
        c.table[1:, :16] = c.table[0, :16]
        want, want_lse = m.kv_attend(c.kv, c.pages, c.table, c.len_t, c.q, c.scale, want_lse=True)
        out, lse = attend(m, c, [0, 4], [512])
        check(c, out, lse, *oracle(c, [0, 4], [512]))
        step = 2.0 ** -7 if dtype != "fp32" else 2.0 ** -18
        assert (np.abs(host(out) - host(want)) <= step * np.abs(host(want)) + 2.0 ** -14).all()
        assert (np.abs(host(lse) - host(want_lse)) <= 2.0 ** -12).all()


def test_captured_replayed_and_on_another_stream(m):  # noqa: F811
    c = Case(m, "bf16", 8, 2, 128, 128, 16, [300, 310, 305, 40], seed=7)
    c.kv.set_shared(True)
    starts, prefix = ints([0, 3, 4]), ints([290, 0])
    out, lse = torch.empty((4, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((4, 8), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.kv_attend_shared(c.kv, c.pages, c.table, c.len_t, starts, prefix, c.q, c.scale, out=out, lse=lse)
    for i in range(4):
        c.q.copy_(torch.randn_like(c.q))
        prefix.copy_(ints([290 - 37 * i, 20]))
        c.len_t.copy_(ints([300 - i, 300, 305, 30 + i]))
        out.fill_(float("nan"))
        graph.replay()
        want, want_lse = m.kv_attend_shared(c.kv, c.pages, c.table, c.len_t, starts, prefix, c.q, c.scale, want_lse=True)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = m.kv_attend_shared(c.kv, c.pages, c.table, c.len_t, starts, prefix, c.q, c.scale, want_lse=True, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want_lse)


def test_packed_queries_and_pages_that_lie_apart(m):  # noqa: F811
    for dtype in ("bf16", "fp8", "fp32"):
        c = Case(m, dtype, 6, 2, 64, 48, 16, [100, 120, 99], seed=7, gap=48)
        room = torch.randn((3, 6 * 64 + 64), device="cuda").to(c.kv.dtype)
        c.q = room[:, 32:32 + 6 * 64].unflatten(1, (6, 64)).copy_(c.q)
        out, lse = attend(m, c, [0, 3], [97])
        check(c, out, lse, *oracle(c, [0, 3], [97]))


def test_refusals(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [40, 50], seed=7)
    args = (c.kv, c.pages, c.table, c.len_t, ints([0, 2]), ints([32]), c.q, c.scale)
    with pytest.raises(m.MoeiError) as e:
        m.kv_attend_shared(*args)
    assert "moei_kv_set_shared" in str(e.value) and e.value.code == -4
    c.kv.set_shared(True)
    m.kv_attend_shared(*args)
    with pytest.raises(m.MoeiError) as e:
        m.kv_attend_shared(*args[:4], ints([0] * 4098), ints([0] * 4097), *args[6:])
    assert "n_groups = 4097" in str(e.value)
    with pytest.raises(m.MoeiError) as e:
        m.kv_attend_shared(*args[:7], 0.0)
    assert "scale" in str(e.value)
    with pytest.raises(AssertionError):
        m.kv_attend_shared(*args[:4], ints([0, 2, 2]), ints([1]), *args[6:])
    with pytest.raises(AssertionError):
        m.kv_attend_shared(*args[:5], torch.ones(1, device="cuda"), *args[6:])
    c.kv.set_shared(False)
    with pytest.raises(m.MoeiError):
        m.kv_attend_shared(*args)


@pytest.mark.parametrize("D,Dv", [(64, 64), (128, 128), (192, 128), (256, 256)])
@pytest.mark.parametrize("B", [1, 40, 70])
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_weights_of_prefixes_keep_24_bits(m, dtype, B, D, Dv):  # noqa: F811
    # The inputs and the bound of tests/test_gpu_kv_exact.py, where two bf16 numbers for a weight would give 0: five tokens, one of weight p = exp(-x) and value 256, four of
    # weight 1 whose values take away 256 times the nearest two.  All five are a prefix, met by 1, 40 and 70 query heads: one, two and four wavefronts of rows.  What is
    # joined with it are sums of nothing, times 0, and itself, times 1: no rounding more.  Allowed: the weight is off by 2^-22.5, seven additions of magnitudes up to 512 p by
    # 2^-23 each, and half a step of the output.
    Hkv, page = 8, 16
    x = logits_whose_weights_need_24_bits(Hkv, dtype, np.random.default_rng(D))
    p = np.exp(-x)
    hi = bf16(p)
    lo = bf16(p - hi)
    take = []
    for part in (256 * hi, 256 * lo):  # four bits each, so that 8-bit pages hold them
        a = e4m3(part)
        take += [a, part - a]
        assert (e4m3(part - a) == part - a).all()
    kv = m.Kv(Hkv, Hkv, D, Dv, page, dtype, max_batch=B, max_pages=1, shared=True)
    k, v = torch.zeros((1, Hkv, page, D), dtype=torch.float64), torch.zeros((1, Hkv, page, Dv), dtype=torch.float64)
    k[0, :, 4, 0] = torch.from_numpy(-np.ones(Hkv) if dtype == "fp8" else -x)
    for t, a in enumerate(take):
        v[0, :, t] = torch.from_numpy(-a)[:, None]
    v[0, :, 4] = 256
    k, v = k.to(kv.page_dtype).cuda(), v.to(kv.page_dtype).cuda()
    scales = dict(k_scale=torch.from_numpy(x).float().cuda(), v_scale=torch.ones(Hkv, device="cuda")) if dtype == "fp8" else {}
    q = torch.zeros((B, Hkv, D), dtype=kv.dtype, device="cuda")
    q[:, :, 0] = 1
    out = m.kv_attend_shared(kv, m.KvPages(kv, k, v, **scales), torch.zeros((B, 1), dtype=torch.int32, device="cuda"), ints([5] * B), ints([0, B]), ints([5]), q, 1.0)
    ref = 256 * (p - hi - lo) / (4 + p)
    tol = (256 * 2.0 ** -22.5 + 7 * 2.0 ** -23 * 512 * p) / (4 + p) + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(ref) > 1.5 * tol).all()
    assert (np.abs(host(out) - ref[None, :, None]) <= tol[None, :, None]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("prefix", [135, 128, 3])
def test_a_sequence_without_tokens_of_its_own_needs_no_pages(m, dtype, prefix):  # noqa: F811
    # as long as the prefix, which ends inside a page or with one, behind the first sequence that has as many: its own row of the table names nothing
    c = Case(m, dtype, 8, 2, 128, 128, 32, [prefix, prefix, 170, prefix], seed=4)
    c.table[1], c.table[3] = -1, c.n_pages
    out, lse = attend(m, c, [0, 4], [prefix])
    check(c, out, lse, *oracle(c, [0, 4], [prefix]))
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("D,Dv", [(128, 128), (192, 128), (256, 256)])
@pytest.mark.parametrize("B", [1, 40, 70])
def test_logits_of_prefixes_in_fp32_are_sums_of_short_sums(m, B, D, Dv):  # noqa: F811
    # Two tokens of equal logits, D (1 + 2^-19): one in a single dimension, one in all of them.  Up to 32 of the latter add up exactly (32 + 2^-14: 20 bits), and so do such
    # sums up to 256 (multiples of 2^-14); one chain loses 2^-18 with every two from 64 on, and would be off by (D - 64) / 2 times that, 2^-13 at least.  Values of 1 and -1 show half
    # of that.  Weights that are equal but for exp2 and its argument, 2^-21, cancel but for that.
    kv = m.Kv(8, 8, D, Dv, 16, "fp32", max_batch=B, max_pages=1, shared=True)
    k, v = torch.zeros((1, 8, 16, D), device="cuda"), torch.zeros((1, 8, 16, Dv), device="cuda")
    k[0, :, 0, 0] = D * (1 + 2.0 ** -19)
    k[0, :, 1] = 1 + 2.0 ** -19
    v[0, :, 0], v[0, :, 1] = 1, -1
    q, table, lens = torch.ones((B, 8, D), device="cuda"), torch.zeros((B, 1), dtype=torch.int32, device="cuda"), ints([2] * B)
    pages = m.KvPages(kv, k, v)
    assert (m.kv_attend_shared(kv, pages, table, lens, ints([0, B]), ints([2]), q, 1.0).abs() <= 2.0 ** -20).all()


@pytest.mark.parametrize("dtype,Hq,Hkv", [("bf16", 1024, 1), ("fp32", 1024, 2), ("fp8", 1024, 1024)])
def test_1024_heads_behind_a_prefix(m, dtype, Hq, Hkv):  # noqa: F811
    c = Case(m, dtype, Hq, Hkv, 16, 32, 16, [100, 90, 133, 45], seed=6, max_sel=0)
    check(c, *attend(m, c, [0, 3, 4], [90, 45]), *oracle(c, [0, 3, 4], [90, 45]))
    assert c.kv.error_flags() == 0
