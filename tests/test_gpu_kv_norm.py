"""Appending tokens whose queries and keys are normed for each head, against the definition in 64 bits (oracle/kv_oracle.py).

Tolerances.  e = 2^-24.  A head's squares are summed by lanes, 16 of them one after another at most, then in 6 steps over lanes: 22 roundings, of
sums without a sign; the division by the width and eps add 2: the root halves them and adds 1, the reciprocal 1, the two products 2: 16 e of the
normed value.  The rotation adds what it adds in kv_append: 2^-20 of |x1| + |x2| bounds all of it, and 2^-20 (16 e) of the normed value is allowed
for the norm, of both elements of a pair.  Then half a step of the type that holds the result.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from tests.test_gpu_kv import APPEND, E, HALF, LEAST, Case, _append_inputs, _freq, bits, host, m  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def weights(c, per_head, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [1.0 + 0.5 * torch.randn((H, c.kv.heads[1]) if per_head else (c.kv.heads[1],), generator=g, device="cuda")
            for H in (c.kv.heads[0], c.kv.k_heads[0])]


def check(c, q, k, v, qw, kw, eps, q_out, q_before, k_before, v_before, seq, pos, freq, interleaved, turn=None):
    """Everything that the call may write, and that it has written nothing else."""
    place = O.places(c.table.cpu().numpy().tolist(), seq, pos, c.page, c.n_pages)
    io = "fp32" if c.dtype == "fp32" else "bf16"
    f = host(freq) if freq is not None else np.zeros(0)
    rot, at = 2 * len(f), [max(p, 0) for p in pos] if turn is None else list(turn)

    def made(x, w):
        y = O.norm(host(x), host(w), eps)
        a = np.abs(y)
        s = a.copy()
        if interleaved:
            s[..., 0:rot:2] = s[..., 1:rot:2] = a[..., 0:rot:2] + a[..., 1:rot:2]
        else:
            s[..., :rot // 2] = s[..., rot // 2:rot] = a[..., :rot // 2] + a[..., rot // 2:rot]
        return O.rotate(y, at, f, interleaved), 2.0 ** -20 * s + 2.0 ** -20 * s * (np.arange(s.shape[-1]) < rot)

    (qr, qs), (kr, ks), vr = made(q, qw), made(k, kw), host(v)
    got_q = host(q_out)
    want_k, want_v = host(k_before), host(v_before)
    tol_k, tol_v = np.zeros_like(want_k), np.zeros_like(want_v)
    for t, to in enumerate(place):
        if to is None:
            assert (bits(q_out[t]) == bits(q_before[t])).all()
            continue
        assert (np.abs(got_q[t] - qr[t]) <= HALF[io] * (np.abs(qr[t]) + qs[t]) + qs[t]).all()
        a, b, sa = kr[t], vr[t], ks[t]
        if c.dtype == "fp8":
            a, b, sa = a / host(c.ks)[:, None], b / host(c.vs)[:, None], sa / host(c.ks)[:, None]
            a, b = np.clip(a, -448, 448), np.clip(b, -448, 448)
        want_k[to[0], :, to[1]], want_v[to[0], :, to[1]] = a, b
        tol_k[to[0], :, to[1]] = HALF[c.dtype] * (np.abs(a) + sa) + LEAST[c.dtype] + sa + 4 * E * np.abs(a)
        tol_v[to[0], :, to[1]] = 0.0 if c.dtype != "fp8" else HALF["fp8"] * np.abs(b) + LEAST["fp8"] + 4 * E * np.abs(b)
    for got, want, tol in ((host(c.k), want_k, tol_k), (host(c.v), want_v, tol_v)):
        same = (got == want) | (np.isnan(got) & np.isnan(want))
        assert (same | (np.abs(got - want) <= tol)).all()
    return place


MORE = [
    ("bf16", 2, 1, 256, 64, 16, 30, True, "odd"),           # element by element: 64 lanes a head, two units each
    ("fp32", 2, 2, 256, 32, 16, 256, False, "dense"),       # 32 lanes a head
    ("fp32", 3, 1, 208, 32, 16, 208, False, "odd"),
    ("bf16", 1, 1, 16, 16, 16, 16, False, "dense"),         # one lane a head
    ("bf16", 40, 8, 96, 96, 32, 96, False, "packed"),       # more heads than a workgroup takes at once
]


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,rot,interleaved,layout", APPEND + MORE)
def test_a_token_to_each_sequence(m, dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, per_head):  # noqa: F811
    pos = [0, page - 1, -1, 2 * page, 3 * page - 1, 2 * page + 5, 3 * page - 1, 7]
    turn = [max(p, 0) + 1000 * i for i, p in enumerate(pos)] if per_head else None
    c = Case(m, dtype, Hq, Hkv, Dk, Dv, page, [max(p, 0) + 1 for p in pos], seed=rot + page, summaries=True, nan_tail=False)
    q, k, v = _append_inputs(c, len(pos), seed=page, layout=layout)
    qw, kw = weights(c, per_head)
    before = [t.clone() for t in (c.k, c.v, c.lo, c.hi)]
    q_out = torch.full((len(pos), Hq, Dk), 7.0, dtype=c.kv.dtype, device="cuda")
    q_before = q_out.clone()
    freq = _freq(rot) if rot else None
    got = m.kv_append_norm(c.kv, c.pages, c.table, ints(pos), q, k, v, qw, kw, freq, eps=1e-5, turn=None if turn is None else ints(turn),
                           interleaved=interleaved, q_out=q_out)
    assert got is q_out
    place = check(c, q, k, v, qw, kw, float(np.float32(1e-5)), q_out, q_before, before[0], before[1], range(len(pos)), pos, freq, interleaved, turn)
    full = [at[0] for at in place if at is not None and at[1] == page - 1]
    assert len(full) == 3
    lo, hi = before[2], before[3]
    for i in full:  # exactly the rows as they are stored, the new one too
        lo[i], hi[i] = c.k[i].to(c.kv.dtype).amin(1), c.k[i].to(c.kv.dtype).amax(1)
    assert (bits(c.lo) == bits(lo)).all() and (bits(c.hi) == bits(hi)).all()
    assert c.kv.error_flags() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("many", [False, True])
def test_prompts(m, dtype, in_place, many):  # noqa: F811
    # three prompts in one call in a mixed order; `many`: as many tokens as make a workgroup take all heads of a token
    page, starts, counts = 16, [0, 21, 1000], [1700, 11, 400] if many else [75, 11, 40]
    rng = np.random.default_rng(3)
    tokens = [(b, starts[b] + i) for b in range(3) for i in range(counts[b])]
    rng.shuffle(tokens)
    seq, pos = [int(t[0]) for t in tokens], [int(t[1]) for t in tokens]
    c = Case(m, dtype, 4, 2, 64, 96, page, [a + n for a, n in zip(starts, counts)], seed=8, summaries=True, nan_tail=False)
    q, k, v = _append_inputs(c, len(tokens), seed=2)
    qw, kw = weights(c, False)
    before = [t.clone() for t in (c.k, c.v, c.lo, c.hi, q)]
    q_out = q if in_place else torch.zeros_like(q)
    m.kv_append_norm(c.kv, c.pages, c.table, ints(pos), q, k, v, qw, kw, _freq(64), seq=ints(seq), q_out=q_out)
    place = check(c, before[4], k, v, qw, kw, float(np.float32(1e-6)), q_out, q_out, before[0], before[1], seq, pos, _freq(64), False)
    lo, hi = before[2], before[3]
    for i in {at[0] for at in place if at[1] == page - 1}:
        lo[i], hi[i] = c.k[i].to(c.kv.dtype).amin(1), c.k[i].to(c.kv.dtype).amax(1)
    assert (bits(c.lo) == bits(lo)).all() and (bits(c.hi) == bits(hi)).all()


def test_far_and_negative_turns(m):  # noqa: F811
    c = Case(m, "fp32", 2, 1, 64, 64, 16, [5, 5, 5, 5], seed=0, nan_tail=False)
    turn = [2 ** 30, -(2 ** 30), 999_999, -3]
    q, k, v = _append_inputs(c, 4, seed=4)
    qw, kw = weights(c, False)
    before = c.k.clone(), c.v.clone()
    q_out = m.kv_append_norm(c.kv, c.pages, c.table, ints([4] * 4), q, k, v, qw, kw, _freq(64), turn=ints(turn))
    check(c, q, k, v, qw, kw, float(np.float32(1e-6)), q_out, q_out, *before, range(4), [4] * 4, _freq(64), False, turn)


def test_tokens_without_a_place_are_left_out(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [32, 32, 32], seed=6, summaries=True, nan_tail=False)
    c.table[1, 0], c.table[2, 1] = -1, c.n_pages
    seq, pos = [0, 0, 1, 2, 3, -1, 2], [5, 32, 7, 31, 1, 1, 2 ** 31 - 1]
    q, k, v = _append_inputs(c, len(seq), seed=6)
    qw, kw = weights(c, True)
    before = [bits(t) for t in (c.lo, c.hi)]
    kb, vb = c.k.clone(), c.v.clone()
    q_out = torch.full_like(q, 3.0)
    m.kv_append_norm(c.kv, c.pages, c.table, ints(pos), q, k, v, qw, kw, _freq(64), seq=ints(seq), q_out=q_out)
    check(c, q, k, v, qw, kw, float(np.float32(1e-6)), q_out, torch.full_like(q, 3.0), kb, vb, seq, pos, _freq(64), False)
    assert (bits(c.lo) == before[0]).all() and (bits(c.hi) == before[1]).all()
    assert c.kv.error_flags() == 3 and c.kv.error_flags() == 0


def test_heads_of_zeros_huge_values_and_no_numbers(m):  # noqa: F811
    c = Case(m, "fp32", 4, 1, 64, 64, 16, [1], seed=0, nan_tail=False)
    q, k, v = _append_inputs(c, 1, seed=4)
    q[0, 0] = 0.0
    q[0, 1] *= 1e30     # the squares pass fp32's range
    q[0, 2, 5] = float("inf")
    q[0, 3, 7] = float("nan")
    k *= 1e-30          # the squares are nothing beside eps
    qw, kw = weights(c, False)
    got = host(m.kv_append_norm(c.kv, c.pages, c.table, ints([0]), q, k, v, qw, kw, None, eps=1e-6))[0]
    assert (got[0] == 0).all() and (got[1] == 0).all()
    assert np.isnan(got[2, 5]) and (np.delete(got[2], 5) == 0).all() and np.isnan(got[3]).all()
    want = host(k)[0, 0] * host(kw) / np.sqrt(float(np.float32(1e-6)))
    assert (np.abs(host(c.k)[int(c.table[0, 0]), 0, 0] - want) <= 2.0 ** -20 * np.abs(want)).all()


def test_nothing_to_append(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [32], seed=6, nan_tail=False)
    q, k, v = (t[:0] for t in _append_inputs(c, 1, seed=6))
    qw, kw = weights(c, False)
    assert m.kv_append_norm(c.kv, c.pages, c.table, ints([]), q, k, v, qw, kw, _freq(64)).shape == (0, 4, 64)


def test_refusals(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [32], seed=6, nan_tail=False)
    q, k, v = _append_inputs(c, 1, seed=6)
    qw, kw = weights(c, False)
    good = dict(q=q, k=k, v=v, q_weight=qw, k_weight=kw, inv_freq=_freq(64))
    before = bits(c.k)

    def refused(text, error=None, **change):
        with pytest.raises(error or m.MoeiError) as e:
            m.kv_append_norm(c.kv, c.pages, c.table, ints([3]), **{**good, **change})
        assert text in str(e.value)

    for eps in (0.0, -1.0, float("inf"), float("nan")):
        refused("eps", eps=eps)
    wide = torch.randn(4 * 64 * 2, device="cuda")
    refused("overlaps", q_weight=wide[:64], q_out=wide[:128].view(torch.bfloat16).view(1, 4, 64))
    refused("", AssertionError, q_weight=qw.bfloat16())
    refused("", AssertionError, q_weight=qw[:32])
    refused("", AssertionError, q_weight=torch.ones(4, 64, device="cuda"))                       # one of the two for each head alone
    refused("", AssertionError, turn=ints([1, 2]))
    refused("", AssertionError, turn=torch.ones(1, device="cuda"))
    refused("rot_dim", inv_freq=_freq(128))
    torch.cuda.synchronize()
    assert (bits(c.k) == before).all()


def test_captured_and_replayed(m):  # noqa: F811
    c = Case(m, "bf16", 4, 2, 64, 64, 16, [32, 8], seed=6, summaries=True, nan_tail=False)
    q, k, v = _append_inputs(c, 2, seed=6)
    qw, kw = weights(c, False)
    pos, turn, q_out, freq = ints([31, 7]), ints([131, 7]), torch.zeros_like(q), _freq(64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.kv_append_norm(c.kv, c.pages, c.table, pos, q, k, v, qw, kw, freq, turn=turn, q_out=q_out)
    for i in range(4):
        q.copy_(torch.randn_like(q))
        turn.add_(1)
        pos.fill_(5 + i)
        graph.replay()
        got, pages = bits(q_out), bits(c.k)
        q_out.zero_()
        want = m.kv_append_norm(c.kv, c.pages, c.table, pos, q, k, v, qw, kw, freq, turn=turn)
        assert (bits(want) == got).all() and (bits(c.k) == pages).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_a_token_to_each_of_many_sequences_with_summaries(m, dtype):  # noqa: F811
    # so many that a workgroup takes all heads of a token, beside those that form the summaries
    rng = np.random.default_rng(7)
    pos = [int(x) for x in rng.choice([0, 14, 15, 31, 30, -1], 2100)]
    c = Case(m, dtype, 4, 2, 32, 48, 16, [max(p, 0) + 1 for p in pos], seed=7, summaries=True, nan_tail=False)
    q, k, v = _append_inputs(c, len(pos), seed=7)
    qw, kw = weights(c, True)
    before = [t.clone() for t in (c.k, c.v, c.lo, c.hi)]
    q_out = torch.zeros_like(q)
    q_before = q_out.clone()
    m.kv_append_norm(c.kv, c.pages, c.table, ints(pos), q, k, v, qw, kw, _freq(32), q_out=q_out)
    place = check(c, q, k, v, qw, kw, float(np.float32(1e-6)), q_out, q_before, before[0], before[1], range(len(pos)), pos, _freq(32), False)
    lo, hi = before[2], before[3]
    for i in {at[0] for at in place if at is not None and at[1] == 15}:
        lo[i], hi[i] = c.k[i].to(c.kv.dtype).amin(1), c.k[i].to(c.kv.dtype).amax(1)
    assert (bits(c.lo) == bits(lo)).all() and (bits(c.hi) == bits(hi)).all()
