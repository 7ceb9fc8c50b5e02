"""Appending as many tokens at once as make a workgroup take a token's heads one after another (from eight tokens a compute unit on),
against the definition in 64 bits, and just below that.

What a rotated element may be off in fp32: sine and cosine 2^-25 each, of |x1| + |x2|; the first product and the result 2^-24 of themselves.  Then
half a step of the type that holds it; 8-bit pages hold the quotient by the head's scale, 2^-24 of itself more.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {"fp32": 0.0, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}   # half a step, besides the fp32 result's own
PAGE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def m():
    import paper_2401_14361_amd as mod
    mod.lib()
    return mod


def turned(x, pos, freq, interleaved):
    """(definition, allowance in fp32) of x [T][heads][D] at pos [T], 64 bits."""
    x, half = x.double(), len(freq)
    angle = pos.double()[:, None, None] * freq.double()
    c, s = angle.cos(), angle.sin()
    first = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    a, b = x[..., first], x[..., second]
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    for at, other in ((first, b), (second, a)):
        tol[..., at] = 2.0 ** -25 * (a.abs() + b.abs()) + 2.0 ** -24 * ((other * s).abs() + y[..., at].abs())
    return y, tol


def inputs(T, heads, dtype, layout, seed):
    """Tensors [T][heads][D] that lie dense, or as parts of one row (at 16 bytes, or anywhere)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    sizes = [h * d for h, d in heads]
    if layout == "dense":
        return [torch.randn((T, h, d), generator=g, device="cuda").to(dtype) for h, d in heads]
    x = torch.randn((T, sum(sizes) + 3), generator=g, device="cuda").to(dtype)
    x = x[:, 3:] if layout == "odd" else x[:, :-3].contiguous()
    return [p.unflatten(1, hd) for p, hd in zip(x.split(sizes, 1), heads)]


def check(m, dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, in_place, B, seq, pos):
    io, T = torch.float32 if dtype == "fp32" else torch.bfloat16, len(pos)
    of = np.arange(T) if seq is None else np.asarray(seq)
    pos = np.asarray(pos)
    width = int(pos.max()) // page + 1
    kv = m.Kv(Hq, Hkv, Dk, Dv, page, dtype, max_batch=B, max_pages=width, max_sel=0)
    rng = np.random.default_rng(T)
    held = np.unique(of[pos >= 0] * width + pos[pos >= 0] // page)
    table = np.full(B * width, 2 ** 30, dtype=np.int32)      # pages that no token of the call lies in are none
    table[held] = rng.permutation(len(held))
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    pool = lambda d: torch.randn((len(held), Hkv, page, d), generator=g, device="cuda").to(PAGE[dtype])  # noqa: E731
    k_pages, v_pages = pool(Dk), pool(Dv)
    lo, hi = torch.full((len(held), Hkv, Dk), 7.0, dtype=io, device="cuda"), torch.full((len(held), Hkv, Dk), -7.0, dtype=io, device="cuda")
    scales = {}
    if dtype == "fp8":
        scales = {n: 0.05 + 0.1 * torch.rand(Hkv, generator=g, device="cuda") for n in ("k_scale", "v_scale")}
    pages = m.KvPages(kv, k_pages, v_pages, k_min=lo, k_max=hi, **scales)
    q, k, v = inputs(T, [(Hq, Dk), (Hkv, Dk), (Hkv, Dv)], io, layout, T)
    q_in, before_k, before_v = q.clone(), k_pages.float(), v_pages.float()
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)).float().cuda()
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).int().cuda()  # noqa: E731
    q_out = m.kv_append(kv, pages, ints(table).view(B, width), ints(pos), q, k, v, freq, seq=None if seq is None else ints(seq), interleaved=interleaved,
                        q_out=q if in_place else torch.full((T, Hq, Dk), 5.0, dtype=io, device="cuda"))
    there = torch.from_numpy(np.flatnonzero(pos >= 0)).cuda()
    gone = torch.from_numpy(np.flatnonzero(pos < 0)).cuda()
    P = torch.from_numpy(np.maximum(pos, 0)).cuda()
    half = HALF["fp32" if dtype == "fp32" else "bf16"]
    ref, tol = turned(q_in, P, freq, interleaved)
    assert ((q_out.double() - ref).abs() <= tol + half * ref.abs())[there].all()
    assert (q_out[gone] == (q_in[gone] if in_place else 5.0)).all()
    at = torch.from_numpy(table[(of * width + np.maximum(pos, 0) // page)[pos >= 0]].astype(np.int64)).cuda()
    row = P[there] % page
    ref, tol = (x[there] for x in turned(k, P, freq, interleaved))
    val = v.double()[there]
    least = 0.0
    if dtype == "fp8":
        ks, vs = (scales[n].double()[None, :, None] for n in ("k_scale", "v_scale"))
        ref, tol, val, least = (ref / ks).clamp(-448, 448), tol / ks + 2.0 ** -24 * (ref / ks).abs(), (val / vs).clamp(-448, 448), 2.0 ** -10
    assert ((k_pages[at, :, row].double() - ref).abs() <= tol + HALF[dtype] * ref.abs() + least).all()
    if dtype == "fp8":
        assert ((v_pages[at, :, row].double() - val).abs() <= (2.0 ** -4 + 2.0 ** -24) * val.abs() + least).all()
    else:
        assert (v_pages[at, :, row].double() == val).all()
    written = torch.zeros((len(held), page), dtype=torch.bool, device="cuda")
    written[at, row] = True
    assert int(written.sum()) == len(there)
    for now, then in ((k_pages, before_k), (v_pages, before_v)):  # nothing else is
        assert ((now.float() == then).all(-1).all(1) | written).all()
    full = torch.zeros(len(held), dtype=torch.bool, device="cuda")
    full[at[row == page - 1]] = True
    assert full.any() and not full.all()
    keys = k_pages[full].float()
    assert (lo[full].float() == keys.amin(2)).all() and (hi[full].float() == keys.amax(2)).all()
    assert (lo[~full] == 7.0).all() and (hi[~full] == -7.0).all()
    assert kv.error_flags() == 0


SHAPES = [
    # dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, in place
    ("bf16", 32, 8, 128, 128, 64, 128, False, "dense", False),
    ("bf16", 32, 8, 128, 128, 64, 128, False, "dense", True),
    ("fp8", 32, 8, 128, 128, 32, 128, True, "packed", False),
    ("fp32", 14, 7, 128, 64, 16, 64, True, "dense", True),      # 21 heads, sixteen at once
    ("fp32", 32, 8, 64, 64, 16, 64, False, "packed", False),
    ("bf16", 24, 4, 192, 128, 16, 64, False, "packed", False),  # 28 heads, 21 at once
    ("bf16", 6, 3, 80, 96, 16, 40, False, "odd", False),        # element by element: nine heads, six at once
    ("fp8", 9, 3, 48, 64, 128, 6, True, "odd", False),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,rot,interleaved,layout,in_place", SHAPES)
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_prompts_of_eight_tokens_a_compute_unit(m, dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, in_place, more):
    T = 8 * torch.cuda.get_device_properties(0).multi_processor_count + more
    starts, counts = [0, 21, 1000], [T // 2, T // 5, T - T // 2 - T // 5]
    tokens = [(b, starts[b] + i) for b in range(3) for i in range(counts[b])]
    np.random.default_rng(T).shuffle(tokens)
    check(m, dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, in_place, 3, [t[0] for t in tokens], [t[1] for t in tokens])


@pytest.mark.parametrize("dtype,Hq,Hkv,Dk,Dv,page,rot,interleaved,layout,in_place", SHAPES)
@pytest.mark.parametrize("more", [-1, 0, 77])
def test_decode_batches_of_eight_sequences_a_compute_unit(m, dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, in_place, more):
    # a token of each sequence: the summaries of the pages that are completed come from the same launch
    B = 8 * torch.cuda.get_device_properties(0).multi_processor_count + more
    pos = np.random.default_rng(B).integers(0, 3 * page, B)
    pos[::3] = pos[::3] // page * page + page - 1
    pos[5::50] = -1
    check(m, dtype, Hq, Hkv, Dk, Dv, page, rot, interleaved, layout, in_place, B, None, pos)


def test_rotated_queries_over_keys_or_values_are_refused(m):  # (no kernel runs but for the calls that are taken)
    kv = m.Kv(4, 2, 64, 64, 16, "bf16", max_batch=4, max_pages=1, max_sel=0)
    pages = m.KvPages(kv, *(torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    table = torch.arange(4, dtype=torch.int32, device="cuda")[:, None].contiguous()
    room = torch.randn(64 * 1024, device="cuda").bfloat16()

    def append(T, q, k, v, out, stride=0):
        view = lambda at, h: (torch.as_strided(room, (T, h, 64), (stride or h * 64, 64, 1), at))  # noqa: E731
        pos = torch.zeros(T, dtype=torch.int32, device="cuda")
        return m.kv_append(kv, pages, table, pos, view(q, 4), view(k, 2), view(v, 2), None, q_out=torch.as_strided(room, (T, 4, 64), (256, 64, 1), out))

    for bad in ((4096, 8192, 4096 + 511), (4096, 8192, 4096 - 1023), (8192, 4096, 4096 + 511), (4096, 4096, 4096)):
        with pytest.raises(m.MoeiError, match="overlaps d_k or d_v"):
            append(4, 0, *bad)
    append(4, 0, 4096, 4608, 4096 + 1024)                       # right behind
    append(4, 0, 4096, 8192, 4096 - 1024)                       # right before
    with pytest.raises(m.MoeiError, match="overlaps d_k or d_v"):  # one row of packed tokens
        append(4, 0, 256, 384, 3 * 4096 + 256, stride=4096)
    append(4, 0, 256, 384, 3 * 4096 - 1024, stride=4096)         # between two rows
    append(1, 0, 256, 384, 0)                                    # in place, keys right behind
    torch.cuda.synchronize()
    assert kv.error_flags() == 0
