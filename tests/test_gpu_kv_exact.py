"""The paged KV cache's attention where its answer shows a single weight: inputs whose sums are known in 64 bits and whose
losses would be larger than what is allowed, by what is derived beside each."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2401_14361_amd as mod
    mod.lib()
    return mod


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).bfloat16().double().numpy()


def e4m3(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.float8_e4m3fn).double().numpy()


def logits_whose_weights_need_24_bits(n, dtype, rng):
    """x in (0.05, 0.69), held by a key of `dtype` (8 bits: by the scale of a code of one), for which p = exp(-x) is at least 0.8 2^-18 off
    the sum of two bf16 numbers (2^-18 is as far as that gets)."""
    x = rng.uniform(0.05, 0.69, 4000)
    x = np.unique(bf16(x) if dtype == "bf16" else x.astype(np.float32).astype(np.float64))
    p = np.exp(-x)
    hi = bf16(p)
    rest = p - hi - bf16(p - hi)
    x = x[np.abs(rest) >= 0.8 * 2.0 ** -18]
    return rng.choice(x, n, replace=len(x) < n)


@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp8", "fp32"])
def test_weights_keep_24_bits(m, dtype, D):
    # Five tokens: one of weight p = exp(-x) and value 256, four of weight 1 whose values take away 256 times the nearest two bf16 numbers.  What is
    # left is 256 (p - hi - lo) / (4 + p), at least 12.8 2^-14 before the division.  Allowed: the weight is off by 2^-22.5 (the exponent's factor and
    # its rounding 2^-23, exp2 2^-24), seven additions of magnitudes up to 512 p by 2^-23 each (twice what rounding to nearest would): 5.8 2^-14.
    Hkv, page, Dv = 32, 16, min(D, 128) if D != 256 else 256
    io = torch.float32 if dtype == "fp32" else torch.bfloat16
    x = logits_whose_weights_need_24_bits(Hkv, dtype, np.random.default_rng(D))
    p = np.exp(-x)
    hi = bf16(p)
    lo = bf16(p - hi)
    take = []
    for part in (256 * hi, 256 * lo):  # four bits each, so that 8-bit pages hold them
        a = e4m3(part)
        take += [a, part - a]
        assert (e4m3(part - a) == part - a).all()
    kv = m.Kv(Hkv, Hkv, D, Dv, page, dtype, max_batch=1, max_pages=1)
    k = torch.zeros((1, Hkv, page, D), dtype=torch.float64)
    v = torch.zeros((1, Hkv, page, Dv), dtype=torch.float64)
    k[0, :, 4, 0] = torch.from_numpy(-np.ones(Hkv) if dtype == "fp8" else -x)
    for t, a in enumerate(take):
        v[0, :, t] = torch.from_numpy(-a)[:, None]
    v[0, :, 4] = 256
    k, v = k.to(kv.page_dtype).cuda(), v.to(kv.page_dtype).cuda()
    scales = dict(k_scale=torch.from_numpy(x).float().cuda(), v_scale=torch.ones(Hkv, device="cuda")) if dtype == "fp8" else {}
    q = torch.zeros((1, Hkv, D), dtype=io, device="cuda")
    q[:, :, 0] = 1
    out = m.kv_attend(kv, m.KvPages(kv, k, v, **scales), torch.zeros((1, 1), dtype=torch.int32, device="cuda"),
                      torch.tensor([5], dtype=torch.int32, device="cuda"), q, 1.0)
    ref = 256 * (p - hi - lo) / (4 + p)
    tol = (256 * 2.0 ** -22.5 + 7 * 2.0 ** -23 * 512 * p) / (4 + p) + 2.0 ** -8 * np.abs(ref)
    assert (np.abs(ref) > 1.5 * tol).all()  # (two parts would give 0)
    assert (np.abs(out[0].double().cpu().numpy() - ref[:, None]) <= tol[:, None]).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(128, 128), (64, 64), (48, 6), (256, 256)])  # (6: element by element)
def test_rotation_rounds_sine_and_cosine_once(m, D, rot, interleaved):
    # x1 c - x2 s in fp32: c and s, which are at most 1, are off by 2^-25 each, the first product by 2^-24 of itself, the result by 2^-24 of itself.
    rng = np.random.default_rng(D + rot)
    T, page = 64, 256
    pos = np.concatenate([[0, 1, 2, 131071, 10 ** 6 - 1, 2 ** 24 + 1, 2 ** 30 - 1, 2 ** 30 - 2], rng.integers(0, 131072, T - 16), rng.integers(0, 2 ** 30, 8)]).astype(np.int64)
    width = 2 ** 30 // page
    kv = m.Kv(4, 2, D, 16, page, "fp32", max_batch=1, max_pages=width, max_sel=0)
    at = np.unique(pos // page)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, torch.from_numpy(at).cuda()] = torch.arange(len(at), dtype=torch.int32, device="cuda")
    k_pages, v_pages = torch.zeros((len(at), 2, page, D), device="cuda"), torch.zeros((len(at), 2, page, 16), device="cuda")
    assert len(np.unique(pos)) == T
    g = torch.Generator(device="cuda")
    g.manual_seed(D)
    q, k = torch.randn((T, 4, D), generator=g, device="cuda"), torch.randn((T, 2, D), generator=g, device="cuda")
    v = torch.randn((T, 2, 16), generator=g, device="cuda")
    freq = (10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)).float()
    q_out = m.kv_append(kv, m.KvPages(kv, k_pages, v_pages), table, torch.from_numpy(pos).int().cuda(), q, k, v, freq.cuda(),
                        seq=torch.zeros(T, dtype=torch.int32, device="cuda"), interleaved=interleaved)
    k_out = k_pages[torch.from_numpy(np.searchsorted(at, pos // page)).cuda(), :, torch.from_numpy(pos % page).cuda()]
    angle = pos[:, None] * freq.double().numpy()
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    first = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    second = first + (1 if interleaved else rot // 2)
    for x, y in ((q, q_out), (k, k_out)):
        x, y = x.double().cpu().numpy(), y.double().cpu().numpy()
        a, b = x[..., first], x[..., second]
        for got, one, other, sign in ((y[..., first], a, b, -1), (y[..., second], b, a, 1)):
            ref = one * c + sign * other * s
            tol = 2.0 ** -25 * (np.abs(a) + np.abs(b)) + 2.0 ** -24 * (np.abs(other * s) + np.abs(ref)) + 1e-12
            assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) / tol).max()
        assert (y[..., rot:] == x[..., rot:]).all()
    assert kv.error_flags() == 0


def test_the_largest_and_smallest_scales(m):
    # equal logits of 0 whatever the scale is; one that is infinite times log2(e) in fp32 is refused: 0 times it would be no number
    kv = m.Kv(2, 1, 64, 64, 16, "fp32", max_batch=1, max_pages=4, max_sel=4)
    k, v = torch.randn((4, 1, 16, 64), device="cuda"), torch.ones((4, 1, 16, 64), device="cuda")
    table, n = torch.arange(4, dtype=torch.int32, device="cuda")[None], torch.tensor([50], dtype=torch.int32, device="cuda")
    pages, q = m.KvPages(kv, k, v, k_min=k.amin(2), k_max=k.amax(2)), torch.zeros((1, 2, 64), device="cuda")
    for scale in (1e-45, 1e-38, 2.35e38):
        out, lse = m.kv_attend(kv, pages, table, n, q, scale, want_lse=True)
        assert (out == 1).all() and ((lse - np.log(50)).abs() < 1e-5).all()
    for scale in (2.4e38, 3.4e38):
        for call in (lambda s: m.kv_attend(kv, pages, table, n, q, s), lambda s: m.kv_attend_blocks(kv, pages, table, n, q, s, 3)):
            with pytest.raises(m.MoeiError, match="scale"):
                call(scale)
