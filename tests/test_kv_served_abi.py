"""Host side of the served cache's calls: what is refused before any device work, and the oracle's own pins (CPU only)."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv_oracle as O
from tests.test_kernel_resources import kernels  # noqa: F401 (a fixture)
from tests.test_kv_abi import m  # noqa: F401 (a fixture)


def test_null_pointers_and_negative_sizes_are_refused_on_the_host(m):  # noqa: F811
    L, one, f = m.lib(), 16, C.c_float(1.0)  # (never dereferenced)

    def err(rc):
        assert rc == -1
        return L.moei_last_error().decode()

    norm = lambda kv=None, T=1, B=1: L.kv_append_norm(kv, one, one, 1, B, None, one, None, T, one, 0, one, 0, one, 0, one, one, 0, f, one, 2, 0, one, None)  # noqa: E731
    shared = lambda kv=None, B=1: L.kv_attend_shared(kv, one, one, 1, one, B, one, one, 1, one, 0, f, one, None, None)  # noqa: E731
    weights = lambda kv=None, B=1: L.kv_attend_weights(kv, one, one, 1, one, B, one, 0, f, 0, one, 0, one, None, None)  # noqa: E731
    evict = lambda kv=None, B=1: L.kv_evict(kv, one, one, 1, one, B, one, 0, 1, 0, 1, one, 1, one, one, 0, one, None)  # noqa: E731
    for call in (norm, shared, weights, evict):
        assert "null" in err(call())
        assert "negative" in err(call(B=-1))
        assert call(B=0) == 0 or call is norm  # nothing to do
    assert "negative" in err(norm(T=-1)) and norm(T=0) == 0
    assert "null" in err(L.moei_kv_set_weights(None, 1)) and "null" in err(L.moei_kv_set_shared(None, 1))


def test_oracle_norm_against_hand_numbers():
    y = O.norm(np.array([[[3.0, 4.0, 0.0, 0.0]]]), [1.0, 2.0, 1.0, 1.0], 0.0)  # mean square 25 / 4
    assert np.allclose(y, [[[1.2, 3.2, 0.0, 0.0]]], rtol=0, atol=1e-15)
    assert (O.norm(np.zeros((1, 1, 4)), np.ones(4), 1e-6) == 0).all()


def test_oracle_weights_add_up_to_the_heads():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((6, 2, 16, 8)), rng.standard_normal((6, 2, 16, 8))
    q, table, lens = rng.standard_normal((2, 6, 8)), np.array([[0, 1, 2], [3, 4, 5]]), [37, 0]
    out, lse = O.attend(q, k, v, table, lens, 0.3)
    w = O.attend_weights(q, k, table, lens, lse, 0.3)
    assert np.allclose(w[0].sum(-1), 3.0) and (w[1] == 0).all() and (w[0, :, 37:] == 0).all()


def test_oracle_shared_is_attention_where_rows_name_the_same_pages():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((9, 1, 16, 8)), rng.standard_normal((9, 1, 16, 8))
    q, table, lens = rng.standard_normal((3, 2, 8)), np.array([[0, 1, 2], [0, 1, 3], [0, 4, 5]]), [40, 33, 16]
    want = O.attend(q, k, v, table, lens, 0.3)
    for a, b in zip(O.attend_shared(q, k, v, table, lens, 0.3, [0, 2, 3], [32, 16]), want):
        assert np.allclose(a, b, rtol=1e-13, atol=1e-13)
    # the third one's first tokens by way of the first row; the second one is too short
    other = O.attend_shared(q, k, v, table, lens, 0.3, [0, 3], [16])
    assert np.allclose(other[0], want[0], rtol=1e-13, atol=1e-13)
    table[2, 0] = 6
    other = O.attend_shared(q, k, v, table, lens, 0.3, [0, 3], [16])
    assert np.allclose(other[0], want[0], rtol=1e-13, atol=1e-13)
    assert not np.allclose(O.attend(q, k, v, table, lens, 0.3)[0][2], want[0][2])


@pytest.mark.parametrize("w,n,keep,first,last,want", [
    ([5, 1, 4, 1, 3, 2], 6, 3, 0, 0, [0, 2, 4]), ([5, 1, 4, 1, 3, 2], 6, 3, 1, 1, [0, 2, 5]), ([1, 1, 1, 1], 4, 2, 0, 0, [0, 1]), ([0, np.nan, -np.inf, 1], 4, 3, 0, 0, [0, 1, 3]),
    ([1, 2], 2, 3, 1, 1, [0, 1]), ([], 0, 3, 1, 1, []), ([3, 2, 1, 0], 4, 2, 0, 2, [2, 3]),
])
def test_oracle_keep(w, n, keep, first, last, want):
    assert O.keep(w, n, keep, first, last) == want


def test_kernels_keep_to_their_registers(kernels):  # noqa: F811
    """As few registers as the wavefronts that a compute unit is to hold at once allow (those of the products' sums among them)."""
    for start, waves_a_simd in (("kv_append_norm_kernel<unsigned short, unsigned short, 8, false>", 6), ("kv_shared_kernel<moei::Bf16, 128, 128, 4>", 2),
                                ("kv_shared_kernel<moei::Fp8, 128, 128, 4>", 2), ("kv_attend_weigh_kernel<moei::Bf16, 128, 128, 2, 8>", 2), ("kv_evict_kernel<1024, false>", 8)):
        got, = [k for n, k in kernels.items() if n.startswith(start)]
        assert got[".private_segment_fixed_size"] == 0
        assert waves_a_simd * (got[".vgpr_count"] + 7 & ~7) <= 512, (start, got[".vgpr_count"])


def test_no_served_kernel_has_private_memory(kernels):  # noqa: F811
    """Every instance, those at the limit of 512 registers too: vectors never leave registers (scalars may stand in lanes of one)."""
    found = {n: k for n, k in kernels.items() if n.startswith(("kv_append_norm_kernel<", "kv_shared_kernel<", "kv_join_kernel<", "kv_attend_weigh_kernel<", "kv_weights_kernel", "kv_evict_kernel<", "kv_move_kernel<"))}
    assert len(found) == 12 + 28 + 2 + 20 + 1 + 2 + 3, sorted(found)
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= 512, n
