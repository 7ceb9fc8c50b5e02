"""Host side of the paged KV cache: layouts of the structures and what is refused before any device work (CPU only)."""
import ctypes as C
import os

import pytest

from tests.test_kernel_resources import kernels  # noqa: F401 (a fixture)


@pytest.fixture(scope="module")
def m():
    import paper_2401_14361_amd as mod
    if not os.path.exists(mod.lib_path()):          # build only if nothing is built
        from paper_2401_14361_amd.build import build
        build()
    mod.lib()
    return mod


def test_structures_match_the_header(m):
    assert C.sizeof(m.KvDesc) == 9 * 4
    assert [f[0] for f in m.KvDesc._fields_] == ["n_q_heads", "n_kv_heads", "k_dim", "v_dim", "page_size", "dtype", "max_batch", "max_pages", "max_sel"]
    from paper_2401_14361_amd.binding import _KvPages
    assert C.sizeof(_KvPages) == 72 and _KvPages.d_k_scale.offset == 40 and _KvPages.n_pages.offset == 32


GOOD = dict(n_q_heads=8, n_kv_heads=2, k_dim=128, v_dim=64, page_size=16, dtype=1, max_batch=4, max_pages=64, max_sel=8)


@pytest.mark.parametrize("change,text", [
    (dict(n_q_heads=7), "multiple"), (dict(n_q_heads=0), "multiple"), (dict(n_kv_heads=0), "multiple"), (dict(n_q_heads=2048), "1024"),
    (dict(k_dim=8), "widths"), (dict(k_dim=272), "widths"), (dict(v_dim=72), "widths"), (dict(v_dim=0), "widths"),
    (dict(page_size=8), "page_size"), (dict(page_size=48), "page_size"), (dict(page_size=512), "page_size"), (dict(page_size=-16), "page_size"),
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(max_batch=0), "max_batch"), (dict(max_batch=5000), "max_batch"),
    (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 27), "max_pages"), (dict(max_sel=-1), "max_sel"), (dict(max_sel=65), "max_sel"),
])
def test_shapes_are_refused_on_the_host(m, change, text):
    L, h = m.lib(), C.c_void_p(0)
    d = m.KvDesc(**{**GOOD, **change})
    assert L.moei_kv_create(C.byref(d), C.byref(h)) == -1 and not h.value
    assert text in L.moei_last_error().decode()


def test_null_pointers_are_refused_on_the_host(m):
    L = m.lib()
    one = 16  # never dereferenced

    def err(rc):
        assert rc == -1
        return L.moei_last_error().decode()

    assert "null" in err(L.moei_kv_create(None, None))
    assert "null" in err(L.kv_attend(None, one, one, 1, one, 1, one, 0, 1.0, 0, one, None, None))
    assert "null" in err(L.kv_attend_blocks(None, one, one, 1, one, 1, one, 0, 1.0, 1, 0, 1, one, None, None, None))
    assert "null" in err(L.kv_append(None, one, one, 1, 1, None, one, 1, one, 0, one, 0, one, 0, one, 2, 0, one, None))
    assert "negative" in err(L.kv_attend(None, one, one, 1, one, -1, one, 0, 1.0, 0, one, None, None))
    assert "null" in err(L.moei_kv_error_flags(None, None, None))
    assert L.moei_kv_destroy(None) == 0


def test_kernels_keep_to_their_registers(kernels):
    """No private memory, and as few registers as the workgroups that a compute unit is to hold at once allow."""
    named = {n: k for n, k in kernels.items() if n.startswith("kv_")}
    assert len(named) >= 4 * 3 + 12 + 6 + 3
    for n, k in named.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n
    for n, waves_a_simd in (("kv_attend_kernel<moei::Bf16, 128, 128, 2, 8>", 2), ("kv_attend_kernel<moei::Fp8, 128, 128, 2, 8>", 2),
                            ("kv_attend_kernel<moei::Bf16, 64, 64, 2, 8>", 4), ("kv_attend_kernel<moei::Bf16, 192, 128, 2, 4>", 2),
                            ("kv_blocks_kernel<unsigned short, 128, 16>", 3), ("kv_append_kernel<unsigned short, unsigned short, 8, false>", 6)):
        got, = [k for name, k in named.items() if name.startswith(n)]
        assert waves_a_simd * (got[".vgpr_count"] + 7 & ~7) <= 512, (n, got[".vgpr_count"])
