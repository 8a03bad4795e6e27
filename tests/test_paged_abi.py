"""Host-side behaviour of the paged-serving entry points that needs no GPU: calls without a context, and the workspace."""
import ctypes

from paper_2506_02572_amd import hata


def workspace(B, Hq, Hkv, L_cap=4096):
    n = ctypes.c_size_t(0)
    cfg = hata.hata_config(B, Hq, Hkv, 128, 128, L_cap, 64, Hkv * L_cap * 128, L_cap * 128, 128)
    assert hata.load_library().hata_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == 0
    return n.value


def test_calls_without_a_context_are_refused():
    lib = hata.load_library()
    p = ctypes.c_void_p(4096)  # (looked at by nobody)
    assert lib.hata_plan_pages(None, p, p, 1, None, None, p, 4, 16, 4, p, p, p, p, None, p, None, 8, None) == -1
    assert lib.hata_write_slots(None, p, p, 128, 128, p, 1, p, p, None, 16, 4, None, None) == -1
    assert lib.hata_dense_decode_paged(None, p, p, p, p, 4, 16, 4, p, 1, None, None, 0, 1.0, p, None, None) == -1


def test_workspace_of_shared_rows():
    """One sequence shares nothing; partial results are laid out for 256 workgroups of at least 64 query rows."""
    row = 130 * 4
    assert workspace(1, 32, 8) < 4 << 20
    assert workspace(2, 32, 8) > 256 * 64 * row
    # 1024 sequences of 64 heads: 65536 query rows, a partial result each and half as many again for what tiles do not fill
    assert workspace(1024, 64, 8) < 1 << 30
