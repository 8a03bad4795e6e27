"""What contexts of two sequences and more hold for rows that groups share: a partial result a query row of the tiles that a launch can
have, no more.  (Host side: needs no GPU.)"""
import ctypes

import pytest

from paper_2506_02572_amd import hata

ROW = (128 + 2) * 4  # bytes of a partial result


def workspace(B, Hq, Hkv, L_cap=64):
    n = ctypes.c_size_t(0)
    cfg = hata.hata_config(B, Hq, Hkv, 128, 32, L_cap, 64, Hkv * L_cap * 128, L_cap * 128, 128)
    assert hata.load_library().hata_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)) == 0
    return n.value


def shared(B, Hq, Hkv):
    """Tiles of 64, 128 or 256 query rows: those that B sequences fill, and for every group, of which half as many as sequences can have
    two members, one that is not full; at least a launch of 256 workgroups.  Larger tiles are for fewer groups (a mean above 64 and 448)."""
    G, most = Hq // Hkv, 0
    for rows, above in ((64, 0), (128, 64), (256, 448)):
        groups = min(B // 2, 1024, (B * G - 1) // above if above else B)
        if groups:
            tiles = (B + groups * (rows // G - 1)) // (rows // G) * Hkv
            most = max(most, max(256, (tiles + 255) // 256 * 256) * rows * ROW)
    return most


def own(B, Hq, Hkv):
    """Partial results of rows that are not shared: one a wave of eight and query head, of every unit or 256 workgroups, and 256 to spare."""
    return (max(256, (B * Hkv + 7) // 8) + 256) * 8 * (Hq // Hkv) * ROW


@pytest.mark.parametrize("B,Hq,Hkv", [(2, 32, 8), (32, 32, 8), (256, 64, 8), (256, 8, 8), (1024, 64, 8), (2048, 8, 1), (3000, 40, 8)])
def test_partial_results(B, Hq, Hkv):
    """The rest (codes, scores, lists, histograms, counters of a cache of 64 rows) is below 1.5 KB a query head and 256 KB."""
    need = shared(B, Hq, Hkv) + own(B, Hq, Hkv)
    got = workspace(B, Hq, Hkv)
    assert need <= got <= need + 1536 * B * Hq + (1 << 18), (need, got)


def test_one_sequence_holds_none():
    assert workspace(1, 64, 8) < 8 << 20
