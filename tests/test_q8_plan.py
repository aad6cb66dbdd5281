"""The grid of the attention over the 8-bit cache, asked of the built library (no GPU)."""
import ctypes

from paper_2609_36546_amd import ops


def grid(cus):
    f = getattr(ops.lib(), "_ZN4ipdv12attn_q8_gridEi")   # ipdv::attn_q8_grid(int)
    f.argtypes, f.restype = [ctypes.c_int], ctypes.c_int
    return f(cus)


def test_every_span_has_a_workgroup():
    """Spans are dealt to the 8 XCDs in runs: workgroup b takes span (b mod 8) ceil(n / 8) + b / 8.
    With 76 workgroups spans 49, 59 and 69 of 76 had none."""
    for cus in [1, 3, 4, 5, 30, 32, 38, 64, 76, 110, 128, 228, 254, 256, 304]:
        g = grid(cus)
        assert g <= max(8, 2 * cus)
        for n in range(1, g + 1):
            each = -(-n // 8)
            taken = {(b & 7) * each + (b >> 3) for b in range(g) if b >> 3 < each}
            assert set(range(n)) <= taken, (cus, n)
    assert grid(256) == 512
