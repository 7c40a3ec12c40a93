"""The plain definitions the GPU tests compare with: the formats' lattices, the
packed layout and the generator's published answers (CPU)."""
import numpy as np
import pytest

import fp4_plain as P
from paper_2306_04235_gb300 import mnmt


def test_lattices():
    assert P.E4M3.max() == 448 and P.E4M3[1] == 2.0 ** -9 and len(P.E4M3) == 127
    # ties go to the even code, beyond 6 to 6
    v = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0001, 7.9])
    assert list(P.E2M1[P.nearest_even(v, P.E2M1)]) == [0, 1, 1, 2, 2, 4, 4, 6, 6]


def test_philox_published_answers():
    """Known answers of Philox4x32-10 published with the generator."""
    for c, k, want in [([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
                       ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
                       ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
                        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])]:
        assert [int(v) for v in P.philox(c, k)] == want


def test_kept_share():
    k, s = P.keep(200, 333, 0.3, 7, 1 << 35)
    t = round(0.3 * 65536)
    assert s == np.float32(65536) / np.float32(65536 - t)
    n = k.size
    assert abs(k.mean() - (1 - t / 65536)) < 5 * (0.21 / n) ** 0.5
    assert not P.keep(5, 9, 1.0, 1, 2)[0].any() and P.keep(5, 9, 0.0, 1, 2)[0].all()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_quantised_values_are_fixed_points(fmt):
    rng = np.random.default_rng(3)
    g = 1.0 if fmt == "mx" else 2.0 ** -6
    x = rng.standard_normal((5, 77)).astype(np.float32)
    byte, code, v, inside = P.quantize(x, fmt, g)
    # an element is off by at most half a step of the widest interval, 1, or was held at 6 of up to 8
    S = np.repeat(P.E4M3[byte] * g if fmt == "nv" else np.ldexp(1.0, byte - 127), P.BLOCK[fmt], 1)[:, :77]
    assert (np.abs(v - x) <= np.where(inside, 1.0 + 1e-6, 2.0) * S).all()
    if fmt == "mx":
        # the largest magnitude stays in the same binade, so a second pass changes nothing
        assert np.array_equal(P.quantize(v, fmt, g)[2], v)


def test_packed_sizes_match_the_library():
    for rows, cols in [(1, 1), (4, 512), (128, 129), (129, 64), (300, 1000)]:
        for fmt, code in (("mx", mnmt.FP4_MX), ("nv", mnmt.FP4_NV)):
            nb = -(-cols // P.BLOCK[fmt])
            c, s = P.pack(np.zeros((rows, nb), np.uint8), np.zeros((rows, nb, P.BLOCK[fmt]), np.uint8), cols)
            assert c.shape[1] == mnmt.mnmt_fp4_pitch(cols) and s.size == mnmt.mnmt_fp4_scale_bytes(rows, cols, code)
    assert mnmt.mnmt_fp4_pitch(0) == 0 and mnmt.mnmt_fp4_scale_bytes(0, 5, 0) == 0
