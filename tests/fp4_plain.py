"""Microscaled 4-bit floating point and counter-based dropout in plain numpy,
64 bits: the definitions the kernels are compared with."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)])[:127]
BLOCK = {"mx": 32, "nv": 16}


def nearest_even(v, lattice):
    """Index of the lattice's nearest entry, ties to the even index, beyond the last the last (v >= 0)."""
    hi = np.clip(np.searchsorted(lattice, v), 1, len(lattice) - 1)
    lo = hi - 1
    d = (v - lattice[lo]) - (lattice[hi] - v)
    return np.where(d < 0, lo, np.where(d > 0, hi, np.where(lo % 2 == 0, lo, hi)))


def bf16(v):
    """Nearest bf16 of float64 values that are fp32 numbers, as fp32."""
    u = np.ascontiguousarray(v, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(v), np.float32(np.nan), r)


def quantize(x, fmt, g=1.0):
    """x [M][K] (fp32 values): scale bytes [M][nb], codes [M][nb][B] and values [M][K] (fp32), straight-through mask."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    B = BLOCK[fmt]
    nb = -(-K // B)
    b = np.zeros((M, nb * B), np.float32)
    b[:, :K] = x
    b = b.reshape(M, nb, B)
    bad = ~np.isfinite(b).all(2)
    a = np.abs(np.where(bad[:, :, None], 1, b)).max(2).astype(np.float64)
    if fmt == "mx":
        e = np.where(a > 0, np.frexp(np.where(a > 0, a, 1))[1] - 3, -127)
        e = np.maximum(e, -127)
        byte, S, r = e + 127, np.ldexp(1.0, e), np.ldexp(1.0, -e)
        byte = np.where(bad, 255, byte)
    else:
        g = float(np.float32(g))
        c = float(np.float32(1 / float(np.float32(6 * g))))
        byte = nearest_even((a * c).astype(np.float32).astype(np.float64), E4M3)
        S = (E4M3[byte] * g).astype(np.float32).astype(np.float64)
        r = np.where(S > 0, 1 / np.where(S > 0, S, 1), 0).astype(np.float32).astype(np.float64)
        byte = np.where(bad, 127, byte)
    t = (np.where(bad[:, :, None], 0, b).astype(np.float64) * r[:, :, None]).astype(np.float32).astype(np.float64)
    q = nearest_even(np.abs(t), E2M1)
    code = np.where(bad[:, :, None], 0, q | (np.signbit(b) << 3))
    S = np.where(bad, np.nan, S)
    with np.errstate(invalid="ignore"):
        v = (np.where(code & 8, -1.0, 1.0) * E2M1[code & 7] * S[:, :, None]).astype(np.float32)
    inside = (np.abs(t) <= 6) & ~bad[:, :, None]
    return byte, code, v.reshape(M, -1)[:, :K], inside.reshape(M, -1)[:, :K]


def pack(byte, code, K):
    """The documented packed form: codes [M][pitch], scales (flat)."""
    M, nb, B = code.shape
    c = np.zeros((M, -(-K // 32) * 32), np.uint8)
    c[:, :K] = code.reshape(M, -1)[:, :K]
    tk = -(-nb // 4)
    s = np.zeros(-(-M // 128) * tk * 512, np.uint8)
    row, blk = np.meshgrid(np.arange(M), np.arange(nb), indexing="ij")
    s[((row // 128) * tk + blk // 4) * 512 + 16 * (row % 32) + 4 * (row % 128 // 32) + blk % 4] = byte
    return c[:, 0::2] | (c[:, 1::2] << 4), s


def philox(c, k):
    """Philox4x32-10: four counter words (arrays) and two key words -> four words."""
    m = 0xFFFFFFFF
    c = [np.asarray(v, np.uint64) for v in c]
    for i in range(10):
        k0, k1 = np.uint64((k[0] + i * 0x9E3779B9) & m), np.uint64((k[1] + i * 0xBB67AE85) & m)
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ k0, p1 & np.uint64(m), (p0 >> np.uint64(32)) ^ c[3] ^ k1, p0 & np.uint64(m)]
    return c


def keep(M, d, p, seed, offset):
    """Boolean [M][d] and the factor of what is kept."""
    n = -(-d // 8)
    col, row = np.meshgrid(np.arange(n), np.arange(M))
    w = philox([col, row, np.full_like(col, offset & 0xFFFFFFFF), np.full_like(col, offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    f = np.stack([w[i // 2] >> np.uint64(16) if i % 2 else w[i // 2] & np.uint64(0xFFFF) for i in range(8)], 2).reshape(M, -1)[:, :d]
    t = int(np.rint(np.float32(p) * np.float32(65536)))
    return f >= t, float(np.float32(65536) / np.float32(65536 - t)) if t < 65536 else 0.0
