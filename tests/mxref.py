"""Microscaled 4-bit floating point and the expert sort in plain numpy / 64 bits, written from the definitions in
include/qmm.h (test infrastructure; shares no code with the library)."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUE = np.concatenate([E2M1, -E2M1])
MXFP4, NVFP4 = 32, 16
# finite e4m3 values by code 0 .. 126 (0x7F is NaN)
E4M3 = np.array([(c & 7) * 2.0**-9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def nearest_code(grid, v):
    """Index of the grid value nearest to v >= 0, ties to the even index, saturating."""
    hi = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = v - grid[lo], grid[hi] - v
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def blocks_of(x, fmt):
    pad = -x.shape[-1] % fmt
    return np.pad(x, ((0, 0), (0, pad))).reshape(x.shape[0], -1, fmt)


def quantize(x, fmt, g=1.0):
    """x float64 [rows, K] (values of a narrower type) -> codes [rows, nb, fmt], scale bytes [rows, nb]."""
    xb = blocks_of(x, fmt)
    finite = np.isfinite(xb).all(-1)
    safe = np.where(finite[..., None], xb, 0.0)
    amax = np.abs(safe).max(-1)
    if fmt == MXFP4:
        e = np.floor(np.log2(np.where(amax > 0, amax, 1.0)))
        b = np.where(amax > 0, np.maximum(e - 2, -127), -127)
        q = np.abs(safe) / np.exp2(b)[..., None]
        scale = (b + 127).astype(np.int64)
        bad = 255
    else:
        g = np.float32(g)
        with np.errstate(over="ignore"):
            s = np.minimum(amax.astype(np.float32) / (np.float32(6) * g), np.float32(448))
        scale = nearest_code(E4M3, s.astype(np.float64))
        D = (E4M3[scale].astype(np.float32) * g)[..., None]
        with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
            q = np.abs(safe).astype(np.float32) / D
        q = np.where(D > 0, q, np.float32(0)).astype(np.float64)
        bad = 127
    codes = nearest_code(E2M1, np.minimum(q, 7.0)) | (np.signbit(safe).astype(np.int64) << 3)
    codes = np.where(finite[..., None], codes, 0)
    return codes, np.where(finite, scale, bad)


def step(scale, fmt, g=1.0):
    """D of every block as float64 (NaN where the scale is NaN)."""
    scale = np.asarray(scale).astype(np.int64)
    if fmt == MXFP4:
        return np.where(scale == 255, np.nan, np.exp2(scale - 127.0))
    d = E4M3[np.minimum(scale, 126)].astype(np.float32) * np.float32(g)
    return np.where(scale == 127, np.nan, d.astype(np.float64))


def values(codes, scale, fmt, K, g=1.0):
    v = VALUE[codes] * step(scale, fmt, g)[..., None]
    return v.reshape(v.shape[0], -1)[:, :K]


def unit_bytes(fmt):
    return 16384 + 128 * 256 // fmt


def units(n):
    return -(-n // 128)


def unpack(packed, fmt, rows, K, row_unit0=0):
    """Packed operand (uint8 numpy) -> codes [rows, KU * 256], scale bytes [rows, KU * 256 / fmt]: everything stored for these rows."""
    ku = -(-K // 256)
    u = packed.reshape(-1, ku, unit_bytes(fmt))[row_unit0: row_unit0 + units(rows)]
    n = u.shape[0]
    chunks = u[:, :, :16384].reshape(n, ku, 128, 8, 16)
    r = np.arange(128)[:, None]
    chunks = np.take_along_axis(chunks, ((np.arange(8)[None, :] ^ (r & 7))[None, None, :, :, None] + np.zeros((n, ku, 1, 1, 1), int)), axis=3)
    by = chunks.reshape(n, ku, 128, 128)
    codes = np.stack([by & 15, by >> 4], -1).reshape(n, ku, 128, 256).transpose(0, 2, 1, 3).reshape(n * 128, ku * 256)
    per = 256 // fmt
    s = u[:, :, 16384:].reshape(n, ku, per // 4, 32, 4, 4).transpose(0, 4, 3, 1, 2, 5).reshape(n * 128, ku * per)
    return codes[:rows].astype(np.int64), s[:rows].astype(np.int64)


def pack(codes, scale, fmt):
    """codes [rows, nb, fmt], scale [rows, nb] -> packed bytes (rows past the matrix: 0xA5)."""
    rows, nb, _ = codes.shape
    ku = -(-nb * fmt // 256)
    c = np.zeros((units(rows) * 128, ku * 256), np.uint8)
    c[:rows, : nb * fmt] = codes.reshape(rows, -1)
    s = np.zeros((units(rows) * 128, ku * 256 // fmt), np.uint8)
    s[:rows, :nb] = scale
    by = c[:, 0::2] | (c[:, 1::2] << 4)
    by[rows:] = 0xA5
    s[rows:] = 0xA5
    n = units(rows)
    out = np.empty((n, ku, unit_bytes(fmt)), np.uint8)
    for i in range(n):
        for j in range(ku):
            for r in range(128):
                for q in range(8):
                    at = 128 * r + 16 * (q ^ (r % 8))
                    out[i, j, at: at + 16] = by[128 * i + r, 128 * j + 16 * q: 128 * j + 16 * q + 16]
                for b in range(256 // fmt):
                    out[i, j, 16384 + 512 * (b // 4) + 16 * (r % 32) + 4 * (r // 32) + b % 4] = s[128 * i + r, j * (256 // fmt) + b]
    return out.reshape(-1)


def sort(idx, E):
    """order, place, offsets, units of the stable sort by expert."""
    flat = idx.reshape(-1).astype(np.int64)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    counts = np.bincount(key, minlength=E + 1)[:E]
    n = int(counts.sum())
    place = np.full(flat.size, -1, np.int64)
    place[order[:n]] = np.arange(n)
    order = np.where(np.arange(flat.size) < n, order, -1)
    return order, place, np.concatenate([[0], np.cumsum(counts)]), np.concatenate([[0], np.cumsum(-(-counts // 128))])


def silu(g):
    return g / (1.0 + np.exp(-g))
