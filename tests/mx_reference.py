"""Microscaled 4-bit records restated in numpy and 64 bits, for the tests: records of rows, and the values of records."""
import numpy as np

MAGNITUDE = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
E4M3 = np.array([(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127])


def record_bytes(d, block):
    return -(-(d // 2 + d // block + (1 if block == 16 else 0)) // 32) * 32


def _power_above(v, unit, lowest):
    """Smallest k >= lowest with unit * 2^k >= v, for every v > 0 (0 gives lowest)."""
    k = np.full(v.shape, lowest, dtype=np.int64)
    for i in range(lowest, 129):
        k = np.where(unit * 2.0 ** i < v, i + 1, k)
    return k


def encode(x, block):
    """x float64 [T, d] (values of bf16 or binary16) -> (records uint8 [T, rec], whether a block was not finite)."""
    T, d = x.shape
    b = x.reshape(T, d // block, block)
    fine = np.isfinite(b).all(-1)
    amax = np.where(fine, np.abs(np.where(np.isfinite(b), b, 0)).max(-1), 0.0)
    if block == 32:
        k = _power_above(amax, 6.0, -127)
        byte, s, r = np.where(amax > 0, k + 127, 0), 2.0 ** k, None
    else:
        top = amax.max(-1)
        r = np.where(top > 0, _power_above(top, 2688.0, -100), 0)
        byte = np.searchsorted(E4M3, amax / 6 / 2.0 ** r[:, None])       # first guess, then by comparison of exact products
        for step in (1, -1, 1):
            at = E4M3[np.clip(byte, 0, 126)] * 6 * 2.0 ** r[:, None]
            below = E4M3[np.clip(byte - 1, 0, 126)] * 6 * 2.0 ** r[:, None]
            byte = np.where(at < amax, byte + 1, np.where((byte > 0) & (below >= amax), byte - 1, byte))
        s = E4M3[byte] * 2.0 ** r[:, None]
    y = np.abs(np.where(fine[..., None], b, 0)) / np.where(s > 0, s, 1)[..., None]
    code = np.zeros(y.shape, dtype=np.int64)
    for i in range(1, 8):
        middle = (MAGNITUDE[i - 1] + MAGNITUDE[i]) / 2
        code += (y >= middle) if i % 2 == 0 else (y > middle)
    code += 8 * (np.signbit(b) & (code > 0))          # a magnitude of 0 has no sign
    code = np.where(fine[..., None], code, 0).reshape(T, d)
    out = np.zeros((T, record_bytes(d, block)), dtype=np.uint8)
    out[:, : d // 2] = code[:, 0::2] | code[:, 1::2] << 4
    out[:, d // 2: d // 2 + d // block] = np.where(fine, byte, 255 if block == 32 else 127)
    if block == 16:
        out[:, d // 2 + d // block] = r.astype(np.int8).view(np.uint8)
    return out, not fine.all()


def decode(rec, d, block):
    """Values float64 [T, d] of records."""
    T = rec.shape[0]
    pair = rec[:, : d // 2]
    code = np.stack((pair & 15, pair >> 4), -1).reshape(T, d)
    v = np.where(code >= 8, -MAGNITUDE[code % 8], MAGNITUDE[code % 8]).reshape(T, d // block, block)
    byte = rec[:, d // 2: d // 2 + d // block].astype(np.int64)
    if block == 32:
        s = np.where(byte == 255, np.nan, 2.0 ** (byte - 127.0))
    else:
        r = np.minimum(rec[:, d // 2 + d // block].view(np.int8).astype(np.int64), 117)
        s = np.append(E4M3, np.nan)[byte & 127] * 2.0 ** r[:, None]
    return (v * s[..., None]).reshape(T, d)


def random_records(T, d, block, rng, spread=2):
    """Records with every code, and scales around 1."""
    rec = np.zeros((T, record_bytes(d, block)), dtype=np.uint8)
    rec[:, : d // 2] = rng.integers(0, 256, (T, d // 2))
    n = d // block
    if block == 32:
        rec[:, d // 2: d // 2 + n] = 127 + rng.integers(-spread, spread + 1, (T, n))
    else:
        rec[:, d // 2: d // 2 + n] = 0x38 + rng.integers(-8 * spread, 8 * spread + 1, (T, n))
        rec[:, d // 2 + n] = rng.integers(-spread, spread + 1, T).astype(np.int8).view(np.uint8)
    return rec
