"""Plain 64-bit statements of the operators on 4-bit floating point and on experts, and of the stored form, in numpy."""
import numpy as np

MX, NV = 0, 1
BLOCK = {MX: 32, NV: 16}
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
_b = np.arange(127)
E4M3 = np.where(_b >> 3 == 0, (_b & 7) * 2.0 ** -9, (1 + (_b & 7) / 8) * 2.0 ** ((_b >> 3) - 7.0))   # bytes 0 .. 126


def pitch(K):
    return -(-K // 32) * 16


def scale_tiles(fmt, K):
    return -(-K // (4 * BLOCK[fmt]))


def nearest(x, grid):
    """Index of the nearest entry of an ascending grid, the even index of two that are equally near (x >= 0)."""
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    up, down = grid[hi] - x, x - grid[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def quantize(x, fmt, exponent=0):
    """x: float64 [rows][K] -> (codes [rows][2 * pitch], scale bytes [rows][4 * scale_tiles])."""
    rows, K = x.shape
    n, wide = BLOCK[fmt], scale_tiles(fmt, K) * 4 * BLOCK[fmt]
    with np.errstate(over="ignore"):
        x = (x * 2.0 ** exponent).astype(np.float32).astype(np.float64)
    b = np.zeros((rows, wide))
    b[:, :K] = x
    b = b.reshape(rows, -1, n)
    most = np.abs(b).max(-1)
    fine = np.isfinite(most)
    safe = np.where(fine, most, 1.0)
    if fmt == MX:
        e = np.where(safe > 0, np.frexp(safe)[1] - 3, -127)
        e = np.clip(e, -127, 127)
        byte, scale = e + 127, 2.0 ** e.astype(np.float64)
    else:
        byte = nearest(np.minimum(safe / 6, 448.0), E4M3)
        scale = E4M3[byte]
    b = np.where(fine[..., None], b, 0.0)
    s = scale[..., None]
    q = nearest(np.minimum(np.where(s > 0, np.abs(b) / np.where(s > 0, s, 1.0), 0.0), 6.0), E2M1)
    code = q + 8 * np.signbit(b)
    code = np.where(fine[..., None], code, 0).reshape(rows, wide)
    byte = np.where(fine, byte, 255 if fmt == MX else 127)
    byte = np.where(np.arange(byte.shape[1]) * n < K, byte, 0)
    out = np.zeros((rows, 2 * pitch(K)), dtype=np.uint8)
    out[:, :min(wide, out.shape[1])] = code[:, :out.shape[1]]
    return out, byte.astype(np.uint8)


def pack(code):
    return code[:, 0::2] | (code[:, 1::2] << 4)


def places(rows, offsets):
    """Row of the scale tiles of each row; -1 where the row is in no group."""
    r = np.arange(rows)
    if offsets is None:
        return r
    at = np.full(rows, -1)
    for g in range(len(offsets) - 1):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        at[lo:hi] = (lo // 128 + g) * 128 + np.arange(hi - lo)
    return at


def store_scales(byte, offsets, groups, fill=0):
    """[rows][4 * kt] -> the tiles, `fill` where no row is."""
    rows, kt = byte.shape[0], byte.shape[1] // 4
    flat = np.full(((rows // 128 + groups) * 128, kt * 4), fill, dtype=np.uint8)
    at = places(rows, offsets)
    flat[at[at >= 0]] = byte[at >= 0]
    return flat.reshape(-1, 4, 32, kt, 4).transpose(0, 3, 2, 1, 4).reshape(-1).copy()


def values(code, byte, fmt, K):
    v = np.where(code & 8, -1.0, 1.0) * E2M1[code & 7]
    s = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127)) if fmt == MX else np.append(E4M3, np.nan)[byte & 127]
    return v[:, :K] * np.repeat(s, BLOCK[fmt], 1)[:, :K]


def random_stored(rng, rows, K, fmt, spread=2):
    """Random codes and scales around 1: (codes [rows][2 * pitch], bytes)."""
    code = rng.integers(0, 16, (rows, 2 * pitch(K)), dtype=np.uint8)
    code[:, K:] = 0
    kt = scale_tiles(fmt, K)
    byte = (127 + rng.integers(-spread, spread + 1, (rows, 4 * kt))) if fmt == MX else rng.integers(0x38 - 8 * spread, 0x39 + 8 * spread, (rows, 4 * kt))
    byte[:, -(-K // BLOCK[fmt]):] = 0
    return code, byte.astype(np.uint8)


def route(x, k, chosen):
    """x: float64 [T][E] -> (index, weight, offsets, slot, source), -1 where there is none."""
    T, E = x.shape
    index, weight = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    for t in range(T):
        key = np.where(np.isnan(x[t]), -np.inf, x[t])
        order = np.argsort(-key, kind="stable")
        order = order[key[order] > -np.inf]
        if len(order) == 0:
            continue
        pick = order[:k]
        with np.errstate(invalid="ignore"):
            p = np.exp(x[t] - key[order[0]])
        total = p[pick].sum() if chosen else p[key > -np.inf].sum()
        index[t, :len(pick)] = pick
        weight[t, :len(pick)] = np.nan if np.isnan(x[t]).any() else p[pick] / total
    slot, source = np.full((T, k), -1, dtype=np.int64), np.full(T * k, -1, dtype=np.int64)
    offsets, at = np.zeros(E + 1, dtype=np.int64), 0
    for e in range(E):
        offsets[e] = at
        for t, j in zip(*np.nonzero(index == e)):
            slot[t, j], source[at] = at, t
            at += 1
    offsets[E] = at
    return index, weight, offsets, slot, source
