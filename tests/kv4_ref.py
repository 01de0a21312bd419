"""Plain 64-bit forms of the 4-bit cache and of the attention over it, for the tests: written from the format's definition,
sharing nothing with the library."""
import numpy as np
import torch

TOP, BAD = 0xC6, 0xFF


def scale_table():
    """float64 value of every scale byte: e = b >> 3, m = b & 7."""
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3, b & 7
        out[b] = m * 2.0 ** -17 if e == 0 else (8 + m) * 2.0 ** (e - 18)
        if e == 31:
            out[b] = np.nan
    return out


TABLE = scale_table()


def quantise(x):
    """x [..., hd] float64 (exact values of the inputs) -> codes c [..., hd] (0..15), scale bytes [..., hd / 16]."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // 16, 16))
    finite = np.isfinite(b).all(-1)
    b = np.where(finite[..., None], b, 0.0)
    amax = np.abs(b).max(-1)
    byte = np.minimum(np.searchsorted(7.0 * TABLE[:TOP + 1], amax, side="left"), TOP)
    s = TABLE[byte][..., None]
    ratio = np.divide(b, s, out=np.zeros_like(b), where=s > 0)
    c = np.clip(np.rint(ratio), -7, 7).astype(np.int64) + 8
    byte = np.where(finite, byte, BAD)
    return c.reshape(x.shape), byte


def values(c, byte):
    return (c - 8.0) * np.repeat(TABLE[byte], 16, axis=-1)


def pack(c, byte, buf, n_kv, capacity, hd, pos0):
    """Codes [n, n_kv, hd] and bytes into rows pos0.. of a packed uint8 numpy array."""
    codes, scales = parts(buf, n_kv, capacity, hd)
    n = c.shape[0]
    two = (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)
    codes[:, pos0:pos0 + n] = two.transpose(1, 0, 2)
    scales[:, pos0:pos0 + n] = byte.astype(np.uint8).transpose(1, 0, 2)


def parts(buf, n_kv, capacity, hd):
    half = n_kv * capacity * hd // 2
    total = half + n_kv * capacity * hd // 16
    return buf[:half].reshape(n_kv, capacity, hd // 2), buf[half:total].reshape(n_kv, capacity, hd // 16)


def unpack(buf, n_kv, capacity, hd):
    """All rows of a packed array as float64 [capacity, n_kv, hd]."""
    codes, scales = parts(buf, n_kv, capacity, hd)
    c = np.stack((codes & 15, codes >> 4), -1).reshape(n_kv, capacity, hd).astype(np.float64)
    return values(c, scales.astype(np.int64)).transpose(1, 0, 2)


def attention(q, k, v, seen):
    """q [R, nq, hd], k / v [N, nkv, hd] float64, seen [R, N] bool -> (out [R, nq, hd], spread of each (row, head): the largest
    sum of |q_d k_d| / sqrt(hd) over its keys, and the largest |v| it sees)."""
    R, nq, hd = q.shape
    G = nq // k.shape[1]
    out, b, a = np.zeros_like(q), np.zeros((R, nq)), np.zeros((R, nq))
    for r in range(R):
        idx = np.nonzero(seen[r])[0]
        if len(idx) == 0:
            continue
        for h in range(nq):
            kk, vv = k[idx, h // G], v[idx, h // G]
            s = kk @ q[r, h] / np.sqrt(hd)
            p = np.exp(s - s.max())
            out[r, h] = p @ vv / p.sum()
            b[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() / np.sqrt(hd)
            a[r, h] = np.abs(vv).max()
    return out, b, a


def tolerance(out, spread, vmax, bf16):
    """Bound on |library - out| from the roundings the kernels make.
      scores: 16-wide multiplies added in fp32 in at most 16 steps (2^-23 of the terms' magnitudes each, truncation counted as a
              whole step), operands exact (bf16 rows) or two half-precision parts (2^-22): d = spread (2^-19 + 2^-22 + 2^-21)
              with two more roundings for the scale to base 2 and the power of two, each 2^-24 of a score <= spread;
      weights: exp2 2^-22, half precision 2^-11 (bf16 models) or two parts 2^-22; weights below 2^-24 of the largest lose at
              most 2^-35 each, 2^-22 x vmax for 2^13 keys of that kind (no test has more);
      sums:   fp32 in runs of at most 64 additions per level, 2^-17;  both enter numerator and denominator.
      result: half a step of its type."""
    d = spread * (2.0 ** -19 + 2.0 ** -21 + 2.0 ** -22) + 2.0 ** -22
    w = 2.0 ** -11 if bf16 else 2.0 ** -21
    rel = 2.0 ** -8 if bf16 else 2.0 ** -24
    return rel * np.abs(out) + (vmax * (2 * d + w + 2.0 ** -18))[..., None]


def seen_mask(R, T, ctx, own, visible=None):
    """[R, ctx (+ R)]: cache positions, then the rows' own."""
    m = np.zeros((R, ctx + (R if own else 0)), dtype=bool)
    for r in range(R):
        m[r, :ctx if visible is None else min(ctx, max(0, int(visible[r])))] = True
        if own:
            m[r, ctx + r // T * T:ctx + r + 1] = True
    return m


def to_np(t):
    return t.double().cpu().numpy()


def bytes_np(t):
    return t.cpu().numpy().copy() if isinstance(t, torch.Tensor) else t
