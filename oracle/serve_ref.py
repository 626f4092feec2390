"""Float64 reference of the serving operators: rotation by positions, the paged
key-value cache with its 8- and 4-bit codes, and attention over packed
sequences and over cached tokens.

TEST INFRASTRUCTURE ONLY (like duo_ref): imported by tests only, shares no code
with the HIP path.

The cache's block of one page and head is [K rows][V rows][K scales][V scales].
Codes are integers: a group of 32 channels of one token and head has the scale
s = bf16(max |x| / q), q = 127 or 7, and the codes rint(x / s), stored with q + 1
added; a group whose s is below 2^-126 is zero, one that is not finite NaN.
"""

from __future__ import annotations

import numpy as np

GROUP = 32
MOST = {"int8": 127, "int4": 7}


def bf16(x):
    """Nearest bfloat16 of float64 values (ties to even; not for subnormals)."""
    m, e = np.frexp(np.asarray(x, dtype=np.float64))
    return np.ldexp(np.rint(m * 256.0), e - 8)


def bits(x):
    """bfloat16 bit patterns of float64 values that are bfloat16 numbers."""
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def rope_at(x, heads, head_dim, pos, theta):
    x = np.asarray(x, dtype=np.float64).reshape(-1, heads, 2, head_dim // 2)
    a = np.asarray(pos, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(head_dim // 2) / head_dim)
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    return np.stack((x[:, :, 0] * c - x[:, :, 1] * s, x[:, :, 1] * c + x[:, :, 0] * s), 2).reshape(len(x), -1)


def quantize(x, fmt):
    """(codes, scales) of rows x (m, kv, hd): integer codes without what is added
    to them, and float64 scales (m, kv, hd / 32)."""
    q = MOST[fmt]
    g = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (-1, GROUP))
    fin = np.isfinite(g).all(-1)
    g = np.where(fin[..., None], g, 0.0)
    s = bf16(np.abs(g).max(-1) / q)
    s = np.where(s < 2.0 ** -126, 0.0, s)
    live = s > 0
    codes = np.where(live[..., None], np.rint(g / np.where(live, s, 1.0)[..., None]), 0.0)
    codes = np.clip(codes, -q, q).astype(np.int64).reshape(x.shape)
    return codes, np.where(fin, s, np.nan)


def numbers(codes, scales):
    return codes * np.repeat(scales, GROUP, -1)


def block_bytes(page, hd, fmt):
    return page * 2 * {"bf16": 2 * hd, "int8": hd + 2 * hd // GROUP, "int4": hd // 2 + 2 * hd // GROUP}[fmt]


def write(data, K, V, slots, page, hd, fmt):
    """The bytes of a cache (pages, kv, block) after rows K and V (m, kv, hd
    float64 holding bfloat16 numbers) went to their slots."""
    out = np.array(data)
    pages, kv = data.shape[:2]
    rb = {"bf16": 2 * hd, "int8": hd, "int4": hd // 2}[fmt]
    sb = 0 if fmt == "bf16" else 2 * hd // GROUP
    for which, x in enumerate((K, V)):
        if fmt != "bf16":
            codes, scales = quantize(x, fmt)
            codes = (codes + MOST[fmt] + 1).astype(np.uint8)
            if fmt == "int4":
                codes = codes[..., 0::2] | codes[..., 1::2] << 4
            sbits = np.where(np.isnan(scales), np.uint16(0x7fc0), bits(np.where(np.isnan(scales), 0.0, scales)))
            sbytes = np.ascontiguousarray(sbits).view(np.uint8)
        for t, s in enumerate(slots):
            if not 0 <= s < pages * page:
                continue
            p, r = divmod(int(s), page)
            at = which * page * rb + r * rb
            out[p, :, at:at + rb] = np.ascontiguousarray(bits(x[t])).view(np.uint8) if fmt == "bf16" else codes[t]
            if sb:
                at = 2 * page * rb + which * page * sb + r * sb
                out[p, :, at:at + sb] = sbytes[t]
    return out


def attend(Q, K, V, scale, seen, extra=0.0):
    """One sequence: Q (lq, H, hd), K and V (lk, Hk, hd), seen (lq, lk) booleans.
    Returns (O, bound): the exact output and how far one may be from it that
    rounds its probabilities (times a scale of V) and its result to bf16 and
    keeps the rest in fp32.  Per element, with A = sum p |V|:
      2^-8 of A and of O for the two roundings (half a unit of eight bits), 2 % more
      for products of them;
      A times the error of a score: of hd products summed in fp32, and again of
      the score times its scale, both ways (numerator and sum);
      A times 2^-24 for every block of 32 keys that is added in fp32, and 2^-20 for
      exponentials and factors of the running maximum.
    extra: an error per score (lq, H, lk) besides, of codes with an offset."""
    lq, H, hd = Q.shape
    Hk = K.shape[1] if K.size else 1
    O = np.zeros((lq, H, hd))
    bound = np.zeros((lq, H, hd))
    if not len(K):
        return O, bound + 1e-37
    for h in range(H):
        k, v = K[:, h // (H // Hk)], V[:, h // (H // Hk)]
        S = np.where(seen, Q[:, h] @ k.T * scale, -np.inf)
        some = seen.any(1)
        p = np.exp(S - np.where(some, S.max(1, initial=-np.inf), 0.0)[:, None])
        p = p / np.where(some, p.sum(1), 1.0)[:, None]
        O[:, h] = p @ v
        A = p @ np.abs(v)
        err = np.where(seen, (np.abs(Q[:, h]) @ np.abs(k).T * hd + np.abs(Q[:, h] @ k.T)) * abs(scale) * 2.0 ** -24, 0.0)
        err = err + (extra[:, h] if np.ndim(extra) else extra)
        slack = 2 * np.where(seen, err, 0.0).max(1)[:, None] + (len(k) / 32 + 1) * 2.0 ** -24 + 2.0 ** -20
        bound[:, h] = (1.02 * 2.0 ** -8 + slack) * A + 1.02 * 2.0 ** -8 * np.abs(O[:, h]) + 1e-37
    return O, bound


def causal(lq, lk):
    return np.arange(lk)[None, :] <= np.arange(lq)[:, None] + lk - lq
