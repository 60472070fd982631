"""A plain form of the 8-bit key/value cache and of attention over it, per
sequence, in numpy (test infrastructure only).

What the cache holds is defined in 32-bit steps (a float32 scale, the float32
quotient rounded to a whole number), so it is computed in those; everything
after that is in 64 bits."""
import numpy as np

BLOCK = 32


def quantised(x):
    """x [BLOCK, heads, hd] float32 -> whole numbers, scales [1, heads, 1] (float32)."""
    amax = np.abs(x).max(axis=(0, 2), keepdims=True)
    scale = (np.maximum(amax, np.float32(2.0 ** -80)) / np.float32(127)).astype(np.float32)
    with np.errstate(all="ignore"):
        scale = np.where(np.isfinite(amax), scale, np.float32(np.nan))
        return np.rint((x / scale).astype(np.float32)), scale


def held(x):
    """What the cache holds of a sequence's rows x [tokens, heads, hd] (float32
    values of 16-bit numbers): float64, the same shape."""
    out = x.astype(np.float64)
    for b in range(x.shape[0] // BLOCK):
        q, scale = quantised(x[b * BLOCK:(b + 1) * BLOCK])
        out[b * BLOCK:(b + 1) * BLOCK] = q.astype(np.float64) * scale.astype(np.float64)
    return out


def attend(q, k, v, pos):
    """q [rows, H, hd], k, v [tokens, KV, hd] as held, row r at position pos[r]
    (sees tokens <= it): (out [rows, H, hd], largest |v| seen [rows, H])."""
    rows, H, hd = q.shape
    rep = H // k.shape[1]
    out, top = np.zeros((rows, H, hd)), np.zeros((rows, H))
    for r in range(rows):
        n = int(pos[r]) + 1
        if n <= 0:
            continue
        for h in range(H):
            s = k[:n, h // rep] @ q[r, h].astype(np.float64) / np.sqrt(hd)
            with np.errstate(invalid="ignore"):
                w = np.exp(s - s.max())
                out[r, h] = (w / w.sum()) @ v[:n, h // rep]
            top[r, h] = np.abs(v[:n, h // rep]).max()
    return out, top
