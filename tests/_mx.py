"""The mxfp4 cache in 64 bits, from its definition: values of E2M1 codes and E8M0 scales, rounding of
rows, and the place of every channel in a slice (by byte address)."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """Rows [..][D] (fp64) -> codes [..][D] (0..15) and scale bytes [..][D/32]."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(g).max(-1)
    bad = ~np.isfinite(top)
    m, e = np.frexp(np.where(bad | (top == 0), 1.0, top))          # top = m 2^e, m in [1/2, 1)
    e = e - 1 + (m >= 0.875)                                       # exponent of top at one mantissa bit
    byte = np.clip(np.where(top == 0, 0, e - 2 + 127), 8, 252)
    a = np.minimum(np.abs(np.where(bad[..., None], 0.0, g)) / np.exp2(byte - 127.0)[..., None], 6.0)
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    code = np.searchsorted(E2M1, np.rint(a / step) * step) + 8 * (np.signbit(g) & ~bad[..., None])
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def values(codes, scales):
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = np.concatenate([E2M1, -E2M1])[codes]
    return (v.reshape(*scales.shape, 32) * s[..., None]).reshape(codes.shape)


def places(ps, D, which):
    """Byte of every channel's code, whether it is the high nibble, and byte of its group's scale, in a
    slice of [ps][D]."""
    t, c = np.arange(ps)[:, None], np.arange(D)[None]
    if which == "k":
        at, sc = t * (D // 2) + c // 2, t * (D // 32) + c // 32
    else:
        at = (((t // 4) * 16 + c // (D // 16)) * 4 + t % 4) * (D // 32) + c % (D // 16) // 2
        sc = ((t // 4) * (D // 32) + c // 32) * 4 + t % 4
    return at, np.broadcast_to(c % 2 == 1, at.shape), ps * D // 2 + sc


def pack(x, which):
    """fp64 [P][H][ps][D] -> uint8 [P][H][ps][17 D / 32]."""
    P, H, ps, D = x.shape
    codes, scales = quantize(x)
    at, high, sc = places(ps, D, which)
    out = np.zeros((P, H, ps * D * 17 // 32), np.uint8)
    for odd in (False, True):
        m = high == odd
        out[..., at[m]] |= (codes[..., m] << (4 * odd)).astype(np.uint8)
    out[..., sc[:, ::32]] = scales
    return out.reshape(P, H, ps, D * 17 // 32)


def unpack(cache, which):
    """uint8 [P][H][ps][17 D / 32] -> fp64 values [P][H][ps][D]."""
    P, H, ps, rb = cache.shape
    D = rb * 32 // 17
    at, high, sc = places(ps, D, which)
    flat = cache.reshape(P, H, -1)
    codes = (flat[..., at] >> (4 * high)) & 15
    return values(codes, flat[..., sc[:, ::32]])


def attend(q, k, v, scale):
    """Softmax attention of heads q [g][D] over rows k, v [n][D] in fp64: output, and the weighted mean
    of |v| and the largest sum |q_c k_c|, which bound its rounding."""
    z = scale * (q @ k.T)
    w = np.exp(z - z.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    return w @ v, w @ np.abs(v), (np.abs(q) @ np.abs(k).T).max()


def attend_tolerance(ref, absv, qk, scale, D, n):
    """Scores: D products added in fp32, each within 2^-23 of the running sum's bound qk; the exponent's
    error is a weight's relative error, twice (numerator and sum).  The weights' split into two bf16
    parts leaves 2^-16, n fp32 additions n 2^-23, the exponentials and rescales a few 2^-22.  The
    result rounds to bf16: 2^-8 of it."""
    delta = 2 * scale * D * 2.0 ** -23 * qk + 2 * (n + 64) * 2.0 ** -23 + 2.0 ** -15
    return 2.0 ** -8 * (np.abs(ref) + delta * absv) + delta * absv + 1e-30
