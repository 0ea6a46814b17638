"""The 4-bit format of the KV cache in float64 NumPy: codes, scales and the bytes of a page (the library's own; the paper has
no cache).  Written from the definition, code by code and byte by byte."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])                        # E2M1 magnitudes, codes 0 .. 7
# scale byte b: 5 exponent bits with bias 15, 3 mantissa bits, no sign; 248 .. 254 are not used, 255 is NaN
SCALES = np.array([(b % 8) * 2.0 ** -17 if b < 8 else (1 + (b % 8) / 8) * 2.0 ** (b // 8 - 15) for b in range(248)])


def quantize(x):
    """x [..., dh] -> (codes uint8 [..., dh], scale bytes uint8 [..., dh / 32])."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    byte = np.minimum(np.searchsorted(6 * SCALES, np.abs(g).max(-1), side="left"), 247)     # the smallest scale with amax <= 6 s
    s = SCALES[byte][..., None]
    y = np.minimum(np.where(s > 0, np.abs(g) / np.where(s > 0, s, 1), 0.0), 8.0)              # above 5: code 7
    far = np.abs(y[..., None] - GRID)
    far[..., 1::2] *= 1 + 2.0 ** -40                                 # a tie goes to the even code
    code = far.argmin(-1) + 8 * (np.signbit(g) & ~bad[..., None])
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, byte).astype(np.uint8)


def values(code, byte):
    """What codes and scale bytes stand for, float64 [..., dh]."""
    s = np.concatenate([SCALES, np.full(8, np.nan)])[byte]
    m = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (m.reshape(byte.shape + (32,)) * s[..., None]).reshape(code.shape)


def places(dh):
    """Where a block of 16 tokens keeps things: (byte, shift) of code d of token s, byte of scale j of token s, for K and V."""
    half = 16 * dh // 2 + 16 * dh // 32
    kc, vc = np.zeros((16, dh), int), np.zeros((16, dh), int)
    ks, vs = np.zeros((16, dh // 32), int), np.zeros((16, dh // 32), int)
    for s in range(16):
        q, i = divmod(s, 4)
        for d in range(dh):
            j, e = divmod(d, 32)
            kc[s, d] = (s % 2 * 8 + s // 2) * (dh // 2) + e // 8 * (dh // 8) + j * 4 + e % 8 // 2
            g = e // 4
            at = (i // 2 * 512 + (g * 4 + q) * 16 + i % 2 * 8) if dh == 128 else (g * 4 + q) * 16 + i * 4
            vc[s, d] = half + at + j * 2 + e % 4 // 2
        for j in range(dh // 32):
            ks[s, j] = 8 * dh + s * (dh // 32) + j
            vs[s, j] = half + 8 * dh + q * (dh // 8) + j * 4 + i
    return kc, vc, ks, vs, np.arange(dh) % 2 * 4


def block_bytes(dh):
    return 17 * dh


def put(pool, page, head, slot, k, v):
    """Write one token's quantised k, v [..., dh] (leading axes: tracks) into pool uint8 [..., page, head, block, bytes]."""
    dh = k.shape[-1]
    kc, vc, ks, vs, shift = places(dh)
    blk = pool[..., page, head, slot // 16, :]
    s = slot % 16
    for x, at, sat in ((k, kc[s], ks[s]), (v, vc[s], vs[s])):
        code, byte = quantize(x)
        blk[..., at[::2]] = code[..., ::2] | code[..., 1::2] << 4
        blk[..., sat] = byte


def get(pool):
    """pool uint8 [..., pages, heads, blocks, bytes] -> values float64 [..., pages, K|V, heads, slots, dh]."""
    dh = pool.shape[-1] // 17
    kc, vc, ks, vs, shift = places(dh)
    out = []
    for at, sat in ((kc, ks), (vc, vs)):
        x = values(pool[..., at] >> shift & 15, pool[..., sat])      # [..., pages, heads, blocks, 16, dh]
        out.append(x.reshape(x.shape[:-3] + (-1, dh)))
    return np.stack(out, -4)
