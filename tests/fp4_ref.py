"""The 4-bit format by its definition, in 64 bits on the CPU."""
import numpy as np

CODES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(w):
    """(values of the codes, scales as bytes) of float64 rows x cols, padded to 128 columns."""
    w = np.asarray(w, dtype=np.float64)
    R, C = w.shape
    n = -(-C // 128) * 128
    v = np.zeros((R, n))
    v[:, :C] = w
    v = v.reshape(R, n // 32, 32)
    with np.errstate(invalid="ignore"):
        bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    amax = np.abs(v).max(-1)
    e = np.zeros(amax.shape, int)
    for t in range(-127, 126):  # the smallest that is enough
        e = np.where((amax > 6 * 2.0 ** (t - 1)) & (t > -127) | (t == -127), t, e)
    e = np.where(amax == 0, 0, e)
    y = np.abs(v) * 2.0 ** -e[..., None].astype(np.float64)
    d = np.abs(y[..., None] - CODES)
    near = d.argmin(-1)
    # halfway: the code with an even number
    tie = (near < 7) & (np.take_along_axis(d, np.minimum(near + 1, 7)[..., None], -1)[..., 0] == d.min(-1))
    near = np.where(tie & (near % 2 == 1), near + 1, near)
    codes = np.copysign(CODES[near], v)
    return np.where(bad[..., None], 0.0, codes).reshape(R, n), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, cols):
    """float64 rows x cols."""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    R = codes.shape[0]
    return (codes.reshape(R, -1, 32) * s[..., None]).reshape(R, -1)[:, :cols]


def unpack(codes, scales, rows, cols):
    """(codes' values, scales' bytes) by row, rows x padded columns, of tiles of 16 x 128
    (uint8 ceil(rows / 16) x pitch each)."""
    down, across = -(-rows // 16), -(-cols // 128)
    v, s = np.zeros((16 * down, 128 * across)), np.zeros((16 * down, 4 * across), np.uint8)
    signed = np.concatenate([CODES, -CODES])
    for i in range(down):
        for j in range(across):
            t = codes[i, 1024 * j: 1024 * (j + 1)].reshape(4, 16, 4, 4)  # g, r, k, b
            for g in range(4):
                for k in range(4):
                    for b in range(4):
                        byte, c = t[g, :, k, b], 128 * j + 32 * k + 8 * g + 2 * b
                        v[16 * i: 16 * i + 16, c], v[16 * i: 16 * i + 16, c + 1] = signed[byte & 15], signed[byte >> 4]
            s[16 * i: 16 * i + 16, 4 * j: 4 * j + 4] = scales[i, 64 * j: 64 * (j + 1)].reshape(16, 4)
    assert (v[rows:] == 0).all() and (s[rows:] == 127).all()
    return v[:rows], s[:rows]
