"""Plain numpy restatement of the matrix operators (microscaled 4-bit floats, their product, the orthogonalised update)
in 64 bits, written from their definitions and sharing no code with the library: test infrastructure only."""
import numpy as np

MX, NV = 0, 1
BLOCK = {MX: 32, NV: 16}
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
# E4M3: sign left out, 4 bits of exponent (bias 7), 3 of mantissa; 0x7F is NaN
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
E8M0 = 2.0 ** np.arange(-127.0, 128.0)


def draws(index, seed, worker, epoch):
    """16-bit draws of element indices: Philox4x32-10 (Salmon, Moraes, Dror, Shaw), counter (i >> 3, worker, epoch)."""
    mask = np.uint64(0xFFFFFFFF)
    i = np.asarray(index, dtype=np.uint64)
    c = [(i >> np.uint64(3)) & mask, i >> np.uint64(35), np.full_like(i, worker), np.full_like(i, epoch)]
    k = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32 & 0xFFFFFFFF)]
    for _ in range(10):
        p, q = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(q >> np.uint64(32)) ^ c[1] ^ k[0], q & mask, (p >> np.uint64(32)) ^ c[3] ^ k[1], p & mask]
        k = [(k[0] + np.uint64(0x9E3779B9)) & mask, (k[1] + np.uint64(0xBB67AE85)) & mask]
    w = np.choose(((i >> np.uint64(1)) & np.uint64(3)).astype(np.int64), c)
    return (w >> (np.uint64(16) * (i & np.uint64(1)))) & np.uint64(0xFFFF)


def tensor_exponent(x):
    x = np.abs(np.asarray(x, dtype=np.float64))
    top = np.max(np.where(np.isfinite(x), x, 0.0))
    t = -126
    while t < 126 and top > 2688.0 * 2.0 ** t:
        t += 1
    return t


def quantize(x, fmt, t=0, seed=None, worker=0, epoch=0):
    """(codes uint8[rows, cols], scale bytes uint8[rows, blocks], whether a block was not finite) of a matrix."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    size = BLOCK[fmt]
    nb = -(-cols // size)
    full = np.zeros((rows, nb * size))
    full[:, :cols] = x
    b = full.reshape(rows, nb, size)
    fine = np.isfinite(b).all(2)
    b = np.where(fine[:, :, None], b, 0.0)
    top = np.abs(b).max(2)
    if fmt == MX:
        byte = np.minimum(np.searchsorted(6.0 * E8M0[:254], top), 253)
        q = np.abs(b) / E8M0[byte][:, :, None]
    else:
        with np.errstate(over="ignore"):
            byte = np.minimum(np.searchsorted(6.0 * E4M3, top * 2.0 ** -t), 126)
            s = np.where(byte > 0, E4M3[byte], 1.0)[:, :, None]
            q = (np.abs(b) * 2.0 ** -t / s).astype(np.float32).astype(np.float64)
    q = np.minimum(q, 6.0)
    low = np.searchsorted(GRID, q, side="right") - 1
    high = np.minimum(low + 1, 7)
    share = np.where(low < 7, (q - GRID[low]) / np.where(low < 7, GRID[high] - GRID[low], 1.0), 0.0)
    if seed is None:
        up = (share > 0.5) | ((share == 0.5) & (low % 2 == 1))
    else:
        index = np.arange(rows)[:, None] * (-(-cols // 32) * 32) + np.arange(nb * size)[None, :]
        up = (draws(index, seed, worker, epoch).reshape(b.shape) + 0.5) / 65536.0 < share
    level = np.where(up, high, low)
    codes = (level + 8 * ((b < 0) & (level > 0))).astype(np.uint8)
    return codes.reshape(rows, nb * size)[:, :cols], byte.astype(np.uint8), bool((~fine).any())


def pack(codes):
    """Two codes to a byte, rows padded with zeros to 32 elements."""
    rows, cols = codes.shape
    full = np.zeros((rows, -(-cols // 32) * 32), dtype=np.uint8)
    full[:, :cols] = codes
    return full[:, 0::2] | (full[:, 1::2] << 4)


def tiles(byte):
    """Scale bytes [rows, blocks] in tiles of 128 rows by 4 blocks."""
    rows, nb = byte.shape
    out = np.zeros((-(-rows // 128), -(-nb // 4), 512), dtype=np.uint8)
    r, k = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    out[r // 128, k // 4, r % 32 * 16 + r // 32 % 4 * 4 + k % 4] = byte
    return out.reshape(-1)


def values(codes, byte, fmt, t=0):
    scale = E8M0[byte] if fmt == MX else E4M3[byte] * 2.0 ** t
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    return v * np.repeat(scale, BLOCK[fmt], axis=1)[:, :codes.shape[1]]


def orthogonalize(x, steps=5, a=3.4445, b=-4.7750, c=2.0315):
    x = np.asarray(x, dtype=np.float64)
    turned = x.shape[0] > x.shape[1]
    x = x.T if turned else x
    norm = np.sqrt((x * x).sum())
    x = x / norm if norm > 0 else x
    for _ in range(steps):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if turned else x
