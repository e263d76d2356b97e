"""What the tests of the residual-block operators (gf_block.h) share: the mask, the 8-bit format and drawn inputs, written
from the definitions on the host."""
import numpy as np
import torch

U = 2.0 ** -24                                                     # half a step of fp32
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step of a type, relative to the value
DTYPES = [torch.float32, torch.bfloat16]


def draw(shape, seed, dtype=torch.float32, scale=1.0, shift=0.0):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype)


def philox_bits(n, key, offset, first=0):
    """16 bits for each of the elements first .. first + n - 1 (first a multiple of 8): Philox4x32, ten rounds."""
    with np.errstate(over="ignore"):
        block = np.arange(-(-n // 8), dtype=np.uint64) + np.uint64(first // 8)
        low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
        c = [block & low, block >> half, np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, (offset >> 32) & 0xFFFFFFFF)]
        k = [key & 0xFFFFFFFF, (key >> 32) & 0xFFFFFFFF]
        for _ in range(10):
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        return np.stack(c, 1).astype("<u4").view("<u2").reshape(-1)[:n]


def seed_words(a, b=0):
    """The device tensor and the two words as unsigned numbers."""
    t = torch.tensor([a, b], dtype=torch.int64)
    return t.cuda(), tuple(int(v) & 0xFFFFFFFFFFFFFFFF for v in t)


def dropped(x, p, words, first=0):
    """x as fp64 after dropout with p: kept elements scaled, the others zero."""
    t = int(round(p * 65536))
    if t == 0:
        return x
    keep = (philox_bits(x.size, *words, first) >= t).reshape(x.shape)
    return np.where(keep, x * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)


def e4m3_values(codes):
    """uint8 codes (numpy) as fp64: sign, 4 exponent bits of bias 7, 3 mantissa bits; S.1111.111 is NaN."""
    c = codes.astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def e4m3_codes(v):
    """Magnitudes of at most 448 (and NaN) to the nearest code, ties to the even one: by searching the table of all values."""
    table = e4m3_values(np.arange(127, dtype=np.uint8))
    a = np.abs(np.asarray(v, dtype=np.float64))
    hi = np.clip(np.searchsorted(table, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = table[hi] - a, a - table[lo]
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    c = np.where(np.isnan(a), 127, c).astype(np.uint8)
    return np.where(np.signbit(v), c | 128, c).astype(np.uint8)


def random_codes(rows, cols, seed):
    """Codes of any finite value, [rows, pitch] with what lies behind the last column filled with NaN codes: it is not to be read."""
    g = np.random.RandomState(seed)
    pitch = -(-cols // 16) * 16
    c = g.randint(0, 254, (rows, pitch)).astype(np.uint8)
    c = np.where(c >= 127, c + 1, c).astype(np.uint8)               # 0 .. 126, 128 .. 254
    c[:, cols:] = 127
    return c
