"""Plain forms of the 8-bit float layers and of dropout for the tests, on the CPU: quantisation in binary32 as the library defines it, values in 64 bits, random bits from
integers of Python's own size or numpy's."""
import numpy as np
import torch

FORMATS = {0: torch.float8_e4m3fn, 1: torch.float8_e5m2}
LARGEST = {0: 448.0, 1: 57344.0}


def quantized(v, format, block):
    """(codes float8 [rows,columns], scales float32 [bands,chunks]) of a matrix; divisions of binary32 numbers on the CPU are rounded once."""
    v = v.float().cpu()
    rows, columns = v.shape
    padded = torch.nn.functional.pad(v, (0, -columns % 128, 0, -rows % block))
    b = padded.view(padded.shape[0] // block, block, -1, 128)
    bits = b.abs().contiguous().view(torch.int32).amax((1, 3))
    scales = (bits.view(torch.float32).double() / LARGEST[format]).float()      # (the quotient of two binary32 numbers rounded to 53 bits, then to 24, is rounded once)
    scales[bits >= 0x7F800000] = float("nan")
    s = scales[:, None, :, None]
    q = torch.where(s > 0, (b / s).clamp(-LARGEST[format], LARGEST[format]), 0.0)
    return q.to(FORMATS[format]).view(padded.shape[0], -1)[:rows, :columns].contiguous(), scales


def values(codes, scales, block):
    """codes times their scales, in 64 bits."""
    rows, columns = codes.shape
    return codes.double() * scales.double().repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :columns]


def product(a, b):
    """(a b^T, the bound of what binary32 sums may be off by) for values [M,K], [N,K]: chunks of 128 products, each sum of at most 128 additions that round or cut off at
    2^-23 of what was added up, a scale and its product (3 roundings), one more addition per chunk."""
    chunks = -(-a.shape[1] // 128)
    return a @ b.T, (128 + 3 + chunks) * 2.0 ** -23 * (a.abs() @ b.abs().T)


def cut_off(a, b, lowest):
    """What a chunk's sums of 16-bit results may lose besides: of eight neighbouring products each but the largest is cut off at less than 2^-13 of the largest one's power of two,
    which is no more than the product of the two largest values (or of the smallest normal codes' values `lowest`, ([M,K], [N,K]) with the scales in them)."""
    def largest(v, low):
        pad = -v.shape[1] % 8
        v, low = (torch.nn.functional.pad(t, (0, pad)).view(v.shape[0], -1, 8).amax(2) for t in (v.abs(), low))
        return torch.maximum(v, low)
    return 7 * 2.0 ** -13 * largest(a, lowest[0]) @ largest(b, lowest[1]).T


def lowest_values(scales, rows, columns, format, block):
    """The value of the smallest normal code at every place."""
    return (2.0 ** -6 if format == 0 else 2.0 ** -14) * scales.double().repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :columns]


def philox(counter, key):
    """Philox 4x32-10 of numpy uint64 arrays (or numbers) below 2^32."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(w) for w in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def random_bits(rows, columns, seed, offset, first_row=0):
    """u of nova_dropout, uint32 [rows,columns]."""
    groups = -(-columns // 8)
    row, column = np.meshgrid(np.arange(first_row, first_row + rows, dtype=np.uint64), np.arange(groups, dtype=np.uint64), indexing="ij")
    o = offset % 2 ** 64

    def halves(second):
        w = philox([column, row + np.uint64(second << 31), np.full_like(row, o & 0xFFFFFFFF), np.full_like(row, o >> 32)], (seed & 0xFFFFFFFF, seed % 2 ** 64 >> 32))
        return np.stack(w, 2).astype("<u4").view("<u2").reshape(rows, groups * 8)[:, :columns].astype(np.uint32)
    return halves(0) << np.uint32(16) | halves(1)


def kept(rows, columns, p, seed, offset):
    return torch.from_numpy(random_bits(rows, columns, seed, offset).astype(np.int64) >= int(p * 2.0 ** 32 + 0.5))
