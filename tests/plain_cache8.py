"""A cache of 8 bits in plain torch: numbers (e4m3), powers of two of blocks of 16 tokens, appending; rotation in 64 bits."""
import torch

BLOCK, LEAST = 16, -110
E4M3 = torch.float8_e4m3fn


def two_to(e):
    """2^e in fp64, from its bits (a power function need not be exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def power(most):
    """The least power of two from 2^LEAST on, 448 times which is not below `most` (fp64, exact)."""
    e = torch.floor(torch.log2(torch.where(most > 0, most, 1.0).double())) - 10        # (448 is below 2^9; log2 may be off by one at powers of two)
    for _ in range(4):
        e = torch.where(448.0 * two_to(e) < most.double(), e + 1, e)
    return two_to(torch.where(most > 0, e, LEAST).clamp(min=LEAST))


def numbers(x, p):
    """x / p rounded to e4m3; what is not finite becomes NaN.  (The division is exact, so x may be fp32 or fp64.)"""
    y = torch.where(torch.isfinite(x), x.double() / p, 0.0).float().to(E4M3).view(torch.uint8)
    return torch.where(torch.isfinite(x), y, 0x7f)


def values(codes, p):
    return codes.view(E4M3).double() * p.double()


def finite_most(x, dims):
    return torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dims)


def quantised(pages):
    """Pages [n, page, H, D] of any type -> codes (uint8), scales [n, H, page / 16] fp32."""
    n, page, H, D = pages.shape
    x = pages.float().reshape(n, page // BLOCK, BLOCK, H, D)
    p = power(finite_most(x, (2, 4)))
    return numbers(x, p[:, :, None, :, None]).view(n, page, H, D), p.float().transpose(1, 2).contiguous()


def dequantised(codes, scales):
    n, page, H, D = codes.shape
    return values(codes.reshape(n, page // BLOCK, BLOCK, H, D), scales.transpose(1, 2)[:, :, None, :, None]).view(n, page, H, D)


def append(codes, scales, x, seqs, table, n_pages):
    """Adds the rows x [T, H, D] (fp64) of sequences (new rows, keys with them) to codes and scales, block by block."""
    page, row = codes.shape[1], 0
    for i, (a, n) in enumerate(seqs):
        first = max(0, n - a)
        for b in range(first // BLOCK, -(-n // BLOCK) if n > first else 0):
            column = b * BLOCK // page
            at = int(table[i, column]) if column < table.shape[1] else -1
            if not 0 <= at < n_pages:
                continue
            lo, hi = max(first, b * BLOCK), min(n, (b + 1) * BLOCK)
            block, r0 = b * BLOCK % page // BLOCK, b * BLOCK % page
            new = x[row + lo - (n - a):row + hi - (n - a)]
            p = power(finite_most(new, (0, 2)))
            if lo > b * BLOCK:
                before = scales[at, :, block].double()
                p = torch.maximum(p, before)
                old = codes[at, r0:r0 + lo - b * BLOCK]
                nan = torch.isnan(old.view(E4M3).float())
                again = (old.view(E4M3).double() * (before / p)[:, None]).float().to(E4M3).view(torch.uint8)
                codes[at, r0:r0 + lo - b * BLOCK] = torch.where(nan, 0x7f, again)
            codes[at, r0 + lo - b * BLOCK:r0 + hi - b * BLOCK] = numbers(new, p[:, None])
            scales[at, :, block] = p.float()
        row += a


def same_numbers(a, b):
    """Equal, any NaN being any other."""
    nan = lambda x: (x & 0x7f) == 0x7f
    return bool(((a == b) | (nan(a) & nan(b))).all())


def turned(x, position, inv_freq, interleaved=False, back=False):
    """x [T, H, D] turned, in fp64; and for tolerances the sizes |a cos| + |b sin| of its sums."""
    x = x.double()
    rot = 2 * inv_freq.numel()
    angle = position.double()[:, None, None] * inv_freq.double()
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if back else 1)
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y, size = x.clone(), x.abs()
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (a * s).abs() + (b * c).abs()
    reach = torch.zeros_like(x)                      # |a| + |b|: what an error of the sines and cosines is multiplied with
    reach[..., first] = reach[..., second] = a.abs() + b.abs()
    return y, size, reach


def turn_tolerance(x, position, inv_freq, interleaved, back, dtype):
    """How far the kernels' results may be off: angles in 64 bits (three roundings, 2^-53 each, of up to `angle`), their part of a turn in fp32 (half a step of a number
    below one half-turn, pi 2^-25), sine and cosine (2 steps of numbers up to 1: 2^-23), fp32 products and their sum (2^-24 each), one rounding to dtype."""
    y, size, reach = turned(x, position, inv_freq, interleaved, back)
    angle = float(position.max()) * float(inv_freq.abs().max())
    w = 3.2 * 2.0 ** -25 + 2.0 ** -23 + 4 * angle * 2.0 ** -53
    rot = 2 * inv_freq.numel()
    size[..., rot:] = 0
    half = torch.finfo(dtype).eps / 2
    return y, half * y.abs() + (1 + half) * (w * reach + 3 * 2.0 ** -24 * size) + 1e-37
