"""The 8-bit row format and its operators in 64 bits, for the tests: by table and search, on the CPU.

Rounding to e4m3 is to the nearest code (half a step is 2^-4 of a value, 2^-10 below 2^-6), ties to the even
code; the power of a block is the first of 2^-126 .. 2^127 that brings its largest finite magnitude to 448
at most, 1 for a block of zeros."""
import torch

BLOCK = 128
TABLE = torch.tensor([(c % 8) * 2.0 ** -9 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)], dtype=torch.float64)
POWERS = torch.tensor([2.0 ** e for e in range(-126, 128)], dtype=torch.float64)


def padded(k):
    blocks = -(-k // BLOCK)
    return blocks, -(-blocks // 4) * 4


def nearest(v):
    """code bytes of 64-bit values within +-448 (NaN and infinities: NaN)"""
    a = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v))
    hi = torch.searchsorted(TABLE, a.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = TABLE[hi] - a, a - TABLE[lo]
    pick = torch.where(up < down, hi, torch.where(down < up, lo, torch.where(hi % 2 == 0, hi, lo)))
    pick = torch.where(torch.isfinite(v), pick, torch.full_like(pick, 127))
    return (pick + 128 * torch.signbit(v)).to(torch.uint8)


def quantise(v):
    """[m][k] 64-bit -> (codes uint8 [m][kp], power bytes uint8 [m][pitch])"""
    m, k = v.shape
    blocks, pitch = padded(k)
    full = torch.zeros(m, blocks * BLOCK, dtype=torch.float64)
    full[:, :k] = v
    full = full.view(m, blocks, BLOCK)
    top = torch.where(torch.isfinite(full), full.abs(), torch.zeros_like(full)).amax(-1)
    e = torch.searchsorted(448 * POWERS, top).clamp(max=253)
    e = torch.where(top > 0, e, torch.full_like(e, 126))
    powers = torch.full((m, pitch), 127, dtype=torch.uint8)
    powers[:, :blocks] = (e + 1).to(torch.uint8)
    return nearest(full / POWERS[e].unsqueeze(-1)).view(m, -1), powers


def values(codes, powers):
    """what codes [m][kp] and power bytes [m][pitch] stand for, 64-bit"""
    c = codes.view(torch.uint8).cpu()
    p = powers.view(torch.uint8).cpu()
    m, kp = c.shape
    mag = (c & 127).long()
    v = torch.where(mag == 127, torch.full(mag.shape, float("nan"), dtype=torch.float64), TABLE[mag.clamp(max=126)])
    v = torch.where(c >= 128, -v, v).view(m, kp // BLOCK, BLOCK)
    return (v * 2.0 ** (p[:, :kp // BLOCK].double() - 127).unsqueeze(-1)).view(m, kp)


def to_type(v, dtype):
    """64-bit values rounded once to fp32 or bf16 (half to even)"""
    if dtype == torch.float32:
        return v.float().double()
    _, e = torch.frexp(v)
    unit = 2.0 ** (e.double().clamp(min=-125) - 8)
    r = torch.round(v / unit) * unit
    return torch.where(torch.isfinite(v), r, v)


def norm(h, y, gain, eps):
    """(h', its norm), 64-bit; h of the stream's type"""
    s = h.double() if y is None else to_type(h.double() + y.double(), h.dtype)
    return s, s / torch.sqrt((s * s).mean(1, keepdim=True) + eps) * gain.double()


def product(x, w):
    """(x w^T, the same of magnitudes)"""
    return x @ w.T, x.abs() @ w.abs().T
