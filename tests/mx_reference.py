"""MXFP4 in 64 bits, from its definition, for the tests of the microscaled layers."""
import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def blocks(k):
    return (k + 31) // 32


def exponents(x):
    """Scale bytes of x's rows (64-bit, whole blocks of 32: ... x 32): ... ."""
    top = x.abs().amax(dim=-1)
    e = torch.frexp(torch.where(torch.isfinite(top) & (top > 0), top, torch.ones(()).double()))[1] - 1
    byte = torch.where(top > 0, (e + 125).clamp_min(0), 0)
    return torch.where(torch.isfinite(top), byte, 255).to(torch.uint8)


def power(byte):
    """What scale bytes are worth, in 64 bits (255: NaN)."""
    v = (byte.long() - 127 + 1023 << 52).view(torch.float64)
    return torch.where(byte == 255, torch.full((), float("nan")).double(), v)


def nearest(a):
    """Codes 0..7 of magnitudes: the nearest number of GRID, the even code of two."""
    code = torch.zeros(a.shape, dtype=torch.uint8)
    for i in range(1, 8):
        middle = (GRID[i - 1] + GRID[i]) / 2
        code += (a >= middle if i % 2 == 0 else a > middle).to(torch.uint8)
    return code


def padded(x):
    """x's rows in 64 bits, in whole blocks: m x blocks x 32."""
    m, k = x.shape
    full = torch.zeros((m, blocks(k) * 32), dtype=torch.float64)
    full[:, :k] = x.double()
    return full.view(m, blocks(k), 32)


def quantize(x):
    """(codes 0..15 of m x blocks x 32, scale bytes) of x's rows."""
    p = padded(x)
    byte = exponents(p)
    scaled = torch.where((byte == 255)[..., None], torch.zeros(()).double(), p / power(byte)[..., None])
    return nearest(scaled.abs()) + 8 * (torch.signbit(p) & (byte != 255)[..., None]).to(torch.uint8), byte


def pack(codes):
    """Bytes of codes (... x blocks x 32): ... x blocks * 16."""
    c = codes.flatten(-2)
    return c[..., 0::2] | c[..., 1::2] << 4


def unpack(w):
    return torch.stack([w & 15, w >> 4], dim=-1).flatten(-2)


def values(w, scale, k):
    """64-bit values of packed rows."""
    c = unpack(w).long()
    v = GRID[c & 7] * (1 - 2.0 * (c >> 3))
    return (v.view(*scale.shape, 32) * power(scale)[..., None]).flatten(-2)[..., :k]


def matrix(g, n, k, spread=3, base=121):
    """Random codes and scales: n rows of k, the padding random too."""
    w = torch.randint(0, 256, (n, blocks(k) * 16), generator=g, dtype=torch.uint8)
    s = torch.randint(base, base + spread, (n, blocks(k)), generator=g, dtype=torch.uint8)
    return w, s
