"""The 8-bit form with block scales and its operators in 64 bits, plain torch on the CPU: what the tests hold the kernels to."""
import torch

B = 128


def blocks(n):
    return (n + B - 1) // B


def decode(codes):
    """E4M3 bytes -> float64, from the format: 1-4-3, bias 7, S.1111.111 NaN."""
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).double()), m / 8 * 2.0 ** -6)
    v = torch.where((c & 127) == 127, torch.full_like(v, float("nan")), v)
    return torch.where(c >= 128, -v, v)


def scale(bytes_):
    s = torch.exp2(bytes_.double() - 127)
    return torch.where(bytes_ == 255, torch.full_like(s, float("nan")), s)


def scale_byte(amax):
    """The least byte >= 1 with amax <= 448 * 2^(byte - 127), by search."""
    byte = torch.ones(amax.shape, dtype=torch.int64)
    for e in range(1, 255):
        byte = torch.where(amax > 448 * 2.0 ** (byte.double() - 127), torch.full_like(byte, e + 1), byte)
    return byte


def round_e4m3(v):
    """|v| <= 448 to the nearest E4M3 value, ties to even; NaN stays."""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 1).clamp_min(-6).double() - 3)
    return torch.round(v / step) * step


def magnitude(x):
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))


def along_rows(x):
    """Scale bytes [blocks x R] of blocks of 1 x 128 of x [R x C], and each element's scale."""
    R, C = x.shape
    m = torch.zeros(R, blocks(C) * B, dtype=torch.float64)
    m[:, :C] = magnitude(x)
    byte = scale_byte(m.reshape(R, -1, B).amax(2)).t().contiguous()
    return byte, per_element(byte, R, C)


def per_element(byte, R, C):
    """float64 [R x C] of scale bytes [blocks x >= R] along the rows."""
    return scale(byte[:, :R].to(torch.int64)).t().repeat_interleave(B, 1)[:, :C]


def per_element_down(byte, R, C):
    return scale(byte[:, :C].to(torch.int64)).repeat_interleave(B, 0)[:R]


def square(x):
    """Scale bytes [blocks of C x R], [blocks of R x C] of blocks of 128 x 128, and each element's scale."""
    R, C = x.shape
    m = torch.zeros(blocks(R) * B, blocks(C) * B, dtype=torch.float64)
    m[:R, :C] = magnitude(x)
    byte = scale_byte(m.reshape(blocks(R), B, blocks(C), B).amax((1, 3)))
    rows = byte.repeat_interleave(B, 0)[:R].t().contiguous()
    cols = byte.repeat_interleave(B, 1)[:, :C].contiguous()
    return rows, cols, per_element(rows, R, C)


def quantized(x):
    """(values in units of the scale, scale bytes [blocks x R])"""
    byte, s = along_rows(x)
    v = torch.where(torch.isfinite(x), x, torch.full_like(x, float("nan")))
    return round_e4m3(v / s), byte


def codes_of(values):
    """E4M3 bytes of values that the format has."""
    return values.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)


def random_codes(g, shape, std=1.0):
    return codes_of(round_e4m3((torch.randn(shape, generator=g, dtype=torch.float64) * std).clamp(-448, 448)))


def random_scales(g, nb, rows, lo=118, hi=132):
    """Scale bytes [nb x rows] at a pitch of whole sixteens; what lies past the rows is 255 (NaN): it must not matter."""
    s = torch.full((nb, (rows + 15) // 16 * 16), 255, dtype=torch.uint8)
    s[:, :rows] = torch.randint(lo, hi + 1, (nb, rows), generator=g, dtype=torch.int64).to(torch.uint8)
    return s


def sigmoid(x):
    return 1 / (1 + torch.exp(-x))


def swiglu(z):
    g, u = z[:, 0::2], z[:, 1::2]
    return g * sigmoid(g) * u


def swiglu_bwd(d, z):
    g, u = z[:, 0::2], z[:, 1::2]
    sg = sigmoid(g)
    out = torch.empty_like(z)
    out[:, 0::2] = d * u * (sg + g * sg * (1 - sg))
    out[:, 1::2] = d * g * sg
    return out
