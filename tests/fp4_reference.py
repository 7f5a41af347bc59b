"""Plain implementations (64 bits, on the CPU) of the residual norm and of 4-bit operands, for the tests to compare with."""
import math

import torch

MX, NV = 0, 1
BLOCK = {MX: 32, NV: 16}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
E2M1_CODES = torch.tensor(E2M1 + [-v for v in E2M1], dtype=torch.float64)
NAN = float("nan")


def e4m3_value(byte: int) -> float:
    e, m = (byte >> 3) & 15, byte & 7
    if e == 15 and m == 7:
        return NAN
    v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -v if byte & 0x80 else v


E4M3_CODES = torch.tensor([e4m3_value(b) for b in range(256)], dtype=torch.float64)
E8M0_CODES = torch.tensor([2.0 ** (b - 127) for b in range(255)] + [NAN], dtype=torch.float64)


def nearest(values, x):
    """Index of the value next to each x >= 0 among `values` (rising, one per code from 0), ties to the even index, beyond the
    last to the last."""
    borders = (values[:-1] + values[1:]) / 2
    up = torch.searchsorted(borders, x.contiguous(), right=False)           # borders strictly below x
    tie = (up < len(borders)) & (x == borders[up.clamp(max=len(borders) - 1)])
    return torch.where(tie & (up % 2 == 1), up + 1, up)


def tensor_scale(top: float) -> float:
    if not (0 < top < math.inf):
        return 1.0
    return 2.0 ** max(-100, min(100, math.floor(math.log2(2688.0 / top))))


def quantise(src, fmt, g=1.0):
    """(codes [R, C] as integers, scale bytes [R, blocks]) of a matrix (fp32 values); v = src * g with one fp32 rounding."""
    n = BLOCK[fmt]
    R, C = src.shape
    v = torch.nn.functional.pad((src.float() * torch.tensor(g, dtype=torch.float32)), (0, -C % n)).view(R, -1, n).double()
    finite = torch.isfinite(v).all(-1)
    v = torch.where(finite[..., None], v, torch.zeros((), dtype=torch.float64))
    top = v.abs().amax(-1)
    if fmt == MX:
        exponent = torch.where(top > 0, torch.frexp(top).exponent - 1, torch.full_like(top, -1000).int())
        byte = (exponent - 2 + 127).clamp(min=0)
        s = E8M0_CODES[byte.long()]
    else:
        byte = nearest(E4M3_CODES[:127], top / 6)
        s = E4M3_CODES[byte]
    q = torch.where(s[..., None] > 0, v / s[..., None], torch.zeros((), dtype=torch.float64))
    code = nearest(torch.tensor(E2M1, dtype=torch.float64), q.abs()) + 8 * (torch.signbit(v) & (s[..., None] > 0)).long()
    byte = torch.where(finite, byte.long(), torch.full_like(byte.long(), 0xff if fmt == MX else 0x7f))
    return code.view(R, -1)[:, :C], byte


def pack_codes(code):
    """[R, C] integers -> bytes, two codes each, rows padded with zeros to 16 bytes."""
    code = torch.nn.functional.pad(code, (0, -code.shape[1] % 32)).to(torch.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4)


def tile_scales(byte):
    """Scale bytes [R, blocks] in the operand's order, entry by entry."""
    R, nb = byte.shape
    tiles = -(-nb // 4)
    out = torch.zeros(-(-R // 128) * tiles * 512, dtype=torch.uint8)
    r, b = torch.arange(R)[:, None], torch.arange(nb)[None, :]
    out[((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4] = byte.to(torch.uint8)
    return out


def untile_scales(tiled, R, nb):
    tiles = -(-nb // 4)
    r, b = torch.arange(R)[:, None], torch.arange(nb)[None, :]
    return tiled[((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4]


def values(code, byte, fmt, g=1.0):
    """What integers [R, C] and scale bytes stand for."""
    table = E8M0_CODES if fmt == MX else E4M3_CODES
    return E2M1_CODES[code.long()] * table[byte.long()].repeat_interleave(BLOCK[fmt], dim=1)[:, :code.shape[1]] / g


def norm(h, gain, eps):
    """(y, rstd) of stored h."""
    h = h.double()
    rstd = 1 / torch.sqrt((h * h).mean(-1) + eps)
    return h * rstd[:, None] * (1.0 if gain is None else gain.double()), rstd


def norm_backward(dy, h, gain, rstd, dh):
    dy, h, rstd = dy.double(), h.double(), rstd.double()[:, None]
    g = dy * (1.0 if gain is None else gain.double())
    dx = rstd * (g - h * rstd * (g * h * rstd).mean(-1, keepdim=True))
    return dx + (0.0 if dh is None else dh.double()), (dy * h * rstd).sum(0)
