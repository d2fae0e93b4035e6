"""Blocks of 32 elements under a power of two, in 64 bits and from the definition (tests only)."""
import torch

E2M1 = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def two_to(e):
    """2^e in f64 for integers -1000 < e < 1000."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exponent(amax, top):
    """The smallest integer e >= -127 with amax <= top 2^e; 128 (a byte of 255) where amax is no number."""
    fine = torch.isfinite(amax)
    a = torch.where(fine, amax, torch.ones_like(amax))
    m, p = torch.frexp(a.clamp_min(2.0 ** -200) / top)     # a / top = m 2^p, .5 <= m < 1
    e = torch.where(m == 0.5, p - 1, p).clamp_min(-127)
    e = torch.where(a > top * two_to(e), e + 1, e)         # the division's own rounding
    return torch.where(fine, e, torch.full_like(e, 128))


def nearest(x, bits, smallest):
    """(x rounded to `bits` bits after the leading one, spacing at least `smallest`, ties to even; the spacing)."""
    m, p = torch.frexp(x.abs().clamp_min(2.0 ** -300))
    step = two_to(p - 1 - bits).clamp_min(smallest)
    return torch.round(x / step) * step, step


def blocks(x):
    n = -(-x.shape[1] // 32)
    full = torch.zeros((x.shape[0], 32 * n), dtype=torch.float64, device=x.device)
    full[:, :x.shape[1]] = x.double()
    return full.reshape(x.shape[0], n, 32)


def quantize4(x):
    """(values [rows, blocks, 32] as multiples of the scale, scale bytes [rows, blocks]) of e2m1 blocks."""
    b = blocks(x)
    e = exponent(b.abs().amax(-1), 6.0)
    v, _ = nearest(torch.nan_to_num(b / two_to(e).unsqueeze(-1)), 1, 0.5)
    return torch.where((e == 128).unsqueeze(-1), torch.zeros_like(v), v), (e + 127).to(torch.uint8)


def round8(x):
    """(values, spacings, both scaled back, scales): x in blocks of e4m3."""
    b = blocks(x)
    s = two_to(exponent(b.abs().amax(-1), 448.0)).unsqueeze(-1)
    v, step = nearest(b / s, 3, 2.0 ** -9)
    return (v * s).reshape(x.shape), (step * s).reshape(x.shape), s.squeeze(-1)


def codes4(codes):
    """Four-bit codes, two to a byte, as f64 values [rows, blocks, 32]."""
    both = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1, 32)
    return E2M1.to(codes.device)[both.long()]


def values4(codes, scales):
    return (codes4(codes) * scales.view(torch.float8_e8m0fnu).double().unsqueeze(-1)).reshape(codes.shape[0], -1)


def tiles(byte):
    """Scale bytes [rows, blocks] in tile order, zeros behind the last row and block."""
    R, C = -(-byte.shape[0] // 128), -(-byte.shape[1] // 4)
    out = torch.zeros((R, C, 32, 4, 4), dtype=torch.uint8, device=byte.device)
    r = torch.arange(byte.shape[0], device=byte.device)[:, None]
    b = torch.arange(byte.shape[1], device=byte.device)[None, :]
    out[r // 128, b // 4, r % 32, r % 128 // 32, b % 4] = byte
    return out


def untiles(s, rows, nblocks):
    r = torch.arange(rows, device=s.device)[:, None]
    b = torch.arange(nblocks, device=s.device)[None, :]
    return s.view(torch.uint8)[r // 128, b // 4, r % 32, r % 128 // 32, b % 4].view(torch.float8_e8m0fnu).double()


def ffn(x, gate, up, down, member):
    """(out, tolerance) [B, d] of the FFN in f64 on f64 operands; member [B, d_ff] bool: the channels of each token's support.

    The kernels add f32 products (exact: 4 + 2 significant bits and powers of two) in f32 over up to K terms and round a, then out.
    Tolerance, element by element:
      bf16 rounding of out                        2^-8 |out|
      f32 sums of the down product                2^-14 sum |a W|: 32 products at a time, so K / 32 <= 2^9 adds of partial sums that
                                                  are at most sum |a W|, each off by 2^-23 at most
      an element of a that lies within its own error of the middle between two e4m3 values, or whose block's largest lies so near the
      border of its scale, may round to the other one: its spacing times |W|.  Its error: f32 sums of K / 32 <= 2^8 adds, 2^-15 of the
      sum of magnitudes, and 2^-20 for the exponential, the division and the product."""
    g, u = x @ gate.t(), x @ up.t()
    ga, ua = x.abs() @ gate.abs().t(), x.abs() @ up.abs().t()
    sig = torch.sigmoid(g)
    silu = g * sig
    a = torch.where(member, silu * u, torch.zeros_like(g))
    # f32 sums: |dg| <= 2^-15 sum |x W|; silu' <= 1.1; the exponential and the division: 2^-20
    da = torch.where(member, 2.0 ** -15 * (1.1 * ga * u.abs() + silu.abs() * ua) + 2.0 ** -20 * a.abs(), torch.zeros_like(g))
    v, step, s = round8(a)
    top = a.abs().reshape(a.shape[0], -1, 32).amax(-1)
    border = ((top + da.reshape(a.shape[0], -1, 32).amax(-1) > 448 * s) | (top - da.reshape(a.shape[0], -1, 32).amax(-1) <= 224 * s))
    border = border.repeat_interleave(32, dim=1)
    tie = ((a / step - torch.floor(a / step) - 0.5).abs() * step <= da)
    # near a border of the scale the small elements of the block may move by the coarser step as well
    loose = torch.where(member & (tie | border), step + border * 2.0 ** -9 * s.repeat_interleave(32, dim=1), torch.zeros_like(a))
    out = v @ down.t()
    tol = 2.0 ** -8 * out.abs() + 2.0 ** -14 * (v.abs() @ down.abs().t()) + loose @ down.abs().t()
    return out, tol * (1 + 2.0 ** -7) + 1e-30
