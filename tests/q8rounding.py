"""Keys of 8-bit caches by the formula in 64 bits (torch, on whatever device the inputs are), and what
may be said of numbers that come out as another e4m3 number than the formula's.

fp32's error of a key's number, u = 2^-24, S = |x_own w_own| + |x_other w_other| over the norm's root:
cosine and sine are within 1.2 ulps, at most 2.4 u of themselves; a product and the joining one rounding
each: 4.4 u S, below 2^-21 S.  With the norm, 1 u for the weight's product, 13 u of the mean of squares
(8 in a lane's chain, at most 4 across lanes, 1 with eps), half of it in the root, 2 u of the root
and 1 u of its product: 15 u S, below 2^-20 S.  A number may round to the other side only as near
to a border.  Numbers whose fp32 form comes within 2 ulps of a border are formed in 64 bits, so that of
those at least 2^-6 of the power which are not a small difference (S <= 1.25 of them) only those are
left that fp32 has more than 2 ulps off: with errors e of root mean square s the share of plain
fp32's that remains is E max(|e| - 2, 0) / E |e| <= (s^2 / 8) / (s / 2) = s / 4 (|e| - 2 <= e^2 / 8; and
E |e| >= s / 2 for anything as compact as a sum of roundings): below 1/4 for s up to 1."""
import torch

E4 = torch.float8_e4m3fn
PLAIN, NORMED = 2.0 ** -21, 2.0 ** -20


def turned64(x, weight, eps, cos, sin):
    """(numbers, S) in 64 bits of x [n, d] (bf16), cos and sin [n, d/2] (fp64)."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    lo, hi = y.chunk(2, dim=-1)
    m = lo.abs() + hi.abs()
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1), torch.cat([m, m], dim=-1)


def turned32(x, weight, eps, cos, sin):
    """The same in plain fp32."""
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * weight
    lo, hi = y.chunk(2, dim=-1)
    c, s = cos.float(), sin.float()
    return torch.cat([lo * c - hi * s, hi * c + lo * s], dim=-1)


def power(top):
    """The smallest 2^e, e in [-60, 119], with top <= 448 2^e, of fp64 magnitudes."""
    m, e = torch.frexp(top)  # m in [0.5, 1): 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.exp2(torch.where(top > 0, e, -60).clamp(-60, 119).double())


def rounded(z):
    """fp64 numbers, |z| <= 448, as e4m3 ones: to nearest, ties to even."""
    _, e = torch.frexp(z)
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(z / step) * step


def judged(number, scale, want, size, bound):
    """Of numbers [n, d] (fp64, as their e4m3 values) and their rows' powers scale [n] against the
    formula's `want` with S = `size`: (how many rows have another power or number than the formula's,
    how many rounded the other way among the numbers counted above).  Fails where one is off by more
    than `bound` S allows."""
    top, p = want.abs().amax(-1), power(want.abs().amax(-1))
    other = scale != p
    if other.any():
        line = 448.0 * torch.minimum(p, scale)[other]
        assert (((scale / p)[other] == 2) | ((scale / p)[other] == 0.5)).all()
        assert ((top[other] - line).abs() <= bound * size.amax(-1)[other]).all()
    z = want / scale[:, None]
    wrong = (number != rounded(z.clamp(-448, 448))) & ~other[:, None]
    # a number on the other side of a border: the border is half way to the formula's number
    right = rounded(z.clamp(-448, 448))
    off = (z - (number + right) / 2).abs() * scale[:, None]
    assert (off[wrong] <= (bound * size)[wrong]).all(), (off[wrong] / size[wrong]).max()
    counted = (z.abs() >= 2.0 ** -6) & (size <= 1.25 * want.abs())
    return int((other | wrong.any(-1)).sum()), int((wrong & counted).sum())


def quantised32(y):
    """Numbers and powers of fp32 keys, as a caller's plain form would have them."""
    p = power(y.abs().amax(-1).double())
    return rounded((y.double() / p[:, None]).clamp(-448, 448)), p
