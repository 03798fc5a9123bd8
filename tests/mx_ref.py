"""Plain 64-bit forms of the operators on microscaled numbers (blocks of 32, a power-of-two scale each) on the CPU."""
import torch

import layer_ref as ref

BLOCK = 32
DTYPES = {"e2m1": torch.uint8, "e4m3": torch.float8_e4m3fn}
# the values of the non-negative codes, in the order of the codes, and what would follow the last one
GRIDS = {"e2m1": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 8.0],
         "e4m3": [i / 512 for i in range(8)] + [(8 + i) / 8 * 2.0 ** e for e in range(-6, 9) for i in range(8)]}
assert GRIDS["e4m3"][-2:] == [448.0, 480.0]


def grid(kind):
    return torch.tensor(GRIDS[kind], dtype=torch.float64)


def two(e):
    return torch.ldexp(torch.ones((), dtype=torch.float64), e.double())


def nearest(a, kind):
    """Place of the nearest grid value of a >= 0; of two equally near ones the even place."""
    g = grid(kind)
    middle = (g[1:] + g[:-1]) / 2
    below, above = torch.searchsorted(middle, a), torch.searchsorted(middle, a, right=True)
    return torch.where(below % 2 == 0, below, above)


def quantise(z, kind):
    """(codes, scale bytes) of rows z [R, K] in 64 bits: codes one to an element, sign in bit 3 (e2m1) or 7."""
    R, K = z.shape
    b = z.double().reshape(R, K // BLOCK, BLOCK)
    most = b.abs().amax(-1)
    bad, some = ~torch.isfinite(most), most >= 2.0 ** -100
    last = len(GRIDS[kind]) - 1
    m = torch.where(some & ~bad, most, 1.0)
    e = torch.floor(torch.log2(m)) - {"e2m1": 2, "e4m3": 8}[kind] - 2
    for _ in range(5):  # up to the least power of two with which the largest magnitude rounds to a value of the type
        y = m / two(e)
        e = torch.where((y > GRIDS[kind][-1]) | (nearest(y, kind) == last), e + 1, e)
    keep = (some & ~bad)[..., None]
    y = torch.where(keep, b, 0.0) / two(e)[..., None]
    codes = nearest(y.abs(), kind) + torch.signbit(y) * {"e2m1": 8, "e4m3": 128}[kind]
    codes = torch.where(keep, codes, 0)
    byte = torch.where(bad, 255.0, torch.where(some, e + 127, 0.0))
    return codes.reshape(R, K).to(torch.uint8), byte.to(torch.uint8)


def pack(codes, kind):
    """The bytes of codes as the operators hold them."""
    if kind == "e4m3":
        return codes
    c = codes.unflatten(-1, (-1, 2))
    return c[..., 0] | c[..., 1] << 4


def raw(codes):
    """Bytes of the operators' codes."""
    return codes.cpu().view(torch.uint8)


def typed(packed, kind):
    return packed.contiguous() if kind == "e2m1" else packed.contiguous().view(torch.float8_e4m3fn)


def values(packed, scales, kind):
    """What bytes of codes [..., K/2 or K] and scales [..., K/32] stand for, 64 bits (a scale of 255: NaN)."""
    p = packed.long()
    c = torch.stack([p & 15, p >> 4], -1).flatten(-2) if kind == "e2m1" else p
    sign = {"e2m1": 8, "e4m3": 128}[kind]
    y = grid(kind)[c % sign] * (1.0 - 2.0 * (c >= sign))
    step = torch.where(scales == 255, float("nan"), two(scales.double() - 127))
    return (y.unflatten(-1, (-1, BLOCK)) * step[..., None]).flatten(-2)


def random_rows(g, R, K, spread=6):
    """fp16 rows whose blocks differ in size by powers of two, with some larger channels."""
    x = ref.randn(g, R, K // BLOCK, BLOCK) * torch.exp2(torch.randint(-spread, spread + 1, (R, K // BLOCK, 1), generator=g).float())
    x[..., ::13] *= 5.0
    return x.reshape(R, K).half()


def product(x, xs, x_kind, w, ws, silu=False):
    """(y, tolerance) in 64 bits of the product of x (bytes) and e2m1 w.

    fp32: an instruction adds the products of 64 or 128 k to the running sum; each addition cuts or rounds by at most 2^-23 of
    what is added so far, at most T = sum |x w|: K / 32 + 16 of them are more than there are.
    e4m3: products are lined up to the largest of their instruction's and cut below 2^-13 of it (seen: 2^-3 beside 6 x 448 is
    kept, 2^-4 is not).  Groups of 128 k in the order of k are no subset of an instruction's k, so the largest is taken over a stage
    of 512 k, and at least the row's share of what is multiplied there is bounded by it: K x 2^-13 x largest over 512.
    Then fp16's half step of the result."""
    X, W = values(x, xs, x_kind), values(w, ws, "e2m1")
    K = X.shape[1]
    y, T = X @ W.t(), X.abs() @ W.abs().t()
    err = (K / 32 + 16) * 2.0 ** -23 * T
    if x_kind == "e4m3":
        for k in range(0, K, 512):
            a, b = X[:, k: k + 512].abs(), W[:, k: k + 512].abs()
            # the largest product of a row and a column is at most the largest over k of the two's product
            err = err + a.shape[1] * 2.0 ** -13 * _largest(a, b)
    if silu:
        gate, up, dg, du = y[:, 0::2], y[:, 1::2], err[:, 0::2], err[:, 1::2]
        s = gate * torch.sigmoid(gate)
        # |SiLU'| <= 1.1; the hardware's exponential and the quotient 2^-20
        y, err = s * up, 1.1 * up.abs() * dg + s.abs() * du + 1.1 * dg * du + 2.0 ** -20 * (s * up).abs()
    return y, err + 2.0 ** -11 * (y.abs() + err) + 2.0 ** -25


def _largest(a, b):
    out = torch.zeros((a.shape[0], b.shape[0]), dtype=torch.float64)
    for k in range(a.shape[1]):
        torch.maximum(out, a[:, k: k + 1] * b[:, k], out=out)
    return out


class Step(ref.Step):
    """A step over a cache of e2m1 blocks; places that no sequence uses have the scale 255 (NaN)."""

    def __init__(self, lens, news, heads, kv_heads, D, page, seed=1, q_scale=1.0, spread=3):
        super().__init__(lens, news, heads, kv_heads, D, page, "fp16", seed, q_scale)
        free = self.k[:, 0, :, 0].isnan()
        g = ref.gen(seed + 1000)
        shape = self.k.shape
        made = []
        for c in (self.k, self.v):
            x = random_rows(g, shape[0] * shape[1] * shape[2], D, spread)
            codes, scales = quantise(x, "e2m1")
            codes, scales = pack(codes, "e2m1").reshape(*shape[:3], D // 2), scales.reshape(*shape[:3], D // 32)
            scales[free[:, None, :].expand(shape[:3])] = 255
            made += [codes, scales]
        self.k, self.ks, self.v, self.vs = made

    def rows(self, b, cache, scales):
        t = torch.arange(self.lens[b])
        pages, place = self.table[b].long()[t // self.page], t % self.page
        return values(cache[pages, :, place], scales[pages, :, place], "e2m1").transpose(0, 1)
