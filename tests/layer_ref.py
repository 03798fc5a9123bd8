"""Plain 64-bit forms of the operators between the linears (residual and norm, paged cache, attention over it) on the CPU,
and inputs for them."""
import numpy as np
import torch

TYPES = {"fp16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
QMAX = {"int8": 127.0, "e4m3": 448.0}
HALF_STEP = {torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float32)


def code_gap(values, kind):
    """Distance of neighbouring codes around these code values (e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6)."""
    if kind == "int8":
        return torch.ones_like(values)
    e = torch.floor(torch.log2(values.abs().clamp(min=2.0 ** -6)))
    return 2.0 ** (e - 3)


def add_rmsnorm(x, residual, gamma, eps):
    """(y, r) in 64 bits: r is exact, y is the norm of r rounded to fp16."""
    r = x.double() + residual.double()
    v = r.half().double()
    return v * gamma.double() / torch.sqrt(v.pow(2).mean(1, keepdim=True) + eps), r


def rotate(x, cos_sin, positions):
    cs = cos_sin.double()[positions.long()][:, None]
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h].double(), x[..., h:].double(), cs[..., :h], cs[..., h:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def cos_sin_table(n, D, theta=1e6):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def make_cache(g, pages, kv_heads, page, D, kind):
    """(codes, scales) of a full cache."""
    shape = (pages, kv_heads, page, D)
    if kind == "fp16":
        c = randn(g, *shape).half()
        c[..., ::37] *= 3
        return c, None
    scales = (1.0 + randn(g, *shape[:3]).abs()) / QMAX[kind] * torch.exp2(torch.randint(-3, 4, shape[:3], generator=g).float())
    if kind == "int8":
        return torch.randint(-127, 128, shape, generator=g, dtype=torch.int8), scales
    return (randn(g, *shape) * 110).clamp(-448, 448).to(torch.float8_e4m3fn), scales


def dequantised(cache, scales):
    return cache.double() if scales is None else cache.float().double() * scales.double()[..., None]


def spoil(cache, scales, free):
    """NaN in the places of a cache that `free` [pages, page] marks (as never written memory may hold)."""
    at = free[:, None, :].expand(cache.shape[:3])
    if cache.dtype == torch.float16:
        cache[at] = float("nan")
    elif cache.dtype == torch.float8_e4m3fn:
        cache.view(torch.uint8)[at] = 0x7f
    if scales is not None:
        scales[at] = float("nan")


class Step:
    """Sequences with `lens` cached tokens, `news` of them new, on shuffled pages; every place of the cache that no
    sequence uses is NaN, and the page table's entries past a sequence's pages lie far outside the cache."""

    def __init__(self, lens, news, heads, kv_heads, D, page, kind, seed=1, q_scale=1.0):
        g = gen(seed)
        self.lens, self.news, self.heads, self.kv_heads, self.D, self.page, self.kind = lens, news, heads, kv_heads, D, page, kind
        need = [-(-n // page) for n in lens]
        pages = sum(need) + 1
        width = max(1, max(need, default=1))
        order = torch.randperm(pages, generator=g).int()
        self.table = torch.tensor([1 << 30, -5], dtype=torch.int32).repeat(len(lens) * width)[: len(lens) * width].reshape(len(lens), width).clone()
        free = torch.ones((pages, page), dtype=torch.bool)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at: at + n]
            for i in range(n):
                free[order[at + i].long(), : lens[b] - i * page] = False
            at += n
        self.k, self.ks = make_cache(g, pages, kv_heads, page, D, kind)
        self.v, self.vs = make_cache(g, pages, kv_heads, page, D, kind)
        self.q = (q_scale * randn(g, sum(news), heads, D)).half()
        spoil(self.k, self.ks, free)
        spoil(self.v, self.vs, free)
        self.starts = torch.tensor([sum(news[:b]) for b in range(len(news) + 1)], dtype=torch.int32)
        self.seq_lens = torch.tensor(lens, dtype=torch.int32)

    def gpu(self, q=None):
        c = lambda t: None if t is None else t.cuda()
        return dict(q=c(self.q if q is None else q), k_cache=c(self.k), v_cache=c(self.v), page_table=c(self.table), seq_lens=c(self.seq_lens),
                    q_starts=c(self.starts), k_scales=c(self.ks), v_scales=c(self.vs))

    def rows(self, b, cache, scales):
        """A sequence's cached tokens in 64 bits [kv_heads, len, D]."""
        t = torch.arange(self.lens[b])
        pages, place = self.table[b].long()[t // self.page], t % self.page
        x = cache.view(torch.uint8)[pages, :, place].view(cache.dtype) if cache.dtype == torch.float8_e4m3fn else cache[pages, :, place]
        return dequantised(x, None if scales is None else scales[pages, :, place]).transpose(0, 1)

    def expected(self, scale=None, rows=None, p_error=2.0 ** -11, rounded=True):
        """(out, tolerance) [T, heads, D] in 64 bits (rows: (sequence, new token, head) to compute, the others are left zero).

        The kernels hold scores, sums and outputs in fp32 and round p to fp16 once, the output once.  With A = sum_j p_j |v_j|:
          output's rounding       2^-11 |o| + 2^-25 (half a step, half of the smallest one)
          p's rounding            2^-11 A, and half of the smallest step per token where p is far below the row's largest
          scores                  a score of D products is off by at most (D + 8) 2^-24 sum_d |q_d k_d| scale, the power of two
                                  by 2^-21: a p by that share, the numerator and the denominator both
          sums over the tokens    len 2^-24 each
        (p_error: p's share; rounded=False: without the output's rounding.)"""
        scale = self.D ** -0.5 if scale is None else scale
        T = self.q.shape[0]
        out, tol = torch.zeros((T, self.heads, self.D), dtype=torch.float64), torch.full((T, self.heads, self.D), 2.0 ** -25 if rounded else 0.0, dtype=torch.float64)
        group = self.heads // self.kv_heads
        for b, (length, n) in enumerate(zip(self.lens, self.news)):
            if length == 0:
                continue
            first = int(self.starts[b])
            k, v = self.rows(b, self.k, self.ks), self.rows(b, self.v, self.vs)
            sees = torch.arange(length)[None, :] <= (length - n + torch.arange(n))[:, None]
            for h in range(self.heads):
                if rows is not None and not any(r[0] == b and r[2] == h for r in rows):
                    continue
                q, kh, vh = self.q[first: first + n, h].double(), k[h // group], v[h // group]
                for i in range(n) if rows is None else [r[1] for r in rows if r[0] == b and r[2] == h]:  # (one row at a time over what it sees: what it does not see may be NaN)
                    m = int(sees[i].sum())
                    if m == 0:
                        continue
                    s = kh[:m] @ q[i] * scale
                    p = torch.softmax(s, 0)
                    size = kh[:m].abs() @ q[i].abs() * scale
                    o, A = p @ vh[:m], p @ vh[:m].abs()
                    e = (self.D + 8) * 2.0 ** -24 * float(size.max()) + 2.0 ** -21
                    out[first + i, h] = o
                    tol[first + i, h] += (2.0 ** -11 * o.abs() if rounded else 0.0) + (p_error + 2 * e + m * 2.0 ** -23) * A + m * 2.0 ** -25 * p.max() * vh[:m].abs().max()
        return out, tol
