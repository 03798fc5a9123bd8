"""GPU parity of the cache's write with plain 32-bit arithmetic, bit for bit."""
import pytest
import torch

import layer_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp16", "int8", "e4m3"])
@pytest.mark.parametrize("T,heads,kv,D", [(1, 4, 4, 64), (16, 64, 8, 128), (301, 10, 10, 128)])
def test_write_is_plain_arithmetic(T, heads, kv, D, kind):
    """Rotation with every product and sum rounded for itself, codes of the products with the inverse step: queries, codes and scales are
    those of elementary operations in 32 bits, rounding's edges included."""
    import paper_2312_03788_amd as sqp
    print("case plain write", T, heads, kv, D, kind, flush=True)
    g = ref.gen(70)
    q, k, v = [ref.randn(g, T, h, D).half() for h in (heads, kv, kv)]
    table, page = ref.cos_sin_table(9000, D), 16
    positions = torch.randint(0, 9000, (T,), generator=g, dtype=torch.int32)
    pages = -(-T // page) + 1
    slots = torch.randperm(pages * page, generator=g)[:T].int()
    cache = [torch.zeros((pages, kv, page, D), dtype=torch.float16, device="cuda").to(ref.TYPES[kind]) for _ in range(2)]
    scales = [None if kind == "fp16" else torch.zeros((pages, kv, page), device="cuda") for _ in range(2)]
    qr = sqp.kv_cache_write(k.cuda(), v.cuda(), slots.cuda(), *cache, *scales, q=q.cuda(), cos_sin=table.cuda(), positions=positions.cuda())

    c, s = table[positions.long()][:, None].chunk(2, -1)

    def turn(x):
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    assert torch.equal(qr.cpu(), turn(q).half())
    at, place = slots.long() // page, slots.long() % page
    for x, got, step in ((turn(k), *(t[0] for t in (cache, scales))), (v.float(), *(t[1] for t in (cache, scales)))):
        got = got.cpu()
        if kind == "fp16":
            assert torch.equal(got[at, :, place], x.half())
            continue
        top, most = x.abs().amax(-1), ref.QMAX[kind]
        z = x * (torch.tensor(most) / top)[..., None]
        codes = torch.round(z).to(torch.int8) if kind == "int8" else z.to(torch.float8_e4m3fn)
        assert torch.equal(step.cpu()[at, :, place], top / most)
        assert torch.equal(got.view(torch.uint8)[at, :, place], codes.view(torch.uint8))
