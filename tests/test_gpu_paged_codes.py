"""How far values of a page in 4 bits may be from what was stored, on the GPU: by the bounds that the header states, at the ends of the range and at far
positions; and rows past the caches against the definition."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2605_06763_amd as L
from test_gpu_paged import D, say
from test_gpu_paged_more import More, values

pytestmark = pytest.mark.gpu


def exponent(top):
    """The least e with top <= 7 * 2^e, from -120 to 125."""
    m, e = torch.frexp(top)
    return (e - 3 + (m > 0.875)).clamp(-120, 125)


def test_how_far_codes_are_off():
    """Blocks of all sizes that bf16 has: off by 2^e at most, less for small codes; what passes 7 * 2^125 becomes 6 * 2^125."""
    with More([(400, 400)], dtype="fp4", hq=4, hkv=4, seed=180) as c:
        x = torch.randn(c.T, c.hkv, 4, 32, generator=c.g, dtype=torch.float64)
        x *= 2.0 ** torch.randint(-135, 126, (c.T, c.hkv, 4, 1), generator=c.g)
        top = torch.tensor([7.0, 7.0625, 7.5, 7.96875, -7.96875, 6.0, 5.0], dtype=torch.float64) * 2.0 ** 125
        x[:40] = top[torch.randint(0, 7, (40, c.hkv, 4, 32), generator=c.g)]
        x[20:40] *= torch.rand(20, c.hkv, 4, 32, generator=c.g, dtype=torch.float64)
        v = x.flatten(2).to(c.dt)
        kp, vp = c.pools()
        start, length, table = c.batch()
        L.lvr_paged_append(c.h, kp, vp, v.cuda(), v.cuda(), start, length, table)
        K, V = (torch.empty(1, c.hkv, c.T, D, dtype=c.dt, device="cuda") for _ in range(2))
        L.lvr_paged_gather(c.h, kp, vp, length, table, K, V)
        x = v.double().unflatten(2, (4, 32))
        step = 2.0 ** exponent(x.abs().amax(dim=3, keepdim=True)).double()
        assert (x.abs() > 7 * 2.0 ** 125).sum() > 1000 and (step == 2.0 ** -120).sum() > 10
        for got in (K, V):
            y = got[0].cpu().double().transpose(0, 1).unflatten(2, (4, 32))
            beyond = x.abs() > 7 * step
            assert torch.equal(y[beyond], torch.sign(x[beyond]) * 6 * 2.0 ** 125)
            err, size = (y - x).abs() / step, x.abs() / step
            bound = torch.where(size < 2, 0.25, torch.where(size < 4, 0.5, 1.0))
            assert (err <= bound)[~beyond].all()


@pytest.mark.parametrize("pairs", [L.LVR_ROT_HALVES, L.LVR_ROT_NEIGHBOURS])
def test_codes_of_keys_at_far_positions(pairs):
    """At the farthest positions, frequencies up to 1e300: a code is that of a value off by |position| * 2^-64 of a turn at most, and by 64-bit arithmetic."""
    bits, two_pi = 1400, 0
    for n, f in ((5, 16), (239, -4)):            # pi = 16 atan(1/5) - 4 atan(1/239)
        term, k = (f << bits) // n, 0
        while term not in (0, -1):
            two_pi += 2 * (-(term // (2 * k + 1)) if k % 2 else term // (2 * k + 1))
            term, k = term // (n * n), k + 1
    freq = [10.0 ** (i / 4) * (-1) ** i for i in range(-8, 40)] + [1e6, 1e17, 2.0 ** 80, 3e300] * 4
    positions = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 10 ** 9 + 7, -10 ** 9, 12345, -1, 0] * 16
    turns = [[float(Fraction(p * Fraction(x).numerator << bits, Fraction(x).denominator * two_pi) % 1) for x in freq] for p in positions]
    angle = torch.tensor(turns, dtype=torch.float64)[:, None] * (2 * math.pi)
    with More([(128, 128)], dtype="fp4", hq=8, hkv=8, rot_dim=128, pairs=pairs, inv_freq=freq, seed=181) as c:
        k = c.randn(c.T, c.hkv, D)
        say(f"codes far off pairs={pairs}")
        kp, vp = c.pools()
        L.lvr_paged_append(c.h, kp, vp, k.cuda(), k.cuda(), *c.batch(), positions=torch.tensor(positions, dtype=torch.int32, device="cuda")[:, None])
        codes, scales = c.unpack(kp)
        at = [(int(c.table[0, p // c.page]), p % c.page) for p in range(c.T)]
        codes, scales = (torch.stack([x[i, :, r] for i, r in at]) for x in (codes, scales))
        got = values(codes, scales).unflatten(2, (4, 32))
        first, second = (slice(0, 64), slice(64, 128)) if pairs == L.LVR_ROT_HALVES else (slice(0, 128, 2), slice(1, 128, 2))
        u, w = k.double()[..., first], k.double()[..., second]
        x, size = torch.empty(c.T, c.hkv, D, dtype=torch.float64), torch.empty(c.T, c.hkv, D, dtype=torch.float64)
        x[..., first], x[..., second] = u * angle.cos() - w * angle.sin(), u * angle.sin() + w * angle.cos()
        size[..., first] = size[..., second] = u.abs() + w.abs()
        # sines off by 2^-50 (theirs) and by some units of 2^-53 here, three roundings of 2^-53 in the rotation
        off = (torch.tensor(positions, dtype=torch.float64).abs()[:, None, None] * (2 * math.pi * 2.0 ** -64) + 2.0 ** -48) * size
        x, off = x.unflatten(2, (4, 32)), off.unflatten(2, (4, 32))
        e = scales[..., None].double() - 127
        assert (e >= exponent((x.abs() - off).amax(dim=3, keepdim=True))).all() and (e <= exponent((x.abs() + off).amax(dim=3, keepdim=True))).all()
        step = 2.0 ** e
        levels = torch.tensor([-6.0, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
        middle = (levels[1:] + levels[:-1]) / 2

        def nearest(t):     # (no value lies on a border between two)
            return levels[torch.searchsorted(middle, t.clamp(-6, 6).contiguous())]
        assert (got / step >= nearest((x - off) / step)).all() and (got / step <= nearest((x + off) / step)).all()
        assert (off / step).max() < 1e-7


def test_rows_past_the_caches_are_the_codes_values():
    """Past 192 MiB of rows the gather stores around the caches: every row against the definition, page by page."""
    n, heads, page, pages = 100003, 8, 64, 1563
    g = torch.Generator(device="cuda").manual_seed(182)
    h = L.lvr_paged_create(L.make_paged_config(n_q_heads=heads, n_kv_heads=heads, kv_dtype=L.LVR_FP4, page_size=page, n_pages=pages, layout="token"))
    try:
        assert n * heads * 256 >= 192 << 20
        kp, vp = (torch.randint(0, 256, (pages, heads * page * 68), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        for p in (kp, vp):
            p[:, heads * page * 64:].clamp_(7, 252)
        table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None].contiguous()
        K, V = (torch.full((1, heads, n, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        L.lvr_paged_gather(h, kp, vp, torch.tensor([n], dtype=torch.int32, device="cuda"), table, K, V)
        levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
        levels = torch.cat([levels, -levels])
        for pool, rows in ((kp, K), (vp, V)):
            for p0 in range(0, pages, 100):
                ids = table[0, p0:p0 + 100].long()
                b = pool[ids, :heads * page * 64].view(-1, page, heads, 64).int()
                s = pool[ids, heads * page * 64:].view(-1, page, heads, 4).long() - 127
                s = (s + 1023 << 52).view(torch.float64)      # 2^s, exactly (pow on the GPU is off by a unit of the last place for some whole numbers)
                x = levels[torch.stack([b & 15, b >> 4], dim=-1).flatten(-2)].unflatten(-1, (4, 32)) * s[..., None]
                x = x.flatten(-2).flatten(0, 1).transpose(0, 1)[:, :n - p0 * page]      # [head][position][128]
                assert torch.equal(rows[0, :, p0 * page:p0 * page + x.shape[1]].double(), x)
    finally:
        L.lvr_paged_destroy(h)
