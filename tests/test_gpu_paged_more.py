"""The paged cache's pages in 4 bits, windows beside which first keys stay visible, and norms of queries and keys, on the GPU, against plain
implementations in 64 bits on the host.

Tolerances are bounds, counted as in test_gpu_paged.py: HALF_STEP is what one rounding to the type is off by relative to the value."""
import math

import numpy as np
import pytest
import torch

import paper_2605_06763_amd as L
from test_gpu_paged import D, HALF_STEP, LENS, Cache, freqs, rotated, say

pytestmark = pytest.mark.gpu

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
TYPES = ["bf16", "f32", "fp4"]


def to_codes(x):
    """Rows [..., 128] in 64 bits as codes [..., 128] and scale bytes [..., 4], by the definition: the least power of two 2^e with A <= 7 * 2^e, the nearest
    level, of two as near the one whose place is even."""
    b = x.double().unflatten(-1, (4, 32))
    top = b.abs().amax(dim=-1)
    odd = ~torch.isfinite(b).all(dim=-1)
    e = torch.full_like(top, -120)
    for k in range(-120, 125):
        e = torch.where(top > 7 * 2.0 ** k, torch.full_like(top, k + 1), e)
    e = torch.where(odd, torch.full_like(top, 128), e)
    t = torch.where(odd[..., None], torch.zeros_like(b), b) / torch.pow(torch.tensor(2.0, dtype=torch.float64), torch.where(odd, 0 * e, e))[..., None]
    far = (t.abs().clamp_max(6)[..., None] - LEVELS).abs()
    near = far.amin(dim=-1, keepdim=True)
    code = torch.where(far == near, torch.arange(8) + 8 * (torch.arange(8) % 2), 99).amin(dim=-1) % 8      # the even one of two
    code = code + 8 * torch.signbit(b).long()
    return code.flatten(-2), (e + 127).long()


def values(codes, scales):
    v = LEVELS[codes % 8] * torch.where(codes >= 8, -1.0, 1.0)
    s = torch.where(scales == 255, torch.tensor(math.nan, dtype=torch.float64), torch.pow(torch.tensor(2.0, dtype=torch.float64), scales.double() - 127))
    return (v.unflatten(-1, (4, 32)) * s[..., None]).flatten(-2)


class More(Cache):
    """Cache, of pages in 4 bits too: codes [page][head][token][128] and scales [page][head][token][4] are what the pages hold then, K and V what that
    stands for."""

    def __init__(self, lens, *, dtype="bf16", **more):
        super().__init__(lens, dtype="bf16" if dtype == "fp4" else dtype, **more)
        self.fp4 = dtype == "fp4"
        if not self.fp4:
            return
        L.lvr_paged_destroy(self.h)
        self.kc, self.ks = to_codes(self.K)
        self.vc, self.vs = to_codes(self.V)
        self.decode()
        c = self.cfg
        self.cfg = L.make_paged_config(n_q_heads=self.hq, n_kv_heads=self.hkv, kv_dtype=L.LVR_FP4, page_size=self.page, n_pages=self.n_pages, layout=self.layout,
                                       scale=c.scale, rot_dim=c.rot_dim, rot_axes=c.rot_axes, rot_pairs=c.rot_pairs)
        self.h = L.lvr_paged_create(self.cfg, inv_freq=more.get("inv_freq"), axis=more.get("axis"))

    def decode(self):
        self.K, self.V = values(self.kc, self.ks).to(self.dt), values(self.vc, self.vs).to(self.dt)

    def pack(self, codes, scales):
        order = (lambda x: x) if self.layout == "head" else (lambda x: x.transpose(1, 2))
        codes = order(codes)
        codes = (codes[..., 0::2] + 16 * codes[..., 1::2]).flatten(1)
        return torch.cat([codes, order(scales).flatten(1)], dim=1).to(torch.uint8)

    def unpack(self, pool):
        pool, rows = pool.cpu().long(), self.hkv * self.page
        shape = (self.n_pages, self.hkv, self.page) if self.layout == "head" else (self.n_pages, self.page, self.hkv)
        b = pool[:, :rows * 64].view(*shape, 64)
        codes, scales = torch.stack([b % 16, b // 16], dim=-1).flatten(-2), pool[:, rows * 64:].view(*shape, 4)
        return (codes, scales) if self.layout == "head" else (codes.transpose(1, 2), scales.transpose(1, 2))

    def pools(self):
        return (self.pack(self.kc, self.ks).cuda(), self.pack(self.vc, self.vs).cuda()) if self.fp4 else super().pools()

    def hide(self, which, unseen, value=math.nan):
        """Rows [page][token] of K or V become no numbers."""
        if self.fp4:
            (self.ks if which == "K" else self.vs).transpose(1, 2)[unseen] = 255
            self.decode()
        else:
            (self.K if which == "K" else self.V).transpose(1, 2)[unseen] = value

    def sink_attention(self, q, window, sinks):
        """The definition in 64 bits and how far off the kernel's may be (counted as in Cache.attention); rows of no sequence NaN."""
        out = torch.full((self.T, self.hq, D), math.nan, dtype=torch.float64)
        tol = torch.zeros_like(out)
        G, step = self.hq // self.hkv, HALF_STEP[self.dtype]
        for b, (t, n) in enumerate(self.lens):
            s0 = int(self.start[b])
            K, V, held = self.rows(b, max(n, 0))
            for i in range(t):
                p, j = n - t + i, torch.arange(max(n, 0))
                sees = (j <= p) & held
                if window:
                    sees &= (j > p - window) | (j < sinks)
                for h in range(self.hq):
                    Kh, Vh, qh = K[h // G][sees], V[h // G][sees], q[s0 + i, h].double()
                    x = Kh @ qh * self.scale
                    w = torch.softmax(x, dim=0)
                    o = w @ Vh if len(x) else torch.zeros(D, dtype=torch.float64)
                    size = w @ Vh.abs() + o.abs() if len(x) else 0 * o
                    S = (Kh.abs() @ qh.abs() * self.scale).amax() if len(x) else torch.tensor(0.0)
                    weight = 2 * (136 * 2.0 ** -24 * S + 2.0 ** -21) + (1.02 * step if self.dtype == "bf16" else 0)
                    out[s0 + i, h], tol[s0 + i, h] = o, (weight + (len(x) + 64) * 2.0 ** -24) * size + step * o.abs()
        return out, tol


def check(c, window=0, sinks=0, q=None, note="", plain=False):
    q = c.randn(c.T, c.hq, D) if q is None else q
    say(f"attention {note} lens={c.lens} {'fp4' if c.fp4 else c.dtype} heads={c.hq}/{c.hkv} page={c.page} {c.layout} window={window} sinks={sinks}")
    out = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
    if plain:
        L.lvr_paged_attention(c.h, *c.pools(), q.cuda(), *c.batch(), out, window=window)
    else:
        L.lvr_paged_sink_attention(c.h, *c.pools(), q.cuda(), *c.batch(), out, window, sinks)
    torch.cuda.synchronize()
    out = out.cpu().double()
    ref, tol = c.sink_attention(q, window, sinks) if sinks else c.attention(q, window)
    # Where the values that have weight are zero, as pages in 4 bits may hold them, outputs come from weights that fp32 does not have: each key's is off by up
    # to 2^-126 against the largest one's, and the sum of all is no less than the largest.
    tol = tol + max([n for _, n in c.lens] + [0]) * 2.0 ** -126 * c.V.double().nan_to_num(0, 0, 0).abs().max()
    inside = torch.zeros(c.T, dtype=torch.bool)
    inside[int(c.start[0]):int(c.start[-1])] = True
    assert (out[~inside] == 7).all(), "rows of no sequence were written"
    out, ref, tol = out[inside], ref[inside], tol[inside]
    finite = torch.isfinite(ref)
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    assert torch.equal(out[~finite & ~torch.isnan(ref)], ref[~finite & ~torch.isnan(ref)])
    err = (out - ref).abs()[finite]
    assert (err <= tol[finite]).all(), float((err - tol[finite]).max())
    return out


# ------------------------------------------------------------------------------------------------ attention over pages in 4 bits
@pytest.mark.parametrize("lens", LENS)
def test_attention_in_4_bits_over_lengths(lens):
    with More(LENS[lens], dtype="fp4", seed=103) as c:
        check(c, plain=True)


@pytest.mark.parametrize("hq, hkv", [(1, 1), (3, 1), (4, 4), (8, 1), (12, 2), (20, 1), (40, 8), (71, 1)])
def test_attention_in_4_bits_over_heads(hq, hkv):
    with More([(1, 70), (9, 41), (1, 200)], dtype="fp4", hq=hq, hkv=hkv, seed=104) as c:
        check(c, plain=True)


@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_attention_in_4_bits_over_pages(page, layout):
    with More([(1, 70), (40, 300), (1, 1040)], dtype="fp4", page=page, layout=layout, seed=105) as c:
        check(c, plain=True)


@pytest.mark.parametrize("hq, hkv, lens, window", [(8, 1, [(1, 20000)], 0), (4, 1, [(1, 9000), (1, 12000)], 7000), (8, 1, [(17, 9000)], 0), (2, 1, [(1, 70000)], 0)])
def test_attention_in_4_bits_cut_into_many_runs(hq, hkv, lens, window):
    with More(lens, dtype="fp4", hq=hq, hkv=hkv, page=64, seed=106) as c:
        check(c, window=window, plain=True)
        q = c.randn(c.T, hq, D).cuda()
        a, b = torch.empty_like(q), torch.empty_like(q)
        pools, batch = c.pools(), c.batch()
        for o in (a, b):
            L.lvr_paged_attention(c.h, *pools, q, *batch, o, window=window)
        assert torch.equal(a, b), "the order of the runs shows in the result"


@pytest.mark.parametrize("window", [1, 33, 64, 300, 2 ** 31 - 1])
def test_attention_in_4_bits_with_a_window(window):
    with More([(1, 400), (90, 333), (5, 5), (1, 30)], dtype="fp4", seed=107) as c:
        check(c, window=window, plain=True)


def test_scales_of_every_size():
    """Blocks whose scales differ by many powers of two, from key to key and within a row."""
    with More([(1, 500), (60, 300), (3, 40)], dtype="fp4", seed=108) as c:
        c.ks += torch.randint(-12, 4, c.ks.shape, generator=c.g)
        c.vs += torch.randint(-60, 60, c.vs.shape, generator=c.g)
        c.decode()
        check(c, plain=True)


def test_large_scores_in_4_bits():
    with More([(1, 500), (30, 100)], dtype="fp4", seed=109) as c:
        c.ks += 6
        c.decode()
        check(c, note="large", plain=True)
        c.kc[:, :, ::2] |= 8
        c.decode()
        check(c, q=c.randn(c.T, c.hq, D).abs() * 30, note="large, of one sign", plain=True)


# ------------------------------------------------------------------------------------------------ first keys that stay visible
SINK_LENS = {
    "singles": [(1, 17), (1, 300), (0, 5), (1, 1), (1, 1500), (1, 64), (1, 129)],
    "chunks": [(33, 100), (1, 257), (70, 700), (16, 64), (3, 3)],
    "prompt": [(200, 200)],
    "tokens_before_the_cache": [(5, 3), (1, 0), (2, 200)],
}
MANY_LENS = [(1 + (i * 7) % 3, 3 + (i * 37) % 400) for i in range(70)] + [(0, 12)] * 70 + [(40, 300), (1, 600)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window, sinks", [(1, 1), (16, 4), (50, 64), (33, 65), (64, 130), (128, 1), (7, 1000), (2 ** 31 - 1, 3), (1, 2 ** 31 - 1), (0, 5)])
@pytest.mark.parametrize("lens", SINK_LENS)
def test_first_keys_stay_visible(lens, window, sinks, dtype):
    with More(SINK_LENS[lens], dtype=dtype, hq=4, hkv=2, seed=110) as c:
        check(c, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq, hkv, page, layout", [(1, 1, 16, "head"), (20, 1, 64, "token"), (24, 8, 32, "head"), (71, 1, 128, "token")])
def test_first_keys_over_heads_and_pages(hq, hkv, page, layout, dtype):
    with More([(1, 900), (9, 341), (40, 600)], dtype=dtype, hq=hq, hkv=hkv, page=page, layout=layout, seed=111) as c:
        check(c, 100, 70)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window, sinks", [(0, 0), (1300, 70)])
@pytest.mark.parametrize("lens", [[(1, 1630)] * 5, [(1, 1168)] * 7, [(1, 1363)] * 3, [(1, 1630), (0, 1630), (0, 0)] * 5, [(1, 1630)] * 4 + [(1, 1400)]])
def test_batches_of_one_length(lens, window, sinks, dtype):
    """Lengths at which as many runs as are wanted are no whole number for each sequence."""
    with More(lens, dtype=dtype, hq=8, hkv=8, page=32, seed=134) as c:
        check(c, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[(97, 208), (97, 107)], [(40, 41), (1, 300), (129, 129)]])
def test_first_keys_with_a_kv_head_to_every_query_head(lens, dtype):
    with More(lens, dtype=dtype, hq=8, hkv=8, page=16, layout="token", seed=133) as c:
        check(c, 54, 4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq, lens, window, sinks", [(8, [(1, 30000)], 6000, 3000), (4, [(17, 9000), (1, 9000)], 3000, 100), (2, [(200, 5000)], 1700, 900)])
def test_first_keys_cut_into_runs(hq, lens, window, sinks, dtype):
    with More(lens, dtype=dtype, hq=hq, hkv=1, page=64, seed=112) as c:
        check(c, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
def test_first_keys_of_many_sequences(dtype):
    with More(MANY_LENS, dtype=dtype, hq=4, hkv=2, seed=119) as c:
        check(c, 40, 20)
    with More([(1, 1 + (i * 53) % 700) for i in range(131)], dtype=dtype, hq=4, hkv=2, seed=118) as c:
        check(c, 40, 20)


@pytest.mark.parametrize("tokens", [8, 9, 16, 17])
def test_a_few_tokens_of_one_sequence_in_4_bits(tokens):
    """Up to 64 rows alone go in tiles of 16, more in tiles of 128."""
    with More([(tokens, 3000)], dtype="fp4", hq=8, hkv=2, seed=117) as c:
        check(c, plain=True)
        check(c, 200, 10)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_first_keys_it_is_the_plain_attention(dtype):
    with More(LENS["beside_decodes"], dtype=dtype, seed=113) as c:
        pools, batch, q = c.pools(), c.batch(), c.randn(c.T, c.hq, D).cuda()
        for window, sinks in ((0, 0), (60, 0), (0, 9), (60, 100000)):
            a, b = torch.empty_like(q), torch.empty_like(q)
            L.lvr_paged_sink_attention(c.h, *pools, q, *batch, a, window, sinks)
            L.lvr_paged_attention(c.h, *pools, q, *batch, b, window=window if sinks < 1000 else 0)
            if sinks < 1000:
                assert torch.equal(a, b)
            else:      # (everything is visible; the runs are cut for the window, so the sums' order may differ)
                assert (a - b).abs().max() <= 4 * HALF_STEP[c.dtype] * b.abs().max() + 2.0 ** -18
                check(c, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_between_may_be_gone(dtype):
    """Pages that neither the window nor the first keys reach, taken out of the table: the same bits; what is in them does not matter either."""
    with More([(1, 900), (40, 700), (1, 2000)], dtype=dtype, seed=114) as c:
        q, window, sinks = c.randn(c.T, c.hq, D), 100, 20
        first = check(c, window, sinks, q=q)
        seen = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
        for b, (t, n) in enumerate(c.lens):
            for p in [*range(sinks), *range(n - t - window + 1, n)]:
                seen[c.table[b, p // c.page], p % c.page] = True
        c.hide("K", ~seen)
        c.hide("V", ~seen)
        assert torch.equal(check(c, window, sinks, q=q, note="unseen"), first)
        for b, (t, n) in enumerate(c.lens):
            c.table[b, 2:(n - t - window + 1) // c.page] = -1
        assert torch.equal(check(c, window, sinks, q=q, note="gone"), first)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_some_tokens_see_reaches_those_alone(dtype):
    """A value that is no number among the first keys, in the window of some tokens of a chunk, and missing pages among the first keys."""
    with More([(20, 300), (60, 400), (1, 500)], dtype=dtype, seed=115) as c:
        window, sinks = 50, 24
        last = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
        last[c.table[0, 297 // c.page], 297 % c.page] = True       # the last three tokens of the first sequence
        early = last.clone()
        early[c.table[1, 300 // c.page], 300 % c.page] = True      # the first ten or so of the second
        c.hide("V", early)
        out = check(c, window, sinks, note="seen by some")
        assert torch.isfinite(out[:17]).all() and not torch.isfinite(out[17:20]).any()
        c.table[2, 0] = -1
        check(c, window, sinks, note="no page")
        sink = torch.zeros_like(last)
        sink[c.table[2, 1], 3] = True
        c.hide("K", sink)
        out = check(c, window, sinks, note="a key")
        assert not torch.isfinite(out[-1]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_far_beyond_the_table_with_first_keys(dtype):
    """Windows that lie behind the table: the first keys are all there is."""
    with More([(1, 60), (5, 60)], dtype=dtype, seed=116, extra_width=0) as c:
        q = c.randn(c.T, c.hq, D)
        outs = []
        for n in (5000, 2 ** 30, 2 ** 31 - 1):
            out = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
            start, _, table = c.batch()
            L.lvr_paged_sink_attention(c.h, *c.pools(), q.cuda(), start, torch.full((2,), n, dtype=torch.int32, device="cuda"), table, out, 100, 30)
            outs.append(out.cpu())
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        c.lens = [(1, 5000), (5, 5000)]
        ref, tol = c.sink_attention(q, 100, 30)
        assert ((outs[0].double() - ref).abs() <= tol).all()


# ------------------------------------------------------------------------------------------------ appends
def new_rows(c, scale=1.0):
    fused = (c.randn(c.T, (c.hq + 2 * c.hkv) * D).float() * scale).to(c.dt)
    return fused, fused.cuda()


def split(c, x):
    return (y.unflatten(1, (-1, D)) for y in x.split([c.hq * D, c.hkv * D, c.hkv * D], dim=1))


def positions_of(c, positions):
    pos = torch.zeros(c.T, max(c.cfg.rot_axes, 1), dtype=torch.int64) if positions is None else positions.long()
    if positions is None:
        for b, (t, n) in enumerate(c.lens):
            s0 = int(c.start[b])
            pos[s0:s0 + t] = torch.arange(n - t, n)[:, None]
    return pos


def normed(x, weight, eps):
    x = x.double()
    y = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)
    return y if weight is None else y * weight.double()


def check_append(c, inv_freq=None, axis=None, positions=None, norm=False, weights=(None, None), eps=1e-6, with_q=True, rows=None, note=""):
    rot, pairs = c.cfg.rot_dim, c.cfg.rot_pairs
    say(f"append {note} lens={c.lens} {'fp4' if c.fp4 else c.dtype} heads={c.hq}/{c.hkv} page={c.page} {c.layout} rot={rot} pairs={pairs} norm={norm} q={with_q}")
    fused, dev = rows or new_rows(c)
    (q, k, v), (dq, dk, dv) = split(c, fused), split(c, dev)
    kp, vp = c.pools()
    before = [c.unpack(p) for p in (kp, vp)] if c.fp4 else None
    qo = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
    more = dict(q=dq if with_q else None, q_out=qo if with_q else None, positions=None if positions is None else positions.cuda())
    if norm:
        L.lvr_paged_norm_append(c.h, kp, vp, dk, dv, *c.batch(), q_weight=None if weights[0] is None else weights[0].cuda(),
                                k_weight=None if weights[1] is None else weights[1].cuda(), eps=eps, **more)
    else:
        L.lvr_paged_append(c.h, kp, vp, dk, dv, *c.batch(), **more)
    torch.cuda.synchronize()
    eps = float(np.float32(eps))
    q, k = (normed(q, weights[0], eps), normed(k, weights[1], eps)) if norm else (q, k)
    pos = positions_of(c, positions)
    axis = [0] * (rot // 2) if axis is None else axis
    kr, ks = rotated(k, pos, inv_freq, axis, rot, pairs) if rot else (k.double(), k.double().abs())
    qr, qs = rotated(q, pos, inv_freq, axis, rot, pairs) if rot else (q.double(), q.double().abs())
    # a rotation as in test_gpu_paged.py; a norm before it: the rounding of 1 / sqrt, and two products.  bf16 sums 16 squares of a lane in fp32, eight steps of at
    # most 2^-23 of the sum each, of which the root halves the error: 8 * 2^-24; fp32 sums in 64 bits.
    of_norm = (0 if not norm else 4 if c.dtype == "f32" else 12) * 2.0 ** -24
    rel, off = HALF_STEP[c.dtype], (12 if rot else 0) * 2.0 ** -24 + of_norm

    def bound(y, size):
        t = rel * y.abs() + off * size
        t[..., rot:] = (rel * y.abs() + of_norm * y.abs())[..., rot:] if norm else 0
        return t

    inside = torch.zeros(c.T, dtype=torch.bool)
    inside[int(c.start[0]):int(c.start[-1])] = with_q
    qo = qo.cpu().double()
    assert (qo[~inside] == 7).all()
    finite = torch.isfinite(qr)
    assert torch.equal(torch.isnan(qo[inside]), torch.isnan(qr[inside]))
    assert ((qo - qr).abs() <= bound(qr, qs))[inside][finite[inside]].all()
    places = {}
    for b, (t, n) in enumerate(c.lens):
        for i in range(t):
            p = n - t + i
            id = int(c.table[b, p // c.page]) if 0 <= p < c.width * c.page else -1
            if 0 <= id < c.n_pages:
                places[(id, p % c.page)] = int(c.start[b]) + i
    ids, at, s = (torch.tensor(x) for x in zip(*((i, a, t) for (i, a), t in places.items()))) if places else (torch.zeros(0, dtype=torch.long),) * 3
    if c.fp4:
        for (codes, scales), pool, x in zip(before, (kp, vp), (kr, v.double())):
            got_codes, got_scales = c.unpack(pool)
            wc, ws = to_codes(x)
            codes[ids, :, at], scales[ids, :, at] = wc[s], ws[s]
            assert torch.equal(got_scales, scales)
            sure = scales.repeat_interleave(32, dim=-1) != 255
            zero = (codes % 8 == 0) & (got_codes % 8 == 0)      # a zero's sign says nothing
            assert torch.equal(got_codes[sure & ~zero], codes[sure & ~zero])
        return kp, vp
    K, V = c.from_pool(kp).double(), c.from_pool(vp).double()
    want_k, want_v, tol = c.K.double().clone(), c.V.double().clone(), torch.zeros(c.K.shape, dtype=torch.float64)
    want_k[ids, :, at], want_v[ids, :, at], tol[ids, :, at] = kr[s], v[s].double(), bound(kr, ks)[s]
    finite = torch.isfinite(want_k)
    assert torch.equal(torch.isnan(K), torch.isnan(want_k)) and torch.equal(V.view(torch.int64), want_v.view(torch.int64))
    assert ((K - want_k).abs() <= tol)[finite].all(), float(((K - want_k).abs() - tol)[finite].max())
    return kp, vp


def weights_of(c):
    return [(1 + 0.3 * torch.randn(D, generator=c.g)).to(c.dt) for _ in range(2)]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", ["one_key", "single_tokens", "whole_prompts", "chunks", "tokens_before_the_cache"])
def test_appends_over_lengths(lens, dtype, norm):
    f = freqs(128)
    with More(LENS[lens], dtype=dtype, rot_dim=128, inv_freq=f, seed=120, behind=3, gap=2) as c:
        check_append(c, f, norm=norm, weights=weights_of(c))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pairs", [L.LVR_ROT_HALVES, L.LVR_ROT_NEIGHBOURS])
@pytest.mark.parametrize("rot", [0, 16, 32, 64, 96, 112, 128])
def test_appends_over_rotations(rot, pairs, dtype):
    f = freqs(rot) if rot else None
    for norm in (True, False):
        with More([(5, 40), (1, 100), (30, 30)], dtype=dtype, rot_dim=rot, pairs=pairs, inv_freq=f, seed=121) as c:
            check_append(c, f, norm=norm, weights=weights_of(c))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq, hkv, axes", [(1, 1, 1), (3, 1, 2), (4, 4, 3), (12, 2, 4), (40, 8, 3), (34, 17, 1), (9, 9, 2)])
def test_appends_over_axes_and_heads(hq, hkv, axes, dtype):
    f, axis = freqs(96), [(i * 7) % axes for i in range(48)]
    with More([(6, 90), (1, 33)], dtype=dtype, hq=hq, hkv=hkv, rot_dim=96, rot_axes=axes, inv_freq=f, axis=axis, layout="token", page=32, seed=122) as c:
        pos = torch.randint(-5000, 5000, (c.T, axes), generator=c.g, dtype=torch.int32)
        check_append(c, f, axis, positions=pos, norm=True, weights=weights_of(c))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq, hkv, lens", [(32, 8, [(300, 300), (80, 200)]), (8, 2, [(1500, 1600)]), (5, 5, [(1200, 1200), (1, 9)])])
def test_appends_of_many_rows(hq, hkv, lens, dtype):
    """Enough rows that a wave takes several of a token."""
    f = freqs(128)
    with More(lens, dtype=dtype, hq=hq, hkv=hkv, rot_dim=128, inv_freq=f, seed=123) as c:
        assert c.T * (hq + 2 * hkv) >= 16384
        check_append(c, f, norm=True, weights=weights_of(c))
        check_append(c, f, norm=False)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [62, 63, 64, 65, 130])
def test_appends_of_as_many_sequences_as_a_wave_has_lanes(n, dtype, norm):
    """On both sides of 63 a token's sequence is found in different ways; among them sequences that bring nothing, the first and the last too."""
    f = freqs(32)
    lens = [((i * 5) % 4, 4 + (i * 37) % 60) for i in range(n - 1)] + [(0, 9)]
    with More(lens, dtype=dtype, hq=2, hkv=2, rot_dim=32, inv_freq=f, seed=132, behind=2, gap=1) as c:
        check_append(c, f, norm=norm, weights=weights_of(c))


@pytest.mark.parametrize("dtype", TYPES)
def test_norms_without_weights_or_queries(dtype):
    f = freqs(64)
    with More([(7, 30), (1, 9)], dtype=dtype, rot_dim=64, inv_freq=f, seed=124) as c:
        w = weights_of(c)
        check_append(c, f, norm=True)
        check_append(c, f, norm=True, weights=(w[0], None), eps=0.5)
        check_append(c, f, norm=True, weights=(None, w[1]), with_q=False)
        check_append(c, f, norm=True, weights=w, eps=0.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_norms_of_rows_of_any_size(dtype):
    """Squares beyond the fp32 range and below it, rows of zeros, and rows with infinities and NaN in them."""
    f = freqs(128)
    with More([(60, 60)], dtype=dtype, rot_dim=128, inv_freq=f, seed=125) as c:
        fused = new_rows(c)[0].float().view(c.T, -1, D)
        fused *= 10.0 ** torch.linspace(-36, 37, c.T)[:, None, None]
        fused[7] = 0
        rows = fused.flatten(1).to(c.dt)
        check_append(c, f, norm=True, weights=weights_of(c), rows=(rows, rows.cuda()), note="sizes")
        check_append(c, f, norm=True, weights=weights_of(c), rows=(rows, rows.cuda()), eps=0.0, note="sizes, without eps")
        for bad in (math.inf, -math.inf, math.nan):
            rows = fused.clone()
            rows[9:40, ::2, 5] = bad
            rows = rows.flatten(1).to(c.dt)
            # of a row with an infinity the formula leaves zeros and, from the infinity, NaN: which a rotation hands to its partner
            check_append(c, f, norm=True, weights=weights_of(c), rows=(rows, rows.cuda()), note=str(bad))


@pytest.mark.parametrize("pairs", [L.LVR_ROT_HALVES, L.LVR_ROT_NEIGHBOURS])
def test_codes_beside_every_border(pairs):
    """Values on the borders between codes and next to them, blocks whose largest value is 7 scales or a little more, zeros, the ends of the range, infinities
    and NaN: V as it is, K without a rotation."""
    f = freqs(32)
    with More([(200, 210)], dtype="fp4", rot_dim=32, pairs=pairs, inv_freq=f, seed=126) as c:
        steps = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.5, 7.0])
        near = torch.cat([steps, steps * (1 + 2.0 ** -7), steps * (1 - 2.0 ** -8)])
        fused = near[torch.randint(0, len(near), (c.T, (c.hq + 2 * c.hkv), D), generator=c.g)]
        fused *= torch.where(torch.rand(fused.shape, generator=c.g) < 0.5, -1.0, 1.0)
        fused[::2, :, ::32] = 7.0
        fused *= 2.0 ** torch.randint(-124, 125, (c.T, 1, 1), generator=c.g).float()
        fused[3] = 0
        fused[4, :, 40:] = 0
        fused[5], fused[6] = 3.3e38, -1e-39
        fused[11, :, 70], fused[12, :, 3], fused[13, :, 127] = math.inf, math.nan, -math.inf
        rows = fused.flatten(1).to(c.dt)
        zeros = torch.zeros(c.T, 1, dtype=torch.int32)      # turned by nothing: K to the bit
        check_append(c, f, positions=zeros, rows=(rows, rows.cuda()), with_q=False)


def test_far_positions_in_4_bits():
    f = [1.0, 0.75, 9.5, 1e-3, 1e6, -2.0, 0.0, 1e-30]
    with More([(40, 90)], dtype="fp4", rot_dim=16, inv_freq=f, seed=127) as c:
        pos = torch.randint(-2000000, 2000000, (c.T, 1), generator=c.g, dtype=torch.int32)
        check_append(c, f, positions=pos, norm=True)


def test_appends_in_4_bits_to_missing_pages_are_dropped():
    f = freqs(128)
    with More([(40, 70), (20, 20), (4, 90)], dtype="fp4", rot_dim=128, inv_freq=f, seed=128) as c:
        c.table[0, 3], c.table[1, 0], c.table[2, 5] = -1, c.n_pages, -2 ** 31
        check_append(c, f, norm=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_normed_queries_in_place(dtype):
    f = freqs(128)
    with More([(7, 30)], dtype=dtype, rot_dim=128, inv_freq=f, seed=129) as c:
        k, q = c.randn(c.T, c.hkv, D).cuda(), c.randn(c.T, c.hq, D).cuda()
        out, again = torch.empty_like(q), q.clone()
        L.lvr_paged_norm_append(c.h, *c.pools(), k, k, *c.batch(), q=q, q_out=out)
        L.lvr_paged_norm_append(c.h, *c.pools(), k, k, *c.batch(), q=again, q_out=again)
        assert torch.equal(out, again) and not torch.equal(out, q)


# ------------------------------------------------------------------------------------------------ gather
@pytest.mark.parametrize("page, layout", [(16, "head"), (16, "token"), (64, "head"), (256, "token")])
def test_gather_in_4_bits(page, layout):
    for n in (1, 15, 16, 300, 333):
        with More([(0, 300), (0, 0), (0, 17), (0, 64), (0, 90)], dtype="fp4", page=page, layout=layout, hkv=3, hq=3, seed=130) as c:
            c.table[4, 0] = -1
            c.vs += torch.randint(-100, 100, c.vs.shape, generator=c.g)
            c.ks[2, 1, 3, 2] = 255
            c.decode()
            say(f"gather n={n} fp4 page={page} {layout}")
            K, V = (torch.full((5, c.hkv, n, D), 7.0, dtype=c.dt, device="cuda") for _ in range(2))
            _, length, table = c.batch()
            L.lvr_paged_gather(c.h, *c.pools(), length, table, K, V)
            for b, (_, held) in enumerate(c.lens):
                Kr, Vr, has = c.rows(b, min(held, n))
                for got, ref in ((K, Kr), (V, Vr)):
                    want = torch.full((c.hkv, n, D), 7.0, dtype=torch.float64)
                    want[:, :min(held, n)][:, has] = ref[:, has]
                    assert torch.equal(got[b].cpu().double().nan_to_num(99), want.nan_to_num(99))


def test_gather_in_4_bits_of_more_than_the_caches_hold():
    """Past 192 MiB of rows, which are stored around the caches then: the same as in pieces."""
    n, heads, page, pages = 100003, 8, 64, 1563
    g = torch.Generator(device="cuda").manual_seed(131)
    h = L.lvr_paged_create(L.make_paged_config(n_q_heads=heads, n_kv_heads=heads, kv_dtype=L.LVR_FP4, page_size=page, n_pages=pages))
    try:
        assert n * heads * 256 >= 192 << 20
        kp, vp = (torch.randint(0, 200, (pages, heads * page * 68), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None].contiguous()
        K, V = (torch.full((1, heads, n, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        L.lvr_paged_gather(h, kp, vp, torch.tensor([n], dtype=torch.int32, device="cuda"), table, K, V)
        for p0 in range(0, pages, 400):
            part = table[:, p0:p0 + 400].contiguous()
            m = min(n - p0 * page, 400 * page)
            k, v = (torch.empty((1, heads, m, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            L.lvr_paged_gather(h, kp, vp, torch.tensor([m], dtype=torch.int32, device="cuda"), part, k, v)
            assert torch.equal(K[:, :, p0 * page:p0 * page + m].view(torch.int16), k.view(torch.int16))
            assert torch.equal(V[:, :, p0 * page:p0 * page + m].view(torch.int16), v.view(torch.int16))
    finally:
        L.lvr_paged_destroy(h)


# ------------------------------------------------------------------------------------------------ refusals
def test_more_calls_refuse_what_they_cannot_take():
    for dtype in ("bf16", "fp4"):
        with More([(2, 20), (1, 40)], dtype=dtype, rot_dim=128, inv_freq=freqs(128), seed=140) as c:
            kp, vp = c.pools()
            start, length, table = c.batch()
            q, k = c.randn(c.T, c.hq, D).cuda(), c.randn(c.T, c.hkv, D).cuda()
            out, w = torch.empty_like(q), torch.ones(D, dtype=c.dt, device="cuda")
            attend = lambda **o: L.lvr_paged_sink_attention(**dict(dict(h=c.h, k_pages=kp, v_pages=vp, q=q, seq_start=start, seq_len=length, table=table, out=out, window=9, sinks=2), **o))   # noqa: E731
            append = lambda **o: L.lvr_paged_norm_append(**dict(dict(h=c.h, k_pages=kp, v_pages=vp, k_new=k, v_new=k, seq_start=start, seq_len=length, table=table, q=q, q_out=out, q_weight=w, k_weight=w), **o))   # noqa: E731
            for call in (attend, append):
                for bad in (dict(k_pages=kp[:-1]), dict(v_pages=vp.float()), dict(v_pages=vp.cpu()), dict(seq_len=length.long()), dict(table=table[0]), dict(q=q.float()),
                            dict(q=q.transpose(0, 1)), dict(seq_start=start[:-1]), dict(k_pages=kp[..., ::2])):
                    with pytest.raises(ValueError):
                        call(**bad)
            for bad in (dict(window=-1), dict(sinks=-1), dict(sinks=1 << 31), dict(window=1 << 40), dict(out=out[:1]), dict(out=out.float())):
                with pytest.raises(ValueError):
                    attend(**bad)
            for bad in (dict(q_weight=w.float()), dict(k_weight=w[:64]), dict(k_weight=w.cpu()), dict(q_weight=torch.ones(2, D, dtype=c.dt, device="cuda")), dict(q_out=None),
                        dict(k_weight=torch.ones(2 * D, dtype=c.dt, device="cuda")[::2])):
                with pytest.raises(ValueError):
                    append(**bad)
            for eps in (-1e-6, math.nan, math.inf):
                with pytest.raises(L.LouverError) as e:
                    append(eps=eps)
                assert e.value.code == L.LVR_E_INVALID
            for x in (torch.ones(D + 8, dtype=c.dt, device="cuda")[1:D + 1],):      # not on 16 bytes
                with pytest.raises(L.LouverError):
                    append(q_weight=x)
            attend()
            append()
            torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
def test_marshalled_arguments_and_plain_ones_give_the_same(monkeypatch, dtype):
    f = freqs(64)
    with More([(5, 40), (1, 20)], dtype=dtype, rot_dim=64, inv_freq=f, seed=142) as c:
        results, w = [], [x.cuda() for x in weights_of(c)]
        for way in ("tensors", "arguments", "general"):
            A = L.tensor_arg if way == "arguments" else (lambda t: t)
            if way == "general":
                monkeypatch.setattr(L.binding, "_call", None)
            kp, vp = c.pools()
            g = torch.Generator().manual_seed(1)
            q, k, v = (torch.randn(c.T, n, D, generator=g).to(c.dt).cuda() for n in (c.hq, c.hkv, c.hkv))
            start, length, table = (A(x) for x in c.batch())
            qo, out = torch.zeros_like(q), torch.zeros_like(q)
            K, V = (torch.zeros(2, c.hkv, 40, D, dtype=c.dt, device="cuda") for _ in range(2))
            L.lvr_paged_norm_append(c.h, A(kp), A(vp), A(k), A(v), start, length, table, q=A(q), q_out=A(qo), q_weight=A(w[0]), k_weight=A(w[1]), eps=1e-5)
            L.lvr_paged_sink_attention(c.h, A(kp), A(vp), A(qo), start, length, table, A(out), 15, 4)
            L.lvr_paged_gather(c.h, A(kp), A(vp), length, table, A(K), A(V))
            results.append([x.clone() for x in (kp, vp, qo, out, K, V)])
        for other in results[1:]:
            assert all(torch.equal(x, y) for x, y in zip(results[0], other))


def test_empty_batches_in_4_bits():
    with More([], dtype="fp4", seed=141) as c:
        z = lambda *s: torch.zeros(s, dtype=c.dt, device="cuda")   # noqa: E731
        L.lvr_paged_sink_attention(c.h, *c.pools(), z(0, c.hq, D), *c.batch(), z(0, c.hq, D), 5, 5)
        L.lvr_paged_norm_append(c.h, *c.pools(), z(0, c.hkv, D), z(0, c.hkv, D), *c.batch())
        L.lvr_paged_gather(c.h, *c.pools(), *c.batch()[1:], z(0, c.hkv, 4, D), z(0, c.hkv, 4, D))
        torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ as they are used
def test_pools_in_4_bits_of_more_than_4_gib():
    """Pages past 2^32 bytes, with a stride wider than a page, hold the same rows as a small pool and give the same bits."""
    lens, hq, hkv, page = [(3, 200), (1, 77), (40, 90)], 16, 8, 64
    size = hkv * page * 68
    stride, big = size + 256, 140000
    with More(lens, dtype="fp4", hq=hq, hkv=hkv, page=page, rot_dim=128, inv_freq=freqs(128), seed=150) as c:
        used = [int(p) for p in c.table.flatten() if p >= 0]
        far = {p: big - 1 - 37 * i for i, p in enumerate(used)}
        assert (big - 1000) * stride > 1 << 32
        h = L.lvr_paged_create(L.make_paged_config(n_q_heads=hq, n_kv_heads=hkv, kv_dtype=L.LVR_FP4, page_size=page, n_pages=big, rot_dim=128,
                                                   page_strides=(stride, 64 * page, 64)), inv_freq=freqs(128))
        try:
            K, V = (torch.empty(big, stride, dtype=torch.uint8, device="cuda") for _ in range(2))
            kp, vp = c.pools()
            for p, f in far.items():
                K[f, :size], V[f, :size] = kp[p], vp[p]
                K[f, size:], V[f, size:] = 77, 77
            table = torch.tensor([[far.get(int(p), -1) for p in row] for row in c.table], dtype=torch.int32, device="cuda")
            start, length, small_table = c.batch()
            k, q = c.randn(c.T, hkv, D).cuda(), c.randn(c.T, hq, D).cuda()
            got = []
            for handle, pools, tab in ((c.h, (kp, vp), small_table), (h, (K[:, :size], V[:, :size]), table)):
                qo, out = torch.empty_like(q), torch.empty_like(q)
                rows = [torch.zeros(3, hkv, 200, D, dtype=c.dt, device="cuda") for _ in range(2)]
                L.lvr_paged_norm_append(handle, *pools, k, k, start, length, tab, q=q, q_out=qo)
                L.lvr_paged_sink_attention(handle, *pools, qo, start, length, tab, out, 60, 5)
                L.lvr_paged_gather(handle, *pools, length, tab, *rows)
                got.append([qo, out, *rows])
            assert all(torch.equal(x, y) for x, y in zip(*got))
            for p, f in far.items():
                assert torch.equal(K[f, :size], kp[p]) and torch.equal(V[f, :size], vp[p]) and (K[f, size:] == 77).all() and (V[f, size:] == 77).all()
        finally:
            L.lvr_paged_destroy(h)


@pytest.mark.parametrize("dtype", TYPES)
def test_normed_prompt_with_first_keys_to_the_index(dtype):
    """A prompt comes in pieces of odd sizes through the normed append and the attention with a window and first keys; its pages become rows, the rows an
    index; the next token is decoded from the index and from the pages: the same keys, the same attention."""
    n, hq, hkv, f, window, sinks = 700, 8, 2, freqs(128), 150, 20
    with More([(n, n + 1)], dtype=dtype, hq=hq, hkv=hkv, rot_dim=128, inv_freq=f, seed=160) as c:
        fused = c.randn(n + 1, (hq + 2 * hkv) * D)
        q, k, v = (x.unflatten(1, (-1, D)) for x in fused.split([hq * D, hkv * D, hkv * D], dim=1))
        dq, dk, dv = (x.unflatten(1, (-1, D)) for x in fused.cuda().split([hq * D, hkv * D, hkv * D], dim=1))
        w = weights_of(c)
        dw = [x.cuda() for x in w]
        kp, vp = c.pools()
        table = c.table.cuda()

        def step(at, m, window, sinks):
            start, length = torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.tensor([at + m], dtype=torch.int32, device="cuda")
            qo, out = (torch.empty(m, hq, D, dtype=c.dt, device="cuda") for _ in range(2))
            L.lvr_paged_norm_append(c.h, kp, vp, dk[at:at + m], dv[at:at + m], start, length, table, q=dq[at:at + m], q_out=qo, q_weight=dw[0], k_weight=dw[1])
            L.lvr_paged_sink_attention(c.h, kp, vp, qo, start, length, table, out, window, sinks)
            return qo, out

        outs, at = [], 0
        for m in (1, 130, 17, 300, 252):
            outs.append(step(at, m, window, sinks))
            at += m
        qo, out = (torch.cat(x).cpu().double() for x in zip(*outs))
        rows = [torch.zeros(1, hkv, n, D, dtype=c.dt, device="cuda") for _ in range(2)]
        L.lvr_paged_gather(c.h, kp, vp, torch.tensor([n], dtype=torch.int32, device="cuda"), table, *rows)
        # the rows are the normed and rotated ones, the attention is that over the rows
        pos, eps = torch.arange(n)[:, None], float(np.float32(1e-6))
        kr = rotated(normed(k[:n], w[1], eps), pos, f, [0] * 64, 128, L.LVR_ROT_HALVES)[0].transpose(0, 1)
        K, V = (x[0].cpu().double() for x in rows)
        if c.fp4:
            assert torch.equal(K, values(*to_codes(kr))) and torch.equal(V, values(*to_codes(v[:n].transpose(0, 1))))
        else:
            assert ((K - kr).abs() <= HALF_STEP[c.dtype] * kr.abs() + 16 * 2.0 ** -24 * 8).all() and torch.equal(V, v[:n].transpose(0, 1).double())
        j = torch.arange(n)
        sees = (j <= pos) & ((j > pos - window) | (j < sinks))
        step_of = HALF_STEP[c.dtype]
        for h in range(hq):
            s = qo[:, h] @ K[h // 4].T / math.sqrt(D)
            ref = torch.softmax(torch.where(sees, s, torch.tensor(-math.inf, dtype=torch.float64)), dim=1)
            S = (qo[:, h].abs() @ K[h // 4].abs().T / math.sqrt(D)).max()
            size = ref @ V[h // 4].abs()
            weight = 2 * (136 * 2.0 ** -24 * S + 2.0 ** -21) + (1.02 * step_of if c.dtype == "bf16" else 0)
            ref = ref @ V[h // 4]
            assert ((out[:, h] - ref).abs() <= (weight + 250 * 2.0 ** -24) * (size + ref.abs()) + step_of * ref.abs()).all()
        cfg = L.make_config(batch=1, n_q_heads=hq, n_kv_heads=hkv, kv_dtype=L.LVR_F32 if dtype == "f32" else L.LVR_BF16, capacity=n + 1,
                            group_size=4 if dtype == "f32" else 1)
        ix = L.lvr_create(cfg)
        try:
            L.lvr_build(ix, *rows)
            qo, paged = step(n, 1, 0, 0)
            new = [torch.zeros(1, hkv, n + 1, D, dtype=c.dt, device="cuda") for _ in range(2)]
            L.lvr_paged_gather(c.h, kp, vp, torch.tensor([n + 1], dtype=torch.int32, device="cuda"), table, *new)
            tau = torch.full((1, hq), -math.inf, device="cuda")
            idx = torch.zeros(1, hq, n + 1, dtype=torch.int32, device="cuda")
            cnt, dense = torch.zeros(1, hq, dtype=torch.int32, device="cuda"), torch.empty(1, hq, D, device="cuda")
            L.lvr_append_decode_step(ix, new[0][:, :, n:].contiguous(), new[1][:, :, n:].contiguous(), qo.float(), tau, dense, idx, cnt)
            torch.cuda.synchronize()
            assert (cnt == n + 1).all()
            got, want = paged.double().cpu(), dense.double().cpu()
            # the index keeps its weights in fp32; the pages' attention rounds them to bf16, and its output
            err = (got - want).abs().amax() / want.abs().amax()
            assert err <= (2e-5 if dtype == "f32" else 4 * step_of), float(err)
        finally:
            L.lvr_destroy(ix)


@pytest.mark.parametrize("dtype", TYPES)
def test_two_handles_on_streams_of_their_own(dtype):
    f = freqs(128)
    a = More([(130, 400), (1, 900)], dtype=dtype, rot_dim=128, inv_freq=f, seed=162)
    b = More([(1, 3000), (3, 50)], dtype=dtype, rot_dim=128, inv_freq=f, seed=163)
    with a, b:
        args = []
        for c in (a, b):
            k, q = c.randn(c.T, c.hkv, D).cuda(), c.randn(c.T, c.hq, D).cuda()
            args.append((c, c.pools(), k, q, c.batch(), torch.empty_like(q), torch.empty_like(q), weights_of(c)[0].cuda()))

        def work(x, stream):
            c, pools, k, q, batch, qo, out, w = x
            L.lvr_paged_norm_append(c.h, *pools, k, k, *batch, q=q, q_out=qo, q_weight=w, k_weight=w, stream=stream)
            L.lvr_paged_sink_attention(c.h, *pools, qo, *batch, out, 80, 12, stream=stream)
        for x in args:
            work(x, None)
        torch.cuda.synchronize()
        want = [x[6].clone() for x in args]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for _ in range(5):
            for x in args:
                x[6].fill_(7)
            torch.cuda.synchronize()
            for x, st in zip(args, streams):
                work(x, st)
            torch.cuda.synchronize()
            assert all(torch.equal(x[6], w) for x, w in zip(args, want))


@pytest.mark.parametrize("dtype", TYPES)
def test_captured_steps_follow_the_arrays(dtype):
    """A decode step and a step with a prompt in it, recorded once each on one handle and replayed in turn while lengths and inputs change: every replay
    gives the eager call's bits.  Rows behind the last sequence (a padded batch) stay as they were."""
    f = freqs(128)
    with More([(1, 900), (1, 40), (1, 2000), (0, 0)], dtype=dtype, rot_dim=128, inv_freq=f, seed=164) as c:
        kp, vp = c.pools()
        table, w = c.table.cuda(), [x.cuda() for x in weights_of(c)]
        steps = []
        for T in (4, 160):
            s = dict(start=torch.zeros(5, dtype=torch.int32, device="cuda"), length=torch.zeros(4, dtype=torch.int32, device="cuda"))
            for name, heads in (("k", c.hkv), ("q", c.hq), ("qo", c.hq), ("out", c.hq)):
                s[name] = torch.zeros(T, heads, D, dtype=c.dt, device="cuda")
            s["K"], s["V"] = (torch.zeros(4, c.hkv, 500, D, dtype=c.dt, device="cuda") for _ in range(2))
            steps.append(s)

        def work(s):
            L.lvr_paged_norm_append(c.h, kp, vp, s["k"], s["k"], s["start"], s["length"], table, q=s["q"], q_out=s["qo"], q_weight=w[0], k_weight=w[1])
            L.lvr_paged_sink_attention(c.h, kp, vp, s["qo"], s["start"], s["length"], table, s["out"], 200, 30)
            L.lvr_paged_gather(c.h, kp, vp, s["length"], table, s["K"], s["V"])

        graphs = []
        for s in steps:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                work(s)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                work(s)
            graphs.append(g)
        for turn, lens in enumerate([([1, 1, 1, 0], [900, 40, 2000, 0]), ([1, 0, 1, 0], [700, 0, 5, 0]), ([90, 1, 1, 0], [880, 33, 1999, 0]), ([1, 1, 1, 0], [64, 16, 17, 0])]):
            for s, g in zip(steps, graphs):
                if sum(lens[0]) > s["q"].shape[0]:
                    continue
                starts = np.concatenate([[0], np.cumsum(lens[0])])
                s["start"].copy_(torch.tensor(starts, dtype=torch.int32))
                s["length"].copy_(torch.tensor(lens[1], dtype=torch.int32))
                for name in ("k", "q"):
                    s[name].copy_(c.randn(*s[name].shape))
                results = []
                for replay in (False, True, True):
                    for name in ("out", "qo", "K", "V"):
                        s[name].fill_(7)
                    torch.cuda.synchronize()
                    g.replay() if replay else work(s)
                    torch.cuda.synchronize()
                    results.append([s[name].clone() for name in ("out", "qo", "K", "V")] + [kp.clone(), vp.clone()])
                for other in results[1:]:
                    assert all(torch.equal(x, y) for x, y in zip(results[0], other)), turn
                assert (results[0][0][int(starts[-1]):] == 7).all() and (results[0][1][int(starts[-1]):] == 7).all()
                assert torch.isfinite(results[0][0].float()).all()


def test_a_batch_of_many_pieces_in_4_bits():
    """4096 sequences of nine tiles each: more pieces than a launch has workgroups in one of its dimensions.  The same bits as from two halves."""
    seqs, t, hq = 4096, 9, 16
    h = L.lvr_paged_create(L.make_paged_config(n_q_heads=hq, n_kv_heads=1, kv_dtype=L.LVR_FP4, page_size=16, n_pages=seqs))
    try:
        g = torch.Generator(device="cuda").manual_seed(5)
        K, V = (torch.randint(0, 256, (seqs, 16 * 68), generator=g, device="cuda", dtype=torch.uint8) for _ in range(2))
        for p in (K, V):
            p[:, 16 * 64:] = 124 + p[:, 16 * 64:] % 4
        q = torch.randn(seqs * t, hq, D, generator=g, device="cuda").to(torch.bfloat16)
        start = torch.arange(0, seqs * t + 1, t, dtype=torch.int32, device="cuda")
        length = (9 + torch.arange(seqs, device="cuda") % 8).to(torch.int32)
        table = torch.randperm(seqs, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
        whole, halves = torch.empty_like(q), torch.empty_like(q)
        L.lvr_paged_sink_attention(h, K, V, q, start, length, table, whole, 3, 2)
        for a, b in ((0, seqs // 2), (seqs // 2, seqs)):
            L.lvr_paged_sink_attention(h, K, V, q[a * t:b * t], start[a:b + 1] - a * t, length[a:b], table[a:b], halves[a * t:b * t], 3, 2)
        assert torch.equal(whole, halves) and torch.isfinite(whole.float()).all()
    finally:
        L.lvr_paged_destroy(h)
