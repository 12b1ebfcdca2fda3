"""The paged cache on the GPU: append with rotation, attention of new tokens, pages to rows, against plain implementations in
64 bits on the host.

Tolerances are bounds: HALF_STEP is what one rounding to the type is off by relative to the value; what else enters is counted
where it is used."""
import math

import numpy as np
import pytest
import torch

import paper_2605_06763_amd as L

pytestmark = pytest.mark.gpu

D = 128
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def say(*a):
    print(*a, flush=True)


class Cache:
    """Pools with scattered pages and the tables of a batch.  lens: (new tokens, keys held) of every sequence."""

    def __init__(self, lens, *, dtype="bf16", hq=8, hkv=2, page=16, layout="head", scale=0.0, rot_dim=0, rot_axes=1, pairs=L.LVR_ROT_HALVES,
                 inv_freq=None, axis=None, seed=0, spare=2, extra_width=1, behind=0, gap=0):
        self.g = torch.Generator().manual_seed(seed + 1)
        self.lens, self.dtype, self.hq, self.hkv, self.page, self.layout = lens, dtype, hq, hkv, page, layout
        self.dt, self.scale = DTYPES[dtype], scale if scale > 0 else 1 / math.sqrt(D)
        used = [max(0, -(-n // page)) for _, n in lens]
        self.width = max(used + [0]) + extra_width
        self.n_pages = sum(used) + spare
        order = torch.randperm(self.n_pages, generator=self.g).tolist()
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        for b, u in enumerate(used):
            for p in range(u):
                self.table[b, p] = order.pop()
        starts = [gap]
        for t, _ in lens:
            starts.append(starts[-1] + t)
        self.T = starts[-1] + behind
        self.start = torch.tensor(starts, dtype=torch.int32)
        self.len = torch.tensor([n for _, n in lens], dtype=torch.int32)
        self.K, self.V = (self.randn(self.n_pages, hkv, page, D) for _ in range(2))     # [page][head][token][D], rounded to the type
        self.cfg = L.make_paged_config(n_q_heads=hq, n_kv_heads=hkv, kv_dtype=L.LVR_BF16 if dtype == "bf16" else L.LVR_F32, page_size=page,
                                       n_pages=self.n_pages, layout=layout, scale=scale, rot_dim=rot_dim, rot_axes=rot_axes, rot_pairs=pairs)
        self.h = L.lvr_paged_create(self.cfg, inv_freq=inv_freq, axis=axis)

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g).to(self.dt)

    def pools(self):
        to = (lambda p: p.cuda()) if self.layout == "head" else (lambda p: p.transpose(1, 2).contiguous().cuda())
        return to(self.K), to(self.V)

    def from_pool(self, p):
        return p.cpu() if self.layout == "head" else p.cpu().transpose(1, 2).contiguous()

    def batch(self):
        return self.start.cuda(), self.len.cuda(), self.table.cuda()

    def close(self):
        L.lvr_paged_destroy(self.h)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def rows(self, b, n):
        """K, V [hkv][n][D] and which of the n positions have a page."""
        K, V = torch.zeros(self.hkv, n, D, dtype=torch.float64), torch.zeros(self.hkv, n, D, dtype=torch.float64)
        held = torch.zeros(n, dtype=torch.bool)
        for p in range(-(-n // self.page)):
            id = int(self.table[b, p]) if p < self.width else -1
            if 0 <= id < self.n_pages:
                e = min(n, (p + 1) * self.page)
                K[:, p * self.page:e], V[:, p * self.page:e] = self.K[id, :, :e - p * self.page].double(), self.V[id, :, :e - p * self.page].double()
                held[p * self.page:e] = True
        return K, V, held

    def attention(self, q, window):
        """The definition in 64 bits: outputs [T][hq][D] and how far off the kernel's may be; NaN rows belong to no sequence."""
        out = torch.full((self.T, self.hq, D), math.nan, dtype=torch.float64)
        tol = torch.zeros_like(out)
        G, step = self.hq // self.hkv, HALF_STEP[self.dtype]
        for b, (t, n) in enumerate(self.lens):
            if t == 0:
                continue
            s0 = int(self.start[b])
            K, V, held = self.rows(b, max(n, 0))
            pos = torch.arange(n - t, n)[:, None]
            j = torch.arange(max(n, 0))[None]
            sees = (j <= pos) & held[None]
            if window:
                sees &= j > pos - window
            for h in range(self.hq):
                Kh, Vh = K[h // G], V[h // G]
                qh = q[s0:s0 + t, h].double()
                x = torch.where(sees, qh @ Kh.T * self.scale, torch.tensor(-math.inf, dtype=torch.float64))
                some = sees.any(dim=1)
                m = torch.where(some, x.amax(dim=1) if n > 0 else torch.zeros(t, dtype=torch.float64), torch.zeros(t, dtype=torch.float64))
                w = torch.exp(x - m[:, None])
                w = w / torch.where(some, w.sum(dim=1), torch.ones(t, dtype=torch.float64))[:, None]
                for i in range(t):      # row by row, so that a value that is no number reaches the rows that see it alone
                    v = sees[i]
                    out[s0 + i, h] = w[i, v] @ Vh[v]
                    size = w[i, v] @ Vh[v].abs() + out[s0 + i, h].abs()
                    # A weight is off by the error of its score (128 products and sums of 2^-24 each, as many in the scaling), by
                    # two roundings of the exponential, and for bf16 by its own rounding; the outputs by the weights' errors against the
                    # size of what is summed, by the sums of up to n terms, and by the last rounding.
                    S = (qh[i].abs() @ Kh[v].abs().T * self.scale).amax() if v.any() else torch.tensor(0.0)
                    weight = 2 * (136 * 2.0 ** -24 * S + 2.0 ** -21) + (1.02 * step if self.dtype == "bf16" else 0)
                    tol[s0 + i, h] = (weight + (int(v.sum()) + 64) * 2.0 ** -24) * size + step * out[s0 + i, h].abs()
        return out, tol


def check_attention(c, window=0, q=None, note=""):
    q = c.randn(c.T, c.hq, D) if q is None else q
    say(f"attention {note} lens={c.lens} {c.dtype} heads={c.hq}/{c.hkv} page={c.page} {c.layout} window={window}")
    out = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
    L.lvr_paged_attention(c.h, *c.pools(), q.cuda(), *c.batch(), out, window=window)
    torch.cuda.synchronize()
    out = out.cpu().double()
    ref, tol = c.attention(q, window)
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


LENS = {
    "one_key": [(1, 1)],
    "single_tokens": [(1, 17), (1, 16), (1, 15), (0, 5), (1, 300), (1, 31), (1, 33)],
    "long_single": [(1, 2500)],
    "whole_prompts": [(5, 5), (17, 17), (0, 0), (64, 64)],
    "chunks": [(33, 100), (1, 257), (7, 129), (16, 64)],
    "one_chunk": [(130, 130)],
    "late_chunk": [(70, 700), (3, 3)],
    "beside_decodes": [(200, 333), (1, 90), (1, 1), (1, 513)],
    "many": [(1 + (i * 7) % 3, 3 + (i * 37) % 90) for i in range(70)] + [(0, 12)] * 70 + [(40, 300), (1, 600)],
    "many_single_tokens": [(1, 1 + (i * 53) % 400) for i in range(131)],
    "cut_both_ways": [(40, 3000), (1, 4000), (2, 2500), (5, 700)],
    "cut_chunk": [(300, 2600)],
    "tokens_before_the_cache": [(5, 3), (1, 0), (4, 0), (2, 40)],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS)
def test_attention_over_lengths(lens, dtype):
    with Cache(LENS[lens], dtype=dtype, seed=3) as c:
        check_attention(c)


@pytest.mark.parametrize("dtype, hq, hkv, lens, window", [
    ("bf16", 8, 1, [(1, 20000)], 0),               # more runs than are merged at once
    ("f32", 16, 1, [(1, 20000)], 0),
    ("bf16", 4, 1, [(1, 9000), (1, 12000)], 7000),
    ("bf16", 2, 1, [(1, 140000)], 0),
    ("bf16", 8, 1, [(17, 9000)], 0),               # several tiles of 16 rows or one of 128, cut
    ("f32", 4, 1, [(30, 5000), (1, 5000)], 0),
])
def test_attention_cut_into_many_runs(dtype, hq, hkv, lens, window):
    with Cache(lens, dtype=dtype, hq=hq, hkv=hkv, page=64, seed=50) as c:
        out = check_attention(c, window=window)
        q = torch.Generator().manual_seed(3)
        q = torch.randn(c.T, hq, D, generator=q).to(c.dt).cuda()
        a, b = torch.empty_like(q), torch.empty_like(q)
        pools, batch = c.pools(), c.batch()
        for o in (a, b):
            L.lvr_paged_attention(c.h, *pools, q, *batch, o, window=window)
        assert torch.equal(a, b), "the order of the runs shows in the result"
        assert out.shape[0] == c.T


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (3, 1), (4, 4), (8, 1), (12, 2), (20, 1), (40, 8), (71, 1)])
def test_attention_over_heads(hq, hkv, dtype):
    with Cache([(1, 70), (9, 41), (1, 200)], dtype=dtype, hq=hq, hkv=hkv, seed=4) as c:
        check_attention(c)


@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_attention_over_pages(page, layout):
    with Cache([(1, 70), (40, 300), (1, 1040)], page=page, layout=layout, seed=5) as c:
        check_attention(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 7, 33, 64, 300, 100000, 2 ** 31 - 1])
def test_attention_with_a_window(window, dtype):
    with Cache([(1, 400), (90, 333), (5, 5), (1, 30)], dtype=dtype, seed=6) as c:
        check_attention(c, window=window)


def test_attention_with_a_scale_of_its_own():
    with Cache([(3, 50)], scale=0.7, seed=7) as c:
        check_attention(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 50])
def test_what_no_token_sees_may_be_anything(window, dtype):
    """NaN and infinities behind the end of a sequence, in spare pages, before every window, and in keys and values of later tokens."""
    with Cache([(20, 90), (1, 200), (1, 17)], dtype=dtype, seed=8) as c:
        seen = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
        for b, (t, n) in enumerate(c.lens):
            for p in range(max(0, n - t - window + 1) if window else 0, n):
                seen[c.table[b, p // c.page], p % c.page] = True
        for pool in (c.K, c.V):
            pool.transpose(1, 2)[~seen] = math.nan
        check_attention(c, window=window, note="unseen")
        c.V[c.table[0, 88 // c.page], :, 88 % c.page, 5] = math.nan      # only the last two tokens of the first sequence see it
        c.V[c.table[0, 85 // c.page], 0, 85 % c.page, 77] = math.inf
        c.V[c.table[1, 199 // c.page], 1, 199 % c.page, 3] = -math.inf
        out = check_attention(c, window=window, note="seen by some")
        assert torch.isfinite(out[:15]).all() and not torch.isfinite(out[18:20]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_pages_take_no_part(dtype):
    with Cache([(1, 300), (40, 200), (1, 20)], dtype=dtype, seed=9) as c:
        c.table[0, 3], c.table[0, 7], c.table[0, 18] = -1, c.n_pages, 2 ** 31 - 1       # the last: the page of the new token
        c.table[1, 0], c.table[1, 11] = -2 ** 31, -5
        c.table[2, :] = -1                                                               # nothing at all: zeros
        out = check_attention(c)
        assert (out[41] == 0).all()


def test_a_sequence_longer_than_its_table():
    with Cache([(4, 60), (1, 30)], seed=10, extra_width=0) as c:
        c.lens = [(4, 90), (1, 30)]
        c.len = torch.tensor([90, 30], dtype=torch.int32)
        check_attention(c)


def test_rows_of_no_sequence_stay_as_they_were():
    with Cache([(3, 20), (0, 9), (2, 40)], seed=11, behind=30, gap=5) as c:
        check_attention(c)


def test_attention_of_large_scores():
    """Scores of some thousands in both directions: the maximum moves by more than the exponents' range from key to key."""
    for dtype in ("bf16", "f32"):
        with Cache([(1, 500), (30, 100)], dtype=dtype, seed=12) as c:
            c.K *= 64
            check_attention(c, note="large")
            c.K[:, :, ::2] = -c.K[:, :, ::2].abs()
            check_attention(c, q=c.randn(c.T, c.hq, D).abs() * 30, note="large, of one sign")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_query_rows_may_be_a_slice_of_a_projection(dtype):
    with Cache([(6, 50), (1, 20)], dtype=dtype, seed=13) as c:
        fused = c.randn(c.T, (c.hq + 2 * c.hkv) * D)
        q = fused[:, :c.hq * D].unflatten(1, (c.hq, D))
        a, b = (torch.zeros(c.T, c.hq, D, dtype=c.dt, device="cuda") for _ in range(2))
        pools, batch, dev = c.pools(), c.batch(), fused.cuda()
        L.lvr_paged_attention(c.h, *pools, dev[:, :c.hq * D].unflatten(1, (c.hq, D)), *batch, a)
        L.lvr_paged_attention(c.h, *pools, q.contiguous().cuda(), *batch, b)
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ append
def rotated(x, pos, inv_freq, axis, rot, pairs):
    """64 bits: x [T][heads][D], pos [T][axes]; and the size of what a rotated value is summed from."""
    y, size = x.double().clone(), x.double().abs()
    angle = pos.double()[:, axis] * torch.tensor(inv_freq, dtype=torch.float64)
    cs, sn = angle.cos()[:, None], angle.sin()[:, None]
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if pairs == L.LVR_ROT_HALVES else (slice(0, rot, 2), slice(1, rot, 2))
    u, w = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = u * cs - w * sn, u * sn + w * cs
    size[..., a] = size[..., b] = u.abs() + w.abs()
    return y, size


def freqs(rot, base=10000.0):
    return [base ** (-2 * c / rot) for c in range(rot // 2)]


def check_append(c, inv_freq, axis, rot, pairs, positions, with_q=True, sliced=True):
    say(f"append lens={c.lens} {c.dtype} heads={c.hq}/{c.hkv} page={c.page} {c.layout} rot={rot} pairs={pairs} q={with_q}")
    fused = c.randn(c.T, (c.hq + 2 * c.hkv) * D)
    q, k, v = (x.unflatten(1, (-1, D)) for x in fused.split([c.hq * D, c.hkv * D, c.hkv * D], dim=1))
    dev = fused.cuda()
    dq, dk, dv = (x.unflatten(1, (-1, D)) for x in dev.split([c.hq * D, c.hkv * D, c.hkv * D], dim=1))
    if not sliced:
        dq, dk, dv = dq.contiguous(), dk.contiguous(), dv.contiguous()
    kp, vp = c.pools()
    qo = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
    L.lvr_paged_append(c.h, kp, vp, dk, dv, *c.batch(), q=dq if with_q else None, q_out=qo if with_q else None,
                       positions=None if positions is None else positions.cuda())
    torch.cuda.synchronize()
    K, V, qo = c.from_pool(kp).double(), c.from_pool(vp).double(), qo.cpu().double()
    pos = torch.zeros(c.T, max(c.cfg.rot_axes, 1), dtype=torch.int64) if positions is None else positions.long()
    if positions is None:
        for b, (t, n) in enumerate(c.lens):
            s0 = int(c.start[b])
            pos[s0:s0 + t] = torch.arange(n - t, n)[:, None]
    kr, ks = rotated(k, pos, inv_freq, axis, rot, pairs) if rot else (k.double(), 0 * k.double())
    qr, qs = rotated(q, pos, inv_freq, axis, rot, pairs) if rot else (q.double(), 0 * q.double())
    # a sine is off by its argument's rounding (2^-24 of at most pi / 4, three times), the series' end and the sums of it, five
    # more steps of 2^-24; the rotation by two products and a sum
    rel, off = HALF_STEP[c.dtype], 12 * 2.0 ** -24
    want_k, want_v = c.K.double().clone(), c.V.double().clone()
    tol_k = torch.zeros_like(want_k)
    for b, (t, n) in enumerate(c.lens):
        for i in range(t):
            p, s = n - t + i, int(c.start[b]) + i
            id = int(c.table[b, p // c.page]) if 0 <= p < c.width * c.page else -1
            if not 0 <= id < c.n_pages:
                continue
            at = (id, slice(None), p % c.page)
            want_k[at], want_v[at] = kr[s], v[s].double()
            tol_k[at] = rel * kr[s].abs() + off * ks[s]
            tol_k[at][:, rot:] = 0
    assert ((K - want_k).abs() <= tol_k).all(), float(((K - want_k).abs() - tol_k).max())
    assert torch.equal(V, want_v)
    inside = torch.zeros(c.T, dtype=torch.bool)
    inside[int(c.start[0]):int(c.start[-1])] = with_q
    assert (qo[~inside] == 7).all()
    tol_q = rel * qr.abs() + off * qs
    tol_q[..., rot:] = 0
    assert ((qo - qr).abs() <= tol_q)[inside].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", ["one_key", "single_tokens", "whole_prompts", "chunks", "tokens_before_the_cache"])
def test_append_over_lengths(lens, dtype):
    f = freqs(128)
    with Cache(LENS[lens], dtype=dtype, rot_dim=128, inv_freq=f, seed=20) as c:
        check_append(c, f, [0] * 64, 128, L.LVR_ROT_HALVES, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [L.LVR_ROT_HALVES, L.LVR_ROT_NEIGHBOURS])
@pytest.mark.parametrize("rot", [0, 16, 64, 96, 128])
def test_append_over_rotations(rot, pairs, dtype):
    f = freqs(rot) if rot else None
    with Cache([(5, 9), (1, 100)], dtype=dtype, rot_dim=rot, pairs=pairs, inv_freq=f, seed=21, layout="token") as c:
        check_append(c, f, [0] * (rot // 2), rot, pairs, None)


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("hq, hkv", [(1, 1), (3, 1), (24, 8), (71, 1)])
def test_append_over_axes_and_heads(hq, hkv, axes):
    f = freqs(128)
    axis = torch.randint(0, axes, (64,), generator=torch.Generator().manual_seed(axes)).tolist()
    with Cache([(5, 9), (0, 3), (12, 40)], hq=hq, hkv=hkv, rot_dim=128, rot_axes=axes, inv_freq=f, axis=axis, seed=22, behind=4, gap=2) as c:
        pos = torch.randint(-50, 5000, (c.T, axes), generator=c.g).to(torch.int32)
        check_append(c, f, axis, 128, L.LVR_ROT_HALVES, pos)


def test_append_of_keys_alone_and_of_whole_arrays():
    f = freqs(64)
    for with_q in (False, True):
        with Cache([(5, 9), (3, 40)], rot_dim=64, inv_freq=f, seed=23) as c:
            check_append(c, f, [0] * 32, 64, L.LVR_ROT_HALVES, None, with_q=with_q, sliced=False)


def test_positions_far_off_and_below_zero():
    """Angles of up to 2^31 radians and of frequencies above a turn per position; the reference's own angle is exact to 2^-53 of them."""
    f = freqs(128, base=500000.0)
    f[3], f[4], f[5] = 0.0, -0.75, 9.5
    with Cache([(8, 8)], dtype="f32", rot_dim=128, inv_freq=f, seed=24) as c:
        pos = torch.tensor([[0], [1], [-1], [10 ** 6], [2 ** 24 + 1], [-(2 ** 24)], [10 ** 8 + 1], [1048577]], dtype=torch.int32)
        check_append(c, f, [0] * 64, 128, L.LVR_ROT_HALVES, pos)


def test_appends_to_missing_pages_are_dropped():
    f = freqs(128)
    with Cache([(30, 50), (3, 20)], rot_dim=128, inv_freq=f, seed=25) as c:
        c.table[0, 1], c.table[0, 2], c.table[1, 1] = -1, c.n_pages, 2 ** 31 - 1
        check_append(c, f, [0] * 64, 128, L.LVR_ROT_HALVES, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [L.LVR_ROT_HALVES, L.LVR_ROT_NEIGHBOURS])
@pytest.mark.parametrize("rot", [64, 128])
@pytest.mark.parametrize("hq, hkv, lens", [(66, 2, [(150, 200), (0, 7), (1, 90), (89, 89)]), (3, 3, [(1801, 1900), (20, 64)])])
def test_append_of_many_rows(hq, hkv, lens, rot, pairs, dtype):
    """At least 16384 rows, from which on a wave takes several and stores around the caches; 70 and 9 rows to a token, no multiple of a wave's."""
    f = freqs(rot)
    axis = [i % 3 for i in range(rot // 2)]
    with Cache(lens, dtype=dtype, hq=hq, hkv=hkv, rot_dim=rot, rot_axes=3, pairs=pairs, inv_freq=f, axis=axis, seed=27, behind=3, gap=2) as c:
        assert c.T * (hq + 2 * hkv) >= 16384
        c.table[0, 2], c.table[3 if len(lens) > 2 else 1, 1] = -1, c.n_pages
        pos = torch.randint(-50, 5000, (c.T, 3), generator=c.g).to(torch.int32)
        check_append(c, f, axis, rot, pairs, pos)


def test_query_is_rotated_in_place():
    f = freqs(128)
    with Cache([(7, 30)], rot_dim=128, inv_freq=f, seed=26) as c:
        k, q = c.randn(c.T, c.hkv, D).cuda(), c.randn(c.T, c.hq, D).cuda()
        out, again = torch.empty_like(q), q.clone()
        L.lvr_paged_append(c.h, *c.pools(), k, k, *c.batch(), q=q, q_out=out)
        L.lvr_paged_append(c.h, *c.pools(), k, k, *c.batch(), q=again, q_out=again)
        assert torch.equal(out, again) and not torch.equal(out, q)


# ------------------------------------------------------------------------------------------------ gather
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page, layout", [(16, "head"), (16, "token"), (64, "head"), (256, "token")])
def test_gather(page, layout, dtype):
    for n in (1, 15, 16, 300, 333):
        with Cache([(0, 300), (0, 0), (0, 17), (0, 64), (0, 90)], dtype=dtype, page=page, layout=layout, seed=30) as c:
            c.table[4, 0] = -1
            say(f"gather n={n} {dtype} page={page} {layout}")
            K, V = (torch.full((5, c.hkv, n, D), 7.0, dtype=c.dt, device="cuda") for _ in range(2))
            kp, vp = c.pools()
            _, length, table = c.batch()
            L.lvr_paged_gather(c.h, kp, vp, length, table, K, V)
            for b, (_, held) in enumerate(c.lens):
                Kr, Vr, has = c.rows(b, min(held, n))
                for got, ref in ((K, Kr), (V, Vr)):
                    want = torch.full((c.hkv, n, D), 7.0, dtype=torch.float64)
                    want[:, :min(held, n)][:, has] = ref[:, has]
                    assert torch.equal(got[b].cpu().double(), want)


@pytest.mark.parametrize("dtype, heads", [("bf16", 8), ("f32", 4)])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_gather_of_more_than_the_caches_hold(dtype, heads, layout):
    """3 sequences of up to 32773 rows: past 192 MiB of keys, where the rows are stored around the caches."""
    n, lens, page = 32773, [32773, 20001, 0], 64
    dt, g = DTYPES[dtype], torch.Generator(device="cuda").manual_seed(31)
    used = [-(-x // page) for x in lens]
    n_pages, width = sum(used) + 1, max(used)
    assert n * heads * len(lens) * D * dt.itemsize >= 192 << 20
    say(f"gather n={n} {dtype} heads={heads} {layout}")
    shape = (n_pages, heads, page, D) if layout == "head" else (n_pages, page, heads, D)
    kp, vp = (torch.randn(shape, generator=g, device="cuda").to(dt) for _ in range(2))
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(32)).tolist()
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    for b, u in enumerate(used):
        table[b, :u] = torch.tensor([order.pop() for _ in range(u)], dtype=torch.int32)
    table[0, 7] = -1
    h = L.lvr_paged_create(L.make_paged_config(n_q_heads=heads, n_kv_heads=heads, kv_dtype=L.LVR_BF16 if dtype == "bf16" else L.LVR_F32, page_size=page,
                                               n_pages=n_pages, layout=layout))
    try:
        K, V = (torch.full((len(lens), heads, n, D), 7.0, dtype=dt, device="cuda") for _ in range(2))
        L.lvr_paged_gather(h, kp, vp, torch.tensor(lens, dtype=torch.int32, device="cuda"), table.cuda(), K, V)
        for got, pool in ((K, kp), (V, vp)):
            by_head = pool if layout == "head" else pool.transpose(1, 2)
            for b, x in enumerate(lens):
                rows = by_head[table[b, :used[b]].long().clamp(min=0).cuda()].transpose(0, 1).reshape(heads, -1, D)[:, :x].clone()
                if b == 0:
                    rows[:, 7 * page:8 * page] = 7
                assert torch.equal(got[b, :, :x], rows) and (got[b, :, x:] == 7).all()
    finally:
        L.lvr_paged_destroy(h)


# ------------------------------------------------------------------------------------------------ refusals
def test_calls_refuse_what_they_cannot_take():
    with Cache([(2, 20), (1, 40)], rot_dim=128, inv_freq=freqs(128), seed=40) as c:
        kp, vp = c.pools()
        start, length, table = c.batch()
        q, k = c.randn(c.T, c.hq, D).cuda(), c.randn(c.T, c.hkv, D).cuda()
        out = torch.empty_like(q)
        K = torch.zeros(2, c.hkv, 40, D, dtype=c.dt, device="cuda")
        attend = lambda **o: L.lvr_paged_attention(**dict(dict(h=c.h, k_pages=kp, v_pages=vp, q=q, seq_start=start, seq_len=length, table=table, out=out), **o))   # noqa: E731
        append = lambda **o: L.lvr_paged_append(**dict(dict(h=c.h, k_pages=kp, v_pages=vp, k_new=k, v_new=k, seq_start=start, seq_len=length, table=table, q=q, q_out=out), **o))   # noqa: E731
        gather = lambda **o: L.lvr_paged_gather(**dict(dict(h=c.h, k_pages=kp, v_pages=vp, seq_len=length, table=table, K_out=K, V_out=K.clone()), **o))   # noqa: E731
        for call in (attend, append, gather):
            for bad in (dict(k_pages=kp[:-1]), dict(v_pages=vp.float()), dict(k_pages=kp[:, :, :, :64]), dict(v_pages=vp.cpu()), dict(k_pages=kp.transpose(1, 2)[:, :, :1]),
                        dict(seq_len=length.long()), dict(seq_len=length[:1]), dict(table=table[0]), dict(table=table[:1]), dict(table=table.T)):
                with pytest.raises(ValueError):
                    call(**bad)
        for call in (attend, append):
            for bad in (dict(seq_start=start[:-1]), dict(seq_start=start.float()), dict(q=q[:, :4]), dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(q=q[..., ::2])):
                with pytest.raises(ValueError):
                    call(**bad)
        for bad in (dict(out=out[:1]), dict(out=out.float()), dict(out=out.cpu()), dict(window=-1), dict(window=1 << 31), dict(window=1 << 70)):
            with pytest.raises(ValueError):
                attend(**bad)
        for bad in (dict(q=None), dict(q_out=None), dict(v_new=k[:1]), dict(k_new=k[:, :1]), dict(positions=torch.zeros(c.T, 2, dtype=torch.int32, device="cuda")),
                    dict(positions=torch.zeros(c.T, 1, dtype=torch.int64, device="cuda"))):
            with pytest.raises(ValueError):
                append(**bad)
        for bad in (dict(K_out=K[:1]), dict(V_out=K[:, :, :3]), dict(K_out=K.float()), dict(K_out=K[0])):
            with pytest.raises(ValueError):
                gather(**bad)

        def refused(code, call, *a):
            assert call(*a) == code

        lib, big = L.lib(), 1 << 40
        p = lambda t, off=0: t.data_ptr() + off   # noqa: E731
        st = lambda *s: (L.binding.C.c_int64 * 3)(*s)   # noqa: E731
        hq, hk = c.hq * D, c.hkv * D
        att = lambda k=p(kp), v=p(vp), q=p(q), qs=hq, s=p(start), n=p(length), t=p(table), w=c.width, b=2, T=c.T, win=0, o=p(out): lib.lvr_paged_attention(c.h, k, v, q, qs, s, n, t, w, b, T, win, o, None)   # noqa: E731
        for kw in (dict(k=None), dict(v=None), dict(q=None), dict(s=None), dict(n=None), dict(t=None), dict(o=None), dict(qs=hq - 8), dict(qs=hq + 4), dict(q=p(q, 2)),
                   dict(k=p(kp, 8)), dict(v=p(vp, 4)), dict(o=p(out, 8)), dict(s=p(start, 2)), dict(n=p(length, 1)), dict(t=p(table, 2)), dict(w=-1), dict(b=-1), dict(T=-1),
                   dict(win=-1), dict(o=p(q)), dict(qs=-hq), dict(qs=big)):
            assert att(**kw) == L.LVR_E_INVALID, kw
        for kw in (dict(b=4097), dict(w=1 << 27), dict(T=1 << 25)):
            assert att(**kw) == L.LVR_E_CAPACITY, kw
        assert att(T=0, q=None, o=None) == L.LVR_OK and att(b=0) == L.LVR_OK and att() == L.LVR_OK
        app = lambda k=p(k), v=p(k), q=p(q), o=p(out), s=st(hk, hk, hq), pos=None, T=c.T: lib.lvr_paged_append(c.h, p(kp), p(vp), k, v, q, o, s, pos, p(start), p(length), p(table), c.width, 2, T, None)   # noqa: E731
        for kw in (dict(k=None), dict(v=None), dict(q=None), dict(o=None), dict(s=None), dict(s=st(hk - 8, hk, hq)), dict(s=st(hk, hk + 4, hq)), dict(s=st(hk, hk, hq - 128)),
                   dict(k=p(k, 8)), dict(q=p(q, 2)), dict(o=p(out, 4)), dict(pos=p(start, 1)), dict(q=p(q), o=p(q), s=st(hk, hk, hq + 128))):
            assert app(**kw) == L.LVR_E_INVALID, kw
        assert app() == L.LVR_OK
        gat = lambda K1=p(K), V1=p(K), n=40: lib.lvr_paged_gather(c.h, p(kp), p(vp), p(length), p(table), c.width, 2, n, K1, V1, None)   # noqa: E731
        for kw in (dict(K1=None), dict(V1=None), dict(K1=p(K, 8)), dict(n=-1)):
            assert gat(**kw) == L.LVR_E_INVALID, kw
        assert gat(n=(1 << 30) + 1) == L.LVR_E_CAPACITY and gat(n=0, K1=None) == L.LVR_OK
        torch.cuda.synchronize()


def test_marshalled_arguments_and_plain_ones_give_the_same(monkeypatch):
    """Tensors, tensors marshalled once, and the general binding without the compiled calls."""
    f = freqs(64)
    with Cache([(5, 40), (1, 20)], rot_dim=64, inv_freq=f, seed=42) as c:
        results = []
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
            L.lvr_paged_append(c.h, A(kp), A(vp), A(k), A(v), start, length, table, q=A(q), q_out=A(qo))
            L.lvr_paged_attention(c.h, A(kp), A(vp), A(qo), start, length, table, A(out), window=30)
            L.lvr_paged_gather(c.h, A(kp), A(vp), length, table, A(K), A(V))
            results.append([x.clone() for x in (kp, vp, qo, out, K, V)])
        for other in results[1:]:
            assert all(torch.equal(x, y) for x, y in zip(results[0], other))


def test_empty_batches():
    with Cache([], seed=41) as c:
        z = lambda *s: torch.zeros(s, dtype=c.dt, device="cuda")   # noqa: E731
        L.lvr_paged_attention(c.h, *c.pools(), z(0, c.hq, D), *c.batch(), z(0, c.hq, D))
        L.lvr_paged_append(c.h, *c.pools(), z(0, c.hkv, D), z(0, c.hkv, D), *c.batch())
        L.lvr_paged_gather(c.h, *c.pools(), *c.batch()[1:], z(0, c.hkv, 4, D), z(0, c.hkv, 4, D))
        torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ as they are used
def test_pools_of_more_than_4_gib():
    """Pages past 2^32 bytes hold the same rows as a small pool and give the same bits."""
    lens, hq, hkv, page = [(3, 200), (1, 77), (40, 90)], 16, 8, 64
    big = 40000                                      # pages of 128 KiB
    with Cache(lens, hq=hq, hkv=hkv, page=page, rot_dim=128, inv_freq=freqs(128), seed=60) as c:
        used = [int(p) for p in c.table.flatten() if p >= 0]
        far = {p: big - 1 - 37 * i for i, p in enumerate(used)}
        cfg = L.make_paged_config(n_q_heads=hq, n_kv_heads=hkv, page_size=page, n_pages=big, rot_dim=128)
        h = L.lvr_paged_create(cfg, inv_freq=freqs(128))
        try:
            K, V = (torch.empty(big, hkv, page, D, dtype=c.dt, device="cuda") for _ in range(2))
            kp, vp = c.pools()
            for p, f in far.items():
                K[f], V[f] = kp[p], vp[p]
            table = torch.tensor([[far.get(int(p), -1) for p in row] for row in c.table], dtype=torch.int32, device="cuda")
            start, length, small_table = c.batch()
            k, q = c.randn(c.T, hkv, D).cuda(), c.randn(c.T, hq, D).cuda()
            got = []
            for handle, pools, tab in ((c.h, (kp, vp), small_table), (h, (K, V), table)):
                qo, out = torch.empty_like(q), torch.empty_like(q)
                rows = [torch.zeros(3, hkv, 200, D, dtype=c.dt, device="cuda") for _ in range(2)]
                L.lvr_paged_append(handle, *pools, k, k, start, length, tab, q=q, q_out=qo)
                L.lvr_paged_attention(handle, *pools, qo, start, length, tab, out)
                L.lvr_paged_gather(handle, *pools, length, tab, *rows)
                got.append([qo, out, *rows])
            assert all(torch.equal(x, y) for x, y in zip(*got))
            for p, f in far.items():
                assert torch.equal(K[f], kp[p]) and torch.equal(V[f], vp[p])
        finally:
            L.lvr_paged_destroy(h)


def _prompt_in_chunks(c, k, v, q, sizes, stream=None):
    """Appends and attends the tokens of one sequence piece by piece; returns pools and outputs."""
    kp, vp = c.pools()
    outs, at = [], 0
    table = c.table.cuda()
    for m in sizes:
        start = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        length = torch.tensor([at + m], dtype=torch.int32, device="cuda")
        qo, out = torch.empty_like(q[at:at + m]), torch.empty_like(q[at:at + m])
        L.lvr_paged_append(c.h, kp, vp, k[at:at + m], v[at:at + m], start, length, table, q=q[at:at + m], q_out=qo, stream=stream)
        L.lvr_paged_attention(c.h, kp, vp, qo, start, length, table, out, stream=stream)
        outs.append(out)
        at += m
    return kp, vp, torch.cat(outs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_from_the_prompt_to_the_index(dtype):
    """A prompt comes in pieces of odd sizes through append and attention, its pages become rows, the rows an index, and the next token
    is decoded from the index and from the pages: the same keys, the same attention."""
    n, hq, hkv, f = 700, 8, 2, freqs(128)
    with Cache([(n, n + 1)], dtype=dtype, hq=hq, hkv=hkv, rot_dim=128, inv_freq=f, seed=61) as c:
        fused = c.randn(n + 1, (hq + 2 * hkv) * D)
        q, k, v = (x.unflatten(1, (-1, D)) for x in fused.split([hq * D, hkv * D, hkv * D], dim=1))
        dq, dk, dv = (x.unflatten(1, (-1, D)) for x in fused.cuda().split([hq * D, hkv * D, hkv * D], dim=1))
        kp, vp, out = _prompt_in_chunks(c, dk[:n], dv[:n], dq[:n], [1, 130, 17, 300, 252])
        # the whole prompt in 64 bits, from the rotated rows as the pages hold them
        pos = torch.arange(n + 1)[:, None]
        Kr = rotated(k, pos, f, [0] * 64, 128, L.LVR_ROT_HALVES)[0].to(c.dt)
        Qr = rotated(q, pos, f, [0] * 64, 128, L.LVR_ROT_HALVES)[0].to(c.dt)
        ref = torch.empty(n, hq, D, dtype=torch.float64)
        for h in range(hq):
            s = Qr[:n, h].double() @ Kr[:n, h // 4].double().T / math.sqrt(D)
            s = torch.where(torch.ones(n, n, dtype=torch.bool).tril(), s, torch.tensor(-math.inf, dtype=torch.float64))
            ref[:, h] = torch.softmax(s, dim=1) @ v[:n, h // 4].double()
        # A key or query component may be rounded the other way than the reference's (its value lies next to a border: one step, 2 * HALF_STEP of
        # it); a score of 128 such products of size S moves by at most 4 * HALF_STEP * S and a weight by twice that, on top of what
        # test_attention_over_lengths counts.  S is at most about 30 here; the outputs are means of values of size 1.
        step = HALF_STEP[dtype]
        S = max(float((Qr[:n, h].double().abs() @ Kr[:n, h // 4].double().abs().T / math.sqrt(D)).max()) for h in range(hq))
        tol = (8 * step * S + 4 * step) * 4
        assert (out.cpu().double() - ref).abs().max() <= tol
        rows = [torch.zeros(1, hkv, n, D, dtype=c.dt, device="cuda") for _ in range(2)]
        length = torch.tensor([n], dtype=torch.int32, device="cuda")
        L.lvr_paged_gather(c.h, kp, vp, length, c.table.cuda(), *rows)
        assert torch.equal(rows[1][0].cpu(), v[:n].transpose(0, 1))
        cfg = L.make_config(batch=1, n_q_heads=hq, n_kv_heads=hkv, kv_dtype=L.LVR_BF16 if dtype == "bf16" else L.LVR_F32, capacity=n + 1,
                            group_size=1 if dtype == "bf16" else 4)
        ix = L.lvr_create(cfg)
        try:
            L.lvr_build(ix, *rows)
            start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
            length = torch.tensor([n + 1], dtype=torch.int32, device="cuda")
            qo, paged = (torch.empty(1, hq, D, dtype=c.dt, device="cuda") for _ in range(2))
            L.lvr_paged_append(c.h, kp, vp, dk[n:], dv[n:], start, length, c.table.cuda(), q=dq[n:], q_out=qo)
            L.lvr_paged_attention(c.h, kp, vp, qo, start, length, c.table.cuda(), paged)
            new = [torch.zeros(1, hkv, n + 1, D, dtype=c.dt, device="cuda") for _ in range(2)]
            L.lvr_paged_gather(c.h, kp, vp, length, c.table.cuda(), *new)
            tau = torch.full((1, hq), -math.inf, device="cuda")
            idx = torch.zeros(1, hq, n + 1, dtype=torch.int32, device="cuda")
            cnt, dense = torch.zeros(1, hq, dtype=torch.int32, device="cuda"), torch.empty(1, hq, D, device="cuda")
            L.lvr_append_decode_step(ix, new[0][:, :, n:].contiguous(), new[1][:, :, n:].contiguous(), qo.float(), tau, dense, idx, cnt)
            torch.cuda.synchronize()
            assert (cnt == n + 1).all()
            got, want = paged.double().cpu(), dense.double().cpu()
            # the index keeps its weights in fp32; the pages' attention rounds them to the cache's type, and its output
            err = (got - want).abs().amax() / want.abs().amax()
            assert err <= (4 * step if dtype == "bf16" else 2e-5), float(err)
        finally:
            L.lvr_destroy(ix)


def test_calls_on_a_stream_of_their_own_and_two_handles_at_once():
    f = freqs(128)
    a = Cache([(130, 400), (1, 900)], rot_dim=128, inv_freq=f, seed=62)
    b = Cache([(1, 3000), (3, 50)], rot_dim=128, inv_freq=f, seed=63)
    with a, b:
        args = []
        for c in (a, b):
            k, q = c.randn(c.T, c.hkv, D).cuda(), c.randn(c.T, c.hq, D).cuda()
            args.append((c, c.pools(), k, q, c.batch(), torch.empty_like(q), torch.empty_like(q)))
        def work(x, stream):
            c, pools, k, q, batch, qo, out = x
            L.lvr_paged_append(c.h, *pools, k, k, *batch, q=q, q_out=qo, stream=stream)
            L.lvr_paged_attention(c.h, *pools, qo, *batch, out, stream=stream)
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_steps_follow_the_arrays(dtype):
    """A decode step and a step with a prompt in it, recorded once each on one handle and replayed in turn while lengths, tables and inputs
    change: every replay gives the eager call's bits.  Rows behind the last sequence (a padded batch) stay as they were."""
    f = freqs(128)
    with Cache([(1, 900), (1, 40), (1, 2000), (0, 0)], dtype=dtype, rot_dim=128, inv_freq=f, seed=64, behind=0) as c:
        kp, vp = c.pools()
        table = c.table.cuda()
        steps = []
        for T in (4, 160):
            s = dict(start=torch.zeros(5, dtype=torch.int32, device="cuda"), length=torch.zeros(4, dtype=torch.int32, device="cuda"))
            for name, heads in (("k", c.hkv), ("q", c.hq), ("qo", c.hq), ("out", c.hq)):
                s[name] = torch.zeros(T, heads, D, dtype=c.dt, device="cuda")
            steps.append(s)

        def work(s):
            L.lvr_paged_append(c.h, kp, vp, s["k"], s["k"], s["start"], s["length"], table, q=s["q"], q_out=s["qo"])
            L.lvr_paged_attention(c.h, kp, vp, s["qo"], s["start"], s["length"], table, s["out"])

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
                    s["out"].fill_(7)
                    s["qo"].fill_(7)
                    torch.cuda.synchronize()
                    g.replay() if replay else work(s)
                    torch.cuda.synchronize()
                    results.append((s["out"].clone(), s["qo"].clone(), kp.clone(), vp.clone()))
                for other in results[1:]:
                    assert all(torch.equal(x, y) for x, y in zip(results[0], other)), turn
                assert (results[0][0][int(starts[-1]):] == 7).all() and (results[0][1][int(starts[-1]):] == 7).all()
                assert torch.isfinite(results[0][0].float()).all()


def test_a_batch_of_many_pieces():
    """4096 sequences of nine tiles each: more pieces than a launch has workgroups in one of its dimensions.  The same bits as from two halves."""
    seqs, t, hq = 4096, 33, 32
    cfg = L.make_paged_config(n_q_heads=hq, n_kv_heads=1, page_size=64, n_pages=seqs)
    h = L.lvr_paged_create(cfg)
    try:
        g = torch.Generator(device="cuda").manual_seed(5)
        K, V = (torch.randn(seqs, 1, 64, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        q = torch.randn(seqs * t, hq, D, generator=g, device="cuda").to(torch.bfloat16)
        start = torch.arange(0, seqs * t + 1, t, dtype=torch.int32, device="cuda")
        length = torch.randint(t, 65, (seqs,), generator=g, device="cuda").to(torch.int32)
        table = torch.randperm(seqs, generator=g, device="cuda").to(torch.int32)[:, None].contiguous()
        whole, halves = torch.empty_like(q), torch.empty_like(q)
        L.lvr_paged_attention(h, K, V, q, start, length, table, whole)
        for a, b in ((0, seqs // 2), (seqs // 2, seqs)):
            L.lvr_paged_attention(h, K, V, q[a * t:b * t], start[a:b + 1] - a * t, length[a:b], table[a:b], halves[a * t:b * t])
        assert torch.equal(whole, halves) and torch.isfinite(whole.float()).all()
    finally:
        L.lvr_paged_destroy(h)


@pytest.mark.parametrize("tokens", [1, 4, 40])
def test_lengths_far_beyond_the_table(tokens):
    """Sequences that claim 2^30 keys with a table of two pages: the division of such a batch stays within the work space of the fewest pieces
    per KV head, and every token attends the keys there are."""
    seqs, heads = 16, 256
    cfg = L.make_paged_config(n_q_heads=heads, n_kv_heads=heads, page_size=16, n_pages=2 * seqs)
    h = L.lvr_paged_create(cfg)
    try:
        g = torch.Generator(device="cuda").manual_seed(6)
        K, V = (torch.randn(2 * seqs, heads, 16, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        q = torch.randn(seqs * tokens, heads, D, generator=g, device="cuda").to(torch.bfloat16)
        start = torch.arange(0, seqs * tokens + 1, tokens, dtype=torch.int32, device="cuda")
        table = torch.arange(2 * seqs, dtype=torch.int32, device="cuda").view(seqs, 2)
        outs = []
        for n in (32 + tokens, 2 ** 30, 2 ** 31 - 1):
            length, out = torch.full((seqs,), n, dtype=torch.int32, device="cuda"), torch.empty_like(q)
            L.lvr_paged_attention(h, K, V, q, start, length, table, out)
            outs.append(out)
        s = torch.einsum("thd,hnd->thn", q[:tokens].float(), K[:2].permute(1, 0, 2, 3).reshape(heads, 32, D).float()) / math.sqrt(D)
        ref = torch.einsum("thn,hnd->thd", torch.softmax(s, dim=2), V[:2].permute(1, 0, 2, 3).reshape(heads, 32, D).float())
        assert (outs[0][:tokens].float() - ref).abs().max() <= 3 * 2.0 ** -8 * 5      # values below 5, each rounding half a step of them
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    finally:
        L.lvr_paged_destroy(h)


def test_sequences_in_no_order_leave_the_handle_usable():
    """seq_start that is not ascending is a mistake of the caller's: nothing is promised for that call's outputs, later calls are as before."""
    with Cache([(1, 3000), (1, 400), (2, 90)], seed=65) as c:
        q = c.randn(c.T, c.hq, D).cuda()
        start, length, table = c.batch()
        pools = c.pools()
        want, out = torch.empty_like(q), torch.empty_like(q)
        L.lvr_paged_attention(c.h, *pools, q, start, length, table, want)
        for bad in ([4, 0, 4, 0], [0, 4, 0, 4], [-5, 100, 2, -7], [2 ** 31 - 1, 0, 1, -2 ** 31], [3, 3, 1, 4]):
            L.lvr_paged_attention(c.h, *pools, q, torch.tensor(bad, dtype=torch.int32, device="cuda"), length, table, out)
            L.lvr_paged_append(c.h, *[p.clone() for p in pools], q[:, :c.hkv].contiguous(), q[:, :c.hkv].contiguous(),
                               torch.tensor(bad, dtype=torch.int32, device="cuda"), length, table)
            torch.cuda.synchronize()
            L.lvr_paged_attention(c.h, *pools, q, start, length, table, out)
            assert torch.equal(out, want)
        odd = torch.tensor([2 ** 31 - 1, -2 ** 31, 5], dtype=torch.int32, device="cuda")      # lengths beyond the table, below zero
        L.lvr_paged_attention(c.h, *pools, q, start, odd, table, out)
        L.lvr_paged_attention(c.h, *pools, q, start, length, table, out)
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq, hkv, lens", [
    (64, 8, [(356, 356)]),
    (32, 8, [(165, 165)] * 8),
    (28, 4, [(546, 546)]),
    (32, 8, [(96, 96), (1, 4000), (338, 352), (400, 400), (130, 131), (1, 1), (200, 900)]),
])
def test_prompts_whose_runs_are_made_longer(hq, hkv, lens, dtype):
    """The shortest runs make more partial results of these than the work space holds (test_paged_division.py has the division itself)."""
    with Cache(lens, dtype=dtype, hq=hq, hkv=hkv, seed=70) as c:
        check_attention(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 100])
def test_a_chunk_longer_than_twice_its_table(window, dtype):
    with Cache([(600, 200), (1, 190), (9, 160)], dtype=dtype, seed=71, extra_width=0) as c:
        c.lens = [(600, 600), (1, 190), (9, 160)]
        c.len = torch.tensor([600, 190, 160], dtype=torch.int32)
        check_attention(c, window=window)


@pytest.mark.parametrize("compiled", [True, False])
def test_pools_of_one_head_in_any_shape(compiled, monkeypatch):
    if not compiled:
        monkeypatch.setattr(L.binding, "_call", None)
    for layout in ("head", "token"):
        with Cache([(5, 40), (1, 20)], hq=4, hkv=1, layout=layout, seed=72) as c:
            q = c.randn(c.T, c.hq, D).cuda()
            outs = []
            for shape in ("as it is", "other order", "other stride"):
                kp, vp = c.K.cuda(), c.V.cuda()      # with one head the memory is the same in both layouts
                if shape == "other order":
                    kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
                elif shape == "other stride":
                    kp, vp = (x.as_strided(x.shape, (x.stride(0), 8, D, 1)) for x in (kp, vp))
                outs.append(torch.empty_like(q))
                L.lvr_paged_attention(c.h, kp, vp, q, *c.batch(), outs[-1])
            assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_frequencies_of_many_turns_per_position(dtype):
    """Frequencies up to 1e300 radians per position at the farthest positions; angles reduced in whole numbers for the reference."""
    from fractions import Fraction
    bits, term, two_pi, k = 1400, 0, 0, 0
    for n, c in ((5, 16), (239, -4)):            # pi = 16 atan(1/5) - 4 atan(1/239)
        term, k = (c << bits) // n, 0
        while term not in (0, -1):
            two_pi += 2 * (-(term // (2 * k + 1)) if k % 2 else term // (2 * k + 1))
            term, k = term // (n * n), k + 1
    f = [10.0 ** (i / 4) * (-1) ** i for i in range(48)] + [1e6, 1e17, 2.0 ** 80, 3e300] * 4
    positions = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 10 ** 9 + 7, 12345]
    turns = [[float(Fraction(p * Fraction(x).numerator << bits, Fraction(x).denominator * two_pi) % 1) for x in f] for p in positions]
    angle = torch.tensor(turns, dtype=torch.float64)[:, None] * (2 * math.pi)
    with Cache([(8, 8)], dtype=dtype, rot_dim=128, inv_freq=f, seed=73) as c:
        k, q = c.randn(c.T, c.hkv, D), c.randn(c.T, c.hq, D)
        kp, vp = c.pools()
        qo = torch.empty_like(q).cuda()
        L.lvr_paged_append(c.h, kp, vp, k.cuda(), k.cuda(), *c.batch(), q=q.cuda(), q_out=qo, positions=torch.tensor(positions, dtype=torch.int32, device="cuda")[:, None])
        kr = c.from_pool(kp)[int(c.table[0, 0]), :, :8].transpose(0, 1)
        for x, got in ((k, kr), (q, qo.cpu())):
            u, w = x.double().split(64, dim=2)
            want = torch.cat([u * angle.cos() - w * angle.sin(), u * angle.sin() + w * angle.cos()], dim=2)
            size = (u.abs() + w.abs()).repeat(1, 1, 2)
            # as in check_append; the angle's 2^-31 of a turn are 0.05 of a step of 2^-24 radians
            assert ((got.double() - want).abs() <= HALF_STEP[dtype] * want.abs() + 12.05 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_in_chunks_token_by_token(dtype):
    """Every chunk's outputs against 64 bits over the rows that append left in the pages, each value within what its own row allows: zeros, a
    mean of the values and attention without the causal mask are all farther off."""
    n, hq, hkv, f = 700, 8, 2, freqs(128)
    with Cache([(n, n)], dtype=dtype, hq=hq, hkv=hkv, rot_dim=128, inv_freq=f, seed=74) as c:
        k, q = c.randn(n, hkv, D), c.randn(n, hq, D)
        v = (c.randn(n, hkv, D).float() + 0.5).to(c.dt)
        kp, vp = c.pools()
        table, at, got, rotated_q = c.table.cuda(), 0, [], []
        for m in (1, 130, 17, 300, 252):
            start = torch.tensor([0, m], dtype=torch.int32, device="cuda")
            length = torch.tensor([at + m], dtype=torch.int32, device="cuda")
            qo, out = (torch.empty(m, hq, D, dtype=c.dt, device="cuda") for _ in range(2))
            L.lvr_paged_append(c.h, kp, vp, k[at:at + m].cuda(), v[at:at + m].cuda(), start, length, table, q=q[at:at + m].cuda(), q_out=qo)
            L.lvr_paged_attention(c.h, kp, vp, qo, start, length, table, out)
            got.append(out.cpu().double())
            rotated_q.append(qo.cpu())
            at += m
        got, rotated_q = torch.cat(got), torch.cat(rotated_q)
        c.K, c.V = c.from_pool(kp), c.from_pool(vp)
        ref, tol = c.attention(rotated_q, 0)
        assert ((got - ref).abs() <= tol).all(), float(((got - ref).abs() - tol).max())
        # the bound tells wrong outputs apart in every row where they differ: the last rows see nearly all keys, the first row one
        Kc, Vc, _ = c.rows(0, n)
        Kc, Vc = Kc.repeat_interleave(hq // hkv, dim=0), Vc.repeat_interleave(hq // hkv, dim=0)
        s = torch.matmul(rotated_q.transpose(0, 1).double(), Kc.transpose(1, 2)) / math.sqrt(D)
        unmasked = torch.matmul(torch.softmax(s, dim=2), Vc).transpose(0, 1)
        mean = (Vc.cumsum(dim=1) / torch.arange(1, n + 1)[:, None]).transpose(0, 1)
        for wrong, rows in ((torch.zeros_like(ref), slice(0, n)), (unmasked, slice(0, n - 50)), (mean, slice(1, n))):
            assert ((wrong - ref).abs() > tol).any(dim=2)[rows].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype):
    """A key whose score is minus infinity has no weight; a token with no other key gives zeros (0 / 0 by the formula), single, in tiles and cut."""
    lens = [(1, 40), (70, 90), (1, 3000), (130, 2000)]
    with Cache(lens, dtype=dtype, seed=75) as c:
        kp, vp = c.pools()
        q = c.randn(c.T, c.hq, D).abs()
        start, length, table = c.batch()
        out = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
        L.lvr_paged_attention(c.h, torch.full_like(kp, -math.inf), vp, q.cuda(), start, length, table, out)
        assert (out == 0).all()
    with Cache(lens, dtype=dtype, seed=75) as c:
        q = c.randn(c.T, c.hq, D).abs() + 0.1
        c.K[:, :, 1::3, 5] = -math.inf                  # position 0 and others between are as they were
        kp, vp = c.pools()
        L.lvr_paged_attention(c.h, kp, vp, q.cuda(), *c.batch(), out)
        got, t0 = out.cpu().double(), 0
        for b, (t, n) in enumerate(lens):
            K, V, _ = c.rows(b, n)
            finite = torch.where(torch.isfinite(K), K, torch.zeros_like(K))
            hidden = torch.arange(n)[None] > torch.arange(n - t, n)[:, None]
            for h in range(c.hq):
                g, qh = h // (c.hq // c.hkv), q[t0:t0 + t, h].double()
                w = torch.softmax((qh @ K[g].T * c.scale).masked_fill(hidden, -math.inf), dim=1)
                ref = w @ V[g]
                # as in Cache.attention, the scores' size over all keys
                S = (qh @ finite[g].abs().T * c.scale).amax()
                weight = 2 * (136 * 2.0 ** -24 * S + 2.0 ** -21) + (1.02 * HALF_STEP[dtype] if dtype == "bf16" else 0)
                tol = (weight + (n + 64) * 2.0 ** -24) * (w @ V[g].abs() + ref.abs()) + HALF_STEP[dtype] * ref.abs()
                assert ((got[t0:t0 + t, h] - ref).abs() <= tol).all()
            t0 += t
