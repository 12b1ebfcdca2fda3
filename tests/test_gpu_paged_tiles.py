"""The attention over pages in tiles of 16 rows, on the GPU, where the tiles of a sequence read the same long runs of keys and where they do not: against the
definition in 64 bits, with tolerances counted as in test_gpu_paged.py."""
import math

import pytest
import torch

import paper_2605_06763_amd as L
from test_gpu_paged import HALF_STEP, say
from test_gpu_paged_more import D, More

pytestmark = pytest.mark.gpu

# 32 KV heads leave eight pieces of a launch to each: two tiles (of 18 rows) go into four runs of 1088 keys.
LENS = {
    "two_tiles": [(18, 4333)],                   # long runs, a workgroup to a compute unit
    "four_tiles": [(50, 9000)],
    "three_tiles": [(40, 4333)],                 # three runs each: more workgroups than that
    "two_short_tiles": [(18, 700)],
    "beside_a_chunk": [(18, 4333), (70, 300)],   # tiles of 128 rows in the same launch
    "one_tile": [(1, 4333)],
}


def definition(c, q, window, sinks):
    """Outputs in 64 bits and how far off the kernel's may be: that of a weight twice the error of its score (128 products and sums of 2^-24 each, as many in
    the scaling) and two roundings of the exponential, for bf16 its own rounding; sums of as many terms as keys are seen; the last rounding."""
    out, tol = (torch.empty(c.T, c.hq, D, dtype=torch.float64) for _ in range(2))
    step = HALF_STEP[c.dtype]
    for b, (t, n) in enumerate(c.lens):
        rows = slice(int(c.start[b]), int(c.start[b]) + t)
        K, V, held = c.rows(b, n)
        p, j = torch.arange(n - t, n)[:, None], torch.arange(n)[None]
        sees = (j <= p) & held & ((j > p - window) | (j < sinks) if window else True)
        for h in range(c.hq):
            odd = ~torch.isfinite(V[h]).all(dim=1)
            Kh, Vh, qh = K[h].nan_to_num(0), V[h].nan_to_num(0, 0, 0), q[rows, h].double()
            x = torch.where(sees, qh @ Kh.T * c.scale, torch.tensor(-math.inf, dtype=torch.float64))
            w = torch.softmax(x, dim=1)
            o, size = w @ Vh, w @ Vh.abs()
            S = torch.where(sees, qh.abs() @ Kh.abs().T * c.scale, torch.zeros(1, dtype=torch.float64)).amax(dim=1, keepdim=True)
            weight = 2 * (136 * 2.0 ** -24 * S + 2.0 ** -21) + (1.02 * step if c.dtype == "bf16" else 0)
            tol[rows, h] = (weight + (sees.sum(dim=1, keepdim=True) + 64) * 2.0 ** -24) * (size + o.abs()) + step * o.abs()
            out[rows, h] = torch.where((sees & odd).any(dim=1, keepdim=True), torch.tensor(math.nan, dtype=torch.float64), o)
    return out, tol


def check(c, q, window, sinks, note=""):
    say(f"tiles {note} lens={c.lens} {c.dtype} heads={c.hq}/{c.hkv} window={window} sinks={sinks}")
    out = torch.full((c.T, c.hq, D), 7.0, dtype=c.dt, device="cuda")
    L.lvr_paged_sink_attention(c.h, *c.pools(), q.cuda(), *c.batch(), out, window, sinks)
    torch.cuda.synchronize()
    out = out.cpu().double()
    ref, tol = definition(c, q, window, sinks)
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    assert ((out - ref).abs() <= tol)[torch.isfinite(ref)].all()
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window, sinks", [(0, 0), (4000, 70)])
@pytest.mark.parametrize("lens", LENS)
def test_tiles_that_read_the_same_runs(lens, window, sinks, dtype):
    with More(LENS[lens], dtype=dtype, hq=32, hkv=32, page=64, seed=170) as c:
        q = c.randn(c.T, c.hq, D)
        first = check(c, q, window, sinks)
        # no numbers where the last two tokens of the first sequence see them alone, and where nobody does
        t, n = c.lens[0]
        bad = torch.zeros(c.n_pages, c.page, dtype=torch.bool)
        for b, (_, m) in enumerate(c.lens):
            bad[c.table[b, m // c.page], m % c.page:] = True
        c.hide("K", bad)
        c.hide("V", bad)
        assert torch.equal(check(c, q, window, sinks, note="unseen"), first)
        if t > 2:
            bad[c.table[0, (n - 2) // c.page], (n - 2) % c.page] = True
            c.hide("V", bad)
            out = check(c, q, window, sinks, note="seen by some")
            assert torch.isfinite(out[:t - 2]).all() and torch.isnan(out[t - 2:t]).any(dim=2).all()
        c.table[0, 1] = -1
        check(c, q, window, sinks, note="no page")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tiles_give_the_same_bits_every_time(dtype):
    """Eager calls and replays of a captured one."""
    with More([(18, 4333)], dtype=dtype, hq=32, hkv=32, page=64, seed=171) as c:
        q, pools, batch = c.randn(c.T, c.hq, D).cuda(), c.pools(), c.batch()
        want, out = torch.empty_like(q), torch.empty_like(q)
        L.lvr_paged_attention(c.h, *pools, q, *batch, want)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            L.lvr_paged_attention(c.h, *pools, q, *batch, out)
        for replay in (True, False, True, True):
            out.fill_(math.nan)
            torch.cuda.synchronize()
            graph.replay() if replay else L.lvr_paged_attention(c.h, *pools, q, *batch, out)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
