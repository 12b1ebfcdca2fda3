"""Timed operators of the paged cache beyond the plain ones: pages that hold keys and values in 4 bits (written by an append, read by
the attention and by the gather that lays out rows for the index), attention with a sliding window and first tokens that stay visible, and
norms of queries and keys per head in the pass that rotates and stores them.

Head counts and lengths follow ``perf/operators.py`` and the benchmark (32 or 64 query heads on 8 KV heads, head_dim 128, 1 to 131072 keys);
batches are ragged, pages are scattered over the pool as a serving program leaves them.

``run`` computes the operators from elementary torch operations in 32 bits (angles, and what is rounded to 4 bits, in 64), or, where ``own`` is
true, calls the library.  ``exact`` follows the definitions in 64 bits, sequence by sequence.

Pages in 4 bits: a page is n_kv_heads * page_size rows of 64 bytes (coordinate 2 i of a row in the low half of byte i, 2 i + 1 in the high half),
then as many groups of 4 bytes, in the same order: the scales of a row's four blocks of 32 coordinates.  A code is a sign and one of 0, 0.5, 1,
1.5, 2, 3, 4, 6; scale byte s stands for 2^(s - 127), 255 for no number.
"""
import math
import random

import torch

own = False

D = 128
EPS = 1e-6
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, kind, *, seqs=1, tokens=1, n=4096, mix="even", hq=32, hkv=8, dtype="bf16", page=16, layout="head", window=0, sinks=0,
          rot=128, axes=1, pairs="halves", query=True, norm=True, pick=1):
    """kind: "attention", "append" (bf16 and f32 pages) or "store" (an append to pages in 4 bits, and the sequences read back).  `seqs` sequences
    hold up to n keys each and bring up to `tokens` new ones: mix "even" (all the same), "ragged" (both lengths vary, a few tokens to the
    most), "chunk" (the first sequence brings all `tokens`, the others one each: a serving step with one prompt in it).  pick: which ragged
    lengths.  dtype: of the pages, "fp4" takes and gives bf16."""
    case = dict(kind=kind, seqs=seqs, tokens=tokens, n=n, mix=mix, hq=hq, hkv=hkv, dtype=dtype, page=page, layout=layout, window=window,
                sinks=sinks, rot=rot, axes=axes, pairs=pairs, query=query, norm=norm, pick=pick)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one sequence decodes one token at 2k of context: the latency of a call
        _case("attn4_1x2k", "attention", n=2048, dtype="fp4"),
        # the benchmark's headline context, one token
        _case("attn4_1x128k", "attention", n=131072, page=64, dtype="fp4"),
        # a serving batch decodes, every sequence as long as it happens to be
        _case("attn4_48_ragged", "attention", seqs=48, n=32768, mix="ragged", dtype="fp4", pick=3),
        # a serving step: a piece of one prompt beside sequences that decode
        _case("attn4_chunk_beside_31", "attention", seqs=32, tokens=1000, n=12000, mix="chunk", page=32, layout="token", dtype="fp4", pick=5),
        # the prompt of the long-output workload in one chunk
        _case("attn4_prompt_16k", "attention", tokens=16384, n=16384, page=64, dtype="fp4"),
        # long conversations decode with a window and a few first tokens: the cost no longer grows with the length
        _case("sinks_24_ragged", "attention", seqs=24, n=100000, mix="ragged", page=64, window=4096, sinks=4, pick=8),
        # a long prompt with a window, over pages in 4 bits
        _case("sinks4_prompt_8k", "attention", tokens=8192, n=8192, page=32, dtype="fp4", window=2048, sinks=16),
        # an fp32 cache, ragged chunks whose first tokens' range ends inside a page and a tile
        _case("sinks_f32_chunks", "attention", seqs=3, tokens=600, n=9001, mix="ragged", dtype="f32", hq=24, window=1024, sinks=70, pick=2),
        # one token of one sequence into the cache: latency
        _case("norm_1", "append", n=2000),
        # a piece of a prompt with images in it: positions on three axes
        _case("norm_8k_3axes", "append", tokens=8192, n=20001, axes=3, page=64, layout="token"),
        # ragged pieces of prompts into pages in 4 bits, and the rows for the index
        _case("store4_5_ragged", "store", seqs=5, tokens=300, n=2000, mix="ragged", hq=64, dtype="fp4", rot=64, pairs="neighbours", pick=6),
        # the end of a prefill: its last piece goes in, all of it comes out
        _case("store4_8k", "store", tokens=8192, n=32768, page=64, dtype="fp4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "attention", "append", "store"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (16, 8), (8, 8), (8, 2), (8, 1), (24, 8), (12, 4), (40, 8)])
    c = dict(hq=hq, hkv=hkv, page=rng.choice([16, 16, 32, 64, 128]), layout=rng.choice(["head", "token"]), pick=rng.randrange(1 << 16),
             mix=rng.choice(["even", "ragged"]))
    if kind != "attention":
        c.update(rot=rng.choice([128, 128, 64, 96, 32]), axes=rng.choice([1, 1, 2, 3]), pairs=rng.choice(["halves", "halves", "neighbours"]),
                 query=rng.random() < 0.8)
        seqs = _log(rng, 1, 64 if kind == "append" else 8)
        tokens = rng.choice([1, _log(rng, 1, 8192 // seqs)])
        if kind == "append":
            return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + _log(rng, 1, 131072 // seqs), dtype=rng.choice(["bf16", "bf16", "f32"]), **c)
        return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + _log(rng, 1, 24000 // seqs), dtype="fp4", norm=rng.random() < 0.7, **c)
    dtype = rng.choice(["fp4", "fp4", "fp4", "fp4", "bf16", "f32"])
    if dtype == "fp4" and rng.random() < 0.6:
        window = sinks = 0
    else:
        window, sinks = _log(rng, 16, 8192), rng.choice([1, 4, 4, 64, _log(rng, 1, 1000)])
    c.update(dtype=dtype, window=window, sinks=sinks)
    what = rng.choice(["decode", "decode", "chunk", "prompts", "few"])
    if what == "decode":
        seqs = rng.choice([1, _log(rng, 1, 48)])
        return _case(None, kind, seqs=seqs, n=_log(rng, 64, min(131072, 524288 // seqs)), **c)
    if what == "few":        # a few tokens a sequence: drafts to be checked
        seqs, tokens = _log(rng, 1, 16), rng.randint(2, 16)
        return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + _log(rng, 64, 65536 // seqs), **c)
    if what == "chunk":
        tokens = _log(rng, 32, 2048)
        return _case(None, kind, seqs=rng.randint(2, 32), tokens=tokens, n=tokens + _log(rng, 64, 8192), **dict(c, mix="chunk"))
    seqs = _log(rng, 1, 8)
    tokens = _log(rng, 16, (2048 if dtype == "f32" else 4096) // seqs)
    return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + rng.choice([0, _log(rng, 1, 8192)]), **c)


# ------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """New tokens and keys held (the new ones among them) of every sequence."""
    r = random.Random(case["pick"])
    new, held = [], []
    for b in range(case["seqs"]):
        t, n = case["tokens"], case["n"]
        if case["mix"] == "ragged":
            t = _log(r, max(1, t // 16), t) if b else t
            n = max(t, _log(r, max(1, n // 64), n) if b else n)
        elif case["mix"] == "chunk":
            t = t if b == 0 else 1
            n = n if b == 0 else max(t, _log(r, max(1, n // 64), n))
        new.append(t)
        held.append(max(n, t))
    return new, held


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _inv_freq(case):
    """Rotations per position in radians, one for each pair."""
    half = case["rot"] // 2
    return [10000.0 ** (-c / half) for c in range(half)]


def _axis(case):
    """Which axis turns a pair: runs of pairs, a quarter (of three axes) or half (of two) for the first."""
    half, axes = case["rot"] // 2, case["axes"]
    if axes == 1:
        return [0] * half
    first = half // 4 if axes == 3 else half // 2
    return [0 if c < first else 1 + (c - first) * (axes - 1) // (half - first) for c in range(half)]


class _Paged:
    """The library's handle and its lifetime."""

    def __init__(self, case, n_pages):
        import paper_2605_06763_amd as L
        self.L = L
        cfg = L.make_paged_config(
            n_q_heads=case["hq"], n_kv_heads=case["hkv"], kv_dtype={"bf16": L.LVR_BF16, "f32": L.LVR_F32, "fp4": L.LVR_FP4}[case["dtype"]],
            page_size=case["page"], n_pages=n_pages, layout=case["layout"], rot_dim=case["rot"], rot_axes=case["axes"],
            rot_pairs=L.LVR_ROT_HALVES if case["pairs"] == "halves" else L.LVR_ROT_NEIGHBOURS)
        self.handle = L.lvr_paged_create(cfg, inv_freq=_inv_freq(case), axis=_axis(case))

    def __del__(self):
        if getattr(self, "handle", None):
            self.L.lvr_paged_destroy(self.handle)


def _power_of_two(e, dtype):
    """2^e of whole numbers e, exactly."""
    return ((e + 1023).long() << 52).view(torch.float64) if dtype == torch.float64 else ((e + 127).int() << 23).view(torch.float32)


def _to_codes(x):
    """x [..., 128] as codes [..., 64] and scales [..., 4], bytes: every block's scale the least power of two that leaves its largest magnitude at
    7 or below, values to the nearest code, ties to the even one.  In the type of x."""
    blocks = x.unflatten(-1, (4, 32))
    m, e = torch.frexp(blocks.abs().amax(dim=-1))
    e = (e - 3 + (m > 0.875)).clamp(-120, 125)
    e[m == 0] = -120
    t = blocks * _power_of_two(-e, x.dtype)[..., None]
    y = t.abs().clamp_max(6)
    half, one, two = (y * 2).round(), y.round(), (y / 2).round()
    code = torch.where(y < 2, half, torch.where(y < 4, one + 2, two + 4)).to(torch.uint8)
    code = (code | (torch.signbit(t).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _views(case, pool):
    """Codes [page][head][token][64] and scales [page][head][token][4] in a pool of pages in 4 bits."""
    hkv, page = case["hkv"], case["page"]
    shape = (-1, hkv, page) if case["layout"] == "head" else (-1, page, hkv)
    codes, scales = pool[:, :hkv * page * 64].unflatten(1, shape[1:] + (64,)), pool[:, hkv * page * 64:].unflatten(1, shape[1:] + (4,))
    return (codes, scales) if case["layout"] == "head" else (codes.transpose(1, 2), scales.transpose(1, 2))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    r = random.Random(int(seed) * 31 + 11)
    new, held = _lengths(case)
    hq, hkv, page, kind, dt = case["hq"], case["hkv"], case["page"], case["kind"], _type(case)
    T = sum(new)
    used = [-(-n // page) for n in held]
    width, n_pages = max(used) + 1, sum(used) + 3
    order = list(range(n_pages))
    r.shuffle(order)                      # pages lie wherever they were free
    table, at = [], 0
    for u in used:
        table.append(order[at:at + u] + [-1] * (width - u))
        at += u
    start = [0]
    for t in new:
        start.append(start[-1] + t)
    shape = (hkv, page, D) if case["layout"] == "head" else (page, hkv, D)

    def pool(scale):                      # [page][head][token][coordinate] in either order of memory
        step = max(1, (1 << 26) // (hkv * page * D))
        p = torch.empty((n_pages,) + ((hkv * page * 68,) if case["dtype"] == "fp4" else shape), device="cuda", dtype=torch.uint8 if case["dtype"] == "fp4" else dt)
        for i in range(0, n_pages, step):
            x = torch.randn((min(step, n_pages - i),) + shape, generator=g, device="cuda")
            if scale is not None:
                x *= scale[:, None] if case["layout"] == "head" else scale
            if case["dtype"] == "fp4":
                codes, scales = _to_codes(x)
                p[i:i + step, :hkv * page * 64] = codes.flatten(1)
                p[i:i + step, hkv * page * 64:] = scales.flatten(1)
            else:
                p[i:i + step] = x
        return p

    # keys whose channels differ in size, as a model's do
    channels = torch.exp(0.4 * torch.randn((hkv, D), generator=g, device="cuda"))
    state = {"case": case, "k_pages": pool(channels), "v_pages": pool(None),
             "table": torch.tensor(table, dtype=torch.int32, device="cuda"),
             "seq_start": torch.tensor(start, dtype=torch.int32, device="cuda"),
             "seq_len": torch.tensor(held, dtype=torch.int32, device="cuda"), "new": new, "held": held}
    if kind == "attention":
        state["q"] = torch.randn((T, hq, D), generator=g, device="cuda").to(dt)
        state["out"] = torch.empty_like(state["q"])
    else:
        fused = torch.randn((T, (hq + 2 * hkv) * D), generator=g, device="cuda").to(dt)   # as one projection writes q, k and v
        state["q"] = fused[:, :hq * D].view(T, hq, D)
        state["k"] = fused[:, hq * D:(hq + hkv) * D].view(T, hkv, D)
        state["v"] = fused[:, (hq + hkv) * D:].view(T, hkv, D)
        state["q_out"] = torch.empty((T, hq, D), device="cuda", dtype=dt) if case["query"] else None
        for name in ("q_weight", "k_weight"):
            state[name] = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt)
        at = torch.cat([torch.arange(n - t, n) for t, n in zip(new, held)])
        pos = torch.stack([at, at // 37 % 411, at % 37 * 3][:case["axes"]], dim=1)        # time, and rows and columns of an image
        state["positions"] = pos.to(torch.int32).cuda().contiguous()
        state["inv_freq"] = torch.tensor(_inv_freq(case), dtype=torch.float64, device="cuda")
        state["axis"] = torch.tensor(_axis(case), device="cuda")
    if kind == "store":
        state["K"] = torch.zeros((case["seqs"], hkv, max(held), D), device="cuda", dtype=dt)   # rows past a sequence's end stay as they are
        state["V"] = torch.zeros_like(state["K"])
    if case["dtype"] == "fp4":
        state["levels"] = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device="cuda")
    if own:
        state["paged"] = _Paged(case, n_pages)
    return state


# ------------------------------------------------------------------------------------------------ the plain forms
def _heads_first(case, pages):
    return pages if case["layout"] == "head" else pages.transpose(1, 2)


def _rows(state, name, table, keys):
    """The rows of the given sequences at positions keys [seq][m]: [seq][head][m][D]; 4-bit pages as 32-bit values."""
    case = state["case"]
    page = table.long().gather(1, keys // case["page"]).clamp_min(0)
    at = keys % case["page"]
    if case["dtype"] != "fp4":
        return _heads_first(case, state[name])[page, :, at].transpose(1, 2)
    codes, scales = _views(case, state[name])
    c = codes[page, :, at]
    values = state["levels"][torch.stack([c & 15, c >> 4], dim=-1).flatten(-2).int()]
    scale = _power_of_two(scales[page, :, at].int() - 127, torch.float32)
    return (values.unflatten(-1, (4, 32)) * scale[..., None]).flatten(-2).transpose(1, 2)


def _attend(q, K, V, sees):
    """q [seq][tokens][hq][D] over K, V [seq][hkv][m][D] in 32 bits; sees [seq][tokens][m]."""
    s, t, hq, _ = q.shape
    hkv, n = K.shape[1], K.shape[2]
    q = (q.float() / math.sqrt(D)).reshape(s, t, hkv, hq // hkv, D).permute(0, 2, 1, 3, 4).reshape(s, hkv, -1, D)
    x = torch.matmul(q, K.float().transpose(2, 3).contiguous()).view(s, hkv, t, hq // hkv, n)
    x.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    x.sub_(x.amax(dim=-1, keepdim=True)).exp_()
    den = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(s, hkv, -1, n), V.float().contiguous()).view(s, hkv, t, hq // hkv, D) / den
    return o.permute(0, 2, 1, 3, 4).reshape(s, t, hq, D)


def _attention(state):
    case, new, held, dt = state["case"], state["new"], state["held"], _type(state["case"])
    window, sinks = case["window"], case["sinks"]

    def piece(b0, b1, tokens, n):
        table, length = state["table"][b0:b1], state["seq_len"][b0:b1].long()
        q = state["q"][sum(new[:b0]):sum(new[:b1])].view(b1 - b0, tokens, case["hq"], D)
        if window and window + tokens - 1 + sinks < n:     # the first keys, and those that some window reaches
            last = length[:, None] - (window + tokens - 1) + torch.arange(window + tokens - 1, device="cuda")
            keys = torch.cat([torch.arange(sinks, device="cuda").expand(b1 - b0, sinks), torch.where(last < sinks, -1, last)], dim=1)
        else:
            keys = torch.arange(n, device="cuda").expand(b1 - b0, n)
        p = (length[:, None] - tokens + torch.arange(tokens, device="cuda"))[:, :, None]
        j = keys[:, None, :]
        sees = (j >= 0) & (j <= p) & ((j > p - window) | (j < sinks)) if window else (j >= 0) & (j <= p)
        at = torch.minimum(keys.clamp_min(0), length[:, None] - 1)
        return _attend(q, _rows(state, "k_pages", table, at), _rows(state, "v_pages", table, at), sees).to(dt).view(-1, case["hq"], D)

    if len(set(new)) == 1:                # one batch, shorter sequences masked
        return piece(0, case["seqs"], new[0], max(held))
    return torch.cat([piece(b, b + 1, new[b], held[b]) for b in range(case["seqs"])])


def _normed(case, x, weight):
    """Rows divided by their root mean square and weighted, in the type of x."""
    return x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * weight.to(x.dtype) if case["norm"] else x


def _rotate(case, y, cos, sin):
    """y [T][heads][D], cos and sin [T][1][rot / 2], in the type of y."""
    rot, y, cos, sin = case["rot"], y.clone(), cos.to(y.dtype), sin.to(y.dtype)
    if case["pairs"] == "halves":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    u, w = a * cos - b * sin, a * sin + b * cos
    a.copy_(u)
    b.copy_(w)
    return y


def _append(state):
    case, start, length, page = state["case"], state["seq_start"].long(), state["seq_len"].long(), state["case"]["page"]
    t = torch.arange(state["k"].shape[0], device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), t, right=True)
    slot = length[b] - start[b + 1] + t
    to = state["table"][b, slot // page].long()
    angle = state["positions"].double()[:, state["axis"]] * state["inv_freq"]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    result = {}
    if case["query"]:
        result["q"] = _rotate(case, _normed(case, state["q"].float(), state["q_weight"]), cos, sin).to(state["q"].dtype)
    if case["dtype"] == "fp4":            # a value beside the border between two codes: in 64 bits
        for name, x in (("k_pages", _rotate(case, _normed(case, state["k"].double(), state["k_weight"]), cos, sin)), ("v_pages", state["v"].double())):
            codes, scales = _views(case, state[name])
            codes[to, :, slot % page], scales[to, :, slot % page] = _to_codes(x)
        return result
    k = _rotate(case, _normed(case, state["k"].float(), state["k_weight"]), cos, sin).to(state["k"].dtype)
    _heads_first(case, state["k_pages"])[to, :, slot % page] = k
    _heads_first(case, state["v_pages"])[to, :, slot % page] = state["v"]
    return dict(result, k_pages=state["k_pages"], v_pages=state["v_pages"])


def _store(state):
    case, n = state["case"], state["K"].shape[2]
    result = _append(state)
    keys = torch.arange(n, device="cuda").expand(case["seqs"], n)
    at = torch.minimum(keys, state["seq_len"][:, None].long() - 1)
    past = (keys >= state["seq_len"][:, None])[:, None, :, None]
    for rows, pages in (("K", "k_pages"), ("V", "v_pages")):
        result[rows] = torch.where(past, state[rows], _rows(state, pages, state["table"], at).to(state[rows].dtype))
    return result


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        return {"out": _attention(state)} if kind == "attention" else _append(state) if kind == "append" else _store(state)
    import paper_2605_06763_amd as L
    h = state["paged"].handle
    if kind == "attention":
        if case["window"]:
            L.lvr_paged_sink_attention(h, state["k_pages"], state["v_pages"], state["q"], state["seq_start"], state["seq_len"],
                                       state["table"], state["out"], case["window"], case["sinks"])
        else:
            L.lvr_paged_attention(h, state["k_pages"], state["v_pages"], state["q"], state["seq_start"], state["seq_len"],
                                  state["table"], state["out"])
        return {"out": state["out"]}
    q = state["q"] if case["query"] else None
    if case["norm"]:
        L.lvr_paged_norm_append(h, state["k_pages"], state["v_pages"], state["k"], state["v"], state["seq_start"], state["seq_len"],
                                state["table"], q=q, q_out=state["q_out"], q_weight=state["q_weight"] if case["query"] else None,
                                k_weight=state["k_weight"], eps=EPS, positions=state["positions"])
    else:
        L.lvr_paged_append(h, state["k_pages"], state["v_pages"], state["k"], state["v"], state["seq_start"], state["seq_len"],
                           state["table"], q=q, q_out=state["q_out"], positions=state["positions"])
    result = {"q": state["q_out"]} if case["query"] else {}
    if kind == "append":
        return dict(result, k_pages=state["k_pages"], v_pages=state["v_pages"])
    L.lvr_paged_gather(h, state["k_pages"], state["v_pages"], state["seq_len"], state["table"], state["K"], state["V"])
    return dict(result, K=state["K"], V=state["V"])


# ------------------------------------------------------------------------------------------------ work, exactness
def work(case):
    """Bytes: every key and value row that some new token sees once, queries, outputs, new rows and rows written once each (68 bytes a row in 4
    bits).  Flops: two products of 128 per visible (query row, key), six per rotated pair, four per normed value."""
    new, held = _lengths(case)
    row, wide = {"fp4": 68, "bf16": 256, "f32": 512}[case["dtype"]], D * (4 if case["dtype"] == "f32" else 2)
    T, hq, hkv, w, s = sum(new), case["hq"], case["hkv"], case["window"], case["sinks"]
    if case["kind"] != "attention":
        q = hq if case["query"] else 0
        moved = T * (2 * hkv + 2 * q) * wide + T * 2 * hkv * row + 4 * T * case["axes"]
        flops = T * (hkv + q) * (3 * case["rot"] + (4 * D if case["norm"] else 0))
        if case["kind"] == "store":
            moved += 2 * sum(held) * hkv * (row + wide)
        return {"bytes": float(moved), "flops": float(flops)}
    keys = seen = 0
    for t, n in zip(new, held):
        some = min(n, w + t - 1) if w else n
        keys += min(n, some + s) if w else n
        first = n - t + 1                 # keys the first new token sees without a window
        seen += sum(min(w, x) + min(s, max(0, x - w)) for x in range(first, n + 1)) if w else (first + n) * t / 2
    return {"bytes": 2.0 * keys * hkv * row + 2.0 * T * hq * wide, "flops": 4.0 * D * hq * seen}


def _values(case, pool, ids, h, n):
    """Rows 0 .. n - 1 of one head of the sequence whose pages are `ids`, in 64 bits."""
    if case["dtype"] != "fp4":
        return (pool if case["layout"] == "head" else pool.transpose(1, 2))[ids, h].reshape(-1, D)[:n].double()
    hkv, page = case["hkv"], case["page"]
    slot = torch.arange(page, device="cuda")
    row = h * page + slot if case["layout"] == "head" else slot * hkv + h
    mine = pool[ids]
    byte = mine[:, (row[:, None] * 64 + torch.arange(64, device="cuda")).flatten()].view(-1, 64)[:n].long()
    scale = mine[:, (hkv * page * 64 + row[:, None] * 4 + torch.arange(4, device="cuda")).flatten()].view(-1, 4)[:n].long()
    code = torch.empty((n, D), dtype=torch.long, device="cuda")
    code[:, 0::2], code[:, 1::2] = byte % 16, byte // 16
    exponent, fraction = code % 8 // 2, code % 2          # one bit of fraction, exponent 0 without the leading one
    size = torch.where(exponent == 0, 0.5 * fraction, (1 + 0.5 * fraction) * 2.0 ** (exponent - 1).double())
    return torch.where(code >= 8, -size, size) * 2.0 ** (scale - 127).double().repeat_interleave(32, dim=1)


def _nearest(x):
    """What 4 bits keep of x [..., 128] (64 bits), by counting the borders below a value."""
    b = x.reshape(x.shape[:-1] + (4, 32))
    top = b.abs().amax(dim=-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 7))
    e = torch.where(top > 7 * 2.0 ** e, e + 1, torch.where(top <= 7 * 2.0 ** (e - 1), e - 1, e)).clamp(-120, 125)
    t = b.abs() / 2.0 ** e
    even = (t > 0.25).int() + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5)
    size = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)[even.long()]
    return (torch.copysign(size, b) * 2.0 ** e).reshape(x.shape)


def exact(case, seed):
    state = prepare(case, seed)
    new, held, page, hkv = state["new"], state["held"], case["page"], case["hkv"]
    G, kind = case["hq"] // hkv, case["kind"]
    table = state["table"].tolist()
    if kind == "attention":
        out = torch.empty((sum(new), case["hq"], D), dtype=torch.float64, device="cuda")
        t0 = 0
        for b, (t, n) in enumerate(zip(new, held)):
            ids = torch.tensor(table[b][:-(-n // page)], device="cuda")
            far = torch.arange(n - t, n, device="cuda")[:, None] - torch.arange(n, device="cuda")     # how far back a key lies
            sees = far >= 0
            if case["window"]:
                sees &= (far < case["window"]) | (torch.arange(n, device="cuda") < case["sinks"])
            for h in range(hkv):
                K, V = (_values(case, state[p], ids, h, n) for p in ("k_pages", "v_pages"))
                for g in range(h * G, h * G + G):
                    s = (state["q"][t0:t0 + t, g].double() @ K.t().contiguous()) * D ** -0.5
                    s = torch.where(sees, s, torch.full_like(s, -math.inf))
                    out[t0:t0 + t, g] = torch.exp(s - torch.logsumexp(s, dim=1, keepdim=True)) @ V
            t0 += t
        return {"out": out}
    # rotation as a product of complex numbers
    turn = torch.exp(1j * (state["positions"].double()[:, state["axis"]] * state["inv_freq"]))[:, None]
    half, rot = case["rot"] // 2, case["rot"]

    def turned(x, weight):
        x = x.double()
        if case["norm"]:
            x = x / ((x * x).sum(dim=-1, keepdim=True) / D + EPS).sqrt() * weight.double()
        first, second = (x[..., :half], x[..., half:rot]) if case["pairs"] == "halves" else (x[..., 0:rot:2], x[..., 1:rot:2])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        parts = [z.real, z.imag] if case["pairs"] == "halves" else [torch.stack([z.real, z.imag], dim=-1).flatten(-2)]
        return torch.cat(parts + [x[..., rot:]], dim=-1)

    result = {"q": turned(state["q"], state["q_weight"])} if case["query"] else {}
    k, v = turned(state["k"], state["k_weight"]), state["v"].double()
    if kind == "store":
        k, v, t0 = _nearest(k), _nearest(v), 0
        result.update(K=state["K"].double(), V=state["V"].double())
        for b, (t, n) in enumerate(zip(new, held)):
            ids = torch.tensor(table[b][:-(-n // page)], device="cuda")
            for rows, pages, x in (("K", "k_pages", k), ("V", "v_pages", v)):
                for h in range(hkv):
                    result[rows][b, h, :n] = _values(case, state[pages], ids, h, n)
                result[rows][b, :, n - t:n] = x[t0:t0 + t].transpose(0, 1)
            t0 += t
        return result
    result.update(k_pages=state["k_pages"].double(), v_pages=state["v_pages"].double())
    rows = [(table[b][p // page], p % page) for b, (t, n) in enumerate(zip(new, held)) for p in range(n - t, n)]
    ids, at = (torch.tensor(x, device="cuda") for x in zip(*rows))
    head = (lambda p: p) if case["layout"] == "head" else (lambda p: p.transpose(1, 2))
    head(result["k_pages"])[ids, :, at] = k
    head(result["v_pages"])[ids, :, at] = v
    return result
