"""Timed operators: the way of a prompt into a paged KV cache, through the attention, and out of the pages into the index.

``lvr_paged_append`` stores the keys and values of new tokens in pages and rotates keys and queries by their positions on
the way, ``lvr_paged_attention`` attends a chunk of new tokens (or a single one) over the pages, ``lvr_paged_gather`` lays the
pages' rows out as ``lvr_build`` reads them.  Head counts follow ``workloads/`` and the benchmark (32 or 64 query heads on 8 KV
heads, head_dim 128, 1 to 131072 keys); batches are ragged, pages are scattered over the pool as a serving program leaves them.

``run`` computes the operators from elementary torch operations in 32 bits (angles in 64), or, where ``own`` is true, calls the
library.  ``exact`` follows the definitions in 64 bits, sequence by sequence.
"""
import math
import random

import torch

own = False

D = 128


def _case(name, kind, *, seqs=1, tokens=1, n=4096, mix="even", hq=32, hkv=8, dtype="bf16", page=16, layout="head", window=0,
          rot=128, axes=1, pairs="halves", query=True, pick=1):
    """kind: "append", "attention" or "gather".  `seqs` sequences hold up to n keys each and bring up to `tokens` new ones:
    mix "even" (all the same), "ragged" (both lengths vary, a few tokens to the most), "chunk" (the first sequence brings all
    `tokens`, the others one each: a serving step with one prompt in it).  pick: which ragged lengths."""
    case = dict(kind=kind, seqs=seqs, tokens=tokens, n=n, mix=mix, hq=hq, hkv=hkv, dtype=dtype, page=page, layout=layout,
                window=window, rot=rot, axes=axes, pairs=pairs, query=query, pick=pick)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one sequence decodes one token at 2k of context: the latency of a call
        _case("attn_1x2k", "attention", n=2048, page=16),
        # the benchmark's headline context, one token
        _case("attn_1x128k", "attention", n=131072, page=64),
        # a serving batch decodes, every sequence as long as it happens to be
        _case("attn_48_ragged", "attention", seqs=48, n=32768, mix="ragged", page=16, pick=3),
        # a serving step: a piece of one prompt beside sequences that decode
        _case("attn_chunk_beside_31", "attention", seqs=32, tokens=1000, n=12000, mix="chunk", page=32, layout="token", pick=5),
        # the prompt of the long-output workload in one chunk
        _case("attn_prompt_16k", "attention", tokens=16384, n=16384, page=64),
        # an fp32 cache, a sliding window, ragged chunks that meet pages in their middle
        _case("attn_f32_window", "attention", seqs=3, tokens=700, n=9001, mix="ragged", dtype="f32", hq=24, window=1500, pick=2),
        # one token of one sequence into the cache: latency
        _case("append_1", "append", n=2000, page=16),
        # one token of each sequence of a serving batch
        _case("append_64", "append", seqs=64, n=32768, mix="ragged", tokens=1, page=16, pick=4),
        # a piece of a prompt with images in it: positions on three axes
        _case("append_8k_3axes", "append", tokens=8192, n=20001, axes=3, page=64, layout="token"),
        # an fp32 cache, neighbouring coordinates rotated together, half of a head left as it is
        _case("append_f32_ragged", "append", seqs=5, tokens=900, n=5000, mix="ragged", dtype="f32", hq=64, rot=64,
              pairs="neighbours", pick=6),
        # the end of a prefill: the pages become the rows an index is built from
        _case("gather_128k", "gather", n=131072, page=64),
        # a batch of shorter prompts in small pages
        _case("gather_8_ragged", "gather", seqs=8, n=3001, mix="ragged", page=16, layout="token", pick=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "append", "append", "gather"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (64, 8), (16, 8), (8, 8), (8, 2), (8, 1), (24, 8), (12, 4), (40, 8)])
    c = dict(hq=hq, hkv=hkv, page=rng.choice([16, 16, 32, 64, 128]), layout=rng.choice(["head", "token"]),
             dtype="f32" if rng.random() < 0.25 else "bf16", pick=rng.randrange(1 << 16), mix=rng.choice(["even", "ragged"]))
    if kind == "gather":
        seqs = _log(rng, 1, 32)
        return _case(None, kind, seqs=seqs, n=_log(rng, 100, 131072 // seqs), **c)
    if kind == "append":
        c.update(rot=rng.choice([128, 128, 64, 96, 32]), axes=rng.choice([1, 1, 2, 3]), pairs=rng.choice(["halves", "halves", "neighbours"]),
                 query=rng.random() < 0.8)
        seqs = _log(rng, 1, 64)
        tokens = rng.choice([1, _log(rng, 1, 8192 // seqs)])
        return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + _log(rng, 1, 131072 // seqs), **c)
    window = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
    what = rng.choice(["decode", "decode", "chunk", "prompts", "few"])
    if what == "decode":
        seqs = rng.choice([1, _log(rng, 1, 48)])
        return _case(None, kind, seqs=seqs, n=_log(rng, 64, min(131072, 524288 // seqs)), window=window, **c)
    if what == "few":        # a few tokens a sequence: drafts to be checked
        seqs = _log(rng, 1, 16)
        tokens = rng.randint(2, 16)
        return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + _log(rng, 64, 65536 // seqs), window=window, **c)
    if what == "chunk":
        tokens = _log(rng, 32, 2048)
        return _case(None, kind, seqs=rng.randint(2, 32), tokens=tokens, n=tokens + _log(rng, 64, 8192), window=window, **dict(c, mix="chunk"))
    seqs = _log(rng, 1, 8)
    tokens = _log(rng, 16, (2048 if c["dtype"] == "f32" else 4096) // seqs)
    return _case(None, kind, seqs=seqs, tokens=tokens, n=tokens + rng.choice([0, _log(rng, 1, 8192)]), window=window, **c)


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
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


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
            n_q_heads=case["hq"], n_kv_heads=case["hkv"], kv_dtype=L.LVR_BF16 if case["dtype"] == "bf16" else L.LVR_F32,
            page_size=case["page"], n_pages=n_pages, layout=case["layout"], rot_dim=case["rot"], rot_axes=case["axes"],
            rot_pairs=L.LVR_ROT_HALVES if case["pairs"] == "halves" else L.LVR_ROT_NEIGHBOURS)
        self.handle = L.lvr_paged_create(cfg, inv_freq=_inv_freq(case), axis=_axis(case))

    def __del__(self):
        if getattr(self, "handle", None):
            self.L.lvr_paged_destroy(self.handle)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 23)
    r = random.Random(int(seed) * 31 + 7)
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
    shape = (n_pages, hkv, page, D) if case["layout"] == "head" else (n_pages, page, hkv, D)

    def pool():                           # [page][head][token][coordinate] in either order of memory
        p = torch.empty(shape, device="cuda", dtype=dt)
        for i in range(0, n_pages, 2048):
            p[i:i + 2048] = torch.randn((min(2048, n_pages - i),) + shape[1:], generator=g, device="cuda")
        return p

    state = {"case": case, "k_pages": pool(), "v_pages": pool(),
             "table": torch.tensor(table, dtype=torch.int32, device="cuda"),
             "seq_start": torch.tensor(start, dtype=torch.int32, device="cuda"),
             "seq_len": torch.tensor(held, dtype=torch.int32, device="cuda"), "new": new, "held": held}
    if kind == "attention":
        # keys whose channels differ in size, as a model's do
        s = torch.exp(0.4 * torch.randn((hkv, D), generator=g, device="cuda"))
        scale = s[None, :, None, :] if case["layout"] == "head" else s[None, None]
        for i in range(0, n_pages, 2048):
            state["k_pages"][i:i + 2048] = state["k_pages"][i:i + 2048].float() * scale
        state["q"] = torch.randn((T, hq, D), generator=g, device="cuda").to(dt)
        state["out"] = torch.empty_like(state["q"])
    elif kind == "append":
        fused = torch.randn((T, (hq + 2 * hkv) * D), generator=g, device="cuda").to(dt)   # as one projection writes q, k and v
        state["q"] = fused[:, :hq * D].view(T, hq, D)
        state["k"] = fused[:, hq * D:(hq + hkv) * D].view(T, hkv, D)
        state["v"] = fused[:, (hq + hkv) * D:].view(T, hkv, D)
        state["q_out"] = torch.empty((T, hq, D), device="cuda", dtype=dt) if case["query"] else None
        at = torch.cat([torch.arange(n - t, n) for t, n in zip(new, held)])
        pos = torch.stack([at, at // 37 % 411, at % 37 * 3][:case["axes"]], dim=1)        # time, and rows and columns of an image
        state["positions"] = pos.to(torch.int32).cuda().contiguous()
        state["inv_freq"] = torch.tensor(_inv_freq(case), dtype=torch.float64, device="cuda")
        state["axis"] = torch.tensor(_axis(case), device="cuda")
    else:
        n = max(held)
        state["K"] = torch.zeros((case["seqs"], hkv, n, D), device="cuda", dtype=dt)      # rows past a sequence's end stay as they are
        state["V"] = torch.zeros_like(state["K"])
    if own:
        state["paged"] = _Paged(case, n_pages)
    return state


# ------------------------------------------------------------------------------------------------ the plain forms
def _heads_first(case, pages):
    return pages if case["layout"] == "head" else pages.transpose(1, 2)


def _rows(case, pages, table, n):
    """The first n rows of the given sequences: [seq][head][n][D]."""
    p = -(-n // case["page"])
    x = _heads_first(case, pages)[table[:, :p].long().clamp_min(0)]
    return x.permute(0, 2, 1, 3, 4).reshape(table.shape[0], case["hkv"], p * case["page"], D)[:, :, :n]


def _attend(case, q, K, V, first, last):
    """q [seq][tokens][hq][D] over K, V [seq][hkv][n][D] in 32 bits; keys first[seq][token] .. last[seq][token] are visible."""
    s, t, hq, _ = q.shape
    hkv, n = K.shape[1], K.shape[2]
    q = (q.float() / math.sqrt(D)).reshape(s, t, hkv, hq // hkv, D).permute(0, 2, 1, 3, 4).reshape(s, hkv, -1, D)
    x = torch.matmul(q, K.float().transpose(2, 3).contiguous()).view(s, hkv, t, hq // hkv, n)
    j = torch.arange(n, device=q.device)
    hidden = (j < first[:, :, None]) | (j > last[:, :, None])
    x.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    x.sub_(x.amax(dim=-1, keepdim=True)).exp_()
    den = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(s, hkv, -1, n), V.float().contiguous()).view(s, hkv, t, hq // hkv, D) / den
    return o.permute(0, 2, 1, 3, 4).reshape(s, t, hq, D)


def _attention(state):
    case, new, held, dt = state["case"], state["new"], state["held"], _type(state["case"])

    def piece(b0, b1, tokens, n):
        table, length = state["table"][b0:b1], state["seq_len"][b0:b1].long()
        q = state["q"][sum(new[:b0]):sum(new[:b1])].view(b1 - b0, tokens, case["hq"], D)
        last = length[:, None] - tokens + torch.arange(tokens, device=q.device)
        first = (last - case["window"] + 1).clamp_min(0) if case["window"] else torch.zeros_like(last)
        K, V = _rows(case, state["k_pages"], table, n), _rows(case, state["v_pages"], table, n)
        return _attend(case, q, K, V, first, last).to(dt).view(-1, case["hq"], D)

    if len(set(new)) == 1:                # one batch, shorter sequences masked
        return piece(0, case["seqs"], new[0], max(held))
    return torch.cat([piece(b, b + 1, new[b], held[b]) for b in range(case["seqs"])])


def _rotate(case, x, cos, sin):
    """x [T][heads][D], cos and sin [T][1][rot / 2], in 32 bits, rounded once."""
    rot, y = case["rot"], x.float().clone()
    if case["pairs"] == "halves":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    u, w = a * cos - b * sin, a * sin + b * cos
    a.copy_(u)
    b.copy_(w)
    return y.to(x.dtype)


def _append(state):
    case, start, length, page = state["case"], state["seq_start"].long(), state["seq_len"].long(), state["case"]["page"]
    t = torch.arange(state["k"].shape[0], device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), t, right=True)
    slot = length[b] - start[b + 1] + t
    to = state["table"][b, slot // page].long()
    angle = state["positions"].double()[:, state["axis"]] * state["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    _heads_first(case, state["k_pages"])[to, :, slot % page] = _rotate(case, state["k"], cos, sin)
    _heads_first(case, state["v_pages"])[to, :, slot % page] = state["v"]
    result = {"k_pages": state["k_pages"], "v_pages": state["v_pages"]}
    if case["query"]:
        result["q"] = _rotate(case, state["q"], cos, sin)
    return result


def _gather(state):
    case, n = state["case"], state["K"].shape[2]
    past = torch.arange(n, device="cuda")[None, None, :, None] >= state["seq_len"][:, None, None, None]
    return {"K": torch.where(past, state["K"], _rows(case, state["k_pages"], state["table"], n)),
            "V": torch.where(past, state["V"], _rows(case, state["v_pages"], state["table"], n))}


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        return {"out": _attention(state)} if kind == "attention" else _append(state) if kind == "append" else _gather(state)
    import paper_2605_06763_amd as L
    h = state["paged"].handle
    if kind == "attention":
        L.lvr_paged_attention(h, state["k_pages"], state["v_pages"], state["q"], state["seq_start"], state["seq_len"],
                              state["table"], state["out"], window=case["window"])
        return {"out": state["out"]}
    if kind == "append":
        q = state["q"] if case["query"] else None
        L.lvr_paged_append(h, state["k_pages"], state["v_pages"], state["k"], state["v"], state["seq_start"], state["seq_len"],
                           state["table"], q=q, q_out=state["q_out"], positions=state["positions"])
        result = {"k_pages": state["k_pages"], "v_pages": state["v_pages"]}
        return dict(result, q=state["q_out"]) if case["query"] else result
    L.lvr_paged_gather(h, state["k_pages"], state["v_pages"], state["seq_len"], state["table"], state["K"], state["V"])
    return {"K": state["K"], "V": state["V"]}


# ------------------------------------------------------------------------------------------------ work, exactness
def work(case):
    """Bytes: every key and value row that some new token sees once (a window hides the older ones), queries, outputs, new rows
    and rows written once each.  Flops: two products of 128 per visible (query row, key), six per rotated pair."""
    new, held = _lengths(case)
    row = D * (2 if case["dtype"] == "bf16" else 4)
    T, hq, hkv, w = sum(new), case["hq"], case["hkv"], case["window"]
    if case["kind"] == "gather":
        return {"bytes": 4.0 * sum(held) * hkv * row + 4 * sum(held) / case["page"], "flops": 0.0}
    if case["kind"] == "append":
        q = hq if case["query"] else 0
        return {"bytes": 2.0 * T * (2 * hkv + q) * row + 4.0 * T * case["axes"], "flops": 6.0 * T * (hkv + q) * case["rot"] / 2}
    keys = seen = 0
    for t, n in zip(new, held):
        keys += min(n, w + t - 1) if w else n
        first = n - t + 1                 # keys the first new token sees without a window
        seen += sum(min(w, x) for x in range(first, n + 1)) if w else (first + n) * t / 2
    return {"bytes": 2.0 * keys * hkv * row + 2.0 * T * hq * row, "flops": 4.0 * D * hq * seen}


def exact(case, seed):
    state = prepare(case, seed)
    new, held, page, hkv = state["new"], state["held"], case["page"], case["hkv"]
    G, kind = case["hq"] // hkv, case["kind"]
    head = (lambda p: p) if case["layout"] == "head" else (lambda p: p.transpose(1, 2))
    table = state["table"].tolist()
    if kind == "attention":
        out = torch.empty((sum(new), case["hq"], D), dtype=torch.float64, device="cuda")
        t0 = 0
        for b, (t, n) in enumerate(zip(new, held)):
            ids = torch.tensor(table[b][:-(-n // page)], device="cuda")
            far = torch.arange(n - t, n, device="cuda")[:, None] - torch.arange(n, device="cuda")     # how far back a key lies
            sees = (far >= 0) & (far < case["window"]) if case["window"] else far >= 0
            for h in range(hkv):
                K = head(state["k_pages"])[ids, h].reshape(-1, D)[:n].double()
                V = head(state["v_pages"])[ids, h].reshape(-1, D)[:n].double()
                for g in range(h * G, h * G + G):
                    s = (state["q"][t0:t0 + t, g].double() @ K.t().contiguous()) * D ** -0.5
                    s = torch.where(sees, s, torch.full_like(s, -math.inf))
                    out[t0:t0 + t, g] = torch.exp(s - torch.logsumexp(s, dim=1, keepdim=True)) @ V
            t0 += t
        return {"out": out}
    if kind == "gather":
        result = {"K": state["K"].double(), "V": state["V"].double()}
        for b, n in enumerate(held):
            ids = torch.tensor(table[b][:-(-n // page)], device="cuda")
            for to, pages in (("K", "k_pages"), ("V", "v_pages")):
                for h in range(hkv):
                    result[to][b, h, :n] = head(state[pages])[ids, h].reshape(-1, D)[:n].double()
        return result
    # rotation as a product of complex numbers
    turn = torch.exp(1j * (state["positions"].double()[:, state["axis"]] * state["inv_freq"]))[:, None]
    half, rot = case["rot"] // 2, case["rot"]

    def rotated(x):
        x = x.double()
        first, second = (x[..., :half], x[..., half:rot]) if case["pairs"] == "halves" else (x[..., 0:rot:2], x[..., 1:rot:2])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        parts = [z.real, z.imag] if case["pairs"] == "halves" else [torch.stack([z.real, z.imag], dim=-1).flatten(-2)]
        return torch.cat(parts + [x[..., rot:]], dim=-1)

    result = {"k_pages": state["k_pages"].double(), "v_pages": state["v_pages"].double()}
    rows = [(table[b][p // page], p % page) for b, (t, n) in enumerate(zip(new, held)) for p in range(n - t, n)]
    ids, at = (torch.tensor(x, device="cuda") for x in zip(*rows))
    head(result["k_pages"])[ids, :, at] = rotated(state["k"])
    head(result["v_pages"])[ids, :, at] = state["v"].double()
    if case["query"]:
        result["q"] = rotated(state["q"])
    return result
