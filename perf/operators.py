"""Performance cases of a decoder's serving operators: appending to a paged 8-bit cache with the position rotation, attention over that
cache, and drawing tokens, for one token per sequence up to whole prompts and for groups of models that answer the same prompts.

Head counts, widths and vocabularies are those of the workload configurations (32 heads of 128, 12 and 16 of 64, 32000 and 30522
tokens, sequences of 2048), their versions with shared key/value heads, and the longer caches that serving meets.

    own                  False: `run` computes the plain form below; True: it calls paper_2107_06469_amd.ops
    listed()             the named cases
    draw(rng)            one more case of the same ranges
    prepare(case, seed)  inputs and what a user's program keeps, on the device
    run(state)           one pass; returns its outputs
    work(case)           bytes and flops that one pass cannot do without
    exact(case, seed)    the same outputs in 64 bits
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

INT8, E4M3 = "int8", "e4m3"
TOP = {INT8: 127.0, E4M3: 448.0}                 # the largest code of a kind
LEAST = 2.0 ** -126                              # the smallest scale of a page


# ---- the cases --------------------------------------------------------------------------------------------------------

def _append(name, G, B, H, HKV, DH, page, kind, q, past, rot, rot_dim):
    """q: new tokens per sequence (the most, where sequences differ); past: tokens that the longest sequence holds already."""
    return dict(name=name, op="append", G=G, B=B, H=H, HKV=HKV, DH=DH, page=page, kind=kind, q=q, past=past, rot=rot, rot_dim=rot_dim)


def _attention(name, G, B, H, HKV, DH, page, kind, q, past, causal=True):
    return dict(name=name, op="attention", G=G, B=B, H=H, HKV=HKV, DH=DH, page=page, kind=kind, q=q, past=past, causal=causal)


def _sample(name, G, rows, V, dtype, filters):
    """filters: "none" (temperature alone), "few" (top-k, then top-p), "mass" (top-p and min-p), "mixed" (each row its own, greedy rows among them)."""
    return dict(name=name, op="sample", G=G, rows=rows, V=V, dtype=dtype, filters=filters)


def listed():
    return [
        # one sequence's next token through the heads of the 4096-wide decoders: nothing but latency
        _append("append_one", 1, 1, 32, 32, 128, 64, E4M3, 1, 700, "halves", 128),
        # the next token of 64 sequences, key/value heads shared by four query heads, two models answering
        _append("append_batch", 2, 64, 32, 8, 128, 64, E4M3, 1, 4000, "halves", 128),
        # whole prompts of up to 2048 tokens of eight sequences into an empty cache
        _append("append_prompts", 1, 8, 32, 32, 128, 64, E4M3, 2048, 0, "halves", 128),
        # prompts of odd lengths behind a shared beginning, heads of 64, half of a head rotated, int8
        _append("append_chunks_int8", 1, 16, 16, 16, 64, 32, INT8, 301, 77, "neighbours", 32),
        # one sequence's next token over a short cache
        _attention("decode_one", 1, 1, 32, 32, 128, 64, INT8, 1, 512),
        # the next token of 64 sequences of up to 2048 tokens, two models answering
        _attention("decode_batch", 2, 64, 32, 8, 128, 64, INT8, 1, 2047),
        # the next token of eight sequences of up to 32768 tokens: the long axis is what there is to split
        _attention("decode_long", 1, 8, 32, 8, 128, 128, E4M3, 1, 32767),
        # up to five tokens at a time (drafted ones being checked), heads of 64, small pages
        _attention("decode_drafts", 1, 24, 16, 4, 64, 16, E4M3, 5, 1500),
        # prompts of 2048 tokens of eight sequences: every query over all keys before it
        _attention("attend_prompts", 1, 8, 32, 32, 128, 64, INT8, 2048, 0),
        # one row of the 4096-wide decoders' vocabulary, top-k and top-p
        _sample("sample_one", 1, 1, 32000, "f32", "few"),
        # 64 sequences of two models, each with settings of its own
        _sample("sample_batch", 2, 64, 32000, "f32", "mixed"),
        # 256 sequences over a wide vocabulary, 16-bit logits, top-p and min-p
        _sample("sample_wide", 1, 256, 131072, "bf16", "mass"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "sample"])
    while True:
        DH = rng.choice([64, 128, 128])
        HKV = rng.choice([1, 2, 3, 4, 8, 12, 16, 32])
        share = rng.choice([1, 1, 2, 4, 5, 8])
        page, kind, G = rng.choice([16, 32, 64, 128]), rng.choice([INT8, E4M3]), rng.choice([1, 1, 2, 3])
        if op == "append":
            q = 1 if rng.random() < 0.4 else _log(rng, 2, 2048)
            rot = rng.choice(["halves", "halves", "neighbours", "none"])
            c = _append("", G, _log(rng, 1, 128), HKV * share, HKV, DH, page, kind, q, _log(rng, 1, 4096), rot,
                        0 if rot == "none" else rng.choice([DH, DH, DH // 2]))
            fits = HKV * share <= 64 and work(c)["bytes"] <= 4.5e8
        elif op == "attention":
            q = 1 if rng.random() < 0.5 else _log(rng, 2, 2048)
            c = _attention("", G, _log(rng, 1, 128), HKV * share, HKV, DH, page, kind, q, _log(rng, 1, 32768), rng.random() < 0.9)
            w = work(c)
            # the plain form holds every score of the call
            scores = G * c["B"] * c["H"] * q * (q + c["past"])
            fits = HKV * share <= 64 and w["bytes"] <= 4.2e8 and w["flops"] <= 2.8e11 and scores <= 1.1e9
        else:
            c = _sample("", G, _log(rng, 1, 256), _log(rng, 1000, 131072), rng.choice(["f32", "bf16"]),
                        rng.choice(["none", "few", "mass", "mixed"]))
            fits = G * c["rows"] * c["V"] <= 256 * 131072
        if fits:
            del c["name"]
            return c


# ---- what a case holds ------------------------------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, tokens in the cache with them) of every sequence: the longest as the case says, the others from half of it on."""
    r = random.Random(case["B"] * 7919 + case["q"] * 104729 + case["past"])
    new = [case["q"] if b == 0 else r.randint((case["q"] + 1) // 2, case["q"]) for b in range(case["B"])]
    past = [case["past"] if b == 0 else r.randint(case["past"] // 2, case["past"]) for b in range(case["B"])]
    return new, [n + p for n, p in zip(new, past)]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape, dtype=torch.bfloat16, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(scale)


def _codes(g, shape, kind):
    """Cached values as they are when a page's largest one has the largest code: a normal distribution of a few widths."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    top = TOP[kind]
    x = x.mul_(top / 3.5).clamp_(-top, top)
    return x.round_().to(torch.int8) if kind == INT8 else x.to(torch.float8_e4m3fn)


def _plan(case, seed):
    """Page table, lengths and offsets of a call; the pages of a sequence lie anywhere in the pool."""
    new, total = _lengths(case)
    page = case["page"]
    need = [-(-n // page) for n in total]
    n_pages = sum(need) + 3
    ids = np.random.RandomState(seed % (2 ** 31)).permutation(n_pages)
    table = np.full((case["B"], max(need)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    ptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    return dict(n_pages=n_pages, table=dev(table), lens=dev(np.array(total, dtype=np.int32)), q_ptr=dev(ptr), n_tok=int(ptr[-1]), max_q=max(new),
                max_len=max(total))


def _cache(case, p, g):
    """The pools of every model of the group and their scales."""
    shape = (p["n_pages"], case["HKV"], case["page"], case["DH"])
    some = lambda: _normal(g, *shape[:2], dtype=torch.float32, scale=0.2).exp_().mul_(2.5 / TOP[case["kind"]])  # noqa: E731
    n = range(case["G"])
    return dict(k=[_codes(g, shape, case["kind"]) for _ in n], v=[_codes(g, shape, case["kind"]) for _ in n], ks=[some() for _ in n],
                vs=[some() for _ in n])


def _angles(case, rows):
    """cos and sin of every position's angles, [rows, rot_dim]: the first half of a row holds the cosines."""
    half = case["rot_dim"] // 2
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(half)[None] / half)
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], axis=1).astype(np.float32)).cuda()


def _settings(case, seed):
    """temperature, top_k, top_p, min_p of every row; 0, 1 and 0 leave a filter out."""
    r, n = np.random.RandomState((seed + 17) % (2 ** 31)), case["rows"]
    t, k, p, m = r.uniform(0.6, 1.3, n), np.zeros(n), np.ones(n), np.zeros(n)
    f = case["filters"]
    if f == "few":
        k, p = r.choice([20, 40, 50], n), r.uniform(0.8, 0.98, n)
    elif f == "mass":
        p, m = r.uniform(0.85, 0.99, n), r.uniform(0.0, 0.05, n)
    elif f == "mixed":
        k = np.where(r.rand(n) < 0.5, r.randint(1, 2000, n), 0)
        p = np.where(r.rand(n) < 0.6, r.uniform(0.3, 1.0, n), 1.0)
        m = np.where(r.rand(n) < 0.3, r.uniform(0.0, 0.2, n), 0.0)
        t = np.where(r.rand(n) < 0.15, 0.0, t)
    dev = lambda a, d: torch.from_numpy(np.ascontiguousarray(a.astype(d))).cuda()  # noqa: E731
    return dict(t=dev(t, np.float32), k=dev(k, np.int32), p=dev(p, np.float32), m=dev(m, np.float32))


def prepare(case, seed):
    g, G = _gen(seed), case["G"]
    s = dict(case=case)
    if case["op"] == "sample":
        rows, V = case["rows"], case["V"]
        # a trained model's logits: falling with a token's rank, ranks dealt over the vocabulary, and noise on top
        step = next(k for k in range(V * 5 // 8 | 1, V + 9, 2) if math.gcd(k, V) == 1)
        rank = (torch.arange(V, device="cuda") * step % V).float()
        s.update(_settings(case, seed))
        s["z"] = [(_normal(g, rows, V, dtype=torch.float32, scale=0.9) - 1.3 * torch.log1p(rank)).to(
            torch.bfloat16 if case["dtype"] == "bf16" else torch.float32) for _ in range(G)]
        s["u"] = [torch.rand((rows, V), generator=g, device="cuda") for _ in range(G)]
        s["token"] = [torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(G)]
        s["logprob"] = [torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(G)]
        return s
    p = _plan(case, seed)
    s.update(p)
    s.update(_cache(case, p, g))
    H, HKV, DH, n = case["H"], case["HKV"], case["DH"], p["n_tok"]
    if case["op"] == "append":
        s["qkv"] = [_normal(g, n, (H + 2 * HKV) * DH) for _ in range(G)]
        s["q"] = [torch.empty((n, H * DH), dtype=torch.bfloat16, device="cuda") for _ in range(G)]
        s["cs"] = _angles(case, p["max_len"]) if case["rot_dim"] else None
    else:
        s["q"] = [_normal(g, n, H * DH) for _ in range(G)]
        s["o"] = [torch.empty((n, H * DH), dtype=torch.bfloat16, device="cuda") for _ in range(G)]
        s["lse"] = [torch.empty((n, H), dtype=torch.float32, device="cuda") for _ in range(G)]
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _tokens(s):
    """Sequence and position of every new token."""
    t = torch.arange(s["n_tok"], device="cuda")
    seq = (t[:, None] >= s["q_ptr"][None, 1:]).sum(1)
    return seq, (s["lens"][seq] - s["q_ptr"][seq + 1]).long() + t


def _rotate(x, cs, case):
    """x [n, heads, DH] with its first rot_dim columns turned by the angles of the tokens' positions, cs [n, rot_dim]."""
    r = case["rot_dim"]
    if not r:
        return x
    c, s = cs[:, None, :r // 2], cs[:, None, r // 2:]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if case["rot"] == "halves" else (x[..., 0:r:2], x[..., 1:r:2])
    u, v = a * c - b * s, b * c + a * s
    turned = torch.cat([u, v], -1) if case["rot"] == "halves" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _to_codes(x, kind):
    x = x.clamp(-TOP[kind], TOP[kind])
    return x.round().to(torch.int8) if kind == INT8 else x.to(torch.float8_e4m3fn).view(torch.int8)


def _from_codes(c, kind):
    return c.float() if kind == INT8 else c.view(torch.float8_e4m3fn).float()


def _into_pages(x, codes, scale, s, seq, pos):
    """New values x [n, HKV, DH] into the pages, whose scale grows where they need it."""
    case, page, kind = s["case"], s["case"]["page"], s["case"]["kind"]
    raw = codes.view(torch.int8)
    at, slot = s["table"][seq, pos // page].long(), pos % page
    most = torch.zeros_like(scale).index_reduce_(0, at, x.abs().amax(-1), "amax")
    first = torch.full((scale.shape[0],), page, device="cuda").index_reduce_(0, at, slot, "amin")  # the first new slot of a page
    held = torch.where(first[:, None] == 0, torch.zeros_like(scale), scale)
    now = torch.maximum(held, (most * (1.0 / TOP[kind])).clamp(min=LEAST))
    now = torch.where(first[:, None] < page, now, scale)
    # what a page holds already: one page of a sequence at most, the one that its first new token goes to
    begin = pos[s["q_ptr"][:-1].long()]
    old = s["table"][torch.arange(case["B"], device="cuda"), begin // page].long()
    c = raw[old]
    again = _to_codes(_from_codes(c, kind) * (held[old] / now[old])[..., None, None], kind)
    kept = torch.arange(page, device="cuda")[None] < (begin % page)[:, None]
    raw[old] = torch.where(kept[:, None, :, None] & (now[old] > held[old])[..., None, None], again, c)
    raw[at, :, slot] = _to_codes(x * (1.0 / now[at])[..., None], kind)
    scale.copy_(now)


def _append_plain(s, g):
    case, n, H, HKV = s["case"], s["n_tok"], s["case"]["H"], s["case"]["HKV"]
    seq, pos = _tokens(s)
    x = s["qkv"][g].float().view(n, H + 2 * HKV, case["DH"])
    cs = s["cs"][pos] if s["cs"] is not None else None
    s["q"][g].copy_(_rotate(x[:, :H], cs, case).reshape(n, -1))
    _into_pages(_rotate(x[:, H:H + HKV], cs, case), s["k"][g], s["ks"][g], s, seq, pos)
    _into_pages(x[:, H + HKV:], s["v"][g], s["vs"][g], s, seq, pos)


def _held(codes, scale, s, case):
    """Cached values [B, HKV, tokens, DH] in 32 bits."""
    tab = s["table"][:, :-(-s["max_len"] // case["page"])].clamp(min=0).long()
    x = _from_codes(codes.view(torch.int8)[tab], case["kind"]) * scale[tab][..., None, None]
    return x.permute(0, 2, 1, 3, 4).reshape(case["B"], case["HKV"], -1, case["DH"])


def _attention_plain(s, g):
    case, B, H, HKV, DH, mq = s["case"], s["case"]["B"], s["case"]["H"], s["case"]["HKV"], s["case"]["DH"], s["max_q"]
    k, v = _held(s["k"][g], s["ks"][g], s, case), _held(s["v"][g], s["vs"][g], s, case)
    j = torch.arange(mq, device="cuda")
    count = (s["q_ptr"][1:] - s["q_ptr"][:-1])[:, None]
    row = (s["q_ptr"][:-1, None] + j).clamp(max=s["n_tok"] - 1).long()
    q = s["q"][g].float()[row].view(B, mq, HKV, H // HKV, DH).permute(0, 2, 1, 3, 4).reshape(B, HKV, -1, DH)
    key = torch.arange(k.shape[2], device="cuda")
    seen = (key < s["lens"][:, None, None]) & (j < count)[..., None]
    if case["causal"]:
        seen = seen & (key <= (s["lens"][:, None] - count + j)[..., None])
    seen = seen[:, None, :, None].expand(B, 1, mq, H // HKV, key.numel()).reshape(B, 1, -1, key.numel())
    z = (q @ k.transpose(-1, -2)).mul_(DH ** -0.5).masked_fill_(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    z = z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    o = (z @ v) / torch.where(total == 0, torch.ones_like(total), total)
    back = lambda x: x.view(B, HKV, mq, H // HKV, -1).permute(0, 2, 1, 3, 4).reshape(B, mq, -1)  # noqa: E731
    seq, _ = _tokens(s)
    at = torch.arange(s["n_tok"], device="cuda") - s["q_ptr"][seq]
    s["o"][g].copy_(back(o)[seq, at])
    s["lse"][g].copy_(back(top + total.log())[seq, at])


def _sample_plain(s, g):
    z, order = s["z"][g].float().sort(dim=1, descending=True, stable=True)
    V = z.shape[1]
    t, k, p, m = (s[n][:, None] for n in "tkpm")
    greedy, t = t <= 0, torch.where(t <= 0, torch.ones_like(t), t)
    rank = torch.arange(V, device="cuda")[None]
    w = ((z - z[:, :1]) / t).exp()
    keep = rank < torch.where(k <= 0, torch.full_like(k, V), k)
    mass = w * keep
    keep &= (mass.cumsum(1) - mass < p * mass.sum(1, keepdim=True)) | (p >= 1) | (rank == 0)
    keep &= w >= m
    u = s["u"][g].gather(1, order)
    score = (z / t - (-u.log()).log()).clamp(min=torch.finfo(torch.float32).min)
    at = torch.where(keep, score, torch.full_like(score, -math.inf)).argmax(1, keepdim=True)
    at = torch.where(greedy, torch.zeros_like(at), at)
    s["token"][g].copy_(order.gather(1, at)[:, 0])
    s["logprob"][g].copy_((z.gather(1, at) - z[:, :1] - (z - z[:, :1]).exp().sum(1, keepdim=True).log())[:, 0])


# ---- one pass ---------------------------------------------------------------------------------------------------------

def _kept(s):
    """The cache's record and attention's scratch, which a program makes once and keeps."""
    from paper_2107_06469_amd import ops
    case = s["case"]
    cache = ops.Cache(ops.CACHE_INT8 if case["kind"] == INT8 else ops.CACHE_E4M3, s["k"], s["v"], s["ks"], s["vs"], s["table"])
    size = 0
    if case["op"] == "attention":
        size = ops.hydra_op_cache_attention_ws_bytes(cache, case["H"], n_tok=s["n_tok"], max_q=s["max_q"], max_len=s["max_len"])
    s["kept"] = cache, [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(case["G"])] if size else None
    return s["kept"]


def _call(s):
    from paper_2107_06469_amd import ops
    case = s["case"]
    H, HKV, DH = (case.get(n) for n in ("H", "HKV", "DH"))
    if case["op"] == "sample":
        ops.hydra_op_sample(ops.BF16 if case["dtype"] == "bf16" else ops.F32, case["rows"], case["V"], case["V"], case["V"], s["z"], s["u"], s["t"],
                            s["k"], s["p"], s["m"], s["token"], s["logprob"])
        return
    cache, ws = s.get("kept") or _kept(s)
    which = dict(n_tok=s["n_tok"], max_q=s["max_q"], max_len=s["max_len"], q_ptr=None if case["q"] == 1 else s["q_ptr"])
    if case["op"] == "append":
        rot = {"none": ops.ROT_NONE, "halves": ops.ROT_HALVES, "neighbours": ops.ROT_NEIGHBOURS}[case["rot"]]
        ops.hydra_op_cache_append(cache, s["lens"], H, (H + 2 * HKV) * DH, H * DH, s["qkv"], s["q"], rot=rot, rot_dim=case["rot_dim"], cos_sin=s["cs"],
                                  **which)
    else:
        ops.hydra_op_cache_attention(cache, s["lens"], H, H * DH, H * DH, case["causal"], DH ** -0.5, s["q"], s["o"], s["lse"], ws=ws, **which)


def _values(codes, scale, kind):
    """A pool as what it stands for: e4m3 codes are numbers already (their scales go beside them), int8 codes times their page's scale."""
    return codes if kind == E4M3 else codes.float().mul_(scale[..., None, None])


def run(state):
    s, case = state, state["case"]
    if own:
        _call(s)
    else:
        plain = {"append": _append_plain, "attention": _attention_plain, "sample": _sample_plain}[case["op"]]
        [plain(s, g) for g in range(case["G"])]
    if case["op"] == "sample":
        return [dict(token=s["token"][g], logprob=s["logprob"][g]) for g in range(case["G"])]
    if case["op"] == "attention":
        return [dict(o=s["o"][g], lse=s["lse"][g]) for g in range(case["G"])]
    return [dict(q=s["q"][g], k=_values(s["k"][g], s["ks"][g], case["kind"]), v=_values(s["v"][g], s["vs"][g], case["kind"]), ks=s["ks"][g], vs=s["vs"][g])
            for g in range(case["G"])]


def work(case):
    G = case["G"]
    if case["op"] == "sample":
        n = G * case["rows"] * case["V"]
        noise = 4 * n if case["filters"] == "none" else 0        # a row whose tokens are filtered needs the numbers of those that are left
        return dict(bytes=n * (2 if case["dtype"] == "bf16" else 4) + noise + 8 * G * case["rows"] + 16 * case["rows"], flops=4.0 * n)
    new, total = _lengths(case)
    H, HKV, DH, page, n = case["H"], case["HKV"], case["DH"], case["page"], sum(new)
    if case["op"] == "append":
        pages = sum(-(-t // page) - (t - m) // page for m, t in zip(new, total))
        each = n * (2 * H + HKV * 2) * DH * 2 + n * HKV * 2 * DH + pages * HKV * 2 * 8
        return dict(bytes=G * each + 4 * n * case["rot_dim"], flops=G * n * (3.0 * (H + HKV) * case["rot_dim"] + 2.0 * HKV * 2 * DH))
    pages = sum(-(-t // page) for t in total)
    each = sum(total) * HKV * DH * 2 + pages * HKV * 8 + n * H * (4 * DH + 4)
    pairs = sum(m * t - (m * (m - 1) // 2 if case["causal"] else 0) for m, t in zip(new, total))
    return dict(bytes=G * each + 4 * pages, flops=4.0 * G * pairs * H * DH)


# ---- in 64 bits -------------------------------------------------------------------------------------------------------

def _wide(codes):
    return codes.double() if codes.dtype == torch.int8 else codes.float().double()


def _exact_append(s, g):
    """Sequence by sequence, page by page, complex numbers for the rotation."""
    case, page, top = s["case"], s["case"]["page"], TOP[s["case"]["kind"]]
    H, HKV, DH, r = case["H"], case["HKV"], case["DH"], case["rot_dim"]
    codes, scales = [_wide(s["k"][g]), _wide(s["v"][g])], [s["ks"][g].double(), s["vs"][g].double()]
    table, lens, ptr = s["table"].tolist(), s["lens"].tolist(), s["q_ptr"].tolist()

    def nearest(x):
        x = x.clamp(-top, top)
        if case["kind"] == INT8:
            return x.round()
        step = torch.exp2(torch.frexp(x)[1].double().sub_(1).clamp_(min=-6) - 3)  # three bits after the first, none below 2^-9
        return (x / step).round() * step

    def turned(x, pos):
        if not r:
            return x
        cs = s["cs"][pos].double()
        by = torch.complex(cs[:, :r // 2], cs[:, r // 2:])[:, None]
        if case["rot"] == "halves":
            z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * by
            return torch.cat([z.real, z.imag, x[..., r:]], -1)
        z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:2], -1, 2).contiguous()) * by
        return torch.cat([torch.view_as_real(z).reshape(*x.shape[:2], r), x[..., r:]], -1)

    q = []
    for b in range(case["B"]):
        n, end = ptr[b + 1] - ptr[b], lens[b]
        pos = torch.arange(end - n, end, device="cuda")
        x = s["qkv"][g][ptr[b]:ptr[b + 1]].double().view(n, H + 2 * HKV, DH)
        q.append(turned(x[:, :H], pos).reshape(n, -1))
        for c, sc, y in zip(codes, scales, (turned(x[:, H:H + HKV], pos), x[:, H + HKV:])):
            for p in range((end - n) // page, (end - 1) // page + 1):
                lo, hi = max(p * page, end - n), min((p + 1) * page, end)
                part, at, k = y[lo - end + n:hi - end + n].transpose(0, 1), table[b][p], lo - p * page
                before = sc[at] if k else torch.zeros_like(sc[at])
                now = torch.maximum(before, (part.abs().amax((1, 2)) / top).clamp(min=LEAST))
                if k:
                    c[at, :, :k] = torch.where((now > before)[:, None, None], nearest(c[at, :, :k] * (before / now)[:, None, None]), c[at, :, :k])
                c[at, :, k:k + hi - lo] = nearest(part / now[:, None, None])
                sc[at] = now
    if case["kind"] == INT8:
        codes = [c * sc[..., None, None] for c, sc in zip(codes, scales)]
    return dict(q=torch.cat(q), k=codes[0], v=codes[1], ks=scales[0], vs=scales[1])


def _exact_attention(s, g):
    """Sequence by sequence and key/value head by head, rows in pieces."""
    case, page, H, HKV, DH = s["case"], s["case"]["page"], s["case"]["H"], s["case"]["HKV"], s["case"]["DH"]
    share = H // HKV
    o = torch.zeros((s["n_tok"], H, DH), dtype=torch.float64, device="cuda")
    lse = torch.full((s["n_tok"], H), -math.inf, dtype=torch.float64, device="cuda")
    lens, ptr = s["lens"].tolist(), s["q_ptr"].tolist()
    for b in range(case["B"]):
        n, end = ptr[b + 1] - ptr[b], lens[b]
        pages = s["table"][b, :-(-end // page)].long()
        for h in range(HKV):
            k, v = ((_wide(c[g][pages, h]) * sc[g][pages, h].double()[:, None, None]).reshape(-1, DH)[:end] for c, sc in ((s["k"], s["ks"]), (s["v"], s["vs"])))
            for lo in range(0, n, 512):
                rows = slice(ptr[b] + lo, ptr[b] + min(n, lo + 512))
                m = rows.stop - rows.start
                x = s["q"][g][rows].double().view(m, H, DH)[:, h * share:(h + 1) * share].reshape(-1, DH)
                z = x @ k.T / math.sqrt(DH)
                if case["causal"]:
                    pos = torch.arange(end - n + lo, end - n + lo + m, device="cuda").repeat_interleave(share)
                    z.masked_fill_(torch.arange(end, device="cuda")[None] > pos[:, None], -math.inf)
                e = torch.logsumexp(z, 1, keepdim=True)
                o[rows, h * share:(h + 1) * share] = (torch.exp(z - e) @ v).view(m, share, DH)
                lse[rows, h * share:(h + 1) * share] = e.view(m, share)
    return dict(o=o.view(s["n_tok"], -1), lse=lse)


def _exact_sample(s, g):
    """Row by row on the host; the draw itself is a whole number, what it is worth is not."""
    logprob = []
    for i, (t, k, p, m) in enumerate(zip(*(s[n].tolist() for n in "tkpm"))):
        z = s["z"][g][i].double().cpu().numpy()
        if t <= 0:
            token = int(np.argmax(z))
        else:
            best = np.argsort(-z, kind="stable")[:k if k > 0 else None]
            w = np.exp((z[best] - z.max()) / t)
            n = len(best) if p >= 1 else max(1, int(np.searchsorted(np.cumsum(w), p * w.sum())) + 1)
            left = best[:n][w[:n] >= m]
            with np.errstate(divide="ignore"):
                token = int(left[np.argmax(z[left] / t - np.log(-np.log(s["u"][g][i].cpu().numpy()[left].astype(np.float64))))])
        logprob.append(z[token] - z.max() - math.log(np.exp(z - z.max()).sum()))
    return dict(token=None, logprob=np.array(logprob))


def exact(case, seed):
    s = prepare(case, seed)
    how = {"append": _exact_append, "attention": _exact_attention, "sample": _exact_sample}[case["op"]]
    return [how(s, g) for g in range(case["G"])]
